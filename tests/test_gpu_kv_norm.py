"""New tokens into a 16- or 32-bit cache with norms of the heads
(nmspmm_kv_append_norm) against plain fp64.

Tolerance, derived, u = 2^-24: the norm's factor is exact to fp64 and rounded
once (u), times the weight (u), times the value (u): a normalised value x is
off by at most 3.1 u |x|.  A turned value is two products of such with cos and
sin and a sum in fp32: (3.1 + 3) u of |a| + |b|.  Then one rounding to the
stored type.
"""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from test_gpu_kv import DTYPES, close, f64, pages_of, tensor  # noqa: E402


def say(msg):
    print(msg, file=sys.stderr, flush=True)


def norm64(x, weight, eps):
    if weight is None:
        return x
    return x * weight / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def turn64(x, cos, sin, rot, interleaved, normed):
    """x (tokens, heads, dim) turned by cos and sin (tokens, rot/2), and the
    error that fp32 makes of it."""
    y, half = x.copy(), rot // 2
    err = (3.1 if normed else 0) * 2.0 ** -24 * np.abs(x)
    for e in range(half):
        i, j = (2 * e, 2 * e + 1) if interleaved else (e, e + half)
        a, b = x[..., i], x[..., j]
        c, s = cos[:, None, e], sin[:, None, e]
        y[..., i], y[..., j] = a * c - b * s, a * s + b * c
        err[..., i] = err[..., j] = (6.1 if normed else 3) * 2.0 ** -24 * (np.abs(a) + np.abs(b))
    return y, err


SHAPES = [
    # tokens, heads, group, dim, page, rot, interleaved, layout
    (1, 1, 1, 64, 16, 64, False, "plain"), (5, 2, 3, 128, 16, 128, False, "plain"), (64, 8, 4, 128, 16, 128, True, "plain"),
    (70, 3, 2, 80, 7, 40, False, "heads"), (33, 2, 1, 96, 24, 96, True, "padded"), (9, 1, 2, 33, 5, 32, False, "odd"),
    (17, 2, 0, 128, 1, 0, False, "joint"), (300, 2, 2, 64, 64, 64, False, "odd"), (12, 1, 1, 1, 3, 0, False, "plain"),
    (11, 2, 2, 512, 16, 256, False, "plain"), (40, 2, 2, 40, 16, 24, True, "plain"), (21, 4, 1, 256, 32, 64, False, "joint"),
    (8, 2, 2, 7, 4, 6, True, "plain"), (13, 2, 1, 24, 8, 4, False, "padded"), (10, 1, 3, 160, 16, 160, False, "plain"),
    (6, 2, 2, 128, 16, 64, False, "plain"), (7, 1, 1, 300, 16, 100, True, "plain")]


def setup(tokens, heads, group, dim, page, rot, interleaved, dtype, seed):
    """Places, projections (queries, keys and values in one row a token) and angles."""
    rng = np.random.default_rng(seed)
    sequences, wide = 4, max(9, -(-tokens // (4 * page)))
    pages = sequences * wide + 2
    table = torch.from_numpy(rng.permutation(pages)[:sequences * wide].reshape(sequences, wide)).int().cuda()
    places = rng.permutation(sequences * wide * page)[:tokens]
    seq, pos = places // (wide * page), places % (wide * page)
    qkv = tensor(rng, (tokens, group * heads + 2 * heads, dim), dtype)
    q, k, v = qkv[:, :group * heads], qkv[:, group * heads::2], qkv[:, group * heads + 1::2]
    half = rot // 2
    cos = sin = None
    if rot:
        angle = rng.uniform(0, 6, (wide * page, half))
        cos, sin = (torch.from_numpy(f(angle).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    c64, s64 = (f64(x)[pos] if rot else np.zeros((tokens, 0)) for x in (cos, sin))
    return rng, pages, table, seq, pos, q, k, v, cos, sin, c64, s64


@pytest.mark.parametrize("norms", ["both", "q", "k", "none"])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32")])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_append_norm(shape, dtype, cache, norms):
    tokens, heads, group, dim, page, rot, interleaved, layout = shape
    say(f"[append norm] {shape} {dtype} {cache} {norms}")
    rng, pages, table, seq, pos, q, k, v, cos, sin, c64, s64 = setup(*shape[:7], dtype, tokens + dim)
    kp, vp = (pages_of((pages, page, heads, dim), cache, layout, 3.0) for _ in range(2))
    weights = {x: torch.from_numpy(rng.uniform(-2, 2, dim).astype(np.float32)).cuda() if norms in ("both", x) else None
               for x in "qk"}
    eps = 1e-3
    handle = nm.nmspmm_kv_cache(kp, vp, table)
    q_out = torch.full((tokens, group * heads, dim + 2), 5.0, dtype=DTYPES[dtype], device="cuda")[..., :dim]
    new = dict(cos=cos, sin=sin, interleaved=interleaved, q_norm=weights["q"], k_norm=weights["k"], eps=eps)
    seq_, pos_ = torch.from_numpy(seq).int().cuda(), torch.from_numpy(pos).int().cuda()
    w64 = {x: None if weights[x] is None else f64(weights[x]) for x in "qk"}
    want_k = turn64(norm64(f64(k), w64["k"], eps), c64, s64, rot, interleaved, weights["k"] is not None)
    want_q = turn64(norm64(f64(q), w64["q"], eps), c64, s64, rot, interleaved, weights["q"] is not None)
    nm.nmspmm_kv_append_norm(handle, k, v, seq_, pos_, q=q if group else None, q_out=q_out if group else None, **new)
    torch.cuda.synchronize()
    at = table.cpu().numpy()[seq, pos // page], pos % page
    for pool, (want, err) in ((kp, want_k), (vp, (f64(v), 0.0))):
        got = f64(pool)
        close(got[at], want, err, cache, "written")
        got[at] = 3.0
        assert np.all(got == 3.0), "a slot that no token names was written"
    if group:
        close(f64(q_out), *want_q, dtype, "queries")
        nm.nmspmm_kv_append_norm(handle, k, v, seq_, pos_, q=q, **new)       # in place
        torch.cuda.synchronize()
        assert torch.equal(q, q_out)


@pytest.mark.parametrize("dim,rot", [(64, 64), (33, 32)])
def test_skips_tokens_without_a_place(dim, rot):
    rng = np.random.default_rng(3)
    heads, page, pages = 2, 4, 6
    kp, vp = (pages_of((pages, page, heads, dim), "bf16", "plain", 3.0) for _ in range(2))
    table = torch.tensor([[0, 1, 99], [-1, 2, 3]], dtype=torch.int32).cuda()
    seq = torch.tensor([0, 0, 2, -1, 1, 0, 0, 1, 1, 0], dtype=torch.int32).cuda()
    pos = torch.tensor([-1, 12, 0, 0, 1, 9, 5, 4, 10, 2 ** 31 - 1], dtype=torch.int32).cuda()
    written = {6: (1, 1), 7: (2, 0)}          # token 8 lies past the angles
    k, v, q = (tensor(rng, (len(seq), heads, dim), "bf16") for _ in range(3))
    q_out = torch.full_like(q, 3.0)
    angle = torch.zeros(10, rot // 2).cuda()
    one = torch.ones(dim, device="cuda")
    nm.nmspmm_kv_append_norm(nm.nmspmm_kv_cache(kp, vp, table), k, v, seq, pos, cos=angle.cos(), sin=angle.sin(), q=q,
                             q_out=q_out, q_norm=one, k_norm=one, eps=0.0)
    torch.cuda.synchronize()
    want_v = torch.full_like(vp, 3.0)
    for t, (pg, slot) in written.items():
        want_v[pg, slot] = v[t]
        for got, x in ((kp[pg, slot], k[t]), (q_out[t], q[t])):
            want = norm64(f64(x), 1.0, 0.0)
            close(f64(got), want, 3.1 * 2.0 ** -24 * np.abs(want), "bf16", "normed")
        kp[pg, slot] = q_out[t] = 3.0
    assert torch.equal(vp, want_v) and torch.all(kp == 3.0) and torch.all(q_out == 3.0)


@pytest.mark.parametrize("scale", [1e-25, 1e25])
def test_norm_of_tiny_and_huge_rows(scale):
    """Squares that overflow or vanish in fp32 do not reach the norm."""
    rng = np.random.default_rng(4)
    dim, page = 128, 16
    kp, vp = (pages_of((1, page, 1, dim), "f32", "plain", 3.0) for _ in range(2))
    k = tensor(rng, (16, 1, dim), "f32") * scale
    q, one = k.clone(), torch.ones(dim, device="cuda")
    pos = torch.arange(16, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv_append_norm(nm.nmspmm_kv_cache(kp, vp, torch.zeros(1, 1, dtype=torch.int32, device="cuda")), k, k,
                             torch.zeros_like(pos), pos, q=q, q_norm=one, k_norm=one, eps=0.0)
    want = norm64(f64(k), 1.0, 0.0)
    for got in (kp[0], q):
        close(f64(got), want, 3.1 * 2.0 ** -24 * np.abs(want), "f32", "normed")
