"""The appends with norms where values are infinite or minus zero: what a head
does not turn is copied bit for bit whatever lies beside it, an infinity stays
in its pair, and a norm makes of it what the formula makes in fp64 (zeros, and
NaN in the infinite places)."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from test_gpu_kv import f64  # noqa: E402
from test_gpu_kv_norm import norm64, turn64  # noqa: E402

# whole pieces, rows of pieces whose pairs are none, single values
FORMS = [(128, 64, False), (128, 64, True), (80, 40, False), (80, 20, True), (33, 32, False), (33, 6, True), (64, 0, False)]


def setup(dim, rot, dtype, tokens=40, heads=3):
    gen = torch.Generator(device="cuda").manual_seed(dim + rot)
    q, k, v = (torch.randn(tokens, heads, dim, generator=gen, device="cuda").to(dtype) for _ in range(3))
    for x in (q, k, v):
        at = torch.randint(0, dim, (tokens, heads, 1), generator=gen, device="cuda")
        x.scatter_(2, at, float("inf"))
        x[1::4] = x[1::4].clamp(max=2.0)            # (rows without one)
        x.scatter_(2, (at + 1) % dim, -0.0)
    pages = (tokens + 15) // 16
    kp, vp = (torch.zeros(pages, 16, heads, dim, dtype=dtype, device="cuda") for _ in range(2))
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    angle = torch.rand(tokens, rot // 2, generator=gen, device="cuda") * 6 if rot else None
    cs = dict(cos=angle.cos(), sin=angle.sin()) if rot else {}
    return q, k, v, kp, vp, nm.nmspmm_kv_cache(kp, vp, table), pos, cs


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=str)
@pytest.mark.parametrize("dim,rot,interleaved", FORMS)
def test_what_does_not_turn(dim, rot, interleaved, dtype):
    print(f"[kv norm edges] {dim} {rot} {interleaved} {dtype}", file=sys.stderr, flush=True)
    q, k, v, kp, vp, cache, pos, cs = setup(dim, rot, dtype)
    q_out = torch.zeros_like(q)
    nm.nmspmm_kv_append_norm(cache, k, v, torch.zeros_like(pos), pos, q=q, q_out=q_out, interleaved=interleaved, **cs)
    torch.cuda.synchronize()
    n = len(pos)
    bits = torch.int16 if dtype is torch.bfloat16 else torch.int32
    got_k, got_v = (x.view(-1, *k.shape[1:])[:n] for x in (kp, vp))
    for got, x, first in ((got_k, k, rot), (q_out, q, rot), (got_v, v, 0)):
        assert torch.equal(got[..., first:].contiguous().view(bits), x[..., first:].contiguous().view(bits))
    if rot:     # an infinity makes its pair, and nothing else, infinite or NaN
        for got, x in ((got_k, k), (q_out, q)):
            bad = np.isinf(f64(x))[..., :rot]
            half = rot // 2
            pair = (bad.reshape(*bad.shape[:2], half, 2).any(-1, keepdims=True).repeat(2, -1).reshape(bad.shape)
                    if interleaved else np.tile(bad[..., :half] | bad[..., half:], 2))
            assert np.array_equal(~np.isfinite(f64(got))[..., :rot], pair)


@pytest.mark.parametrize("dim,rot,interleaved", FORMS)
def test_norm_of_infinite_rows(dim, rot, interleaved):
    print(f"[kv norm edges] norm {dim} {rot} {interleaved}", file=sys.stderr, flush=True)
    q, k, v, kp, vp, cache, pos, cs = setup(dim, rot, torch.float32)
    weight = torch.rand(dim, device="cuda") + 0.5
    q_out = torch.zeros_like(q)
    nm.nmspmm_kv_append_norm(cache, k, v, torch.zeros_like(pos), pos, q=q, q_out=q_out, q_norm=weight, k_norm=weight,
                             eps=1e-3, interleaved=interleaved, **cs)
    torch.cuda.synchronize()
    c, s = (f64(cs[x]) if rot else np.zeros((len(pos), 0)) for x in ("cos", "sin"))
    with np.errstate(invalid="ignore"):
        for got, x in ((kp.view(-1, *k.shape[1:])[:len(pos)], k), (q_out, q)):
            want, err = turn64(norm64(f64(x), f64(weight), 1e-3), c, s, rot, interleaved, True)
            g = f64(got)
            assert np.array_equal(np.isnan(g), np.isnan(want))
            fine = ~np.isnan(want)
            assert np.all(np.abs(g - want)[fine] <= (err + 2.0 ** -24 * np.abs(want))[fine])


@pytest.mark.parametrize("power,eps", [(127, 1e-6), (120, 0.0), (-100, 0.0), (-126, 0.0), (-140, 0.0), (-140, 1e-6)])
@pytest.mark.parametrize("dim,rot,interleaved", [(128, 64, False), (33, 6, True)])
def test_norm_of_huge_and_tiny_rows(dim, rot, interleaved, power, eps):
    """fp32 rows of values near 2^power, beside ordinary ones; the tolerance of
    test_gpu_kv_norm.py, and half of the last place of fp32 (2^-150) where
    results are subnormal."""
    print(f"[kv norm edges] 2^{power} {dim} {eps}", file=sys.stderr, flush=True)
    q, k, v, kp, vp, cache, pos, cs = setup(dim, rot, torch.float32)
    gen = torch.Generator(device="cuda").manual_seed(power + 200)
    for x in (q, k):
        x.copy_(torch.rand(x.shape, generator=gen, device="cuda") - 0.5)
        x[::3] = torch.ldexp(x[::3].double(), torch.tensor(power, device="cuda")).float()
    weight = torch.rand(dim, device="cuda") + 0.5
    q_out = torch.zeros_like(q)
    nm.nmspmm_kv_append_norm(cache, k, v, torch.zeros_like(pos), pos, q=q, q_out=q_out, q_norm=weight, k_norm=weight,
                             eps=eps, interleaved=interleaved, **cs)
    torch.cuda.synchronize()
    c, s = (f64(cs[x]) for x in ("cos", "sin"))
    for got, x in ((kp.view(-1, *k.shape[1:])[:len(pos)], k), (q_out, q)):
        want, err = turn64(norm64(f64(x), f64(weight), np.float64(np.float32(eps))), c, s, rot, interleaved, True)
        assert np.all(np.isfinite(want))
        # (the two products of a subnormal result round to its last place each)
        assert np.all(np.abs(f64(got) - want) <= err + 2.0 ** -24 * np.abs(want) + 3 * 2.0 ** -150)
