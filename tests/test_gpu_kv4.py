"""The paged cache in 4 bits (nmspmm_kv4_*) against plain fp64.

What is written is compared by value, to the bit: keys are normalised and
turned in fp64, so that their codes differ from the plain ones only where both
come within some 2^-45 of a border, which no input here does.

Attention, tolerance derived as for the 16-bit cache: a score is a dot product
of dim terms and a scaling in fp32, off by at most es = (dim + 8) * 2^-24 *
scale * sum |q||k| (queries enter with all their bits); a weight is then off by
a factor of 1 +- (2 es + 2^-20) and a sum of L terms by L * 2^-24, all relative
to sum w|v|; weights enter with 24 bits (2^-24 each, within the 2^-20).  A
weight relative to the largest is an fp32 value, of which what lies below 2^-126
may be lost: L * 2^-126 * max|v| absolute (4-bit values are often zero, so that
a dimension may be left with nothing but such weights: e^-121 was met where
fp32 ends at e^-87).  The store rounds once.
"""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import mx4_plain as plain  # noqa: E402
import paper_2503_01253_amd as nm  # noqa: E402
from test_gpu_kv import DTYPES, LENGTHS, ROUND, attend64, close, f64, tensor  # noqa: E402
from test_gpu_kv_norm import SHAPES, norm64, setup, turn64  # noqa: E402


def say(msg):
    print(msg, file=sys.stderr, flush=True)


def pool_of(pages, page, heads, dim, pad=0, fill=0xff):
    """Pages full of NaN scales and codes, `pad` bytes apart."""
    size = nm.nmspmm_kv4_page_bytes(page, heads, dim)
    return torch.full((pages, size + pad), fill, dtype=torch.uint8, device="cuda")[:, :size]


def places(table, page, seq, pos):
    return torch.from_numpy(np.asarray(seq)).int().cuda(), torch.from_numpy(np.asarray(pos)).int().cuda()


@pytest.mark.parametrize("norms", ["both", "k", "none"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_append_and_read(shape, dtype, norms):
    tokens, heads, group, dim, page, rot, interleaved, layout = shape
    say(f"[kv4 append] {shape} {dtype} {norms}")
    rng, pages, table, seq, pos, q, k, v, cos, sin, c64, s64 = setup(*shape[:7], dtype, tokens + dim + 1)
    pool = pool_of(pages, page, heads, dim, pad=48 if layout == "padded" else 0)
    before = pool.clone()
    weights = {x: torch.from_numpy(rng.uniform(-2, 2, dim).astype(np.float32)).cuda() if norms in ("both", x) else None
               for x in "qk"}
    eps = 1e-3
    handle = nm.nmspmm_kv4_cache(pool, table, page, heads, dim)
    q_out = torch.full((tokens, group * heads, dim + 2), 5.0, dtype=DTYPES[dtype], device="cuda")[..., :dim]
    new = dict(cos=cos, sin=sin, interleaved=interleaved, q_norm=weights["q"], k_norm=weights["k"], eps=eps)
    at = places(table, page, seq, pos)
    w64 = {x: None if weights[x] is None else f64(weights[x]) for x in "qk"}
    want_k, _ = turn64(norm64(f64(k), w64["k"], eps), c64, s64, rot, interleaved, True)
    want_q = turn64(norm64(f64(q), w64["q"], eps), c64, s64, rot, interleaved, weights["q"] is not None)
    nm.nmspmm_kv4_append(handle, k, v, *at, q=q if group else None, q_out=q_out if group else None, **new)
    if group:
        close(f64(q_out), *want_q, dtype, "queries")
    for out in ("f32", "bf16", "f16"):
        wide = torch.full((2, tokens, heads, dim + 3), 9.0, dtype=DTYPES[out], device="cuda")
        k_out, v_out = wide[0, ..., :dim], wide[1, ..., :dim]
        nm.nmspmm_kv4_read(handle, *at, k_out, v_out)
        torch.cuda.synchronize()
        assert torch.all(wide[..., dim:] == 9.0)
        for got, want in ((k_out, plain.rounded(want_k)), (v_out, plain.rounded(f64(v)))):
            want = torch.from_numpy(want).to(DTYPES[out]).double().numpy()
            assert np.array_equal(f64(got), want), f"{np.sum(f64(got) != want)} values differ"
    # what is read back and written again is what was there
    k_out, v_out = (torch.empty(tokens, heads, dim, device="cuda") for _ in range(2))
    nm.nmspmm_kv4_read(handle, *at, k_out, v_out)
    written = pool.clone()
    nm.nmspmm_kv4_append(handle, k_out, v_out, *at)
    k_again, v_again = (torch.empty_like(k_out) for _ in range(2))
    nm.nmspmm_kv4_read(handle, *at, k_again, v_again)
    assert torch.equal(k_again, k_out) and torch.equal(v_again, v_out)
    # pages that no token names are as they were
    used = np.unique(table.cpu().numpy()[seq, pos // page])
    rest = torch.from_numpy(np.setdiff1d(np.arange(pages), used)).cuda()
    assert torch.equal(written[rest], before[rest])


def test_neighbours_stay():
    """Tokens written one after another into one page, in any order, leave
    each other's rows alone, and slots that none names read as they were."""
    rng = np.random.default_rng(2)
    for page, dim in ((16, 128), (7, 64), (24, 80), (1, 96), (6, 300)):
        heads, pages = 2, 3
        pool = pool_of(pages, page, heads, dim)
        table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
        handle = nm.nmspmm_kv4_cache(pool, table, page, heads, dim)
        k, v = (tensor(rng, (pages * page, heads, dim), "f32") for _ in range(2))
        order = rng.permutation(pages * page)[:pages * page - 1]
        for t in order:
            nm.nmspmm_kv4_append(handle, k[t:t + 1], v[t:t + 1], *places(table, page, [0], [t]))
        k_out, v_out = (torch.empty_like(k) for _ in range(2))
        nm.nmspmm_kv4_read(handle, *places(table, page, [0] * (pages * page), range(pages * page)), k_out, v_out)
        missing = np.setdiff1d(np.arange(pages * page), order)[0]
        for got, x in ((f64(k_out), k), (f64(v_out), v)):
            assert np.all(np.isnan(got[missing]))
            want = plain.rounded(f64(x))
            assert np.array_equal(np.delete(got, missing, 0), np.delete(want, missing, 0)), (page, dim)


def test_ties_borders_and_infinities():
    """Values on ties and on the scale's border, tiny and huge ones; a group
    with an infinity or NaN reads as NaN, its neighbours do not."""
    dim, page = 96, 16
    rng = np.random.default_rng(5)
    x = rng.choice([0.25, -0.75, 1.25, 1.75, 2.5, -3.5, 5.0, 0.0, 6.0, -0.0], (16, 1, dim))
    x[0, 0, 0], x[1, 0, 5], x[2, 0, 64] = 7.0, 7.03125, -7.0
    x[3], x[4], x[5], x[6] = 0, x[4] * 1e-39, x[5] * 5e37, 3.3e38
    x[7, 0, 40], x[8, 0, 0], x[9, 0, 95] = np.inf, np.nan, -np.inf
    k = torch.from_numpy(x.astype(np.float32)).cuda()
    pool = pool_of(1, page, 1, dim)
    handle = nm.nmspmm_kv4_cache(pool, torch.zeros(1, 1, dtype=torch.int32, device="cuda"), page, 1, dim)
    at = torch.zeros(16, dtype=torch.int32, device="cuda"), torch.arange(16, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(handle, k, -k, *at)
    k_out, v_out = (torch.empty_like(k) for _ in range(2))
    nm.nmspmm_kv4_read(handle, *at, k_out, v_out)
    want = plain.rounded(f64(k))
    assert np.array_equal(f64(k_out), want, equal_nan=True) and np.array_equal(f64(v_out), -want, equal_nan=True)
    assert np.isnan(want[7, 0, 32:64]).all() and np.isfinite(want[7, 0, :32]).all()
    # the same through a rotation by nothing, in fp64
    ones, none = torch.ones(16, dim // 2, device="cuda"), torch.zeros(16, dim // 2, device="cuda")
    finite = torch.nan_to_num(k, nan=1.0, posinf=2.0, neginf=3.0)
    nm.nmspmm_kv4_append(handle, finite, finite, *at, cos=ones, sin=none)
    nm.nmspmm_kv4_read(handle, *at, k_out, v_out)
    assert np.array_equal(f64(k_out), plain.rounded(f64(finite))) and torch.equal(k_out, v_out)


def test_keys_next_to_a_border():
    """Turned keys whose fp32 value would fall on a tie or on its other side:
    the codes are those of the exact value."""
    dim, page, T = 64, 64, 64
    rng = np.random.default_rng(6)
    # pairs (a, b) with a*c - b*s = a border and a little: c = 1, s = 2^-30 to 2^-28
    k = np.zeros((T, 1, dim))
    k[..., :32] = rng.choice([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], (T, 1, 32))
    k[..., 0] = 6.0
    k[..., 32:] = rng.choice([-1.0, 1.0], (T, 1, 32))
    cos = np.ones((T, 32))
    sin = rng.integers(1, 5, (T, 32)) * 2.0 ** -30
    t = torch.from_numpy(k.astype(np.float32)).cuda()
    handle = nm.nmspmm_kv4_cache(pool_of(1, page, 1, dim), torch.zeros(1, 1, dtype=torch.int32, device="cuda"), page, 1, dim)
    at = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(handle, t, t, *at, cos=torch.from_numpy(cos).float().cuda(), sin=torch.from_numpy(sin).float().cuda())
    k_out = torch.empty_like(t)
    nm.nmspmm_kv4_read(handle, *at, k_out)
    want = k.copy()
    want[..., :32], want[..., 32:] = k[..., :32] - k[..., 32:] * sin[:, None], k[..., :32] * sin[:, None] + k[..., 32:]
    assert np.array_equal(f64(k_out), plain.rounded(want))
    assert not np.array_equal(plain.rounded(want), plain.rounded(want.astype(np.float32).astype(np.float64)))


def test_skips_tokens_without_a_place():
    rng = np.random.default_rng(3)
    heads, dim, page, pages = 2, 64, 4, 6
    pool = pool_of(pages, page, heads, dim)
    table = torch.tensor([[0, 1, 99], [-1, 2, 3]], dtype=torch.int32).cuda()
    seq = torch.tensor([0, 0, 2, -1, 1, 0, 0, 1, 1, 0], dtype=torch.int32).cuda()
    pos = torch.tensor([-1, 12, 0, 0, 1, 9, 5, 4, 10, 2 ** 31 - 1], dtype=torch.int32).cuda()
    written = {6, 7}          # token 8 lies past the angles
    k, v, q = (tensor(rng, (len(seq), heads, dim), "bf16") for _ in range(3))
    q_out = torch.full_like(q, 3.0)
    angle = torch.zeros(10, 32).cuda()
    handle = nm.nmspmm_kv4_cache(pool, table, page, heads, dim)
    nm.nmspmm_kv4_append(handle, k, v, seq, pos, cos=angle.cos(), sin=angle.sin(), q=q, q_out=q_out)
    k_out, v_out = (torch.full((len(seq), heads, dim), 3.0, device="cuda") for _ in range(2))
    nm.nmspmm_kv4_read(handle, seq, pos, k_out, v_out)
    want_k, want_v = plain.rounded(f64(k)), plain.rounded(f64(v))
    for t in range(len(seq)):
        if t in written:
            assert np.array_equal(f64(k_out[t]), want_k[t]) and np.array_equal(f64(v_out[t]), want_v[t])
            assert torch.equal(q_out[t], q[t])
        elif t == 8:        # a place of its own, never written
            assert torch.isnan(k_out[t]).all() and torch.isnan(v_out[t]).all() and torch.all(q_out[t] == 3.0)
        else:
            assert torch.all(k_out[t] == 3.0) and torch.all(v_out[t] == 3.0) and torch.all(q_out[t] == 3.0)
    for only, other in (({"k_out": k_out}, k_out), ({"v_out": v_out}, v_out)):
        again = other.clone()
        other.fill_(3.0)
        nm.nmspmm_kv4_read(handle, seq, pos, **only)
        assert torch.equal(other.nan_to_num(), again.nan_to_num())


# ---- attend ----------------------------------------------------------------

def run_attend(lengths, heads, group, dim, page, dtype, window=0, scale=None, seed=0, spread=1.0, workspace="library",
               max_length=None, wide=None, pad=0):
    rng = np.random.default_rng(seed + dim + sum(lengths))
    B = len(lengths)
    need = [-(-max(x, 0) // page) for x in lengths]
    wide = wide or max(need + [1])
    pages = sum(need) + 2
    pool = pool_of(pages, page, heads, dim, pad=pad)      # what no sequence holds is NaN: it must not matter
    table = torch.full((B, wide), 2 ** 30, dtype=torch.int32)
    order = iter(rng.permutation(pages - 1) + 1)
    for b in range(B):
        ids = [int(next(order)) for _ in range(need[b])]
        table[b, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    handle = nm.nmspmm_kv4_cache(pool, table.cuda(), page, heads, dim)
    K, V = [], []
    for b, x in enumerate(lengths):
        x = max(x, 0)
        k, v = tensor(rng, (x, heads, dim), "f32") * spread, tensor(rng, (x, heads, dim), "f32")
        at = torch.full((x,), b, dtype=torch.int32, device="cuda"), torch.arange(x, dtype=torch.int32, device="cuda")
        if x:       # (numpy's empty arrays have strides of their own)
            nm.nmspmm_kv4_append(handle, k, v, *at)
            nm.nmspmm_kv4_read(handle, *at, k, v)
        K.append(f64(k))
        V.append(f64(v))
    q = tensor(rng, (B, heads * group, dim), dtype)
    out = torch.full((B, heads * group, dim + 3), 9.0, dtype=DTYPES[dtype], device="cuda")
    lse = torch.full((B, heads * group), float("nan"), device="cuda")
    ws = None
    if workspace == "caller":
        size = nm.nmspmm_kv4_attend_workspace_bytes(handle, heads * group, max_length or wide * page, window)
        assert size >= 0
        ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
    nm.nmspmm_kv4_attend(handle, q, torch.tensor(lengths, dtype=torch.int32).cuda(), out[..., :dim], scale=scale,
                         window=window, max_length=max_length, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    assert torch.all(out[..., dim:] == 9.0)
    got, got_lse, q64 = f64(out[..., :dim]), f64(lse), f64(q)
    scale = dim ** -0.5 if scale is None else scale
    for b, x in enumerate(lengths):
        x = min(max(x, 0), wide * page, max_length if max_length is not None else x)
        first = max(0, x - window) if window else 0
        want, err, want_lse = attend64(q64[b].reshape(heads, group, dim), K[b][first:x], V[b][first:x], scale, False)
        tol = err * (1 + 2.0 ** -6) + np.abs(want) * ROUND[dtype] + (2.0 ** -25 if dtype == "f16" else 0)
        tol += (x - first) * 2.0 ** -126 * np.abs(V[b][first:x]).max(initial=0)
        diff = np.abs(got[b].reshape(want.shape) - want)
        worst = np.unravel_index(np.argmax(diff / np.maximum(tol, 1e-300)), diff.shape)
        assert np.all(diff <= tol), f"sequence {b} of length {x}: {got[b].reshape(want.shape)[worst]} for " \
                                    f"{want[worst]}, {np.sum(diff > tol)} off, tolerance {tol[worst]}"
        if x > first:
            L = x - first
            bound = np.abs(want_lse) * 2.0 ** -22 + (dim + 8) * 2.0 ** -24 * abs(scale) * np.einsum(
                "hgd,lhd->hgl", np.abs(q64[b].reshape(heads, group, dim)), np.abs(K[b][first:x])).max(-1) + \
                L * 2.0 ** -24 + 2.0 ** -20
            assert np.all(np.abs(got_lse[b].reshape(want_lse.shape) - want_lse) <= bound)
        else:
            assert np.all(got_lse[b] == -np.inf) and np.all(got[b] == 0)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("heads,group,dim,page", [
    (1, 1, 64, 16), (8, 4, 128, 16), (2, 8, 128, 16), (4, 1, 64, 32), (2, 3, 80, 24), (3, 7, 96, 1), (1, 16, 128, 64),
    (2, 5, 256, 16), (1, 2, 33, 7), (2, 4, 128, 8), (1, 20, 64, 16), (1, 1, 512, 16), (1, 33, 128, 16), (2, 2, 8, 3),
    (1, 1, 1, 5), (2, 2, 300, 9), (2, 16, 112, 48), (1, 6, 192, 16), (2, 8, 48, 16), (1, 4, 16, 16), (1, 4, 160, 20),
    (2, 2, 32, 4), (1, 3, 96, 16), (1, 2, 224, 32), (1, 8, 128, 2), (2, 4, 64, 12)])
def test_attend(heads, group, dim, page, dtype):
    say(f"[kv4 attend] {heads}x{group} dim {dim} page {page} {dtype}")
    run_attend(LENGTHS, heads, group, dim, page, dtype, pad=32 if page == 24 else 0)


@pytest.mark.parametrize("workspace", ["library", "caller"])
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("lengths,heads,group,dim,page", [
    ([5000], 2, 4, 128, 16), ([4097, 3, 0, 2048], 1, 8, 64, 64), ([3000, 2999], 2, 1, 80, 24), ([9001], 1, 16, 128, 16),
    ([2500, 1], 1, 3, 256, 32), ([3001], 1, 2, 128, 7)])
def test_attend_split(lengths, heads, group, dim, page, dtype, workspace):
    say(f"[kv4 attend] split {lengths} {heads}x{group} dim {dim} page {page} {dtype} {workspace}")
    run_attend(lengths, heads, group, dim, page, dtype, workspace=workspace)


@pytest.mark.parametrize("window", [1, 15, 64, 100, 1024, 10 ** 6])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 24), (128, 5)])
def test_attend_window(window, dim, page):
    say(f"[kv4 attend] window {window} {dim} {page}")
    run_attend([0, 1, 64, 65, 99, 101, 1500, 4096], 2, 4, dim, page, "bf16", window=window)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("page", [16, 6])
def test_attend_bounds_and_scales(dtype, page):
    """Lengths beyond max_length and beyond the table are cut; a scale of 0
    averages, a negative one inverts; large scores neither overflow nor
    underflow into NaN."""
    say(f"[kv4 attend] bounds {dtype} {page}")
    run_attend([10, 100, 300, 299], 2, 4, 64, page, dtype, max_length=100)
    run_attend([0, 7, 300], 2, 4, 64, page, dtype, scale=0.0)
    run_attend([1, 7, 300], 2, 4, 64, page, dtype, scale=-0.3)
    run_attend([1, 40, 3000], 2, 4, 64, page, dtype, scale=4.0, spread=8.0)
    run_attend([0, 0, 0], 2, 4, 64, page, dtype)


@pytest.mark.parametrize("dim,page", [(128, 16), (33, 16), (128, 8), (96, 5)])
def test_attend_leaves_out_pages_outside_the_cache(dim, page):
    """A table entry below 0 or past the cache's pages: its positions do not
    count, as if the sequence did not hold them."""
    rng = np.random.default_rng(5)
    heads, group, pages = 2, 4, 5
    pool = pool_of(pages, page, heads, dim)
    q = tensor(rng, (3, heads * group, dim), "f32")
    full = torch.tensor([[4, -1, 2, 2 ** 31 - 1, 0], [-5, 7, 9, 5, -1], [1, 2, 3, 0, 4]], dtype=torch.int32).cuda()
    near = torch.tensor([[4, 2, 0], [0, 0, 0], [1, 2, 3]], dtype=torch.int32).cuda()
    whole = nm.nmspmm_kv4_cache(pool, torch.arange(pages, dtype=torch.int32, device="cuda")[None], page, heads, dim)
    k, v = (tensor(rng, (pages * page, heads, dim), "f32") for _ in range(2))
    pos = torch.arange(pages * page, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(whole, k, v, torch.zeros_like(pos), pos)
    out, want = torch.empty_like(q), torch.empty_like(q)
    last = page - 3
    cache = [nm.nmspmm_kv4_cache(pool, t, page, heads, dim) for t in (full, near)]
    nm.nmspmm_kv4_attend(cache[0], q, torch.tensor([4 * page + last, 5 * page, 3 * page]).int().cuda(), out)
    nm.nmspmm_kv4_attend(cache[1], q, torch.tensor([2 * page + last, 0, 3 * page]).int().cuda(), want)
    torch.cuda.synchronize()
    assert torch.all(out[1] == 0)
    assert torch.all((out - want).abs() <= 2.0 ** -18 * (want.abs() + 1))      # order of the sums


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("dim", [32, 64, 96, 128, 256])
@pytest.mark.parametrize("page", [8, 24, 16, 4, 5, 32])
def test_attend_counts_the_positions_that_are_there(page, dim, dtype):
    """With a scale of 0 every position weighs 1: the log-sum-exp counts them,
    over tables whose pages are there, one or all missing, at lengths that end
    inside and at the end of a page."""
    say(f"[kv4 attend] counts {page} {dim} {dtype}")
    rng = np.random.default_rng(6)
    heads, group, pages = 2, 4, 5
    pool = pool_of(pages, page, heads, dim)
    whole = nm.nmspmm_kv4_cache(pool, torch.arange(pages, dtype=torch.int32, device="cuda")[None], page, heads, dim)
    k, v = (tensor(rng, (pages * page, heads, dim), "f32") for _ in range(2))
    pos = torch.arange(pages * page, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(whole, k, v, torch.zeros_like(pos), pos)
    tables = [[-5, 7, 9, 5, -1], [4, -1, 2 ** 31 - 1, -2 ** 31, 5], [-1, 4, -1, -1, -1], [-1, -1, 4, -1, -1],
              [-1, -1, -1, -1, 4], [0, 1, 2, 3, 4], [3, 2, -1, 1, 0]]
    handle = nm.nmspmm_kv4_cache(pool, torch.tensor(tables, dtype=torch.int32).cuda(), page, heads, dim)
    q = tensor(rng, (len(tables), heads * group, dim), dtype)
    out, lse = torch.empty_like(q), torch.empty(len(tables), heads * group, device="cuda")
    for length in (1, page, page + 1, 2 * page, 3 * page - 1, 5 * page):
        for window in (0, 1, page, 2 * page + 1):
            nm.nmspmm_kv4_attend(handle, q, torch.full((len(tables),), length, dtype=torch.int32, device="cuda"), out,
                                 lse=lse, scale=0.0, window=window)
            first = max(0, length - window) if window else 0
            want = [sum(0 <= table[i // page] < pages for i in range(first, length)) for table in tables]
            got = np.exp(f64(lse))
            assert np.all(np.abs(got - np.array(want)[:, None]) <= 1e-4 * np.array(want)[:, None]), (length, window)


def test_attend_a_row_of_infinite_scores():
    """Keys whose scores are all minus infinity (q of -3e38 times k of 2^125): a zero
    row with lse minus infinity; a NaN group inside the range makes its heads NaN,
    outside it does not matter."""
    dim, page = 64, 16
    pool = pool_of(4, page, 2, dim)
    handle = nm.nmspmm_kv4_cache(pool, torch.arange(4, dtype=torch.int32, device="cuda")[None], page, 2, dim)
    k = torch.full((40, 2, dim), 2.0 ** 126, device="cuda")
    k[:, 1] = 1.0
    v = torch.ones(40, 2, dim, device="cuda")
    v[20, 1, 40] = float("nan")
    at = torch.zeros(40, dtype=torch.int32, device="cuda"), torch.arange(40, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(handle, k, v, *at)
    for dtype in ("bf16", "f32"):
        q = torch.full((1, 2, dim), -3e38, dtype=DTYPES[dtype], device="cuda")
        q[:, 1] = 1.0
        for length, first in ((40, False), (20, True)):
            out = torch.empty_like(q)
            lse = torch.empty(1, 2, device="cuda")
            nm.nmspmm_kv4_attend(handle, q, torch.tensor([length]).int().cuda(), out, lse=lse, scale=1.0)
            assert torch.all(out[0, 0] == 0) and lse[0, 0] == -float("inf")
            assert torch.all(out[0, 1, :32] == 1.0)
            assert torch.all(out[0, 1, 32:] == 1.0) if first else torch.isnan(out[0, 1, 32:]).all()


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("first", [0, 1, 199])
@pytest.mark.parametrize("page", [8, 16, 5])
def test_many_weights_below_half_a_step(first, dtype, page):
    """One position 17.5 above the others, whose values are zero: the others'
    weights, e^-17.5 each, make the whole result."""
    say(f"[kv4] small weights {first} {dtype} {page}")
    dim, length = 64, 200
    pages = 40
    handle = nm.nmspmm_kv4_cache(pool_of(pages, page, 1, dim), torch.arange(pages, dtype=torch.int32, device="cuda")[None],
                                 page, 1, dim)
    k, v = torch.zeros(length, 1, dim, device="cuda"), torch.full((length, 1, dim), 768.0, device="cuda")
    k[first, 0, 0], k[first, 0, 1], v[first] = 16.0, 1.5, 0.0       # 1.5 in units of 4: 2 (a tie goes to the even code)
    at = torch.zeros(length, dtype=torch.int32, device="cuda"), torch.arange(length, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(handle, k, v, *at)
    nm.nmspmm_kv4_read(handle, *at, k, v)
    q = torch.zeros(1, 3, dim)
    q[..., 0], q[..., 1] = 1.0, 0.75
    out = torch.empty(1, 3, dim, dtype=DTYPES[dtype], device="cuda")
    nm.nmspmm_kv4_attend(handle, q.to(DTYPES[dtype]).cuda(), torch.tensor([length]).int().cuda(), out, scale=1.0)
    top = float(k[first, 0, 0] + 0.75 * k[first, 0, 1])
    small = (length - 1) * np.exp(-top)
    want = 768.0 * small / (1.0 + small)
    assert np.all(np.abs(f64(out) - want) <= (2.0 ** -15 + ROUND[dtype]) * want)


def test_offsets_past_32_bits():
    """Pages whose bytes lie past 2^32, and past 2^32 pieces of 16 bytes between the strides of a few
    pages: written, read back, attended."""
    heads, dim, page, group = 2, 128, 16, 4
    size = nm.nmspmm_kv4_page_bytes(page, heads, dim)
    pages = 2 ** 33 // size + 40
    pool = torch.empty(pages, size, dtype=torch.uint8, device="cuda")
    wide = torch.empty(3 * 2 ** 34 + size, dtype=torch.uint8, device="cuda")      # 48 GiB
    far = wide.as_strided((4, size), (2 ** 34, 1))
    rng = np.random.default_rng(1)
    T = 40
    for store, ids in ((pool, [pages - 1, 0, pages - 7]), (far, [3, 0, 2])):
        handle = nm.nmspmm_kv4_cache(store, torch.tensor([ids], dtype=torch.int32).cuda(), page, heads, dim)
        k, v = (tensor(rng, (T, heads, dim), "f32") for _ in range(2))
        at = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.arange(T, dtype=torch.int32, device="cuda")
        nm.nmspmm_kv4_append(handle, k, v, *at)
        want = plain.rounded(f64(k)), plain.rounded(f64(v))
        nm.nmspmm_kv4_read(handle, *at, k, v)
        assert np.array_equal(f64(k), want[0]) and np.array_equal(f64(v), want[1])
        q = tensor(rng, (1, heads * group, dim), "f32")
        out = torch.empty_like(q)
        nm.nmspmm_kv4_attend(handle, q, torch.tensor([T]).int().cuda(), out)
        y, err, _ = attend64(f64(q)[0].reshape(heads, group, dim), *want, dim ** -0.5, False)
        assert np.all(np.abs(f64(out)[0].reshape(y.shape) - y) <= 1.02 * err + np.abs(y) * ROUND["f32"])


@pytest.mark.parametrize("page", [16, 24, 5])
def test_streams_graphs_and_determinism(page):
    """Append and attend on a stream of their own and replayed from graphs,
    lengths growing between replays: the same bits as eager calls."""
    say(f"[kv4] graph {page}")
    rng = np.random.default_rng(2)
    heads, group, dim, B, wide = 2, 4, 128, 3, 250
    pool = pool_of(B * wide, page, heads, dim, fill=120)
    table = torch.arange(B * wide, dtype=torch.int32).view(B, wide).cuda()
    handle = nm.nmspmm_kv4_cache(pool, table, page, heads, dim)
    k, v = (tensor(rng, (B, heads, dim), "bf16") for _ in range(2))
    q = tensor(rng, (B, heads * group, dim), "bf16")
    angle = torch.rand(wide * page, dim // 2).cuda()
    cos, sin, one = angle.cos(), angle.sin(), torch.ones(dim, device="cuda")
    seq = torch.arange(B).int().cuda()
    pos = torch.tensor([0, 777, 1200]).int().cuda()
    lengths = pos + 1
    size = nm.nmspmm_kv4_attend_workspace_bytes(handle, heads * group, wide * page)
    assert size > 0
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")

    def step(out, turned, stream=None, workspace=ws):
        nm.nmspmm_kv4_append(handle, k, v, seq, pos, cos=cos, sin=sin, q=q, q_out=turned, q_norm=one, k_norm=one,
                             stream=stream)
        nm.nmspmm_kv4_attend(handle, turned, lengths, out, stream=stream, workspace=workspace)

    turned, first, out, bare_out = (torch.empty_like(q) for _ in range(4))
    side = torch.cuda.Stream()
    step(first, turned)
    torch.cuda.synchronize()
    step(out, turned, stream=side, workspace=None)
    torch.cuda.synchronize()
    assert torch.equal(out, first)
    graph, bare = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out, turned)
    with torch.cuda.graph(bare):
        step(bare_out, turned, workspace=None)
    for _ in range(4):
        pos += 5
        lengths += 5
        out.fill_(float("nan"))
        bare_out.fill_(float("nan"))
        graph.replay()
        bare.replay()
        torch.cuda.synchronize()
        step(first, turned)
        torch.cuda.synchronize()
        assert torch.equal(out, first)
        tol = 2.0 ** -7      # one split or several: the order of the sums
        assert torch.all((bare_out.float() - first.float()).abs() <= tol * (first.float().abs() + 0.1))
