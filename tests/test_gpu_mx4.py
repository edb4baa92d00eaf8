"""The product with a 4-bit weight (nmspmm_mx4_*) against plain fp64.

Tolerance, derived: the product of a 16-bit value and one of 4 bits is exact in
fp32, and so is its product with a power of two; a sum of w terms in any order
errs by at most w * 2^-24 of the sum of absolute terms; the epilogue as in the
16-bit product: a few roundings of 2^-24, the activation's own error below
2^-20 of its argument, slopes of at most 1.13; the store rounds once, by at
most u = 2^-8 (bf16), 2^-11 (fp16) or 2^-24 (fp32) of the result, or 2^-25
absolute where fp16 is subnormal.
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

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def say(msg):
    print(msg, file=sys.stderr, flush=True)


def f64(t):
    return t.double().cpu().numpy()


def pattern(rng, k, n, N, M, V):
    """Offsets (w x q), increasing within a window."""
    keep = np.sort(rng.random((k // M, n // V, M)).argsort(-1)[..., :N], axis=-1)
    return np.ascontiguousarray(keep.transpose(0, 2, 1).reshape(k // M * N, n // V).astype(np.uint8))


def dense(kept, idx, k, n, N, M, V):
    """The weight as a k x n matrix of its kept rows' values."""
    B = np.zeros((k, n))
    at = np.arange(kept.shape[0])[:, None] // N * M + np.repeat(idx.astype(np.int64), V, axis=1)
    np.put_along_axis(B, at, kept, axis=0)
    return B


def weight_of(rng, k, n, N, M, V, scales=None, ints=False):
    """A packed weight of random codes, and the matrix it stands for.  Scales
    are drawn from `scales` (bytes)."""
    w, groups = k // M * N, (k // M * N + 31) // 32
    codes = rng.integers(0, 16, (w, n)).astype(np.uint8)
    if ints:
        codes = rng.choice(np.array([0, 2, 4, 5, 6, 7, 10, 12, 13, 14, 15], dtype=np.uint8), (w, n))
    byte = rng.choice(np.array([127] if ints else scales or range(115, 125)), (groups, n)).astype(np.uint8)
    idx = pattern(rng, k, n, N, M, V)
    weight = nm.nmspmm_mx4_pack(*(torch.from_numpy(x).cuda() for x in (codes, byte, idx)), n, k, N, M, V)
    full = np.repeat(byte.astype(np.int64), 32, axis=0)[:w]
    return weight, dense(plain.values_of(codes.astype(np.int64), full), idx, k, n, N, M, V)


def rows_of(rng, m, k, dtype, ints=False, pad=0, off=0):
    x = rng.integers(-2, 3, (m, k)) if ints else rng.standard_normal((m, k))
    wide = torch.full((m, off + k + pad), float("nan"), dtype=DTYPES[dtype], device="cuda")
    A = wide[:, off:off + k]
    A.copy_(torch.from_numpy(x.astype(np.float32)))
    return A


def act64(y, act):
    from scipy.special import erfc
    if act == "relu":
        return np.maximum(y, 0)
    if act == "gelu":
        return 0.5 * y * erfc(-y / np.sqrt(2))
    if act == "silu":
        return y / (1 + np.exp(-y))
    return y


def reference(A, B, alpha, bias, act, mul, residual, out):
    """The fp64 result and its tolerance."""
    w = max(1, B.shape[0])
    y = alpha * (A @ B)
    err = abs(alpha) * (np.abs(A) @ np.abs(B)) * (w + 4) * 2.0 ** -24
    if bias is not None:
        y = y + bias
        err = err + np.abs(y) * 2.0 ** -23
    err = 1.13 * err + np.abs(y) * 2.0 ** -20
    y = act64(y, act)
    if mul is not None:
        y, err = y * mul, err * np.abs(mul) + np.abs(y * mul) * 2.0 ** -24
    if residual is not None:
        y = y + residual
        err = err + np.abs(y) * 2.0 ** -24
    return y, err * (1 + 2.0 ** -6) + np.abs(y) * ROUND[out] + (2.0 ** -25 if out == "f16" else 0)


def check(C, y, tol, what):
    got = f64(C)
    assert np.all(np.isfinite(got)), what
    err = np.abs(got - y)
    bad = err > tol
    assert not bad.any(), f"{what}: {bad.sum()} off, worst err/tol {np.max(err / np.maximum(tol, 1e-300)):.3f} at " \
                          f"{np.unravel_index(np.argmax(err - tol), err.shape)}"


SHAPES = [
    # m, k, n, N, M, V
    (1, 32, 16, 32, 32, 16), (1, 32, 16, 16, 32, 16), (1, 64, 32, 4, 32, 32), (1, 4096, 512, 4, 32, 64),
    (1, 1024, 1056, 32, 32, 32), (1, 8192, 128, 4, 32, 64), (2, 256, 64, 8, 32, 32), (3, 2048, 256, 2, 4, 16),
    (4, 4000, 64, 32, 32, 64), (5, 96, 48, 12, 32, 48), (7, 1120, 128, 12, 32, 32), (8, 512, 128, 32, 32, 32),
    (13, 1600, 320, 8, 32, 32), (15, 1600, 320, 12, 32, 32), (16, 8192, 256, 32, 32, 64), (16, 11008, 64, 16, 32, 32),
    (17, 256, 192, 1, 32, 64), (31, 512, 64, 4, 16, 16), (33, 1056, 96, 16, 32, 32), (37, 4096, 352, 8, 32, 32),
    (48, 768, 128, 32, 32, 128), (64, 2048, 224, 20, 32, 32), (65, 512, 160, 31, 32, 32), (100, 288, 272, 16, 32, 16),
    (200, 1024, 96, 32, 32, 96), (6, 131072, 32, 2, 32, 32), (1, 70000, 16, 5, 100, 16),
    # patterns and blocks that fit no matrix instruction, rows off 16 bytes
    (7, 24, 10, 3, 8, 2), (40, 28, 21, 2, 7, 3), (9, 512, 40, 5, 256, 8), (20, 100, 48, 7, 10, 16),
    (33, 243, 64, 4, 9, 32), (70, 770, 96, 1, 77, 32), (12, 256, 96, 1, 256, 32), (66, 1024, 32, 255, 256, 32),
    (4, 16, 16, 1, 1, 16), (130, 21, 33, 3, 3, 11), (3, 2560, 32, 1, 256, 16), (2, 7, 16, 7, 7, 16), (5, 65, 32, 2, 5, 32),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product(shape, dtype):
    m, k, n, N, M, V = shape
    say(f"[mx4] {shape} {dtype}")
    rng = np.random.default_rng(m + k + n)
    weight, B = weight_of(rng, *shape[1:])
    A = rows_of(rng, m, k, dtype)
    for out in (dtype, "f32"):
        C = torch.full((m, n), float("nan"), dtype=DTYPES[out], device="cuda")
        nm.nmspmm_mx4_run(A, weight, C)
        torch.cuda.synchronize()
        check(C, *reference(f64(A), B, 1.0, None, "none", None, None, out), f"{shape} {dtype}->{out}")


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product_exact_on_integers(shape, dtype):
    """Small integers: every partial sum is an exact fp32 integer, so any
    order of summation gives the exact result; with the library's workspace, a
    caller's, and one that is too small."""
    m, k, n, N, M, V = shape
    say(f"[mx4] exact {shape} {dtype}")
    rng = np.random.default_rng(m + k + n + 1)
    weight, B = weight_of(rng, *shape[1:], ints=True)
    A = rows_of(rng, m, k, dtype, ints=True)
    size = nm.nmspmm_mx4_workspace_bytes(m, weight)
    assert size >= 0
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
    for workspace in (None, ws, ws, ws[:1]):
        C = torch.full((m, n), float("nan"), device="cuda")
        nm.nmspmm_mx4_run(A, weight, C, workspace=workspace)
        assert np.array_equal(f64(C), f64(A) @ B)


EPILOGUES = [(1.0, False, "none", False, True), (8.0, True, "gelu", False, False), (2.0, True, "silu", True, False),
             (-0.5, False, "relu", True, True), (1.0, True, "none", True, True)]


@pytest.mark.parametrize("alpha,bias,act,mul,residual", EPILOGUES)
@pytest.mark.parametrize("dtype,out", [("bf16", "bf16"), ("bf16", "f32"), ("f16", "f16"), ("f16", "f32")])
@pytest.mark.parametrize("shape", [(1, 512, 96, 4, 32, 32), (9, 320, 64, 32, 32, 64), (21, 60, 36, 3, 12, 6),
                                   (40, 4096, 64, 16, 32, 32)], ids=lambda s: "x".join(map(str, s)))
def test_epilogue(shape, dtype, out, alpha, bias, act, mul, residual):
    """Every epilogue, on rows of odd strides, in place of the factor or the term."""
    m, k, n, N, M, V = shape
    say(f"[mx4] epilogue {shape} {dtype}->{out} {alpha} {bias} {act} {mul} {residual}")
    rng = np.random.default_rng(m + n)
    weight, B = weight_of(rng, *shape[1:])
    for pad, off in ((0, 0), (5, 3), (8, 8)):
        A = rows_of(rng, m, k, dtype, pad=pad, off=off)
        b = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() if bias else None
        x, y = (rows_of(rng, m, n, out, pad=pad, off=off) if on else None for on in (mul, residual))
        want, tol = reference(f64(A), B, alpha, f64(b) if bias else None, act, f64(x) if mul else None,
                              f64(y) if residual else None, out)
        C = torch.full((m, n + pad), 7.0, dtype=DTYPES[out], device="cuda")
        nm.nmspmm_mx4_run(A, weight, C[:, :n], alpha=alpha, bias=b, act=act, mul=x, residual=y)
        check(C[:, :n], want, tol, "apart")
        assert torch.all(C[:, n:] == 7.0)
        place = y if residual else x
        if place is not None:
            nm.nmspmm_mx4_run(A, weight, place, alpha=alpha, bias=b, act=act, mul=x, residual=y)
            check(place, want, tol, "in place")


def test_dense_without_offsets():
    """N = M: the offsets are the rows themselves, and idx may be left out."""
    rng = np.random.default_rng(4)
    k, n, N, M, V = 320, 64, 32, 32, 32
    codes = torch.from_numpy(rng.integers(0, 16, (k, n)).astype(np.uint8)).cuda()
    byte = torch.from_numpy(rng.integers(118, 124, (k // 32, n)).astype(np.uint8)).cuda()
    idx = torch.from_numpy(pattern(rng, k, n, N, M, V)).cuda()
    one = nm.nmspmm_mx4_pack(codes, byte, None, n, k, N, M, V)
    two = nm.nmspmm_mx4_pack(codes, byte, idx, n, k, N, M, V)
    A = rows_of(rng, 3, k, "bf16")
    C = [torch.empty(3, n, device="cuda") for _ in range(2)]
    nm.nmspmm_mx4_run(A, one, C[0])
    nm.nmspmm_mx4_run(A, two, C[1])
    B = plain.values_of(codes.cpu().numpy().astype(np.int64),
                        np.repeat(byte.cpu().numpy().astype(np.int64), 32, axis=0))
    check(C[0], *reference(f64(A), B, 1.0, None, "none", None, None, "f32"), "no idx")
    assert torch.equal(C[0], C[1])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_every_scale(dtype):
    """Scales over their whole range: a group of scale s times rows that bring
    it back near 1 (bf16 rows reach 2^-100 and 2^100, fp16 rows 2^-14 and
    2^14), other groups zero."""
    say(f"[mx4] scales {dtype}")
    rng = np.random.default_rng(6)
    k, n = 96, 32
    reach = 100 if dtype == "bf16" else 14
    for s in (0, 1, 2, 13, 60, 113, 127, 141, 200, 240, 251, 252):
        e = int(np.clip(127 - s, -reach, reach))
        codes = rng.integers(0, 16, (k, n)).astype(np.uint8)
        codes[:32] = codes[64:] = 0
        byte = np.full((3, n), s, dtype=np.uint8)
        weight = nm.nmspmm_mx4_pack(torch.from_numpy(codes).cuda(), torch.from_numpy(byte).cuda(), None, n, k, 32, 32, 32)
        A = torch.from_numpy(rng.integers(-2, 3, (5, k)) * 2.0 ** e).to(DTYPES[dtype]).cuda()
        C = torch.empty(5, n, device="cuda")
        nm.nmspmm_mx4_run(A, weight, C)
        B = plain.values_of(codes.astype(np.int64), np.full((k, n), s))
        assert np.array_equal(f64(C), f64(A) @ B), s      # halves of integers times one power of two


def test_nan_scale_and_infinite_rows():
    """A group of scale 255 makes its column NaN; an infinity in a column of A
    that no kept row of a block meets leaves that block alone, where there are
    padding rows too (a weight of 8 kept rows)."""
    rng = np.random.default_rng(7)
    k, n, N, M, V = 64, 64, 4, 32, 32
    codes = rng.integers(1, 8, (8, n)).astype(np.uint8)
    byte = np.full((1, n), 127, dtype=np.uint8)
    byte[0, 40] = 255
    idx = np.zeros((8, 2), dtype=np.uint8)
    idx[:, 0], idx[:, 1] = [0, 1, 2, 3] * 2, [4, 5, 6, 31] * 2
    weight = nm.nmspmm_mx4_pack(*(torch.from_numpy(x).cuda() for x in (codes, byte, idx)), n, k, N, M, V)
    for dtype in ("bf16", "f16"):
        A = torch.ones(3, k, dtype=DTYPES[dtype], device="cuda")
        A[1, 0], A[1, 10], A[2, 63], A[0, 40] = float("inf"), float("nan"), float("-inf"), float("nan")
        C = torch.empty(3, n, device="cuda")
        nm.nmspmm_mx4_run(A, weight, C)
        got = f64(C)
        want = dense(plain.values_of(codes.astype(np.int64), np.full(codes.shape, 127)), idx, k, n, N, M, V).sum(0)
        assert np.all(np.isnan(got[:, 40]))
        got, want = np.delete(got, 40, 1), np.delete(want, 40)
        assert np.array_equal(got[0], want)
        assert np.all(np.isposinf(got[1, :32])) and np.array_equal(got[1, 32:], want[32:])
        assert np.array_equal(got[2, :32], want[:32]) and np.all(np.isneginf(got[2, 32:]))


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("w,n", [(1, 1), (31, 5), (32, 64), (33, 70), (128, 300), (100, 1)])
def test_quantize(w, n, dtype):
    """Codes and scales are those of the rule, to the bit: ordinary values,
    ties and borders of the scale, zeros, tiny and huge values, infinities."""
    rng = np.random.default_rng(w + n)
    x = rng.standard_normal((w, n)) * np.exp(rng.uniform(-9, 9, (1, n)))
    x = np.where(rng.random((w, n)) < 0.3, rng.choice([0.25, -0.75, 1.25, 1.75, 2.5, -3.5, 5.0, 7.0, 0.0], (w, n)), x)
    if n >= 5:
        x[:, 1], x[:, 2], x[0, 2] = 0, 0.25, 7.0
        x[0, 3] = np.inf
        x[:, 4] = x[:, 4] * (1e-42 if dtype != "f16" else 1e-6)
    if n >= 64:
        x[:, 10] = 3e38 if dtype != "f16" else 6e4
        x[w // 2, 11] = np.nan
    with np.errstate(over="ignore"):
        t = torch.from_numpy(x.astype(np.float32)).to(DTYPES[dtype])
    codes, scales = nm.nmspmm_mx4_quantize(t.cuda())
    v = t.double().numpy()
    byte = plain.group_bytes(v, 0)
    with np.errstate(invalid="ignore"):
        assert np.array_equal(scales.cpu().numpy(), byte[::32])
        assert np.array_equal(codes.cpu().numpy(), plain.codes_of(v, byte))


def test_quantized_weight_end_to_end():
    """Pruned on the GPU, brought to 4 bits, packed and multiplied: the product
    with the rounded values; rounding them again changes nothing."""
    rng = np.random.default_rng(8)
    k, n, N, M, V = 512, 128, 8, 32, 32
    B = torch.from_numpy(rng.standard_normal((k, n)).astype(np.float32)).cuda()
    Bc = torch.empty(k // M * N, n, device="cuda")
    idx = torch.empty(k // M * N, n // V, dtype=torch.uint8, device="cuda")
    nm.nmspmm_compress_device(B, Bc, idx, N, M, V)
    codes, scales = nm.nmspmm_mx4_quantize(Bc)
    weight = nm.nmspmm_mx4_pack(codes, scales, idx, n, k, N, M, V)
    kept = plain.rounded(f64(Bc), 0)
    A = rows_of(rng, 3, k, "bf16")
    C = torch.empty(3, n, device="cuda")
    nm.nmspmm_mx4_run(A, weight, C)
    check(C, *reference(f64(A), dense(kept, idx.cpu().numpy(), k, n, N, M, V), 1.0, None, "none", None, None, "f32"),
          "end to end")
    again = nm.nmspmm_mx4_quantize(torch.from_numpy(kept).float().cuda())
    full = np.repeat(again[1].cpu().numpy().astype(np.int64), 32, axis=0)
    assert np.array_equal(plain.values_of(again[0].cpu().numpy().astype(np.int64), full), kept)


@pytest.mark.parametrize("shape", [(1, 2048, 64, 32, 32, 32), (40, 4096, 64, 8, 32, 32)])
def test_streams_and_graphs(shape):
    """On a stream of its own, and replayed from graphs with and without a
    workspace between eager calls: the same bits."""
    m, k, n, N, M, V = shape
    rng = np.random.default_rng(9)
    weight, B = weight_of(rng, *shape[1:], ints=True)
    A = rows_of(rng, m, k, "bf16", ints=True)
    size = nm.nmspmm_mx4_workspace_bytes(m, weight)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda") if size else None
    out, bare, eager = (torch.empty(m, n, device="cuda") for _ in range(3))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    nm.nmspmm_mx4_run(A, weight, out, stream=side)
    torch.cuda.synchronize()
    assert np.array_equal(f64(out), f64(A) @ B)
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        nm.nmspmm_mx4_run(A, weight, out, workspace=ws)
    with torch.cuda.graph(g2):
        nm.nmspmm_mx4_run(A, weight, bare)
    for i in range(4):
        A.copy_(torch.from_numpy(rng.integers(-2, 3, (m, k)).astype(np.float32)))
        out.fill_(float("nan"))
        bare.fill_(float("nan"))
        g1.replay()
        g2.replay()
        nm.nmspmm_mx4_run(A, weight, eager)
        torch.cuda.synchronize()
        want = f64(A) @ B
        for got in (out, bare, eager):
            assert np.array_equal(f64(got), want), i
