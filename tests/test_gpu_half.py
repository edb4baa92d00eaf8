"""The 16-bit N:M product (nmspmm_half_*) against a plain fp64 product of the
kept rows.

Tolerance, derived: the product of two 16-bit values is exact in fp32, and a
sum of w terms in any order errs by at most w * 2^-24 of the sum of absolute
terms; the epilogue adds a few roundings of 2^-24 and the activation's own
error (below 2^-20 of its argument); the activations' slopes are at most 1.13;
the store rounds once, by at most u = 2^-8 (bf16), 2^-11 (fp16) or 2^-24 (fp32)
of the result, or 2^-25 absolute where fp16 is subnormal.
"""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from nm_workloads import make_inputs  # noqa: E402

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def say(msg):
    print(msg, file=sys.stderr, flush=True)


def f64(t):
    return t.double().cpu().numpy()


def setup(m, k, n, N, M, V, dtype, seed=0, ints=False, a_pad=0, a_off=0):
    """Operands on the GPU (A with padded rows where asked) and the pruned
    weight's 16-bit values as a dense fp64 matrix."""
    A, Bp, _ = make_inputs(m, k, n, N, M, V, seed=seed + 7 * m + k + 3 * n, dist="int" if ints else "normal")
    if ints:
        A, Bp = np.clip(A, -2, 2), np.clip(Bp, -2, 2)
    Bc, idx = nm.nmspmm_compress(Bp, N, M, V)
    wide = torch.full((m, k + a_pad + a_off), float("nan"), dtype=DTYPES[dtype], device="cuda")
    dA = wide[:, a_off:a_off + k]
    dA.copy_(torch.from_numpy(A))
    weight = nm.nmspmm_half_pack(torch.from_numpy(Bc).cuda(), torch.from_numpy(idx).cuda(), n, k, N, M, V,
                                 dtype=DTYPES[dtype])
    B = f64(torch.from_numpy(Bp).to(DTYPES[dtype]))
    return dA, weight, B


def act64(y, act):
    from scipy.special import erf
    if act == "relu":
        return np.maximum(y, 0)
    if act == "gelu":
        return 0.5 * y * (1 + erf(y / np.sqrt(2)))
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
    (1, 32, 16, 16, 32, 16), (1, 64, 32, 4, 32, 32), (1, 1024, 512, 4, 32, 64), (1, 4096, 1056, 16, 32, 32),
    (2, 256, 64, 8, 32, 32), (3, 2048, 256, 2, 4, 16), (5, 96, 48, 12, 32, 48), (8, 512, 128, 32, 32, 32),
    (15, 1600, 320, 12, 32, 32), (16, 8192, 256, 4, 32, 64), (17, 256, 192, 1, 32, 64), (31, 512, 64, 4, 16, 16),
    (33, 1056, 96, 16, 32, 32), (37, 4096, 352, 8, 32, 32), (64, 768, 128, 12, 32, 128), (65, 320, 224, 20, 32, 32),
    (100, 512, 160, 31, 32, 32), (128, 2048, 256, 4, 32, 32), (129, 64, 512, 16, 32, 64), (200, 288, 272, 16, 32, 16),
    (257, 1024, 288, 8, 32, 32), (300, 2560, 544, 16, 32, 32), (512, 512, 512, 12, 32, 32), (1000, 256, 768, 4, 32, 64),
    # patterns and blocks that fit no matrix instruction
    (7, 24, 10, 3, 8, 2), (40, 28, 21, 2, 7, 3), (9, 512, 40, 5, 256, 8), (20, 100, 48, 7, 10, 16),
    (33, 243, 64, 4, 9, 32), (70, 770, 96, 1, 77, 32), (12, 256, 96, 1, 256, 32), (66, 1024, 32, 255, 256, 32),
    (4, 16, 16, 1, 1, 16), (130, 21, 33, 3, 3, 11),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product(shape, dtype):
    m, k, n, N, M, V = shape
    say(f"[half] {shape} {dtype}")
    A, weight, B = setup(*shape, dtype)
    for out in (dtype, "f32"):
        C = torch.full((m, n), float("nan"), dtype=DTYPES[out], device="cuda")
        nm.nmspmm_half_run(A, weight, C)
        torch.cuda.synchronize()
        check(C, *reference(f64(A), B, 1.0, None, "none", None, None, out), f"{shape} {dtype}->{out}")


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product_exact_on_integers(shape):
    """Small integers: every partial sum is an exact fp32 integer, so any
    order of summation gives the exact result."""
    m, k, n, N, M, V = shape
    say(f"[half] exact {shape}")
    A, weight, B = setup(*shape, "bf16", ints=True)
    C = torch.full((m, n), float("nan"), device="cuda")
    nm.nmspmm_half_run(A, weight, C)
    torch.cuda.synchronize()
    assert np.array_equal(f64(C), f64(A) @ B)
    # without the library's cached workspace, and with a caller's, twice
    size = nm.nmspmm_half_workspace_bytes(m, weight)
    assert size >= 0
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
    for _ in range(2):
        C.fill_(float("nan"))
        nm.nmspmm_half_run(A, weight, C, workspace=ws)
        assert np.array_equal(f64(C), f64(A) @ B)


EPILOGUES = [
    dict(alpha=2.0, bias=True, act="none", mul=False, residual=False),
    dict(alpha=1.0, bias=False, act="relu", mul=False, residual=True),
    dict(alpha=0.5, bias=True, act="gelu", mul=False, residual=False),
    dict(alpha=1.0, bias=False, act="silu", mul=True, residual=False),
    dict(alpha=-1.5, bias=True, act="silu", mul=True, residual=True),
]


@pytest.mark.parametrize("e", range(len(EPILOGUES)))
@pytest.mark.parametrize("shape,dtype,out", [
    ((1, 2048, 512, 4, 32, 64), "bf16", "bf16"), ((1, 24, 10, 3, 8, 2), "f16", "f32"),
    ((16, 1024, 96, 8, 32, 32), "f16", "f16"), ((37, 4096, 352, 8, 32, 32), "f16", "f16"),
    ((130, 512, 288, 12, 32, 32), "bf16", "f32"), ((520, 768, 544, 16, 32, 32), "bf16", "bf16"),
    ((300, 1024, 256, 4, 32, 64), "f16", "f32")],
    ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else x)
def test_epilogue_and_strides(shape, dtype, out, e):
    """Every part of the epilogue, with rows of every operand further apart
    than their length, A starting off a 16-byte boundary, and what lies
    between the rows untouched."""
    m, k, n, N, M, V = shape
    E = EPILOGUES[e]
    say(f"[half] epilogue {shape} {dtype} {out} {E}")
    A, weight, B = setup(*shape, dtype, a_pad=e * 3, a_off=e % 3)
    rng = np.random.default_rng(e + m)
    t = DTYPES[out]

    def matrix(pad):
        return torch.from_numpy(rng.standard_normal((m, n + pad))).to(t).cuda()[:, :n]

    bias = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).cuda() if E["bias"] else None
    mul = matrix(3) if E["mul"] else None
    residual = matrix(8) if E["residual"] else None
    whole = torch.full((m, n + 5), 7.0, dtype=t, device="cuda")
    C = whole[:, :n]
    nm.nmspmm_half_run(A, weight, C, alpha=E["alpha"], bias=bias, act=E["act"], mul=mul, residual=residual)
    torch.cuda.synchronize()
    y, tol = reference(f64(A), B, E["alpha"], None if bias is None else f64(bias), E["act"],
                       None if mul is None else f64(mul), None if residual is None else f64(residual), out)
    check(C, y, tol, f"{shape} {E}")
    assert torch.all(whole[:, n:] == 7.0)
    # in place: the residual (or the factor) is C itself
    if residual is not None or mul is not None:
        part = residual if residual is not None else mul
        kw = dict(mul=mul, residual=residual)
        kw["residual" if residual is not None else "mul"] = C
        C.copy_(part)
        nm.nmspmm_half_run(A, weight, C, alpha=E["alpha"], bias=bias, act=E["act"], **kw)
        torch.cuda.synchronize()
        check(C, y, tol, f"{shape} {E} in place")


@pytest.mark.parametrize("shape", [(1, 1024, 128, 4, 32, 64), (20, 1024, 128, 12, 32, 32), (300, 1024, 128, 3, 32, 32),
                                   (5, 60, 10, 3, 12, 5)], ids=lambda s: "x".join(map(str, s)))
def test_unkept_columns_do_not_enter(shape):
    """Infinities and NaN in columns of A that no block keeps leave the result
    alone; those that are kept reach exactly the blocks that keep them."""
    m, k, n, N, M, V = shape
    say(f"[half] infinities {shape}")
    A, weight, B = setup(*shape, "bf16")
    kept = (B != 0).any(axis=1)
    A0 = f64(A)
    dead = np.flatnonzero(~kept)
    A[:, torch.from_numpy(dead[::2]).cuda()] = float("nan")
    A[:, torch.from_numpy(dead[1::2]).cuda()] = float("inf")
    C = torch.full((m, n), float("nan"), device="cuda")
    nm.nmspmm_half_run(A, weight, C)
    torch.cuda.synchronize()
    A0[:, dead] = 0
    check(C, *reference(A0, B, 1.0, None, "none", None, None, "f32"), shape)
    live = int(np.flatnonzero(kept)[-1])
    A[m - 1, live] = float("inf")
    nm.nmspmm_half_run(A, weight, C)
    torch.cuda.synchronize()
    got = f64(C)
    touched = np.zeros((m, n), bool)
    touched[m - 1] = B[live] != 0
    assert np.all(np.isfinite(got[~touched])) and np.all(np.isinf(got[touched]))


def test_pack_from_every_type_and_clamped_offsets():
    m, k, n, N, M, V = 19, 256, 64, 8, 32, 32
    A, weight, B = setup(m, k, n, N, M, V, "f16")
    _, Bp, _ = make_inputs(m, k, n, N, M, V, seed=7 * m + k + 3 * n, dist="normal")
    Bc, idx = nm.nmspmm_compress(Bp, N, M, V)
    dBc, didx = torch.from_numpy(Bc).cuda(), torch.from_numpy(idx).cuda()
    other = nm.nmspmm_half_pack(dBc.half(), didx, n, k, N, M, V)
    assert other.dtype == torch.float16 and torch.equal(other.packed, weight.packed)
    assert nm.nmspmm_half_pack(dBc, didx, n, k, N, M, V).dtype == torch.bfloat16
    # offsets past the window are clamped: every access stays inside A
    bad = didx.clone()
    bad[3, 1] = 255
    clamped = didx.clone()
    clamped[3, 1] = M - 1
    C, D = (torch.empty(m, n, device="cuda") for _ in range(2))
    nm.nmspmm_half_run(A, nm.nmspmm_half_pack(dBc.half(), bad, n, k, N, M, V), C)
    nm.nmspmm_half_run(A, nm.nmspmm_half_pack(dBc.half(), clamped, n, k, N, M, V), D)
    torch.cuda.synchronize()
    assert torch.equal(C, D)


def test_empty_products():
    for m, k, n in ((0, 64, 32), (3, 64, 0), (3, 0, 32)):
        Bc = torch.zeros(k // 32 * 4, n, device="cuda")
        idx = torch.zeros(k // 32 * 4, n // 16, dtype=torch.uint8, device="cuda")
        weight = nm.nmspmm_half_pack(Bc, idx, n, k, 4, 32, 16)
        A = torch.ones(m, k, dtype=torch.bfloat16, device="cuda")
        C = torch.full((m, n), float("nan"), device="cuda")
        bias = torch.arange(n, device="cuda").float()
        nm.nmspmm_half_run(A, weight, C, bias=bias, act="relu")
        torch.cuda.synchronize()
        assert torch.equal(C, bias.expand(m, n))


@pytest.mark.parametrize("m", [1, 16, 40, 300])
def test_streams_graphs_and_determinism(m):
    """On a stream of its own, and replayed from a graph several times between
    eager calls: the same bits every time."""
    k, n, N, M, V = 2048, 256, 8, 32, 32
    say(f"[half] graph m={m}")
    A, weight, B = setup(m, k, n, N, M, V, "bf16")
    size = nm.nmspmm_half_workspace_bytes(m, weight)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    residual = torch.randn(m, n, device="cuda")
    first = torch.empty(m, n, device="cuda")
    nm.nmspmm_half_run(A, weight, first, residual=residual, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    C = torch.empty(m, n, device="cuda")
    torch.cuda.synchronize()
    nm.nmspmm_half_run(A, weight, C, residual=residual, stream=side)      # the library's workspace
    torch.cuda.synchronize()
    assert torch.equal(C, first)
    with torch.cuda.stream(side):
        nm.nmspmm_half_run(A, weight, C, residual=residual, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nmspmm_half_run(A, weight, C, residual=residual, workspace=ws)
    bare = torch.cuda.CUDAGraph()
    D = torch.empty(m, n, device="cuda")
    with torch.cuda.graph(bare):
        nm.nmspmm_half_run(A, weight, D, residual=residual)               # no workspace under capture
    for _ in range(4):
        C.fill_(float("nan"))
        D.fill_(float("nan"))
        graph.replay()
        bare.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, first)
        check(D, *reference(f64(A), B, 1.0, None, "none", None, f64(residual), "f32"), "graph without workspace")
        nm.nmspmm_half_run(A, weight, C, residual=residual)
        torch.cuda.synchronize()
        assert torch.equal(C, first)


def test_handle_refuses_what_is_no_packed_weight():
    size = nm.nmspmm_half_bytes(256, 64, 8, 32, 32)
    packed = torch.zeros(size, dtype=torch.uint8, device="cuda")
    assert nm.HalfWeight(packed, torch.bfloat16, 256, 64, 8, 32, 32).k == 256
    with pytest.raises(ValueError):
        nm.HalfWeight(packed[:-1], torch.bfloat16, 256, 64, 8, 32, 32)
    with pytest.raises(TypeError):
        nm.HalfWeight(packed, torch.float32, 256, 64, 8, 32, 32)
    with pytest.raises(TypeError):
        nm.HalfWeight(packed.float(), torch.bfloat16, 256, 64, 8, 32, 32)
    with pytest.raises(TypeError):
        nm.HalfWeight(packed.cpu(), torch.bfloat16, 256, 64, 8, 32, 32)
    with pytest.raises(nm.NmSpmmError):
        nm.HalfWeight(packed, torch.bfloat16, 250, 64, 8, 32, 32)
