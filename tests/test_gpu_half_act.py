"""The activations of the 16-bit product's epilogue, against fp64, relative to
their own values: the product is zero and the bias is the argument, so that
fp32 results show every digit.

Tolerances, derived.  GELU y * Phi(y), Phi(y) = erfc(-y / sqrt 2) / 2: the
argument of erfc is rounded twice (the factor and the product), by 2^-23 of
itself together, and erfc's logarithm changes by at most 2x^2 + 2 times that
for an x = |y| / sqrt 2, that is by (y^2 + 2) * 2^-23; erfc itself is off by at
most 16 * 2^-24 of its value (OpenCL's bound, which the device library keeps,
is 16 units of 2^-23), so 16 * 2^-23, and three products by 3 * 2^-24.
SiLU y / (1 + e^-y): an exponential (at most 2 * 2^-23), a sum, a quotient and
a product, 8 * 2^-24 together at most.  16-bit results are rounded once more.
Values below fp32's smallest normal number, 2^-126, may be taken as zero."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
ROUND = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}


def results(y, act, m, vector, out="f32", mul=None):
    """act(y) for every y, from each of the kernels' epilogues: one row or
    several, rows on 16 bytes or not, one run over k or slices of it."""
    n = y.size
    assert n % 64 == 0
    k = 256
    dtype = DTYPES["bf16" if out == "f32" else out]
    Bc = torch.zeros(k // 4, n, dtype=dtype, device="cuda")
    idx = (torch.arange(k // 4, device="cuda") % 8).byte()[:, None].repeat(1, n // 32)
    weight = nm.nmspmm_half_pack(Bc, idx, n, k, 8, 32, 32)
    A = torch.ones(m, k, dtype=dtype, device="cuda")
    C = torch.full((m, n + (8 if vector else 3)), float("nan"), dtype=DTYPES[out], device="cuda")[:, :n]
    bias = torch.from_numpy(y).cuda()
    factor = None if mul is None else torch.full_like(C, mul)
    nm.nmspmm_half_run(A, weight, C, bias=bias, act=act, mul=factor)
    torch.cuda.synchronize()
    got = C.double().cpu().numpy()
    assert np.array_equal(got, np.broadcast_to(got[0], got.shape), equal_nan=True)
    return got[0]


def values(lo, hi):
    rng = np.random.default_rng(1)
    return np.concatenate([rng.uniform(lo, hi, 1000), np.linspace(lo, hi, 24)]).astype(np.float32)


@pytest.mark.parametrize("vector", [False, True])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_gelu(m, vector):
    from scipy.special import erfc
    print(f"[half act] gelu {m} {vector}", file=sys.stderr, flush=True)
    for lo, hi in ((-12.5, -8), (-8, -3), (-3, 3), (3, 20)):
        y = values(lo, hi)
        want = 0.5 * y.astype(np.float64) * erfc(-y.astype(np.float64) / np.sqrt(2.0))
        tol = np.abs(want) * ((y.astype(np.float64) ** 2 + 2) * 2.0 ** -23 + 16 * 2.0 ** -23 + 3 * 2.0 ** -24) + 2.0 ** -126
        err = np.abs(results(y, "gelu", m, vector) - want)
        assert np.all(err <= tol), f"{lo} to {hi}: worst {np.max(err / tol)} of the tolerance at {y[np.argmax(err / tol)]}"


@pytest.mark.parametrize("out", ["bf16", "f16"])
def test_gelu_times_a_large_factor(out):
    """A factor brings the tail back into the range of 16-bit types."""
    from scipy.special import erfc
    y = values(-8, -5)
    want = 0.5 * y.astype(np.float64) * erfc(-y.astype(np.float64) / np.sqrt(2.0)) * 32768.0
    tol = np.abs(want) * (ROUND[out] + 2.0 ** -16) + (2.0 ** -25 if out == "f16" else 0)
    err = np.abs(results(y, "gelu", 40, True, out, 32768.0) - want)
    assert np.all(err <= tol), f"worst {np.max(err / tol)} of the tolerance"


@pytest.mark.parametrize("vector", [False, True])
@pytest.mark.parametrize("m", [1, 40, 300])
def test_silu(m, vector):
    print(f"[half act] silu {m} {vector}", file=sys.stderr, flush=True)
    for lo, hi in ((-86, -30), (-30, -3), (-3, 3), (3, 100)):
        y = values(lo, hi)
        y64 = y.astype(np.float64)
        want = y64 * np.where(y64 < 0, np.exp(y64), 1) / (1 + np.exp(-np.abs(y64)))
        tol = np.abs(want) * 8 * 2.0 ** -24 + 2.0 ** -126
        err = np.abs(results(y, "silu", m, vector) - want)
        assert np.all(err <= tol), f"{lo} to {hi}: worst {np.max(err / tol)} of the tolerance at {y[np.argmax(err / tol)]}"


@pytest.mark.parametrize("vector", [False, True])
@pytest.mark.parametrize("m", [1, 40])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
def test_infinities_and_nan(act, m, vector):
    """Plus infinity stays, NaN stays, and what is finite beside them does."""
    y = np.ones(64, np.float32)
    y[3], y[10], y[20], y[21] = np.inf, np.nan, 3e38, -3e38
    got = results(y, act, m, vector)
    assert got[3] == np.inf and np.isnan(got[10]) and np.isfinite(np.delete(got, [3, 10])).all()
    assert got[20] == np.float64(y[20]) and got[21] == (np.float64(y[21]) if act == "none" else 0)
