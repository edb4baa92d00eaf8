"""How many bits of a weight reach the attention's sums (nmspmm_kv_attend),
against fp64 at places where lost bits show.

Tolerance of the sums, derived: queries with one 1 among zeros make every
score exact; its scaling, the exponent's product and its exponential (one step)
leave a weight of e^-t, t <= 0.5, within (2 + 2) * 2^-24 of itself; a sum of
four terms that are not zero, in parts or whole, and its joining round at most
16 times by 2^-24 of the absolute terms: together 2^-22 + 2^-20 of sum w|v|.
The store rounds once, by at most u = 2^-8 (bf16), 2^-11 (fp16, 2^-25 absolute
where subnormal) or 2^-24 (fp32) of the result.
"""
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
TYPES = [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f16", "bf16"), ("f32", "f32"), ("bf16", "f16")]


def f64(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("dim", [64, 96, 128, 200])
def test_every_bit_of_a_weight_counts(dim, dtype, cache):
    """Three positions of weight 1 whose values add up to minus the weighted
    value of a fourth, as far as the cache's type holds them: what is left is
    what the weight's last bits make of it."""
    print(f"[kv] weight's bits {dim} {dtype} {cache}", file=sys.stderr, flush=True)
    rng = np.random.default_rng(dim)
    B, heads, length, page = 16, 4, 40, 8
    per = length // page
    t = (128 + rng.permutation(128)[:B * heads].reshape(B, heads)) / 512.0      # eight bits: exact in every type
    K = np.zeros((B, length, heads, dim))
    V = torch.zeros(B, length, heads, dim, dtype=DTYPES[cache])
    for b in range(B):
        places = rng.permutation(length)[:4]
        K[b, places[3], :, 0] = -t[b]
        last = torch.from_numpy(rng.uniform(1, 2, (heads, dim))).to(DTYPES[cache])
        V[b, places[3]] = last
        left = -np.exp(-t[b])[:, None] * f64(last)
        for p in places[:3]:
            V[b, p] = torch.from_numpy(left).to(DTYPES[cache])
            left = left - f64(V[b, p])
    shape = (B * per, page, heads, dim)
    handle = nm.nmspmm_kv_cache(torch.from_numpy(K).to(DTYPES[cache]).view(shape).cuda(), V.view(shape).cuda(),
                                torch.arange(B * per, dtype=torch.int32).view(B, per).cuda())
    q = torch.zeros(B, 2 * heads, dim, dtype=DTYPES[dtype], device="cuda")
    q[..., 0] = 1.0
    out = torch.full_like(q, float("nan"))
    nm.nmspmm_kv_attend(handle, q, torch.full((B,), length, dtype=torch.int32, device="cuda"), out, scale=1.0)
    torch.cuda.synchronize()
    w = np.exp(K[..., 0])
    p = (w / w.sum(1, keepdims=True))[..., None]
    want, size = (p * f64(V)).sum(1), (p * np.abs(f64(V))).sum(1)
    tol = (2.0 ** -22 + 2.0 ** -20) * size + ROUND[dtype] * np.abs(want) + (2.0 ** -25 if dtype == "f16" else 0)
    for g in range(2):
        err = np.abs(f64(out)[:, g::2] - want)
        assert np.all(err <= tol), f"{np.sum(err > tol)} off, worst {np.max(err / tol)} of the tolerance"


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("below", [25.0, 30.0, 32.0])
def test_weights_far_below_the_largest_count(below, dtype, cache):
    """One position far above the others, whose value is zero: the others'
    weights, under 2^-36 each, make the whole result."""
    print(f"[kv] far weights {below} {dtype} {cache}", file=sys.stderr, flush=True)
    dim, length, page = 64, 2000, 8
    pages = length // page
    k, v = torch.zeros(pages, page, 1, dim), torch.full((pages, page, 1, dim), 60000.0)
    k[3, 5, 0, 0] = below
    v[3, 5] = 0.0
    v = v.to(DTYPES[cache])
    value = float(v[0, 0, 0, 0])
    handle = nm.nmspmm_kv_cache(k.to(DTYPES[cache]).cuda(), v.cuda(),
                                torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages))
    q = torch.zeros(1, 3, dim, dtype=DTYPES[dtype], device="cuda")
    q[..., 0] = 1.0
    out = torch.full_like(q, float("nan"))
    nm.nmspmm_kv_attend(handle, q, torch.tensor([length]).int().cuda(), out, scale=1.0)
    torch.cuda.synchronize()
    small = (length - 1) * np.exp(-below)
    want = value * small / (1.0 + small)
    # an exponent of up to 47 doublings, rounded twice, and the sum of equal terms
    rel = 2 * below * 2.0 ** -24 + 2.0 ** -22 + length * 2.0 ** -24
    tol = want * (rel + ROUND[dtype]) + (2.0 ** -25 if dtype == "f16" else 0)
    assert np.all(np.abs(f64(out) - want) <= tol), f"{f64(out).min()} to {f64(out).max()}, expected {want}"
