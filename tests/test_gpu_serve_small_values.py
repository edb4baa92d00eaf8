"""Subnormal 16-bit values in the decoding-step operators: they are values like
others in every kernel (products and sums of powers of two, so that every
result is exact), and the attention's vector kernel at its largest tile."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


def say(msg):
    print(msg, file=sys.stderr, flush=True)


@pytest.mark.parametrize("dtype,small", [(torch.float16, 2.0 ** -20), (torch.bfloat16, 2.0 ** -130)])
@pytest.mark.parametrize("shape", [(1, 256, 64, 8, 32, 32), (16, 256, 64, 8, 32, 32), (40, 256, 64, 8, 32, 32),
                                   (300, 256, 256, 8, 32, 64), (40, 256, 48, 8, 32, 16), (9, 256, 40, 8, 32, 8)],
                         ids=lambda s: "x".join(map(str, s)))
def test_product(shape, dtype, small):
    say(f"[small] product {shape} {dtype}")
    m, k, n, N, M, V = shape
    w = k // M * N
    idx = (torch.arange(w, device="cuda") % N).byte()[:, None].repeat(1, n // V)
    gen = torch.Generator(device="cuda").manual_seed(1)
    whole = torch.randint(-2, 3, (w, n), generator=gen, device="cuda").float()
    rows = torch.randint(-2, 3, (m, k), generator=gen, device="cuda").float()
    at = torch.arange(w, device="cuda") // N * M + torch.arange(w, device="cuda") % N
    want = rows[:, at] @ whole
    # small weights times whole rows, and the other way round
    for a, b in ((1.0, small), (small, 1.0)):
        weight = nm.nmspmm_half_pack((whole * b).to(dtype), idx, n, k, N, M, V)
        A = (rows * a).to(dtype)
        assert torch.equal(A.double(), rows.double() * a)
        C = torch.full((m, n), float("nan"), device="cuda")
        nm.nmspmm_half_run(A, weight, C, alpha=2.0 ** 20)
        torch.cuda.synchronize()
        assert torch.equal(C.double(), want.double() * small * 2.0 ** 20)


@pytest.mark.parametrize("dtype,cache,small", [
    (torch.float16, torch.float16, 2.0 ** -20), (torch.float32, torch.float16, 2.0 ** -20),
    (torch.bfloat16, torch.bfloat16, 2.0 ** -130), (torch.float32, torch.bfloat16, 2.0 ** -130)])
@pytest.mark.parametrize("dim", [64, 33])
def test_attend(dim, dtype, cache, small):
    say(f"[small] attend {dim} {dtype} {cache}")
    if dtype == torch.float16:
        dim *= 2
    k = torch.zeros(2, 16, 1, dim, dtype=cache, device="cuda")
    v = torch.full((2, 16, 1, dim), small, dtype=cache, device="cuda")
    v[0, 3], v[1, 2] = 5 * small, -3 * small
    q = torch.ones(1, 3, dim, dtype=dtype, device="cuda")
    out = torch.full_like(q, float("nan"))
    table = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda")
    nm.nmspmm_kv_attend(nm.nmspmm_kv_cache(k, v, table), q, torch.tensor([32], dtype=torch.int32, device="cuda"), out)
    torch.cuda.synchronize()
    assert torch.equal(out.double(), torch.full_like(out, small).double())      # (30 + 5 - 3) / 32
    # small keys: scores of 2^-20 and less, told apart by a scale
    if small == 2.0 ** -20:
        k[0, 3, 0, 0], v[0, 3] = small, 1.0
        nm.nmspmm_kv_attend(nm.nmspmm_kv_cache(k, v, table), q, torch.tensor([32], dtype=torch.int32, device="cuda"), out,
                            scale=50.0 / small)
        torch.cuda.synchronize()
        assert torch.equal(out, torch.ones_like(out))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dim,group", [(300, 8), (511, 7), (512, 16), (33, 9)])
def test_rows_off_16_bytes_with_many_heads(dim, group, dtype):
    """Eight heads a workgroup on the vector kernel, up to its longest rows:
    the results of one head a workgroup."""
    say(f"[small] many heads {dim} {group} {dtype}")
    gen = torch.Generator(device="cuda").manual_seed(dim)
    kp, vp = (torch.randn(30, 8, 1, dim + 1, generator=gen, device="cuda").to(dtype)[..., 1:] for _ in range(2))
    table = torch.randperm(30, generator=gen, device="cuda").int().view(2, 15)
    cache = nm.nmspmm_kv_cache(kp, vp, table)
    lengths = torch.tensor([117, 40], dtype=torch.int32, device="cuda")
    q = torch.randn(2, group, dim, generator=gen, device="cuda").to(dtype)
    out = torch.full_like(q, float("nan"))
    nm.nmspmm_kv_attend(cache, q, lengths, out)
    for h in range(group):
        one = torch.full((2, 1, dim), float("nan"), dtype=dtype, device="cuda")
        nm.nmspmm_kv_attend(cache, q[:, h:h + 1], lengths, one)
        torch.cuda.synchronize()
        assert torch.equal(out[:, h:h + 1], one)
