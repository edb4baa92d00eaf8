"""Memory layouts of the decoding-step operators that choose other kernels or
other loads than the usual ones: each gives the result of the plain layout,
exactly (integers for the product, the same arithmetic for the attention)."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from nm_workloads import make_inputs  # noqa: E402


def say(msg):
    print(msg, file=sys.stderr, flush=True)


def product(m, k, n, N, M, V, dtype=torch.bfloat16):
    A, Bp, _ = make_inputs(m, k, n, N, M, V, seed=m + k + n, dist="int")
    A, Bp = np.clip(A, -2, 2), np.clip(Bp, -2, 2)
    Bc, idx = nm.nmspmm_compress(Bp, N, M, V)
    weight = nm.nmspmm_half_pack(torch.from_numpy(Bc).cuda(), torch.from_numpy(idx).cuda(), n, k, N, M, V, dtype=dtype)
    want = torch.from_numpy(A.astype(np.float64) @ Bp.astype(np.float64)).float().cuda()
    return torch.from_numpy(A).to(dtype).cuda(), weight, want


@pytest.mark.parametrize("offset,stride", [(0, 2 ** 21), (0, 2 ** 21 + 8), (1, 1000), (3, 1027), (8, 1032), (4, 1028)])
@pytest.mark.parametrize("shape", [(3, 512, 96, 8, 32, 32), (20, 512, 128, 12, 32, 64), (70, 256, 48, 16, 32, 16)],
                         ids=lambda s: "x".join(map(str, s)))
def test_rows_of_a_at_any_place(shape, offset, stride):
    """Rows so far apart that no tile spans them, and rows on no 16-byte boundary."""
    say(f"[layout] {shape} offset {offset} stride {stride}")
    m, k = shape[:2]
    A, weight, want = product(*shape)
    flat = torch.zeros(offset + (m - 1) * stride + k, dtype=A.dtype, device="cuda")
    far = torch.as_strided(flat, (m, k), (stride, 1), offset)
    far.copy_(A)
    C = torch.full_like(want, float("nan"))
    nm.nmspmm_half_run(far, weight, C)
    torch.cuda.synchronize()
    assert torch.equal(C, want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", [(1, 512, 96, 8, 32, 32), (33, 512, 128, 12, 32, 64), (300, 256, 256, 16, 32, 32),
                                   (130, 256, 48, 16, 32, 16)], ids=lambda s: "x".join(map(str, s)))
def test_factor_and_term_far_apart(shape, dtype):
    """mul and residual whose rows lie 2^21 elements apart or on odd places, C
    in the middle of wider rows: (A*B) * mul + residual on integers."""
    say(f"[layout] factor {shape} {dtype}")
    m, n = shape[0], shape[2]
    A, weight, want = product(*shape, dtype=dtype)
    rng = np.random.default_rng(m)
    rows = min(m, 40)       # 40 fp32 rows 2^21 apart are 336 MB

    def values(stride, offset):
        t = torch.from_numpy(rng.integers(-3, 4, (rows, n))).to(torch.float32).cuda()
        place = torch.as_strided(torch.zeros(offset + (rows - 1) * stride + n, device="cuda"), (rows, n), (stride, 1), offset)
        place.copy_(t)
        return place

    for stride, offset in ((2 ** 21, 0), (n + 3, 1), (n + 8, 8)):
        mul, residual = values(stride, offset), values(stride, offset)
        C = torch.full((rows, n + 16), 7.0, device="cuda")
        nm.nmspmm_half_run(A[:rows], weight, C[:, 8:8 + n], mul=mul, residual=residual)
        torch.cuda.synchronize()
        assert torch.equal(C[:, 8:8 + n], want[:rows] * mul + residual)
        assert torch.all(C[:, :8] == 7.0) and torch.all(C[:, 8 + n:] == 7.0)


@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("f32", "bf16"), ("f16", "bf16"),
                                         ("f32", "f32")])
@pytest.mark.parametrize("dim", [64, 96, 128, 256])
def test_queries_at_any_place(dim, dtype, cache):
    """Queries and results in rows of odd length: bit for bit those of contiguous ones."""
    types = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
    say(f"[layout] queries dim {dim} {dtype} {cache}")
    gen = torch.Generator(device="cuda").manual_seed(dim)
    heads, group, page, B = 2, 5, 16, 3
    kp, vp = (torch.randn(40, page, heads, dim, generator=gen, device="cuda").to(types[cache]) for _ in range(2))
    table = torch.randperm(40, generator=gen, device="cuda")[:39].int().view(B, 13)
    handle = nm.nmspmm_kv_cache(kp, vp, table)
    lengths = torch.tensor([200, 1, 33]).int().cuda()
    q = torch.randn(B, heads * group, dim, generator=gen, device="cuda").to(types[dtype])
    out = torch.empty_like(q)
    nm.nmspmm_kv_attend(handle, q, lengths, out)
    wide = torch.zeros(B, heads * group + 1, dim + 3, dtype=q.dtype, device="cuda")
    odd, odd_out = wide[:, 1:, 1:dim + 1], torch.zeros_like(wide)[:, :-1, 2:dim + 2]
    odd.copy_(q)
    nm.nmspmm_kv_attend(handle, odd, lengths, odd_out)
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)      # heads first in memory
    turned_out = torch.empty_like(turned)
    nm.nmspmm_kv_attend(handle, turned, lengths, turned_out)
    torch.cuda.synchronize()
    assert torch.equal(odd_out, out) and torch.equal(turned_out, out)


@pytest.mark.parametrize("shape", [
    # m, k, n, N, M, V: k of no whole pieces of eight
    (1, 243, 64, 4, 9, 32), (1, 27, 32, 4, 9, 32), (33, 243, 64, 4, 9, 32), (130, 45, 96, 3, 5, 32),
    (3, 770, 96, 1, 77, 32), (1, 12, 32, 2, 4, 32), (16, 52, 64, 2, 4, 32), (40, 84, 48, 2, 4, 16),
    (1, 90, 48, 8, 10, 16), (2, 88, 32, 8, 8, 32), (1, 5, 16, 5, 5, 16), (70, 35, 32, 7, 7, 32), (1, 1, 32, 1, 1, 32),
    (9, 4, 32, 4, 4, 32), (17, 66, 32, 8, 22, 32)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_last_columns_of_a_beside_nothing(shape, dtype):
    """A's rows start on 16 bytes and end inside a piece of eight: the last
    columns count, and NaN between them and the next row does not."""
    say(f"[layout] ends {shape} {dtype}")
    m, k, n, N, M, V = shape
    A, weight, want = product(*shape, dtype=dtype)
    for stride in (k, (k + 7) // 8 * 8, (k + 7) // 8 * 8 + 8):
        flat = torch.full(((m - 1) * stride + k + 64,), float("nan"), dtype=dtype, device="cuda")
        rows = torch.as_strided(flat, (m, k), (stride, 1))
        rows.copy_(A)
        C = torch.full_like(want, float("nan"))
        nm.nmspmm_half_run(rows, weight, C)
        torch.cuda.synchronize()
        assert torch.equal(C, want)
