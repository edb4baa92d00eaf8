"""The 4-bit product of up to 16 rows from the debug build (as in
test_gpu_mx4_poison.py), where A comes in several chunks: the next one lands in
the other slot while this one is computed, by DMA (rows in whole 16-byte pieces)
or by plain stores (rows that are not)."""
import ctypes
import os
import re
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from paper_2503_01253_amd import binding, mx4, serve  # noqa: E402
from paper_2503_01253_amd.build import POISON_LIB_PATH  # noqa: E402
from test_gpu_threads import pruned  # noqa: E402


@pytest.fixture(scope="module")
def poisoned():
    assert os.path.exists(POISON_LIB_PATH), "build() makes the debug library"
    return mx4.declare(serve.declare(binding.load(POISON_LIB_PATH)))


@pytest.mark.parametrize("pitch", [0, 1])
@pytest.mark.parametrize("m,k,n,N,M,V", [
    (16, 11008, 64, 16, 32, 32), (9, 11008, 64, 16, 32, 16), (16, 11008, 128, 16, 32, 64), (6, 131072, 32, 2, 32, 32),
    (16, 8192, 4816, 16, 32, 16), (16, 8192, 9600, 8, 32, 32), (5, 8192, 16656, 4, 32, 16),
    (16, 60000, 16, 5, 100, 16), (64, 65536, 64, 1, 256, 64)], ids=lambda x: str(x))
def test_poisoned_chunks(poisoned, m, k, n, N, M, V, pitch):
    print(f"[mx4 poison] chunks {m} {k} {n} {N}:{M} V={V} +{pitch}", file=sys.stderr, flush=True)
    _, _, idx = pruned(1, k, n, N, M, V, m + k)
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    w = k // M * N
    Bc = torch.tensor([0., 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], device="cuda")[
        torch.randint(0, 11, (w, n), generator=gen, device="cuda")]
    A = torch.randint(-2, 3, (m, k + pitch), generator=gen, device="cuda").float()[:, :k]
    codes, scales = nm.nmspmm_mx4_quantize(Bc)
    weight = nm.nmspmm_mx4_pack(codes, scales, idx, n, k, N, M, V)
    name = nm.nmspmm_mx4_kernel_name(m, weight)
    assert name.startswith("nm_mx4_sparse_kernel") and int(re.search(r"chunk(\d+)", name)[1]) < (w + 31) // 32, name
    at = torch.arange(w, device="cuda")[:, None] // N * M + idx.long().repeat_interleave(V, dim=1)
    B = torch.zeros(k, n, device="cuda").scatter_(0, at, Bc)
    want = (A.double() @ B.double()).float()
    A = torch.zeros(m, k + pitch, dtype=torch.bfloat16, device="cuda")[:, :k].copy_(A)
    for _ in range(3):
        C = torch.full((m, n), float("nan"), device="cuda")
        st = poisoned.nmspmm_mx4_run(A.data_ptr(), A.stride(0), nm.NMSPMM_BF16, weight._ref, C.data_ptr(), n,
                                     nm.NMSPMM_F32, m, 1.0, None, 0, None, 0, None, 0, None, ctypes.c_size_t(0),
                                     torch.cuda.current_stream().cuda_stream)
        assert st == nm.NMSPMM_OK
        torch.cuda.synchronize()
        assert torch.equal(C, want)
