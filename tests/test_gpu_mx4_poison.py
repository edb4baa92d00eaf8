"""The 4-bit product from the debug build of the library, which fills the
places of every coming LDS write of A with NaN: a wave that reads a slot before
the barrier that completes it then gives NaN.  Small integers that 4 bits hold
(0, 1, 2, 3, 4, 6 and their negatives), so that every result is exact."""
import ctypes
import os
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


@pytest.mark.parametrize("pitch", [0, 1])      # rows of A in whole 16-byte pieces, and not
@pytest.mark.parametrize("m,k,n,N,M,V", [
    (1, 8192, 256, 4, 32, 64), (7, 4096, 64, 16, 32, 32), (16, 4096, 96, 8, 32, 16), (13, 2080, 160, 12, 32, 32),
    (3, 1000, 64, 3, 8, 16), (17, 1024, 128, 12, 32, 32), (40, 2048, 192, 8, 32, 32), (64, 8192, 128, 16, 32, 32),
    (100, 2048, 512, 4, 32, 64), (33, 1504, 96, 8, 32, 16), (60, 2048, 64, 32, 32, 32)], ids=lambda x: str(x))
def test_poisoned_slots(poisoned, m, k, n, N, M, V, pitch):
    print(f"[mx4 poison] {m} {k} {n} {N}:{M} V={V} +{pitch}", file=sys.stderr, flush=True)
    _, _, idx = pruned(1, k, n, N, M, V, m + k)
    gen = torch.Generator(device="cuda").manual_seed(m + n)
    w = k // M * N
    Bc = torch.tensor([0., 1, 2, 3, 4, 6, -1, -2, -3, -4, -6], device="cuda")[
        torch.randint(0, 11, (w, n), generator=gen, device="cuda")]
    A = torch.randint(-2, 3, (m, k + pitch), generator=gen, device="cuda").float()[:, :k]
    codes, scales = nm.nmspmm_mx4_quantize(Bc)
    weight = nm.nmspmm_mx4_pack(codes, scales, idx, n, k, N, M, V)
    at = torch.arange(w, device="cuda")[:, None] // N * M + idx.long().repeat_interleave(V, dim=1)
    B = torch.zeros(k, n, device="cuda").scatter_(0, at, Bc)
    want = (A.double() @ B.double()).float()
    A = torch.zeros(m, k + pitch, dtype=torch.bfloat16, device="cuda")[:, :k].copy_(A)
    size = nm.nmspmm_mx4_workspace_bytes(m, weight)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        C = torch.full((m, n), float("nan"), device="cuda")
        st = poisoned.nmspmm_mx4_run(A.data_ptr(), A.stride(0), nm.NMSPMM_BF16, weight._ref, C.data_ptr(), n,
                                     nm.NMSPMM_F32, m, 1.0, None, 0, None, 0, None, 0, ws.data_ptr(),
                                     ctypes.c_size_t(size), torch.cuda.current_stream().cuda_stream)
        assert st == nm.NMSPMM_OK
        torch.cuda.synchronize()
        assert torch.equal(C, want)
