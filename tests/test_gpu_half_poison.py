"""The 16-bit product from the debug build of the library, which fills the
places of every coming LDS write with NaN: a wave that reads a slot of A before
the barrier that completes it then gives NaN.  Small integers, so that every
result is exact."""
import ctypes
import os
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from nm_workloads import make_inputs  # noqa: E402
from paper_2503_01253_amd import binding, serve  # noqa: E402
from paper_2503_01253_amd.build import POISON_LIB_PATH  # noqa: E402


@pytest.fixture(scope="module")
def poisoned():
    assert os.path.exists(POISON_LIB_PATH), "build() makes the debug library"
    return serve.declare(binding.load(POISON_LIB_PATH))


@pytest.mark.parametrize("m,k,n,N,M,V", [
    (1, 8192, 256, 4, 32, 64), (7, 4096, 64, 16, 32, 32), (16, 4096, 96, 8, 32, 16), (40, 2048, 192, 8, 32, 32),
    (64, 1024, 128, 12, 32, 32), (100, 2048, 512, 4, 32, 64), (128, 1024, 256, 16, 32, 16), (300, 2048, 512, 16, 32, 32),
    (520, 1024, 1024, 8, 32, 64), (1100, 640, 2112, 12, 32, 32), (1100, 640, 2112, 16, 32, 64)],
    ids=lambda x: str(x))
def test_poisoned_slots(poisoned, m, k, n, N, M, V):
    print(f"[half poison] {m} {k} {n} {N}:{M} V={V}", file=sys.stderr, flush=True)
    A, Bp, _ = make_inputs(m, k, n, N, M, V, seed=m + k, dist="int")
    A, Bp = np.clip(A, -2, 2), np.clip(Bp, -2, 2)
    Bc, idx = nm.nmspmm_compress(Bp, N, M, V)
    weight = nm.nmspmm_half_pack(torch.from_numpy(Bc).cuda(), torch.from_numpy(idx).cuda(), n, k, N, M, V)
    dA = torch.from_numpy(A).bfloat16().cuda()
    want = torch.from_numpy(A.astype(np.float64) @ Bp.astype(np.float64)).float().cuda()
    size = nm.nmspmm_half_workspace_bytes(m, weight)
    ws = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        C = torch.full((m, n), float("nan"), device="cuda")
        st = poisoned.nmspmm_half_run(dA.data_ptr(), k, weight._ref, C.data_ptr(), n, nm.NMSPMM_F32, m, 1.0, None, 0,
                                      None, 0, None, 0, ws.data_ptr(), ctypes.c_size_t(size),
                                      torch.cuda.current_stream().cuda_stream)
        assert st == nm.NMSPMM_OK
        torch.cuda.synchronize()
        assert torch.equal(C, want)
