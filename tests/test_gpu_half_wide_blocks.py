"""The largest tiles of the 16-bit product where V is a multiple of 64 and one
gathered row serves two operands: small integers, so that every result is
exact, from the product library and from the debug build that fills the places
of coming LDS writes with NaN."""
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

SHAPES = [
    # m, k, n, N, M, V: stages of one to four operands, partial last units and tiles
    (1990, 256, 4288, 4, 32, 64), (1990, 256, 4224, 8, 32, 192), (1990, 256, 4288, 12, 32, 64),
    (2500, 160, 4288, 16, 32, 64), (2500, 96, 4352, 2, 4, 128), (2500, 210, 4160, 3, 7, 64), (3000, 320, 4160, 1, 32, 64)]


def operands(shape, dtype):
    m, k, n, N, M, V = shape
    A, Bp, _ = make_inputs(m, k, n, N, M, V, seed=m + k + n, dist="int")
    A, Bp = np.clip(A, -2, 2), np.clip(Bp, -2, 2)
    Bc, idx = nm.nmspmm_compress(Bp, N, M, V)
    weight = nm.nmspmm_half_pack(torch.from_numpy(Bc).cuda(), torch.from_numpy(idx).cuda(), n, k, N, M, V, dtype=dtype)
    assert "<128x256,mi32,ct2," in nm.nmspmm_half_kernel_name(m, weight)
    return torch.from_numpy(A).to(dtype).cuda(), weight, torch.from_numpy(A @ Bp).cuda()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_product_factor_and_term(shape, dtype):
    print(f"[half wide] {shape} {dtype}", file=sys.stderr, flush=True)
    A, weight, want = operands(shape, dtype)
    C = torch.full_like(want, float("nan"))
    nm.nmspmm_half_run(A, weight, C)
    torch.cuda.synchronize()
    assert torch.equal(C, want)
    gen = torch.Generator(device="cuda").manual_seed(1)
    mul, residual = (torch.randint(-1, 2, want.shape, generator=gen, device="cuda").to(dtype) for _ in range(2))
    out = torch.full_like(want, float("nan"), dtype=dtype)
    nm.nmspmm_half_run(A, weight, out, alpha=0.25, mul=mul, residual=residual)
    torch.cuda.synchronize()
    assert torch.equal(out, (0.25 * want * mul + residual).to(dtype))


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_poisoned_slots(shape):
    print(f"[half wide poison] {shape}", file=sys.stderr, flush=True)
    assert os.path.exists(POISON_LIB_PATH), "build() makes the debug library"
    poisoned = serve.declare(binding.load(POISON_LIB_PATH))
    A, weight, want = operands(shape, torch.bfloat16)
    for _ in range(3):
        C = torch.full_like(want, float("nan"))
        st = poisoned.nmspmm_half_run(A.data_ptr(), A.stride(0), weight._ref, C.data_ptr(), C.stride(0), nm.NMSPMM_F32,
                                      A.shape[0], 1.0, None, 0, None, 0, None, 0, None, ctypes.c_size_t(0),
                                      torch.cuda.current_stream().cuda_stream)
        assert st == nm.NMSPMM_OK
        torch.cuda.synchronize()
        assert torch.equal(C, want)
