"""The 4-bit product with the two largest scales, which no rounding gives: the
values that fp32 holds are exact."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import mx4_plain as plain  # noqa: E402
import paper_2503_01253_amd as nm  # noqa: E402
from test_gpu_mx4 import dense, pattern  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("m,k,n,N,M,V", [(5, 96, 32, 32, 32, 32), (5, 192, 32, 16, 32, 32), (20, 192, 32, 16, 32, 32),
                                         (5, 96, 24, 16, 32, 8)], ids=lambda x: str(x))
def test_largest_scales(m, k, n, N, M, V, dtype):
    print(f"[mx4 scales] {m} {k} {n} {N}:{M} V={V} {dtype}", file=sys.stderr, flush=True)
    rng = np.random.default_rng(m + k)
    w = k // M * N
    for s in (253, 254):
        least = 2.0 ** (255 - s)
        codes = rng.choice([c for c in range(16) if plain.MAGNITUDES[c & 7] < least], (w, n)).astype(np.uint8)
        codes[32:] = 0      # (one group: its terms are whole multiples of one power of two)
        byte = np.full(((w + 31) // 32, n), s, dtype=np.uint8)
        idx = pattern(rng, k, n, N, M, V)
        weight = nm.nmspmm_mx4_pack(*(torch.from_numpy(x).cuda() for x in (codes, byte, idx)), n, k, N, M, V)
        B = dense(plain.values_of(codes.astype(np.int64), np.full((w, n), s)), idx, k, n, N, M, V)
        A = torch.from_numpy(rng.integers(-2, 3, (m, k)) * 2.0 ** (-100 if dtype is torch.bfloat16 else -14)).to(dtype).cuda()
        C = torch.empty(m, n, device="cuda")
        nm.nmspmm_mx4_run(A, weight, C)
        assert np.array_equal(C.double().cpu().numpy(), A.double().cpu().numpy() @ B)
