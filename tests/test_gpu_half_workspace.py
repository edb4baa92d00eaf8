"""The 16-bit product with a caller's workspace where A's rows start off 16
bytes: captured into a graph, where the library takes no buffer of its own, it
gives the bits of the eager call, so the workspace of the size that the query
names was enough.  (Slices of k add up in another order than one run over k.)"""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402
from nm_workloads import make_inputs  # noqa: E402


@pytest.mark.parametrize("offset,stride", [(0, 0), (1, 0), (8, 4), (4, 8)])
@pytest.mark.parametrize("shape", [
    # m, k, n, N, M, V
    (1, 8192, 256, 4, 32, 64), (8, 4096, 4096, 8, 32, 32), (16, 8192, 512, 16, 32, 32), (3, 4096, 64, 8, 32, 16),
    (40, 4096, 352, 8, 32, 32), (200, 2048, 256, 12, 32, 64), (100, 4096, 48, 4, 32, 16)],
    ids=lambda s: "x".join(map(str, s)))
def test_caller_workspace_serves_rows_at_any_place(shape, offset, stride):
    print(f"[half workspace] {shape} offset {offset} stride + {stride}", file=sys.stderr, flush=True)
    m, k, n, N, M, V = shape
    A, Bp, _ = make_inputs(m, k, n, N, M, V, seed=m + k, dist="normal")
    Bc, idx = nm.nmspmm_compress(Bp, N, M, V)
    weight = nm.nmspmm_half_pack(torch.from_numpy(Bc).cuda(), torch.from_numpy(idx).cuda(), n, k, N, M, V)
    rows = torch.zeros(offset + m * (k + stride), dtype=torch.bfloat16, device="cuda").as_strided(
        (m, k), (k + stride, 1), offset)
    rows.copy_(torch.from_numpy(A))
    size = nm.nmspmm_half_workspace_bytes(m, weight)
    ws = torch.full((max(size, 1),), 255, dtype=torch.uint8, device="cuda")
    first, C = (torch.full((m, n), float("nan"), device="cuda") for _ in range(2))
    nm.nmspmm_half_run(rows, weight, first)                             # the library's buffer
    torch.cuda.synchronize()
    want = rows.double().cpu().numpy() @ torch.from_numpy(Bp).bfloat16().double().numpy()
    assert np.allclose(first.double().cpu().numpy(), want, rtol=0, atol=k * 2.0 ** -24 * np.abs(want).max() * 8)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nmspmm_half_run(rows, weight, C, workspace=ws)
    for _ in range(3):
        C.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(C, first)
        nm.nmspmm_half_run(rows, weight, C, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(C, first)
