"""Attention over tables that name more positions than 2^31 - 1, with and
without a workspace, captured and not: the results of a narrow table."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("sequences", [1, 3])
def test_table_of_more_positions_than_an_int(sequences, dtype):
    print(f"[kv] wide table {sequences} {dtype}", file=sys.stderr, flush=True)
    page, heads, dim = 65536, 1, 64
    gen = torch.Generator(device="cuda").manual_seed(sequences)
    kp, vp = (torch.randn(sequences, page, heads, dim, generator=gen, device="cuda").to(dtype) for _ in range(2))
    near = torch.arange(sequences, dtype=torch.int32, device="cuda").view(sequences, 1)
    far = torch.full((sequences, 32768), -1, dtype=torch.int32, device="cuda")
    far[:, :1] = near
    lengths = torch.tensor([700, 1, 33][:sequences], dtype=torch.int32, device="cuda")
    q = torch.randn(sequences, 2, dim, generator=gen, device="cuda").to(dtype)
    want, out = torch.empty_like(q), torch.empty_like(q)
    nm.nmspmm_kv_attend(nm.nmspmm_kv_cache(kp, vp, near), q, lengths, want, max_length=700)
    handle = nm.nmspmm_kv_cache(kp, vp, far)
    tol = 2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -18      # two roundings; order of the sums
    nm.nmspmm_kv_attend(handle, q, lengths, out)
    torch.cuda.synchronize()
    assert torch.all((out - want).abs() <= tol * (want.abs() + 1))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nm.nmspmm_kv_attend(handle, q, lengths, out)        # no workspace under capture: not split
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.all((out - want).abs() <= tol * (want.abs() + 1))
        nm.nmspmm_kv_attend(handle, q, lengths, out)
        torch.cuda.synchronize()
