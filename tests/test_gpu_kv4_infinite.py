"""Infinite queries over the 4-bit cache, of every type: scores of minus
infinity weigh nothing, a row that has no others is zero and its lse minus
infinity, and a score of plus infinity makes its head NaN, no other."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=str)
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 8), (96, 4), (256, 16), (64, 5)])
@pytest.mark.parametrize("length", [1, 40, 3000])
def test_infinite_queries(length, dim, page, dtype):
    print(f"[kv4] infinite queries {length} {dim} {page} {dtype}", file=sys.stderr, flush=True)
    pages = 3000 // page + 1
    pool = torch.full((pages, nm.nmspmm_kv4_page_bytes(page, 1, dim)), 255, dtype=torch.uint8, device="cuda")
    cache = nm.nmspmm_kv4_cache(pool, torch.arange(pages, dtype=torch.int32, device="cuda")[None], page, 1, dim)
    gen = torch.Generator(device="cuda").manual_seed(length)
    k, v = (torch.randn(length, 1, dim, generator=gen, device="cuda") for _ in range(2))
    k[..., 3] = 3.0         # (not rounded to zero)
    at = torch.zeros(length, dtype=torch.int32, device="cuda"), torch.arange(length, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv4_append(cache, k, v, *at)
    q = torch.randn(1, 4, dim, generator=gen, device="cuda").to(dtype)
    q[0, 0, 3], q[0, 1, 3], q[0, 3, 3] = float("-inf"), float("inf"), float("nan")
    lengths = torch.tensor([length], dtype=torch.int32, device="cuda")
    out, lse = torch.full_like(q, 7.0), torch.zeros(1, 4, device="cuda")
    nm.nmspmm_kv4_attend(cache, q, lengths, out, lse=lse)
    torch.cuda.synchronize()
    assert torch.all(out[0, 0] == 0) and lse[0, 0] == float("-inf")
    assert torch.isnan(out[0, 1]).all() and torch.isnan(out[0, 3]).all()
    assert torch.isfinite(out[0, 2]).all() and torch.isfinite(lse[0, 2])
    # one finite score among them takes all: a key of zero there would be NaN, a group
    # of its own magnitude is not
    x = length // 2
    k[x] = -k[x]
    nm.nmspmm_kv4_append(cache, k, v, *at)
    v_out = torch.empty_like(v)
    nm.nmspmm_kv4_read(cache, *at, None, v_out)
    q[0, 0, 3] = float("inf")       # the one at x minus infinity now, the others plus
    nm.nmspmm_kv4_attend(cache, q, lengths, out, lse=lse)
    torch.cuda.synchronize()
    if length == 1:
        assert torch.all(out[0, 0] == 0) and lse[0, 0] == float("-inf")
    else:
        assert torch.isnan(out[0, 0]).all()
    assert torch.isfinite(out[0, 2]).all()
