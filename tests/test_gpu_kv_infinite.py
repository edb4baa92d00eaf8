"""Scores of minus infinity in the attention: they weigh nothing, and a row that
has no others is zero, its lse minus infinity, whether split or not."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


@pytest.mark.parametrize("dtype,cache", [(torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16),
                                         (torch.float32, torch.float32), (torch.bfloat16, torch.float16)])
@pytest.mark.parametrize("length", [1, 40, 3000])
def test_scores_of_minus_infinity(length, dtype, cache):
    print(f"[kv] minus infinity {length} {dtype} {cache}", file=sys.stderr, flush=True)
    dim, page = 64, 8
    pages = 375
    gen = torch.Generator(device="cuda").manual_seed(length)
    k, v = (torch.randn(pages, page, 1, dim, generator=gen, device="cuda").to(cache) for _ in range(2))
    k[..., 0] = float("-inf")
    table = torch.arange(pages, dtype=torch.int32, device="cuda").view(1, pages)
    q = torch.randn(1, 3, dim, generator=gen, device="cuda").to(dtype)
    q[..., 0] = 1.0
    out, lse = torch.full_like(q, 7.0), torch.zeros(1, 3, device="cuda")
    lengths = torch.tensor([length], dtype=torch.int32, device="cuda")
    nm.nmspmm_kv_attend(nm.nmspmm_kv_cache(k, v, table), q, lengths, out, lse=lse)
    torch.cuda.synchronize()
    assert torch.all(out == 0) and torch.all(lse == float("-inf"))
    # one finite score among them takes all
    at = length // 2
    k[at // page, at % page, 0, 0] = 1.0
    nm.nmspmm_kv_attend(nm.nmspmm_kv_cache(k, v, table), q, lengths, out, lse=lse)
    torch.cuda.synchronize()
    assert torch.equal(out, v[at // page, at % page].to(dtype).expand(1, 3, dim)) and torch.all(torch.isfinite(lse))
