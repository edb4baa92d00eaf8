"""More new tokens than one launch takes, queries in place: every token is
normalised once.  Tolerance as in test_gpu_kv_norm.py: 3.1 u of the value in
fp32, then a rounding to bf16 (2^-8 of it); the norms of fp64 here."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


# (25 waves a token, of which a launch takes 2^25: the last workgroup of the first would
# have waves left for the queries of the next token)
@pytest.mark.parametrize("tokens,q_heads,dim", [((1 << 24) - 1, 1, 8), ((1 << 23) - 5, 33, 8),
                                                ((1 << 25) // 25 + 1000, 360, 1)])
def test_many_tokens(tokens, q_heads, dim):
    page = 4096
    print(f"[kv norm sizes] {tokens} tokens, {q_heads} query heads of {dim}", file=sys.stderr, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(1)
    pages = (tokens + page - 1) // page
    kp, vp = (torch.zeros(pages, page, 1, dim, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = torch.randperm(pages, generator=gen, device="cuda").int()[None]
    cache = nm.nmspmm_kv_cache(kp, vp, table)
    k, v = (torch.randn(tokens, 1, dim, generator=gen, device="cuda").bfloat16() for _ in range(2))
    q = torch.randn(tokens, q_heads, dim, generator=gen, device="cuda").bfloat16()
    weight = torch.full((dim,), 2.0, device="cuda")
    before = q.clone()
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    nm.nmspmm_kv_append_norm(cache, k, v, torch.zeros_like(pos), pos, q=q, q_norm=weight, k_norm=weight, eps=1.0)

    def far(got, x):
        """The largest error over the tolerance."""
        worst = 0.0
        for g, y in zip(got.split(1 << 20), x.split(1 << 20)):
            y = y.double()
            want = 2 * y / y.square().mean(-1, keepdim=True).add(1.0).sqrt()
            err = (g.double() - want).abs() / (want.abs() * (2.0 ** -8 + 3.2 * 2.0 ** -24) + 1e-30)
            worst = max(worst, err.max().item())
        return worst

    assert far(q, before) <= 1
    assert far(kp[table[0].long()].view(-1, 1, dim)[:tokens], k) <= 1
    assert torch.equal(vp[table[0].long()].view(-1, 1, dim)[:tokens], v)
