"""The appends with norms, head by head: the bits of a head do not depend on
what lies in the other heads of its token."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


@pytest.mark.parametrize("four", [False, True])
@pytest.mark.parametrize("power", [-140, -125, 126])
@pytest.mark.parametrize("tokens,dim,rot,interleaved", [(40, 128, 128, False), (40, 128, 64, True), (40, 80, 40, False),
                                                        (40, 33, 6, True), (2100, 128, 128, False)])
def test_a_head_is_its_own(tokens, dim, rot, interleaved, power, four):
    print(f"[kv norm heads] {tokens} {dim} {rot} {interleaved} 2^{power} {four}", file=sys.stderr, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(tokens + dim + rot)
    page, heads, group = 16, 3, 4
    pages = -(-tokens // page)
    table = torch.randperm(pages, generator=gen, device="cuda").int()[None]
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    seq = torch.zeros_like(pos)
    q, k, v = (torch.randn(tokens, h, dim, generator=gen, device="cuda") for h in (heads * group, heads, heads))
    weight = torch.rand(dim, generator=gen, device="cuda") + 0.5
    angle = torch.rand(tokens, rot // 2, generator=gen, device="cuda") * 6

    def written(q, k):
        q_out, k_out = torch.empty_like(q), torch.empty_like(k)
        new = dict(cos=angle.cos(), sin=angle.sin(), q=q, q_out=q_out, interleaved=interleaved, q_norm=weight,
                   k_norm=weight, eps=0.0)
        if four:
            pool = torch.zeros(pages, nm.nmspmm_kv4_page_bytes(page, heads, dim), dtype=torch.uint8, device="cuda")
            cache = nm.nmspmm_kv4_cache(pool, table, page, heads, dim)
            nm.nmspmm_kv4_append(cache, k, v, seq, pos, **new)
            nm.nmspmm_kv4_read(cache, seq, pos, k_out)
            return q_out, k_out
        kp, vp = (torch.zeros(pages, page, heads, dim, device="cuda") for _ in range(2))
        nm.nmspmm_kv_append_norm(nm.nmspmm_kv_cache(kp, vp, table), k, v, seq, pos, **new)
        return q_out, kp[table[0].long()].view(-1, heads, dim)[:tokens]

    alone = written(q, k)
    # every third head, another one from token to token, tiny or huge
    far = [(torch.arange(x.shape[1], device="cuda")[None] + pos[:, None]) % 3 == 0 for x in (q, k)]
    beside = written(*(torch.where(f[..., None], torch.ldexp(x.double(), torch.tensor(power, device="cuda")).float(), x)
                       for x, f in zip((q, k), far)))
    for a, b, f in zip(alone, beside, far):
        assert torch.equal(a[~f], b[~f])
