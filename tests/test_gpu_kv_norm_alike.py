"""The append with norms where a norm is left out: keys without k_norm and
queries without q_norm are those of nmspmm_kv_append, to the bit, whatever the
other has."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402

BITS = {torch.float32: torch.int32, torch.bfloat16: torch.int16, torch.float16: torch.int16}


# whole pieces, pieces whose pairs are none, single values; the last: two steps of heads a wave
@pytest.mark.parametrize("tokens,heads,group,dim,rot,interleaved", [
    (40, 3, 2, 128, 128, False), (40, 3, 2, 128, 64, True), (40, 2, 2, 80, 40, False), (40, 2, 2, 80, 20, True),
    (40, 3, 1, 33, 32, False), (40, 3, 1, 33, 6, True), (40, 2, 2, 64, 0, False), (2100, 3, 4, 128, 128, False),
    (2100, 3, 4, 80, 40, False)])
@pytest.mark.parametrize("dtype,cache", [
    (torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.float32, torch.float16),
    (torch.bfloat16, torch.bfloat16), (torch.float16, torch.float16), (torch.bfloat16, torch.float32)], ids=str)
def test_without_weights(tokens, heads, group, dim, rot, interleaved, dtype, cache):
    print(f"[kv norm alike] {tokens} {heads} {group} {dim} {rot} {interleaved} {dtype} {cache}", file=sys.stderr, flush=True)
    gen = torch.Generator(device="cuda").manual_seed(tokens + dim + rot)
    page = 16
    pages = -(-tokens // page)
    table = torch.randperm(pages, generator=gen, device="cuda").int()[None]
    pos = torch.arange(tokens, dtype=torch.int32, device="cuda")
    seq = torch.zeros_like(pos)
    q, k, v = (torch.randn(tokens, h, dim, generator=gen, device="cuda").to(dtype) for h in (heads * group, heads, heads))
    q[::5, 0], k[::5, 0] = -0.0, -0.0
    weight = torch.rand(dim, generator=gen, device="cuda") + 0.5
    angle = torch.rand(tokens, rot // 2, generator=gen, device="cuda") * 6
    new = dict(cos=angle.cos(), sin=angle.sin(), interleaved=interleaved) if rot else {}

    def written(call, **norms):
        kp, vp = (torch.zeros(pages, page, heads, dim, dtype=cache, device="cuda") for _ in range(2))
        q_out = torch.empty_like(q)
        call(nm.nmspmm_kv_cache(kp, vp, table), k, v, seq, pos, q=q, q_out=q_out, **new, **norms)
        return [x.view(BITS[x.dtype]) for x in (kp, vp, q_out)]

    keys, values, queries = written(nm.nmspmm_kv_append)
    got = written(nm.nmspmm_kv_append_norm)
    assert torch.equal(got[0], keys) and torch.equal(got[1], values) and torch.equal(got[2], queries)
    got = written(nm.nmspmm_kv_append_norm, q_norm=weight)
    assert torch.equal(got[0], keys) and torch.equal(got[1], values) and not torch.equal(got[2], queries)
    got = written(nm.nmspmm_kv_append_norm, k_norm=weight)
    assert not torch.equal(got[0], keys) and torch.equal(got[1], values) and torch.equal(got[2], queries)
