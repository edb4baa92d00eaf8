"""The appends with norms of whole prompts, where a wave takes two steps of
heads (from 8192 waves on): all types, both caches, with rotations, against
fp64.  Tolerance as in test_gpu_kv_norm.py; in 4 bits by value, to the bit."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import mx4_plain as plain  # noqa: E402
import paper_2503_01253_amd as nm  # noqa: E402
from test_gpu_kv import DTYPES, close, f64, pages_of  # noqa: E402
from test_gpu_kv_norm import norm64, setup, turn64  # noqa: E402


@pytest.mark.parametrize("norms", ["both", "q", "k"])
@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f32", "bf16"), ("f16", "f16"), ("f32", "f32"), ("bf16", "f32"),
                                         ("bf16", "4bit"), ("f16", "4bit"), ("f32", "4bit")])
@pytest.mark.parametrize("tokens,heads,group,dim,page,rot,interleaved", [
    (2101, 3, 4, 128, 16, 128, False), (2101, 3, 4, 128, 16, 64, True), (2101, 3, 4, 80, 16, 40, False),
    (2101, 5, 2, 96, 24, 96, True), (1101, 3, 4, 256, 16, 64, False), (4001, 3, 4, 64, 64, 64, False),
    (2101, 9, 1, 128, 16, 0, False)])
def test_prompt(tokens, heads, group, dim, page, rot, interleaved, dtype, cache, norms):
    print(f"[kv norm prompts] {tokens} {heads} {group} {dim} {rot} {interleaved} {dtype} {cache} {norms}", file=sys.stderr,
          flush=True)
    lanes = next(x for x in (4, 8, 16, 32, 64) if 8 * x >= dim)
    assert tokens * lanes // 64 * (2 + group) * heads >= 8192
    rng, pages, table, seq, pos, q, k, v, cos, sin, c64, s64 = setup(tokens, heads, group, dim, page, rot, interleaved,
                                                                     dtype, tokens + dim)
    weights = {x: torch.from_numpy(rng.uniform(-2, 2, dim).astype(np.float32)).cuda() if norms in ("both", x) else None
               for x in "qk"}
    w64 = {x: None if weights[x] is None else f64(weights[x]) for x in "qk"}
    eps = 1e-3
    q_out = torch.full_like(q, 5.0)
    new = dict(cos=cos, sin=sin, interleaved=interleaved, q=q, q_out=q_out, q_norm=weights["q"], k_norm=weights["k"], eps=eps)
    seq_, pos_ = torch.from_numpy(seq).int().cuda(), torch.from_numpy(pos).int().cuda()
    want_k, want_q = (turn64(norm64(f64(x), w64[y], eps), c64, s64, rot, interleaved, w64[y] is not None)
                      for x, y in ((k, "k"), (q, "q")))
    if cache == "4bit":
        pool = torch.full((pages, nm.nmspmm_kv4_page_bytes(page, heads, dim)), 255, dtype=torch.uint8, device="cuda")
        handle = nm.nmspmm_kv4_cache(pool, table, page, heads, dim)
        nm.nmspmm_kv4_append(handle, k, v, seq_, pos_, **new)
        k_out, v_out = (torch.empty(tokens, heads, dim, device="cuda") for _ in range(2))
        nm.nmspmm_kv4_read(handle, seq_, pos_, k_out, v_out)
        assert np.array_equal(f64(k_out), plain.rounded(want_k[0])) and np.array_equal(f64(v_out), plain.rounded(f64(v)))
    else:
        kp, vp = (pages_of((pages, page, heads, dim), cache, "plain", 3.0) for _ in range(2))
        nm.nmspmm_kv_append_norm(nm.nmspmm_kv_cache(kp, vp, table), k, v, seq_, pos_, **new)
        at = table.cpu().numpy()[seq, pos // page], pos % page
        for got, (want, err) in ((f64(kp), want_k), (f64(vp), (f64(v), 0.0))):
            close(got[at], want, err, cache, "written")
            got[at] = 3.0
            assert np.all(got == 3.0), "a slot that no token names was written"
    close(f64(q_out), *want_q, dtype, "queries")
