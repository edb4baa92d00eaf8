"""Memory that the binding of the decoding-step operators allocates for a call
on a stream of its own."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


def test_pack_takes_no_block_of_another_stream():
    """A block that the current stream has freed may still be written by work
    queued there: a pack on another stream must not get it."""
    k, n, N, M, V = 2048, 2048, 8, 32, 32
    gen = torch.Generator(device="cuda").manual_seed(1)
    Bc = torch.randn(k // M * N, n, generator=gen, device="cuda")
    idx = torch.sort(torch.rand(k // M, n // V, M, generator=gen, device="cuda").argsort(-1)[..., :N], -1).values
    idx = idx.permute(0, 2, 1).reshape(k // M * N, n // V).byte().contiguous()
    want = nm.nmspmm_half_pack(Bc, idx, n, k, N, M, V)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        held = [torch.empty_like(want.packed) for _ in range(4)]
        places = {t.data_ptr() for t in held}
        del held                       # freed on the current stream, nothing queued on them
        torch.cuda.synchronize()
        weight = nm.nmspmm_half_pack(Bc, idx, n, k, N, M, V, stream=side)
        assert weight.packed.data_ptr() not in places
        torch.cuda.synchronize()
        assert torch.equal(weight.packed, want.packed)
    # on the current stream, named or not, as ever
    for stream in (None, torch.cuda.current_stream()):
        assert torch.equal(nm.nmspmm_half_pack(Bc, idx, n, k, N, M, V, stream=stream).packed, want.packed)
