"""Host threads that call the library at once on one stream, without a
workspace of their own: the calls share the stream's cached buffer, and each
gives the bits that it gives alone."""
import sys
import threading

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402


def pruned(m, k, n, N, M, V, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    keep = torch.rand(k // M, n // V, M, generator=gen, device="cuda").argsort(-1)[..., :N].sort(-1).values
    return (torch.randn(m, k, generator=gen, device="cuda"), torch.randn(k // M * N, n, generator=gen, device="cuda"),
            keep.permute(0, 2, 1).reshape(k // M * N, n // V).byte().contiguous())


def fp32_product(seed):
    """A transposed copy of A in the buffer, then the product from it."""
    m, n, k, N, M, V = 64, 8192, 8192, 4, 32, 64
    assert "gather" in nm.nmspmm_kernel_name_ws(m, n, k, N, M, V)
    A, Bc, idx = pruned(m, k, n, N, M, V, seed)
    return torch.empty(m, n, device="cuda"), lambda C: nm.nmspmm_run(A, Bc, idx, C, m, n, k, N, M, V)


def half_product(seed):
    """Slices of k, joined by a second kernel."""
    m, k, n, N, M, V = 40, 4096, 512, 8, 32, 32
    A, Bc, idx = pruned(m, k, n, N, M, V, seed)
    weight = nm.nmspmm_half_pack(Bc, idx, n, k, N, M, V)
    assert nm.nmspmm_half_workspace_bytes(m, weight) > 0
    A = A.bfloat16()
    return torch.empty(m, n, device="cuda"), lambda C: nm.nmspmm_half_run(A, weight, C)


def attention(seed):
    """Sequences in chunks, joined by a second kernel."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kp, vp = (torch.randn(256, 16, 2, 64, generator=gen, device="cuda").bfloat16() for _ in range(2))
    cache = nm.nmspmm_kv_cache(kp, vp, torch.arange(256, dtype=torch.int32, device="cuda").view(1, 256))
    assert nm.nmspmm_kv_attend_workspace_bytes(cache, 8, 4096) > 0
    q = torch.randn(1, 8, 64, generator=gen, device="cuda").bfloat16()
    lengths = torch.tensor([4000], dtype=torch.int32, device="cuda")
    return torch.empty_like(q), lambda out: nm.nmspmm_kv_attend(cache, q, lengths, out)


@pytest.mark.parametrize("own_stream", [False, True])
def test_calls_at_once_on_one_stream(own_stream):
    print(f"[threads] own stream {own_stream}", file=sys.stderr, flush=True)
    calls = 60
    stream = torch.cuda.Stream() if own_stream else torch.cuda.current_stream()
    work = [make(seed) for seed in (1, 2) for make in (fp32_product, half_product, attention)]
    want, outs = [], []
    with torch.cuda.stream(stream):
        for like, run in work:
            want.append(run(like).clone())
            outs.append([torch.full_like(like, float("nan")) for _ in range(calls)])
    torch.cuda.synchronize()
    start, failed = threading.Barrier(len(work)), []

    def worker(run, results):
        try:
            start.wait()
            with torch.cuda.stream(stream):
                for out in results:
                    run(out)
        except Exception as e:       # reported below, in the main thread
            failed.append(e)

    threads = [threading.Thread(target=worker, args=(run, results)) for (_, run), results in zip(work, outs)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed, failed
    for i, results in enumerate(outs):
        wrong = [j for j, out in enumerate(results) if not torch.equal(out, want[i])]
        assert not wrong, f"work {i}: {len(wrong)} of {calls} calls differ"
