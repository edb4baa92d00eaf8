"""The 4-bit product in every form of its kernels: each case names the one that
it is there for, and runs it with rows of A in whole 16-byte pieces and not, in
both types, against fp64 and exactly on integers.

Tolerance as derived in test_gpu_mx4.py, with the number of the weight's kept
rows, w, in the place of k: products are exact in fp32, a sum of w terms in any
order errs by at most w * 2^-24 of the sum of absolute terms, alpha, bias and
residual by a rounding each, the store by half a step of C's type."""
import sys

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import paper_2503_01253_amd as nm  # noqa: E402

STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}

DENSE = [(1, 1, (3, 416, 96, 32, 32, 32)), (1, 2, (1, 160, 4112, 32, 32, 16)), (1, 2, (16, 1440, 8192, 32, 32, 32)),
         (1, 3, (1, 4096, 11008, 32, 32, 32)), (1, 3, (5, 160, 8208, 32, 32, 16)), (1, 3, (16, 1440, 8224, 32, 32, 16)),
         (1, 4, (1, 160, 12304, 32, 32, 16)), (1, 4, (2, 4096, 16448, 32, 32, 64)), (1, 4, (16, 1440, 12320, 32, 32, 32)),
         (1, 1, (5, 770, 64, 7, 7, 16)), (1, 2, (7, 770, 4128, 7, 7, 16)), (2, 4, (17, 160, 96, 32, 32, 32)),
         (2, 4, (32, 4096, 96, 32, 32, 32)), (2, 4, (31, 1440, 4112, 32, 32, 16)), (2, 4, (20, 770, 64, 7, 7, 16)),
         (4, 4, (33, 160, 96, 32, 32, 32)), (4, 4, (64, 4096, 112, 32, 32, 16)), (4, 4, (300, 1440, 160, 32, 32, 32))]
# up to 16 rows, or patterns whose windows the kernel of more rows does not hold: columns
# tiles a wave, waves side by side; whether A comes in chunks
SPARSE = [(1, 1, False, (16, 1056, 96, 16, 32, 16)), (1, 2, False, (13, 1056, 4816, 8, 32, 16)),
          (1, 4, False, (1, 512, 8224, 4, 32, 16)), (1, 4, False, (16, 1056, 16656, 16, 32, 16)),
          (2, 1, False, (7, 2048, 160, 8, 32, 32)), (2, 2, False, (13, 4096, 11008, 8, 32, 32)),
          (2, 4, False, (2, 512, 16448, 8, 32, 32)), (2, 4, False, (3, 96, 33312, 4, 32, 32)),
          (4, 1, False, (1, 4096, 512, 4, 32, 64)), (4, 2, False, (16, 2048, 24640, 4, 32, 64)),
          (4, 4, False, (4, 256, 32832, 8, 32, 64)), (4, 4, False, (16, 512, 66624, 4, 32, 64)),
          (1, 2, True, (16, 8192, 4816, 16, 32, 16)), (2, 2, True, (16, 8192, 9600, 8, 32, 32)),
          (4, 1, True, (16, 11008, 128, 16, 32, 64)), (1, 4, True, (16, 4096, 16656, 16, 32, 16)),
          (1, 4, True, (16, 60000, 16, 5, 100, 16)), (4, 4, True, (64, 65536, 64, 1, 256, 64)),
          (2, 1, False, (40, 4096, 160, 1, 128, 32))]
# of more rows: row tiles, column tiles, waves side by side, groups of a chunk of A
WIDE = [(MT, V // 16, 8 if groups == 1 else 4, groups, (m, k, 5 * V, N, 32, V))
        for MT, m, kept in ((2, 20, (1, 2, 4, 8)), (4, 50, (2, 4, 8, 16)))
        for V in (16, 32, 64) for N, groups, k in zip(kept, (1, 2, 4, 8), (2080, 2080, 2080, 6176))]
WIDE += [(2, 2, 4, 8, (32, 4096, 96, 8, 32, 32)), (4, 2, 4, 4, (300, 1056, 160, 8, 32, 32)),
         (4, 1, 4, 4, (64, 4096, 96, 12, 32, 16))]
CASES = [(f"nm_mx4_dense_kernel<mt{mt},ct{ct}>", "", s) for mt, ct, s in DENSE]
CASES += [(f"nm_mx4_sparse_kernel<mt1,ct{ct},wc{wc}>", chunks, s) for ct, wc, chunks, s in SPARSE]
CASES += [(f"nm_mx4_wide_kernel<mt{mt},ct{ct},wc{wc}>", f",chunk{chunk},", s) for mt, ct, wc, chunk, s in WIDE]


def made(gen, k, n, N, M, V, ints):
    """A packed weight and the matrix that it stands for (fp64)."""
    w = k // M * N
    keep = torch.rand(k // M, n // V, M, generator=gen, device="cuda").argsort(-1)[..., :N].sort(-1).values
    idx = keep.permute(0, 2, 1).reshape(w, n // V).byte().contiguous()
    mag = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    if ints:        # whole numbers: no halves, no scale
        codes = torch.tensor([0, 2, 4, 5, 6, 7, 10, 12, 13, 14, 15], dtype=torch.uint8, device="cuda")[
            torch.randint(0, 11, (w, n), generator=gen, device="cuda")]
        scales = torch.full(((w + 31) // 32, n), 127, dtype=torch.uint8, device="cuda")
    else:
        codes = torch.randint(0, 16, (w, n), generator=gen, device="cuda").byte()
        scales = torch.randint(115, 125, ((w + 31) // 32, n), generator=gen, device="cuda").byte()
    weight = nm.nmspmm_mx4_pack(codes, scales, idx, n, k, N, M, V)
    kept = mag[codes.long() & 7] * (1 - 2 * (codes >= 8).double())
    kept *= torch.exp2(scales.double() - 127).repeat_interleave(32, dim=0)[:w]
    at = torch.arange(w, device="cuda")[:, None] // N * M + idx.long().repeat_interleave(V, dim=1)
    return weight, torch.zeros(k, n, dtype=torch.float64, device="cuda").scatter_(0, at, kept)


def strided(x, pad, dtype):
    wide = torch.full((x.shape[0], x.shape[1] + pad), float("nan"), dtype=dtype, device="cuda")
    return wide[:, :x.shape[1]].copy_(x)


@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=str)
@pytest.mark.parametrize("name,chunks,shape", CASES, ids=lambda x: "x".join(map(str, x)) if isinstance(x, tuple) else None)
def test_instance(name, chunks, shape, dtype, pad):
    print(f"[mx4 instance] {name} {shape} {dtype} +{pad}", file=sys.stderr, flush=True)
    m, k, n, N, M, V = shape
    gen = torch.Generator(device="cuda").manual_seed(m + k + n)
    w = k // M * N
    for ints in (True, False):
        weight, B = made(gen, k, n, N, M, V, ints)
        got = nm.nmspmm_mx4_kernel_name(m, weight)
        assert got.startswith(name), got
        if isinstance(chunks, str):
            assert chunks in got, got
        else:
            assert (int(got.split("chunk")[1].split(",")[0]) < (w + 31) // 32) == chunks, got
        x = (torch.randint(-2, 3, (m, k), generator=gen, device="cuda").double() if ints
             else torch.randn(m, k, generator=gen, device="cuda"))
        A = strided(x, pad, dtype)
        # the library's workspace, and a caller's
        for workspace in (None, torch.empty(max(1, nm.nmspmm_mx4_workspace_bytes(m, weight)), dtype=torch.uint8, device="cuda")):
            if ints:
                C = torch.full((m, n), float("nan"), device="cuda")
                nm.nmspmm_mx4_run(A, weight, C, workspace=workspace)
                assert torch.equal(C.double(), A.double() @ B)
                continue
            for out in (dtype, torch.float32):
                bias = torch.randn(n, generator=gen, device="cuda")
                term = strided(torch.randn(m, n, generator=gen, device="cuda"), pad, out)
                sums, size = A.double() @ B, A.double().abs() @ B.abs()
                for form, want, tol in (
                        ({}, sums, size * (w * 2.0 ** -24)),
                        (dict(alpha=0.75, bias=bias, residual=term), 0.75 * sums + bias.double() + term.double(),
                         0.75 * size * ((w + 2) * 2.0 ** -24) + (bias.double().abs() + term.double().abs()) * 2.0 ** -23)):
                    C = strided(torch.full((m, n), 7.0, device="cuda"), pad, out)
                    nm.nmspmm_mx4_run(A, weight, C, workspace=workspace, **form)
                    bound = tol * (1 + 2.0 ** -6) + want.abs() * STEP[out] + (2.0 ** -25 if out is torch.float16 else 0)
                    assert torch.all((C.double() - want).abs() <= bound)
