"""CPU tests of the sizes that the decoding-step operators plan with, at the
ends of what their ABI takes: no kernel is launched."""
import ctypes

import pytest

import paper_2503_01253_amd as nm
from paper_2503_01253_amd import serve

PTR = 1 << 20      # an address that is never used


@pytest.mark.parametrize("window", [0, 2 ** 31 - 1, 2 ** 40])
@pytest.mark.parametrize("table_pages,page_size", [
    (32767, 65536), (1, 2 ** 31 - 128), (1, 2 ** 31 - 127), (1, 2 ** 31 - 1), (32768, 65536), (2 ** 31 - 1, 1),
    (2 ** 31 - 1, 2 ** 31 - 1), (1, 2 ** 31 - 4097), (1, 2 ** 31 - 4096)])
def test_attend_that_does_not_split_needs_no_workspace(table_pages, page_size, window):
    """Enough sequences to fill the GPU without splitting any: no workspace,
    however many positions the table names (a second split without one would
    be written nowhere)."""
    strides = (ctypes.c_int64 * 3)(0, 0, 64)
    cache = ctypes.pointer(serve._Cache(PTR, PTR, strides, strides, 1, PTR, table_pages, 20000, table_pages, page_size,
                                        1, 64, nm.NMSPMM_BF16))
    size = serve._library().nmspmm_kv_attend_workspace_bytes
    for max_length in (table_pages * page_size, 2 ** 31 - 129, 2 ** 31 - 1, 2 ** 40, 2 ** 62):
        assert size(cache, 1, max_length, window) == 0, max_length


@pytest.mark.parametrize("m,k,n,N,M,V", [(1, 8192, 256, 4, 32, 64), (8, 4096, 4096, 8, 32, 32), (16, 8192, 512, 16, 32, 32),
                                         (3, 4096, 64, 8, 32, 16)])
def test_half_workspace_counts_rows_of_a_off_16_bytes(m, k, n, N, M, V):
    """Rows on 16 bytes take the kernel of few rows, which needs no workspace;
    others cut k into slices, and one size has to hold for both."""
    weight = ctypes.pointer(serve._Weight(PTR, nm.NMSPMM_BF16, N, M, V, k, n))
    L = serve._library()
    assert L.nmspmm_half_kernel_name(m, weight, 1).startswith(b"nm_half_short_kernel")
    size = L.nmspmm_half_workspace_bytes(m, weight)
    assert size >= 2 * m * n * 4 and size % (m * n * 4) == 0


@pytest.mark.parametrize("m,k,n,N,M", [(4096, 4096, 4096, 16, 32), (4096, 4096, 4096, 4, 32), (2048, 4096, 11008, 8, 32),
                                       (2500, 160, 4608, 16, 32)])
def test_half_large_tiles_gather_once_for_two_operands(m, k, n, N, M):
    """Where V is a multiple of 64 a gathered row serves two operands in the
    largest tiles, and cannot where it is not."""
    for V, ct in ((32, b",ct1,"), (64, b",ct2,"), (192, b",ct2,"), (96, b",ct1,")):
        weight = ctypes.pointer(serve._Weight(PTR, nm.NMSPMM_BF16, N, M, V, k, n // (2 * V) * 2 * V))
        name = serve._library().nmspmm_half_kernel_name(m, weight, 1)
        assert name.startswith(b"nm_half_tile_kernel<128x256,mi32") and ct in name, (V, name)


@pytest.mark.parametrize("n,V,short", [(2 ** 28 - 2 ** 20, 2 ** 20, True), (2 ** 28, 2 ** 20, False),
                                       (2 ** 30, 2 ** 28, False), (2 ** 27, 2 ** 20 + 16, False)])
def test_half_few_rows_within_a_launch(n, V, short):
    """A launch takes fewer than 2^32 threads: weights of 2^28 columns (2^27 in
    operands of 16) are not the few-row kernel's, 512 threads an operand."""
    if V % 32:
        n = (n // V + 1) * V
    weight = ctypes.pointer(serve._Weight(PTR, nm.NMSPMM_BF16, 4, 32, V, 256, n))
    assert serve._library().nmspmm_half_kernel_name(1, weight, 1).startswith(b"nm_half_short_kernel") == short


def test_sizes_that_the_header_names():
    """The first sizes that are refused, before anything is read."""
    L = serve._library()
    P2 = (ctypes.c_int64 * 2)(128, 64)
    strides = (ctypes.c_int64 * 3)(2048, 128, 64)

    def append(tokens=1, q_heads=0, positions=0):
        cache = ctypes.pointer(serve._Cache(PTR, PTR, strides, strides, 4, PTR, 4, 1, 4, 16, 2, 64, nm.NMSPMM_BF16))
        return L.nmspmm_kv_append(cache, PTR, P2, PTR, P2, nm.NMSPMM_BF16, tokens, PTR, PTR, None, None, positions, 0, 0,
                                  PTR, P2, PTR, P2, q_heads, None)

    assert append(tokens=2 ** 24) == nm.NMSPMM_ERR_UNSUPPORTED
    assert append(positions=2 ** 31) == nm.NMSPMM_ERR_UNSUPPORTED
    assert append(q_heads=(2 ** 24 - 256) // 32 - 4 + 1) == nm.NMSPMM_ERR_UNSUPPORTED
    wide = ctypes.pointer(serve._Weight(PTR, nm.NMSPMM_BF16, 4, 32, 32, 32, 2 ** 31))
    assert L.nmspmm_half_pack(PTR, nm.NMSPMM_F32, PTR, wide, None) == nm.NMSPMM_ERR_UNSUPPORTED
    assert L.nmspmm_half_run(PTR, 32, wide, PTR, 2 ** 31, nm.NMSPMM_BF16, 1, 1.0, None, 0, None, 0, None, 0, None, 0,
                             None) == nm.NMSPMM_ERR_UNSUPPORTED
