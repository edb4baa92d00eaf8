"""CPU tests of the 4-bit operators' C ABI (include/nmspmm_mx4.h) and of the
append with norms: every declared symbol is exported, sizes are right, and bad
arguments are refused before anything reaches the GPU."""
import ctypes
import os
import re

import pytest

import paper_2503_01253_amd as nm
from paper_2503_01253_amd import mx4, serve
from test_serve_abi import PAIR, PTR
from test_serve_abi import cache as cache16

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED = nm.NMSPMM_OK, nm.NMSPMM_ERR_INVALID_ARG, nm.NMSPMM_ERR_UNSUPPORTED
BF16, F16, F32 = nm.NMSPMM_BF16, nm.NMSPMM_F16, nm.NMSPMM_F32


def test_library_exports_every_declared_symbol():
    text = open(os.path.join(ROOT, "include", "nmspmm_mx4.h")).read()
    names = sorted(set(re.findall(r"NMSPMM_API\s+[\w\s\*]*?\b(nmspmm_\w+)\s*\(", text)))
    assert names == sorted(nm.MX4_EXPORTS)
    L = mx4._library()
    for name in names:
        assert ctypes.cast(getattr(L, name), ctypes.c_void_p).value, name
        assert getattr(L, name).argtypes is not None, name
        assert getattr(nm, name) is not None


# ---- the product -----------------------------------------------------------

def weight(packed=PTR, k=64, n=64, N=4, M=32, V=32):
    return ctypes.pointer(mx4._Weight(packed, N, M, V, k, n))


def run(w=None, A=PTR, lda=64, a_dtype=BF16, C=PTR, ldc=64, c_dtype=BF16, m=8, bias=None, act=0, mul=None, ld_mul=64,
        residual=None, ld_residual=64, ws=None, ws_bytes=0):
    return mx4._library().nmspmm_mx4_run(A, lda, a_dtype, w or weight(), C, ldc, c_dtype, m, 1.0, bias, act, mul, ld_mul,
                                         residual, ld_residual, ws, ws_bytes, None)


def test_run_refusals():
    for bad in (dict(k=65), dict(n=65), dict(N=0), dict(N=33), dict(M=257, N=1, k=257), dict(V=0), dict(k=-32)):
        assert run(weight(**bad)) == INVALID, bad
    for bad in (dict(m=-1), dict(A=None), dict(C=None), dict(w=weight(packed=None)), dict(act=4), dict(act=-1),
                dict(c_dtype=F16), dict(c_dtype=7), dict(a_dtype=F32), dict(a_dtype=9), dict(lda=63), dict(ldc=63),
                dict(mul=PTR, ld_mul=63), dict(residual=PTR, ld_residual=63)):
        assert run(**bad) == INVALID, bad
    for bad in (dict(A=PTR + 1), dict(C=PTR + 1), dict(C=PTR + 2, c_dtype=F32), dict(bias=PTR + 2), dict(mul=PTR + 1),
                dict(residual=PTR + 1), dict(w=weight(packed=PTR + 128)), dict(ws=PTR + 16), dict(m=1 << 62),
                dict(lda=1 << 62), dict(w=weight(n=1 << 31))):
        assert run(**bad) == UNSUPPORTED, bad
    assert run(m=0, A=None, C=None) == OK
    assert run(weight(n=0), C=None) == OK
    assert mx4._library().nmspmm_mx4_run(PTR, 64, BF16, None, PTR, 64, 1, 8, 1.0, None, 0, None, 0, None, 0, None, 0,
                                         None) == INVALID


def test_pack_and_quantize_refusals():
    pack = mx4._library().nmspmm_mx4_pack
    assert pack(None, PTR, PTR, weight(), None) == INVALID
    assert pack(PTR, None, PTR, weight(), None) == INVALID
    assert pack(PTR, PTR, None, weight(), None) == INVALID
    assert pack(PTR, PTR, PTR, weight(packed=None), None) == INVALID
    assert pack(PTR, PTR, PTR, weight(k=63), None) == INVALID
    assert pack(PTR, PTR, PTR, None, None) == INVALID
    assert pack(PTR, PTR, PTR, weight(packed=PTR + 64), None) == UNSUPPORTED
    assert pack(None, None, None, weight(k=0), None) == OK
    quantize = mx4._library().nmspmm_mx4_quantize
    assert quantize(PTR, 3, 32, 32, PTR, PTR, None) == INVALID
    assert quantize(PTR, F32, -1, 32, PTR, PTR, None) == INVALID
    for bad in ((None, PTR, PTR), (PTR, None, PTR), (PTR, PTR, None)):
        assert quantize(bad[0], F32, 32, 32, bad[1], bad[2], None) == INVALID
    assert quantize(PTR + 2, F32, 32, 32, PTR, PTR, None) == UNSUPPORTED
    assert quantize(PTR + 1, BF16, 32, 32, PTR, PTR, None) == UNSUPPORTED
    assert quantize(PTR, F32, 1 << 31, 32, PTR, PTR, None) == UNSUPPORTED
    assert quantize(None, F32, 0, 32, None, None, None) == OK
    assert quantize(None, F32, 32, 0, None, None, None) == OK


def test_weight_sizes():
    for k, n, N, M, V in ((64, 64, 4, 32, 32), (4096, 11008, 8, 32, 32), (4096, 11008, 32, 32, 32), (24, 10, 3, 8, 2),
                          (100, 48, 7, 10, 16)):
        w = k // M * N
        size = nm.nmspmm_mx4_bytes(k, n, N, M, V)
        assert size >= (w * n + 1) // 2 + -(-w // 32) * n
        if w % 128 == 0:        # no padding to speak of: half a byte, the scale, two bytes an offset
            assert size <= w * n // 2 + w // 32 * n + 2 * w * (n // V) + 1024
    assert nm.nmspmm_mx4_bytes(65, 64, 4, 32, 32) == -1
    assert nm.nmspmm_mx4_bytes(0, 64, 4, 32, 32) == 0
    L = mx4._library()
    assert L.nmspmm_mx4_workspace_bytes(-1, weight()) == -1
    assert L.nmspmm_mx4_workspace_bytes(0, weight()) == 0
    assert L.nmspmm_mx4_kernel_name(-1, weight(), 1) == b"invalid"
    assert L.nmspmm_mx4_kernel_name(0, weight(), 1) == b"none"


# ---- the appends -----------------------------------------------------------

def cache4(pages=PTR, page_stride=None, page_count=10, table=PTR, sequences=3, table_pages=4, page_size=16, heads=2,
           dim=64):
    if page_stride is None:
        page_stride = max(nm.nmspmm_kv4_page_bytes(page_size, heads, dim), 0)
    return ctypes.pointer(mx4._Cache(pages, page_stride, page_count, table, table_pages, sequences, table_pages, page_size,
                                     heads, dim))


def append(fn, c, k=PTR, ks=PAIR, v=PTR, vs=PAIR, dtype=BF16, tokens=4, seq=PTR, pos=PTR, cos=PTR, sin=PTR,
           positions=64, rot=64, q_norm=PTR, k_norm=PTR, eps=1e-6, q=PTR, qs=PAIR, q_out=PTR, qos=PAIR, q_heads=4):
    return fn(c, k, ks, v, vs, dtype, tokens, seq, pos, cos, sin, positions, rot, 0, q_norm, k_norm, eps, q, qs, q_out,
              qos, q_heads, None)


@pytest.mark.parametrize("four", [False, True])
def test_append_refusals(four):
    fn = mx4._library().nmspmm_kv4_append if four else serve._library().nmspmm_kv_append_norm
    cache = cache4 if four else cache16
    sizes = [dict(page_size=0), dict(heads=0), dict(dim=0), dict(sequences=-1), dict(table_pages=-1), dict(table=None)]
    sizes += [dict(page_count=-1), dict(pages=None), dict(page_stride=16)] if four else \
        [dict(pages=-1), dict(dtype=3), dict(k_pages=None), dict(v_pages=None)]
    for bad in sizes:
        assert append(fn, cache(**bad)) == INVALID, bad
    for bad in (dict(tokens=-1), dict(rot=3), dict(rot=-2), dict(rot=66), dict(positions=-1), dict(q_heads=-1),
                dict(dtype=5), dict(k=None), dict(v=None), dict(ks=None), dict(vs=None), dict(seq=None), dict(pos=None),
                dict(cos=None), dict(sin=None), dict(q=None), dict(q_out=None), dict(qs=None), dict(qos=None),
                dict(eps=-1e-6), dict(eps=float("nan"))):
        assert append(fn, cache(), **bad) == INVALID, bad
    for bad in (dict(k=PTR + 1), dict(v=PTR + 1), dict(q=PTR + 1), dict(q_out=PTR + 1), dict(seq=PTR + 2),
                dict(pos=PTR + 2), dict(cos=PTR + 2), dict(sin=PTR + 1), dict(q_norm=PTR + 2), dict(k_norm=PTR + 1),
                dict(tokens=1 << 24), dict(q_heads=1 << 17), dict(q_heads=1 << 62), dict(positions=1 << 31)):
        assert append(fn, cache(), **bad) == UNSUPPORTED, bad
    for bad in [dict(dim=513), dict(table=PTR + 2)] + ([dict(pages=PTR + 8), dict(page_stride=1 << 20 | 8)] if four else
                                                       [dict(k_pages=PTR + 1), dict(dtype=F32, v_pages=PTR + 2)]):
        assert append(fn, cache(**bad)) == UNSUPPORTED, bad
    assert append(fn, cache(), tokens=0, k=None, v=None) == OK
    assert append(fn, None) == INVALID


def test_read_refusals():
    fn = mx4._library().nmspmm_kv4_read

    def read(c=None, tokens=4, seq=PTR, pos=PTR, dtype=BF16, k=PTR, ks=PAIR, v=PTR, vs=PAIR):
        return fn(c or cache4(), tokens, seq, pos, dtype, k, ks, v, vs, None)

    for bad in (dict(tokens=-1), dict(dtype=3), dict(seq=None), dict(pos=None), dict(ks=None), dict(vs=None),
                dict(c=cache4(heads=0)), dict(c=cache4(pages=None)), dict(c=cache4(table=None))):
        assert read(**bad) == INVALID, bad
    for bad in (dict(k=PTR + 1), dict(v=PTR + 1), dict(dtype=F32, v=PTR + 2), dict(seq=PTR + 2), dict(pos=PTR + 1),
                dict(tokens=1 << 24), dict(c=cache4(dim=513)), dict(c=cache4(pages=PTR + 4))):
        assert read(**bad) == UNSUPPORTED, bad
    assert read(tokens=0, seq=None) == OK
    assert read(k=None, v=None, seq=None) == OK
    assert fn(None, 1, PTR, PTR, BF16, PTR, PAIR, PTR, PAIR, None) == INVALID


# ---- attention -------------------------------------------------------------

def attend(c=None, q=PTR, qs=PAIR, dtype=BF16, q_heads=4, lengths=PTR, max_length=64, window=0, out=PTR, os_=PAIR,
           lse=None, ws=None, ws_bytes=0):
    return mx4._library().nmspmm_kv4_attend(c or cache4(), q, qs, dtype, q_heads, lengths, max_length, window, 1.0, out,
                                            os_, lse, ws, ws_bytes, None)


def test_attend_refusals():
    for bad in (dict(page_size=0), dict(heads=0), dict(dim=0), dict(pages=None), dict(table=None), dict(page_stride=16)):
        assert attend(cache4(**bad)) == INVALID, bad
    for bad in (dict(q_heads=3), dict(q_heads=-2), dict(max_length=-1), dict(window=-1), dict(dtype=3), dict(q=None),
                dict(qs=None), dict(lengths=None), dict(out=None), dict(os_=None)):
        assert attend(**bad) == INVALID, bad
    for bad in (dict(q=PTR + 1), dict(out=PTR + 1), dict(lengths=PTR + 2), dict(lse=PTR + 2), dict(ws=PTR + 64),
                dict(c=cache4(dim=513)), dict(q_heads=1 << 40), dict(c=cache4(sequences=1 << 31)),
                dict(c=cache4(pages=PTR + 1)), dict(dtype=F32, q=PTR + 2)):
        assert attend(**bad) == UNSUPPORTED, bad
    assert attend(q_heads=0, q=None, out=None) == OK
    assert attend(cache4(sequences=0, table=None)) == OK
    L = mx4._library()
    assert L.nmspmm_kv4_attend_workspace_bytes(cache4(), 3, 64, 0) == -1
    assert L.nmspmm_kv4_attend_workspace_bytes(cache4(heads=0), 4, 64, 0) == -1
    assert L.nmspmm_kv4_attend_workspace_bytes(None, 4, 64, 0) == -1
    assert L.nmspmm_kv4_attend_workspace_bytes(cache4(), 0, 64, 0) == 0
    long = cache4(sequences=1, table_pages=10000)
    assert L.nmspmm_kv4_attend_workspace_bytes(long, 4, 160000, 0) > 0


def test_page_bytes():
    for page, heads, dim in ((16, 8, 128), (64, 1, 64), (16, 2, 80), (1, 1, 1), (7, 3, 300), (24, 4, 256)):
        size, groups = nm.nmspmm_kv4_page_bytes(page, heads, dim), -(-dim // 32)
        assert size % 16 == 0 and size >= 2 * page * heads * 17 * groups
        assert page % 4 or size <= 2 * heads * (page * (16 * groups + 2 * groups) + 32)
    assert nm.nmspmm_kv4_page_bytes(16, 8, 128) == 16 * 8 * 2 * (64 + 4)        # no padding
    for bad in ((0, 1, 64), (16, 0, 64), (16, 1, 0), (16, 1, 513), (-1, 1, 1), (2 ** 31 - 1, 2 ** 31 - 1, 512)):
        assert nm.nmspmm_kv4_page_bytes(*bad) == -1, bad
    # such a page has no cache either
    assert attend(cache4(page_size=2 ** 31 - 1, heads=2 ** 31 - 2, dim=512, page_stride=1 << 40), q_heads=0) == UNSUPPORTED


def test_binding_checks_before_any_gpu_call():
    torch = pytest.importorskip("torch")
    host, i32 = torch.zeros(4, 4096, dtype=torch.uint8), torch.zeros(1, 1, dtype=torch.int32)
    with pytest.raises(TypeError, match="pages must be a CUDA tensor"):
        nm.nmspmm_kv4_cache(host, i32, 16, 2, 64)
    with pytest.raises(nm.NmSpmmError):
        nm.nmspmm_kv4_cache(host, i32, 16, 2, 513)
    with pytest.raises(TypeError, match="codes must be a contiguous CUDA tensor"):
        nm.nmspmm_mx4_pack(torch.zeros(8, 64, dtype=torch.uint8), torch.zeros(1, 64, dtype=torch.uint8), None, 64, 64, 4,
                           32, 32)
    with pytest.raises(nm.NmSpmmError):
        nm.nmspmm_mx4_pack(host, host, host, 64, 65, 4, 32, 32)
    with pytest.raises(TypeError, match="Bc must be a contiguous CUDA tensor"):
        nm.nmspmm_mx4_quantize(torch.zeros(32, 32))
    for call, kind in ((nm.nmspmm_kv_append_norm, "KvCache"), (nm.nmspmm_kv4_append, "Kv4Cache")):
        with pytest.raises(TypeError, match=f"cache must be a {kind}"):
            call(None, torch.zeros(1, 1, 1), torch.zeros(1, 1, 1), i32[0], i32[0])
        with pytest.raises(ValueError, match="cos and sin go together"):
            call(None, None, None, None, None, cos=torch.zeros(1, 1))
        with pytest.raises(ValueError, match="q_out without q"):
            call(None, None, None, None, None, q_out=torch.zeros(1, 1))
    with pytest.raises(TypeError, match="cache must be a Kv4Cache"):
        nm.nmspmm_kv4_read(None, i32[0], i32[0])
    with pytest.raises(TypeError, match="cache must be a Kv4Cache"):
        nm.nmspmm_kv4_attend(None, None, None, None)
    with pytest.raises(TypeError, match="weight must be an Mx4Weight"):
        nm.nmspmm_mx4_run(None, None, None)
