"""ctypes binding of the 4-bit operators (include/nmspmm_mx4.h): the product
with a 4-bit weight and the paged key-value cache in 4 bits, under the C names.

Argument marshalling only, as in serve.py.  A packed weight (``Mx4Weight``) and
a cache (``Kv4Cache``) are handles that a program makes once and passes to
every call; they hold the tensors and their description, nothing of a call.
"""
from __future__ import annotations

import ctypes

from . import binding, serve
from .binding import _call, _check, _raw_stream
from .serve import HALF_ACTS, _append_norm, _check_cache, _Pair, _require, _shape, _workspace

MX4_EXPORTS = (
    "nmspmm_mx4_bytes", "nmspmm_mx4_quantize", "nmspmm_mx4_pack", "nmspmm_mx4_workspace_bytes", "nmspmm_mx4_run",
    "nmspmm_mx4_kernel_name", "nmspmm_kv4_page_bytes", "nmspmm_kv4_append", "nmspmm_kv4_read",
    "nmspmm_kv4_attend_workspace_bytes", "nmspmm_kv4_attend",
)


class _Weight(ctypes.Structure):
    _fields_ = [("packed", ctypes.c_void_p), ("N", ctypes.c_int32), ("M", ctypes.c_int32), ("V", ctypes.c_int32),
                ("k", ctypes.c_int64), ("n", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("pages", ctypes.c_void_p), ("page_stride", ctypes.c_int64), ("page_count", ctypes.c_int64),
                ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("sequences", ctypes.c_int64),
                ("table_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32),
                ("dim", ctypes.c_int32)]


_lib = None
_dtypes = None


def _library():
    """The library with this header's signatures declared."""
    global _lib, _dtypes
    if _lib is None:
        L = serve._library()
        declare(L)
        _dtypes = serve._dtypes
        _lib = L
    return _lib


def declare(L):
    """Declares the signatures of nmspmm_mx4.h on a handle of the library."""
    I64, I, P, F, Z = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
    W, C = ctypes.POINTER(_Weight), ctypes.POINTER(_Cache)
    S = ctypes.POINTER(ctypes.c_int64)
    L.nmspmm_mx4_bytes.argtypes = [I64, I64, I, I, I]
    L.nmspmm_mx4_bytes.restype = I64
    L.nmspmm_mx4_quantize.argtypes = [P, I, I64, I64, P, P, P]
    L.nmspmm_mx4_quantize.restype = I
    L.nmspmm_mx4_pack.argtypes = [P, P, P, W, P]
    L.nmspmm_mx4_pack.restype = I
    L.nmspmm_mx4_workspace_bytes.argtypes = [I64, W]
    L.nmspmm_mx4_workspace_bytes.restype = I64
    L.nmspmm_mx4_kernel_name.argtypes = [I64, W, I]
    L.nmspmm_mx4_kernel_name.restype = ctypes.c_char_p
    L.nmspmm_mx4_run.argtypes = [P, I64, I, W, P, I64, I, I64, F, P, I, P, I64, P, I64, P, Z, P]
    L.nmspmm_mx4_run.restype = I
    L.nmspmm_kv4_page_bytes.argtypes = [I64, I64, I64]
    L.nmspmm_kv4_page_bytes.restype = I64
    L.nmspmm_kv4_append.argtypes = [C, P, P, P, P, I, I64, P, P, P, P, I64, I, I, P, P, F, P, P, P, P, I64, P]
    L.nmspmm_kv4_append.restype = I
    L.nmspmm_kv4_read.argtypes = [C, I64, P, P, I, P, S, P, S, P]
    L.nmspmm_kv4_read.restype = I
    L.nmspmm_kv4_attend_workspace_bytes.argtypes = [C, I64, I64, I64]
    L.nmspmm_kv4_attend_workspace_bytes.restype = I64
    L.nmspmm_kv4_attend.argtypes = [C, P, S, I, I64, P, I64, I64, F, P, S, P, P, Z, P]
    L.nmspmm_kv4_attend.restype = I
    return L


# ---- the product -----------------------------------------------------------

class Mx4Weight:
    """An N:M sparse weight in 4 bits laid out by nmspmm_mx4_pack for nmspmm_mx4_run."""

    def __init__(self, packed, k, n, N, M, V):
        size, held = nmspmm_mx4_bytes(k, n, N, M, V), _workspace(packed, getattr(packed, "device", None), "packed")[1]
        if size < 0:
            raise binding.NmSpmmError("Mx4Weight", binding.NMSPMM_ERR_INVALID_ARG,
                                      f"invalid shape k={k} n={n} N={N} M={M} V={V}")
        if held < size:
            raise ValueError(f"packed has {held} bytes, {size} needed")
        self.packed, self.device, self.at = packed, packed.device, packed.get_device()
        self.k, self.n, self.N, self.M, self.V = k, n, N, M, V
        self._c = _Weight(packed.data_ptr(), N, M, V, k, n)
        self._ref = ctypes.pointer(self._c)


def nmspmm_mx4_bytes(k: int, n: int, N: int, M: int, V: int) -> int:
    return int(_library().nmspmm_mx4_bytes(k, n, N, M, V))


def _bytes_of(name, t, shape, device):
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of torch.uint8")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, {device} expected")
    _shape(name, t, shape)


def _new_bytes(torch, shape, device, at, stream):
    """Memory for a call on `stream`, from that stream's pool: a block of the
    current stream's may still be in use by work queued there."""
    with torch.cuda.stream(stream):     # (None: the current one)
        t = torch.empty(shape, dtype=torch.uint8, device=device)
    if stream is not None:
        t.record_stream(torch.cuda.current_stream(at))
    return t


def nmspmm_mx4_quantize(Bc, codes=None, scales=None, stream=None):
    """Brings Bc (w x n, contiguous, fp32 or 16-bit) to 4 bits and returns
    (codes, scales): codes (w x n) uint8 of 0 to 15, scales (ceil(w/32) x n)
    uint8, one for 32 rows of a column (default: new tensors)."""
    import torch
    L = _lib or _library()
    if not isinstance(Bc, torch.Tensor) or Bc.dtype not in _dtypes or not Bc.is_cuda or not Bc.is_contiguous():
        raise TypeError(f"Bc must be a contiguous CUDA tensor of {' or '.join(str(d) for d in _dtypes)}")
    if Bc.dim() != 2:
        raise ValueError("Bc must be 2-D")
    (w, n), at = Bc.shape, Bc.get_device()
    groups = (w + 31) // 32
    if codes is None:
        codes = _new_bytes(torch, (w, n), Bc.device, at, stream)
    if scales is None:
        scales = _new_bytes(torch, (groups, n), Bc.device, at, stream)
    _bytes_of("codes", codes, (w, n), Bc.device)
    _bytes_of("scales", scales, (groups, n), Bc.device)
    st = _call(torch, at, L.nmspmm_mx4_quantize, Bc.data_ptr(), _dtypes[Bc.dtype], w, n, codes.data_ptr(),
               scales.data_ptr(), _raw_stream(torch, at, stream))
    _check("nmspmm_mx4_quantize", st)
    return codes, scales


def nmspmm_mx4_pack(codes, scales, idx, n: int, k: int, N: int, M: int, V: int, packed=None, stream=None):
    """Lays codes (w x n), scales (ceil(w/32) x n) and idx (w x q; None where
    N = M), contiguous CUDA tensors of uint8, out for nmspmm_mx4_run and returns
    the ``Mx4Weight``.  ``packed``: the uint8 tensor to write, nmspmm_mx4_bytes
    long (default: a new one)."""
    import torch
    L = _lib or _library()
    size = nmspmm_mx4_bytes(k, n, N, M, V)
    if size < 0:
        raise binding.NmSpmmError("nmspmm_mx4_pack", binding.NMSPMM_ERR_INVALID_ARG,
                                  f"invalid shape k={k} n={n} N={N} M={M} V={V}")
    w = k // M * N
    _bytes_of("codes", codes, (w, n), None)
    _bytes_of("scales", scales, ((w + 31) // 32, n), codes.device)
    if idx is not None or N != M:
        _bytes_of("idx", idx, (w, n // V), codes.device)
    at = codes.get_device()
    if packed is None:
        packed = _new_bytes(torch, (size,), codes.device, at, stream)
    elif _workspace(packed, codes.device, "packed")[1] < size:
        raise ValueError(f"packed has {packed.numel()} bytes, {size} needed")
    weight = Mx4Weight(packed, k, n, N, M, V)
    st = _call(torch, at, L.nmspmm_mx4_pack, codes.data_ptr(), scales.data_ptr(),
               None if idx is None else idx.data_ptr(), weight._ref, _raw_stream(torch, at, stream))
    _check("nmspmm_mx4_pack", st)
    return weight


def nmspmm_mx4_workspace_bytes(m: int, weight: Mx4Weight) -> int:
    """Workspace bytes with which nmspmm_mx4_run splits k for m rows (0: it does not; -1: bad shape)."""
    return int(_library().nmspmm_mx4_workspace_bytes(m, weight._ref))


def nmspmm_mx4_kernel_name(m: int, weight: Mx4Weight, with_workspace: bool = True) -> str:
    return _library().nmspmm_mx4_kernel_name(m, weight._ref, int(with_workspace)).decode()


def nmspmm_mx4_run(A, weight: Mx4Weight, C, alpha: float = 1.0, bias=None, act: str = "none", mul=None, residual=None,
                   workspace=None, stream=None):
    """C = act(alpha * (A * B) + bias) * mul + residual on the GPU,
    asynchronously on ``stream`` (default: torch's current stream).  A (m x k)
    is bfloat16 or float16; C (m x n) A's type or fp32; mul and residual C's
    shape and type (either may be C itself); bias is n contiguous fp32 values.
    Rows of A, C, mul and residual may lie any stride apart.  act: "none",
    "relu", "gelu" or "silu".  ``workspace``: a contiguous uint8 tensor,
    256-byte aligned, of nmspmm_mx4_workspace_bytes bytes (or None: the
    library's own)."""
    import torch
    L = _lib or _library()
    # one expression for what holds in every good call, as in nmspmm_half_run
    try:
        at, dtype, c_dtype, shape, n = weight.at, A.dtype, C.dtype, C.shape, weight.n
        good = (type(weight) is Mx4Weight and (dtype is torch.bfloat16 or dtype is torch.float16)
                and (c_dtype is dtype or c_dtype is torch.float32) and A.get_device() == at
                and C.get_device() == at and len(shape) == 2 and A.shape == (shape[0], weight.k) and shape[1] == n
                and A.stride(1) == 1 and C.stride(1) == 1
                and (mul is None or (mul.dtype is c_dtype and mul.get_device() == at and mul.shape == shape
                                     and mul.stride(1) == 1))
                and (residual is None or (residual.dtype is c_dtype and residual.get_device() == at
                                          and residual.shape == shape and residual.stride(1) == 1))
                and (bias is None or (bias.dtype is torch.float32 and bias.get_device() == at and bias.shape == (n,)
                                      and bias.stride(0) == 1)))
    except AttributeError:      # no tensor, or no handle
        good = False
    if not good:
        _check_run(A, weight, C, bias, mul, residual)
    if act not in HALF_ACTS:
        raise ValueError(f"act must be one of {sorted(HALF_ACTS)}")
    ws, size = (None, 0) if workspace is None else _workspace(workspace, weight.device)
    st = _call(torch, at, L.nmspmm_mx4_run, A.data_ptr(), A.stride(0), _dtypes[dtype], weight._ref, C.data_ptr(),
               C.stride(0), _dtypes[c_dtype], shape[0], alpha, None if bias is None else bias.data_ptr(),
               HALF_ACTS[act], None if mul is None else mul.data_ptr(), 0 if mul is None else mul.stride(0),
               None if residual is None else residual.data_ptr(), 0 if residual is None else residual.stride(0),
               ws, size, _raw_stream(torch, at, stream))
    if st:
        _check("nmspmm_mx4_run", st)
    return C


def _check_run(A, weight, C, bias, mul, residual):
    import torch
    if not isinstance(weight, Mx4Weight):
        raise TypeError("weight must be an Mx4Weight")
    dev = weight.device
    _require("A", A, (torch.bfloat16, torch.float16), 2, dev)
    _shape("A", A, (A.shape[0], weight.k))
    _require("C", C, (A.dtype, torch.float32), 2, dev)
    _shape("C", C, (A.shape[0], weight.n))
    for name, t in (("mul", mul), ("residual", residual)):
        if t is not None:
            _require(name, t, (C.dtype,), 2, dev)
            _shape(name, t, C.shape)
    if bias is not None:
        _require("bias", bias, (torch.float32,), 1, dev)
        _shape("bias", bias, (weight.n,))


# ---- the cache -------------------------------------------------------------

def nmspmm_kv4_page_bytes(page_size: int, heads: int, dim: int) -> int:
    """Bytes of a page of the 4-bit cache (-1: bad sizes)."""
    return int(_library().nmspmm_kv4_page_bytes(page_size, heads, dim))


class Kv4Cache:
    """A paged key-value cache in 4 bits: ``pages`` (pages, at least
    nmspmm_kv4_page_bytes) uint8 with a contiguous last dimension, and the
    table (sequences, table_pages) of int32 page numbers.  The tensors stay
    the caller's; pages need no clearing."""

    def __init__(self, pages, table, page_size, heads, dim):
        import torch
        size = nmspmm_kv4_page_bytes(page_size, heads, dim)
        if size < 0:
            raise binding.NmSpmmError("Kv4Cache", binding.NMSPMM_ERR_INVALID_ARG,
                                      f"invalid sizes page_size={page_size} heads={heads} dim={dim}")
        _require("pages", pages, (torch.uint8,), 2, None)
        _require("table", table, (torch.int32,), 2, pages.device)
        if pages.shape[1] < size:
            raise ValueError(f"pages has rows of {pages.shape[1]} bytes, {size} needed")
        self.pages, self.table = pages, table
        self.device, self.at = pages.device, pages.get_device()
        self.page_size, self.heads, self.dim = page_size, heads, dim
        self.page_count = pages.shape[0]
        self.sequences, self.table_pages = table.shape
        # (one page's stride may be anything)
        stride = pages.stride(0) if self.page_count > 1 else size
        self._c = _Cache(pages.data_ptr(), stride, self.page_count, table.data_ptr(), table.stride(0), self.sequences,
                         self.table_pages, page_size, heads, dim)
        self._ref = ctypes.pointer(self._c)


def nmspmm_kv4_cache(pages, table, page_size: int, heads: int, dim: int) -> Kv4Cache:
    """The handle of a paged cache in 4 bits, for the calls below."""
    return Kv4Cache(pages, table, page_size, heads, dim)


def nmspmm_kv4_append(cache: Kv4Cache, k, v, seq, pos, cos=None, sin=None, q=None, q_out=None, interleaved=False,
                      q_norm=None, k_norm=None, eps: float = 1e-6, stream=None):
    """nmspmm_kv_append_norm into a 4-bit cache: k and v (tokens, heads, dim)
    of new tokens, token t at position pos[t] of sequence seq[t], keys (and
    queries) normalised and turned first.  The tokens' places must differ."""
    L = _lib or _library()
    return _append_norm("nmspmm_kv4_append", L.nmspmm_kv4_append, Kv4Cache, cache, k, v, seq, pos, cos, sin, q, q_out,
                        interleaved, q_norm, k_norm, eps, stream)


def nmspmm_kv4_read(cache: Kv4Cache, seq, pos, k_out=None, v_out=None, stream=None):
    """Reads the keys and values of the places (seq[t], pos[t]) back into
    k_out and v_out (tokens, heads, dim) of one type, either of which may be
    None; rows of tokens without a place are left as they were.  Returns
    (k_out, v_out)."""
    import torch
    L = _lib or _library()
    some = v_out if k_out is None else k_out
    # as in nmspmm_half_run: one expression, and _check_read words the rest
    try:
        at, tokens = cache.at, seq.shape
        good = (type(cache) is Kv4Cache and seq.dtype is torch.int32 and pos.dtype is torch.int32
                and seq.get_device() == at and pos.get_device() == at and len(tokens) == 1 and pos.shape == tokens
                and seq.is_contiguous() and pos.is_contiguous())
        dtype, ks, vs = torch.float32, (0, 0), (0, 0)
        if some is not None:
            dtype, shape = some.dtype, (tokens[0], cache.heads, cache.dim)
            good = good and dtype in _dtypes
        if k_out is not None:
            ks = k_out.stride()
            good = good and k_out.shape == shape and k_out.get_device() == at and ks[2] == 1
        if v_out is not None:
            vs = v_out.stride()
            good = good and v_out.shape == shape and v_out.dtype is dtype and v_out.get_device() == at and vs[2] == 1
    except (AttributeError, IndexError):
        good = False
    if not good:
        _check_read(cache, seq, pos, k_out, v_out)
    st = _call(torch, at, L.nmspmm_kv4_read, cache._ref, tokens[0], seq.data_ptr(), pos.data_ptr(), _dtypes[dtype],
               0 if k_out is None else k_out.data_ptr(), _Pair(ks[0], ks[1]), 0 if v_out is None else v_out.data_ptr(),
               _Pair(vs[0], vs[1]), _raw_stream(torch, at, stream))
    if st:
        _check("nmspmm_kv4_read", st)
    return k_out, v_out


def _check_read(cache, seq, pos, k_out, v_out):
    import torch
    _check_cache(cache, Kv4Cache)
    _require("seq", seq, (torch.int32,), 1, cache.device)
    _require("pos", pos, (torch.int32,), 1, cache.device)
    _shape("pos", pos, seq.shape)
    dtypes = tuple(_dtypes)
    for name, t in (("k_out", k_out), ("v_out", v_out)):
        if t is not None:
            _require(name, t, dtypes, 3, cache.device)
            _shape(name, t, (seq.shape[0], cache.heads, cache.dim))
            dtypes = (t.dtype,)


def nmspmm_kv4_attend_workspace_bytes(cache: Kv4Cache, q_heads: int, max_length: int, window: int = 0) -> int:
    """Workspace bytes with which nmspmm_kv4_attend splits sequences (0: it does not; -1: bad sizes)."""
    return int(_library().nmspmm_kv4_attend_workspace_bytes(cache._ref, q_heads, max_length, window))


def nmspmm_kv4_attend(cache: Kv4Cache, q, lengths, out, scale=None, window: int = 0, max_length=None, lse=None,
                      workspace=None, stream=None):
    """Attention of one new token per sequence over the 4-bit cache; arguments
    as for nmspmm_kv_attend (``workspace``: nmspmm_kv4_attend_workspace_bytes
    bytes)."""
    import torch
    L = _lib or _library()
    try:
        at, dtype, shape, qs, outs = cache.at, q.dtype, q.shape, q.stride(), out.stride()
        good = (type(cache) is Kv4Cache and dtype in _dtypes and out.dtype is dtype and q.get_device() == at
                and out.get_device() == at and len(shape) == 3 and shape[0] == cache.sequences
                and shape[2] == cache.dim and out.shape == shape and qs[2] == 1 and outs[2] == 1
                and lengths.dtype is torch.int32 and lengths.get_device() == at and lengths.shape == shape[:1]
                and lengths.stride(0) == 1 and lse is None)
    except AttributeError:
        good = False
    if not good:
        serve._check_attend(cache, q, lengths, out, lse, Kv4Cache)
    if max_length is None:
        max_length = cache.table_pages * cache.page_size
    if scale is None:
        scale = cache.dim ** -0.5
    ws, size = (None, 0) if workspace is None else _workspace(workspace, cache.device)
    st = _call(torch, at, L.nmspmm_kv4_attend, cache._ref, q.data_ptr(), _Pair(qs[0], qs[1]), _dtypes[dtype], shape[1],
               lengths.data_ptr(), max_length, window, scale, out.data_ptr(), _Pair(outs[0], outs[1]),
               None if lse is None else lse.data_ptr(), ws, size, _raw_stream(torch, at, stream))
    if st:
        _check("nmspmm_kv4_attend", st)
    return out
