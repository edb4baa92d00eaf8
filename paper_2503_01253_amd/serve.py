"""ctypes binding of the decoding-step operators (include/nmspmm_serve.h): the
16-bit N:M product and the paged key-value cache, under the C names.

Argument marshalling only, as in binding.py: every step runs in the library's
HIP kernels, and there is no fallback.  A packed weight (``HalfWeight``) and a
cache (``KvCache``) are handles that a program makes once and passes to every
call; they hold the tensors and their description, nothing of a call.
"""
from __future__ import annotations

import ctypes

from . import binding
from .binding import _call, _check, _raw_stream

NMSPMM_F32, NMSPMM_BF16, NMSPMM_F16 = 0, 1, 2
HALF_ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}

SERVE_EXPORTS = (
    "nmspmm_half_bytes", "nmspmm_half_pack", "nmspmm_half_workspace_bytes", "nmspmm_half_run",
    "nmspmm_half_kernel_name", "nmspmm_kv_append", "nmspmm_kv_append_norm", "nmspmm_kv_attend_workspace_bytes",
    "nmspmm_kv_attend",
)


class _Weight(ctypes.Structure):
    _fields_ = [("packed", ctypes.c_void_p), ("dtype", ctypes.c_int), ("N", ctypes.c_int32), ("M", ctypes.c_int32),
                ("V", ctypes.c_int32), ("k", ctypes.c_int64), ("n", ctypes.c_int64)]


class _Cache(ctypes.Structure):
    _fields_ = [("k_pages", ctypes.c_void_p), ("v_pages", ctypes.c_void_p), ("k_stride", ctypes.c_int64 * 3),
                ("v_stride", ctypes.c_int64 * 3), ("pages", ctypes.c_int64), ("table", ctypes.c_void_p),
                ("table_stride", ctypes.c_int64), ("sequences", ctypes.c_int64), ("table_pages", ctypes.c_int64),
                ("page_size", ctypes.c_int32), ("heads", ctypes.c_int32), ("dim", ctypes.c_int32),
                ("dtype", ctypes.c_int)]


_Pair = ctypes.c_int64 * 2
_Strides = ctypes.c_int64 * 8
_lib = None
_dtypes = None


def _library():
    """The library with this header's signatures declared."""
    global _lib, _dtypes
    if _lib is None:
        import torch
        L = binding.lib()
        declare(L)
        _dtypes = {torch.float32: NMSPMM_F32, torch.bfloat16: NMSPMM_BF16, torch.float16: NMSPMM_F16}
        _lib = L
    return _lib


def declare(L):
    """Declares the signatures of nmspmm_serve.h on a handle of the library."""
    I64, I, P, F, Z = ctypes.c_int64, ctypes.c_int, ctypes.c_void_p, ctypes.c_float, ctypes.c_size_t
    W, C = ctypes.POINTER(_Weight), ctypes.POINTER(_Cache)
    S = ctypes.POINTER(ctypes.c_int64)
    L.nmspmm_half_bytes.argtypes = [I64, I64, I, I, I]
    L.nmspmm_half_bytes.restype = I64
    L.nmspmm_half_pack.argtypes = [P, I, P, W, P]
    L.nmspmm_half_pack.restype = I
    L.nmspmm_half_workspace_bytes.argtypes = [I64, W]
    L.nmspmm_half_workspace_bytes.restype = I64
    L.nmspmm_half_kernel_name.argtypes = [I64, W, I]
    L.nmspmm_half_kernel_name.restype = ctypes.c_char_p
    L.nmspmm_half_run.argtypes = [P, I64, W, P, I64, I, I64, F, P, I, P, I64, P, I64, P, Z, P]
    L.nmspmm_half_run.restype = I
    L.nmspmm_kv_append.argtypes = [C, P, S, P, S, I, I64, P, P, P, P, I64, I, I, P, S, P, S, I64, P]
    L.nmspmm_kv_append.restype = I
    # (strides as addresses: four in one array of _append_norm's)
    L.nmspmm_kv_append_norm.argtypes = [C, P, P, P, P, I, I64, P, P, P, P, I64, I, I, P, P, F, P, P, P, P, I64, P]
    L.nmspmm_kv_append_norm.restype = I
    L.nmspmm_kv_attend_workspace_bytes.argtypes = [C, I64, I64, I64]
    L.nmspmm_kv_attend_workspace_bytes.restype = I64
    L.nmspmm_kv_attend.argtypes = [C, P, S, I, I64, P, I64, I64, F, P, S, P, P, Z, P]
    L.nmspmm_kv_attend.restype = I
    return L


def _require(name, t, dtypes, dim, device):
    """A tensor of one of `dtypes` with `dim` dimensions on `device` (None:
    any CUDA device), its last dimension contiguous."""
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA tensor of {' or '.join(str(d) for d in dtypes)}")
    if t.dim() != dim:
        raise ValueError(f"{name} must be {dim}-D")
    if t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}'s last dimension must be contiguous")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, {device} expected")


def _shape(name, t, shape):
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")


def _workspace(t, device, name="workspace"):
    """Address and size of a workspace tensor, or nothing."""
    if t is None:
        return None, 0
    import torch
    if not isinstance(t, torch.Tensor) or t.dtype != torch.uint8 or not t.is_cuda or not t.is_contiguous():
        raise TypeError(f"{name} must be a contiguous CUDA tensor of torch.uint8")
    if t.device != device:
        raise ValueError(f"{name} is on {t.device}, {device} expected")
    return t.data_ptr(), t.numel()


class HalfWeight:
    """An N:M sparse weight laid out by nmspmm_half_pack for nmspmm_half_run."""

    def __init__(self, packed, dtype, k, n, N, M, V):
        _library()
        if _dtypes.get(dtype) not in (NMSPMM_BF16, NMSPMM_F16):
            raise TypeError(f"dtype must be torch.bfloat16 or torch.float16, not {dtype}")
        size, held = nmspmm_half_bytes(k, n, N, M, V), _workspace(packed, getattr(packed, "device", None), "packed")[1]
        if size < 0:
            raise binding.NmSpmmError("HalfWeight", binding.NMSPMM_ERR_INVALID_ARG,
                                      f"invalid shape k={k} n={n} N={N} M={M} V={V}")
        if held < size:
            raise ValueError(f"packed has {held} bytes, {size} needed")
        self.packed, self.dtype, self.device, self.at = packed, dtype, packed.device, packed.get_device()
        self.k, self.n, self.N, self.M, self.V = k, n, N, M, V
        self._c = _Weight(packed.data_ptr(), _dtypes[dtype], N, M, V, k, n)
        self._ref = ctypes.pointer(self._c)


def nmspmm_half_bytes(k: int, n: int, N: int, M: int, V: int) -> int:
    return int(_library().nmspmm_half_bytes(k, n, N, M, V))


def nmspmm_half_pack(Bc, idx, n: int, k: int, N: int, M: int, V: int, dtype=None, packed=None, stream=None):
    """Lays Bc (w x n, fp32 or 16-bit) and idx (w x q uint8), contiguous CUDA
    tensors as nmspmm_compress_device writes them, out for nmspmm_half_run and
    returns the ``HalfWeight``.  ``dtype`` is the weight's type (default: Bc's,
    bfloat16 for an fp32 Bc).  ``packed``: the uint8 tensor to write,
    nmspmm_half_bytes long (default: a new one)."""
    import torch
    L = _library()
    size = nmspmm_half_bytes(k, n, N, M, V)
    if size < 0:
        raise binding.NmSpmmError("nmspmm_half_pack", binding.NMSPMM_ERR_INVALID_ARG,
                                  f"invalid shape k={k} n={n} N={N} M={M} V={V}")
    for name, t, dtypes, numel in (("Bc", Bc, tuple(_dtypes), (k // M) * N * n),
                                   ("idx", idx, (torch.uint8,), (k // M) * N * (n // V))):
        if not isinstance(t, torch.Tensor) or t.dtype not in dtypes or not t.is_cuda or not t.is_contiguous():
            raise TypeError(f"{name} must be a contiguous CUDA tensor of {' or '.join(str(d) for d in dtypes)}")
        if t.device != Bc.device:
            raise ValueError(f"{name} is on {t.device}, {Bc.device} expected")
        if t.numel() != numel:
            raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    if dtype is None:
        dtype = torch.bfloat16 if Bc.dtype == torch.float32 else Bc.dtype
    at = Bc.get_device()
    if packed is None:
        # from the pool of the stream that writes it: a block of the current
        # stream's may still be in use by work queued there
        with torch.cuda.stream(stream):     # (None: the current one)
            packed = torch.empty(size, dtype=torch.uint8, device=Bc.device)
        if stream is not None:
            packed.record_stream(torch.cuda.current_stream(at))
    elif _workspace(packed, Bc.device, "packed")[1] < size:
        raise ValueError(f"packed has {packed.numel()} bytes, {size} needed")
    weight = HalfWeight(packed, dtype, k, n, N, M, V)
    st = _call(torch, at, L.nmspmm_half_pack, Bc.data_ptr(), _dtypes[Bc.dtype], idx.data_ptr(), weight._ref,
               _raw_stream(torch, at, stream))
    _check("nmspmm_half_pack", st)
    return weight


def nmspmm_half_workspace_bytes(m: int, weight: HalfWeight) -> int:
    """Workspace bytes with which nmspmm_half_run splits k for m rows (0: it does not; -1: bad shape)."""
    return int(_library().nmspmm_half_workspace_bytes(m, weight._ref))


def nmspmm_half_kernel_name(m: int, weight: HalfWeight, with_workspace: bool = True) -> str:
    return _library().nmspmm_half_kernel_name(m, weight._ref, int(with_workspace)).decode()


def nmspmm_half_run(A, weight: HalfWeight, C, alpha: float = 1.0, bias=None, act: str = "none", mul=None,
                    residual=None, workspace=None, stream=None):
    """C = act(alpha * (A * B) + bias) * mul + residual on the GPU,
    asynchronously on ``stream`` (default: torch's current stream).  A (m x k)
    has the weight's type; C (m x n) that type or fp32; mul and residual C's
    shape and type (either may be C itself); bias is n contiguous fp32 values.  Rows of A, C, mul
    and residual may lie any stride apart.  act: "none", "relu", "gelu" or
    "silu".  ``workspace``: a contiguous uint8 tensor, 256-byte aligned, of
    nmspmm_half_workspace_bytes bytes (or None: the library's own)."""
    import torch
    L = _lib or _library()
    # one expression for what holds in every good call (a call's host time is
    # of the order of a small product's GPU time); _check_half words the rest
    try:
        at, dtype, c_dtype, shape, n = weight.at, weight.dtype, C.dtype, C.shape, weight.n
        good = (A.dtype is dtype and (c_dtype is dtype or c_dtype is torch.float32) and A.get_device() == at
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
        _check_half(A, weight, C, bias, mul, residual)
    if act not in HALF_ACTS:
        raise ValueError(f"act must be one of {sorted(HALF_ACTS)}")
    ws, size = (None, 0) if workspace is None else _workspace(workspace, weight.device)
    st = _call(torch, at, L.nmspmm_half_run, A.data_ptr(), A.stride(0), weight._ref, C.data_ptr(), C.stride(0),
               _dtypes[c_dtype], shape[0], alpha, None if bias is None else bias.data_ptr(), HALF_ACTS[act],
               None if mul is None else mul.data_ptr(), 0 if mul is None else mul.stride(0),
               None if residual is None else residual.data_ptr(), 0 if residual is None else residual.stride(0),
               ws, size, _raw_stream(torch, at, stream))
    if st:
        _check("nmspmm_half_run", st)
    return C


def _check_half(A, weight, C, bias, mul, residual):
    import torch
    if not isinstance(weight, HalfWeight):
        raise TypeError("weight must be a HalfWeight")
    dev = weight.device
    _require("A", A, (weight.dtype,), 2, dev)
    _shape("A", A, (A.shape[0], weight.k))
    _require("C", C, (weight.dtype, torch.float32), 2, dev)
    _shape("C", C, (A.shape[0], weight.n))
    for name, t in (("mul", mul), ("residual", residual)):
        if t is not None:
            _require(name, t, (C.dtype,), 2, dev)
            _shape(name, t, C.shape)
    if bias is not None:
        _require("bias", bias, (torch.float32,), 1, dev)
        _shape("bias", bias, (weight.n,))


class KvCache:
    """A paged key-value cache: k_pages and v_pages (pages, page_size, heads,
    dim), any strides with a contiguous last dimension, and the table
    (sequences, table_pages) of int32 page numbers.  The tensors stay the
    caller's: their contents, the table's among them, are read on the device
    by every call."""

    def __init__(self, k_pages, v_pages, table):
        import torch
        _library()
        _require("k_pages", k_pages, tuple(_dtypes), 4, None)
        _require("v_pages", v_pages, (k_pages.dtype,), 4, k_pages.device)
        _shape("v_pages", v_pages, k_pages.shape)
        _require("table", table, (torch.int32,), 2, k_pages.device)
        if max(k_pages.shape[1:]) > 2 ** 31 - 1:
            raise ValueError(f"k_pages has shape {tuple(k_pages.shape)}: a page's sizes are 32-bit")
        self.k_pages, self.v_pages, self.table = k_pages, v_pages, table
        self.device, self.dtype, self.at = k_pages.device, k_pages.dtype, k_pages.get_device()
        self.pages, self.page_size, self.heads, self.dim = k_pages.shape
        self.sequences, self.table_pages = table.shape
        S = ctypes.c_int64 * 3
        self._c = _Cache(k_pages.data_ptr(), v_pages.data_ptr(), S(*k_pages.stride()[:3]), S(*v_pages.stride()[:3]),
                         self.pages, table.data_ptr(), table.stride(0), self.sequences, self.table_pages,
                         self.page_size, self.heads, self.dim, _dtypes[k_pages.dtype])
        self._ref = ctypes.pointer(self._c)


def nmspmm_kv_cache(k_pages, v_pages, table) -> KvCache:
    """The handle of a paged cache, for the calls below."""
    return KvCache(k_pages, v_pages, table)


def nmspmm_kv_append(cache: KvCache, k, v, seq, pos, cos=None, sin=None, q=None, q_out=None, interleaved=False,
                     stream=None):
    """Writes k and v (tokens, heads, dim) of new tokens into the cache, token
    t at position pos[t] of sequence seq[t] (int32), asynchronously on
    ``stream``.  With cos and sin (positions, rot/2, contiguous fp32) the first
    rot dimensions of k, and of q (tokens, q_heads, dim) into q_out (default:
    in place), are turned by their position's angles, in pairs (d, d + rot/2)
    or, ``interleaved``, (2d, 2d + 1).  k, v, q and q_out have one type; their
    first two dimensions may have any strides.  Tokens without a place (a
    negative position, say) are skipped.  Returns q_out."""
    import torch
    L = _lib or _library()
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin go together")
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    if q is not None and q_out is None:
        q_out = q
    angles, queries = (None, None, 0, 0), (None, None, None, None, 0)
    # as in nmspmm_half_run: one expression, and the _check_ functions word the rest
    try:
        at, dtype, shape, ks, vs = cache.at, k.dtype, k.shape, k.stride(), v.stride()
        good = (dtype in _dtypes and v.dtype is dtype and k.get_device() == at and v.get_device() == at
                and len(shape) == 3 and v.shape == shape and shape[1] == cache.heads and shape[2] == cache.dim
                and ks[2] == 1 and vs[2] == 1 and seq.dtype is torch.int32 and pos.dtype is torch.int32
                and seq.get_device() == at and pos.get_device() == at and seq.shape == shape[:1]
                and pos.shape == seq.shape and seq.stride(0) == 1 and pos.stride(0) == 1)
    except AttributeError:
        good = False
    if not good:
        _check_append(cache, k, v, seq, pos)
    if cos is not None:
        try:
            good = (cos.dtype is torch.float32 and sin.dtype is torch.float32 and cos.get_device() == at
                    and sin.get_device() == at and cos.dim() == 2 and sin.shape == cos.shape and cos.is_contiguous()
                    and sin.is_contiguous())
        except AttributeError:
            good = False
        if not good:
            _check_angles(cache, cos, sin)
        rows, half = cos.shape
        angles = (cos.data_ptr(), sin.data_ptr(), rows, 2 * half)
    if q is not None:
        try:
            heads, qs, qos = q.shape[1], q.stride(), q_out.stride()
            good = (q.dtype is dtype and q_out.dtype is dtype and q.get_device() == at and q_out.get_device() == at
                    and q.shape == (shape[0], heads, cache.dim) and q_out.shape == q.shape and qs[2] == 1
                    and qos[2] == 1)
        except (AttributeError, IndexError):
            good = False
        if not good:
            _check_queries(cache, k, q, q_out)
        queries = (q.data_ptr(), _Pair(qs[0], qs[1]), q_out.data_ptr(), _Pair(qos[0], qos[1]), heads)
    st = _call(torch, at, L.nmspmm_kv_append, cache._ref, k.data_ptr(), _Pair(ks[0], ks[1]), v.data_ptr(),
               _Pair(vs[0], vs[1]), _dtypes[dtype], shape[0], seq.data_ptr(), pos.data_ptr(), *angles,
               interleaved, *queries, _raw_stream(torch, at, stream))
    if st:
        _check("nmspmm_kv_append", st)
    return q_out


def nmspmm_kv_append_norm(cache: KvCache, k, v, seq, pos, cos=None, sin=None, q=None, q_out=None, interleaved=False,
                          q_norm=None, k_norm=None, eps: float = 1e-6, stream=None):
    """nmspmm_kv_append with a norm of every head before the rotation: with
    q_norm and k_norm (dim contiguous fp32 weights, either may be None) a query
    or key x becomes x * weight / sqrt(mean(x^2) + eps).  All else as there."""
    L = _lib or _library()
    return _append_norm("nmspmm_kv_append_norm", L.nmspmm_kv_append_norm, KvCache, cache, k, v, seq, pos, cos, sin, q,
                        q_out, interleaved, q_norm, k_norm, eps, stream)


def _append_norm(name, call, kind, cache, k, v, seq, pos, cos, sin, q, q_out, interleaved, q_norm, k_norm, eps, stream):
    """What the appends with norms share; ``kind``: the cache's class."""
    import torch
    if (cos is None) != (sin is None):
        raise ValueError("cos and sin go together")
    if q is None and q_out is not None:
        raise ValueError("q_out without q")
    if q is not None and q_out is None:
        q_out = q
    # as in nmspmm_half_run: one expression each, and the _check_ functions word the rest
    try:
        at, dtype, shape, ks, vs, dim = cache.at, k.dtype, k.shape, k.stride(), v.stride(), cache.dim
        tokens = shape[:1]
        good = (type(cache) is kind and dtype in _dtypes and v.dtype is dtype and k.get_device() == at
                and v.get_device() == at and v.shape == shape and shape[1:] == (cache.heads, dim)
                and ks[2] == 1 and vs[2] == 1 and seq.dtype is torch.int32 and pos.dtype is torch.int32
                and seq.get_device() == at and pos.get_device() == at and seq.shape == tokens
                and pos.shape == tokens and seq.is_contiguous() and pos.is_contiguous())
    except (AttributeError, IndexError):
        good = False
    if not good:
        _check_append(cache, k, v, seq, pos, kind)
    cosp = sinp = rows = rot = 0
    if cos is not None:
        try:
            angles = cos.shape
            good = (cos.dtype is torch.float32 and sin.dtype is torch.float32 and cos.get_device() == at
                    and sin.get_device() == at and len(angles) == 2 and sin.shape == angles and cos.is_contiguous()
                    and sin.is_contiguous())
        except AttributeError:
            good = False
        if not good:
            _check_angles(cache, cos, sin)
        rows, rot = angles[0], 2 * angles[1]
        cosp, sinp = cos.data_ptr(), sin.data_ptr()
    qp = qop = heads = 0
    qs = qos = (0, 0)
    if q is not None:
        try:
            heads, qs, qos = q.shape[1], q.stride(), q_out.stride()
            good = (q.dtype is dtype and q_out.dtype is dtype and q.get_device() == at and q_out.get_device() == at
                    and q.shape == (shape[0], heads, dim) and q_out.shape == q.shape and qs[2] == 1
                    and qos[2] == 1)
        except (AttributeError, IndexError):
            good = False
        if not good:
            _check_queries(cache, k, q, q_out)
        qp, qop = q.data_ptr(), q_out.data_ptr()
    qn = kn = 0
    if q_norm is not None:
        qn = _norm_weight("q_norm", q_norm, cache, torch)
    if k_norm is not None:
        kn = _norm_weight("k_norm", k_norm, cache, torch)
    strides = _Strides(ks[0], ks[1], vs[0], vs[1], qs[0], qs[1], qos[0], qos[1])
    here = ctypes.addressof(strides)
    st = _call(torch, at, call, cache._ref, k.data_ptr(), here, v.data_ptr(), here + 16, _dtypes[dtype], shape[0],
               seq.data_ptr(), pos.data_ptr(), cosp, sinp, rows, rot, interleaved, qn, kn, eps, qp, here + 32, qop,
               here + 48, heads, _raw_stream(torch, at, stream))
    if st:
        _check(name, st)
    return q_out


def _norm_weight(name, w, cache, torch):
    """The address of a norm's weights."""
    try:
        good = w.dtype is torch.float32 and w.get_device() == cache.at and w.shape == (cache.dim,) and w.is_contiguous()
    except AttributeError:
        good = False
    if not good:
        _require(name, w, (torch.float32,), 1, cache.device)
        _shape(name, w, (cache.dim,))
    return w.data_ptr()


def _check_cache(cache, kind=None):
    kind = kind or KvCache
    if not isinstance(cache, kind):
        raise TypeError(f"cache must be a {kind.__name__}")


def _check_append(cache, k, v, seq, pos, kind=None):
    import torch
    _check_cache(cache, kind)
    _require("k", k, tuple(_dtypes), 3, cache.device)
    _shape("k", k, (k.shape[0], cache.heads, cache.dim))
    _require("v", v, (k.dtype,), 3, cache.device)
    _shape("v", v, k.shape)
    for name, t in (("seq", seq), ("pos", pos)):
        _require(name, t, (torch.int32,), 1, cache.device)
        _shape(name, t, k.shape[:1])


def _check_angles(cache, cos, sin):
    import torch
    for name, t in (("cos", cos), ("sin", sin)):
        _require(name, t, (torch.float32,), 2, cache.device)
        _shape(name, t, cos.shape)
        if not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")


def _check_queries(cache, k, q, q_out):
    _require("q", q, (k.dtype,), 3, cache.device)
    _shape("q", q, (k.shape[0], q.shape[1], cache.dim))
    _require("q_out", q_out, (k.dtype,), 3, cache.device)
    _shape("q_out", q_out, q.shape)


def nmspmm_kv_attend_workspace_bytes(cache: KvCache, q_heads: int, max_length: int, window: int = 0) -> int:
    """Workspace bytes with which nmspmm_kv_attend splits sequences (0: it does not; -1: bad sizes)."""
    return int(_library().nmspmm_kv_attend_workspace_bytes(cache._ref, q_heads, max_length, window))


def nmspmm_kv_attend(cache: KvCache, q, lengths, out, scale=None, window: int = 0, max_length=None, lse=None,
                     workspace=None, stream=None):
    """Attention of one new token per sequence over the cache, asynchronously
    on ``stream``: q and out (sequences, q_heads, dim) of one type, any strides
    in the first two dimensions; lengths (sequences,) int32, the new token
    included.  ``scale``: default dim ** -0.5.  ``window`` > 0: the last
    ``window`` positions only.  ``max_length``: an upper bound of the lengths
    (default: what the table can hold); a tighter one splits the work better.
    ``lse``: (sequences, q_heads) contiguous fp32 for the log-sum-exp, or None.
    ``workspace``: as for nmspmm_half_run, nmspmm_kv_attend_workspace_bytes
    bytes."""
    import torch
    L = _lib or _library()
    # as in nmspmm_half_run: one expression, and _check_attend words the rest
    try:
        at, dtype, shape, qs, outs = cache.at, q.dtype, q.shape, q.stride(), out.stride()
        good = (dtype in _dtypes and out.dtype is dtype and q.get_device() == at and out.get_device() == at
                and len(shape) == 3 and shape[0] == cache.sequences and shape[2] == cache.dim and out.shape == shape
                and qs[2] == 1 and outs[2] == 1 and lengths.dtype is torch.int32 and lengths.get_device() == at
                and lengths.shape == shape[:1] and lengths.stride(0) == 1 and lse is None)
    except AttributeError:
        good = False
    if not good:
        _check_attend(cache, q, lengths, out, lse)
    if max_length is None:
        max_length = cache.table_pages * cache.page_size
    if scale is None:
        scale = cache.dim ** -0.5
    ws, size = (None, 0) if workspace is None else _workspace(workspace, cache.device)
    st = _call(torch, at, L.nmspmm_kv_attend, cache._ref, q.data_ptr(), _Pair(qs[0], qs[1]), _dtypes[dtype],
               shape[1], lengths.data_ptr(), max_length, window, scale, out.data_ptr(), _Pair(outs[0], outs[1]),
               None if lse is None else lse.data_ptr(), ws, size, _raw_stream(torch, at, stream))
    if st:
        _check("nmspmm_kv_attend", st)
    return out


def _check_attend(cache, q, lengths, out, lse, kind=None):
    import torch
    _check_cache(cache, kind)
    dev = cache.device
    _require("q", q, tuple(_dtypes), 3, dev)
    _shape("q", q, (cache.sequences, q.shape[1], cache.dim))
    _require("out", out, (q.dtype,), 3, dev)
    _shape("out", out, q.shape)
    _require("lengths", lengths, (torch.int32,), 1, dev)
    _shape("lengths", lengths, (cache.sequences,))
    if lse is not None:
        _require("lse", lse, (torch.float32,), 2, dev)
        _shape("lse", lse, q.shape[:2])
        if not lse.is_contiguous():
            raise ValueError("lse must be contiguous")
