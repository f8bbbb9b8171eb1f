"""Operators around the recurrence in a hybrid model: binding of
``include/swr_hybrid.h``.

The normed residual stream (``swr_rms_norm``), the projections of decoded
tokens with 4-bit weights (``swr_fp4_pack``, ``swr_fp4_linear``) and the
attention layers over a paged key-value cache (``swr_block_tables``,
``swr_cache_append``, ``swr_paged_attention``).  The functions marshal torch
tensors into pointers, strides and the current HIP stream, the ordinary call in
native code (``csrc/swr_binding.cpp``); every step of the computation runs in
the library's HIP kernels.  There is no CPU fallback.
"""
import ctypes
import math

import paper_2512_13921_amd as _package

from . import (SWR_ABI_VERSION, SWR_DTYPE_BF16, SWR_DTYPE_F32, SwrError, _checked, _on, _opt, _ptr, _raw, _stream,
               _torch, load)

__all__ = ["swr_rms_norm", "swr_rms_norm_backward", "swr_fp4_pack", "swr_fp4_linear", "swr_block_tables",
           "swr_cache_append", "swr_paged_attention", "SWRNormFunction"]

SWR_DTYPE_FP8 = 2
FP4_GROUP = 32   # weights that share a power

_i32, _i64, _f32, _vp = ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class SwrNorm(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("weight_dtype", _i32), ("out_dtype", _i32),
                ("outer", _i64), ("inner", _i64), ("width", _i64), ("eps", _f32), ("reserved", _i32),
                ("sx_o", _i64), ("sx_i", _i64), ("sr_o", _i64), ("sr_i", _i64), ("sh_o", _i64), ("sh_i", _i64),
                ("sy_o", _i64), ("sy_i", _i64)]


class SwrFp4(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("out_dtype", _i32), ("reserved", _i32),
                ("M", _i64), ("N", _i64), ("K", _i64), ("sx", _i64), ("sy", _i64), ("sc", _i64), ("sp", _i64)]


class SwrTables(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("reserved", _i32), ("batch", _i64), ("max_pages", _i64), ("st", _i64),
                ("page_size", _i64), ("tokens", _i64), ("free_pages", _i64)]


class SwrCache(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("pages", _i64), ("page_size", _i64), ("heads", _i64),
                ("D", _i64), ("s_page", _i64), ("s_token", _i64), ("s_head", _i64)]


class SwrPaged(ctypes.Structure):
    _fields_ = [("cache", SwrCache), ("batch", _i64), ("q_heads", _i64), ("max_pages", _i64), ("st", _i64),
                ("window", _i64), ("sq_b", _i64), ("sq_h", _i64), ("sy_b", _i64), ("sy_h", _i64), ("scale", _f32),
                ("reserved", _i32)]


_bound = None


def _lib():
    """The loaded library, with the argument types of this header's calls."""
    global _bound
    lib = load()
    if _bound is not lib:
        P = ctypes.POINTER
        for name, restype, args in (
                ("swr_rms_norm", ctypes.c_int, [P(SwrNorm)] + [_vp] * 7),
                ("swr_rms_norm_workspace_bytes", _i64, [P(SwrNorm)]),
                ("swr_rms_norm_backward", ctypes.c_int, [P(SwrNorm)] + [_vp] * 8),
                ("swr_fp4_linear", ctypes.c_int, [P(SwrFp4)] + [_vp] * 6),
                ("swr_fp4_pack", ctypes.c_int, [P(SwrFp4)] + [_vp] * 4),
                ("swr_block_tables", ctypes.c_int, [P(SwrTables)] + [_vp] * 10),
                ("swr_cache_append", ctypes.c_int, [P(SwrCache), _i64, P(_i64), P(_i64)] + [_vp] * 6),
                ("swr_paged_attention", ctypes.c_int, [P(SwrPaged)] + [_vp] * 9),
                ("swr_paged_workspace_bytes", _i64, [P(SwrPaged)])):
            entry = getattr(lib, name)
            entry.restype, entry.argtypes = restype, args
        _bound = lib
    return lib


# The entry points that the native marshalling calls, in its order.
_BOUND = ("swr_rms_norm", "swr_rms_norm_workspace_bytes", "swr_rms_norm_backward", "swr_fp4_linear",
          "swr_block_tables", "swr_cache_append", "swr_paged_workspace_bytes", "swr_paged_attention")
_native = None   # (the package's native marshalling, the library that it is bound to)


def _fast():
    """The native marshalling, bound to the loaded library's entry points."""
    global _native
    module = _package._fast()
    if _native is None or _native[0] is not module or _native[1] is not _bound:
        lib = _lib()
        module.bind_hybrid(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _BOUND))
        _native = (module, lib)
    return module


def _check(rc, what):
    if rc < 0:
        raise SwrError(int(rc), what)
    return rc


def _code(t, what, fp8=False):
    torch = _torch()
    if t.dtype == torch.bfloat16:
        return SWR_DTYPE_BF16
    if t.dtype == torch.float32:
        return SWR_DTYPE_F32
    if fp8 and t.dtype == torch.float8_e4m3fn:
        return SWR_DTYPE_FP8
    raise TypeError(f"{what}: unsupported dtype {t.dtype}")


def _gpu(t, what):
    # The kernels dereference every pointer on the GPU: a host tensor would be
    # a memory fault, not an error, so it is refused here.
    if not t.is_cuda:
        raise ValueError(f"{what} must be a GPU tensor")


def _like(t, what, shape, dtype, device, contiguous=False):
    if tuple(t.shape) != tuple(shape) or t.dtype != dtype or t.device != device:
        raise ValueError(f"{what} must be a {dtype} tensor of shape {tuple(shape)} on {device}")
    if contiguous and not t.is_contiguous():
        raise ValueError(f"{what} must be contiguous")
    return t


def _workspace(nbytes, workspace, device, stream):
    if workspace is None:
        with _on(stream, device):
            return _torch().empty(max(nbytes // 4, 4), dtype=_torch().float32, device=device)
    if (workspace.numel() * workspace.element_size() < nbytes or not workspace.is_contiguous()
            or workspace.device != device):
        raise ValueError(f"workspace must be a contiguous tensor of at least {nbytes} bytes on the inputs' device")
    return workspace


# ----------------------------------------------------------------------------- norm


def _rows(t, what):
    """(outer, inner, strides) of a tensor's rows, [.., width] with contiguous
    channels; more leading dimensions have to be one by their strides."""
    if t.dim() < 1:
        raise ValueError(f"{what} must have a dimension")
    if t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"the last dimension of {what} must be contiguous")
    if t.dim() == 1:
        return 1, 1, (0, 0)
    if t.dim() == 2:
        return 1, t.shape[0], (0, t.stride(0))
    outer, so = t.shape[0], t.stride(0)
    inner, si = t.shape[-2], t.stride(-2)
    for i in range(t.dim() - 3, 0, -1):
        if t.shape[i] != 1 and inner > 1 and t.stride(i) != inner * si:
            raise ValueError(f"the leading dimensions of {what} must be a batch and a run of equally spaced rows")
        if inner == 1:
            si = t.stride(i)
        inner *= t.shape[i]
    return outer, inner, (so, si)


def _norm(x, weight, eps, out_dtype):
    _gpu(x, "x")
    dtype = _code(x, "x")
    outer, inner, (so, si) = _rows(x, "x")
    if tuple(weight.shape) != (x.shape[-1],) or weight.device != x.device:
        raise ValueError(f"weight must have shape {(x.shape[-1],)} and x's device")
    if not weight.is_contiguous():
        raise ValueError("weight must be contiguous")
    n = SwrNorm()
    n.abi_version, n.dtype, n.weight_dtype = SWR_ABI_VERSION, dtype, _code(weight, "weight")
    n.out_dtype = dtype if out_dtype is None else out_dtype
    n.outer, n.inner, n.width, n.eps = outer, inner, x.shape[-1], float(eps)
    n.sx_o, n.sx_i = so, si
    return n


def _same(x, t, what, dtype=None):
    """t's row strides; it has x's shape and device, and x's dtype or `dtype`."""
    _like(t, what, x.shape, dtype or x.dtype, x.device)
    return _rows(t, what)[2]


def swr_rms_norm(x, weight, residual=None, eps=1e-6, fp8=False, y=None, h=None, stream=None):
    """Residual addition and root-mean-square norm of rows x [.., width] (see
    ``include/swr_hybrid.h``): h = x + residual, y = h / rms(h) * weight.

    Returns y; with a ``residual`` (or an ``h`` to fill) (y, h); with ``fp8``, y is a
    ``float8_e4m3fn`` tensor q followed by its rows' float32 scales: (q, scale)
    or (q, scale, h).  ``h`` may be x or residual itself (updated in place)."""
    if y is None and h is None:
        r = _fast().rms_norm(x, weight, residual, eps, bool(fp8), _raw(stream))
        if r is not None:
            y, scale, h = _checked(r, "swr_rms_norm")
            if h is None:
                return (y, scale) if fp8 else y
            return (y, scale, h) if fp8 else (y, h)
    torch = _torch()
    n = _norm(x, weight, eps, SWR_DTYPE_FP8 if fp8 else None)
    if residual is not None:
        n.sr_o, n.sr_i = _same(x, residual, "residual")
    want_h = residual is not None or h is not None
    out = torch.float8_e4m3fn if fp8 else x.dtype
    if y is None:
        y = torch.empty(x.shape, dtype=out, device=x.device)
    n.sy_o, n.sy_i = _same(x, y, "y", out)
    if want_h:
        if h is None:
            h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        n.sh_o, n.sh_i = _same(x, h, "h")
    scale = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device) if fp8 else None
    _check(_lib().swr_rms_norm(ctypes.byref(n), _ptr(x), _opt(residual), _ptr(weight), _ptr(y), _opt(scale), _opt(h),
                               _stream(stream, x.device)), "swr_rms_norm")
    r = (y,) + ((scale,) if fp8 else ()) + ((h,) if want_h else ())
    return r[0] if len(r) == 1 else r


def swr_rms_norm_backward(h, weight, dy, dh=None, eps=1e-6, dx=None, dweight=None, workspace=None, stream=None):
    """(dx, dweight) of ``swr_rms_norm`` at its sum h, given dy and the gradient
    dh (or None) that reaches h on its other ways.  dx is the gradient of x and of the
    residual alike (it may be dy or dh itself); dweight is float32."""
    if dx is None and dweight is None and workspace is None:
        r = _fast().rms_norm_backward(h, weight, dy, dh, eps, _raw(stream))
        if r is not None:
            return _checked(r, "swr_rms_norm_backward")
    torch = _torch()
    n = _norm(h, weight, eps, None)
    n.sy_o, n.sy_i = _same(h, dy, "dy")
    if dh is not None:
        n.sr_o, n.sr_i = _same(h, dh, "dh")
    if dx is None:
        dx = torch.empty(h.shape, dtype=h.dtype, device=h.device)
    n.sh_o, n.sh_i = _same(h, dx, "dx")
    if dweight is None:
        dweight = torch.empty(weight.shape, dtype=torch.float32, device=h.device)
    _like(dweight, "dweight", weight.shape, torch.float32, h.device, contiguous=True)
    lib = _lib()
    nbytes = _check(lib.swr_rms_norm_workspace_bytes(ctypes.byref(n)), "swr_rms_norm_workspace_bytes")
    workspace = _workspace(nbytes, workspace, h.device, stream)
    _check(lib.swr_rms_norm_backward(ctypes.byref(n), _ptr(h), _ptr(weight), _ptr(dy), _opt(dh), _ptr(dx),
                                     _ptr(dweight), _ptr(workspace), _stream(stream, h.device)),
           "swr_rms_norm_backward")
    return dx, dweight


# ----------------------------------------------------------------------------- 4-bit weights


def _matrix(t, what):
    if t.dim() != 2 or (t.stride(1) != 1 and t.shape[1] > 1):
        raise ValueError(f"{what} must be a matrix with contiguous rows")
    return t.stride(0)


def swr_fp4_pack(w, codes=None, powers=None, stream=None):
    """(codes, powers) of a weight matrix w [N, K] (see ``include/swr_hybrid.h``):
    uint8 tensors [N, 16 ceil(K / 32)] and [N, ceil(K / 32)]."""
    torch = _torch()
    _gpu(w, "w")
    p = SwrFp4()
    p.abi_version, p.dtype, p.sx = SWR_ABI_VERSION, _code(w, "w"), _matrix(w, "w")
    p.N, p.K = w.shape
    groups = -(-p.K // FP4_GROUP)
    if codes is None:
        codes = torch.empty((p.N, 16 * groups), dtype=torch.uint8, device=w.device)
    if powers is None:
        powers = torch.empty((p.N, groups), dtype=torch.uint8, device=w.device)
    p.sc = _matrix(_like(codes, "codes", (p.N, 16 * groups), torch.uint8, w.device), "codes")
    p.sp = _matrix(_like(powers, "powers", (p.N, groups), torch.uint8, w.device), "powers")
    _check(_lib().swr_fp4_pack(ctypes.byref(p), _ptr(w), _ptr(codes), _ptr(powers), _stream(stream, w.device)),
           "swr_fp4_pack")
    return codes, powers


def swr_fp4_linear(x, codes, powers, scale=None, out_dtype=None, y=None, stream=None):
    """y = x W^T of rows x [.., K] (float32, bfloat16, or ``float8_e4m3fn``) with
    packed weights W [N, K], times ``scale`` [..] (float32, a factor per row)
    where given.  y is in ``out_dtype``: x's by default, bfloat16 for 8-bit rows."""
    if y is None and out_dtype is None:
        r = _fast().fp4_linear(x, codes, powers, scale, _raw(stream))
        if r is not None:
            return _checked(r, "swr_fp4_linear")
    torch = _torch()
    _gpu(x, "x")
    p = SwrFp4()
    p.abi_version, p.dtype = SWR_ABI_VERSION, _code(x, "x", fp8=True)
    outer, inner, (so, si) = _rows(x, "x")
    if outer > 1 and inner > 1 and so != inner * si:
        raise ValueError("the rows of x must be equally spaced")
    p.M, p.K, p.sx = outer * inner, x.shape[-1], si if inner > 1 else so
    if codes.dim() != 2 or powers.dim() != 2:
        raise ValueError("codes and powers must be matrices")
    p.N, groups = codes.shape[0], -(-p.K // FP4_GROUP)
    p.sc = _matrix(_like(codes, "codes", (p.N, 16 * groups), torch.uint8, x.device), "codes")
    p.sp = _matrix(_like(powers, "powers", (p.N, groups), torch.uint8, x.device), "powers")
    if scale is not None:
        _like(scale, "scale", x.shape[:-1], torch.float32, x.device, contiguous=True)
    shape = (*x.shape[:-1], p.N)
    if y is None:
        if out_dtype is None:
            out_dtype = torch.bfloat16 if p.dtype == SWR_DTYPE_FP8 else x.dtype
        y = torch.empty(shape, dtype=out_dtype, device=x.device)
    _like(y, "y", shape, y.dtype if out_dtype is None else out_dtype, x.device)
    p.out_dtype = _code(y, "y")
    yo, yi, (to, ti) = _rows(y, "y")
    if yo > 1 and yi > 1 and to != yi * ti:
        raise ValueError("the rows of y must be equally spaced")
    p.sy = ti if yi > 1 else to
    _check(_lib().swr_fp4_linear(ctypes.byref(p), _ptr(x), _opt(scale), _ptr(codes), _ptr(powers), _ptr(y),
                                 _stream(stream, x.device)), "swr_fp4_linear")
    return y


# ----------------------------------------------------------------------------- paged cache


def swr_block_tables(lengths, new_tokens, block_table, free_stack, free_count, page_size, tokens, slots=None,
                     starts=None, new_lengths=None, new_free_count=None, stream=None):
    """A step's tables from the requests' lengths (see ``include/swr_hybrid.h``):
    pages for ``new_tokens`` [batch] more tokens a request are taken from the
    top of ``free_stack`` and entered into ``block_table`` [batch, max_pages] in
    place (all int32).  Returns (slots, starts, new_lengths, new_free_count):
    the new tokens' slots in the cache (int64 [tokens]; -1 for none), the first
    of each request's (int32 [batch + 1]), the requests' new lengths, and the
    free pages left.  ``tokens`` is the number of new tokens, or a bound on it."""
    if slots is None and starts is None and new_lengths is None and new_free_count is None:
        r = _fast().block_tables(lengths, new_tokens, block_table, free_stack, free_count, page_size, tokens,
                                 _raw(stream))
        if r is not None:
            return _checked(r, "swr_block_tables")
    torch = _torch()
    i32 = torch.int32
    _gpu(lengths, "lengths")
    dev, batch = lengths.device, lengths.shape[0] if lengths.dim() == 1 else -1
    _like(lengths, "lengths", (batch,), i32, dev, contiguous=True)
    _like(new_tokens, "new_tokens", (batch,), i32, dev, contiguous=True)
    if free_stack.dim() != 1 or block_table.dim() != 2:
        raise ValueError("free_stack must have one dimension, block_table two")
    _like(free_stack, "free_stack", free_stack.shape, i32, dev, contiguous=True)
    _like(free_count, "free_count", (1,), i32, dev)
    p = SwrTables()
    p.abi_version, p.batch, p.max_pages, p.tokens = SWR_ABI_VERSION, batch, block_table.shape[1], int(tokens)
    p.page_size, p.free_pages = int(page_size), free_stack.shape[0]
    p.st = _matrix(_like(block_table, "block_table", (batch, p.max_pages), i32, dev), "block_table")
    if p.tokens < 0:
        raise ValueError("tokens must not be negative")

    def out(t, what, shape, dtype):
        if t is None:
            return torch.empty(shape, dtype=dtype, device=dev)
        return _like(t, what, shape, dtype, dev, contiguous=True)

    slots = out(slots, "slots", (p.tokens,), torch.int64)
    starts = out(starts, "starts", (batch + 1,), i32)
    new_lengths = out(new_lengths, "new_lengths", (batch,), i32)
    new_free_count = out(new_free_count, "new_free_count", (1,), i32)
    _check(_lib().swr_block_tables(ctypes.byref(p), _ptr(lengths), _ptr(new_tokens), _ptr(free_stack),
                                   _ptr(free_count), _ptr(block_table), _ptr(slots), _ptr(starts), _ptr(new_lengths),
                                   _ptr(new_free_count), _stream(stream, dev)), "swr_block_tables")
    return slots, starts, new_lengths, new_free_count


def _cache(c, k_cache, v_cache):
    _gpu(k_cache, "k_cache")
    if k_cache.dim() != 4:
        raise ValueError("k_cache must be [pages, page_size, heads, D]")
    _like(v_cache, "v_cache", k_cache.shape, k_cache.dtype, k_cache.device)
    if k_cache.stride() != v_cache.stride() or (k_cache.stride(3) != 1 and k_cache.shape[3] > 1):
        raise ValueError("k_cache and v_cache must have the same strides and contiguous channels")
    c.abi_version, c.dtype = SWR_ABI_VERSION, _code(k_cache, "k_cache")
    c.pages, c.page_size, c.heads, c.D = k_cache.shape
    c.s_page, c.s_token, c.s_head = k_cache.stride()[:3]


def _heads(t, what, shape, cache):
    _like(t, what, shape, cache.dtype, cache.device)
    if t.stride(2) != 1 and t.shape[2] > 1:
        raise ValueError(f"the channels of {what} must be contiguous")
    return t.stride(0), t.stride(1)


def swr_cache_append(k, v, k_cache, v_cache, slots, stream=None):
    """New keys and values, [tokens, heads, D], into their ``slots`` (int64
    [tokens]) of a layer's cache [pages, page_size, heads, D], in place.  A token
    whose slot is not within the cache is left out."""
    r = _fast().cache_append(k, v, k_cache, v_cache, slots, _raw(stream))
    if r is not None:
        _checked(r, "swr_cache_append")
        return
    torch = _torch()
    c = SwrCache()
    _cache(c, k_cache, v_cache)
    if slots.dim() != 1:
        raise ValueError("slots must have one dimension")
    tokens = slots.shape[0]
    _like(slots, "slots", (tokens,), torch.int64, k_cache.device, contiguous=True)
    sk = (_i64 * 2)(*_heads(k, "k", (tokens, c.heads, c.D), k_cache))
    sv = (_i64 * 2)(*_heads(v, "v", (tokens, c.heads, c.D), k_cache))
    _check(_lib().swr_cache_append(ctypes.byref(c), tokens, sk, sv, _ptr(k), _ptr(v), _ptr(slots), _ptr(k_cache),
                                   _ptr(v_cache), _stream(stream, k_cache.device)), "swr_cache_append")


def swr_paged_attention(q, k_cache, v_cache, block_table, lengths, scale=None, window=0, want_lse=False, y=None,
                        workspace=None, stream=None):
    """Attention of one query token a request, q [batch, q_heads, D], over its
    ``lengths`` [batch] cached tokens (see ``include/swr_hybrid.h``); the last ``window`` of them
    where that is not 0.  ``scale`` is 1 / sqrt(D) by default.  Returns y, or
    (y, lse) with the logarithms of the softmax sums, float32 [batch, q_heads]."""
    if y is None and workspace is None and q.dim() == 3:
        r = _fast().paged_attention(q, k_cache, v_cache, block_table, lengths,
                                    q.shape[2] ** -0.5 if scale is None else scale, window, bool(want_lse),
                                    _raw(stream))
        if r is not None:
            y, lse = _checked(r, "swr_paged_attention")
            return (y, lse) if want_lse else y
    torch = _torch()
    p = SwrPaged()
    _cache(p.cache, k_cache, v_cache)
    if q.dim() != 3 or block_table.dim() != 2:
        raise ValueError("q must be [batch, q_heads, D] and block_table [batch, max_pages]")
    p.batch, p.q_heads = q.shape[:2]
    if p.q_heads < 1 or p.q_heads % max(p.cache.heads, 1) != 0:
        raise ValueError("q_heads must be a multiple of the cache's heads")
    p.sq_b, p.sq_h = _heads(q, "q", (p.batch, p.q_heads, p.cache.D), k_cache)
    if y is None:
        y = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    p.sy_b, p.sy_h = _heads(y, "y", q.shape, k_cache)
    p.max_pages = block_table.shape[1]
    p.st = _matrix(_like(block_table, "block_table", (p.batch, p.max_pages), torch.int32, q.device), "block_table")
    _like(lengths, "lengths", (p.batch,), torch.int32, q.device, contiguous=True)
    p.window = int(window)
    p.scale = p.cache.D ** -0.5 if scale is None else float(scale)
    if not math.isfinite(p.scale):
        raise ValueError("scale must be finite")
    lse = torch.empty((p.batch, p.q_heads), dtype=torch.float32, device=q.device) if want_lse else None
    lib = _lib()
    nbytes = _check(lib.swr_paged_workspace_bytes(ctypes.byref(p)), "swr_paged_workspace_bytes")
    workspace = _workspace(nbytes, workspace, q.device, stream)
    _check(lib.swr_paged_attention(ctypes.byref(p), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
                                   _ptr(lengths), _ptr(y), _opt(lse), _ptr(workspace), _stream(stream, q.device)),
           "swr_paged_attention")
    return (y, lse) if want_lse else y


# ----------------------------------------------------------------------------- autograd


def _as_rows(g):
    """A gradient as it comes, or a copy where the calls cannot take its layout (an
    expanded or a transposed one)."""
    try:
        _rows(g, "gradient")
    except ValueError:
        return g.contiguous()
    return g


def _autograd_function():
    torch = _torch()

    class _SWRNormFunction(torch.autograd.Function):
        """Autograd wrapper of the norm with its residual: (y, h) of (x, weight,
        residual, eps); only h and the weight are kept for the backward.  Without a
        residual (None) h is x."""

        @staticmethod
        def forward(ctx, x, weight, residual, eps=1e-6):
            if residual is None:
                y, h = swr_rms_norm(x, weight, eps=eps), x
            else:
                y, h = swr_rms_norm(x, weight, residual=residual, eps=eps)
            ctx.eps, ctx.has_residual = eps, residual is not None
            ctx.save_for_backward(h, weight)
            return y, h

        @staticmethod
        def backward(ctx, dy, dh):
            h, weight = ctx.saved_tensors
            dx, dw = swr_rms_norm_backward(h, weight, _as_rows(dy), dh=_as_rows(dh), eps=ctx.eps)
            return dx, dw.to(weight.dtype), dx if ctx.has_residual else None, None

    return _SWRNormFunction


_function = None


def __getattr__(name):
    global _function
    if name == "SWRNormFunction":
        if _function is None:
            _function = _autograd_function()
        return _function
    raise AttributeError(name)
