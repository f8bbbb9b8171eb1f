"""Operators of a recurrent language model around the recurrence, its norms and
projections: binding of ``include/swr_lm.h``.

The embedding of tokens (``swr_embedding``), the short causal convolution
(``swr_causal_conv``) and the selective state space scan (``swr_selective_scan``) of
a mixer, and the log probabilities of given tokens (``swr_log_probs``), with their
gradients and, for the mixer, their forms for single tokens.  The functions marshal
torch tensors into pointers, strides and the current HIP stream, the ordinary call
in native code (``csrc/swr_binding.cpp``); every step of the computation runs in
the library's HIP kernels.  There is no CPU fallback.
"""
import ctypes
import math

import paper_2512_13921_amd as _package

from . import (SWR_ABI_VERSION, SWR_DTYPE_BF16, SWR_DTYPE_F32, _checked, _on, _opt, _ptr, _raw, _stream, _torch, load)
from .hybrid import _check, _code, _gpu, _like, _rows, _workspace

__all__ = ["swr_embedding", "swr_embedding_backward", "swr_causal_conv", "swr_causal_conv_step",
           "swr_causal_conv_backward", "swr_selective_scan", "swr_selective_step", "swr_selective_scan_backward",
           "swr_log_probs", "swr_log_probs_backward", "SWREmbeddingFunction", "SWRCausalConvFunction",
           "SWRSelectiveScanFunction", "SWRLogProbsFunction"]

SWR_CONV_SILU = 1
SWR_SCAN_SOFTPLUS = 1
SWR_SCAN_BLOCK = 16
SWR_TOP_MOST = 64

_i32, _u32, _i64, _f32, _vp = ctypes.c_int32, ctypes.c_uint32, ctypes.c_int64, ctypes.c_float, ctypes.c_void_p


class SwrEmbed(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("out_dtype", _i32), ("token_bytes", _i32),
                ("tokens", _i64), ("vocab", _i64), ("width", _i64), ("st", _i64), ("sy", _i64), ("scale", _f32),
                ("reserved", _i32)]


class SwrConv(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("flags", _u32), ("taps", _i32), ("B", _i64), ("T", _i64),
                ("C", _i64), ("sx_b", _i64), ("sx_t", _i64), ("sy_b", _i64), ("sy_t", _i64), ("sd_b", _i64),
                ("sd_t", _i64)]


class SwrScan(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("flags", _u32), ("N", _i32), ("B", _i64), ("T", _i64),
                ("D", _i64), ("G", _i64), ("sx_b", _i64), ("sx_t", _i64), ("sdt_b", _i64), ("sdt_t", _i64),
                ("sz_b", _i64), ("sz_t", _i64), ("sy_b", _i64), ("sy_t", _i64), ("sB_b", _i64), ("sB_t", _i64),
                ("sB_g", _i64), ("sC_b", _i64), ("sC_t", _i64), ("sC_g", _i64)]


class SwrScanInputs(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("x", "dt", "A", "B", "C", "bias", "skip", "z", "h0", "lengths")]


class SwrScanGradients(ctypes.Structure):
    _fields_ = [(n, _vp) for n in ("dx", "ddt", "dA", "dB", "dC", "dbias", "dskip", "dz", "dh0")]


class SwrLogProb(ctypes.Structure):
    _fields_ = [("abi_version", _i32), ("dtype", _i32), ("token_bytes", _i32), ("top", _i32), ("rows", _i64),
                ("vocab", _i64), ("sl", _i64), ("sd", _i64), ("scale", _f32), ("reserved", _i32)]


_bound = None


def _lib():
    """The loaded library, with the argument types of this header's calls."""
    global _bound
    lib = load()
    if _bound is not lib:
        P, i32 = ctypes.POINTER, ctypes.c_int
        for name, restype, args in (
                ("swr_embedding", i32, [P(SwrEmbed)] + [_vp] * 4),
                ("swr_embedding_workspace_bytes", _i64, [P(SwrEmbed)]),
                ("swr_embedding_backward", i32, [P(SwrEmbed)] + [_vp] * 5),
                ("swr_causal_conv", i32, [P(SwrConv)] + [_vp] * 8),
                ("swr_causal_conv_workspace_bytes", _i64, [P(SwrConv)]),
                ("swr_causal_conv_backward", i32, [P(SwrConv)] + [_vp] * 10),
                ("swr_selective_scan", i32, [P(SwrScan), P(SwrScanInputs)] + [_vp] * 5),
                ("swr_selective_scan_workspace_bytes", _i64, [P(SwrScan)]),
                ("swr_selective_scan_backward", i32, [P(SwrScan), P(SwrScanInputs)] + [_vp] * 3 +
                 [P(SwrScanGradients)] + [_vp] * 2),
                ("swr_selective_scan_backward_workspace_bytes", _i64, [P(SwrScan)]),
                ("swr_log_probs", i32, [P(SwrLogProb)] + [_vp] * 9),
                ("swr_log_probs_workspace_bytes", _i64, [P(SwrLogProb)]),
                ("swr_log_probs_backward", i32, [P(SwrLogProb)] + [_vp] * 9)):
            entry = getattr(lib, name)
            entry.restype, entry.argtypes = restype, args
        _bound = lib
    return lib


# The entry points that the native marshalling calls, in its order.
_BOUND = ("swr_embedding", "swr_embedding_workspace_bytes", "swr_embedding_backward", "swr_causal_conv",
          "swr_causal_conv_workspace_bytes", "swr_causal_conv_backward", "swr_selective_scan",
          "swr_selective_scan_workspace_bytes", "swr_selective_scan_backward",
          "swr_selective_scan_backward_workspace_bytes", "swr_log_probs", "swr_log_probs_workspace_bytes",
          "swr_log_probs_backward")
_native = None   # (the package's native marshalling, the library that it is bound to)


def _fast():
    """The native marshalling, bound to the loaded library's entry points."""
    global _native
    module = _package._fast()
    if _native is None or _native[0] is not module or _native[1] is not _bound:
        lib = _lib()
        module.bind_lm(*(ctypes.cast(getattr(lib, n), ctypes.c_void_p).value for n in _BOUND))
        _native = (module, lib)
    return _native[0]


def _even_rows(t, what):
    """(rows, row stride) of a tensor [.., width] whose rows are equally spaced."""
    outer, inner, (so, si) = _rows(t, what)
    if outer > 1 and inner > 1 and so != inner * si:
        raise ValueError(f"the rows of {what} must be equally spaced")
    return outer * inner, si if inner > 1 else so


def _tokens(tokens, shape, device):
    """A token's bytes; tokens is an int32 or int64 tensor of the shape."""
    torch = _torch()
    if tokens.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"tokens: unsupported dtype {tokens.dtype} (int32 or int64)")
    _like(tokens, "tokens", shape, tokens.dtype, device, contiguous=True)
    return 4 if tokens.dtype == torch.int32 else 8


def _finite(v, what):
    v = float(v)
    if not math.isfinite(v):
        raise ValueError(f"{what} must be finite")
    return v


def _lengths(lengths, batch, device):
    if lengths is not None:
        _like(lengths, "lengths", (batch,), _torch().int32, device, contiguous=True)
    return lengths


def _vector(t, what, n, dtype, device):
    if t is not None:
        _like(t, what, (n,), dtype, device, contiguous=True)
    return t


# ----------------------------------------------------------------------------- embedding


def _embed(tokens, rows, vocab, scale, what):
    e = SwrEmbed()
    e.abi_version, e.dtype = SWR_ABI_VERSION, _code(rows, what)
    e.out_dtype = e.dtype
    e.tokens, e.vocab, e.width = tokens.numel(), vocab, rows.shape[-1]
    e.scale = _finite(scale, "scale")
    return e


def swr_embedding(tokens, table, scale=1.0, y=None, stream=None):
    """Rows of a table [vocab, width] for tokens [..] (int32 or int64), times ``scale``:
    y [.., width].  A token outside the table (padding) has a row of zeros."""
    if y is None:
        r = _fast().embedding(tokens, table, scale, _raw(stream))
        if r is not None:
            return _checked(r, "swr_embedding")
    torch = _torch()
    _gpu(table, "table")
    if table.dim() != 2 or (table.stride(1) != 1 and table.shape[1] > 1):
        raise ValueError("table must be a matrix with contiguous rows")
    e = _embed(tokens, table, table.shape[0], scale, "table")
    e.token_bytes, e.st = _tokens(tokens, tokens.shape, table.device), table.stride(0)
    shape = (*tokens.shape, e.width)
    if y is None:
        y = torch.empty(shape, dtype=table.dtype, device=table.device)
    _, e.sy = _even_rows(_like(y, "y", shape, table.dtype, table.device), "y")
    _check(_lib().swr_embedding(ctypes.byref(e), _ptr(tokens), _ptr(table), _ptr(y), _stream(stream, table.device)),
           "swr_embedding")
    return y


def swr_embedding_backward(tokens, dy, vocab, scale=1.0, dtype=None, dtable=None, workspace=None, stream=None):
    """The table's gradient [vocab, width], of dy [.., width]: float32, or ``dtype`` (dy's)."""
    if dtable is None and workspace is None and dtype in (None, dy.dtype, _torch().float32):
        r = _fast().embedding_backward(tokens, dy, vocab, scale, dtype == dy.dtype, _raw(stream))
        if r is not None:
            return _checked(r, "swr_embedding_backward")
    torch = _torch()
    _gpu(dy, "dy")
    e = _embed(tokens, dy, int(vocab), scale, "dy")
    e.token_bytes = _tokens(tokens, dy.shape[:-1], dy.device)
    _, e.sy = _even_rows(dy, "dy")
    if dtable is None:
        dtable = torch.empty((e.vocab, e.width), dtype=dtype or torch.float32, device=dy.device)
    _like(dtable, "dtable", (e.vocab, e.width), dtable.dtype if dtype is None else dtype, dy.device)
    e.out_dtype, e.st = _code(dtable, "dtable"), dtable.stride(0)
    if dtable.stride(1) != 1 and e.width > 1:
        raise ValueError("dtable must be a matrix with contiguous rows")
    lib = _lib()
    nbytes = _check(lib.swr_embedding_workspace_bytes(ctypes.byref(e)), "swr_embedding_workspace_bytes")
    workspace = _workspace(nbytes, workspace, dy.device, stream)
    _check(lib.swr_embedding_backward(ctypes.byref(e), _ptr(tokens), _ptr(dy), _ptr(dtable), _ptr(workspace),
                                      _stream(stream, dy.device)), "swr_embedding_backward")
    return dtable


# ----------------------------------------------------------------------------- convolution


def _sequence(t, what, shape, dtype, device):
    """(batch, token) strides of a tensor [B, T, channels] with contiguous channels."""
    _like(t, what, shape, dtype, device)
    if t.stride(2) != 1 and t.shape[2] > 1:
        raise ValueError(f"the channels of {what} must be contiguous")
    return t.stride(0), t.stride(1)


def _conv(x, weight, bias, silu, lengths):
    _gpu(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be [B, T, channels]")
    p = SwrConv()
    p.abi_version, p.dtype, p.flags = SWR_ABI_VERSION, _code(x, "x"), SWR_CONV_SILU if silu else 0
    p.B, p.T, p.C = x.shape
    if weight.dim() != 2:
        raise ValueError("weight must be [channels, taps]")
    _like(weight, "weight", (p.C, weight.shape[1]), x.dtype, x.device, contiguous=True)
    p.taps = weight.shape[1]
    _vector(bias, "bias", p.C, x.dtype, x.device)
    _lengths(lengths, p.B, x.device)
    p.sx_b, p.sx_t = _sequence(x, "x", x.shape, x.dtype, x.device)
    return p


def swr_causal_conv(x, weight, bias=None, silu=True, state=None, lengths=None, state_out=None, want_state=False,
                    y=None, stream=None):
    """Depthwise causal convolution of x [B, T, channels] with weight [channels, taps] (1 to
    8 taps, the last of them the token's own), its SiLU where ``silu`` (see ``include/swr_lm.h``):
    (y, state).  ``state`` [B, taps - 1, channels] holds the tokens before; the new one
    is returned where ``want_state`` (None otherwise) or written to ``state_out`` (it may be ``state``).  ``lengths``
    [B] (int32): tokens of each batch; y is zero past them."""
    if y is None and state_out is None:
        r = _fast().causal_conv(x, weight, bias, bool(silu), state, lengths, bool(want_state), _raw(stream))
        if r is not None:
            return _checked(r, "swr_causal_conv")
    torch = _torch()
    p = _conv(x, weight, bias, silu, lengths)
    shape = (p.B, p.taps - 1, p.C)
    for t, what in ((state, "state"), (state_out, "state_out")):
        if t is not None:
            _like(t, what, shape, x.dtype, x.device, contiguous=True)
    if want_state and state_out is None:
        state_out = torch.empty(shape, dtype=x.dtype, device=x.device)
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    p.sy_b, p.sy_t = _sequence(y, "y", x.shape, x.dtype, x.device)
    _check(_lib().swr_causal_conv(ctypes.byref(p), _ptr(x), _ptr(weight), _opt(bias), _opt(state), _opt(lengths),
                                  _ptr(y), _opt(state_out), _stream(stream, x.device)), "swr_causal_conv")
    return y, state_out


def swr_causal_conv_step(x, weight, state, bias=None, silu=True, y=None, stream=None):
    """The convolution of one more token a request, x [B, channels]: y [B, channels].  ``state``
    [B, taps - 1, channels] is updated in place."""
    if y is None:
        r = _fast().causal_conv_step(x, weight, state, bias, bool(silu), _raw(stream))
        if r is not None:
            return _checked(r, "swr_causal_conv_step")
    if x.dim() != 2:
        raise ValueError("x must be [B, channels]")
    if y is not None:
        _like(y, "y", x.shape, x.dtype, x.device)
    r, _ = swr_causal_conv(x[:, None], weight, bias, silu, state, state_out=state,
                           y=None if y is None else y[:, None], stream=stream)
    return r[:, 0] if y is None else y


def swr_causal_conv_backward(x, weight, dy, bias=None, silu=True, lengths=None, dx=None, dweight=None, dbias=None,
                             workspace=None, stream=None):
    """(dx, dweight, dbias) of ``swr_causal_conv`` without a state; dweight [channels, taps] and
    dbias [channels] (None without a bias) are float32."""
    if dx is None and dweight is None and dbias is None and workspace is None:
        r = _fast().causal_conv_backward(x, weight, dy, bias, bool(silu), lengths, _raw(stream))
        if r is not None:
            return _checked(r, "swr_causal_conv_backward")
    torch = _torch()
    p = _conv(x, weight, bias, silu, lengths)
    p.sy_b, p.sy_t = _sequence(dy, "dy", x.shape, x.dtype, x.device)
    if dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    p.sd_b, p.sd_t = _sequence(dx, "dx", x.shape, x.dtype, x.device)
    f32 = dict(dtype=torch.float32, device=x.device)
    if dweight is None:
        dweight = torch.empty((p.C, p.taps), **f32)
    _like(dweight, "dweight", (p.C, p.taps), torch.float32, x.device, contiguous=True)
    if dbias is None and bias is not None:
        dbias = torch.empty((p.C,), **f32)
    _vector(dbias, "dbias", p.C, torch.float32, x.device)
    lib = _lib()
    nbytes = _check(lib.swr_causal_conv_workspace_bytes(ctypes.byref(p)), "swr_causal_conv_workspace_bytes")
    workspace = _workspace(nbytes, workspace, x.device, stream)
    _check(lib.swr_causal_conv_backward(ctypes.byref(p), _ptr(x), _ptr(weight), _opt(bias), _ptr(dy), _opt(lengths),
                                        _ptr(dx), _ptr(dweight), _opt(dbias), _ptr(workspace),
                                        _stream(stream, x.device)), "swr_causal_conv_backward")
    return dx, dweight, dbias


# ----------------------------------------------------------------------------- scan


def _scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, lengths):
    """The problem and its inputs; B and C may leave out their groups, [B, T, N]."""
    torch = _torch()
    _gpu(x, "x")
    if x.dim() != 3:
        raise ValueError("x must be [B, T, channels]")
    if A.dim() != 2:
        raise ValueError("A must be [channels, states]")
    p, q = SwrScan(), SwrScanInputs()
    p.abi_version, p.dtype, p.flags = SWR_ABI_VERSION, _code(x, "x"), SWR_SCAN_SOFTPLUS if softplus else 0
    p.B, p.T, p.D = x.shape
    p.N = A.shape[1]
    f32, dev = torch.float32, x.device
    _like(A, "A", (p.D, p.N), f32, dev, contiguous=True)
    p.sx_b, p.sx_t = _sequence(x, "x", x.shape, x.dtype, dev)
    p.sdt_b, p.sdt_t = _sequence(dt, "dt", x.shape, x.dtype, dev)
    if z is not None:
        p.sz_b, p.sz_t = _sequence(z, "z", x.shape, x.dtype, dev)
    if B.dim() not in (3, 4) or B.dim() != C.dim():
        raise ValueError("B and C must be [B, T, groups, states] or [B, T, states]")
    p.G = B.shape[2] if B.dim() == 4 else 1
    strides = []
    for t, what in ((B, "B"), (C, "C")):
        _like(t, what, (p.B, p.T, p.G, p.N) if B.dim() == 4 else (p.B, p.T, p.N), x.dtype, dev)
        if t.stride(-1) != 1 and p.N > 1:
            raise ValueError(f"the states of {what} must be contiguous")
        strides += [t.stride(0), t.stride(1), t.stride(2) if B.dim() == 4 else 0]
    if p.G < 1 or p.D % p.G != 0:
        raise ValueError("the groups of B and C must divide the channels")
    p.sB_b, p.sB_t, p.sB_g, p.sC_b, p.sC_t, p.sC_g = strides
    _vector(D, "D", p.D, f32, dev)
    _vector(dt_bias, "dt_bias", p.D, f32, dev)
    if h0 is not None:
        _like(h0, "h0", (p.B, p.D, p.N), f32, dev, contiguous=True)
    _lengths(lengths, p.B, dev)
    for name, t in (("x", x), ("dt", dt), ("A", A), ("B", B), ("C", C), ("bias", dt_bias), ("skip", D), ("z", z),
                    ("h0", h0), ("lengths", lengths)):
        setattr(q, name, None if t is None else t.data_ptr())
    return p, q


def _carriers(p, device, carriers=None):
    torch = _torch()
    shape = (p.B, -(-p.T // SWR_SCAN_BLOCK), p.D, p.N)
    if carriers is None:
        return torch.empty(shape, dtype=torch.float32, device=device)
    return _like(carriers, "carriers", shape, torch.float32, device, contiguous=True)


def swr_selective_scan(x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, h0=None, lengths=None,
                       save_carriers=False, want_state=False, h_last=None, y=None, workspace=None, stream=None):
    """Selective state space scan (see ``include/swr_lm.h``): (y, carriers, h_last).

    x, dt and z are [B, T, channels], A [channels, states] (float32, 1 to 64 states),
    B and C [B, T, groups, states] (or without the groups), D and dt_bias [channels]
    (float32).  ``h0`` and the final state are float32 [B, channels, states]; the final state is
    returned where ``want_state`` (None otherwise) or written to ``h_last`` (it may be ``h0``).  ``lengths`` [B]
    (int32): tokens of each batch; y is zero past them.  ``save_carriers``: the states that the
    backward starts from (None otherwise)."""
    if y is None and workspace is None and h_last is None:
        r = _fast().selective_scan(x, dt, A, B, C, D, z, dt_bias, bool(softplus), h0, lengths, bool(save_carriers),
                                   bool(want_state), _raw(stream))
        if r is not None:
            return _checked(r, "swr_selective_scan")
    torch = _torch()
    p, q = _scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, lengths)
    if y is None:
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    p.sy_b, p.sy_t = _sequence(y, "y", x.shape, x.dtype, x.device)
    carriers = _carriers(p, x.device) if save_carriers else None
    if want_state and h_last is None:
        h_last = torch.empty((p.B, p.D, p.N), dtype=torch.float32, device=x.device)
    if h_last is not None:
        _like(h_last, "h_last", (p.B, p.D, p.N), torch.float32, x.device, contiguous=True)
    lib = _lib()
    nbytes = _check(lib.swr_selective_scan_workspace_bytes(ctypes.byref(p)), "swr_selective_scan_workspace_bytes")
    workspace = _workspace(nbytes, workspace, x.device, stream)
    _check(lib.swr_selective_scan(ctypes.byref(p), ctypes.byref(q), _ptr(y), _opt(carriers), _opt(h_last),
                                  _ptr(workspace), _stream(stream, x.device)), "swr_selective_scan")
    return y, carriers, h_last


def swr_selective_step(x, dt, A, B, C, state, D=None, z=None, dt_bias=None, softplus=True, y=None, stream=None):
    """The scan of one more token a request, x, dt and z [B, channels], B and C [B, groups, states]
    (or without the groups): y [B, channels].  ``state`` [B, channels, states] (float32) is updated in place."""
    if y is None:
        r = _fast().selective_step(x, dt, A, B, C, state, D, z, dt_bias, bool(softplus), _raw(stream))
        if r is not None:
            return _checked(r, "swr_selective_step")
    if x.dim() != 2 or B.dim() not in (2, 3):
        raise ValueError("x must be [B, channels], B and C [B, groups, states] or [B, states]")
    if y is not None:
        _like(y, "y", x.shape, x.dtype, x.device)

    def token(t):
        return None if t is None else t[:, None]

    r, _, _ = swr_selective_scan(token(x), token(dt), A, token(B), token(C), D, token(z), dt_bias, softplus, state,
                                 h_last=state, y=token(y), stream=stream)
    return r[:, 0] if y is None else y


def swr_selective_scan_backward(x, dt, A, B, C, dy, carriers, D=None, z=None, dt_bias=None, softplus=True, h0=None,
                                dh_last=None, lengths=None, want_dh0=False, workspace=None, stream=None):
    """Gradients of ``swr_selective_scan``, of dy and of the final state's ``dh_last``:
    (dx, ddt, dA, dB, dC, dD, dz, ddt_bias, dh0), None for what is not there (dh0:
    unless ``want_dh0``).  ``carriers`` are the forward's, or None: they are computed anew.  Those of float32
    inputs are float32, the others of x's dtype."""
    if carriers is not None and workspace is None:
        r = _fast().selective_scan_backward(x, dt, A, B, C, dy, carriers, D, z, dt_bias, bool(softplus), dh_last,
                                            lengths, bool(want_dh0), _raw(stream))
        if r is not None:
            return _checked(r, "swr_selective_scan_backward")
    torch = _torch()
    p, q = _scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, lengths)
    dev, lib = x.device, _lib()
    if carriers is None:
        with _on(stream, dev):   # (let go when this call returns)
            _, carriers, _ = swr_selective_scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, lengths,
                                                save_carriers=True, stream=stream)
    carriers = _carriers(p, dev, carriers)
    p.sy_b, p.sy_t = _sequence(dy, "dy", x.shape, x.dtype, dev)
    if dh_last is not None:
        _like(dh_last, "dh_last", (p.B, p.D, p.N), torch.float32, dev, contiguous=True)

    def like(t, shape=None):
        return None if t is None else torch.empty(t.shape if shape is None else shape, dtype=t.dtype, device=dev)

    out = {"dx": like(x), "ddt": like(dt), "dA": like(A), "dB": like(B), "dC": like(C), "dskip": like(D),
           "dz": like(z), "dbias": like(dt_bias), "dh0": like(A, (p.B, p.D, p.N)) if want_dh0 else None}
    g = SwrScanGradients()
    for name, t in out.items():
        setattr(g, name, None if t is None else t.data_ptr())
    nbytes = _check(lib.swr_selective_scan_backward_workspace_bytes(ctypes.byref(p)),
                    "swr_selective_scan_backward_workspace_bytes")
    workspace = _workspace(nbytes, workspace, dev, stream)
    _check(lib.swr_selective_scan_backward(ctypes.byref(p), ctypes.byref(q), _ptr(dy), _ptr(carriers), _opt(dh_last),
                                           ctypes.byref(g), _ptr(workspace), _stream(stream, dev)),
           "swr_selective_scan_backward")
    return tuple(out.values())


# ----------------------------------------------------------------------------- log probabilities


def _log_probs(logits, tokens, top, scale):
    _gpu(logits, "logits")
    p = SwrLogProb()
    p.abi_version, p.dtype, p.top = SWR_ABI_VERSION, _code(logits, "logits"), int(top)
    p.rows, p.sl = _even_rows(logits, "logits")
    p.vocab = logits.shape[-1]
    p.token_bytes = _tokens(tokens, logits.shape[:-1], logits.device)
    p.scale = _finite(scale, "scale")
    if not 0 <= p.top <= min(SWR_TOP_MOST, p.vocab):
        raise ValueError(f"top must be between 0 and {SWR_TOP_MOST}, and no more than the vocabulary")
    return p


def swr_log_probs(logits, tokens, top=0, scale=1.0, workspace=None, stream=None):
    """Log probabilities of tokens [..] under softmax(scale logits), logits [.., vocab] (see
    ``include/swr_lm.h``): (logp, lse, entropy), float32 [..]; with ``top``, the log probabilities
    and tokens (int64) of as many best alternatives [.., top] too.  A token outside the
    vocabulary (not scored) has logp 0."""
    if workspace is None:
        r = _fast().log_probs(logits, tokens, top, scale, _raw(stream))
        if r is not None:
            r = _checked(r, "swr_log_probs")
            return r if top else r[:3]
    torch = _torch()
    p = _log_probs(logits, tokens, top, scale)
    lead, dev = tuple(logits.shape[:-1]), logits.device
    out = [torch.empty(lead, dtype=torch.float32, device=dev) for _ in range(3)]
    best = ([torch.empty((*lead, p.top), dtype=t, device=dev) for t in (torch.float32, torch.int64)] if p.top
            else [None, None])
    lib = _lib()
    nbytes = _check(lib.swr_log_probs_workspace_bytes(ctypes.byref(p)), "swr_log_probs_workspace_bytes")
    workspace = _workspace(nbytes, workspace, dev, stream)
    _check(lib.swr_log_probs(ctypes.byref(p), _ptr(logits), _ptr(tokens), *map(_ptr, out), *map(_opt, best),
                             _ptr(workspace), _stream(stream, dev)), "swr_log_probs")
    return (*out, *best) if p.top else tuple(out)


def swr_log_probs_backward(logits, tokens, lse, entropy, dlogp=None, dentropy=None, dlse=None, scale=1.0, dlogits=None,
                           stream=None):
    """The logits' gradient, of the gradients of logp, of the entropy and of lse (each may be
    None); lse and entropy are the forward's.  ``dlogits`` may be the logits themselves."""
    if dlogits is None:
        r = _fast().log_probs_backward(logits, tokens, lse, entropy, dlogp, dentropy, dlse, scale, _raw(stream))
        if r is not None:
            return _checked(r, "swr_log_probs_backward")
    torch = _torch()
    p = _log_probs(logits, tokens, 0, scale)
    dev = logits.device
    for t, what in ((lse, "lse"), (entropy, "entropy"), (dlogp, "dlogp"), (dentropy, "dentropy"), (dlse, "dlse")):
        if t is not None:
            _like(t, what, logits.shape[:-1], torch.float32, dev, contiguous=True)
    if dlogits is None:
        dlogits = torch.empty(logits.shape, dtype=logits.dtype, device=dev)
    _, p.sd = _even_rows(_like(dlogits, "dlogits", logits.shape, logits.dtype, dev), "dlogits")
    _check(_lib().swr_log_probs_backward(ctypes.byref(p), _ptr(logits), _ptr(tokens), _ptr(lse), _ptr(entropy),
                                         _opt(dlogp), _opt(dlse), _opt(dentropy), _ptr(dlogits),
                                         _stream(stream, dev)), "swr_log_probs_backward")
    return dlogits


# ----------------------------------------------------------------------------- autograd


def _even(g):
    """A gradient as it comes, or a copy where the calls cannot take its layout."""
    try:
        _even_rows(g, "gradient")
    except ValueError:
        return g.contiguous()
    return g


def _channels(g):
    return g if g.stride(-1) == 1 or g.shape[-1] <= 1 else g.contiguous()


def _functions():
    torch = _torch()
    once = torch.autograd.function.once_differentiable   # (a second derivative is refused)

    class _SWREmbeddingFunction(torch.autograd.Function):
        """Autograd wrapper of the embedding: y of (tokens, table, scale); the table's gradient
        has the table's dtype."""

        @staticmethod
        def forward(ctx, tokens, table, scale=1.0):
            ctx.scale, ctx.vocab, ctx.dtype = scale, table.shape[0], table.dtype
            ctx.save_for_backward(tokens)
            return swr_embedding(tokens, table, scale)

        @staticmethod
        @once
        def backward(ctx, dy):
            tokens, = ctx.saved_tensors
            return None, swr_embedding_backward(tokens, _even(dy), ctx.vocab, ctx.scale, ctx.dtype), None

    class _SWRCausalConvFunction(torch.autograd.Function):
        """Autograd wrapper of the convolution, from no state: y of (x, weight, bias, silu, lengths)."""

        @staticmethod
        def forward(ctx, x, weight, bias=None, silu=True, lengths=None):
            ctx.silu = silu
            ctx.save_for_backward(x, weight, bias, lengths)
            return swr_causal_conv(x, weight, bias, silu, lengths=lengths)[0]

        @staticmethod
        @once
        def backward(ctx, dy):
            x, weight, bias, lengths = ctx.saved_tensors
            dx, dw, db = swr_causal_conv_backward(x, weight, _channels(dy), bias, ctx.silu, lengths)
            return dx, dw.to(weight.dtype), None if db is None else db.to(bias.dtype), None, None

    class _SWRSelectiveScanFunction(torch.autograd.Function):
        """Autograd wrapper of the scan: (y, h_last) of (x, dt, A, B, C, D, z, dt_bias,
        softplus, h0, lengths)."""

        @staticmethod
        def forward(ctx, x, dt, A, B, C, D=None, z=None, dt_bias=None, softplus=True, h0=None, lengths=None):
            y, carriers, h_last = swr_selective_scan(x, dt, A, B, C, D, z, dt_bias, softplus, h0, lengths,
                                                     save_carriers=True, want_state=True)
            ctx.softplus = softplus
            ctx.save_for_backward(x, dt, A, B, C, D, z, dt_bias, h0, lengths, carriers)
            ctx.set_materialize_grads(False)
            return y, h_last

        @staticmethod
        @once
        def backward(ctx, dy, dh):
            x, dt, A, B, C, D, z, dt_bias, h0, lengths, carriers = ctx.saved_tensors
            if dy is None and dh is None:
                return (None,) * 11
            dy = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if dy is None else _channels(dy)
            dx, ddt, dA, dB, dC, dD, dz, dbias, dh0 = swr_selective_scan_backward(
                x, dt, A, B, C, dy, carriers, D, z, dt_bias, ctx.softplus, h0, None if dh is None else dh.contiguous(),
                lengths, want_dh0=h0 is not None)
            return dx, ddt, dA, dB, dC, dD, dz, dbias, None, dh0, None

    class _SWRLogProbsFunction(torch.autograd.Function):
        """Autograd wrapper of the log probabilities: (logp, lse, entropy) of (logits, tokens, scale)."""

        @staticmethod
        def forward(ctx, logits, tokens, scale=1.0):
            logp, lse, entropy = swr_log_probs(logits, tokens, scale=scale)
            ctx.scale = scale
            ctx.save_for_backward(logits, tokens, lse, entropy)
            ctx.set_materialize_grads(False)
            return logp, lse, entropy

        @staticmethod
        @once
        def backward(ctx, dlogp, dlse, dentropy):
            logits, tokens, lse, entropy = ctx.saved_tensors
            if dlogp is None and dlse is None and dentropy is None:
                return None, None, None
            dlogp, dlse, dentropy = (None if g is None else g.contiguous() for g in (dlogp, dlse, dentropy))
            return swr_log_probs_backward(logits, tokens, lse, entropy, dlogp, dentropy, dlse, ctx.scale), None, None

    return {f.__name__[1:]: f for f in (_SWREmbeddingFunction, _SWRCausalConvFunction, _SWRSelectiveScanFunction,
                                        _SWRLogProbsFunction)}


_made = None


def __getattr__(name):
    global _made
    if name in ("SWREmbeddingFunction", "SWRCausalConvFunction", "SWRSelectiveScanFunction", "SWRLogProbsFunction"):
        if _made is None:
            _made = _functions()
        return _made[name]
    raise AttributeError(name)
