"""The C ABI of a recurrent language model's operators and its binding, checked without a
GPU: exports, struct layouts, and every refusal, made before any HIP call and with nothing
touched."""
import ctypes
import os
import re

import pytest

import paper_2512_13921_amd as swr
from paper_2512_13921_amd import lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "swr_lm.h")
F32, BF16, FP8 = 0, 1, 2
OK, E_NULL, E_SHAPE, E_DTYPE, E_PAGE, E_ALIGN, E_ALIAS, E_UNSUP, E_VER = 0, -1, -2, -3, -4, -5, -6, -7, -9

# Fake, well-aligned "device" addresses far apart: validation never dereferences them.
GB = 1 << 30
ADDRESS = [GB * 64 * (i + 1) for i in range(32)]
v = ctypes.c_void_p
ref = ctypes.byref


def _at(i):
    return None if i is None else ADDRESS[i] if i < 32 else i


def _set(s, values, kw):
    for k, x in {**values, **kw}.items():
        setattr(s, k, x)
    return s


def test_library_exports_every_declared_symbol():
    text = open(HEADER).read()
    names = set(re.findall(r"^\s*(?:int|int64_t)\s+(swr_\w+)\s*\(", text, re.M))
    assert names == set(lm._BOUND)
    lib = lm._lib()
    for name in names:
        assert hasattr(lib, name), name


def test_names_are_the_packages():
    for name in lm.__all__:
        if name.startswith("swr_"):
            assert getattr(swr, name) is getattr(lm, name)
            assert getattr(lm, name).__doc__
        else:
            assert getattr(swr, name).__doc__
        assert name in swr.__all__


def test_struct_layouts():
    assert ctypes.sizeof(lm.SwrEmbed) == 16 + 40 + 8
    assert ctypes.sizeof(lm.SwrConv) == 16 + 24 + 48
    assert ctypes.sizeof(lm.SwrScan) == 16 + 32 + 64 + 48
    assert ctypes.sizeof(lm.SwrScanInputs) == 80
    assert ctypes.sizeof(lm.SwrScanGradients) == 72
    assert ctypes.sizeof(lm.SwrLogProb) == 16 + 32 + 8
    text = open(HEADER).read()
    for name, value in (("SWR_CONV_SILU", lm.SWR_CONV_SILU), ("SWR_SCAN_SOFTPLUS", lm.SWR_SCAN_SOFTPLUS),
                        ("SWR_SCAN_BLOCK", lm.SWR_SCAN_BLOCK), ("SWR_TOP_MOST", lm.SWR_TOP_MOST)):
        assert int(re.search(rf"#define {name} (\d+)u?$", text, re.M).group(1)) == value


# ----------------------------------------------------------------------------- embedding


def _embed(**kw):
    return _set(lm.SwrEmbed(), dict(abi_version=1, dtype=BF16, out_dtype=BF16, token_bytes=8, tokens=10, vocab=100,
                                    width=64, st=64, sy=64, scale=1.0), kw)


def _lookup(e, tokens=0, table=1, y=2):
    return lm._lib().swr_embedding(None if e is None else ref(e), *(v(_at(i)) for i in (tokens, table, y)), None)


def _lookup_back(e, tokens=0, dy=1, dtable=2, ws=3):
    return lm._lib().swr_embedding_backward(None if e is None else ref(e),
                                            *(v(_at(i)) for i in (tokens, dy, dtable, ws)), None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=2), E_VER), (dict(dtype=FP8), E_DTYPE), (dict(dtype=7, out_dtype=7), E_DTYPE),
    (dict(token_bytes=2), E_DTYPE), (dict(token_bytes=0), E_DTYPE), (dict(dtype=F32), E_DTYPE),
    (dict(reserved=1), E_UNSUP), (dict(scale=float("inf")), E_UNSUP), (dict(scale=float("nan")), E_UNSUP),
    (dict(tokens=-1), E_SHAPE), (dict(vocab=0), E_SHAPE), (dict(width=0), E_SHAPE), (dict(st=-64), E_SHAPE),
    (dict(sy=-1), E_SHAPE), (dict(tokens=1 << 31), E_UNSUP), (dict(vocab=(1 << 30) + 1), E_UNSUP),
    (dict(width=(1 << 30) + 1, st=1 << 31, sy=1 << 31), E_UNSUP), (dict(st=1 << 62), E_SHAPE)])
def test_embedding_refuses(kw, code):
    assert _lookup(_embed(**kw)) == code
    assert _lookup_back(_embed(**kw)) == code
    assert lm._lib().swr_embedding_workspace_bytes(ref(_embed(**kw))) == code


def test_embedding_refuses_pointers_and_overlaps():
    assert _lookup(None) == E_NULL and _lookup_back(None) == E_NULL
    assert lm._lib().swr_embedding_workspace_bytes(None) == E_NULL
    for name in ("tokens", "table", "y"):
        assert _lookup(_embed(), **{name: None}) == E_NULL
    for name in ("tokens", "dy", "dtable", "ws"):
        assert _lookup_back(_embed(), **{name: None}) == E_NULL
    for name, off in (("tokens", 4), ("table", 1), ("y", 1)):
        assert _lookup(_embed(), **{name: ADDRESS[5] + off}) == E_ALIGN
    for name, off in (("tokens", 4), ("dy", 1), ("dtable", 1), ("ws", 8)):
        assert _lookup_back(_embed(), **{name: ADDRESS[5] + off}) == E_ALIGN
    assert _lookup_back(_embed(out_dtype=F32), dtable=ADDRESS[5] + 2) == E_ALIGN
    # Rows that overlap can be read, not written.
    assert _lookup(_embed(sy=63)) == E_SHAPE
    assert _lookup_back(_embed(st=63)) == E_SHAPE
    assert _lookup(_embed(out_dtype=F32)) == E_DTYPE
    # The last row ends where the next tensor may begin.
    assert _lookup(_embed(), y=ADDRESS[1] + 100 * 64 * 2 - 2) == E_ALIAS
    assert _lookup(_embed(), y=ADDRESS[0] + 72) == E_ALIAS
    assert _lookup_back(_embed(), dtable=1) == E_ALIAS
    assert _lookup_back(_embed(), ws=1) == E_ALIAS
    assert _lookup_back(_embed(), ws=2) == E_ALIAS
    assert _lookup_back(_embed(), ws=0) == E_ALIAS


def test_embedding_of_nothing():
    e = _embed(tokens=0)
    assert _lookup(e, None, None, None) == OK
    assert _lookup_back(e, dtable=None) == E_NULL
    bytes_of = lm._lib().swr_embedding_workspace_bytes
    assert bytes_of(ref(_embed(tokens=1))) > 0
    # It grows with the tokens.
    sizes = [bytes_of(ref(_embed(tokens=n, vocab=1 << 16, width=512, st=512, sy=512))) for n in (1, 100, 10000, 1000000)]
    assert sizes == sorted(sizes)


# ----------------------------------------------------------------------------- convolution


def _conv(**kw):
    return _set(lm.SwrConv(), dict(abi_version=1, dtype=BF16, flags=1, taps=4, B=2, T=50, C=64, sx_b=3200, sx_t=64,
                                   sy_b=3200, sy_t=64, sd_b=3200, sd_t=64), kw)


def _convolve(p, x=0, w=1, bias=2, state=3, lengths=4, y=5, out=6):
    return lm._lib().swr_causal_conv(None if p is None else ref(p),
                                     *(v(_at(i)) for i in (x, w, bias, state, lengths, y, out)), None)


def _convolve_back(p, x=0, w=1, bias=2, dy=3, lengths=4, dx=5, dw=6, dbias=7, ws=8):
    return lm._lib().swr_causal_conv_backward(None if p is None else ref(p),
                                              *(v(_at(i)) for i in (x, w, bias, dy, lengths, dx, dw, dbias, ws)), None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=0), E_VER), (dict(dtype=FP8), E_DTYPE), (dict(flags=2), E_UNSUP), (dict(taps=0), E_SHAPE),
    (dict(taps=-1), E_SHAPE), (dict(taps=9), E_UNSUP), (dict(B=-1), E_SHAPE), (dict(T=-1), E_SHAPE), (dict(C=0), E_SHAPE),
    (dict(B=(1 << 30) + 1), E_UNSUP), (dict(T=(1 << 30) + 1), E_UNSUP), (dict(C=(1 << 30) + 1), E_UNSUP),
    (dict(B=1 << 30, T=1 << 30), E_UNSUP), (dict(sx_t=-1), E_SHAPE), (dict(sx_b=-1), E_SHAPE), (dict(sy_t=-1), E_SHAPE),
    (dict(sx_b=1 << 61), E_SHAPE)])
def test_convolution_refuses(kw, code):
    assert _convolve(_conv(**kw)) == code
    assert _convolve_back(_conv(**kw)) == code
    assert lm._lib().swr_causal_conv_workspace_bytes(ref(_conv(**kw))) == code


def test_convolution_refuses_pointers_and_overlaps():
    assert _convolve(None) == E_NULL and _convolve_back(None) == E_NULL
    assert lm._lib().swr_causal_conv_workspace_bytes(None) == E_NULL
    for name in ("x", "w", "y"):
        assert _convolve(_conv(), **{name: None}) == E_NULL
    for name in ("x", "w", "dy", "dx", "dw", "ws"):
        assert _convolve_back(_conv(), **{name: None}) == E_NULL
    for name in ("x", "w", "bias", "state", "y", "out"):
        assert _convolve(_conv(), **{name: ADDRESS[9] + 1}) == E_ALIGN
    assert _convolve(_conv(), lengths=ADDRESS[9] + 2) == E_ALIGN
    for name, off in (("x", 1), ("dy", 1), ("dx", 1), ("dw", 2), ("dbias", 2), ("lengths", 2), ("ws", 8)):
        assert _convolve_back(_conv(), **{name: ADDRESS[12] + off}) == E_ALIGN
    assert _convolve(_conv(sy_t=63)) == E_SHAPE
    assert _convolve(_conv(sy_b=64)) == E_SHAPE
    assert _convolve_back(_conv(sd_t=63)) == E_SHAPE
    assert lm._lib().swr_causal_conv_workspace_bytes(ref(_conv(sd_t=63))) == E_SHAPE
    for other in (0, 1, 2, 3, 4, 6):
        assert _convolve(_conv(), y=other) == E_ALIAS
    for other in (0, 1, 2, 4):
        assert _convolve(_conv(), out=other) == E_ALIAS
    assert _convolve(_conv(), out=ADDRESS[3] + 128) == E_ALIAS   # (the state itself is allowed, a part of it is not)
    for name in ("dx", "dw", "dbias", "ws"):
        for other in (0, 1, 2, 3, 4):
            assert _convolve_back(_conv(), **{name: other}) == E_ALIAS
    assert _convolve_back(_conv(), ws=6) == E_ALIAS


def test_convolution_of_nothing():
    for kw in (dict(B=0), dict(T=0)):
        assert _convolve(_conv(**kw), x=None, y=None, out=None) == OK
    assert _convolve(_conv(B=0), x=None, y=None) == OK
    assert _convolve(_conv(T=0, taps=1), x=None, y=None) == OK   # one tap keeps nothing


# ----------------------------------------------------------------------------- scan

INPUTS = ("x", "dt", "A", "B", "C", "bias", "skip", "z", "h0", "lengths")
GRADIENTS = ("dx", "ddt", "dA", "dB", "dC", "dbias", "dskip", "dz", "dh0")


def _scan(**kw):
    rows, shared = 50 * 64, 50 * 2 * 16
    return _set(lm.SwrScan(), dict(abi_version=1, dtype=BF16, flags=1, N=16, B=2, T=50, D=64, G=2,
                                   sx_b=rows, sx_t=64, sdt_b=rows, sdt_t=64, sz_b=rows, sz_t=64, sy_b=rows, sy_t=64,
                                   sB_b=shared, sB_t=32, sB_g=16, sC_b=shared, sC_t=32, sC_g=16), kw)


def _inputs(kw):
    q = lm.SwrScanInputs()
    for i, name in enumerate(INPUTS):
        setattr(q, name, _at(kw.get(name, i)))
    return q


def _run(p, y=10, carriers=11, last=12, ws=13, **kw):
    return lm._lib().swr_selective_scan(None if p is None else ref(p), ref(_inputs(kw)),
                                        *(v(_at(i)) for i in (y, carriers, last, ws)), None)


def _run_back(p, dy=10, carriers=11, dlast=12, ws=13, **kw):
    g = lm.SwrScanGradients()
    for i, name in enumerate(GRADIENTS):
        setattr(g, name, _at(kw.get(name, 16 + i)))
    return lm._lib().swr_selective_scan_backward(None if p is None else ref(p), ref(_inputs(kw)), v(_at(dy)),
                                                 v(_at(carriers)), v(_at(dlast)), ref(g), v(_at(ws)), None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=3), E_VER), (dict(dtype=FP8), E_DTYPE), (dict(flags=4), E_UNSUP), (dict(N=0), E_SHAPE),
    (dict(N=65, sB_t=130, sC_t=130), E_UNSUP), (dict(B=-1), E_SHAPE), (dict(T=-1), E_SHAPE), (dict(D=0), E_SHAPE),
    (dict(G=0), E_SHAPE), (dict(G=3), E_SHAPE), (dict(G=-2), E_SHAPE), (dict(B=(1 << 30) + 1), E_UNSUP),
    (dict(T=(1 << 30) + 1), E_UNSUP), (dict(D=(1 << 28) + 2), E_UNSUP), (dict(B=1 << 30, T=1 << 30), E_UNSUP),
    (dict(sx_t=-1), E_SHAPE), (dict(sdt_b=-1), E_SHAPE), (dict(sB_g=-16), E_SHAPE), (dict(sC_t=-1), E_SHAPE),
    (dict(sy_t=-1), E_SHAPE), (dict(sx_b=1 << 61), E_SHAPE)])
def test_scan_refuses(kw, code):
    lib = lm._lib()
    assert _run(_scan(**kw)) == code
    assert _run_back(_scan(**kw)) == code
    assert lib.swr_selective_scan_workspace_bytes(ref(_scan(**kw))) == code
    assert lib.swr_selective_scan_backward_workspace_bytes(ref(_scan(**kw))) == code


def test_scan_refuses_pointers():
    lib = lm._lib()
    assert _run(None) == E_NULL and _run_back(None) == E_NULL
    assert lib.swr_selective_scan_workspace_bytes(None) == E_NULL
    assert lib.swr_selective_scan_backward_workspace_bytes(None) == E_NULL
    assert lib.swr_selective_scan(ref(_scan()), None, *(v(_at(i)) for i in range(4)), None) == E_NULL
    for name in ("x", "dt", "A", "B", "C", "y"):
        assert _run(_scan(), **{name: None}) == E_NULL, name
    for name in ("x", "dt", "A", "B", "C", "dy", "carriers", "ws", "dx", "ddt", "dA", "dB", "dC"):
        assert _run_back(_scan(), **{name: None}) == E_NULL, name
    # A gradient is there with its input, and only then.
    for name in ("z", "bias", "skip"):
        assert _run_back(_scan(), **{name: None}) == E_NULL
        assert _run_back(_scan(), **{"d" + name: None}) == E_NULL
    # Long runs of few channels are cut, which takes a workspace.
    long = _scan(T=5000, sx_b=1 << 20, sdt_b=1 << 20, sz_b=1 << 20, sy_b=1 << 20, sB_b=1 << 20, sC_b=1 << 20)
    assert lib.swr_selective_scan_workspace_bytes(ref(long)) > 0
    assert _run(long, ws=None) == E_NULL


def test_scan_refuses_alignments():
    for name in INPUTS:
        off = 1 if name in ("x", "dt", "B", "C", "z") else 2
        assert _run(_scan(), **{name: ADDRESS[30] + off}) == E_ALIGN, name
        assert _run_back(_scan(), **{name: ADDRESS[30] + off}) == E_ALIGN, name
    for name, off in (("y", 1), ("carriers", 2), ("last", 2), ("ws", 4)):
        assert _run(_scan(), **{name: ADDRESS[30] + off}) == E_ALIGN, name
    for name in GRADIENTS + ("dy", "carriers", "dlast", "ws"):
        off = 1 if name in ("dx", "ddt", "dB", "dC", "dz", "dy") else 2
        assert _run_back(_scan(), **{name: ADDRESS[30] + off}) == E_ALIGN, name


def test_scan_refuses_overlaps():
    assert _run(_scan(sy_t=63)) == E_SHAPE and _run(_scan(sy_b=64)) == E_SHAPE
    for i, name in enumerate(INPUTS):
        for out in ("y", "carriers") + (() if name == "h0" else ("last",)):
            assert _run(_scan(), **{out: i}) == E_ALIAS, (name, out)
    assert _run(_scan(), last=ADDRESS[8] + 4) == E_ALIAS   # (h0 itself is allowed, a part of it is not)
    assert _run(_scan(), carriers=10) == E_ALIAS and _run(_scan(), last=10) == E_ALIAS
    for i in range(13):
        for name in GRADIENTS + ("ws",):
            assert _run_back(_scan(), **{name: i}) == E_ALIAS, (name, i)
    for name in GRADIENTS[1:]:
        assert _run_back(_scan(), **{name: 16}) == E_ALIAS, name


def test_scan_of_nothing():
    lib = lm._lib()
    none = {n: None for n in INPUTS}
    assert _run(_scan(B=0), y=None, carriers=None, last=None, ws=None, **none) == OK
    assert _run(_scan(T=0), y=None, carriers=None, last=None, ws=None, **none) == OK
    assert lib.swr_selective_scan_workspace_bytes(ref(_scan(B=0))) == 0


# ----------------------------------------------------------------------------- log probabilities


def _logp(**kw):
    return _set(lm.SwrLogProb(), dict(abi_version=1, dtype=F32, token_bytes=8, top=4, rows=10, vocab=100, sl=100,
                                      sd=100, scale=1.0), kw)


def _score(p, logits=0, tokens=1, logp=2, lse=3, entropy=4, top=5, best=6, ws=7):
    return lm._lib().swr_log_probs(None if p is None else ref(p),
                                   *(v(_at(i)) for i in (logits, tokens, logp, lse, entropy, top, best, ws)), None)


def _score_back(p, logits=0, tokens=1, lse=2, entropy=3, dlogp=4, dlse=5, dentropy=6, dlogits=7):
    return lm._lib().swr_log_probs_backward(None if p is None else ref(p),
                                            *(v(_at(i)) for i in (logits, tokens, lse, entropy, dlogp, dlse, dentropy,
                                                                  dlogits)), None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=2), E_VER), (dict(dtype=FP8), E_DTYPE), (dict(token_bytes=1), E_DTYPE), (dict(reserved=1), E_UNSUP),
    (dict(scale=0.0), E_UNSUP), (dict(scale=-1.0), E_UNSUP), (dict(scale=float("nan")), E_UNSUP),
    (dict(scale=float("inf")), E_UNSUP), (dict(scale=3.0e38), E_UNSUP), (dict(rows=-1), E_SHAPE), (dict(vocab=0), E_SHAPE),
    (dict(top=-1), E_SHAPE), (dict(top=101), E_SHAPE), (dict(top=65), E_UNSUP), (dict(rows=1 << 31), E_UNSUP),
    (dict(vocab=(1 << 30) + 1, sl=1 << 31, sd=1 << 31), E_UNSUP), (dict(sl=-1), E_SHAPE), (dict(sl=1 << 61), E_SHAPE)])
def test_log_probs_refuses(kw, code):
    assert _score(_logp(**kw)) == code
    assert _score_back(_logp(**kw)) == code
    assert lm._lib().swr_log_probs_workspace_bytes(ref(_logp(**kw))) == code


def test_log_probs_refuses_pointers_and_overlaps():
    assert _score(None) == E_NULL and _score_back(None) == E_NULL
    assert lm._lib().swr_log_probs_workspace_bytes(None) == E_NULL
    for name in ("logits", "tokens", "logp", "lse", "entropy", "top", "best"):
        assert _score(_logp(), **{name: None}) == E_NULL
    for name in ("logits", "tokens", "lse", "entropy", "dlogits"):
        assert _score_back(_logp(), **{name: None}) == E_NULL
    for name, off in (("logits", 2), ("tokens", 4), ("logp", 2), ("lse", 2), ("entropy", 2), ("top", 2), ("best", 4),
                      ("ws", 8)):
        assert _score(_logp(), **{name: ADDRESS[9] + off}) == E_ALIGN
    for name, off in (("logits", 2), ("tokens", 4), ("lse", 2), ("entropy", 2), ("dlogp", 2), ("dlse", 2),
                      ("dentropy", 2), ("dlogits", 2)):
        assert _score_back(_logp(), **{name: ADDRESS[9] + off}) == E_ALIGN
    for name in ("logp", "lse", "entropy", "top", "best"):
        for other in (0, 1):
            assert _score(_logp(), **{name: other}) == E_ALIAS
    assert _score(_logp(), logp=3) == E_ALIAS and _score(_logp(), top=6) == E_ALIAS
    assert _score_back(_logp(sd=99)) == E_SHAPE
    for other in range(1, 7):
        assert _score_back(_logp(), dlogits=other) == E_ALIAS
    # The logits themselves are allowed, in their own layout only.
    assert _score_back(_logp(sd=128), dlogits=0) == E_ALIAS
    assert _score_back(_logp(), dlogits=ADDRESS[0] + 4) == E_ALIAS
    # A few long rows are cut, which takes a workspace.
    few = _logp(rows=1, vocab=1 << 18, sl=1 << 18)
    assert lm._lib().swr_log_probs_workspace_bytes(ref(few)) > 0
    assert _score(few, ws=None) == E_NULL and _score(few, ws=0) == E_ALIAS


def test_log_probs_of_nothing():
    assert _score(_logp(rows=0), *(None,) * 8) == OK
    assert _score_back(_logp(rows=0), *(None,) * 8) == OK


# ----------------------------------------------------------------------------- the binding


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(2, 3, 4)
    tokens = torch.zeros(2, 3, dtype=torch.int64)
    with pytest.raises(ValueError):
        swr.swr_embedding(tokens, torch.zeros(5, 4))
    with pytest.raises(ValueError):
        swr.swr_embedding_backward(tokens, x, 5)
    with pytest.raises(ValueError):
        swr.swr_causal_conv(x, torch.zeros(4, 2))
    with pytest.raises(ValueError):
        swr.swr_causal_conv_step(x[:, 0], torch.zeros(4, 2), torch.zeros(2, 1, 4))
    with pytest.raises(ValueError):
        swr.swr_causal_conv_backward(x, torch.zeros(4, 2), x)
    rates, shared = torch.zeros(4, 2), torch.zeros(2, 3, 2)
    with pytest.raises(ValueError):
        swr.swr_selective_scan(x, x, rates, shared, shared)
    with pytest.raises(ValueError):
        swr.swr_selective_step(x[:, 0], x[:, 0], rates, shared[:, 0], shared[:, 0], torch.zeros(2, 4, 2))
    with pytest.raises(ValueError):
        swr.swr_selective_scan_backward(x, x, rates, shared, shared, x, torch.zeros(2, 1, 4, 2))
    with pytest.raises(ValueError):
        swr.swr_log_probs(x, tokens)
    with pytest.raises(ValueError):
        swr.swr_log_probs_backward(x, tokens, x[..., 0].contiguous(), x[..., 0].contiguous())
