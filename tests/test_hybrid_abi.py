"""The hybrid model's C ABI and its binding, checked without a GPU: exports,
struct layouts, and every refusal, made before any HIP call and with nothing
touched."""
import ctypes
import os
import re

import pytest

import paper_2512_13921_amd as swr
from paper_2512_13921_amd import hybrid

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "swr_hybrid.h")
F32, BF16, FP8 = 0, 1, 2
OK, E_NULL, E_SHAPE, E_DTYPE, E_PAGE, E_ALIGN, E_ALIAS, E_UNSUP, E_VER = 0, -1, -2, -3, -4, -5, -6, -7, -9

# Fake, well-aligned "device" addresses far apart: validation never dereferences them.
GB = 1 << 30
ADDRESS = [GB * 64 * (i + 1) for i in range(12)]
v = ctypes.c_void_p


def test_library_exports_every_declared_symbol():
    text = open(HEADER).read()
    names = set(re.findall(r"^\s*(?:int|int64_t)\s+(swr_\w+)\s*\(", text, re.M))
    assert names == {"swr_rms_norm", "swr_rms_norm_backward", "swr_rms_norm_workspace_bytes", "swr_fp4_linear",
                     "swr_fp4_pack", "swr_block_tables", "swr_cache_append", "swr_paged_attention",
                     "swr_paged_workspace_bytes"}
    lib = hybrid._lib()
    for name in names:
        assert hasattr(lib, name), name


def test_struct_layouts():
    assert ctypes.sizeof(hybrid.SwrNorm) == 16 + 24 + 8 + 64
    assert ctypes.sizeof(hybrid.SwrFp4) == 16 + 56
    assert ctypes.sizeof(hybrid.SwrTables) == 8 + 48
    assert ctypes.sizeof(hybrid.SwrCache) == 8 + 56
    assert ctypes.sizeof(hybrid.SwrPaged) == 64 + 72 + 8


# ----------------------------------------------------------------------------- norm


def _norm(**kw):
    n = hybrid.SwrNorm()
    n.abi_version, n.dtype, n.weight_dtype, n.out_dtype = 1, BF16, BF16, BF16
    n.outer, n.inner, n.width, n.eps = 2, 8, 64, 1e-6
    for f in ("sx", "sr", "sh", "sy"):
        setattr(n, f + "_o", 8 * 64)
        setattr(n, f + "_i", 64)
    for k, x in kw.items():
        setattr(n, k, x)
    return n


def _forward(n, x=0, r=1, w=2, y=3, scale=4, h=5):
    a = [None if i is None else ADDRESS[i] if i < 12 else i for i in (x, r, w, y, scale, h)]
    return hybrid._lib().swr_rms_norm(ctypes.byref(n) if n is not None else None, *(v(i) for i in a), None)


def _backward(n, h=0, w=1, dy=2, dh=3, dx=4, dw=5, ws=6):
    a = [None if i is None else ADDRESS[i] if i < 12 else i for i in (h, w, dy, dh, dx, dw, ws)]
    return hybrid._lib().swr_rms_norm_backward(ctypes.byref(n) if n is not None else None, *(v(i) for i in a), None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=2), E_VER), (dict(dtype=3), E_DTYPE), (dict(dtype=FP8), E_DTYPE), (dict(out_dtype=F32), E_DTYPE),
    (dict(dtype=F32, out_dtype=F32), E_DTYPE), (dict(weight_dtype=FP8), E_DTYPE), (dict(reserved=1), E_UNSUP),
    (dict(eps=-1.0), E_UNSUP), (dict(eps=float("nan")), E_UNSUP), (dict(eps=float("inf")), E_UNSUP),
    (dict(outer=-1), E_SHAPE), (dict(inner=-1), E_SHAPE), (dict(width=0), E_SHAPE), (dict(width=(1 << 30) + 1), E_UNSUP),
    (dict(outer=1 << 16, inner=1 << 16), E_UNSUP), (dict(sx_i=-64), E_SHAPE), (dict(sx_o=1 << 62), E_SHAPE),
    (dict(sh_i=63), E_SHAPE), (dict(sh_o=64), E_SHAPE), (dict(sy_i=10), E_SHAPE)])
def test_norm_refuses(kw, code):
    assert _forward(_norm(**kw)) == code
    if "sy_i" not in kw:   # (the backward only reads there)
        assert _backward(_norm(**kw)) == code
        assert hybrid._lib().swr_rms_norm_workspace_bytes(ctypes.byref(_norm(**kw))) == code


def test_norm_refuses_pointers():
    assert _forward(None) == _backward(None) == E_NULL
    for which in ("x", "w", "y"):
        assert _forward(_norm(), **{which: None}) == E_NULL
    assert _forward(_norm(out_dtype=FP8), scale=None) == E_NULL
    assert _backward(_norm(out_dtype=FP8)) == E_DTYPE
    for which in ("h", "w", "dy", "dx", "dw", "ws"):
        assert _backward(_norm(), **{which: None}) == E_NULL
    for which in ("x", "r", "w", "y", "h"):
        assert _forward(_norm(), **{which: GB * 64 * 11 + 1}) == E_ALIGN
    for which in ("h", "w", "dy", "dh", "dx", "dw"):
        assert _backward(_norm(), **{which: GB * 64 * 11 + 1}) == E_ALIGN
    assert _backward(_norm(), ws=GB * 64 * 11 + 4) == E_ALIGN


def test_norm_refuses_overlaps():
    n, base = _norm(), ADDRESS[0]
    for kw in (dict(y=0), dict(y=1), dict(y=2), dict(y=5), dict(h=2), dict(h=base + 2), dict(h=base + 128),
               dict(y=base + 1022 * 2)):
        assert _forward(n, **kw) == E_ALIAS, kw
    assert _forward(_norm(out_dtype=FP8), scale=0) == E_ALIAS
    assert _forward(_norm(sh_o=8 * 64 + 64), h=0) == E_ALIAS          # in place, other strides
    for kw in (dict(dx=0), dict(dx=1), dict(dw=0), dict(dw=2), dict(ws=4), dict(ws=0), dict(dx=ADDRESS[2] + 128)):
        assert _backward(n, **kw) == E_ALIAS, kw
    # rows between each other's, of one larger tensor [2, 8, 3, 64]: apart unless shifted
    s = {f + d: k for f in ("sx", "sr", "sh", "sy") for d, k in (("_o", 8 * 192), ("_i", 192))}
    assert _forward(_norm(**s), r=base + 128, h=base + 256, y=base + 256) == E_ALIAS
    assert _forward(_norm(**s), r=base + 128, h=base + 130) == E_ALIAS
    assert _forward(_norm(**s), r=base + 128, h=base + 254) == E_ALIAS
    assert _forward(_norm(**s), r=base + 384, h=base + 384 + 8 * 384 - 126) == E_ALIAS


def test_norm_of_nothing_is_a_no_op():
    assert _forward(_norm(outer=0), None, None, None, None, None, None) == OK
    assert _forward(_norm(inner=0), None, None, None, None, None, None) == OK
    assert hybrid._lib().swr_rms_norm_workspace_bytes(ctypes.byref(_norm(outer=0))) == 0


@pytest.mark.parametrize("dtype,rows,width", [(BF16, 1, 1), (F32, 700, 5), (BF16, 100000, 2048), (F32, 33, 20000)])
def test_norm_workspace(dtype, rows, width):
    n = _norm(dtype=dtype, out_dtype=dtype, weight_dtype=dtype, outer=1, inner=rows, width=width,
              **{f + "_i": width for f in ("sx", "sr", "sh", "sy")})
    size = hybrid._lib().swr_rms_norm_workspace_bytes(ctypes.byref(n))
    assert size >= width * 4 and size % 4 == 0 and size <= 4 * width * min(rows, 1024) + 8 * rows + 16


# ----------------------------------------------------------------------------- 4-bit weights


def _fp4(**kw):
    p = hybrid.SwrFp4()
    p.abi_version, p.dtype, p.out_dtype = 1, BF16, BF16
    p.M, p.N, p.K, p.sx, p.sy, p.sc, p.sp = 4, 100, 96, 96, 100, 48, 3
    for k, x in kw.items():
        setattr(p, k, x)
    return p


def _linear(p, x=0, scale=1, codes=2, powers=3, y=4):
    a = [None if i is None else ADDRESS[i] if i < 12 else i for i in (x, scale, codes, powers, y)]
    return hybrid._lib().swr_fp4_linear(ctypes.byref(p) if p is not None else None, *(v(i) for i in a), None)


def _pack(p, w=0, codes=2, powers=3):
    a = [None if i is None else ADDRESS[i] if i < 12 else i for i in (w, codes, powers)]
    return hybrid._lib().swr_fp4_pack(ctypes.byref(p) if p is not None else None, *(v(i) for i in a), None)


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=0), E_VER), (dict(dtype=3), E_DTYPE), (dict(reserved=1), E_UNSUP), (dict(N=-1), E_SHAPE),
    (dict(K=0), E_SHAPE), (dict(K=(1 << 30) + 1, sx=1 << 31, sc=1 << 31, sp=1 << 31), E_UNSUP), (dict(sx=-96), E_SHAPE),
    (dict(sc=-48), E_SHAPE), (dict(sp=-1), E_SHAPE), (dict(sc=1 << 60), E_SHAPE), (dict(sc=40), None)])
def test_fp4_refuses(kw, code):
    for call in (_linear, _pack):
        got = call(_fp4(**kw))
        assert got == code if code is not None else got in (E_SHAPE, E_ALIGN), call


def test_fp4_refuses_each_of_the_two():
    assert _linear(None) == _pack(None) == E_NULL
    assert _linear(_fp4(out_dtype=FP8)) == E_DTYPE and _pack(_fp4(dtype=FP8)) == E_DTYPE
    assert _linear(_fp4(M=-1)) == E_SHAPE and _linear(_fp4(sy=99)) == E_SHAPE
    assert _pack(_fp4(sc=32)) == E_SHAPE and _pack(_fp4(sp=2)) == E_SHAPE
    for which in ("x", "codes", "powers", "y"):
        assert _linear(_fp4(), **{which: None}) == E_NULL
    for which in ("w", "codes", "powers"):
        assert _pack(_fp4(), **{which: None}) == E_NULL
    odd = GB * 64 * 11
    assert _linear(_fp4(), x=odd + 1) == _linear(_fp4(), y=odd + 1) == _linear(_fp4(), codes=odd + 8) == E_ALIGN
    assert _linear(_fp4(), scale=odd + 2) == E_ALIGN and _pack(_fp4(), codes=odd + 4) == E_ALIGN
    for kw in (dict(y=0), dict(y=1), dict(y=2), dict(y=3)):
        assert _linear(_fp4(), **kw) == E_ALIAS
    assert _pack(_fp4(), codes=0) == _pack(_fp4(), powers=0) == _pack(_fp4(), powers=2) == E_ALIAS
    assert _linear(_fp4(M=0), None, None, None, None, None) == _linear(_fp4(N=0), None, None, None, None, None) == OK
    assert _pack(_fp4(N=0), None, None, None) == OK


# ----------------------------------------------------------------------------- paged cache


def _tables(p, **kw):
    names = ("lengths", "news", "stack", "count", "table", "slots", "starts", "new_lengths", "new_count")
    a = {n: ADDRESS[i] for i, n in enumerate(names)}
    a.update(kw)
    return hybrid._lib().swr_block_tables(ctypes.byref(p) if p is not None else None, *(v(a[n]) for n in names), None)


def _table_problem(**kw):
    p = hybrid.SwrTables()
    p.abi_version, p.batch, p.max_pages, p.st, p.page_size, p.tokens, p.free_pages = 1, 4, 10, 10, 16, 20, 30
    for k, x in kw.items():
        setattr(p, k, x)
    return p


@pytest.mark.parametrize("kw,code", [
    (dict(abi_version=0), E_VER), (dict(reserved=1), E_UNSUP), (dict(batch=-1), E_SHAPE), (dict(max_pages=-1), E_SHAPE),
    (dict(tokens=-1), E_SHAPE), (dict(free_pages=-1), E_SHAPE), (dict(page_size=0), E_PAGE), (dict(page_size=65537), E_PAGE),
    (dict(st=9), E_SHAPE), (dict(st=-10), E_SHAPE), (dict(batch=1 << 31), E_UNSUP), (dict(tokens=1 << 31), E_UNSUP)])
def test_tables_refuse(kw, code):
    assert _tables(_table_problem(**kw)) == code


def test_tables_refuse_pointers():
    assert _tables(None) == E_NULL
    names = ("lengths", "news", "stack", "count", "table", "slots", "starts", "new_lengths", "new_count")
    for n in names:
        assert _tables(_table_problem(), **{n: None}) == E_NULL, n
        assert _tables(_table_problem(), **{n: ADDRESS[11] + 2}) == E_ALIGN, n
    assert _tables(_table_problem(), slots=ADDRESS[11] + 4) == E_ALIGN
    for out in names[4:]:
        for other in names:
            if other != out:
                i = names.index(other)
                assert _tables(_table_problem(), **{out: ADDRESS[i]}) == E_ALIAS, (out, other)


def _cache_of(p=None, **kw):
    c = hybrid.SwrCache() if p is None else p.cache
    c.abi_version, c.dtype, c.pages, c.page_size, c.heads, c.D = 1, BF16, 50, 16, 4, 64
    c.s_page, c.s_token, c.s_head = 16 * 4 * 64, 4 * 64, 64
    for k, x in kw.items():
        setattr(c, k, x)
    return c


BAD_CACHES = [
    (dict(abi_version=0), E_VER), (dict(dtype=FP8), E_DTYPE), (dict(pages=-1), E_SHAPE), (dict(heads=0), E_SHAPE),
    (dict(D=0), E_SHAPE), (dict(D=24, s_head=24), E_UNSUP), (dict(D=272, s_head=272, s_token=4 * 272, s_page=64 * 272), E_UNSUP),
    (dict(page_size=0), E_PAGE), (dict(page_size=65537), E_PAGE), (dict(s_token=4 * 64 - 1), E_SHAPE),
    (dict(s_head=60), E_SHAPE), (dict(s_token=4 * 64 + 4), E_SHAPE), (dict(s_head=-64), E_SHAPE),
    (dict(s_page=16 * 4 * 64 + 4), E_ALIGN), (dict(pages=1 << 24), E_UNSUP), (dict(s_page=1 << 61), E_SHAPE)]


def _append(c, tokens=5, sk=(256, 64), sv=(256, 64), k=0, v_=1, slots=2, kc=3, vc=4):
    a = [None if i is None else ADDRESS[i] if i < 12 else i for i in (k, v_, slots, kc, vc)]
    two = ctypes.c_int64 * 2
    return hybrid._lib().swr_cache_append(ctypes.byref(c) if c is not None else None, tokens, two(*sk), two(*sv),
                                          *(v(i) for i in a), None)


@pytest.mark.parametrize("kw,code", BAD_CACHES)
def test_append_and_attention_refuse_caches(kw, code):
    assert _append(_cache_of(**kw)) == code
    p = _paged()
    _cache_of(p, **kw)
    assert _attention(p) == code
    assert hybrid._lib().swr_paged_workspace_bytes(ctypes.byref(p)) == code


def test_append_refuses():
    c = _cache_of()
    assert _append(None) == E_NULL
    assert _append(c, tokens=-1) == E_SHAPE and _append(c, tokens=1 << 31) == E_UNSUP
    assert _append(c, sk=(-256, 64)) == E_SHAPE and _append(c, sv=(256, 4)) == E_ALIGN
    for which in ("k", "v_", "slots", "kc", "vc"):
        assert _append(c, **{which: None}) == E_NULL
        assert _append(c, **{which: ADDRESS[11] + 4}) == E_ALIGN
    for kw in (dict(kc=4), dict(kc=0), dict(vc=0), dict(vc=1), dict(kc=2)):
        assert _append(c, **kw) == E_ALIAS
    assert _append(c, tokens=0, k=None, v_=None, slots=None, kc=None, vc=None) == OK
    assert _append(_cache_of(pages=0), k=None, v_=None, slots=None, kc=None, vc=None) == OK


def _paged(**kw):
    p = hybrid.SwrPaged()
    _cache_of(p)
    p.batch, p.q_heads, p.max_pages, p.st, p.window, p.scale = 3, 8, 100, 100, 0, 0.125
    p.sq_b = p.sy_b = 8 * 64
    p.sq_h = p.sy_h = 64
    for k, x in kw.items():
        setattr(p, k, x)
    return p


def _attention(p, q=0, kc=1, vc=2, table=3, lengths=4, y=5, lse=6, ws=7):
    a = [None if i is None else ADDRESS[i] if i < 12 else i for i in (q, kc, vc, table, lengths, y, lse, ws)]
    return hybrid._lib().swr_paged_attention(ctypes.byref(p) if p is not None else None, *(v(i) for i in a), None)


@pytest.mark.parametrize("kw,code", [
    (dict(batch=-1), E_SHAPE), (dict(q_heads=0), E_SHAPE), (dict(q_heads=6), E_SHAPE), (dict(max_pages=-1), E_SHAPE),
    (dict(window=-1), E_SHAPE), (dict(st=-1), E_SHAPE), (dict(reserved=1), E_UNSUP), (dict(scale=float("nan")), E_UNSUP),
    (dict(scale=float("inf")), E_UNSUP), (dict(q_heads=65540), E_UNSUP), (dict(batch=1 << 20), E_UNSUP),
    (dict(sy_h=60), E_SHAPE), (dict(sy_b=64), E_SHAPE), (dict(sq_h=-64), E_SHAPE), (dict(sq_h=68), E_ALIGN),
    (dict(sy_b=8 * 64 + 4), E_ALIGN)])
def test_attention_refuses(kw, code):
    assert _attention(_paged(**kw)) == code
    assert hybrid._lib().swr_paged_workspace_bytes(ctypes.byref(_paged(**kw))) == code


def test_attention_refuses_pointers():
    assert _attention(None) == E_NULL
    for which in ("q", "kc", "vc", "table", "lengths", "y", "ws"):
        assert _attention(_paged(), **{which: None}) == E_NULL, which
    for which in ("q", "kc", "vc", "y", "ws"):
        assert _attention(_paged(), **{which: ADDRESS[11] + 8}) == E_ALIGN
    for which in ("table", "lengths", "lse"):
        assert _attention(_paged(), **{which: ADDRESS[11] + 2}) == E_ALIGN
    for out in ("y", "lse", "ws"):
        for i in range(5):
            assert _attention(_paged(), **{out: i}) == E_ALIAS
    assert _attention(_paged(), lse=5) == _attention(_paged(), ws=5) == _attention(_paged(), ws=6) == E_ALIAS
    # a table of few positions, or a short window, is attended to without a workspace
    size = hybrid._lib().swr_paged_workspace_bytes
    assert size(ctypes.byref(_paged())) > 0
    assert size(ctypes.byref(_paged(max_pages=10, st=10))) == size(ctypes.byref(_paged(window=64))) == 0
    assert _attention(_paged(batch=0), None, None, None, None, None, None, None, None) == OK


# ----------------------------------------------------------------------------- the binding's own refusals

torch = pytest.importorskip("torch")


def test_binding_refuses_host_tensors():
    x, w = torch.zeros(2, 64), torch.zeros(64)
    c, i = torch.zeros(3, 16, 1, 64), torch.zeros(2, dtype=torch.int32)
    u = torch.zeros(5, 32, dtype=torch.uint8)
    for call in (lambda: swr.swr_rms_norm(x, w), lambda: swr.swr_rms_norm_backward(x, w, x),
                 lambda: swr.swr_fp4_pack(x), lambda: swr.swr_fp4_linear(x, u, u[:, :2]),
                 lambda: swr.swr_block_tables(i, i, torch.zeros(2, 3, dtype=torch.int32), i, i[:1], 16, 2),
                 lambda: swr.swr_cache_append(x[:, None], x[:, None], c, c, i.long()),
                 lambda: swr.swr_paged_attention(x[:, None], c, c, torch.zeros(2, 3, dtype=torch.int32), i)):
        with pytest.raises(ValueError, match="GPU tensor"):
            call()


def test_rows_of_a_tensor():
    t = torch.zeros(4, 3, 5, 8)
    assert hybrid._rows(t, "t") == (4, 15, (120, 8))
    assert hybrid._rows(t[:, 1], "t") == (4, 5, (120, 8))
    assert hybrid._rows(t[0, 0], "t") == (1, 5, (0, 8))
    assert hybrid._rows(t[0, 0, 0], "t") == (1, 1, (0, 0))
    assert hybrid._rows(t[:, :, :1], "t") == (4, 3, (120, 40))
    assert hybrid._rows(t[:, :1, 2:], "t") == (4, 3, (120, 8))
    for bad in (t[:, :, 1:], t.transpose(2, 3), t[..., ::2]):
        with pytest.raises(ValueError):
            hybrid._rows(bad, "t")
