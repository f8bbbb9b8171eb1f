"""Strides of tensors that a call of the norm does not have are not read (CPU only:
the calls are refused for their alignment, which is checked after the strides)."""
import pytest

from test_hybrid_abi import ADDRESS, BF16, E_ALIGN, E_SHAPE, FP8, _backward, _forward, _norm

ODD = ADDRESS[11] + 1
# none, negative, of overlapping rows, out of range
STRIDES = [(0, 0), (-512, -64), (64, 0), (1 << 62, 1 << 62)]


@pytest.mark.parametrize("out", [BF16, FP8])
@pytest.mark.parametrize("outer,inner", STRIDES)
def test_forward(outer, inner, out):
    h = dict(sh_o=outer, sh_i=inner)
    assert _forward(_norm(out_dtype=out, **h), h=None, x=ODD) == E_ALIGN
    assert _forward(_norm(out_dtype=out, **h), r=None, h=None, x=ODD) == E_ALIGN
    assert _forward(_norm(out_dtype=out, **h), x=ODD) == E_SHAPE
    r = dict(sr_o=outer, sr_i=inner)
    assert _forward(_norm(out_dtype=out, **r), r=None, x=ODD) == E_ALIGN
    assert _forward(_norm(out_dtype=out, **r), x=ODD) == (E_SHAPE if inner < 0 or outer > 1 << 60 else E_ALIGN)


@pytest.mark.parametrize("outer,inner", STRIDES)
def test_backward(outer, inner):
    r = dict(sr_o=outer, sr_i=inner)
    assert _backward(_norm(**r), dh=None, h=ODD) == E_ALIGN
    assert _backward(_norm(**r), h=ODD) == (E_SHAPE if inner < 0 or outer > 1 << 60 else E_ALIGN)
    assert _backward(_norm(sh_o=outer, sh_i=inner), h=ODD) == E_SHAPE
