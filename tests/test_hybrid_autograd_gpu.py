"""The norm under autograd: with and without a residual, against the 64-bit
form."""
import pytest

import hybrid_ref as ref
from hybrid_ref import ROUND, TINY, U
from test_hybrid_norm_gpu import _rand, _terms

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def _check_gradients(h, w, dy, dh, dx, dw):
    """dx and dw against the formula's, with the bounds that the direct calls keep."""
    dtype, width, rows = h.dtype, h.shape[-1], h.numel() // h.shape[-1]
    flat = [t.reshape(rows, width) for t in (h, dy, dh)]
    want_x, want_w, size_x, size_w = ref.norm_backward(flat[0], w, flat[1], flat[2], 1e-6)
    ref.close(dx.reshape(rows, width), want_x, want_x.abs() * ROUND[dtype] + size_x * U * (2 * _terms(width) + 16) + TINY,
              "dx")
    ref.close(dw, want_w, want_w.abs() * ROUND[w.dtype] + size_w * U * (rows + _terms(width) + 64) + TINY, "dw")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(2, 96), (2, 3, 64), (1, 40), (5, 100)])
def test_without_a_residual(swr, dtype, shape):
    # (two leading rows: the case in which a lone y would be taken for a pair)
    x, w = _rand(1, shape, dtype).requires_grad_(True), _rand(2, shape[-1:], dtype).requires_grad_(True)
    gy, gh = _rand(3, shape, dtype), _rand(4, shape, dtype)
    y, h = swr.SWRNormFunction.apply(x, w, None)
    assert y.shape == h.shape == x.shape
    assert torch.equal(y, swr.swr_rms_norm(x.detach(), w.detach())) and torch.equal(h, x)
    dx, dw = torch.autograd.grad((y, h), (x, w), (gy, gh))
    _check_gradients(x.detach(), w.detach(), gy, gh, dx, dw)
    y, h = swr.SWRNormFunction.apply(x, w, None, 1e-6)
    dx, dw = torch.autograd.grad(y, (x, w), gy)
    _check_gradients(x.detach(), w.detach(), gy, torch.zeros_like(gy), dx, dw)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(2, 96), (2, 3, 64)])
def test_with_a_residual(swr, dtype, shape):
    x, r, w = (_rand(i, s, dtype).requires_grad_(True) for i, s in ((5, shape), (6, shape), (7, shape[-1:])))
    gy, gh = _rand(8, shape, dtype), _rand(9, shape, dtype)
    y, h = swr.SWRNormFunction.apply(x, w, r)
    dx, dr, dw = torch.autograd.grad((y, h), (x, r, w), (gy, gh))
    _check_gradients(h.detach(), w.detach(), gy, gh, dx, dw)
    assert torch.equal(dx, dr)
