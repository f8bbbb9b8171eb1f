"""The norm under autograd: with and without a residual, and with gradients of any
layout that autograd passes, against the 64-bit form."""
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


def _layouts(shape, dtype):
    """Gradients of a shape as autograd passes them: expanded, transposed, of steps and
    in an order whose rows are no run."""
    yield "expanded", _rand(10, (1,) * len(shape), dtype).expand(shape)
    yield "a row for all", _rand(11, shape[-1:], dtype).expand(shape)
    yield "a value a row", _rand(12, (*shape[:-1], 1), dtype).expand(shape)
    yield "transposed", _rand(13, (*shape[:-2], shape[-1], shape[-2]), dtype).transpose(-1, -2)
    yield "every second channel", _rand(14, (*shape[:-1], 2 * shape[-1]), dtype)[..., ::2]
    if len(shape) > 2:
        yield "batch inside", _rand(15, (*shape[1:-1], shape[0], shape[-1]), dtype).movedim(-2, 0)
    if len(shape) == 4:
        yield "swapped", _rand(16, (shape[2], shape[1], shape[0], shape[3]), dtype).permute(2, 1, 0, 3)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(6, 40), (2, 5, 64), (3, 2, 4, 48)])
@pytest.mark.parametrize("with_residual", [True, False])
def test_gradients_of_any_layout(swr, dtype, shape, with_residual):
    x, w = _rand(17, shape, dtype).requires_grad_(True), _rand(18, shape[-1:], dtype).requires_grad_(True)
    r = _rand(19, shape, dtype) if with_residual else None
    dense = _rand(20, shape, dtype)
    for what, g in _layouts(shape, dtype):
        for gy, gh in ((g, dense), (dense, g), (g, g)):
            y, h = swr.SWRNormFunction.apply(x, w, r)
            dx, dw = torch.autograd.grad((y, h), (x, w), (gy, gh))
            y, h = swr.SWRNormFunction.apply(x, w, r)
            want = torch.autograd.grad((y, h), (x, w), (gy.contiguous(), gh.contiguous()))
            assert torch.equal(dx, want[0]) and torch.equal(dw, want[1]), what
            _check_gradients(h.detach(), w.detach(), gy, gh, dx, dw)


@pytest.mark.parametrize("loss", [lambda y, h: y.sum(), lambda y, h: h.mean(), lambda y, h: y.sum() + h.sum(),
                                  lambda y, h: (y.transpose(0, 1) @ h).sum()])
def test_ordinary_losses(swr, loss):
    x, r, w = (_rand(i, s, F32).requires_grad_(True) for i, s in ((21, (7, 33)), (22, (7, 33)), (23, (33,))))
    y, h = swr.SWRNormFunction.apply(x, w, r)
    loss(y, h).backward()
    plain = [t.detach().double().requires_grad_(True) for t in (x, w, r)]
    s = plain[0] + plain[2]
    loss(s * torch.rsqrt(s.square().mean(-1, keepdim=True) + 1e-6) * plain[1], s).backward()
    for got, want in zip((x, w, r), plain):
        want = torch.zeros_like(want) if want.grad is None else want.grad     # (h does not depend on the weight)
        # sums of 33 or 7 float32 terms of a few units, of a product of two matrices at most
        assert (got.grad.double() - want).abs().max() <= 2e-5 * (1 + want.abs().max())
