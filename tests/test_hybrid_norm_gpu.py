"""Residual addition and root-mean-square norm against its 64-bit form: types,
widths on both sides of every plan's edge, strides, 8-bit rows, rows of zeros,
infinities and NaN, and the gradient by the formula and by differences."""
import pytest

import hybrid_ref as ref
from hybrid_ref import ROUND, TINY, U

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


def _rand(seed, shape, dtype, size=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * size).to(dtype).cuda()


# Terms that a float32 sum over a row adds one after another are at most 32 a
# thread, 6 steps in a wave and 16 waves; wide rows add width / 1024 a thread.
def _terms(width):
    return 32 + 6 + 16 + width / 1024 + 8


def _check_forward(swr, x, w, r, eps=1e-6, **kw):
    y, h64, _ = ref.norm(x, r, w, eps)
    got = swr.swr_rms_norm(x, w, residual=r, eps=eps, **kw)
    torch.cuda.synchronize()
    gy, gh = got if r is not None else (got, None)
    assert gy.dtype == x.dtype
    ref.close(gy, y, y.abs() * (ROUND[x.dtype] + U * _terms(x.shape[-1])) + TINY, "y")
    if gh is not None:
        want = (x.float() + r.float()).to(x.dtype)
        assert torch.equal(gh, want), "h is the float32 sum, rounded once"


WIDTHS = [1, 2, 3, 7, 8, 64, 100, 255, 512, 513, 1000, 2048, 2049, 4099, 8192, 8200, 16384, 16390, 32768, 40003]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", WIDTHS)
def test_forward(swr, dtype, width):
    for rows, seed in ((1, 1), (5, 2), (259, 3)):
        if rows * width > 1 << 22:
            continue
        x, r = _rand(seed, (rows, width), dtype), _rand(seed + 10, (rows, width), dtype, 3.0)
        w = _rand(seed + 20, (width,), dtype)
        _check_forward(swr, x, w, r)
        _check_forward(swr, x, w, None)
        _check_forward(swr, x, w.float(), r, eps=0.25)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [96, 1500, 5000, 40003])
def test_strides_and_in_place(swr, dtype, width):
    big = _rand(4, (3, 2, 5, width + 3), dtype)
    x, r = big[:, 0, :, 1:width + 1], big[:, 1, :, 3:]          # unaligned rows, two strides
    w = _rand(5, (width,), dtype)
    _check_forward(swr, x, w, r)
    _check_forward(swr, x.transpose(0, 1), w, r.transpose(0, 1))
    want_y, want_h = swr.swr_rms_norm(x, w, residual=r)
    for target in ("x", "r"):
        c = big.clone()
        x2, r2 = c[:, 0, :, 1:width + 1], c[:, 1, :, 3:]
        y, h = swr.swr_rms_norm(x2, w, residual=r2, h=x2 if target == "x" else r2)
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(h, want_h)
        other, was = (r2, r) if target == "x" else (x2, x)
        assert torch.equal(other, was)
    y = torch.full((3, 5, width + 5), 7.0, dtype=dtype, device="cuda")
    swr.swr_rms_norm(x, w, residual=r, y=y[..., 2:width + 2])
    torch.cuda.synchronize()
    assert torch.equal(y[..., 2:width + 2], want_y) and (y[..., :2] == 7).all() and (y[..., width + 2:] == 7).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [1, 5, 130, 2048, 2051, 9000, 33000])
def test_eight_bits(swr, dtype, width):
    x, r, w = _rand(6, (7, width), dtype), _rand(7, (7, width), dtype), _rand(8, (width,), dtype)
    x[2], r[2] = 0, 0
    q, scale, h = swr.swr_rms_norm(x, w, residual=r, fp8=True)
    torch.cuda.synchronize()
    assert q.dtype == torch.float8_e4m3fn and scale.shape == (7,) and scale.dtype == F32
    assert torch.equal(h, (x.float() + r.float()).to(dtype))
    y, _, _ = ref.norm(x, r, w, 1e-6)
    s = y.abs().amax(-1) / 448
    room = 1 + U * (_terms(width) + 8)
    ref.close(scale, s, s * (room - 1), "scale")
    # nearest of 4 significant bits, or of the smallest steps of 2^-9
    ref.close(ref.f64(q.float()) * s[:, None], y, torch.maximum(y.abs() / 16, s[:, None] * 2.0 ** -10) * room + y.abs() * (room - 1) + TINY, "q")
    assert float(scale[2]) == 0 and (q[2].float() == 0).all()
    top = q.float().abs().amax(-1)
    assert all(float(top[i]) == 448 for i in range(7) if i != 2)


def test_eight_bits_of_the_smallest_rows(swr):
    # Scales below the normal floats: |y| up to 448 * 2^-130.
    x = _rand(9, (4, 300), F32)
    w = torch.full((300,), 2.0 ** -125, device="cuda")
    q, scale = swr.swr_rms_norm(x, w, fp8=True)
    torch.cuda.synchronize()
    y, _, _ = ref.norm(x, None, w, 1e-6)
    s = y.abs().amax(-1) / 448
    step = 2.0 ** -149
    ref.close(scale, s, s * 1e-5 + step, "scale")
    ref.close(q, (y / s[:, None]), torch.maximum((y / s[:, None]).abs() / 16, torch.tensor(2.0 ** -10, dtype=torch.float64)) * 1.001, "q")


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [40, 3000, 40000])
def test_infinities_and_nan_stay_in_their_rows(swr, dtype, fp8, width):
    x = _rand(10, (6, width), dtype)
    w = _rand(11, (width,), dtype)
    want = swr.swr_rms_norm(x, w, fp8=fp8)
    x2 = x.clone()
    x2[1, 3], x2[3, 7], x2[4, width - 1] = float("inf"), float("nan"), float("-inf")
    got = swr.swr_rms_norm(x2, w, fp8=fp8)
    torch.cuda.synchronize()
    clean = [0, 2, 5]
    if fp8:
        assert torch.equal(got[0].view(torch.uint8)[clean], want[0].view(torch.uint8)[clean])
        assert torch.equal(got[1][clean], want[1][clean]) and torch.isnan(got[1][[1, 3, 4]]).all()
    else:
        assert torch.equal(got[clean], want[clean])
        y, _, _ = ref.norm(x2, None, w, 1e-6)
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(y))
    zero = torch.zeros(2, width, dtype=dtype, device="cuda")
    assert (swr.swr_rms_norm(zero, w).float() == 0).all()                    # eps > 0
    assert torch.isnan(swr.swr_rms_norm(zero, w, eps=0.0).float()).all()     # 0 / 0


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [1, 3, 64, 100, 511, 513, 2048, 2050, 4096, 8193, 16384, 16391, 20000])
def test_backward(swr, dtype, width):
    for rows, seed in ((1, 1), (6, 2), (2600, 3)):
        if rows * width > 1 << 23:
            continue
        h, dy, dh = (_rand(seed + i, (rows, width), dtype) for i in range(3))
        for w, d in ((_rand(9, (width,), dtype), dh), (_rand(9, (width,), F32), None)):
            dx, dw = swr.swr_rms_norm_backward(h, w, dy, dh=d)
            again = swr.swr_rms_norm_backward(h, w, dy, dh=d)
            torch.cuda.synchronize()
            assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
            want_x, want_w, size_x, size_w = ref.norm_backward(h, w, dy, d, 1e-6)
            assert dx.dtype == dtype and dw.dtype == F32
            ref.close(dx, want_x, want_x.abs() * ROUND[dtype] + size_x * U * (2 * _terms(width) + 16) + TINY, "dx")
            # rows a block's thread adds, then up to 512 blocks in 16 parts
            ref.close(dw, want_w, size_w * U * (rows / 512 + 32 + 16 + _terms(width) + 16) + TINY, "dw")


def test_backward_strides_and_in_place(swr):
    for dtype, width in ((BF16, 500), (F32, 21), (BF16, 17000)):
        big = _rand(12, (4, 3, 3, width + 1), dtype)
        h, dy, dh = (big[:, i, :, i % 2:width + i % 2] for i in range(3))
        w = _rand(13, (width,), dtype)
        dx, dw = swr.swr_rms_norm_backward(h, w, dy, dh=dh)
        dense = swr.swr_rms_norm_backward(h.contiguous(), w, dy.contiguous(), dh=dh.contiguous())
        torch.cuda.synchronize()
        want_x, want_w, size_x, size_w = ref.norm_backward(h, w, dy, dh, 1e-6)
        ref.close(dx, want_x, want_x.abs() * ROUND[dtype] + size_x * U * (2 * _terms(width) + 16) + TINY, "dx")
        ref.close(dw, want_w, size_w * U * (_terms(width) + 64), "dw")
        assert torch.equal(dx, dense[0]) and torch.equal(dw, dense[1])
        for i in (1, 2):
            c = big.clone()
            h2, dy2, dh2 = (c[:, j, :, j % 2:width + j % 2] for j in range(3))
            out = (None, dy2, dh2)[i]
            got, gw = swr.swr_rms_norm_backward(h2, w, dy2, dh=dh2, dx=out)
            torch.cuda.synchronize()
            assert torch.equal(got, dx) and torch.equal(gw, dw)


def test_gradient_by_differences(swr):
    """The autograd function's gradients against differences of the 64-bit form."""
    x, r, w = _rand(14, (3, 37), F32), _rand(15, (3, 37), F32), _rand(16, (37,), F32)
    gy, gh = _rand(17, (3, 37), F32), _rand(18, (3, 37), F32)
    leaves = [t.clone().requires_grad_(True) for t in (x, w, r)]
    y, h = swr.SWRNormFunction.apply(leaves[0], leaves[1], leaves[2], 0.1)
    grads = torch.autograd.grad((y, h), leaves, (gy, gh))
    torch.cuda.synchronize()
    a, b = ref.f64(gy), ref.f64(gh)

    def loss(x, w, r):
        y, h, _ = ref.norm(x, r, w, 0.1)
        return float((y * a).sum() + (h * b).sum())

    step = 1e-5
    for i, g in enumerate(grads):
        args = [ref.f64(t) for t in (x, w, r)]
        base = args[i]
        for j in range(0, base.numel(), 5):
            up, down = base.clone(), base.clone()
            up.view(-1)[j] += step
            down.view(-1)[j] -= step
            d = (loss(*args[:i], up, *args[i + 1:]) - loss(*args[:i], down, *args[i + 1:])) / (2 * step)
            assert abs(float(g.reshape(-1)[j]) - d) <= 1e-4 * (1 + abs(d))   # (float32 sums of 37 terms of size 1)


def test_empty(swr):
    w = _rand(1, (24,), F32)
    x = torch.empty((0, 24), device="cuda")
    y, h = swr.swr_rms_norm(x, w, residual=x)
    assert y.shape == h.shape == (0, 24)
    dx, dw = swr.swr_rms_norm_backward(x, w, x)
    torch.cuda.synchronize()
    assert dx.shape == (0, 24) and (dw == 0).all()


def test_another_stream(swr):
    x, r, w = _rand(20, (300, 2048), BF16), _rand(21, (300, 2048), BF16), _rand(22, (2048,), BF16)
    y, h = swr.swr_rms_norm(x, w, residual=r)
    dx, dw = swr.swr_rms_norm_backward(h, w, x, dh=r)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        y2, h2 = swr.swr_rms_norm(x, w, residual=r, stream=s)
        dx2, dw2 = swr.swr_rms_norm_backward(h2, w, x, dh=r, stream=s)
        junk = [torch.full((1 << 16,), 3.0, device="cuda") for _ in range(8)]   # (what a freed workspace would become)
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(dx, dx2) and torch.equal(dw, dw2)
        del junk
