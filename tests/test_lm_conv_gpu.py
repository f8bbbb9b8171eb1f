"""The short causal convolution on the GPU against its definition in 64 bits."""
import pytest

import lm_ref as ref
from lm_ref import ROUND, TINY, U, rand

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


def make(seed, B, T, C, K, dtype):
    x = rand(seed, (B, T, C + 9), dtype).cuda()[..., 5:5 + C]
    return x, rand(seed + 1, (C, K), dtype, 0.6).cuda(), rand(seed + 2, (C,), dtype).cuda()


def check_forward(y, x, w, bias, silu, state=None, lengths=None, last=None):
    want, pre, size, tail = ref.conv(x, w, bias, silu, state, lengths)
    # A sum's error, what the SiLU makes of it (its slope is below 1.1), and the gate's own roundings.
    bound = want.abs() * ROUND[y.dtype] + U * (1.1 * size * (w.shape[1] + 2) + want.abs() * (2 * pre.abs() + 8)) + TINY
    ref.close(y, want, bound, "y")
    if last is not None:
        ref.close(last, tail, 0.0, "state")


def check_backward(got, x, w, bias, silu, dy, lengths=None):
    dx, dw, db, sx, sw, sb = ref.conv_backward(x, w, bias, silu, lengths, dy)
    K, n = w.shape[1], x.shape[0] * x.shape[1]
    ref.close(got[0], dx, dx.abs() * ROUND[x.dtype] + sx * U * (2 * K + 12) * (1 + ROUND[x.dtype]) + TINY, "dx")
    ref.close(got[1], dw, dw.abs() * ROUND[got[1].dtype] + sw * U * (2 * K + 12 + n) + TINY, "dw")
    if bias is None:
        assert got[2] is None
    else:
        ref.close(got[2], db, db.abs() * ROUND[got[2].dtype] + sb * U * (2 * K + 12 + n) + TINY, "db")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [1, 2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("B,T,C", [(1, 1, 1), (2, 3, 5), (1, 16, 64), (3, 17, 70), (2, 40, 520), (1, 65, 2100), (5, 33, 24)])
def test_forward_and_backward(swr, dtype, K, B, T, C):
    x, w, bias = make(1, B, T, C, K, dtype)
    dy = rand(9, (B, T, C + 2), dtype).cuda()[..., 1:1 + C]
    for silu, b in ((True, bias), (False, None)):
        y, none = swr.swr_causal_conv(x, w, b, silu)
        assert none is None
        check_forward(y, x, w, b, silu)
        got = swr.swr_causal_conv_backward(x, w, dy, b, silu)
        check_backward(got, x, w, b, silu, dy)
        again = swr.swr_causal_conv_backward(x, w, dy, b, silu)
        assert all(p is q or torch.equal(p, q) for p, q in zip(got, again))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [1, 4, 8])
@pytest.mark.parametrize("lengths", [[0, 1, 2, 20], [7, 33, -1, 3], [16, 17, 500, 32]])
def test_lengths_and_state(swr, dtype, K, lengths):
    B, T, C = 4, 33, 40
    x, w, bias = make(2, B, T, C, K, dtype)
    dy = rand(10, (B, T, C), dtype).cuda()
    for i, n in enumerate(lengths):
        x[i, max(n, 0):], dy[i, max(n, 0):] = float("nan"), float("inf")
    state, n = rand(11, (B, K - 1, C), dtype).cuda(), torch.tensor(lengths, dtype=torch.int32).cuda()
    for s in (None, state):
        y, last = swr.swr_causal_conv(x, w, bias, state=s, lengths=n, want_state=True)
        check_forward(y, x, w, bias, True, s, n, last)
    kept = state.clone()
    y2, out = swr.swr_causal_conv(x, w, bias, state=kept, lengths=n, state_out=kept)
    assert out is kept and torch.equal(kept, last) and torch.equal(y, y2)
    check_backward(swr.swr_causal_conv_backward(x, w, dy, bias, lengths=n), x, w, bias, True, dy, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K,C", [(4, 70), (2, 512), (1, 8), (8, 33)])
def test_tokens_one_by_one(swr, dtype, K, C):
    B, T = 3, 12
    x, w, bias = make(3, B, T, C, K, dtype)
    want, _ = swr.swr_causal_conv(x, w, bias)
    y, state = swr.swr_causal_conv(x[:, :2], w, bias, want_state=True)
    ys = [y]
    for t in range(2, T):
        if t % 2:
            yt = torch.empty(B, 2 * C, dtype=dtype, device="cuda")[:, C:]
            assert swr.swr_causal_conv_step(x[:, t], w, state, bias, y=yt) is yt
        else:
            yt = swr.swr_causal_conv_step(x[:, t], w, state, bias)
        ys.append(yt[:, None])
    assert torch.equal(torch.cat(ys, 1), want)
    check_forward(want, x, w, bias, True)


def test_long_sequences(swr):
    """Several turns of a block over its runs."""
    x, w, bias = make(4, 3, 3001, 8, 4, BF16)
    dy = rand(12, x.shape, BF16).cuda()
    check_forward(swr.swr_causal_conv(x, w, bias)[0], x, w, bias, True)
    check_backward(swr.swr_causal_conv_backward(x, w, dy, bias), x, w, bias, True, dy)
    x, w, bias = make(5, 2, 9000, 1100, 2, F32)
    dy = rand(13, x.shape, F32).cuda()
    check_backward(swr.swr_causal_conv_backward(x, w, dy, bias), x, w, bias, True, dy)


def test_outputs_in_place_and_layouts(swr):
    B, T, C, K = 2, 20, 48, 4
    x, w, bias = make(6, B, T, C, K, BF16)
    want, _ = swr.swr_causal_conv(x, w, bias)
    wide = torch.full((B, T, 3 * C), 5.0, dtype=BF16, device="cuda")
    y, _ = swr.swr_causal_conv(x, w, bias, y=wide[..., C:2 * C])
    assert torch.equal(y, want) and (wide[..., :C] == 5).all() and (wide[..., 2 * C:] == 5).all()
    one = x[:1].expand(3, T, C)
    assert torch.equal(swr.swr_causal_conv(one, w, bias)[0][2], want[0])
    dy = rand(14, (T, B, C), BF16).cuda().transpose(0, 1)
    dx = torch.full((B, T, 2 * C), 5.0, dtype=BF16, device="cuda")
    got = swr.swr_causal_conv_backward(x, w, dy, bias, dx=dx[..., C:],
                                       workspace=torch.empty(1 << 16, dtype=torch.uint8, device="cuda"))
    check_backward(got, x, w, bias, True, dy)
    assert (dx[..., :C] == 5).all()
    with pytest.raises(ValueError):
        swr.swr_causal_conv(x.transpose(1, 2).contiguous().transpose(1, 2), w, bias)
    with pytest.raises(ValueError):
        swr.swr_causal_conv(x, w.t().contiguous().t(), bias)
    with pytest.raises(swr.SwrError):
        swr.swr_causal_conv(x, w, bias, y=x)
    with pytest.raises(swr.SwrError):
        swr.swr_causal_conv(x, rand(1, (C, 9), BF16).cuda(), bias)


def test_saturated_gates(swr):
    """Sums so large that the SiLU is the identity or zero, and infinite ones."""
    x = torch.tensor([-3e38, -200.0, -90.0, -1e-30, 0.0, 1e-30, 90.0, 200.0, 3e38], device="cuda").reshape(1, -1, 1)
    w = torch.ones(1, 1, device="cuda")
    y, _ = swr.swr_causal_conv(x, w)
    check_forward(y, x, w, None, True)
    dy = torch.ones_like(x)
    dx, dw, _ = swr.swr_causal_conv_backward(x[:, 1:-1].contiguous(), w, dy[:, 1:-1].contiguous())
    want = ref.conv_backward(x[:, 1:-1], w, None, True, None, dy[:, 1:-1])
    ref.close(dx, want[0], want[3] * U * 32 + TINY, "dx")


def test_nothing(swr):
    w, bias = rand(1, (6, 4), F32).cuda(), rand(2, (6,), F32).cuda()
    state = rand(3, (2, 3, 6), F32).cuda()
    x = torch.zeros(2, 0, 6, device="cuda")
    y, last = swr.swr_causal_conv(x, w, bias, state=state, want_state=True)
    assert y.shape == (2, 0, 6) and torch.equal(last, state)
    dx, dw, db = swr.swr_causal_conv_backward(x, w, x, bias)
    assert dx.shape == x.shape and (dw == 0).all() and (db == 0).all()
    x = torch.zeros(0, 5, 6, device="cuda")
    assert swr.swr_causal_conv(x, w, bias)[0].shape == (0, 5, 6)
    dx, dw, db = swr.swr_causal_conv_backward(x, w, x, bias)
    assert (dw == 0).all() and (db == 0).all()


def test_autograd(swr):
    B, T, C, K = 2, 19, 20, 4
    x, w, bias = (t.detach().clone().requires_grad_(True) for t in make(7, B, T, C, K, F32))
    n = torch.tensor([19, 11], dtype=torch.int32).cuda()
    y = swr.SWRCausalConvFunction.apply(x, w, bias, True, n)
    for dy in (rand(15, (B, T, C), F32).cuda(), rand(16, (1, 1, C), F32).cuda().expand(B, T, C),
               rand(17, (B, C, T), F32).cuda().transpose(1, 2)):
        got = torch.autograd.grad(y, (x, w, bias), dy, retain_graph=True)
        check_backward(got, x.detach(), w.detach(), bias.detach(), True, dy, n)
    x16, w16 = x.detach().to(BF16).requires_grad_(True), w.detach().to(BF16).requires_grad_(True)
    y = swr.SWRCausalConvFunction.apply(x16, w16)
    dy = rand(18, (B, T, C), BF16).cuda()
    dx, dw = torch.autograd.grad(y, (x16, w16), dy)
    assert dw.dtype == BF16
    check_backward((dx, dw, None), x16.detach(), w16.detach(), None, True, dy)


@pytest.mark.parametrize("seed", range(12))
def test_mixed_shapes(swr, seed):
    """Shapes and options drawn at random; lengths, the state in place, NaN past the lengths."""
    import random
    rng = random.Random(seed)
    B, T, C, K = rng.randint(1, 9), rng.choice((1, 2, rng.randint(1, 150))), rng.randint(1, 600), rng.randint(1, 8)
    dtype, silu = rng.choice((BF16, F32)), rng.random() < 0.7
    x, w, bias = make(60 + seed, B, T, C, K, dtype)
    lengths = torch.tensor([rng.randint(0, T) for _ in range(B)], dtype=torch.int32).cuda()
    for i, n in enumerate(lengths.tolist()):
        x[i, n:] = float("nan")
    state = rand(80, (B, K - 1, C), dtype).cuda()
    before = state.clone()
    y, last = swr.swr_causal_conv(x, w, bias, silu, state, lengths, state_out=state)
    assert last is state
    check_forward(y, x, w, bias, silu, before, lengths, state)
    dy = rand(81, (B, T, C), dtype).cuda()
    for i, n in enumerate(lengths.tolist()):
        dy[i, n:] = float("inf")
    check_backward(swr.swr_causal_conv_backward(x, w, dy, bias, silu, lengths), x, w, bias, silu, dy, lengths)
