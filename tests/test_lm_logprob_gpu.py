"""Log probabilities, entropy, alternatives and the logits' gradient on the GPU against
their definitions in 64 bits."""
import pytest

import lm_ref as ref
from lm_ref import ROUND, TINY, U, rand

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def _tokens(seed, shape, vocab, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(-1, vocab + 1, shape, generator=g).to(dtype).cuda()


def check(got, logits, tokens, scale=1.0, top=0):
    logp, lse, entropy = got[:3]
    want = ref.log_probs(logits, tokens, scale)
    V = logits.shape[-1]
    z = ref.f64(logits) * scale
    most = torch.where(torch.isfinite(z), z.abs(), 0.0).max(-1).values
    # Of an exponent (the distance from the largest logit, two products) and of a sum of V terms, in
    # any grouping of its additions, each rescaled at most once for a tile of a thread and for a join.
    logs = torch.where(torch.isfinite(want[3]), want[3].abs(), 0.0)
    p = torch.where(torch.isfinite(want[3]), torch.exp(want[3]), 0.0)
    spread = (p * logs).sum(-1)
    total = V + 64 + 8 * (spread + 40)
    ref.close(lse, want[1], U * (total + 3 * most + 4), "lse")
    fine = want[0].abs().nan_to_num(0, 0, 0)
    ref.close(logp, want[0], U * (total + 4 * fine + 4) + TINY, "logp")
    ref.close(entropy, want[2], U * (2 * total + 8) * (1 + spread + torch.log(torch.tensor(float(V)))) + TINY, "entropy")
    if top:
        order = ref.top_tokens(logits, top)
        assert got[4].dtype == torch.int64 and torch.equal(got[4].cpu(), order)
        best = torch.gather(want[3], -1, order)
        ref.close(got[3], best, U * (total[..., None] + 4 * best.abs().nan_to_num(0, 0, 0) + 4) + TINY, "top_logp")


SIZES = [(1, 1), (3, 2), (5, 7), (2, 64), (4, 65), (9, 257), (3, 2048), (2, 2049), (3, 5000), (2, 16384), (2, 16385),
         (2, 40001), (1, 131072), (1, 140001)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", SIZES)
def test_forward(swr, dtype, rows, vocab):
    logits, tokens = rand(1, (rows, vocab), dtype, 3.0).cuda(), _tokens(2, (rows,), vocab)
    plain = swr.swr_log_probs(logits, tokens)
    assert len(plain) == 3
    check(plain, logits, tokens)
    for top in sorted({1, min(5, vocab), min(20, vocab), min(64, vocab)}):
        got = swr.swr_log_probs(logits, tokens, top=top)
        check(got, logits, tokens, top=top)
    check(swr.swr_log_probs(logits, tokens.int(), scale=0.37), logits, tokens, 0.37)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [70, 3000, 20000, 131072])
def test_orders_and_ties(swr, dtype, vocab):
    """Rows sorted up and down, all equal, of few values, and of large ones next to each other."""
    rows = torch.stack([torch.linspace(-9, 9, vocab), torch.linspace(9, -9, vocab), torch.full((vocab,), 0.25),
                        (torch.arange(vocab) * 7919 % 5).float(), 1000 + (torch.arange(vocab) % 3).float() * 4,
                        torch.where(torch.arange(vocab) == vocab - 1, 40.0, -40.0),
                        torch.where(torch.arange(vocab) % 2 == 0, 0.0, -0.0)]).to(dtype).cuda()
    tokens = _tokens(3, (7,), vocab)
    for top in (1, 20, 64):
        check(swr.swr_log_probs(rows, tokens, top=top), rows, tokens, top=top)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [10, 2048, 9000, 40000, 131073])
def test_masked_rows(swr, dtype, vocab):
    """Logits of -infinity, rows of nothing else, of a type's lowest value, NaN and +infinity."""
    low = torch.finfo(dtype).min
    x = rand(4, (9, vocab), dtype, 2.0)
    x[0, : vocab - 3] = -INF
    x[1] = -INF
    x[2, 2:] = low
    x[3] = low
    x[4, vocab // 2] = NAN
    x[5, vocab - 1] = INF
    x[6] = -INF
    x[6, vocab - 1] = NAN
    x[7] = -INF
    x[7, 3] = low
    x = x.cuda()
    tokens = torch.tensor([vocab - 1, 0, 5, 7, 1, 2, vocab - 1, 3, -1]).cuda()
    got = swr.swr_log_probs(x, tokens, top=8)
    # (of a row that holds NaN or +infinity the alternatives' tokens are as defined, their values NaN)
    check(got, x, tokens, top=8)
    zeros = torch.zeros(9, device="cuda")
    g = rand(5, (9,), F32).cuda()
    d = swr.swr_log_probs_backward(x, tokens, got[1], got[2], g, g, zeros)
    assert (d[1] == 0).all() and torch.isnan(d[4]).all() and torch.isnan(d[5]).all()
    assert torch.isfinite(d[0]).all() and (d[0, :vocab - 3] == 0).all()
    assert torch.isfinite(d[2]).all() and (d[2, 2:5] == 0).all()
    want, size = ref.log_probs_backward(x[[0, 8]], tokens[[0, 8]], 1.0, g[[0, 8]], zeros[[0, 8]], g[[0, 8]])
    ref.close(d[[0, 8]], want, want.abs() * ROUND[dtype] + size * U * (4 * vocab + 400) + TINY, "d")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,vocab", [(1, 1), (3, 5), (7, 300), (2, 5000), (70, 130), (3, 40001)])
def test_gradient(swr, dtype, rows, vocab):
    logits, tokens = rand(6, (rows, vocab), dtype, 3.0).cuda(), _tokens(7, (rows,), vocab)
    a, b, c = (rand(i, (rows,), F32).cuda() for i in (8, 9, 10))
    for scale in (1.0, 1.7):
        logp, lse, entropy = swr.swr_log_probs(logits, tokens, scale=scale)
        for dlogp, dlse, dentropy in ((a, None, None), (None, b, None), (None, None, c), (a, b, c), (None, None, None)):
            want, size = ref.log_probs_backward(logits, tokens, scale, dlogp, dlse, dentropy)
            most = float((ref.f64(logits) * scale).abs().max())
            # p's exponent has lse's error (a sum of vocab terms, its own rounding) and the products'.
            bound = want.abs() * ROUND[dtype] + size * U * (2 * vocab + 8 * most + 500) * (1 + ROUND[dtype]) + TINY
            d = swr.swr_log_probs_backward(logits, tokens, lse, entropy, dlogp, dentropy, dlse, scale)
            ref.close(d, want, bound, "dlogits")
        place = logits.clone()
        assert swr.swr_log_probs_backward(place, tokens, lse, entropy, a, c, b, scale, dlogits=place) is place
        assert torch.equal(place, swr.swr_log_probs_backward(logits, tokens, lse, entropy, a, c, b, scale))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [9, 5000, 40001])
def test_gradient_far_out(swr, dtype, vocab):
    """Rows whose lse holds nothing, or little, of what p goes by: all of a type's lowest value, or far from zero."""
    low, up = torch.finfo(dtype).min, rand(30, (vocab,), F32, 2.0)
    x = torch.stack([torch.full((vocab,), low), torch.full((vocab,), low), up * 8 - 70000, up + 5000, up - 255, up,
                     torch.full((vocab,), -low)])
    x[1, vocab // 2] = low / 2
    x = x.to(dtype).cuda()
    tokens = torch.tensor([3, 0, 1, vocab - 1, 2, -1, 7]).cuda()
    a, b, c = (rand(i, (7,), F32).cuda() for i in (31, 32, 33))
    _, lse, entropy = swr.swr_log_probs(x, tokens)
    for dlogp, dlse, dentropy in ((a, None, None), (a, b, c), (None, None, None)):
        want, size = ref.log_probs_backward(x, tokens, 1.0, dlogp, dlse, dentropy)
        # As above, with an lse of at most 256 (farther out p goes by the distance from the row's largest logit).
        bound = want.abs() * ROUND[dtype] + size * U * (2 * vocab + 8 * 256 + 500) * (1 + ROUND[dtype]) + TINY
        d = swr.swr_log_probs_backward(x, tokens, lse, entropy, dlogp, dentropy, dlse)
        ref.close(d, want, bound, "dlogits")
        place = x.clone()
        assert torch.equal(swr.swr_log_probs_backward(place, tokens, lse, entropy, dlogp, dentropy, dlse, dlogits=place), d)


def test_layouts(swr):
    """Rows that are parts of wider ones, at odd addresses, and leading dimensions."""
    wide = rand(11, (3, 4, 3011), BF16).cuda()
    logits, tokens = wide[..., 5:3006], _tokens(12, (3, 4), 3001)
    got = swr.swr_log_probs(logits, tokens, top=3)
    assert got[0].shape == (3, 4) and got[3].shape == (3, 4, 3)
    check(got, logits, tokens, top=3)
    out = torch.full((3, 4, 3100), 4.0, dtype=BF16, device="cuda")
    g = rand(13, (3, 4), F32).cuda()
    d = swr.swr_log_probs_backward(logits, tokens, got[1], got[2], g, dlogits=out[..., 7:3008])
    want, size = ref.log_probs_backward(logits, tokens, 1.0, g, None, None)
    ref.close(d, want, want.abs() * ROUND[BF16] + size * U * 8000 + TINY, "d")
    assert (out[..., :7] == 4).all() and (out[..., 3008:] == 4).all()
    one = logits[:1, :1].expand(3, 1, 3001)   # the same row for all
    check(swr.swr_log_probs(one, tokens[:, :1].contiguous()), one, tokens[:, :1])


def test_many_rows(swr):
    """More rows than a launch has blocks for at once, of every kind of block."""
    for rows, vocab in ((40000, 3), (5000, 2100), (700, 17000)):
        logits, tokens = rand(14, (rows, vocab), BF16, 2.0).cuda(), _tokens(15, (rows,), vocab)
        check(swr.swr_log_probs(logits, tokens), logits, tokens)


def test_nothing(swr):
    got = swr.swr_log_probs(torch.zeros(0, 5, device="cuda"), torch.zeros(0, dtype=torch.int64, device="cuda"), top=2)
    assert [tuple(t.shape) for t in got] == [(0,), (0,), (0,), (0, 2), (0, 2)]


def test_autograd(swr):
    logits = rand(16, (6, 50), F32, 2.0).cuda().requires_grad_(True)
    tokens = _tokens(17, (6,), 50)
    a, b, c = (rand(i, (6,), F32).cuda() for i in (18, 19, 20))
    logp, lse, entropy = swr.SWRLogProbsFunction.apply(logits, tokens, 0.8)
    for pick in ((a, b, c), (a, None, None), (None, b, None), (None, None, c)):
        chosen = [(o, g) for o, g in zip((logp, lse, entropy), pick) if g is not None]
        d, = torch.autograd.grad([o for o, _ in chosen], logits, [g for _, g in chosen], retain_graph=True)
        want, size = ref.log_probs_backward(logits, tokens, 0.8, *pick)
        ref.close(d, want, want.abs() * ROUND[F32] + size * U * 800 + TINY, "dlogits")
    d, = torch.autograd.grad(-logp.mean(), logits)   # an expanded gradient
    want, size = ref.log_probs_backward(logits, tokens, 0.8, torch.full((6,), -1 / 6), None, None)
    ref.close(d, want, want.abs() * ROUND[F32] + size * U * 800 + TINY, "dlogits")


def test_refusals(swr):
    logits, tokens = rand(21, (4, 30), F32).cuda(), _tokens(22, (4,), 30)
    for bad in (lambda: swr.swr_log_probs(logits, tokens, top=65), lambda: swr.swr_log_probs(logits, tokens, top=31),
                lambda: swr.swr_log_probs(logits, tokens, top=-1), lambda: swr.swr_log_probs(logits, tokens, scale=NAN),
                lambda: swr.swr_log_probs(logits, tokens[:3]), lambda: swr.swr_log_probs(logits.t(), tokens),
                lambda: swr.swr_log_probs(logits, tokens.cpu()), lambda: swr.swr_log_probs(logits.cpu(), tokens.cpu())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: swr.swr_log_probs(logits, tokens, scale=0.0), lambda: swr.swr_log_probs(logits, tokens, scale=-1.0)):
        with pytest.raises(swr.SwrError):
            bad()
    with pytest.raises(TypeError):
        swr.swr_log_probs(logits, tokens.float())
