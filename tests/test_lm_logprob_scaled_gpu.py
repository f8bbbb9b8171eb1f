"""The logits' gradient where scale times the logits leaves float32, or is so far from zero
that lse holds nothing of what p goes by: against the definition in 64 bits."""
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


def _rows(dtype, vocab):
    """Rows of a type's lowest and largest value, with others among them, masked ones, and ordinary ones."""
    low, up = torch.finfo(dtype).min, rand(30, (vocab,), F32, 2.0)
    x = torch.stack([torch.full((vocab,), low), torch.full((vocab,), low), torch.full((vocab,), -low),
                     torch.full((vocab,), -low), torch.full((vocab,), low), torch.full((vocab,), -INF), up, up - 1000])
    x[1, vocab // 2] = low / 2
    x[3, 1:] = low
    x[4, : vocab // 2] = -INF
    return x.to(dtype).cuda(), torch.tensor([3, 0, vocab - 1, 0, vocab - 1, 2, -1, 5]).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [9, 5000, 40001])
@pytest.mark.parametrize("scale", [0.7, 1.25, 1.7, 64.0])
def test_gradient_past_the_range(swr, dtype, vocab, scale):
    x, tokens = _rows(dtype, vocab)
    a, b, c = (rand(i, (8,), F32).cuda() for i in (31, 32, 33))
    logp, lse, entropy = swr.swr_log_probs(x, tokens, scale=scale)
    want = ref.log_probs(x, tokens, scale)
    # lse itself, rounded to float32, may be infinite; what is taken from the largest logit is not.
    exact = want[1].to(F32)
    assert torch.equal(torch.isinf(lse.cpu()), torch.isinf(exact)) and not torch.isnan(lse).any()
    for dlogp, dlse, dentropy in ((a, None, None), (None, b, None), (a, b, c)):
        d = swr.swr_log_probs_backward(x, tokens, lse, entropy, dlogp, dentropy, dlse, scale)
        value, size = ref.log_probs_backward(x, tokens, scale, dlogp, dlse, dentropy)
        value[5] = 0.0   # (a row of nothing but -infinity has no gradient, its token's neither)
        # As of ordinary rows: a sum of vocab terms, an exponent of at most 256 by lse or the distance from the
        # row's largest logit (p is 0 below 2^-160), the products' own.
        bound = value.abs() * ROUND[dtype] + size * U * (2 * vocab + 8 * 256 + 500) * (1 + ROUND[dtype]) + TINY
        ref.close(d, value, bound, "dlogits")
        place = x.clone()
        assert torch.equal(swr.swr_log_probs_backward(place, tokens, lse, entropy, dlogp, dentropy, dlse, scale,
                                                      dlogits=place), d)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [1.25, 1.7])
def test_not_a_number_past_the_range(swr, dtype, scale):
    """NaN and +infinity in such a row make its gradient NaN, as in any other."""
    x, tokens = _rows(dtype, 3000)
    x[0, 7], x[2, 2999], x[4, 0] = NAN, INF, NAN
    _, lse, entropy = swr.swr_log_probs(x, tokens, scale=scale)
    d = swr.swr_log_probs_backward(x, tokens, lse, entropy, torch.ones(8, device="cuda"), scale=scale)
    nan = torch.isnan(d)
    assert nan[[0, 2, 4]].all() and not nan[[1, 3, 5, 6, 7]].any()
