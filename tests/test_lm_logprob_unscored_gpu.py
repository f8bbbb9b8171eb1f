"""Rows that nothing is learned from (gradients of zero) have a gradient of zero, however far their
logits are from zero."""
import pytest

import lm_ref as ref
from lm_ref import ROUND, U, rand

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


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", [5, 3000, 9001])
@pytest.mark.parametrize("scale", [0.3, 0.7, 0.9, 1.0, 1.1, 1.3, 3.7])
def test_far_rows_without_a_gradient(swr, dtype, vocab, scale):
    low = torch.finfo(dtype).min
    base = torch.tensor([low, low * 0.77, low / 1000, -1e30, -1e12, -5e9, -7e4, 0.0, 7e4, 5e9, 1e12, 1e30, -low / 1000, -low * 0.77])
    x = (base[:, None] + rand(1, (len(base), vocab), F32)).clamp(low, -low).to(dtype).cuda()
    x[:, 1] = float("-inf")
    n = len(base)
    tokens = (torch.arange(n) % 5).cuda()
    _, lse, entropy = swr.swr_log_probs(x, tokens, scale=scale)
    zero, g = torch.zeros(n, device="cuda"), rand(2, (n,), F32).cuda()
    for dlogp, dlse, dentropy in ((zero, None, None), (zero, zero, zero), (None, None, None), (None, -zero, zero)):
        d = swr.swr_log_probs_backward(x, tokens, lse, entropy, dlogp, dentropy, dlse, scale)
        assert (d == 0).all()
    # Padding: its dlogp counts for nothing.
    none = torch.full((n,), -1, device="cuda")
    assert (swr.swr_log_probs_backward(x, none, lse, entropy, g, scale=scale) == 0).all()
    # p's parts cancel where dlse = dlogp: what is left is the token's own.
    d = swr.swr_log_probs_backward(x, tokens, lse, entropy, g, None, g, scale)
    want = torch.zeros(n, vocab, dtype=torch.float64).scatter_(1, tokens.cpu()[:, None], scale * ref.f64(g)[:, None])
    ref.close(d, want, want.abs() * (ROUND[dtype] + 2 * U), "dlogits")
