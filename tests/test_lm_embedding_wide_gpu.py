"""The embedding's gradient of rows wider than a block takes at a time, of tokens that go on over
windows of positions."""
import pytest

from test_lm_embedding_gpu import _check, _tokens, swr  # noqa: F401  (a fixture)
from lm_ref import rand

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["one", "words", "any"])
@pytest.mark.parametrize("n,vocab,width", [(1001, 503, 1001), (500, 3, 2056), (300, 5, 4100), (70, 2, 513), (4100, 40, 1030)])
def test_gradient(swr, dtype, kind, n, vocab, width):  # noqa: F811
    t, dy = _tokens(21, n, vocab, kind), rand(22, (n, width), dtype).cuda()
    d = _check(swr, t, dy, vocab, 1.5)
    assert torch.equal(d, swr.swr_embedding_backward(t, dy, vocab, 1.5))
    _check(swr, t, dy, vocab, 1.5, dtype)
