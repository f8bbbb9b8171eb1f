"""Token embedding and its gradient on the GPU against their definitions in 64 bits."""
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


def _tokens(seed, n, vocab, kind, dtype=torch.int64):
    g = torch.Generator().manual_seed(seed)
    if kind == "one":
        t = torch.full((n,), min(3, vocab - 1))
    elif kind == "words":
        t = (vocab ** torch.rand(n, generator=g, dtype=torch.float64)).long() - 1
    else:
        t = torch.randint(-2, vocab + 2, (n,), generator=g)   # (some of them none)
    return t.to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens", [torch.int32, torch.int64])
@pytest.mark.parametrize("n,vocab,width", [(1, 1, 1), (3, 5, 7), (8, 100, 2048), (300, 17, 40), (70, 33, 8), (5, 9, 5001)])
def test_rows(swr, dtype, tokens, n, vocab, width):
    t, table = _tokens(1, n, vocab, "any", tokens), rand(2, (vocab, width), dtype).cuda()
    for scale in (1.0, 45.25, -0.3):
        want = ref.embedding(t, table, scale)
        ref.close(swr.swr_embedding(t, table, scale), want, want.abs() * (ROUND[dtype] + U) + TINY, "y")


def _check(swr, t, dy, vocab, scale, dtype=None, **kw):
    d = swr.swr_embedding_backward(t, dy, vocab, scale, dtype, **kw)
    want, size, most = ref.embedding_backward(t, dy, vocab, scale)
    assert d.dtype == (dtype or F32)
    ref.close(d, want, want.abs() * ROUND[d.dtype] + size * U * (most + 1) * (1 + ROUND[d.dtype]) + TINY, "dtable")
    return d


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("kind", ["any", "words", "one"])
@pytest.mark.parametrize("n,vocab,width", [
    (1, 1, 1), (1, 7, 3), (31, 5, 9), (32, 2, 16), (33, 300, 24), (64, 64, 8), (65, 1000, 130), (500, 3, 40),
    (4096, 70000, 4), (4097, 300, 12), (9000, 255, 17), (9000, 256, 8), (20000, 65536, 3)])
def test_gradient(swr, dtype, kind, n, vocab, width):
    t, dy = _tokens(3, n, vocab, kind), rand(4, (n, width), dtype).cuda()
    d = _check(swr, t, dy, vocab, 3.5)
    assert torch.equal(d, swr.swr_embedding_backward(t, dy, vocab, 3.5))   # (a fixed order)
    _check(swr, t, dy, vocab, 1.0, dtype)


def test_many_tiles(swr):
    """More tiles of positions than a pass's blocks sum by themselves, and three digits of tokens."""
    n, vocab = 300000, 70001
    t, dy = _tokens(5, n, vocab, "words", torch.int32), rand(6, (n, 2), F32).cuda()
    d = swr.swr_embedding_backward(t, dy, vocab)
    want, size = (torch.zeros(vocab, 2, dtype=torch.float64) for _ in range(2))
    want.index_add_(0, t.cpu().long(), ref.f64(dy))
    size.index_add_(0, t.cpu().long(), ref.f64(dy).abs())
    most = int(torch.bincount(t.cpu().long()).max())
    ref.close(d, want, size * U * (most + 1) + TINY, "dtable")


def test_layouts(swr):
    """Tokens of two dimensions, dy of one row for all and of spaced rows, a gradient within a larger tensor."""
    t = _tokens(7, 60, 11, "any").reshape(4, 15)
    wide = rand(8, (4, 15, 50), BF16).cuda()
    _check(swr, t, wide[..., 7:40], 11, 2.0)
    _check(swr, t, wide[:1, :1, :33].expand(4, 15, 33), 11, 2.0)
    out = torch.full((11, 60), 9.0, device="cuda")
    d = _check(swr, t, wide[..., :30], 11, 2.0, dtable=out[:, 10:40],
               workspace=torch.empty(1 << 16, dtype=torch.float32, device="cuda"))
    assert d.data_ptr() == out[:, 10:40].data_ptr() and (out[:, :10] == 9).all() and (out[:, 40:] == 9).all()
    table = rand(9, (11, 64), BF16).cuda()[:, 3:36]
    ys = torch.full((4, 15, 40), 9.0, dtype=BF16, device="cuda")
    y = swr.swr_embedding(t, table, y=ys[..., 2:35])
    ref.close(y, ref.embedding(t, table, 1.0), TINY, "y")
    assert (ys[..., :2] == 9).all() and (ys[..., 35:] == 9).all()


def test_nothing(swr):
    t = torch.zeros(0, dtype=torch.int64, device="cuda")
    table = rand(1, (5, 8), F32).cuda()
    assert swr.swr_embedding(t, table).shape == (0, 8)
    d = swr.swr_embedding_backward(t, torch.zeros(0, 8, device="cuda"), 5)
    assert d.shape == (5, 8) and (d == 0).all()


def test_values_of_other_rows_do_not_matter(swr):
    """NaN and infinities reach their own token's row only; padding's rows are not looked at."""
    t = torch.tensor([4, -1, 2, 9, 4, 0], device="cuda")
    dy = rand(10, (6, 12), F32).cuda()
    dy[1], dy[3], dy[2, 5] = float("nan"), float("inf"), float("nan")
    d = swr.swr_embedding_backward(t, dy, 9)
    want, _, _ = ref.embedding_backward(t, dy, 9, 1.0)
    ref.close(d, want, want.abs().nan_to_num() * 4 * U + TINY, "dtable")


def test_autograd(swr):
    t, table = _tokens(11, 40, 30, "any"), rand(12, (30, 24), BF16).cuda().requires_grad_(True)
    y = swr.SWREmbeddingFunction.apply(t, table, 4.0)
    for g in (rand(13, (40, 24), BF16).cuda(), rand(14, (1, 24), BF16).cuda().expand(40, 24),
              rand(15, (24, 40), BF16).cuda().t()):
        d, = torch.autograd.grad(y, table, g, retain_graph=True)
        want, size, most = ref.embedding_backward(t, g, 30, 4.0)
        assert d.dtype == BF16
        ref.close(d, want, want.abs() * ROUND[BF16] + size * U * (most + 1) * 1.01 + TINY, "dtable")


def test_refusals(swr):
    t, table = _tokens(1, 4, 9, "any"), rand(1, (9, 8), F32).cuda()
    dy = rand(2, (4, 8), F32).cuda()
    for bad in (lambda: swr.swr_embedding(t.float(), table), lambda: swr.swr_embedding(t, table.half()),
                lambda: swr.swr_embedding_backward(t, dy, 9, dtype=BF16)):
        with pytest.raises((TypeError, swr.SwrError)):
            bad()
    for bad in (lambda: swr.swr_embedding(t, table.t()), lambda: swr.swr_embedding(t, table[0]),
                lambda: swr.swr_embedding(t, table, float("nan")), lambda: swr.swr_embedding(t.cpu(), table),
                lambda: swr.swr_embedding(t, table.cpu()), lambda: swr.swr_embedding_backward(t[:3], dy, 9)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(swr.SwrError):
        swr.swr_embedding_backward(t, dy, 0)


@pytest.mark.parametrize("n", [63, 64, 65, 1024, 4095, 4096, 4097])
def test_orders_of_equal_tokens(swr, n):
    """Sums whose order shows in their bits, repeated, of positions around a tile's and a block's."""
    g = torch.Generator().manual_seed(n)
    tokens = torch.randint(-1, 4, (n,), generator=g).cuda()
    dy = (torch.randn(n, 3, generator=g) * 2.0 ** torch.randint(-20, 20, (n, 3), generator=g)).cuda()
    first = swr.swr_embedding_backward(tokens, dy, 3)
    for _ in range(3):
        assert torch.equal(swr.swr_embedding_backward(tokens, dy, 3), first)
    # Padding counts for nothing, NaN in its rows neither.
    for v in range(3):
        own = tokens == v
        alone = swr.swr_embedding_backward(torch.where(own, tokens, -1), torch.where(own[:, None], dy, float("nan")), 3)
        rows = ref.f64(dy[own])
        ref.close(first[v], rows.sum(0), rows.abs().sum(0) * ref.U * n + ref.TINY, "sum")
        ref.close(alone[v], rows.sum(0), rows.abs().sum(0) * ref.U * n + ref.TINY, "alone")
        assert (alone[[i for i in range(3) if i != v]] == 0).all()
