"""Paged attention by shares of the work, as tables of more than 1024 positions have
it: every width, head layout, page size, window and cache layout, missing pages and
large scores, rows cut between workgroups, and the two ways in which their parts are
found and joined."""
import pytest

from test_hybrid_paged_gpu import _check, _i32, _paged, _q

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


def _shared(seed, lengths, heads, D, page, dtype, **kw):
    """As _paged, with a table of 2048 positions at least, more columns than its requests use."""
    kc, vc, table, n = _paged(seed, lengths, heads, D, page, dtype, **kw)
    more = max(0, 2048 // page + 1 - table.shape[1])
    return kc, vc, torch.nn.functional.pad(table, (0, more), value=-1), n


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 240, 256])
def test_widths(swr, dtype, D):
    lengths = [1, 0, 33, 200, 64, 31, 32, 700, 1500]
    kc, vc, table, n = _shared(D, lengths, 2, D, 16, dtype)
    _check(swr, _q(1, len(lengths), 6, D, dtype), kc, vc, table, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,group", [(1, 1), (3, 2), (5, 3), (2, 8), (1, 16), (2, 17), (1, 40), (8, 4), (4, 5)])
def test_heads(swr, dtype, heads, group):
    # (groups of 17 and 40: several tiles of heads a key head)
    lengths = [5, 1300, 0, 1, 257]
    kc, vc, table, n = _shared(heads + group, lengths, heads, 64, 16, dtype)
    _check(swr, _q(2, 5, heads * group, 64, dtype), kc, vc, table, n)


@pytest.mark.parametrize("page", [1, 2, 5, 16, 24, 48, 100, 128, 1000])
def test_pages(swr, page):
    lengths = [99, 100, 101, 1, 0, 640, 37, 1999]
    for dtype in (BF16, F32):
        kc, vc, table, n = _shared(page, lengths, 2, 32, page, dtype)
        _check(swr, _q(3, 8, 4, 32, dtype), kc, vc, table, n)


@pytest.mark.parametrize("window", [1025, 1500, 1504, 2900])
@pytest.mark.parametrize("heads,group", [(2, 4), (1, 20)])
def test_windows(swr, window, heads, group):
    # Windows that begin past 0, inside a page and at its edge, in rows that are cut.
    lengths = [3000, 16, 1600, 2999, 0, 1503, 3200]
    for dtype in (BF16, F32):
        kc, vc, table, n = _shared(window, lengths, heads, 64, 16, dtype, poison=False)
        q = _q(4, 7, heads * group, 64, dtype)
        y = _check(swr, q, kc, vc, table, n, window=window)
        for b, length in enumerate(lengths):     # what lies before the window is not read into the result
            for t in range(max(0, length - window)):
                page, at = int(table[b, t // 16]), t % 16
                kc[page, at], vc[page, at] = float("nan"), float("nan")
        assert torch.equal(swr.swr_paged_attention(q, kc, vc, table, n, window=window), y)


def test_missing_pages(swr):
    lengths = [2000, 500, 64, 10, 1300]
    kc, vc, table, n = _shared(11, lengths, 2, 64, 16, BF16, poison=False)
    table[0, 3], table[0, 7], table[1, 0], table[3, 0] = -1, kc.shape[0], 2 ** 31 - 1, -2 ** 31
    table[0, 40:60], table[1, 1:20], table[4] = -1, -5, -1       # whole tiles, and a whole request
    _check(swr, _q(8, 5, 4, 64, BF16), kc, vc, table, n)
    # lengths past the table's columns end with it
    q, end = _q(8, 5, 4, 64, BF16), 16 * table.shape[1]
    want = _check(swr, q, kc, vc, table, _i32([end, 500, end, 10, 1300]))
    assert torch.equal(swr.swr_paged_attention(q, kc, vc, table, _i32([5000, 500, 2 ** 31 - 1, 10, 1300])), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(swr, dtype):
    lengths = [70, 3, 0, 1250]
    base = _shared(12, lengths, 3, 64, 16, dtype)
    q = _q(9, 4, 6, 64, dtype)
    want = _check(swr, q, *base)
    heads_first = _shared(12, lengths, 3, 64, 16, dtype, order=(0, 2, 1, 3))
    assert heads_first[0].stride() != base[0].stride()
    assert torch.equal(_check(swr, q, *heads_first), want)
    fused = torch.cat([q, _q(10, 4, 9, 64, dtype)], 1)[:, :6]
    wide = torch.nn.functional.pad(base[2], (5, 9), value=-7)
    y = torch.full((4, 8, 64), 2.0, dtype=dtype, device="cuda")
    swr.swr_paged_attention(fused, base[0], base[1], wide[:, 5:-9], base[3], y=y[:, 1:7])
    torch.cuda.synchronize()
    assert torch.equal(y[:, 1:7], want) and (y[:, 0] == 2).all() and (y[:, 7] == 2).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_large_scores(swr, dtype):
    # One position far above the others, in one of each row's shares; negative and zero scales.
    lengths = [1097] * 37
    kc, vc, table, n = _shared(13, lengths, 1, 32, 32, dtype)
    q = _q(11, 37, 2, 32, dtype)
    for b in range(37):
        t = 29 * b + 3
        kc[int(table[b, t // 32]), t % 32, 0] = q[b, 0] * 30
    for scale in (1.0, -0.5, 0.0):
        _check(swr, q, kc, vc, table, n, scale=scale)


@pytest.mark.parametrize("batch,heads,group", [(40, 1, 2), (30, 3, 1), (100, 2, 2), (230, 1, 4), (60, 2, 20), (700, 1, 2)])
def test_many_rows_are_cut(swr, batch, heads, group):
    # From few rows (a block finds each) to many (each share joins what begins in it): rows of one
    # tile to some that go through many shares, next to each other and apart, and none.
    g = torch.Generator().manual_seed(batch)
    lengths = torch.randint(0, 400, (batch,), generator=g).tolist()
    for b in range(0, batch, 9):
        lengths[b] = 1000 + 211 * (b % 7)
    lengths[batch // 2], lengths[batch // 2 + 1], lengths[-1] = 4000, 3500, 0
    kc, vc, table, n = _shared(batch, lengths, heads, 32, 16, BF16)
    q = _q(6, batch, heads * group, 32, BF16)
    y = _check(swr, q, kc, vc, table, n)
    assert torch.equal(swr.swr_paged_attention(q, kc, vc, table, n), y)
