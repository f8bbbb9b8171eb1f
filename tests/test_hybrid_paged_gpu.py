"""The paged key-value cache against its definitions on the host: tables and
slots, appends, and attention over lengths from none to many workgroups' shares,
every head layout and width, pages of any size, windows, strides, and what lies in
slots that no position uses."""
import pytest

import hybrid_ref as ref
from hybrid_ref import ROUND, U

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


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ----------------------------------------------------------------------------- tables


def _table_case(swr, lengths, news, page, max_pages, stack, count, tokens, seed=0):
    g = torch.Generator().manual_seed(seed)
    table = torch.randint(-1, 50, (len(lengths), max_pages), generator=g, dtype=torch.int32)
    want = ref.tables(lengths, news, table.tolist(), stack, count, page, tokens)
    t = table.cuda()
    got = swr.swr_block_tables(_i32(lengths), _i32(news), t, _i32(stack), _i32([count]), page, tokens)
    torch.cuda.synchronize()
    # (a page that no listed token is on is entered too)
    assert t.cpu().tolist() == want[0]
    assert got[0].dtype == torch.int64 and got[0].tolist() == want[1]
    assert got[1].tolist() == want[2] and got[2].tolist() == want[3] and got[3].tolist() == [want[4]]


@pytest.mark.parametrize("page", [1, 3, 16, 64])
@pytest.mark.parametrize("batch", [0, 1, 5, 255, 256, 257, 1030])
def test_tables(swr, page, batch):
    g = torch.Generator().manual_seed(batch + page)
    lengths = torch.randint(0, 70, (batch,), generator=g).tolist()
    news = torch.randint(0, 20, (batch,), generator=g).tolist()
    stack = torch.randperm(batch * 20 + 3, generator=g).tolist()
    total = sum(news)
    for tokens in (total, total + 1500, max(total - 7, 0), 0):
        _table_case(swr, lengths, news, page, 90 // page + 2, stack, len(stack), tokens)


def test_tables_one_token_each(swr):
    _table_case(swr, [0, 15, 16, 17, 31], [1] * 5, 16, 3, [9, 8, 7, 6], 4, 5)
    _table_case(swr, [0, 15, 16, 17, 31], [0] * 5, 16, 3, [9, 8, 7, 6], 4, 5)


def test_tables_long_prompts(swr):
    _table_case(swr, [0, 5, 1000, 0], [5000, 0, 3001, 1], 16, 400, list(range(1000)), 900, 8002)


def test_tables_at_their_limits(swr):
    # No page left, a stack count past the stack or below zero, positions past
    # the table, numbers below zero.
    _table_case(swr, [4, 4, 4], [5, 5, 5], 4, 8, [1, 2, 3], 3, 15)
    _table_case(swr, [4, 4, 4], [5, 5, 5], 4, 8, [1, 2, 3], 0, 15)
    _table_case(swr, [4, 4, 4], [5, 5, 5], 4, 8, [1, 2, 3], -5, 15)
    _table_case(swr, [4, 4, 4], [5, 5, 5], 4, 8, [1, 2, 3, 4, 5, 6], 99, 15)
    _table_case(swr, [4, 30, 4, 7], [5, 9, 40, 1], 4, 8, list(range(40)), 40, 60)
    _table_case(swr, [-3, 5, -1], [4, -2, 0], 4, 8, list(range(9)), 9, 8)
    _table_case(swr, [3, 5], [4, 2], 4, 0, [], 0, 6)


def test_tables_of_huge_numbers(swr):
    # 2^31 - 1 tokens asked of a small table end as quickly as any.
    big = 2 ** 31 - 1
    t = torch.full((3, 4), -1, dtype=torch.int32, device="cuda")
    slots, starts, lengths, left = swr.swr_block_tables(_i32([0, big, 5]), _i32([big, big, 1]), t, _i32(list(range(20))),
                                                        _i32([20]), 2, 6)
    torch.cuda.synchronize()
    assert t.tolist() == [[19, 18, 17, 16], [-1] * 4, [-1, -1, -1, -1]]
    assert slots.tolist() == [38, 39, 36, 37, 34, 35] and left.tolist() == [16]
    assert lengths.tolist() == [big, big, 6] and starts.tolist() == [0, big, big, big]


# ----------------------------------------------------------------------------- append


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("tokens,heads,D,page", [(1, 1, 16, 1), (3, 5, 48, 7), (40, 8, 128, 16), (1000, 3, 80, 64), (65, 2, 256, 5)])
def test_append(swr, dtype, tokens, heads, D, page):
    g = torch.Generator().manual_seed(tokens)
    pages = tokens // page + 3
    k, v = torch.randn((2, tokens, heads, D), generator=g).to(dtype).cuda()
    fused = torch.randn((tokens, 3 * heads, D), generator=g).to(dtype).cuda()
    slots = torch.randperm(pages * page, generator=g)[:tokens]
    slots[tokens // 2] = -1
    if tokens > 2:
        slots[0], slots[1] = pages * page, 2 ** 62
    for kk, vv in ((k, v), (fused[:, heads:2 * heads], fused[:, 2 * heads:])):
        for order in ((0, 1, 2, 3), (0, 2, 1, 3)):     # pages of tokens, or of heads
            shape = [(pages, page, heads, D)[i] for i in order]
            kc, vc = torch.randn((2, *shape), generator=g).to(dtype).cuda()
            kc, vc = kc.permute(*order), vc.permute(*order)
            want_k, want_v = kc.clone(), vc.clone()
            for i, s in enumerate(slots.tolist()):
                if 0 <= s < pages * page:
                    want_k[s // page, s % page], want_v[s // page, s % page] = kk[i], vv[i]
            swr.swr_cache_append(kk, vv, kc, vc, slots.cuda())
            torch.cuda.synchronize()
            assert torch.equal(kc, want_k) and torch.equal(vc, want_v)


# ----------------------------------------------------------------------------- attention


def _paged(seed, lengths, heads, D, page, dtype, extra=3, poison=True, order=(0, 1, 2, 3)):
    """A cache whose requests' pages lie in any order; slots that no position
    uses hold NaN, unused pages infinities."""
    g = torch.Generator().manual_seed(seed)
    counts = [-(-max(n, 0) // page) for n in lengths]
    pages = sum(counts) + extra
    kc, vc = torch.randn((2, pages, page, heads, D), generator=g)
    ids = torch.randperm(pages, generator=g).tolist()
    table = torch.full((len(lengths), max(counts + [1])), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = torch.tensor(ids[at:at + c], dtype=torch.int32)
        if poison and c and lengths[b] % page:
            for t in (kc, vc):
                t[ids[at + c - 1], lengths[b] % page:] = float("nan")
        at += c
    if poison:
        for i in ids[at:]:
            kc[i], vc[i] = float("inf"), float("-inf")
    shape = [(pages, page, heads, D)[i] for i in order]
    back = [order.index(i) for i in range(4)]

    def place(t):
        return t.permute(*order).contiguous().view(shape).to(dtype).cuda().permute(*back)

    return place(kc), place(vc), table.cuda(), _i32(lengths)


def _check(swr, q, kc, vc, table, lengths, scale=None, window=0, **kw):
    D = q.shape[-1]
    s = D ** -0.5 if scale is None else scale
    y, lse = swr.swr_paged_attention(q, kc, vc, table, lengths, scale=scale, window=window, want_lse=True, **kw)
    torch.cuda.synchronize()
    want, wl, vmax, smax = ref.attention(q, kc, vc, table, lengths, s, window)
    n = int(lengths.max()) if lengths.numel() else 0
    # A score is a float32 sum of D products, scaled and exponentiated (off by
    # its error, both in the weights and in their sum); then sums of n weights.
    score = smax * U * (D + 8) + U * 16
    rel = 2 * score + U * (n / 8 + 64)
    ref.close(y, want, want.abs() * ROUND[q.dtype] + rel * vmax, "y")
    ref.close(lse, wl, rel[..., 0] + wl.abs().nan_to_num(posinf=0) * U * 4, "lse")
    return y


def _q(seed, B, H, D, dtype):
    g = torch.Generator().manual_seed(seed)
    return torch.randn((B, H, D), generator=g).to(dtype).cuda()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("D", [16, 32, 48, 64, 80, 96, 112, 128, 144, 192, 240, 256])
def test_attention_widths(swr, dtype, D):
    lengths = [1, 0, 33, 200, 64, 31, 32, 700]
    kc, vc, table, n = _paged(D, lengths, 2, D, 16, dtype)
    _check(swr, _q(1, len(lengths), 6, D, dtype), kc, vc, table, n)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("heads,group", [(1, 1), (3, 2), (5, 3), (2, 8), (1, 16), (2, 17), (1, 40), (8, 4), (4, 5)])
def test_attention_heads(swr, dtype, heads, group):
    lengths = [5, 130, 0, 1, 257]
    kc, vc, table, n = _paged(heads + group, lengths, heads, 64, 16, dtype)
    _check(swr, _q(2, 5, heads * group, 64, dtype), kc, vc, table, n)


@pytest.mark.parametrize("page", [1, 2, 5, 16, 24, 32, 48, 64, 100, 128, 1000])
def test_attention_pages(swr, page):
    lengths = [99, 100, 101, 1, 0, 640, 37]
    for dtype in (BF16, F32):
        kc, vc, table, n = _paged(page, lengths, 2, 32, page, dtype)
        _check(swr, _q(3, 7, 4, 32, dtype), kc, vc, table, n)


@pytest.mark.parametrize("window", [1, 16, 31, 32, 33, 100, 5000])
def test_attention_windows(swr, window):
    lengths = [1, 16, 33, 100, 0, 1500, 32]
    for dtype in (BF16, F32):
        kc, vc, table, n = _paged(window, lengths, 2, 64, 16, dtype, poison=False)
        y = _check(swr, _q(4, 7, 8, 64, dtype), kc, vc, table, n, window=window)
        # what lies before the window is not read into the result
        for b, length in enumerate(lengths):
            for t in range(max(0, length - window)):
                page, at = int(table[b, t // 16]), t % 16
                kc[page, at], vc[page, at] = float("nan"), float("nan")
        assert torch.equal(swr.swr_paged_attention(_q(4, 7, 8, 64, dtype), kc, vc, table, n, window=window), y)


def test_attention_long_rows_are_split(swr):
    # Rows cut between many workgroups, of very different lengths.
    for dtype, D, group in ((BF16, 128, 4), (F32, 64, 2), (BF16, 256, 1)):
        lengths = [20011, 1, 0, 300, 7777, 64, 12000, 2]
        kc, vc, table, n = _paged(D, lengths, 2, D, 16, dtype)
        _check(swr, _q(5, len(lengths), 2 * group, D, dtype), kc, vc, table, n)


def test_attention_many_short_requests(swr):
    g = torch.Generator().manual_seed(8)
    lengths = torch.randint(0, 90, (700,), generator=g).tolist()
    kc, vc, table, n = _paged(9, lengths, 1, 32, 16, BF16)
    _check(swr, _q(6, 700, 2, 32, BF16), kc, vc, table, n)


def test_attention_no_request_has_a_token(swr):
    kc, vc, table, n = _paged(1, [0, 0, -4], 2, 64, 16, BF16)
    y, lse = swr.swr_paged_attention(_q(7, 3, 4, 64, BF16), kc, vc, table, n, want_lse=True)
    torch.cuda.synchronize()
    assert (y == 0).all() and (lse == float("-inf")).all()
    assert swr.swr_paged_attention(_q(7, 0, 4, 64, BF16), kc, vc, table[:0], n[:0]).shape == (0, 4, 64)
    y = swr.swr_paged_attention(_q(7, 3, 4, 64, BF16), kc[:0], vc[:0], table, _i32([5, 40, 0]))
    torch.cuda.synchronize()
    assert (y == 0).all()


def test_attention_leaves_out_pages_that_are_none(swr):
    lengths = [200, 50, 64, 10]
    kc, vc, table, n = _paged(11, lengths, 2, 64, 16, BF16, poison=False)
    table[0, 3], table[0, 7], table[1, 0], table[3, 0] = -1, kc.shape[0], 2 ** 31 - 1, -2 ** 31
    _check(swr, _q(8, 4, 4, 64, BF16), kc, vc, table, n)
    # lengths past the table's columns end with it
    _check(swr, _q(8, 4, 4, 64, BF16), kc, vc, table, _i32([5000, 50, 2 ** 31 - 1, 10]))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_layouts(swr, dtype):
    lengths = [70, 3, 0, 250]
    base = _paged(12, lengths, 3, 64, 16, dtype)
    q = _q(9, 4, 6, 64, dtype)
    want = _check(swr, q, *base)
    heads_first = _paged(12, lengths, 3, 64, 16, dtype, order=(0, 2, 1, 3))
    assert heads_first[0].stride() != base[0].stride()
    assert torch.equal(_check(swr, q, *heads_first), want)
    fused = torch.cat([q, _q(10, 4, 9, 64, dtype)], 1)[:, :6]          # q as part of one projection's rows
    wide = torch.full((4, 30), -7, dtype=torch.int32, device="cuda")
    wide[:, 5:5 + base[2].shape[1]] = base[2]
    y = torch.full((4, 8, 64), 2.0, dtype=dtype, device="cuda")
    swr.swr_paged_attention(fused, base[0], base[1], wide[:, 5:5 + base[2].shape[1]], base[3], y=y[:, 1:7])
    torch.cuda.synchronize()
    assert torch.equal(y[:, 1:7], want) and (y[:, 0] == 2).all() and (y[:, 7] == 2).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_of_large_scores(swr, dtype):
    # One position far above the others, at each place of a tile; negative and zero scales.
    lengths = [97] * 97
    kc, vc, table, n = _paged(13, lengths, 1, 32, 32, dtype)
    q = _q(11, 97, 2, 32, dtype)
    for b in range(97):
        page = int(table[b, b // 32])
        kc[page, b % 32, 0] = q[b, 0] * 30
    _check(swr, q, kc, vc, table, n, scale=1.0)
    _check(swr, q, kc, vc, table, n, scale=-0.5)
    _check(swr, q, kc, vc, table, n, scale=0.0)


def test_attention_nan_stays_with_its_head(swr):
    kc, vc, table, n = _paged(14, [80, 200], 2, 64, 16, BF16)
    q = _q(12, 2, 4, 64, BF16)
    want = swr.swr_paged_attention(q, kc, vc, table, n)
    q2 = q.clone()
    q2[1, 2, 5] = float("nan")
    got = swr.swr_paged_attention(q2, kc, vc, table, n)
    torch.cuda.synchronize()
    assert torch.isnan(got[1, 2]).all()
    got[1, 2] = want[1, 2]
    assert torch.equal(got, want)


def test_attention_repeats_and_streams(swr):
    lengths = [9000, 100, 1, 4000]
    kc, vc, table, n = _paged(15, lengths, 4, 128, 16, BF16)
    q = _q(13, 4, 16, 128, BF16)
    want = swr.swr_paged_attention(q, kc, vc, table, n)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        got = swr.swr_paged_attention(q, kc, vc, table, n, stream=s)
        junk = [torch.full((1 << 18,), float("nan"), device="cuda") for _ in range(8)]
        torch.cuda.current_stream().wait_stream(s)
        assert torch.equal(got, want)
        del junk


def test_offsets_past_32_bits(swr):
    # A cache of more than 2^32 bytes: pages at its end and its start.
    pages, page, heads, D = 70000, 16, 16, 128
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("needs 40 GB of device memory")
    kc, vc = (torch.zeros((pages, page, heads, D), dtype=BF16, device="cuda") for _ in range(2))
    lengths = [100, 40]
    table = torch.full((2, 7), -1, dtype=torch.int32)
    table[0] = torch.tensor([69999, 0, 65536, 69998, 32768, 12345, 69000])
    table[1, :3] = torch.tensor([69997, 1, 50000])
    slots = [int(table[b, t // page]) * page + t % page for b, n in enumerate(lengths) for t in range(n)]
    g = torch.Generator().manual_seed(1)
    k, v = torch.randn((2, 140, heads, D), generator=g).to(BF16).cuda()
    swr.swr_cache_append(k, v, kc, vc, torch.tensor(slots, device="cuda"))
    q = _q(14, 2, heads, D, BF16)
    got = swr.swr_paged_attention(q, kc, vc, table.cuda(), _i32(lengths))
    # the same tokens in a small cache
    small_k, small_v = (torch.zeros((10, page, heads, D), dtype=BF16, device="cuda") for _ in range(2))
    order = {int(p): i for i, p in enumerate(table[table >= 0].tolist())}
    small = table.clone()
    small[table >= 0] = torch.arange(10, dtype=torch.int32)
    at = torch.tensor([order[s // page] * page + s % page for s in slots], device="cuda")
    swr.swr_cache_append(k, v, small_k, small_v, at)
    want = swr.swr_paged_attention(q, small_k, small_v, small.cuda(), _i32(lengths))
    torch.cuda.synchronize()
    assert torch.equal(got, want) and got.abs().max() > 0.01
    del kc, vc


def test_a_captured_step_replays(swr):
    """Append and attention in a HIP graph: every replay gives the eager result."""
    lengths = [50, 333]
    kc, vc, table, n = _paged(16, [x + 1 for x in lengths], 2, 64, 16, BF16)
    q, k, v = _q(15, 2, 4, 64, BF16), _q(16, 2, 2, 64, BF16), _q(17, 2, 2, 64, BF16)
    slots = torch.tensor([int(table[b, x // 16]) * 16 + x % 16 for b, x in enumerate(lengths)], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        swr.swr_cache_append(k, v, kc, vc, slots)
        swr.swr_paged_attention(q, kc, vc, table, n)
    torch.cuda.current_stream().wait_stream(s)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        swr.swr_cache_append(k, v, kc, vc, slots)
        y = swr.swr_paged_attention(q, kc, vc, table, n)
    for i in range(4):
        for t, seed in ((q, 30), (k, 40), (v, 50)):
            t.copy_(_q(seed + i, *t.shape, BF16))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(kc.reshape(-1, 2, 64)[slots], k) and torch.equal(vc.reshape(-1, 2, 64)[slots], v)
        assert torch.equal(swr.swr_paged_attention(q, kc, vc, table, n), got)
