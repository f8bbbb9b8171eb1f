"""What paged attention makes of its values: weights of all 24 bits, infinite
values, scores of -infinity, on both routes (a workgroup a row, and shares of the work)."""
import math

import pytest

from hybrid_ref import f64
from test_hybrid_paged_gpu import _i32

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


def _cache(tokens, seed, dtype, pages, page=16, heads=1, D=16):
    """A cache, and the table of requests that hold `tokens` of its tokens each in turn."""
    g = torch.Generator().manual_seed(seed)
    kc, vc = torch.randn((2, pages, page, heads, D), generator=g)
    counts = [-(-n // page) for n in tokens]
    table = torch.full((len(tokens), max(counts)), -1, dtype=torch.int32)
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = torch.arange(at, at + c)
        at += c
    assert at <= pages
    return kc.to(dtype), vc.to(dtype), table


# Columns that the table has besides: past 1024 positions the work goes by shares.
ROUTES = [0, 100]


def _widened(table, more):
    return torch.nn.functional.pad(table, (0, more), value=-1).cuda()


@pytest.mark.parametrize("more", ROUTES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weights_keep_their_bits(swr, dtype, more):
    # Token 0 weighs p = exp(q) in [0.5, 1), the next three 1 (scores of 0); their values are 1
    # and the three parts of -p to 24 bits, so that y is what the weights' and the sums' roundings leave.
    # p: two roundings of a score below 0.7 (1.5 2^-24 p) and the exponential's last place
    # (2^-23); then at most 12 products, each cut off at worst at 2^-23 of a sum below 1.
    B, D = 64, 16
    kc, vc, table = _cache([4] * B, 0, dtype, B, D=D)
    q = torch.zeros(B, 1, D)
    q[:, 0, 0] = -(torch.arange(1, B + 1) / (B + 1) * 0.69).to(dtype).float()
    kc.zero_()
    kc[:, 0, 0, 0] = 1
    p = torch.exp(q[:, 0, 0].double())
    vc[:, 0] = 1
    left = p.clone()
    for t in range(1, 4):
        part = left.to(BF16)
        vc[:, t] = -part.to(dtype)[:, None, None]
        left -= part.double()
    assert left.abs().max() < 2.0 ** -25
    y = swr.swr_paged_attention(q.to(dtype).cuda(), kc.cuda(), vc.cuda(), _widened(table, more), _i32([4] * B), scale=1.0)
    torch.cuda.synchronize()
    off = (f64(y) * (3 + p)[:, None, None]).abs().max()
    assert off <= (1.5 + 2 + 24 + 0.5) * 2.0 ** -24 * 1.01, off * 2 ** 24
    assert math.isfinite(off)


@pytest.mark.parametrize("more", ROUTES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinite_values(swr, dtype, more):
    # An infinite value makes its channel of every head infinite, whatever its weight's bits:
    # of a single token (a weight of 1), and of others; of both signs NaN.
    lengths = [1, 2, 40, 300, 33, 64, 7]
    kc, vc, table = _cache(lengths, 1, dtype, 40, heads=2, D=32)
    q = torch.randn((len(lengths), 6, 32), generator=torch.Generator().manual_seed(2)).to(dtype).cuda()
    run = lambda v: swr.swr_paged_attention(q, kc.cuda(), v.cuda(), _widened(table, more), _i32(lengths))
    want = run(vc)
    inf = float("inf")

    def put(b, t, head, c, value):
        vc[table[b, t // 16], t % 16, head, c] = value
        y = want[b, 3 * head:3 * head + 3, c]
        y[:] = value if (torch.isfinite(y) | (y == value)).all() else float("nan")

    for b, n in enumerate(lengths):
        for t in {0, n // 2, n - 1}:
            put(b, t, 0, (5 * b + t) % 16, inf if t % 2 else -inf)
            put(b, t, 1, 31 - t % 8, inf)
    for t in (1, 2, 30, 31, 32, 200, 299):
        put(3, t, 1, t % 20, -inf)
    put(2, 3, 0, 17, inf)
    put(2, 4, 0, 17, -inf)
    got = run(vc)
    torch.cuda.synchronize()
    assert torch.isinf(want).any() and torch.isnan(want).any()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=0.0, posinf=inf, neginf=-inf),
                                                                            want.nan_to_num(nan=0.0, posinf=inf, neginf=-inf))


@pytest.mark.parametrize("more", ROUTES)
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_scores_of_minus_infinity(swr, dtype, more):
    # Tokens of such scores weigh nothing (as those of very low ones do); where a request has no
    # others, y is 0 / 0 and the sum's logarithm -infinity.  Only a request without a position has y = 0.
    lengths = [1, 40, 300, 1000, 1000, 64, 0, 20]
    kc, vc, table = _cache(lengths, 3, dtype, 160, heads=1, D=64)
    q = torch.randn((len(lengths), 3, 64), generator=torch.Generator().manual_seed(4))
    q[..., 0] = q[..., 0].abs().clamp(0.1, 1)
    q = q.to(dtype).cuda()
    spots = {b: range(n) for b, n in enumerate(lengths) if b in (0, 2, 3)}     # all of a request's tokens
    spots.update({1: range(32), 4: list(range(600)) + [999], 5: [63]})         # its first, most, its last
    table[7] = -1                                                              # tokens on no page: no position
    run = lambda k: swr.swr_paged_attention(q, k.cuda(), vc.cuda(), _widened(table, more), _i32(lengths), want_lse=True)
    low = kc.clone()
    for b, at in spots.items():
        for t in at:
            kc[table[b, t // 16], t % 16, 0, 0], low[table[b, t // 16], t % 16, 0, 0] = float("-inf"), -1e38
    y, lse = run(kc)
    want, wl = run(low)
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        if b in (0, 2, 3):
            assert torch.isnan(y[b]).all() and (lse[b] == float("-inf")).all(), b
        elif n == 0 or b == 7:
            assert (y[b] == 0).all() and (lse[b] == float("-inf")).all(), b
        else:
            assert torch.equal(y[b], want[b]) and torch.equal(lse[b], wl[b]) and torch.isfinite(y[b]).all(), b
