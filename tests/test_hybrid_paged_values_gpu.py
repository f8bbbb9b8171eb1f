"""What paged attention makes of its values: weights of all 24 bits, on both
routes (a workgroup a row, and shares of the work)."""
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
