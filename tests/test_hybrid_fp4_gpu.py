"""Products with 4-bit weights against their 64-bit form: every code and power,
types, row counts, lengths that end inside a group and a block, strides,
infinities and NaN; and packing."""
import pytest

import hybrid_ref as ref
from hybrid_ref import ROUND, TINY, U

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32, FP8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def _weights(seed, N, K, low=118, high=130):
    g = torch.Generator().manual_seed(seed)
    groups = -(-K // 32)
    return (torch.randint(0, 256, (N, 16 * groups), generator=g, dtype=torch.uint8).cuda(),
            torch.randint(low, high, (N, groups), generator=g, dtype=torch.uint8).cuda())


def _rows(seed, M, K, dtype):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((M, K), generator=g) * (10 if dtype == FP8 else 1)
    return x.clamp(-448, 448).to(dtype).cuda()


def _check(swr, x, codes, powers, scale=None, out=None):
    y = swr.swr_fp4_linear(x, codes, powers, scale=scale, out_dtype=out)
    torch.cuda.synchronize()
    want, size = ref.linear(x, codes, powers, scale)
    assert y.dtype == (out or (BF16 if x.dtype == FP8 else x.dtype))
    # float32 sums of K products (bf16 and 8-bit products are exact; float32 ones
    # are sums of three), and the row factor
    ref.close(y, want, want.abs() * ROUND[y.dtype] + size * U * (x.shape[-1] / 4 + 40) + TINY, "y")
    return y


SHAPES = [(1, 1, 1), (1, 16, 32), (2, 17, 31), (3, 5, 33), (16, 64, 128), (5, 1001, 1000), (17, 33, 130), (1, 6176, 2048),
          (32, 100, 257), (33, 48, 96), (64, 65, 511), (65, 130, 1024), (130, 31, 100), (7, 20, 5000), (8, 256, 4096)]


@pytest.mark.parametrize("dtype", [BF16, F32, FP8])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(swr, dtype, M, N, K):
    codes, powers = _weights(M * 7 + N, N, K)
    x = _rows(K, M, K, dtype)
    _check(swr, x, codes, powers)
    g = torch.Generator().manual_seed(1)
    scale = torch.rand((M,), generator=g).cuda() + 0.1
    for out in (BF16, F32):
        _check(swr, x, codes, powers, scale, out)


# Each way through the kernels: x held in registers of every length (one to eight blocks
# of 128 k a wave), 16 and 32 rows at a time; several meetings of a workgroup's waves, the
# last one short; x that does not fit; one tile of W a wave and two.
LONG = [(9, 40, 1100), (12, 50, 3000), (16, 33, 4097), (10, 50, 6000), (16, 40, 8191), (11, 48, 16384), (10, 33, 16390),
        (20, 40, 2049), (40, 35, 4000), (18, 47, 5200), (33, 18, 8192), (3, 20003, 40), (12, 8200, 300), (40, 9000, 300),
        (17, 4500, 1500), (300, 5000, 100), (3, 4200, 2100), (8, 4099, 4500), (70, 4111, 2300)]


@pytest.mark.parametrize("dtype", [BF16, F32, FP8])
@pytest.mark.parametrize("M,N,K", LONG)
def test_long_rows_and_many_tiles(swr, dtype, M, N, K):
    codes, powers = _weights(M + N + K, N, K)
    x = _rows(K, M, K, dtype)
    scale = torch.rand((M,), generator=torch.Generator().manual_seed(2)).cuda() + 0.1
    y = _check(swr, x, codes, powers, scale)
    _check(swr, x, codes, powers, None, F32)
    again = swr.swr_fp4_linear(x, codes, powers, scale=scale)
    torch.cuda.synchronize()
    assert torch.equal(y, again)


@pytest.mark.parametrize("dtype", [BF16, F32, FP8])
def test_every_code_and_power(swr, dtype):
    # Row n of W has one group of one power, all 16 codes in it twice.
    codes = (torch.arange(0, 256, 17, dtype=torch.uint8)).repeat(253, 1).cuda()    # byte 0x11 i: code i twice
    powers = torch.arange(0, 253, dtype=torch.uint8)[:, None].cuda()
    x = torch.zeros((16, 32))
    for i in range(16):
        x[i, 2 * i] = 1.0
    y = swr.swr_fp4_linear(x.to(dtype).cuda(), codes, powers, out_dtype=F32)
    torch.cuda.synchronize()
    w = ref.unpack(codes, powers, 32)[:, ::2]                                     # [power, code]
    assert torch.equal(ref.f64(y), w.t())


@pytest.mark.parametrize("dtype", [BF16, F32, FP8])
def test_strides_and_alignment(swr, dtype):
    M, N, K = 6, 70, 333
    codes, powers = _weights(3, N, K)
    room = torch.full((N, codes.shape[1] + 32), 255, dtype=torch.uint8, device="cuda")
    room[:, 16:16 + codes.shape[1]] = codes
    wide = torch.full((N, powers.shape[1] + 3), 255, dtype=torch.uint8, device="cuda")
    wide[:, 1:1 + powers.shape[1]] = powers
    x = _rows(4, M, K, dtype)
    big = torch.full((M, K + 9), float("nan"), device="cuda").to(dtype)
    big[:, 5:K + 5] = x
    want = _check(swr, x, codes, powers)
    y = torch.full((M, N + 4), 3.0, dtype=want.dtype, device="cuda")
    swr.swr_fp4_linear(big[:, 5:K + 5], room[:, 16:16 + codes.shape[1]], wide[:, 1:1 + powers.shape[1]],
                       y=y[:, 1:N + 1])
    torch.cuda.synchronize()
    assert torch.equal(y[:, 1:N + 1], want) and (y[:, 0] == 3).all() and (y[:, N + 1:] == 3).all()
    three = x.reshape(2, 3, K)
    assert torch.equal(swr.swr_fp4_linear(three, codes, powers), want.reshape(2, 3, N))


def test_codes_past_the_end_are_not_used(swr):
    for dtype in (BF16, F32, FP8):
        codes, powers = _weights(5, 40, 37)
        x = _rows(6, 3, 37, dtype)
        want = swr.swr_fp4_linear(x, codes, powers)
        codes[:, 19:] = 0x77    # k = 38 and later
        codes[:, 18] |= 0x70    # k = 37
        assert torch.equal(swr.swr_fp4_linear(x, codes, powers), want)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_infinities_and_nan(swr, dtype):
    codes, powers = _weights(7, 50, 200)
    codes[:, 0] = 0x22                        # weights 0 and 1 are not zero (an infinity times one is no NaN)
    x = _rows(8, 20, 200, dtype)
    want = swr.swr_fp4_linear(x, codes, powers)
    x[3, 0], x[5, 1], x[18, 190] = float("inf"), float("-inf"), float("nan")
    powers[17, 2] = 255
    got = swr.swr_fp4_linear(x, codes, powers)
    torch.cuda.synchronize()
    rows = [i for i in range(20) if i not in (3, 5, 18)]
    cols = [i for i in range(50) if i != 17]
    assert torch.equal(got[rows][:, cols], want[rows][:, cols])
    assert (got[3, cols] == float("inf")).all() and (got[5, cols] == float("-inf")).all()
    assert torch.isnan(got[18]).all() and torch.isnan(got[:, 17]).all()


def test_large_and_small_floats(swr):
    # Activations at both ends of float32 keep their bits.
    codes, powers = _weights(9, 16, 32, 127, 128)
    codes[:] = 0
    codes[:, 0] = 0x02                        # W = 1 at k = 0 only
    x = torch.zeros(6, 32)
    x[:, 0] = torch.tensor([3.4028234e38, -3.4e38, 1.17549435e-38, 1.0000001, -7.123456e-20, 16777215.0])
    y = swr.swr_fp4_linear(x.cuda(), codes, powers)
    torch.cuda.synchronize()
    got = y[:, 0].cpu()
    assert ((got - x[:, 0]).abs() <= x[:, 0].abs() * 2.0 ** -24 + 2.0 ** -140).all(), (got, x[:, 0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,K", [(1, 1), (3, 32), (17, 100), (64, 4097)])
def test_pack(swr, dtype, N, K):
    g = torch.Generator().manual_seed(N)
    w = torch.randn((N, K + 2), generator=g) * torch.exp(4 * torch.randn((N, 1), generator=g))
    w = w.to(dtype).cuda()[:, 1:K + 1]
    w[N // 2, K // 2] = 0
    codes, powers = swr.swr_fp4_pack(w)
    torch.cuda.synchronize()
    groups = -(-K // 32)
    assert codes.shape == (N, 16 * groups) and powers.shape == (N, groups)
    got = ref.unpack(codes, powers, 32 * groups)
    w64 = torch.nn.functional.pad(ref.f64(w), (0, 32 * groups - K))
    top = w64.reshape(N, groups, 32).abs().amax(-1)
    p = 2.0 ** (powers.cpu().double() - 127)
    live = top > 0
    assert (top <= 6 * p).all() and (top[live] > 3 * p[live]).all()           # the least power that holds the group
    # the nearest value: no other code is nearer
    size = (w64.reshape(N, groups, 32) / p[..., None])[..., None]
    best = (torch.cat([ref.SIZES, -ref.SIZES]) - size).abs().amin(-1)
    mine = (got.reshape(N, groups, 32) / p[..., None] - size[..., 0]).abs()
    assert torch.equal(mine, best)
    assert (got[:, K:] == 0).all()


def test_pack_edges(swr):
    w = torch.zeros(6, 64)
    w[1, :10] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -5.0])   # ties to the even code
    w[2, 3], w[3, 40] = float("inf"), float("nan")
    w[4, 0] = 3.0e38
    w[5, 0] = 1e-42
    codes, powers = swr.swr_fp4_pack(w.cuda())
    torch.cuda.synchronize()
    got = ref.unpack(codes, powers, 64)
    assert (powers[0] == 127).all() and (codes[0] == 0).all()
    assert got[1, :10].tolist() == [0, 1, 1, 2, 2, 4, 4, 6, 0, -4]
    assert powers[2].tolist() == [255, 127] and powers[3].tolist() == [127, 255]
    assert abs(float(got[4, 0]) / 3.0e38 - 1) <= 0.25 and int(powers[5, 0]) == 1
    y = swr.swr_fp4_linear(torch.ones(1, 64, device="cuda"), codes, powers)
    torch.cuda.synchronize()
    assert torch.isnan(y[0, 2]) and torch.isnan(y[0, 3]) and torch.isfinite(y[0, [0, 1, 4, 5]]).all()


def test_empty_and_another_stream(swr):
    codes, powers = _weights(1, 30, 64)
    assert swr.swr_fp4_linear(torch.empty(0, 64, device="cuda"), codes, powers).shape == (0, 30)
    assert swr.swr_fp4_linear(torch.ones(2, 64, device="cuda"), codes[:0], powers[:0]).shape == (2, 0)
    x = _rows(2, 16, 64, BF16)
    want = swr.swr_fp4_linear(x, codes, powers)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = swr.swr_fp4_linear(x, codes, powers, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(got, want)
