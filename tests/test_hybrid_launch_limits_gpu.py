"""Calls whose blocks would pass a launch's 2^32 threads."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32, FP8 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GB of device memory")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def test_attention_of_more_short_rows_than_a_launch_has_blocks(swr):
    # 32767 requests of 257 key heads: 8421119 rows, which as a block of 512 threads each were 2^32 threads.
    B, H, D, pages = 32767, 257, 16, 40
    assert B * H >= 1 << 23
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((B, H, D), generator=g, device="cuda").to(BF16)
    kc, vc = torch.randn((2, pages, 1, H, D), generator=g, device="cuda").to(BF16)
    table = torch.randint(0, pages, (B, 2), generator=g, device="cuda", dtype=torch.int32)
    lengths = torch.randint(0, 3, (B,), generator=g, device="cuda", dtype=torch.int32)
    y = swr.swr_paged_attention(q, kc, vc, table, lengths, scale=0.25)
    torch.cuda.synchronize()
    worst = 0.0
    for b in range(0, B, 4096):
        at = slice(b, b + 4096)
        rows, n = table[at].long(), lengths[at]
        k, v = (c[:, 0].double()[rows] for c in (kc, vc))                  # [requests, 2, H, D]
        s = (k * q[at].double()[:, None]).sum(-1) * 0.25                   # [requests, 2, H]
        s = s.masked_fill(torch.arange(2, device="cuda")[None, :, None] >= n[:, None, None], float("-inf"))
        p = torch.softmax(s, 1).nan_to_num(0.0)
        want = (p[..., None] * v).sum(1)
        assert (y[at][n == 0] == 0).all()
        # bf16's rounding; scores of 16 products of a few units
        worst = max(worst, float(((y[at].double() - want).abs() - want.abs() * 2.0 ** -8).max()))
    assert worst <= 1e-5


@pytest.mark.parametrize("M,N", [((1 << 28) + 37, 1), (3, (1 << 27) + 21), ((1 << 22) + 3, 600)])
def test_products_of_more_tiles_than_a_launch_has_blocks(swr, M, N):
    # y of more than 2^23 tiles of 16 x 16, each the product of one weight and one value.
    g = torch.Generator(device="cuda").manual_seed(2)
    x = torch.randn((M, 1), generator=g, device="cuda").to(FP8)
    scale = torch.rand((M,), generator=g, device="cuda") + 0.5
    codes = torch.zeros((N, 16), dtype=torch.uint8, device="cuda")
    codes[:, 0] = torch.randint(0, 16, (N,), generator=g, device="cuda", dtype=torch.uint8)
    powers = torch.randint(120, 130, (N, 1), generator=g, device="cuda", dtype=torch.uint8)
    y = swr.swr_fp4_linear(x, codes, powers, scale=scale)
    sizes = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device="cuda")
    w = torch.cat([sizes, -sizes])[codes[:, 0].int()] * torch.exp2(powers[:, 0].float() - 127)
    step = max(1, (1 << 26) // N)
    for m in range(0, M, step):     # exact products, rounded once by the scale's and once to bf16
        want = ((x[m:m + step].float() * w) * scale[m:m + step, None]).to(BF16)
        assert torch.equal(y[m:m + step], want), m
