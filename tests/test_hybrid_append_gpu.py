"""Keys and values whose caches are parts of one allocation, and those that share
elements."""
import pytest

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


def _layouts(pages, page, heads, D, dtype):
    """(allocation, keys' and values' cache): halves of the pages, of a page, of a token, of a
    head's place, of its channels, pages taken in turn, and heads before tokens."""
    def made(*shape):
        g = torch.Generator(device="cuda").manual_seed(len(shape))
        return torch.randn(shape, generator=g, device="cuda").to(dtype)

    for at, shape in enumerate(((2, pages, page, heads, D), (pages, 2, page, heads, D), (pages, page, 2, heads, D),
                                (pages, page, heads, 2, D))):
        whole = made(*shape)
        yield whole, whole.select(at, 0), whole.select(at, 1)
    whole = made(pages, page, heads, 2 * D)
    yield whole, whole[..., D:], whole[..., :D]
    whole = made(2 * pages, page, heads, D)
    yield whole, whole[1::2], whole[::2]
    whole = made(pages, 2, heads, page, D)
    yield whole, whole[:, 0].transpose(1, 2), whole[:, 1].transpose(1, 2)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("pages,page,heads,D", [(6, 16, 2, 64), (9, 5, 3, 48), (4, 1, 1, 16), (1, 40, 4, 32)])
def test_caches_of_one_allocation(swr, dtype, pages, page, heads, D):
    g = torch.Generator(device="cuda").manual_seed(pages)
    n = pages * page
    k, v = torch.randn((2, n, heads, D), generator=g, device="cuda").to(dtype)
    slots = torch.randperm(n, generator=g, device="cuda")
    slots[0] = -1
    kept = slots >= 0
    q = torch.randn((1, 2 * heads, D), generator=g, device="cuda").to(dtype)
    table = torch.arange(pages, dtype=torch.int32, device="cuda")[None]
    length = torch.full((1,), n, dtype=torch.int32, device="cuda")
    for whole, kc, vc in _layouts(pages, page, heads, D, dtype):
        want = []
        for cache, new in ((kc, k), (vc, v)):
            flat = cache.reshape(n, heads, D).clone()
            flat[slots[kept]] = new[kept]
            want.append(flat.view(pages, page, heads, D))
        total = whole.numel()
        assert total == kc.numel() + vc.numel()     # (what is not a cache's element is none of the allocation's)
        swr.swr_cache_append(k, v, kc, vc, slots)
        torch.cuda.synchronize()
        assert torch.equal(kc, want[0]) and torch.equal(vc, want[1])
        got = swr.swr_paged_attention(q, kc, vc, table, length)
        assert torch.equal(got, swr.swr_paged_attention(q, want[0], want[1], table, length))


def test_caches_that_share_elements_are_refused(swr):
    whole = torch.zeros(5, 16, 2, 64, device="cuda", dtype=BF16)
    k = torch.ones(3, 2, 64, device="cuda", dtype=BF16)
    slots = torch.arange(3, device="cuda")
    wide = torch.zeros(4, 16, 2, 136, device="cuda", dtype=BF16)
    for kc, vc in ((whole, whole), (whole[1:], whole[:-1]), (whole[::2], whole[::2]), (whole[:2], whole[1:3]),
                   (whole[:, 1:], whole[:, :-1]), (wide[..., :64], wide[..., 56:120]), (wide[..., 64:128], wide[..., 8:72])):
        assert kc.shape == vc.shape and kc.stride() == vc.stride()
        with pytest.raises(swr.SwrError):
            swr.swr_cache_append(k, k, kc, vc, slots)
    torch.cuda.synchronize()
    assert (whole == 0).all() and (wide == 0).all()
