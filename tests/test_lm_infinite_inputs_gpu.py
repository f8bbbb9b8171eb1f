"""Infinite inputs: what the definitions make of them, and nothing else, wherever runs of tokens and sequences end."""
import pytest

import lm_ref as ref
from lm_ref import rand

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32
INF = float("inf")


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def same_kinds(got, want, what):
    """Infinities and NaN where the definition has them."""
    got, want = ref.f64(got), want.to(torch.float64)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what
    assert torch.equal(torch.isinf(got), torch.isinf(want)), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("K", [1, 2, 4, 8])
@pytest.mark.parametrize("at", [0, 15, 16, 17, 31, 32, 36, 39])
def test_convolution(swr, dtype, K, at):
    """An infinite x next to the places where runs of 16 tokens meet: without the SiLU its weights' gradients are
    infinite, not NaN (no gradient there is zero)."""
    B, T, C = 2, 40, 9
    x, w = rand(1, (B, T, C), dtype).cuda(), rand(2, (C, K), dtype).cuda()
    dy = (rand(3, (B, T, C), dtype).abs() + 0.5).to(dtype).cuda()
    x[0, at, 3], x[1, at, 5] = INF, -INF
    want = ref.conv_backward(x, w, None, False, None, dy)
    got = swr.swr_causal_conv_backward(x, w, dy, silu=False)
    same_kinds(got[0], want[0], "dx")
    same_kinds(got[1], want[1], "dw")
    assert torch.isinf(want[1][[3, 5]]).any() and not torch.isnan(want[1]).any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N", [3, 16, 20, 64])
@pytest.mark.parametrize("T", [21, 200])
def test_scan_past_the_lengths(swr, dtype, N, T):
    """A state that is infinite at its batch's last token: outputs and gradients past it are zeros all the same."""
    B, D, n = 3, 5, [T - 3, T - 11, T]
    x, dt, z, dy = (rand(i, (B, T, D), dtype).cuda() for i in (1, 2, 3, 4))
    b, c = (rand(i, (B, T, 1, N), dtype).cuda() for i in (5, 6))
    A, dh = -torch.exp(rand(7, (D, N), F32)).cuda(), rand(8, (B, D, N), F32).cuda()
    lengths = torch.tensor(n, dtype=torch.int32).cuda()
    for i in range(B):
        x[i, n[i] - 1, 1] = INF
    y, carriers, h = swr.swr_selective_scan(x, dt, A, b, c, z=z, lengths=lengths, save_carriers=True, want_state=True)
    assert not torch.isfinite(h[:, 1]).any() and torch.isfinite(h[:, [0, 2, 3, 4]]).all()
    got = swr.swr_selective_scan_backward(x, dt, A, b, c, dy, carriers, z=z, dh_last=dh, lengths=lengths)
    for i in range(B):
        for t in (y, got[0], got[1], got[3], got[4], got[6]):
            assert (t[i, n[i]:] == 0).all()
