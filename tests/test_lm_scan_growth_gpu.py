"""Runs of the selective scan whose product of decays leaves float32, while no state does: against the
definition in 64 bits, and the same call in one run."""
import pytest

import lm_ref as ref
from lm_ref import TINY, rand
from lm_scan_ref import Bounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32 = torch.float32


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def problem(steps, N, D=16, seed=1):
    """One sequence with the given steps, B and C of one sign and size (sums do not cancel)."""
    T = len(steps)
    s = {"x": rand(seed, (1, T, D), F32, 0.5).abs() + 0.1, "dt": torch.tensor(steps).reshape(1, T, 1).expand(1, T, D).contiguous(),
         "A": 1.0 - 0.05 * torch.arange(N) / N * torch.ones(D, 1), "B": rand(seed + 1, (1, T, 1, N), F32, 0.5).abs() + 0.1,
         "C": rand(seed + 2, (1, T, 1, N), F32, 0.5).abs() + 0.1}
    return {k: v.cuda().contiguous() for k, v in s.items()}


def check(swr, s, dy, h0=None, dh=None):
    """Forward and backward against the definition; the sequence is cut (few channels, runs of 64 tokens)."""
    r = Bounded(s["x"], s["dt"], s["A"], s["B"], s["C"], use_softplus=False, h0=h0, adds=s["x"].shape[1])
    r.forward()
    assert float(r.h_size.max()) < 1e38   # (of a state in float32)
    y, carriers, h = swr.swr_selective_scan(**s, softplus=False, h0=h0, save_carriers=True, want_state=True)
    ref.close(y, r.y, r.y.abs() * ref.ROUND[F32] + r.bounds["y"] + TINY, "y")
    ref.close(h, r.h[:, -1], r.bounds["h"][:, -1] + TINY, "h_last")
    ref.close(carriers, r.h[:, :-1:16], r.bounds["h"][:, :-1:16] + TINY, "carriers")
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, softplus=False, h0=h0,
                                          dh_last=dh, want_dh0=True)
    want = r.backward(dy, dh)
    for name, g in zip(("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "dt_bias", "dh0"), got):
        if g is not None:
            value, bound = (t.reshape(g.shape) for t in want[name])
            assert float(value.abs().max()) < 1e37, name
            ref.close(g, value, value.abs() * ref.ROUND[F32] + bound + TINY, name)


GROW = [1.7] * 64           # exp(103) and more, 2^149: past float32, and its inverse too
FADE = [-1.7] * 64
FLAT = [0.01, -0.01] * 32


@pytest.mark.parametrize("N", [2, 4, 16, 20, 40])
def test_nothing_enters_a_growing_run(swr, N):
    """No state comes into the first run that grows, no gradient into the last: 0 times the product is 0."""
    s = problem(FLAT + GROW + FADE, N)
    s["x"][:, : 64 + 40] = 0.0   # (the state begins when it has 24 tokens left to grow)
    dy = torch.zeros_like(s["x"])
    dy[:, :88] = rand(5, (1, 88, 16), F32).cuda()   # (... and its gradient where 24 are left before)
    check(swr, s, dy)


@pytest.mark.parametrize("N", [4, 16, 40])
@pytest.mark.parametrize("steps", [GROW + FADE, FADE + GROW, FLAT + GROW + FADE, GROW + FLAT + FADE + FLAT])
def test_small_and_large_states(swr, N, steps):
    """A state that runs take from 1e-28 to 1e16 and more and back, or from 1e28 and back, and a gradient that they take
    from the end the other way."""
    s = problem(steps, N)
    s["x"][:] = 0.0
    small, large = (torch.full((1, 16, N), v, device="cuda") for v in (1e-28, 1e28))
    h0, dh = (large, small) if steps[0] < 0 else (small, large)
    check(swr, s, torch.zeros_like(s["x"]), h0, dh)


def test_infinite_and_missing_states_stay_so(swr):
    """What is infinite or no number in a run is it behind the run too; rates of minus infinity forget."""
    for rate, what in ((float("-inf"), 0.0), (0.0, 1.0)):
        s = problem([0.5] * 64 + [0.0] * 64, 16)
        s["A"][:] = rate
        h0 = rand(7, (1, 16, 16), F32).cuda()
        s["x"][:] = 0.0
        _, _, h = swr.swr_selective_scan(**s, softplus=False, h0=h0, want_state=True)
        assert torch.equal(h, h0 * what)
    s = problem([0.5] * 128, 16)
    s["dt"][:, 3, 2] = float("nan")
    _, _, h = swr.swr_selective_scan(**s, softplus=False, want_state=True)
    assert torch.isnan(h[:, 2]).all() and torch.isfinite(h[:, :2]).all() and torch.isfinite(h[:, 3:]).all()
