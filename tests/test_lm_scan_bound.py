"""The scan's bounds hold for a plain float32 evaluation, cut into runs or not, and are narrow: outputs of
zeros, or of runs that do not hand on their states, are outside."""
import pytest

import lm_ref as ref
from lm_ref import TINY, rand

torch = pytest.importorskip("torch")
F32 = torch.float32
from lm_scan_ref import Bounded  # noqa: E402
from test_lm_scan_gpu import NAMES  # noqa: E402

SHAPES = [(200, 6, 16), (515, 9, 16), (300, 20, 8), (1030, 24, 4), (260, 5, 64)]   # T, channels, states


def inputs(T, D, N, slow, lengths=None):
    s = {"x": rand(1, (2, T, D), F32), "dt": rand(2, (2, T, D), F32, 0.5),
         "A": -torch.exp(rand(3, (D, N), F32, 0.7)) * (0.02 if slow else 1.0), "B": rand(4, (2, T, 1, N), F32),
         "C": rand(5, (2, T, 1, N), F32), "D": rand(6, (D,), F32), "z": rand(7, (2, T, D), F32),
         "dt_bias": rand(8, (D,), F32) - 2.0, "h0": rand(9, (2, D, N), F32)}
    return {**s, "lengths": None if lengths is None else torch.tensor(lengths, dtype=torch.int32)}


def evaluate(s, chunk, hand_on=True):
    """y and h by float32 operations, the sequence in runs of `chunk` tokens chained by their sums of steps."""
    st = torch.nn.functional.softplus(s["dt"] + s["dt_bias"])
    T = st.shape[1]
    h, ys = s["h0"], []
    for first in range(0, T, chunk):
        own, start = torch.zeros_like(h), h
        total = torch.zeros_like(st[:, 0])
        for t in range(first, min(first + chunk, T)):
            a = torch.exp(st[:, t, :, None] * s["A"])
            u = (st[:, t] * s["x"][:, t])[..., None] * s["B"][:, t]
            own, h = a * own + u, a * h + u
            total = total + st[:, t]
            y = (s["C"][:, t] * h).sum(-1) + s["D"] * s["x"][:, t]
            ys.append(y * s["z"][:, t] * torch.sigmoid(s["z"][:, t]))
        h = torch.exp(total[..., None] * s["A"]) * start + own if hand_on else own
    return torch.stack(ys, 1), h


@pytest.mark.parametrize("slow", [False, True])
@pytest.mark.parametrize("T,D,N", SHAPES)
def test_bounds(T, D, N, slow):
    s = inputs(T, D, N, slow)
    r = Bounded(**s, adds=T)
    r.forward()
    for chunk in (T, 64):
        y, h = evaluate(s, chunk)
        ref.close(y, r.y, r.bounds["y"] + TINY, "y")
        ref.close(h, r.h[:, -1], r.bounds["h"][:, -1] + TINY, "h")
    if slow:   # (fast decays leave nothing of a run's start at its end)
        y, _ = evaluate(s, 64, hand_on=False)
        wrong = (ref.f64(y) - r.y).abs() > r.bounds["y"] + TINY
        assert wrong[:, 64:].float().mean() > 0.9 and not wrong[:, :64].any()
    for name, bound, want in (("y", r.bounds["y"], r.y), ("h", r.bounds["h"][:, 1:], r.h[:, 1:])):
        assert (want.abs() > bound + TINY).float().mean() > 0.97, name
    dy, dh = rand(10, (2, T, D), F32), rand(11, (2, D, N), F32)
    got = r.backward(dy, dh)
    assert set(got) == set(NAMES)
    for name, (value, bound) in got.items():
        assert (value.abs() > bound + TINY).float().mean() > 0.9, name


@pytest.mark.parametrize("T,D,N", [(200, 6, 16), (300, 5, 8)])
def test_bounds_of_gradients(T, D, N):
    """Gradients by float32 operations (torch's, of the definition) are within them."""
    s = inputs(T, D, N, True)
    r = Bounded(**s, adds=T)
    r.forward()
    leaves = {k: (v.clone().requires_grad_(True) if v is not None else None) for k, v in s.items()}
    y, h = evaluate(leaves, T)
    dy, dh = rand(10, (2, T, D), F32), rand(11, (2, D, N), F32)
    torch.autograd.backward((y, h), (dy, dh))
    names = {"dx": "x", "ddt": "dt", "dA": "A", "dB": "B", "dC": "C", "dD": "D", "dz": "z", "dt_bias": "dt_bias", "dh0": "h0"}
    for name, (value, bound) in r.backward(dy, dh).items():
        ref.close(leaves[names[name]].grad.reshape(value.shape), value, bound + TINY, name)
