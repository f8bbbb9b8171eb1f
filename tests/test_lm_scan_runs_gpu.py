"""Sequences of the selective scan that are cut into runs, and many whole ones, on the GPU against the
definition in 64 bits, within bounds that follow each state (lm_scan_ref)."""
import random

import pytest

import lm_ref as ref
from lm_ref import ROUND, TINY, rand
from lm_scan_ref import Bounded

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32
from test_lm_scan_gpu import NAMES, make  # noqa: E402


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def check(swr, s, softplus=True, dh=True):
    """Forward and backward of inputs as test_lm_scan_gpu.make has them."""
    B, T, D = s["x"].shape
    dtype = s["x"].dtype
    r = Bounded(s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["z"], s["dt_bias"], softplus, s["h0"], s["lengths"],
                adds=T)
    r.forward()
    y, carriers, h = swr.swr_selective_scan(**s, softplus=softplus, save_carriers=True, want_state=True)
    ref.close(y, r.y, r.y.abs() * ROUND[dtype] + r.bounds["y"] * (1 + ROUND[dtype]) + TINY, "y")
    ref.close(h, r.h[:, -1], r.bounds["h"][:, -1] + TINY, "h_last")
    ref.close(carriers, r.h[:, :-1:16], r.bounds["h"][:, :-1:16] + TINY, "carriers")
    y2, _, h2 = swr.swr_selective_scan(**s, softplus=softplus, want_state=True)
    assert torch.equal(y2, y) and torch.equal(h2, h)
    dy = rand(91, (B, T, D), dtype).cuda()
    dlast = rand(92, tuple(h.shape), F32).cuda() if dh else None
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                          s["dt_bias"], softplus=softplus, h0=s["h0"], dh_last=dlast,
                                          lengths=s["lengths"], want_dh0=True)
    want = r.backward(dy, dlast)
    there = {"dD": s["D"], "dz": s["z"], "dt_bias": s["dt_bias"]}
    for name, g in zip(NAMES, got):
        if name in there and there[name] is None:
            assert g is None, name
            continue
        value, bound = (t.reshape(g.shape) for t in want[name])
        ref.close(g, value, value.abs() * ROUND[g.dtype] + bound * (1 + ROUND[g.dtype]) + TINY, name)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("slow", [False, True])
@pytest.mark.parametrize("T,D,N,G", [(200, 6, 16, 1), (515, 70, 16, 1), (300, 20, 8, 2), (1030, 3, 4, 1), (260, 5, 64, 1),
                                     (700, 12, 24, 3), (130, 300, 1, 1), (200, 40, 33, 2)])
def test_runs(swr, dtype, slow, T, D, N, G):
    """Slow decays, so that a run's start is seen to the end of the sequence, and ordinary ones."""
    s = make(2, 2, T, D, N, G, dtype, h0=True, lengths=[T, T - 77])
    if slow:
        s["A"] = s["A"] * 0.02
    check(swr, s)


@pytest.mark.parametrize("seed", range(10))
def test_mixed_runs(swr, seed):
    """Shapes and options drawn at random, of sequences that are cut."""
    rng = random.Random(seed)
    G, B, T, N = rng.choice((1, 1, 2, 3)), rng.randint(1, 4), rng.randint(128, 900), rng.randint(1, 64)
    D, dtype = G * rng.randint(1, 24), rng.choice((BF16, F32))
    lengths = [rng.randint(0, T) for _ in range(B)] if rng.random() < 0.6 else None
    z, skip, bias, h0 = (rng.random() < 0.7 for _ in range(4))
    s = make(200 + seed, B, T, D, N, G, dtype, z, skip, bias, h0, lengths)
    s["A"] = s["A"] * rng.choice((1.0, 0.1, 0.01))
    check(swr, s, dh=rng.random() < 0.7)


@pytest.mark.parametrize("N,D", [(16, 2200), (32, 1100), (8, 4100), (3, 9000)])
def test_many_whole_sequences(swr, N, D):
    """Enough channels and batches that no sequence is cut, forward and backward, over several tiles of tokens."""
    check(swr, make(3, 4, 37, D, N, 1, BF16, lengths=[37, 16, 0, 33]))
