"""The selective scan on the GPU against its definition in 64 bits: forward, backward, single
tokens, over state counts, groups, lengths, layouts and the ways that the work is cut."""
import pytest

import lm_ref as ref
from lm_ref import ROUND, TINY, U, rand

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


def make(seed, B, T, D, N, G, dtype, z=True, skip=True, bias=True, h0=False, lengths=None, groups_dim=True):
    """Inputs on the GPU as a model has them: parts of projections' rows, strided."""
    s = {}
    both = rand(seed, (B, T, 2 * D + 3), dtype).cuda()
    s["x"] = both[..., 1:1 + D]
    s["dt"] = rand(seed + 1, (B, T, D), dtype, 0.5).cuda()
    s["A"] = -torch.exp(rand(seed + 2, (D, N), F32, 0.7)).cuda()
    parts = rand(seed + 3, (B, T, 2 * G * N + 5), dtype).cuda()
    s["B"], s["C"] = (parts[..., o:o + G * N].unflatten(2, (G, N)) for o in (5, 5 + G * N))
    if not groups_dim:
        s["B"], s["C"] = s["B"][:, :, 0], s["C"][:, :, 0]
    s["D"] = rand(seed + 4, (D,), F32).cuda() if skip else None
    s["z"] = both[..., 1 + D:1 + 2 * D] if z else None
    s["dt_bias"] = (rand(seed + 5, (D,), F32) - 2.0).cuda() if bias else None
    s["h0"] = rand(seed + 6, (B, D, N), F32).cuda() if h0 else None
    s["lengths"] = None if lengths is None else torch.tensor(lengths, dtype=torch.int32).cuda()
    return s


def definition(s, softplus=True):
    r = ref.Scan(s["x"], s["dt"], s["A"], s["B"], s["C"], s["D"], s["z"], s["dt_bias"], softplus, s["h0"], s["lengths"])
    r.forward()
    return r


def check_forward(r, y, h=None, carriers=None):
    dtype = y.dtype
    ref.close(y, r.y, r.y.abs() * ROUND[dtype] + r.y_bound * (1 + ROUND[dtype]) + TINY, "y")
    if h is not None:
        ref.close(h, r.h[:, -1], r.h_size[:, -1] * U * r.terms + TINY, "h_last")
    if carriers is not None:
        ref.close(carriers, r.h[:, :-1:16], r.h_size[:, :-1:16] * U * r.terms + TINY, "carriers")


NAMES = ("dx", "ddt", "dA", "dB", "dC", "dD", "dz", "dt_bias", "dh0")


def check_backward(s, r, got, dy, dh=None):
    want = r.backward(dy, dh)
    B, T, D = s["x"].shape
    for name, g in zip(NAMES, got):
        if name not in want or (name == "dD" and s["D"] is None) or (name == "dt_bias" and s["dt_bias"] is None) \
                or (name == "dz" and s["z"] is None):
            assert g is None, name
            continue
        if g is None:
            assert name == "dh0"
            continue
        value, size = want[name]
        # Sums over the channels of a group, over all tokens, beyond what lies on a term's way twice
        # (the states' and the gradients'), and the gates' roundings.
        terms = 2 * r.terms + {"dB": D, "dC": D, "dA": B * T, "dD": B * T, "dt_bias": B * T}.get(name, 0) + 32
        if s["z"] is not None:
            terms += 2 * float(s["z"].abs().float().nan_to_num(0, 0, 0).max()) + 8
        value = value.reshape(g.shape)
        ref.close(g, value, value.abs() * ROUND[g.dtype] + size.reshape(g.shape) * U * terms * (1 + ROUND[g.dtype])
                  + TINY, name)


SHAPES = [  # B, T, D, N, G
    (1, 1, 1, 1, 1), (2, 1, 70, 16, 1), (3, 7, 24, 4, 2), (2, 8, 5, 3, 1), (1, 9, 130, 16, 1), (2, 16, 64, 16, 1),
    (2, 17, 65, 8, 1), (1, 33, 66, 16, 3), (2, 40, 48, 5, 2), (1, 50, 20, 64, 2), (1, 31, 10, 33, 1),
    (1, 45, 36, 32, 1), (2, 29, 12, 24, 4), (1, 20, 300, 2, 1), (1, 130, 8, 16, 1)]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_forward_and_backward(swr, shape, dtype):
    B, T, D, N, G = shape
    s = make(1, *shape, dtype, h0=T % 2 == 1)
    r = definition(s)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(r, y, h, carriers)
    y2, none, none2 = swr.swr_selective_scan(**s)
    assert none is None and none2 is None and torch.equal(y, y2)
    dy, dh = rand(11, (B, T, D), dtype).cuda(), rand(12, (B, D, N), F32).cuda()
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                          s["dt_bias"], h0=s["h0"], dh_last=dh, want_dh0=True)
    check_backward(s, r, got, dy, dh)
    again = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, None, s["D"], s["z"],
                                            s["dt_bias"], h0=s["h0"], dh_last=dh, want_dh0=True)
    check_backward(s, r, again, dy, dh)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,D,N", [(200, 6, 16), (515, 70, 16), (300, 20, 8), (1030, 3, 4), (260, 5, 64)])
def test_runs(swr, dtype, T, D, N):
    """Few channels and many tokens: the sequence in runs, with a state before and after."""
    s = make(2, 2, T, D, N, 1, dtype, h0=True, lengths=[T, T - 77])
    r = definition(s)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(r, y, h, carriers)
    dy, dh = rand(13, (2, T, D), dtype).cuda(), rand(14, (2, D, N), F32).cuda()
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                          s["dt_bias"], h0=s["h0"], dh_last=dh, lengths=s["lengths"], want_dh0=True)
    check_backward(s, r, got, dy, dh)


def test_many_channels(swr):
    """Enough channels that a lane has 16 states and the sequences are whole."""
    for N, D in ((16, 9000), (32, 5000)):
        s = make(3, 16, 20, D, N, 1, BF16)
        r = definition(s)
        y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
        check_forward(r, y, h, carriers)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("lengths", [[0, 1, 5, 16], [17, 40, 0, 39], [100, -3, 33, 40]])
def test_lengths(swr, dtype, lengths):
    """Batches of different lengths (0, past T, negative); what is behind them is not looked at."""
    B, T, D, N = 4, 40, 20, 16
    s = make(4, B, T, D, N, 2, dtype, h0=True, lengths=lengths)
    dy, dh = rand(15, (B, T, D), dtype).cuda(), rand(16, (B, D, N), F32).cuda()
    for i, n in enumerate(lengths):
        for k, t in enumerate((s["x"], s["dt"], s["B"], s["C"], s["z"], dy)):
            t[i, max(n, 0):] = (float("nan"), float("inf"))[(i + k) % 2]
    r = definition(s)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(r, y, h, carriers)
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                          s["dt_bias"], h0=s["h0"], dh_last=dh, lengths=s["lengths"], want_dh0=True)
    check_backward(s, r, got, dy, dh)


@pytest.mark.parametrize("z", [False, True])
@pytest.mark.parametrize("skip", [False, True])
@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("softplus", [False, True])
def test_options(swr, z, skip, bias, softplus):
    for T in (3, 21):
        s = make(5, 2, T, 18, 6, 1, F32, z=z, skip=skip, bias=bias, groups_dim=False)
        if not softplus:
            s["dt"] = s["dt"].abs()
            if bias:
                s["dt_bias"] = s["dt_bias"].abs()
        r = definition(s, softplus)
        y, carriers, h = swr.swr_selective_scan(**s, softplus=softplus, save_carriers=True, want_state=True)
        check_forward(r, y, h, carriers)
        dy = rand(17, s["x"].shape, F32).cuda()
        got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                              s["dt_bias"], softplus=softplus)
        assert got[3].shape == s["B"].shape and got[8] is None
        check_backward(s, r, got, dy)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("N,G", [(16, 1), (16, 2), (3, 1), (64, 1), (24, 2), (1, 1)])
def test_tokens_one_by_one(swr, dtype, N, G):
    """A prompt, then single tokens: each step's output, the state in place, as the whole sequence has them."""
    B, T, D = 3, 26, 34
    s = make(6, B, T, D, N, G, dtype)
    r = definition(s)
    part = {k: (v[:, :20] if k in ("x", "dt", "B", "C", "z") else v) for k, v in s.items()}
    y, _, state = swr.swr_selective_scan(**part, want_state=True)
    check_forward(definition(part), y, state)
    ys = [y]
    for t in range(20, T):
        x, dt, b, c, z = (s[k][:, t] for k in ("x", "dt", "B", "C", "z"))
        held = state
        if t % 2:
            yt = swr.swr_selective_step(x, dt, s["A"], b, c, state, s["D"], z, s["dt_bias"])
        else:
            yt = torch.empty(B, 3 * D, dtype=dtype, device="cuda")[:, D:2 * D]
            out = swr.swr_selective_step(x, dt, s["A"], b, c, state, s["D"], z, s["dt_bias"], y=yt)
            assert out is yt
        assert state is held
        ys.append(yt[:, None])
    check_forward(r, torch.cat(ys, 1), state)


def test_extreme_values(swr):
    """Steps from 1e-30 to large ones, rates of zero and minus infinity, growth, an infinite state."""
    B, T, D, N = 1, 24, 8, 16
    s = make(7, B, T, D, N, 1, F32, z=False, skip=False, bias=False)
    s["dt"] = torch.linspace(-75, 30, T).reshape(1, T, 1).expand(B, T, D).contiguous().cuda()
    s["A"][0] = 0.0
    s["A"][1] = float("-inf")
    s["A"][2] = 1e-3
    s["A"] = s["A"].contiguous()
    keep = [c for c in range(D) if c != 1]
    r = definition({**s, "x": s["x"][..., keep], "dt": s["dt"][..., keep], "A": s["A"][keep]})
    y, _, h = swr.swr_selective_scan(**s, want_state=True)
    check_forward(r, y[..., keep].contiguous(), h[:, keep].contiguous())
    # A rate of minus infinity forgets everything but the token's own input.
    u = ref.softplus(ref.f64(s["dt"][:, -1, 1])) * ref.f64(s["x"][:, -1, 1])
    want = u[:, None] * ref.f64(s["B"][:, -1, 0])
    ref.close(h[:, 1], want, want.abs() * U * 128 + TINY, "forgotten")


def test_strides_and_reuse(swr):
    """Outputs into given tensors (strided), the state in place, an explicit workspace, and
    transposed or stepped inputs that have to be refused."""
    B, T, D, N = 2, 70, 40, 16
    s = make(8, B, T, D, N, 1, BF16, h0=True)
    want, _, h = swr.swr_selective_scan(**s, want_state=True)
    wide = torch.full((B, T, 3 * D), 7.0, dtype=BF16, device="cuda")
    state = s["h0"].clone()
    y, none, out = swr.swr_selective_scan(**{**s, "h0": state}, h_last=state, y=wide[..., D:2 * D],
                                          workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    assert out is state and none is None
    assert torch.equal(y, want) and torch.equal(state, h)
    assert (wide[..., :D] == 7).all() and (wide[..., 2 * D:] == 7).all()
    # a batch expanded from one
    one = {k: (v[:1].expand(3, *v.shape[1:]) if k in ("x", "dt", "B", "C", "z") else v) for k, v in s.items()}
    one["h0"] = None
    y3, _, _ = swr.swr_selective_scan(**one)
    assert torch.equal(y3[0], y3[2])
    with pytest.raises(ValueError):
        swr.swr_selective_scan(**{**s, "x": s["x"].transpose(1, 2).contiguous().transpose(1, 2)})
    with pytest.raises(ValueError):
        swr.swr_selective_scan(**{**s, "A": s["A"].t().contiguous().t()})
    with pytest.raises(swr.SwrError):
        swr.swr_selective_scan(**s, y=s["x"])


def test_empty(swr):
    s = make(9, 2, 0, 8, 16, 1, BF16, h0=True)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    assert y.shape == (2, 0, 8) and carriers.numel() == 0 and torch.equal(h, s["h0"])
    dh = rand(18, h.shape, F32).cuda()
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], y, carriers, s["D"], s["z"],
                                          s["dt_bias"], h0=s["h0"], dh_last=dh, want_dh0=True)
    assert (got[2] == 0).all() and (got[5] == 0).all() and (got[7] == 0).all() and torch.equal(got[8], dh)
    s = make(9, 0, 5, 8, 16, 1, BF16)
    y, _, h = swr.swr_selective_scan(**s, want_state=True)
    assert y.shape == (0, 5, 8) and h.shape == (0, 8, 16)
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], y, None, s["D"], s["z"], s["dt_bias"])
    assert (got[2] == 0).all()


def test_autograd(swr):
    s = make(10, 2, 37, 12, 8, 1, F32, h0=True)
    names = [k for k in s if k != "lengths"]
    leaves = {k: s[k].detach().clone().requires_grad_(True) for k in names}
    y, h = swr.SWRSelectiveScanFunction.apply(*(leaves[k] for k in ("x", "dt", "A", "B", "C", "D", "z", "dt_bias")),
                                              True, leaves["h0"], None)
    dy, dh = rand(19, y.shape, F32).cuda(), rand(20, h.shape, F32).cuda()
    (y * dy).sum().backward(retain_graph=True)
    r = definition({**{k: v.detach() for k, v in leaves.items()}, "lengths": None})
    order = ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "h0")
    check_backward(s, r, [leaves[k].grad for k in order], dy)
    for k in names:
        leaves[k].grad = None
    torch.autograd.backward((y, h), (dy, dh), retain_graph=True)
    check_backward(s, r, [leaves[k].grad for k in order], dy, dh)
    for k in names:
        leaves[k].grad = None
    (h * dh).sum().backward()
    check_backward(s, definition({**{k: v.detach() for k, v in leaves.items()}, "lengths": None}),
                   [leaves[k].grad for k in order], torch.zeros_like(dy), dh)


def test_far_rows(swr):
    """Tokens so far apart that a tile of them passes 31 bits of bytes."""
    B, T, D, N = 1, 40, 6, 16
    s = make(21, B, T, D, N, 1, BF16)
    far = torch.zeros((T, (1 << 22) + 64), dtype=BF16, device="cuda")
    far[:, :D] = s["x"][0]
    want = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    s["x"] = far[None, :, :D]
    r = definition(s)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(r, y, h, carriers)
    check_forward(r, want[0], want[2], want[1])
    dy = rand(22, (B, T, D), BF16).cuda()
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                          s["dt_bias"])
    check_backward(s, r, got, dy)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 2, 8, 9])
@pytest.mark.parametrize("B,D,N,G", [(1, 5, 16, 5), (5, 130, 16, 2), (3, 7, 6, 1), (2, 9, 64, 9), (7, 6, 1, 3)])
def test_few_tokens(swr, dtype, T, B, D, N, G):
    """Odd numbers of batches, groups of one channel, lengths of all kinds, the state in place."""
    lengths = [(T, 0, 1, T + 3, -1, T // 2, T - 1)[i] for i in range(B)]
    s = make(40, B, T, D, N, G, dtype, h0=True, lengths=lengths)
    for i, n in enumerate(lengths):
        for k, t in enumerate((s["x"], s["dt"], s["B"], s["C"], s["z"])):
            t[i, max(n, 0):] = (float("nan"), float("inf"))[(i + k) % 2]
    r = definition(s)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(r, y, h, carriers)
    state = s["h0"].clone()
    again, none, last = swr.swr_selective_scan(**{**s, "h0": state}, h_last=state)
    assert last is state and none is None and torch.equal(again, y) and torch.equal(state, h)
    s["lengths"] = None
    for k in ("x", "dt", "B", "C", "z"):
        s[k] = torch.nan_to_num(s[k].contiguous(), 0.5, 0.5, -0.5)
    bare = {**s, "h0": None, "z": None, "D": None, "dt_bias": None}
    for given in (s, bare):
        r = definition(given)
        y, _, h = swr.swr_selective_scan(**given, want_state=True)
        check_forward(r, y, h)


@pytest.mark.parametrize("seed", range(12))
def test_mixed_shapes(swr, seed):
    """Shapes and options drawn at random, forward and backward."""
    import random
    rng = random.Random(seed)
    G, B, T, N = rng.choice((1, 1, 2, 5)), rng.randint(1, 5), rng.randint(1, 100), rng.randint(1, 64)
    D, dtype = G * rng.randint(1, 40), rng.choice((BF16, F32))
    lengths = [rng.randint(0, T) for _ in range(B)] if rng.random() < 0.6 else None
    z, skip, bias, h0 = (rng.random() < 0.7 for _ in range(4))
    s = make(50 + seed, B, T, D, N, G, dtype, z, skip, bias, h0, lengths)
    r = definition(s)
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(r, y, h, carriers)
    dy, dh = rand(70, (B, T, D), dtype).cuda(), rand(71, (B, D, N), F32).cuda()
    got = swr.swr_selective_scan_backward(s["x"], s["dt"], s["A"], s["B"], s["C"], dy, carriers, s["D"], s["z"],
                                          s["dt_bias"], h0=s["h0"], dh_last=dh, lengths=s["lengths"], want_dh0=True)
    check_backward(s, r, got, dy, dh)
