"""The language model operators' native marshalling against the Python path (the same results, the
same refusals), streams, captured graphs, and calls side by side."""
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


class _Nothing:
    """A native module that handles no call."""
    def __getattr__(self, name):
        return lambda *args: None


def _python(swr, monkeypatch):
    monkeypatch.setattr(swr, "_native", (swr._lib, _Nothing()))


def _inputs(dtype, T=150):
    g = torch.Generator(device="cuda").manual_seed(3)

    def t(*shape, by=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * by).to(dtype)

    B, D, N, G, V = 3, 64, 16, 2, 1009
    tokens = torch.randint(-1, V + 1, (B, T), generator=g, device="cuda")
    both = t(B, T, 2 * D)
    lengths = torch.tensor([T, 0, T // 2 + 1], dtype=torch.int32, device="cuda")
    return {"tokens": tokens, "tokens32": tokens.int(), "table": t(V, D), "dy": t(B, T, D), "x": both[..., :D],
            "z": both[..., D:], "w": t(D, 4), "bias": t(D), "past": t(B, 3, D), "dt": t(B, T, D, by=0.5),
            "A": -torch.exp(t(D, N).float()), "B": t(B, T, G, N), "C": t(B, T, G, N), "skip": t(D).float(),
            "dt_bias": t(D).float() - 2, "h0": t(B, D, N).float(), "lengths": lengths, "logits": t(B, T, V),
            "few": t(2, 50001), "few_tokens": torch.tensor([5, 50000], device="cuda"),
            "dlogp": t(B, T).float(), "dent": t(B, T).float(), "vocab": V}


def _scan_args(i):
    return (i["x"], i["dt"], i["A"], i["B"], i["C"])


def _calls(swr, i):
    V = i["vocab"]
    yield swr.swr_embedding(i["tokens"], i["table"])
    yield swr.swr_embedding(i["tokens32"], i["table"], 0.5)
    yield swr.swr_embedding(i["tokens"][0, 0], i["table"])
    yield swr.swr_embedding_backward(i["tokens"], i["dy"], V)
    yield swr.swr_embedding_backward(i["tokens32"], i["dy"], V, 2.0, i["dy"].dtype)
    yield swr.swr_embedding_backward(i["tokens"], i["x"], V, dtype=F32)
    yield swr.swr_causal_conv(i["x"], i["w"])
    yield swr.swr_causal_conv(i["x"], i["w"], i["bias"], False, i["past"], i["lengths"], want_state=True)
    yield swr.swr_causal_conv(i["x"], i["w"][:, :1].contiguous(), want_state=True)
    past = i["past"].clone()
    yield swr.swr_causal_conv_step(i["x"][:, 0], i["w"], past, i["bias"]), past
    yield swr.swr_causal_conv_backward(i["x"], i["w"], i["dy"])
    yield swr.swr_causal_conv_backward(i["x"], i["w"], i["dy"], i["bias"], False, i["lengths"])
    yield swr.swr_selective_scan(*_scan_args(i))
    y, carriers, h = swr.swr_selective_scan(*_scan_args(i), i["skip"], i["z"], i["dt_bias"], True, i["h0"], i["lengths"],
                                            True, True)
    yield y, carriers, h
    state = i["h0"].clone()
    yield swr.swr_selective_step(i["x"][:, 0], i["dt"][:, 0], i["A"], i["B"][:, 0], i["C"][:, 0], state, i["skip"],
                                 i["z"][:, 0], i["dt_bias"]), state
    state = i["h0"].clone()
    yield swr.swr_selective_step(i["x"][:, 0], i["dt"][:, 0], i["A"], i["B"][:, 0, 0], i["C"][:, 0, 1], state), state
    yield swr.swr_selective_scan_backward(*_scan_args(i), i["dy"], carriers, i["skip"], i["z"], i["dt_bias"], True,
                                          i["h0"], i["h0"], i["lengths"], True)
    yield swr.swr_selective_scan_backward(i["x"], i["dt"], i["A"], i["B"][:, :, 0], i["C"][:, :, 0], i["dy"],
                                          swr.swr_selective_scan(i["x"], i["dt"], i["A"], i["B"][:, :, 0], i["C"][:, :, 0],
                                                                 save_carriers=True)[1])
    yield swr.swr_log_probs(i["logits"], i["tokens"])
    logp, lse, ent, top, best = swr.swr_log_probs(i["logits"], i["tokens32"], 20, 0.7)
    yield logp, lse, ent, top, best
    yield swr.swr_log_probs(i["few"], i["few_tokens"], 64)
    yield swr.swr_log_probs(i["few"][0], i["few_tokens"][0], 1)
    yield swr.swr_log_probs_backward(i["logits"], i["tokens"], lse, ent, i["dlogp"], scale=0.7)
    yield swr.swr_log_probs_backward(i["logits"], i["tokens"], lse, ent, i["dlogp"], i["dent"], i["dent"], 0.7)


def _same(u, w, what):
    u, w = (r if isinstance(r, (tuple, list)) else (r,) for r in (u, w))
    assert len(u) == len(w), what
    for p, q in zip(u, w):
        assert (p is None) == (q is None), what
        if p is not None:
            assert p.dtype == q.dtype and p.shape == q.shape and p.stride() == q.stride(), what
            assert torch.equal(*(t.contiguous().view(-1).view(torch.uint8) for t in (p, q))), what


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_native_and_python_paths_agree(swr, monkeypatch, dtype):
    inputs = _inputs(dtype)
    native = list(_calls(swr, inputs))
    _python(swr, monkeypatch)
    python = list(_calls(swr, inputs))
    torch.cuda.synchronize()
    assert len(native) == len(python)
    for n, (u, w) in enumerate(zip(native, python)):
        _same(u, w, n)


@pytest.mark.parametrize("native", [True, False])
def test_refusals(swr, monkeypatch, native):
    if not native:
        _python(swr, monkeypatch)
    i = _inputs(BF16)
    x, w, dy, tokens, table, logits, V = (i[k] for k in ("x", "w", "dy", "tokens", "table", "logits", "vocab"))
    dt, A, B, C = (i[k] for k in ("dt", "A", "B", "C"))
    y, carriers, _ = swr.swr_selective_scan(x, dt, A, B, C, save_carriers=True)
    logp, lse, ent = swr.swr_log_probs(logits, tokens)
    state = i["h0"].clone()
    for n, (error, call) in enumerate((
            (TypeError, lambda: swr.swr_embedding(tokens.short(), table)),
            (TypeError, lambda: swr.swr_embedding(tokens, table.half())),
            (ValueError, lambda: swr.swr_embedding(tokens, table[0])),
            (ValueError, lambda: swr.swr_embedding(tokens, table.t())),
            (ValueError, lambda: swr.swr_embedding(tokens.cpu(), table)),
            (ValueError, lambda: swr.swr_embedding(tokens.t(), table)),
            (ValueError, lambda: swr.swr_embedding(tokens, table, float("nan"))),
            (ValueError, lambda: swr.swr_embedding(tokens, table, y=x[:, :3])),
            (swr.SwrError, lambda: swr.swr_embedding(tokens, table[:0])),
            (ValueError, lambda: swr.swr_embedding_backward(tokens[:, :3], dy, V)),
            (TypeError, lambda: swr.swr_embedding_backward(tokens, dy.half(), V)),
            (swr.SwrError, lambda: swr.swr_embedding_backward(tokens, dy, 0)),
            (ValueError, lambda: swr.swr_embedding_backward(tokens, dy, V, workspace=torch.empty(4, device="cuda"))),
            (TypeError, lambda: swr.swr_causal_conv(x.half(), w)),
            (ValueError, lambda: swr.swr_causal_conv(x, w[:60])),
            (ValueError, lambda: swr.swr_causal_conv(x, w.float())),
            (ValueError, lambda: swr.swr_causal_conv(x[0], w)),
            (ValueError, lambda: swr.swr_causal_conv(x.transpose(1, 2), w)),
            (ValueError, lambda: swr.swr_causal_conv(x, w, i["bias"].float())),
            (ValueError, lambda: swr.swr_causal_conv(x, w, state=i["past"][:, :2])),
            (ValueError, lambda: swr.swr_causal_conv(x, w, lengths=i["lengths"].long())),
            (ValueError, lambda: swr.swr_causal_conv(x, w, lengths=i["lengths"][:2])),
            (swr.SwrError, lambda: swr.swr_causal_conv(x, w.repeat(1, 3))),
            (swr.SwrError, lambda: swr.swr_causal_conv(x, w[:, :0].contiguous())),
            (swr.SwrError, lambda: swr.swr_causal_conv(x, w, y=x)),
            (ValueError, lambda: swr.swr_causal_conv_step(x, w, i["past"])),
            (ValueError, lambda: swr.swr_causal_conv_step(x[:, 0], w, i["past"][:2])),
            (ValueError, lambda: swr.swr_causal_conv_backward(x, w, dy[:, :5])),
            (ValueError, lambda: swr.swr_causal_conv_backward(x, w, dy.float())),
            (TypeError, lambda: swr.swr_selective_scan(x.half(), dt, A, B, C)),
            (ValueError, lambda: swr.swr_selective_scan(x, dt[:, :5], A, B, C)),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A.bfloat16(), B, C)),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A[:32], B, C)),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B, C[:, :, 0])),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B[..., :8], C)),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B.float(), C)),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B[:, :, [0, 1, 0]], C[:, :, [0, 1, 0]])),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B, C, i["skip"].bfloat16())),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B, C, z=i["z"][:2])),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B, C, h0=i["h0"][:2])),
            (ValueError, lambda: swr.swr_selective_scan(x, dt, A, B, C, lengths=i["lengths"].long())),
            (swr.SwrError, lambda: swr.swr_selective_scan(x, dt, A.repeat(1, 5), B.repeat(1, 1, 1, 5), C.repeat(1, 1, 1, 5))),
            (swr.SwrError, lambda: swr.swr_selective_scan(x, dt, A, B, C, y=x)),
            (ValueError, lambda: swr.swr_selective_step(x, dt, A, B, C, state)),
            (ValueError, lambda: swr.swr_selective_step(x[:, 0], dt[:, 0], A, B[:, 0], C[:, 0], state[:2])),
            (ValueError, lambda: swr.swr_selective_scan_backward(x, dt, A, B, C, dy, carriers[:, :2])),
            (ValueError, lambda: swr.swr_selective_scan_backward(x, dt, A, B, C, dy[:, :2], carriers)),
            (ValueError, lambda: swr.swr_selective_scan_backward(x, dt, A, B, C, dy, carriers, dh_last=state[:1])),
            (TypeError, lambda: swr.swr_log_probs(logits.half(), tokens)),
            (TypeError, lambda: swr.swr_log_probs(logits, tokens.float())),
            (ValueError, lambda: swr.swr_log_probs(logits, tokens[:2])),
            (ValueError, lambda: swr.swr_log_probs(logits, tokens, 65)),
            (ValueError, lambda: swr.swr_log_probs(logits[..., :4], tokens, 5)),
            (ValueError, lambda: swr.swr_log_probs(logits, tokens, scale=float("inf"))),
            (swr.SwrError, lambda: swr.swr_log_probs(logits, tokens, scale=0.0)),
            (ValueError, lambda: swr.swr_log_probs(logits.transpose(0, 1), tokens)),
            (ValueError, lambda: swr.swr_log_probs_backward(logits, tokens, lse[:1], ent, logp)),
            (ValueError, lambda: swr.swr_log_probs_backward(logits, tokens, lse, ent, logp.bfloat16())),
            (swr.SwrError, lambda: swr.swr_log_probs_backward(logits, tokens, lse, ent, logp, scale=-1.0)))):
        with pytest.raises(error):
            call()
            raise AssertionError(n)
    torch.cuda.synchronize()


def _used(t):
    return [r for r in (t if isinstance(t, (tuple, list)) else (t,)) if r is not None]


@pytest.mark.parametrize("native", [True, False])
def test_the_current_and_a_given_stream(swr, monkeypatch, native):
    """Both paths launch on torch's current stream, or on the one that is given, workspaces too."""
    if not native:
        _python(swr, monkeypatch)
    i = _inputs(BF16)
    _, carriers, _ = swr.swr_selective_scan(*_scan_args(i), save_carriers=True)
    _, lse, ent = swr.swr_log_probs(i["logits"], i["tokens"])
    calls = {
        "dy": lambda t, **kw: swr.swr_embedding_backward(i["tokens"], t, i["vocab"], **kw),
        "table": lambda t, **kw: swr.swr_embedding(i["tokens"], t, **kw),
        "x": lambda t, **kw: swr.swr_causal_conv(t, i["w"], want_state=True, **kw),
        "w": lambda t, **kw: swr.swr_causal_conv_backward(i["x"], t, i["dy"], **kw),
        "dt": lambda t, **kw: swr.swr_selective_scan(i["x"], t, i["A"], i["B"], i["C"], want_state=True, **kw),
        "B": lambda t, **kw: swr.swr_selective_scan_backward(i["x"], i["dt"], i["A"], t, i["C"], i["dy"], carriers, **kw),
        "few": lambda t, **kw: swr.swr_log_probs(t, i["few_tokens"], 30, **kw),
        "logits": lambda t, **kw: swr.swr_log_probs_backward(t, i["tokens"], lse, ent, i["dlogp"], **kw)}
    s = torch.cuda.Stream()
    for name, call in calls.items():
        want = _used(call(i[name]))
        t = torch.zeros(i[name].shape, dtype=i[name].dtype, device="cuda")
        for given in (False, True):
            t.zero_()
            torch.cuda.synchronize()
            with torch.cuda.stream(s):
                for _ in range(50):   # work that the call has to come after
                    big = torch.randn(1 << 20, device="cuda")
                t.copy_(i[name])
                if not given:
                    got = call(t)
            if given:
                got = call(t, stream=s)
            s.synchronize()
            for a, b in zip(_used(got), want):
                assert torch.equal(a, b), (name, given)
            del big


@pytest.mark.parametrize("T", [150, 1])
def test_captured_graphs(swr, T):
    """Every call captured, two graphs of the same calls at once; replays with eager calls and
    synchronizations between them equal the eager results, for inputs that change too."""
    i = _inputs(BF16, T)
    eager = [_used(r) for r in _calls(swr, i)]
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = [_used(r) for r in _calls(swr, i)]
        graphs.append((graph, out))
    changed = _inputs(BF16, T)
    for n in range(4):
        if n == 2:   # other inputs in place, and the eager results of those
            for name, t in changed.items():
                if name in ("table", "dy", "logits", "few", "dt", "B"):
                    i[name].copy_(torch.roll(t.flatten(), 7).view(t.shape))
            eager = [_used(r) for r in _calls(swr, i)]
        for _, out in graphs:
            for r in out:
                for t in r:
                    t.zero_()
        streams = [torch.cuda.Stream() for _ in graphs]
        torch.cuda.synchronize()
        for (graph, _), s in zip(graphs, streams):   # the two side by side
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            for k, (a, b) in enumerate(zip(out, eager)):
                for p, q in zip(a, b):
                    assert torch.equal(p, q), (n, k)
        swr.swr_embedding_backward(i["tokens"], i["dy"], i["vocab"])
        swr.swr_log_probs(i["few"], i["few_tokens"], 10)


def test_a_captured_training_step(swr):
    """Forward and backward of a chain of the operators in a graph, replayed."""
    i = _inputs(BF16)
    V, D = i["vocab"], 64
    leaves = [i[k].detach().clone().requires_grad_() for k in ("table", "w", "bias", "A", "skip", "dt_bias")]

    def grads():
        table, w, bias, A, skip, dt_bias = leaves
        h = swr.SWREmbeddingFunction.apply(i["tokens"], table)
        x = swr.SWRCausalConvFunction.apply(h, w, bias, True, i["lengths"])
        y, _ = swr.SWRSelectiveScanFunction.apply(x, h, A, i["B"], i["C"], skip, i["z"], dt_bias, True, None, i["lengths"])
        logits = y @ table.t()
        logp, _, ent = swr.SWRLogProbsFunction.apply(logits, i["tokens"])
        return [logp.detach(), *torch.autograd.grad([logp, ent], leaves, ones)]

    ones = [torch.ones(3, 150, device="cuda"), torch.full((3, 150), 0.01, device="cuda")]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(2):
            want = [t.clone() for t in grads()]
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = grads()
    for n in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for k, (a, b) in enumerate(zip(got, want)):
            assert torch.equal(a, b), (n, k)
        torch.randn(1 << 16, device="cuda").sum().item()
    assert got[1].shape == (V, D)


def test_gradients_of_broadcast_inputs(swr):
    """Inputs that were expanded, and gradients that come expanded."""
    i = _inputs(F32, 20)
    row = i["dy"][:1, :1].clone().requires_grad_()
    x = row.expand(3, 20, 64)
    y = swr.SWRCausalConvFunction.apply(x, i["w"])
    y, _ = swr.SWRSelectiveScanFunction.apply(y, x, i["A"], i["B"], i["C"])
    got, = torch.autograd.grad(y.sum(), row)   # (the sum's gradient is one number, expanded)
    dense = x.detach().contiguous()
    c = swr.swr_causal_conv(dense, i["w"])[0]
    carriers = swr.swr_selective_scan(c, dense, i["A"], i["B"], i["C"], save_carriers=True)[1]
    dc, ddt, *_ = swr.swr_selective_scan_backward(c, dense, i["A"], i["B"], i["C"], torch.ones_like(c), carriers)
    dx = swr.swr_causal_conv_backward(dense, i["w"], dc)[0] + ddt
    assert torch.equal(got, dx.sum((0, 1), keepdim=True))
    logits = i["logits"][:1, :1].clone().requires_grad_()
    rows = logits.expand(3, 20, -1)
    logp, _, _ = swr.SWRLogProbsFunction.apply(rows, i["tokens"])
    d, = torch.autograd.grad(logp.sum(), logits)
    dense = rows.detach().contiguous()
    _, lse, ent = swr.swr_log_probs(dense, i["tokens"])
    assert torch.equal(d, swr.swr_log_probs_backward(dense, i["tokens"], lse, ent,
                                                     torch.ones_like(lse)).sum((0, 1), keepdim=True))
    table = i["table"].clone().requires_grad_()
    out = swr.SWREmbeddingFunction.apply(i["tokens"], table)
    d, = torch.autograd.grad(out.sum(), table)
    assert torch.equal(d, swr.swr_embedding_backward(i["tokens"], torch.ones_like(out), i["vocab"]))


def test_second_derivatives_are_refused(swr):
    i = _inputs(F32, 20)
    table = i["table"].clone().requires_grad_()
    y = swr.SWREmbeddingFunction.apply(i["tokens"], table)
    d, = torch.autograd.grad((y * y).sum(), table, create_graph=True)
    with pytest.raises(RuntimeError):
        d.sum().backward()


def test_far_offsets(swr):
    """Rows past 2^31 elements: of the table, of the gradient, of the logits."""
    V, width = 40, 1 << 26   # 2.7e9 elements of bfloat16, 5.4 GB
    table = torch.zeros(V, width, dtype=BF16, device="cuda")
    table[V - 1, -5:] = 3.0
    table[V - 2, :5] = 2.0
    y = swr.swr_embedding(torch.tensor([V - 1, V - 2, V], device="cuda"), table)
    assert (y[0, -5:] == 3).all() and (y[1, :5] == 2).all()
    assert float(y[0, :-5].float().abs().max()) == 0 and float(y[2].float().abs().max()) == 0
    dt = swr.swr_embedding_backward(torch.tensor([V - 1, V - 1, V - 2], device="cuda"), y, V, dtype=BF16)
    assert torch.equal(dt[V - 1], (y[0].float() + y[1].float()).to(BF16)) and torch.equal(dt[V - 2], y[2])
    assert float(dt[:V - 2].abs().max()) == 0
    del table, dt, y
    rows, vocab = 33, 1 << 26
    logits = torch.full((rows, vocab), -20.0, dtype=BF16, device="cuda")
    logits[-1, -1] = 20.0   # e^40 against 2^26 of e^0: log p = -2^26 e^-40, about -2.9e-10
    tokens = torch.full((rows,), vocab - 1, device="cuda")
    logp, lse, ent, top, best = swr.swr_log_probs(logits, tokens, 1)
    assert int(best[-1, 0]) == vocab - 1 and int(best[-2, 0]) == 0
    assert abs(float(lse[-1]) - 20) < 1e-5 and abs(float(logp[-1])) < 1e-5
    # A row of equal logits: -log 2^26; the sum in float32 of 2^26 ones in parts, each exact.
    assert abs(float(logp[0]) + 18.021826694558577) < 1e-5
    d = swr.swr_log_probs_backward(logits, tokens, lse, ent, torch.ones_like(logp))
    assert float(d[0, -1]) == 1.0 and abs(float(d[0, 5]) * 2 ** 26 + 1) < 2 ** -7
    assert abs(float(d[-1, -1])) < 1e-5 and abs(float(d[-1, 7])) < 1e-15


def test_far_tokens_of_the_convolution(swr):
    """Tokens past 2^31 elements of x, y and dx."""
    B, T, D = 1, 9000, 1 << 18   # 2.4e9 elements of bfloat16, 4.7 GB each
    x = torch.zeros(B, T, D, dtype=BF16, device="cuda")
    x[0, -3:, -1] = 1.0
    w = torch.zeros(D, 4, dtype=BF16, device="cuda")
    w[:, 2:] = torch.tensor([0.5, 1.0], dtype=BF16)
    y, _ = swr.swr_causal_conv(x, w, silu=False)
    assert y[0, -4:, -1].tolist() == [0, 1, 1.5, 1.5] and float(y[..., :-1].abs().max()) == 0
    dx, dw, _ = swr.swr_causal_conv_backward(x, w, x, silu=False)
    assert dx[0, -5:, -1].tolist() == [0, 0.5, 1.5, 1.5, 1.0] and dw[-1].tolist() == [0, 1, 2, 3]


@pytest.mark.parametrize("N", [2, 16])
def test_far_tokens_of_the_scan(swr, N):
    """Tokens past 2^31 elements of x, y, dx, and of the carriers of 16 states."""
    B, T, D = 1, 9000, 1 << 18
    x = torch.zeros(B, T, D, dtype=BF16, device="cuda")
    x[0, -3:, -1] = 1.0
    A = torch.zeros(D, N, device="cuda")
    ones = torch.ones(B, T, N, dtype=BF16, device="cuda")
    # Steps of x times x: the states of the last channel count the ones, y sums N of them.
    y, carriers, h = swr.swr_selective_scan(x, x, A, ones, ones, softplus=False, save_carriers=True, want_state=True)
    assert y[0, -4:, -1].tolist() == [0, N, 2 * N, 3 * N] and (h[0, -1] == 3).all()
    assert float(y[0, :-3].abs().max()) == 0 and float(h[0, :-1].abs().max()) == 0
    assert float(carriers.abs().max()) == 0
    del y
    dx, ddt, dA, dB, dC, *_ = swr.swr_selective_scan_backward(x, x, A, ones, ones, x, carriers, softplus=False)
    for d in (dx, ddt):
        assert d[0, -4:, -1].tolist() == [0, 3 * N, 2 * N, N] and float(d[0, :-3].abs().max()) == 0
    assert (dA[-1] == 4).all() and float(dA[:-1].abs().max()) == 0   # 2 h[1] + 1 h[2]
    assert dB[0, -4:, 0].tolist() == [0, 3, 2, 1] and dC[0, -4:, N - 1].tolist() == [0, 1, 2, 3]
