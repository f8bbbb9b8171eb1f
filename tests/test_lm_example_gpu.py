"""The operators together, as the selective language model's example uses them: log
probabilities and every parameter's gradient against a plain 64-bit evaluation with torch's own
differentiation on the host, single tokens against whole prompts, and the program itself.

Bounds, of float32.  Between two products a value is rounded at most 30 times a layer (norm,
convolution, gates, a scan over up to 40 tokens), and a product of up to 96 terms is off by 96 2^-24 of
its absolute sum, some 8 times the result's root mean square: a layer adds at most 2^-24 (30 + 4 96 8),
2e-4, of a tensor's root mean square, were none of it averaged.  The backward passes as
many again: two layers, there and back, 8e-4, which the norms and the softmax pass on without
enlarging it on the whole.  The tests take 1e-3 of a gradient's root mean square."""
import importlib.util
import os
import sys

import pytest
import torch

import lm_ref as ref
from lm_ref import f64

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "selective_lm.py")
SIZES = dict(width=64, inner=96, states=16, groups=2, rank=8, taps=4, vocab=75)
CLOSE = 1e-3


@pytest.fixture()
def example():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    spec = importlib.util.spec_from_file_location("selective_lm", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _norm(x, w):
    return x * torch.rsqrt((x * x).mean(-1, keepdim=True) + 1e-6) * w


def plain(m, leaves, tokens, lengths):
    """Outputs before the logits, and the logits, of 64-bit copies of the model's parameters."""
    table, norms = leaves[0], leaves[1:2 + len(m.layers)]
    rest = iter(leaves[2 + len(m.layers):])
    B, T = tokens.shape
    live = torch.arange(T)[None] < lengths[:, None]
    h = torch.where(((tokens >= 0) & (tokens < len(table)))[..., None], table[tokens.clamp(0, len(table) - 1)], 0.0)
    y = 0.0
    for norm, names in zip(norms, m.layers):
        p = {k: next(rest) for k in names}
        h = h + y
        x, z = (_norm(h, norm) @ p["into"].t()).split(m.inner, -1)
        padded = torch.cat([torch.zeros(B, p["conv"].shape[1] - 1, m.inner, dtype=x.dtype), x], 1)
        pre = p["conv_bias"] + sum(p["conv"][:, k] * padded[:, k:k + T] for k in range(p["conv"].shape[1]))
        x = torch.where(live[..., None], ref.silu(pre), 0.0)
        dt, shared = torch.split(x @ p["mix"].t(), [m.rank, 2 * m.groups * m.states], -1)
        b, c = (t.repeat_interleave(m.inner // m.groups, 2) for t in
                shared.unflatten(-1, (2, m.groups, m.states)).unbind(-3))
        s = ref.softplus(dt @ p["dt"].t() + p["dt_bias"])
        state, out = torch.zeros(B, m.inner, m.states, dtype=x.dtype), []
        for t in range(T):
            state = torch.exp(s[:, t, :, None] * -torch.exp(p["rates"])) * state + (s * x)[:, t, :, None] * b[:, t]
            out.append((c[:, t] * state).sum(-1) + p["skip"] * x[:, t])
        x = torch.where(live[..., None], torch.stack(out, 1) * ref.silu(z), 0.0)
        y = x @ p["out"].t()
    u = _norm(h + y, norms[-1])
    return u, u @ table.t()


def _off(got, want):
    """The difference's root mean square relative to the wanted one's."""
    got, want = f64(got), f64(want)
    return float((got - want).square().mean().sqrt() / want.square().mean().sqrt())


@pytest.mark.parametrize("T,lengths", [(1, [1, 1]), (17, [17, 5]), (40, [40, 33])])
def test_training_matches_64_bits(example, T, lengths):
    m = example.SelectiveLM(2, dtype=torch.float32, **SIZES)
    g = torch.Generator().manual_seed(T)
    tokens, targets = (torch.randint(SIZES["vocab"], (2, T), generator=g) for _ in range(2))
    n = torch.tensor(lengths)
    live = torch.arange(T)[None] < n[:, None]
    tokens, targets = torch.where(live, tokens, -1), torch.where(live, targets, -1)   # padding

    logp = m.log_probs(tokens.cuda(), targets.cuda(), n.int().cuda())
    got = torch.autograd.grad(-logp.sum(), m.parameters())
    leaves = [f64(p.detach()).requires_grad_() for p in m.parameters()]
    _, logits = plain(m, leaves, tokens, n)
    want = torch.where(live, torch.gather(torch.log_softmax(logits, -1), -1, targets.clamp(min=0)[..., None])[..., 0], 0.0)
    grads = torch.autograd.grad(-want.sum(), leaves)
    assert _off(logp.detach(), want.detach()) < CLOSE
    assert (logp.detach().cpu()[~live] == 0).all()
    for i, (a, b) in enumerate(zip(got, grads)):
        if b.square().sum() == 0:
            assert (a == 0).all(), i
        else:
            assert _off(a, b) < CLOSE, i


def test_single_tokens_carry_prompts_on(example):
    m = example.SelectiveLM(2, dtype=torch.float32, **SIZES)
    B, T, lengths = 3, 30, torch.tensor([20, 1, 7])
    tokens = torch.randint(SIZES["vocab"], (B, T), generator=torch.Generator().manual_seed(2))
    whole, _ = m.prompt(tokens.cuda())
    want, logits = plain(m, [f64(p.detach()) for p in m.parameters()], tokens, torch.full((B,), T))
    assert _off(whole, want) < CLOSE
    u, states = m.prompt(tokens.cuda(), lengths.int().cuda())
    rows = torch.arange(B)
    assert _off(u[rows, lengths - 1], want[rows, lengths - 1]) < CLOSE
    for i in range(T - int(lengths.max())):
        at = lengths + i
        u = m.step(tokens[rows, at].cuda(), states)
        assert _off(u, want[rows, at]) < CLOSE, i
    chosen, logp = m.best(u, top=3)
    logs = torch.log_softmax(logits[rows, at], -1)
    # (the largest log probability is 4.3 = log 75 at least below nothing: 1e-3 of the logits' size, which is about 1)
    assert (f64(logp) - logs.topk(3).values).abs().max() < 4 * CLOSE
    assert (torch.gather(logs, 1, chosen.cpu()) - logs.topk(3).values).abs().max() < 4 * CLOSE


def test_steps_in_a_captured_graph(example):
    """Generation captured once: every replay, with other work between, is the eager step."""
    m = example.SelectiveLM(2, **SIZES)
    tokens = torch.randint(SIZES["vocab"], (4, 9), generator=torch.Generator().manual_seed(3)).cuda()
    u, states = m.prompt(tokens)
    first, _ = m.best(u[:, -1])
    eager, token = [], first[:, 0].contiguous()
    moved = [tuple(t.clone() for t in s) for s in states]
    for _ in range(6):
        token = m.best(m.step(token, moved))[0][:, 0].contiguous()
        eager.append(token)
    kept, at = [tuple(t.clone() for t in s) for s in states], first[:, 0].contiguous()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):   # (loads kernels and libraries)
        m.best(m.step(at, [tuple(t.clone() for t in s) for s in states]))
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        at.copy_(m.best(m.step(at, kept))[0][:, 0])
    for i in range(6):
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(at, eager[i]), i
        m.prompt(tokens)
    for a, b in zip(kept, moved):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_runs_as_a_program(example, monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["selective_lm.py", "--layers", "2", "--batch", "2", "--tokens", "100", "--steps", "2",
                                      "--generate", "5"])
    example.main()
    out = capsys.readouterr().out
    assert "2 steps" in out and "5 tokens each" in out
