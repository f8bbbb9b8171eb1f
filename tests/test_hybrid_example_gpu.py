"""The hybrid model's decoding example against a plain 64-bit evaluation of the whole
sequence: recurrences by the oracle, attention dense and causal, 4-bit weights
unpacked, the norm's 8-bit rows rounded as the format says.

Bound.  The decoder rounds to bf16 five times a layer (sum, projection, mixer, mixed
projection, embedding or norm), each 2^-9 of a value at most in the mean square sense
(2^-8 / sqrt 3), and an 8-bit value next to a rounding boundary may fall on its
other side, an eighth of it at most; of a bf16 perturbation of 2^-8.8 against
steps of 2^-3, one value in 50 does, in the mean square 2^-3 / sqrt(50) = 0.018 a
layer.  Four layers add to sqrt(4 (5 2^-17.6 + 0.018^2)) = 0.037 of the logits' root
mean square, were none of it averaged in the products and the residual sums; the
test takes 0.05 over all logits of a token."""
import importlib.util
import os
import sys

import numpy as np
import pytest
import torch

import oracle
from tests.hybrid_ref import f64, norm, unpack

pytestmark = pytest.mark.gpu

PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "hybrid_decode.py")


def _example():
    spec = importlib.util.spec_from_file_location("hybrid_decode", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _eight(y):
    """y rounded to 8 bits with a scale a row."""
    s = y.abs().amax(-1, keepdim=True) / 448
    return f64((y / s).to(torch.float32).to(torch.float8_e4m3fn).float()) * s


def _plain(m, tokens):
    """Logits [batch, T, vocab] of tokens [batch, T]."""
    B, T = tokens.shape
    h, y = f64(m.embedding)[tokens], None
    for i, kind in enumerate(m.layers):
        u, h, _ = norm(h, y, m.norms[i], 1e-6)
        z = _eight(u) @ unpack(*m.into[i], m.width).t()
        if kind == "R":
            n = m.width
            x, b, c = (z[..., j * n:(j + 1) * n].reshape(B, T, m.heads, -1).numpy() for j in range(3))
            mixed = torch.from_numpy(oracle.forward(x, z[..., 3 * n:].numpy(), b, c, 16, sigmoid_decay=True,
                                                    sigmoid_pregate=True)).reshape(B, T, n)
        else:
            z = z.reshape(B, T, -1, m.dim).transpose(1, 2)
            q, k, v = z[:, :m.q_heads], z[:, m.q_heads:m.q_heads + m.kv_heads], z[:, m.q_heads + m.kv_heads:]
            k, v = (t.repeat_interleave(m.q_heads // m.kv_heads, 1) for t in (k, v))
            s = (q @ k.transpose(2, 3)) * m.dim ** -0.5
            s = s.masked_fill(torch.ones(T, T, dtype=torch.bool).triu(1), -np.inf)
            mixed = (s.softmax(-1) @ v).transpose(1, 2).reshape(B, T, -1)
        y = mixed @ unpack(*m.out[i], mixed.shape[-1]).t()
    u, _, _ = norm(h, y, m.norms[-1], 1e-6)
    return u @ unpack(*m.head, m.width).t()


@pytest.mark.parametrize("layers,batch,page_size", [("RAAR", 3, 8), ("R", 1, 16), ("AA", 5, 16), ("RARR", 2, 3)])
def test_decoding_matches_the_whole_sequence(layers, batch, page_size):
    T = 37   # past two blocks of the recurrence, and pages that end within one
    m = _example().HybridDecoder(layers, batch, width=128, heads=8, q_heads=4, kv_heads=2, dim=32, vocab=100,
                                 max_tokens=T, page_size=page_size, seed=len(layers) + batch)
    tokens = torch.randint(100, (batch, T), generator=torch.Generator().manual_seed(1))
    got = torch.stack([m.step(tokens[:, t].to("cuda:0")) for t in range(T)], 1)
    torch.cuda.synchronize()
    want = _plain(m, tokens)
    off = (f64(got) - want).square().mean(-1).sqrt() / want.square().mean(-1).sqrt()
    assert off.max() < 0.05, off
    assert m.lengths.tolist() == [T] * batch
    used = batch * -(-T // page_size)
    assert m.free_count.item() == m.free.numel() - used
    assert len(set(m.table[m.table >= 0].tolist())) == used


def test_runs_as_a_program(monkeypatch, capsys):
    monkeypatch.setattr(sys, "argv", ["hybrid_decode.py", "--layers", "RA", "--batch", "2", "--tokens", "20"])
    _example().main()
    assert "20 tokens each" in capsys.readouterr().out
