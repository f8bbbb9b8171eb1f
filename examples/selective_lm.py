"""A language model of selective state space layers: training, prompts, single tokens.

Tokens become rows of the table (``swr_embedding``).  A layer norms the sum of the residual
stream and the last layer's output (``swr_rms_norm``), projects it to the mixer's inputs and
gates, convolves the inputs over a few tokens (``swr_causal_conv``), derives steps, B and C
of the scan from them (``swr_selective_scan``), and projects the gated result back.  The
logits are products with the table once more, and what is learned from are the log
probabilities of the next tokens (``swr_log_probs``), whose alternatives also choose
the next token when it generates.

A prompt of each request leaves two states a layer, the convolution's last inputs and the
scan's states, which single tokens then carry on in place (``swr_causal_conv_step``,
``swr_selective_step``).

The weights start random and the text is a made-up one: what it shows is how the calls fit
together, and what they take.  Run it on a GPU:

    python examples/selective_lm.py [--layers 4] [--batch 8] [--tokens 2048] [--steps 10] [--generate 100]
"""
import argparse
import os
import sys
import time

sys.path.insert(0, os.path.join(os.path.dirname(os.path.abspath(__file__)), ".."))
import torch  # noqa: E402

import paper_2512_13921_amd as swr  # noqa: E402


class SelectiveLM:
    """``width`` channels of the residual stream, ``inner`` of the mixer with ``states`` each; B
    and C are shared by ``groups`` of them, steps come through a bottleneck of ``rank``."""

    def __init__(self, layers, width, inner, states, groups, rank, taps, vocab, dtype=torch.bfloat16, seed=0,
                 device="cuda:0"):
        self.inner, self.states, self.groups, self.rank = inner, states, groups, rank
        rng = torch.Generator().manual_seed(seed)

        def normal(*shape, by=None):
            return torch.randn(shape, generator=rng) * (shape[-1] ** -0.5 if by is None else by)

        def leaf(t, kind=dtype):
            return t.to(device, kind).requires_grad_()

        self.table = leaf(normal(vocab, width))
        self.norms = [leaf(torch.ones(width)) for _ in range(layers + 1)]
        f32 = torch.float32
        self.layers = [dict(into=leaf(normal(2 * inner, width)), conv=leaf(normal(inner, taps)),
                            conv_bias=leaf(normal(inner, by=0.1)), mix=leaf(normal(rank + 2 * groups * states, inner)),
                            dt=leaf(normal(inner, rank)), dt_bias=leaf(normal(inner, by=0.5) - 3.0, f32),
                            rates=leaf(torch.log(torch.arange(1.0, states + 1)).repeat(inner, 1), f32),
                            skip=leaf(torch.ones(inner), f32), out=leaf(normal(width, inner)))
                       for _ in range(layers)]

    def parameters(self):
        return [self.table, *self.norms, *(t for layer in self.layers for t in layer.values())]

    def mixed(self, layer, x):
        """What the scan takes of the convolved inputs: steps, rates, B and C."""
        dt, shared = torch.split(x @ layer["mix"].t(), [self.rank, 2 * self.groups * self.states], -1)
        B, C = shared.unflatten(-1, (2, self.groups, self.states)).unbind(-3)
        return dt @ layer["dt"].t(), -torch.exp(layer["rates"]), B, C

    def log_probs(self, tokens, targets, lengths=None):
        """Log probabilities of targets [B, T] after tokens [B, T], with gradients."""
        h, y = swr.SWREmbeddingFunction.apply(tokens, self.table), None
        for norm, layer in zip(self.norms, self.layers):
            u, h = swr.SWRNormFunction.apply(h, norm, y)
            x, z = (u @ layer["into"].t()).split(self.inner, -1)
            x = swr.SWRCausalConvFunction.apply(x, layer["conv"], layer["conv_bias"], True, lengths)
            dt, A, B, C = self.mixed(layer, x)
            x, _ = swr.SWRSelectiveScanFunction.apply(x, dt, A, B, C, layer["skip"], z, layer["dt_bias"], True, None,
                                                      lengths)
            y = x @ layer["out"].t()
        u, _ = swr.SWRNormFunction.apply(h, self.norms[-1], y)
        return swr.SWRLogProbsFunction.apply(u @ self.table.t(), targets)[0]

    @torch.no_grad()
    def prompt(self, tokens, lengths=None):
        """Outputs [B, T, width] of prompts [B, T] (of lengths [B]), and the states after them."""
        h, y, states = swr.swr_embedding(tokens, self.table), None, []
        for norm, layer in zip(self.norms, self.layers):
            if y is None:
                u = swr.swr_rms_norm(h, norm)
            else:
                u, h = swr.swr_rms_norm(h, norm, y)
            x, z = (u @ layer["into"].t()).split(self.inner, -1)
            x, past = swr.swr_causal_conv(x, layer["conv"], layer["conv_bias"], lengths=lengths, want_state=True)
            dt, A, B, C = self.mixed(layer, x)
            x, _, state = swr.swr_selective_scan(x, dt, A, B, C, layer["skip"], z, layer["dt_bias"], lengths=lengths,
                                                 want_state=True)
            states.append((past, state))
            y = x @ layer["out"].t()
        return swr.swr_rms_norm(h, self.norms[-1], y)[0], states

    @torch.no_grad()
    def step(self, tokens, states):
        """Outputs [B, width] after one more token of each request; the states move on."""
        h, y = swr.swr_embedding(tokens, self.table), None
        for norm, layer, (past, state) in zip(self.norms, self.layers, states):
            if y is None:
                u = swr.swr_rms_norm(h, norm)
            else:
                u, h = swr.swr_rms_norm(h, norm, y)
            x, z = (u @ layer["into"].t()).split(self.inner, -1)
            x = swr.swr_causal_conv_step(x, layer["conv"], past, layer["conv_bias"])
            dt, A, B, C = self.mixed(layer, x)
            x = swr.swr_selective_step(x, dt, A, B, C, state, layer["skip"], z, layer["dt_bias"])
            y = x @ layer["out"].t()
        return swr.swr_rms_norm(h, self.norms[-1], y)[0]

    @torch.no_grad()
    def best(self, u, top=1):
        """The most probable next tokens after outputs [B, width], and their log probabilities."""
        logits = u @ self.table.t()
        nothing = torch.full(u.shape[:-1], -1, dtype=torch.int64, device=u.device)
        _, _, _, logp, tokens = swr.swr_log_probs(logits, nothing, top=top)
        return tokens, logp


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--layers", type=int, default=4)
    ap.add_argument("--batch", type=int, default=8)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--steps", type=int, default=10)
    ap.add_argument("--generate", type=int, default=100)
    args = ap.parse_args()
    if min(args.layers, args.batch, args.tokens, args.steps, args.generate) < 1:
        ap.error("layers, batch, tokens, steps and generate must be positive")
    vocab = 8192
    model = SelectiveLM(args.layers, width=1024, inner=2048, states=16, groups=1, rank=64, taps=4, vocab=vocab)
    optimizer = torch.optim.AdamW(model.parameters(), lr=1e-3)
    # A text that repeats itself, each request from another place.
    text = torch.randint(vocab, (997,), generator=torch.Generator().manual_seed(1)).cuda()
    at = torch.arange(args.tokens + 1, device="cuda") + 100 * torch.arange(args.batch, device="cuda")[:, None]
    rows = text[at % len(text)]
    tokens, targets = rows[:, :-1].contiguous(), rows[:, 1:].contiguous()

    def train():
        optimizer.zero_grad()
        loss = -model.log_probs(tokens, targets).mean()
        loss.backward()
        optimizer.step()
        return loss

    first = train()   # (first calls load the kernels)
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(args.steps):
        loss = train()
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"training: {args.layers} layers, {args.batch} x {args.tokens} tokens, {args.steps} steps: "
          f"{1e3 * took / args.steps:.1f} ms a step, loss {first.item():.3f} to {loss.item():.3f}")

    u, states = model.prompt(tokens)
    token, _ = model.best(u[:, -1])
    token, _ = model.best(model.step(token[:, 0].contiguous(), states))
    torch.cuda.synchronize()
    start = time.perf_counter()
    for _ in range(args.generate):
        token, _ = model.best(model.step(token[:, 0].contiguous(), states))
    torch.cuda.synchronize()
    took = time.perf_counter() - start
    print(f"generation: {args.batch} requests, {args.generate} tokens each: {1e6 * took / args.generate:.0f} us a step")


if __name__ == "__main__":
    main()
