"""Plain 64-bit forms of a recurrent language model's operators, on the host,
written from their definitions (no code of the library), and the absolute sums that
their float32 evaluations' errors go by (hybrid_ref has the comparison)."""
import numpy as np
import torch

from hybrid_ref import ROUND, TINY, U, close, f64  # noqa: F401  (the tests' too)


def rand(seed, shape, dtype, by=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g, dtype=torch.float64) * by).to(dtype)


# ----------------------------------------------------------------------------- embedding


def embedding(tokens, table, scale):
    tokens, table = tokens.cpu().long(), f64(table)
    fine = (tokens >= 0) & (tokens < table.shape[0])
    return torch.where(fine[..., None], table[torch.where(fine, tokens, 0)] * scale, 0.0)


def embedding_backward(tokens, dy, vocab, scale):
    """The gradient, its absolute sums, and the most rows of one token."""
    tokens, dy = tokens.cpu().long().reshape(-1), f64(dy).reshape(-1, dy.shape[-1])
    d, size = (torch.zeros(vocab, dy.shape[-1], dtype=torch.float64) for _ in range(2))
    most = 0
    for v in tokens[(tokens >= 0) & (tokens < vocab)].unique().tolist():
        rows = dy[tokens == v]
        d[v], size[v] = rows.sum(0) * scale, rows.abs().sum(0) * abs(scale)
        most = max(most, rows.shape[0])
    return d, size, most


# ----------------------------------------------------------------------------- convolution


def silu(v):
    return v / (1 + torch.exp(-v))


def silu_slope(v):
    gate = 1 / (1 + torch.exp(-v))
    return gate * (1 + v * (1 - gate))


def _live(T, lengths, B):
    n = torch.full((B,), T) if lengths is None else lengths.cpu().long().clamp(0, T)
    return torch.arange(T)[None] < n[:, None], n


def conv(x, w, bias, with_silu, state, lengths):
    """y, the sums before the SiLU, their absolute sums, and the last taps - 1 tokens."""
    x, w = f64(x), f64(w)
    B, T, C = x.shape
    K = w.shape[1]
    live, n = _live(T, lengths, B)
    past = torch.zeros(B, K - 1, C, dtype=torch.float64) if state is None else f64(state)
    rows = torch.cat([past, torch.where(live[..., None], x, 0.0)], 1)
    b = torch.zeros(C, dtype=torch.float64) if bias is None else f64(bias)
    pre = b.expand(B, T, C) + sum(w[:, k] * rows[:, k:k + T] for k in range(K))
    size = b.abs().expand(B, T, C) + sum((w[:, k] * rows[:, k:k + T]).abs() for k in range(K))
    y = torch.where(live[..., None], silu(pre) if with_silu else pre, 0.0)
    last = torch.stack([rows[i, n[i]:n[i] + K - 1] for i in range(B)]) if B else past
    return y, pre, size, last


def conv_backward(x, w, bias, with_silu, lengths, dy):
    """dx, dw, dbias and their absolute sums; `wobble` is how far a gate's error takes g."""
    y, pre, size, _ = conv(x, w, bias, with_silu, None, lengths)
    x, w, dy = f64(x), f64(w), f64(dy)
    B, T, C = x.shape
    K = w.shape[1]
    live, _ = _live(T, lengths, B)
    x, dy = torch.where(live[..., None], x, 0.0), torch.where(live[..., None], dy, 0.0)
    g = dy * (silu_slope(pre) if with_silu else 1.0)
    # |g|, with what an error of pre (size, relative U) and of the gate does to it
    err = dy.abs() * ((1.2 + pre.abs()) * 8 + size) if with_silu else dy.abs()
    out = []
    for t, xs in ((g, x), (err, x.abs())):
        dx, dw = torch.zeros_like(x), torch.zeros_like(w)
        for k in range(K):
            lag = K - 1 - k
            ws = w[:, k] if xs is x else w[:, k].abs()
            if lag < T:
                dx[:, :T - lag] += ws * t[:, lag:]
                dw[:, k] = (t[:, lag:] * xs[:, :T - lag]).sum((0, 1))
        out += [torch.where(live[..., None], dx, 0.0), dw, t.sum((0, 1))]
    return out


# ----------------------------------------------------------------------------- scan


def softplus(v):
    return torch.logaddexp(v, torch.zeros((), dtype=v.dtype))


class Scan:
    """The scan's definition token by token, its gradients, and their absolute sums."""

    def __init__(self, x, dt, A, B, C, D=None, z=None, dt_bias=None, use_softplus=True, h0=None, lengths=None):
        self.x, self.A = f64(x), f64(A)
        n, T, ch = self.x.shape
        self.G = B.shape[2] if B.dim() == 4 else 1
        self.B, self.C = (f64(t).reshape(n, T, self.G, -1).repeat_interleave(ch // self.G, 2) for t in (B, C))
        zeros = torch.zeros(ch, dtype=torch.float64)
        self.skip = zeros if D is None else f64(D)
        self.z = None if z is None else f64(z)
        self.v = f64(dt) + (zeros if dt_bias is None else f64(dt_bias))
        self.use_softplus = use_softplus
        live, _ = _live(T, lengths, n)
        self.live = live[..., None]
        self.s = torch.where(self.live, softplus(self.v) if use_softplus else self.v, 0.0)
        self.x = torch.where(self.live, self.x, 0.0)
        # Past the lengths nothing counts, whatever is there.
        self.B, self.C = (torch.where(self.live[..., None], t, 0.0) for t in (self.B, self.C))
        if z is not None:
            self.z = torch.where(self.live, self.z, 0.0)
        self.a = torch.exp(self.s[..., None] * self.A)
        self.u = (self.s * self.x)[..., None] * self.B
        self.h0 = torch.zeros(n, ch, self.A.shape[1], dtype=torch.float64) if h0 is None else f64(h0)
        # How many roundings of a value lie on its way: a step's own (its sum, exponential and
        # logarithm), a decay's, for every token, and the runs' sums of steps.
        rate = (self.s[..., None] * self.A).abs()
        far = float(rate.max()) if rate.numel() else 0.0
        big = float(torch.where(self.live, self.v, 0.0).abs().max()) if self.v.numel() else 0.0
        step = 3 * big + 16
        self.terms = T * (far * (step + 3 + T) + 4) + step + self.A.shape[1] + 16

    def forward(self):
        h, hs, size, sizes = self.h0, [self.h0], self.h0.abs(), [self.h0.abs()]
        for t in range(self.x.shape[1]):
            h = self.a[:, t] * h + self.u[:, t]
            size = self.a[:, t] * size + self.u[:, t].abs()
            hs.append(h)
            sizes.append(size)
        self.h, self.h_size = torch.stack(hs, 1), torch.stack(sizes, 1)
        self.y0 = (self.C * self.h[:, 1:]).sum(-1) + self.skip * self.x
        size = (self.C.abs() * self.h_size[:, 1:]).sum(-1) + (self.skip * self.x).abs()
        self.y0_size = size
        gate = 1.0 if self.z is None else silu(self.z)
        more = 0.0 if self.z is None else 2 * self.z.abs() + 8
        self.y = torch.where(self.live, self.y0 * gate, 0.0)
        self.y_bound = torch.where(self.live, size * abs(gate) * U * (self.terms + more), 0.0)
        return self.y

    def backward(self, dy, dh_last=None):
        """{name: (gradient, absolute sum)}; after forward()."""
        dy = torch.where(self.live, f64(dy), 0.0)
        n, T, ch = self.x.shape
        gate = 1.0 if self.z is None else silu(self.z)
        slope = 1 / (1 + torch.exp(-self.v)) if self.use_softplus else torch.ones_like(self.v)
        out = {}
        for absolute in (False, True):
            mod = torch.abs if absolute else (lambda t: t)
            w = mod(dy * gate)
            g = torch.zeros_like(self.h0) if dh_last is None else mod(f64(dh_last))
            h = self.h_size if absolute else self.h
            C, B, A, x, skip, s = (mod(t) for t in (self.C, self.B, self.A, self.x, self.skip, self.s))
            dx, ddt = torch.zeros_like(self.x), torch.zeros_like(self.x)
            dA, dB, dC = torch.zeros_like(self.A), torch.zeros_like(self.B), torch.zeros_like(self.C)
            for t in reversed(range(T)):
                g = g + C[:, t] * w[:, t, :, None]
                dC[:, t] = h[:, t + 1] * w[:, t, :, None]
                dB[:, t] = g * (s[:, t] * x[:, t])[..., None]
                along = (g * B[:, t]).sum(-1)
                g = g * self.a[:, t]
                past = g * h[:, t]
                dA += (past * s[:, t, :, None]).sum(0)
                ddt[:, t] = (along * x[:, t] + (past * A).sum(-1)) * slope[:, t]
                dx[:, t] = along * s[:, t] + skip * w[:, t]
            dB, dC = (t.unflatten(2, (self.G, -1)).sum(3) for t in (dB, dC))
            res = {"dx": dx, "ddt": torch.where(self.live, ddt, 0.0), "dA": dA, "dB": dB, "dC": dC,
                   "dD": (w * x).sum((0, 1)), "dh0": g}
            res["dt_bias"] = res["ddt"].sum((0, 1))
            if self.z is not None:
                turn = (1.2 + self.z.abs()) if absolute else silu_slope(self.z)
                res["dz"] = mod(dy) * (self.y0_size if absolute else self.y0) * turn
            for k, v in res.items():
                out[k] = (out[k][0], v) if absolute else (v, None)
        return out


# ----------------------------------------------------------------------------- log probabilities


def log_probs(logits, tokens, scale):
    """logp, lse, entropy (defined as the header has them), and each row's largest |z|."""
    z, tokens = f64(logits) * scale, tokens.cpu().long()
    V = z.shape[-1]
    top = z.max(-1).values
    empty = top == -np.inf
    bad = torch.isnan(z).any(-1) | (z == np.inf).any(-1)
    # (From the largest: even in 64 bits a sum with a type's lowest value loses the logarithm.)
    far = z - torch.where(empty, 0.0, top)[..., None]
    total = torch.log(torch.exp(far).sum(-1))
    lse = torch.where(bad, np.nan, torch.where(empty, -np.inf, top + total))
    logs = torch.where(empty[..., None], -np.inf, torch.where(bad[..., None], np.nan, far - total[..., None]))
    p = torch.exp(logs)
    entropy = -torch.where(p == 0, 0.0, p * logs).sum(-1)
    entropy = torch.where(empty, 0.0, torch.where(bad, np.nan, entropy))
    fine = (tokens >= 0) & (tokens < V)
    logp = torch.gather(logs, -1, torch.where(fine, tokens, 0)[..., None])[..., 0]
    return torch.where(fine, logp, 0.0), lse, entropy, logs


def top_tokens(logits, top):
    """Indices of the largest, the first of equal ones first, NaN before all."""
    z = f64(logits)
    z = torch.where(torch.isnan(z), np.inf, z) + 0.0
    odd = torch.isnan(f64(logits))
    order = [sorted(range(r.numel()), key=lambda i: (not bool(o[i]), -float(r[i]), i))[:top]
             for r, o in zip(z.reshape(-1, z.shape[-1]), odd.reshape(-1, z.shape[-1]))]
    return torch.tensor(order, dtype=torch.int64).reshape(*z.shape[:-1], top)


def log_probs_backward(logits, tokens, scale, dlogp, dlse, dentropy):
    """The logits' gradient and its absolute sums."""
    _, _, entropy, logs = log_probs(logits, tokens, scale)
    tokens = tokens.cpu().long()
    V = logs.shape[-1]
    zero = torch.zeros_like(entropy)
    dlogp, dlse, dentropy = (zero if t is None else f64(t) for t in (dlogp, dlse, dentropy))
    fine = (tokens >= 0) & (tokens < V)
    dlogp = torch.where(fine, dlogp, 0.0)
    p = torch.exp(logs)
    hit = torch.zeros_like(p)
    hit.scatter_(-1, torch.where(fine, tokens, 0)[..., None], 1.0)
    turn = torch.where(p == 0, 0.0, logs + entropy[..., None])
    d = dlogp[..., None] * (hit - p) + dlse[..., None] * p - dentropy[..., None] * p * turn
    size = (dlogp.abs()[..., None] * (hit + p) + dlse.abs()[..., None] * p
            + dentropy.abs()[..., None] * p * (turn.abs() + 2 * entropy.abs()[..., None] + 1))
    return scale * d, scale * size
