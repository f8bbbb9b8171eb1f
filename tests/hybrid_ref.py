"""Plain 64-bit forms of the hybrid model's operators, on the host, written from
their definitions (no code of the library), and the bounds that a float32
evaluation with one rounding to the output's type keeps.

A float32 sum of n terms in any order is off by at most n 2^-24 times the sum of
their absolute values; U stands for that unit with room for the second order."""
import numpy as np
import torch

U = 2.0 ** -24 * 1.01
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}   # one rounding, relative
TINY = 1e-30


def f64(t):
    return t.detach().to("cpu").to(torch.float64)


def close(got, want, bound, what):
    """|got - want| <= bound element by element (bound: tensor or number); NaN and
    infinities have to be where the definition has them."""
    got, want = f64(got), want.to(torch.float64)
    assert got.shape == want.shape, what
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got[odd]), torch.isnan(want[odd])), what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), what
    err = (got - want).abs()
    bound = torch.as_tensor(bound, dtype=torch.float64).expand(want.shape)
    bad = ~odd & ~(err <= bound)
    if bad.any():
        i = int((err - bound).masked_fill(~bad, -1).argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {want.numel()} values off; worst at {i}: "
                             f"{got.reshape(-1)[i]} for {want.reshape(-1)[i]}, bound {bound.reshape(-1)[i]}")


# ----------------------------------------------------------------------------- norm


def norm(x, r, w, eps):
    h = f64(x) + (f64(r) if r is not None else 0)
    rho = 1 / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    return h * rho * f64(w), h, rho


def norm_backward(h, w, dy, dh, eps):
    """dx, dw and the absolute sums that their errors go by."""
    h, w, dy = f64(h), f64(w), f64(dy)
    rho = 1 / torch.sqrt(h.square().mean(-1, keepdim=True) + eps)
    g = dy * w
    dx = rho * (g - h * (g * h).mean(-1, keepdim=True) * rho ** 2)
    size = rho * (g.abs() + h.abs() * (g * h).abs().mean(-1, keepdim=True) * rho ** 2)
    if dh is not None:
        dx, size = dx + f64(dh), size + f64(dh).abs()
    n = (dy * h * rho).reshape(-1, h.shape[-1])
    return dx, n.sum(0), size, n.abs().sum(0)


# ----------------------------------------------------------------------------- 4-bit weights

SIZES = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)


def unpack(codes, powers, K):
    codes, powers = codes.cpu(), powers.cpu()
    c = torch.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1).long()
    v = SIZES[c & 7] * torch.where(c > 7, -1.0, 1.0)
    p = torch.where(powers == 255, float("nan"), 2.0 ** (powers.to(torch.float64) - 127))
    return (v * p.repeat_interleave(32, 1))[:, :K]


def linear(x, codes, powers, scale):
    """y, and the absolute sums that its error goes by."""
    x = f64(x.float())
    w = unpack(codes, powers, x.shape[-1])
    y, size = x @ w.t(), x.abs() @ w.abs().t()
    if scale is not None:
        s = f64(scale)[..., None]
        y, size = y * s, size * s.abs()
    return y, size


# ----------------------------------------------------------------------------- paged cache


def tables(lengths, news, table, stack, count, page, tokens):
    """The definition, request by request: (table, slots, starts, lengths, count)."""
    table = [list(r) for r in table]
    count = min(max(count, 0), len(stack))
    slots, starts = [], [0]
    for i, (n, more) in enumerate(zip(lengths, news)):
        n, more = max(n, 0), max(more, 0)
        for at in range(n, n + more):
            column = at // page
            if column >= len(table[i]):
                slots.append(-1)
                continue
            if at % page == 0:
                count -= 1
                table[i][column] = stack[count] if count >= 0 else -1
            entry = table[i][column]
            slots.append(entry * page + at % page if entry >= 0 else -1)
        starts.append(starts[-1] + more)
    slots = (slots + [-1] * tokens)[:tokens]
    return table, slots, starts, [max(a, 0) + max(b, 0) for a, b in zip(lengths, news)], max(count, 0)


def attention(q, k_cache, v_cache, table, lengths, scale, window):
    """y, lse and the largest |v| and |scores| of each row."""
    q, k_cache, v_cache = f64(q), f64(k_cache), f64(v_cache)
    table, lengths = table.cpu().tolist(), lengths.cpu().tolist()
    B, Hq, D = q.shape
    pages, page, H, _ = k_cache.shape
    group = Hq // H
    y, lse = torch.zeros(B, Hq, D, dtype=torch.float64), torch.full((B, Hq), -np.inf, dtype=torch.float64)
    vmax, smax = torch.zeros(B, Hq, 1, dtype=torch.float64), torch.zeros(B, Hq, 1, dtype=torch.float64)
    for b in range(B):
        n = max(lengths[b], 0)
        at = [t for t in range(max(0, n - window) if window else 0, n)
              if t // page < len(table[b]) and 0 <= table[b][t // page] < pages]
        if not at:
            continue
        rows = torch.tensor([[table[b][t // page], t % page] for t in at])
        k, v = k_cache[rows[:, 0], rows[:, 1]], v_cache[rows[:, 0], rows[:, 1]]   # [n, H, D]
        for h in range(Hq):
            s = (k[:, h // group] @ q[b, h]) * scale
            top = s.max()
            p = torch.exp(s - top)
            y[b, h] = p @ v[:, h // group] / p.sum()
            lse[b, h] = top + torch.log(p.sum())
            vmax[b, h] = v[:, h // group].abs().max()
            smax[b, h] = (k[:, h // group].abs() @ q[b, h].abs()).max() * abs(scale)
    return y, lse, vmax, smax
