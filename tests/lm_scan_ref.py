"""Bounds of a float32 evaluation of the selective scan, element by element: an error is carried along the
recurrence as the state itself is, so that it fades where the state does (lm_ref has the definition).

In units of U (half a step of float32, with room for the second order), relative:
* a step: v = dt + bias has 1 of |v|; the softplus 3 |v| + 16 of the step (its exponential's argument, twice,
  and some sixteen operations), without it 1;
* a decay exp(s A): |s A| times the step's error and 3 (log2 e, two products), and 2 of its own.  Where a sequence
  is cut into runs, a run's decay is the exponential of a sum of steps: with at most `adds` additions
  that many more for |s A|;
* sums over all tokens are of a run's tokens in a row (at most T), then of the batches' runs (of 64 tokens and
  more) in a row, and some of lanes;
* products and additions 1 each, of the absolute sums."""
import torch

from lm_ref import U, Scan, f64, silu, silu_slope

SECOND = 1.02   # room for products of errors (which are below 1e-3 here)


class Bounded(Scan):
    """lm_ref.Scan's values with bounds: `bounds` of y, h (before every token and after the last), and gradients."""

    def __init__(self, *args, adds=0, **kw):
        super().__init__(*args, **kw)
        v = torch.where(self.live, self.v, 0.0).abs()
        self.step = torch.where(self.live, 3 * v + 16, 0.0) if self.use_softplus else torch.ones_like(v)
        self.size = self.s.abs()
        rate = self.size[..., None] * self.A.abs()
        self.decay = rate * (self.step[..., None] + 3 + adds) + 2        # relative, of a
        self.n = self.A.shape[1]
        if self.z is not None:
            self.gate = silu(self.z)
            self.gate_err = 2 * self.z.abs() + 9
        else:
            self.gate = torch.ones_like(self.s)
            self.gate_err = torch.zeros_like(self.s)

    def forward(self):
        super().forward()
        T = self.x.shape[1]
        err, errs = torch.zeros_like(self.h0), [torch.zeros_like(self.h0)]
        for t in range(T):
            err = (self.a[:, t] * (err + self.h_size[:, t] * self.decay[:, t])
                   + self.u[:, t].abs() * (self.step[:, t, :, None] + 2) + 2 * self.h_size[:, t + 1])
            errs.append(err)
        self.h_err = torch.stack(errs, 1)
        self.y0_err = ((self.C.abs() * self.h_err[:, 1:]).sum(-1) + (self.n + 4) * self.y0_size)
        own = torch.where(self.live, (self.y0_err + self.y0_size * self.gate_err) * self.gate.abs(), 0.0)
        self.bounds = {"y": own * U * SECOND, "h": self.h_err * U * SECOND}
        return self.y

    def backward(self, dy, dh_last=None):
        """{name: (gradient, bound)}; after forward()."""
        values = super().backward(dy, dh_last)
        dy = torch.where(self.live, f64(dy), 0.0)
        n, T, ch = self.x.shape
        # Factors of a gradient: the gated dy, and how the step goes with dt.
        w, w_err = (dy * self.gate).abs(), self.gate_err
        slope = 1 / (1 + torch.exp(-self.v)) if self.use_softplus else torch.ones_like(self.v)
        slope = torch.where(self.live, slope, 0.0)
        slope_err = self.step + 4
        C, B, A, x, skip, s = (t.abs() for t in (self.C, self.B, self.A, self.x, self.skip, self.s))
        g = torch.zeros_like(self.h0) if dh_last is None else f64(dh_last).abs()
        e = torch.zeros_like(g)
        zeros = torch.zeros_like
        dx, ddt, ddt_size = zeros(x), zeros(x), zeros(x)
        dA, dA_size, dB, dB_size, dC, dC_size = zeros(A), zeros(A), zeros(B), zeros(B), zeros(C), zeros(C)
        for t in reversed(range(T)):
            wt, we, st, se = w[:, t, :, None], w_err[:, t, :, None], s[:, t, :, None], self.step[:, t, :, None]
            g = g + C[:, t] * wt
            e = e + C[:, t] * wt * (we + 1) + g
            h, h_err = self.h_size[:, t + 1], self.h_err[:, t + 1]
            dC_size[:, t] = h * wt
            dC[:, t] = h_err * wt + h * wt * (we + 1)
            u = st * x[:, t, :, None]
            dB_size[:, t] = g * u
            dB[:, t] = e * u + g * u * (se + 2)
            along = (g * B[:, t]).sum(-1)
            along_err = (e * B[:, t]).sum(-1) + (self.n + 1) * along
            # (from the token before: its gradient and state, each with its own error)
            e = self.a[:, t] * (e + g * (self.decay[:, t] + 1))
            g = self.a[:, t] * g
            past = g * self.h_size[:, t]
            past_err = e * self.h_size[:, t] + g * self.h_err[:, t] + past
            dA_size += (past * st).sum(0)
            dA += (past_err * st + past * st * (se + 2)).sum(0)
            decay = (past * A).sum(-1)
            decay_err = (past_err * A).sum(-1) + (self.n + 2) * decay
            size = along * x[:, t] + decay
            ddt_size[:, t] = size * slope[:, t]
            ddt[:, t] = (along_err * x[:, t] + decay_err + 2 * size) * slope[:, t] + size * slope[:, t] * slope_err[:, t]
            dx[:, t] = (along_err * s[:, t] + along * s[:, t] * (self.step[:, t] + 1)
                        + skip * w[:, t] * (w_err[:, t] + 1) + 2 * (along * s[:, t] + skip * w[:, t]))
        live = torch.where(self.live, 1.0, 0.0)
        ddt, ddt_size = ddt * live, ddt_size * live
        group = lambda t: t.unflatten(2, (self.G, -1)).sum(3)   # noqa: E731
        per, tokens = ch // self.G, T + n * max(1, T // 64) + 16
        bound = {"dx": dx, "ddt": ddt, "dA": dA + tokens * dA_size, "dB": group(dB) + per * group(dB_size),
                 "dC": group(dC) + per * group(dC_size), "dh0": e,
                 "dD": (w * x * (w_err + 1)).sum((0, 1)) + tokens * (w * x).sum((0, 1)),
                 "dt_bias": ddt.sum((0, 1)) + tokens * ddt_size.sum((0, 1))}
        if self.z is not None:
            turn = silu_slope(self.z).abs()
            turn_err = (1.2 + self.z.abs()) * (2 * self.z.abs() + 10)
            bound["dz"] = dy.abs() * (self.y0_err * turn + self.y0_size * turn_err + 2 * self.y0_size * turn) * live
        return {k: (values[k][0], v * U * SECOND) for k, v in bound.items()}
