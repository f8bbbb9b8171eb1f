"""Performance cases of the operators that a recurrent language model is made of
around its norms and projections, from its tokens to what it learns from: the
embedding of tokens, the short causal convolution and the selective state space
scan of its mixer, and the log probabilities of given tokens.

Each case is one call, or the forward and the backward of a training step:

* ``lookup``, ``lookup_grad``: scaled rows of an embedding table, and the table's
  gradient;
* ``conv``, ``conv_step``: the mixer's depthwise causal convolution with its SiLU,
  in training (forward and backward) and for one new token a request;
* ``scan``, ``scan_train``, ``scan_step``: the selective scan over prompts, in
  training, and for one new token a request;
* ``score``, ``score_train``: log probabilities of given tokens with their rows'
  entropy, with the top alternatives, or with the logits' gradient.

``run`` computes them by elementary torch operations in 32 bits, rounded once at
the end, or (``own``) by the library's calls; ``exact`` in 64 bits.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
_BYTES = {"bf16": 2, "f32": 4}


def listed():
    return [
        # A decoding step's embedding for a batch of 8 at width 2048: latency.
        {"name": "lookup_decode", "kind": "lookup", "rows": 8, "vocab": 65536, "width": 2048, "dtype": "bf16"},
        # A training batch's embedding gradient, at an odd length: tokens as
        # frequent as words are, most of the vocabulary absent.
        {"name": "lookup_grad", "kind": "lookup_grad", "rows": 5 * 4099, "vocab": 65536, "width": 2048,
         "dtype": "bf16", "out": "bf16"},
        # A small model's debugging run in float32, everything odd.
        {"name": "lookup_grad_odd_f32", "kind": "lookup_grad", "rows": 1001, "vocab": 5003, "width": 1001,
         "dtype": "f32", "out": "f32"},
        # The mixer's convolution in a training step, 4096 channels (twice the
        # width), odd length.
        {"name": "conv_train", "kind": "conv", "batch": 5, "length": 4099, "channels": 4096, "taps": 4,
         "dtype": "bf16"},
        # The same for one new token of 64 requests.
        {"name": "conv_step", "kind": "conv_step", "batch": 64, "channels": 4096, "taps": 4, "dtype": "bf16"},
        # One long prompt: one sequence alone has to fill the GPU.
        {"name": "scan_prompt", "kind": "scan", "batch": 1, "length": 16387, "channels": 4096, "states": 16,
         "groups": 1, "dtype": "bf16", "ragged": False},
        # A batch of prompts of different lengths, padded to the longest.
        {"name": "scan_prompts_ragged", "kind": "scan", "batch": 8, "length": 1500, "channels": 4096, "states": 16,
         "groups": 1, "dtype": "bf16", "ragged": True},
        # A training step's scan, forward and backward.
        {"name": "scan_train", "kind": "scan_train", "batch": 2, "length": 2048, "channels": 4096, "states": 16,
         "groups": 1, "dtype": "bf16"},
        # One new token of 128 requests: the states are read and written once.
        {"name": "scan_step", "kind": "scan_step", "batch": 128, "channels": 4096, "states": 16, "groups": 1,
         "dtype": "bf16"},
        # A decoding step's log probabilities with the 20 best alternatives.
        {"name": "score_decode", "kind": "score", "rows": 8, "vocab": 65536, "top": 20, "dtype": "bf16"},
        # Scoring a text without alternatives, float32 logits of an odd vocabulary.
        {"name": "score_text_f32", "kind": "score", "rows": 1027, "vocab": 50001, "top": 0, "dtype": "f32"},
        # A training step's loss: log probabilities, entropy and the logits' gradient.
        {"name": "score_train", "kind": "score_train", "rows": 5 * 819, "vocab": 65536, "dtype": "bf16"},
    ]


def _spread(rng, low, high):
    """A whole number between low and high, even over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("lookup", "lookup_grad", "lookup_grad", "conv", "conv", "conv_step", "scan", "scan", "scan",
                       "scan_train", "scan_train", "scan_step", "score", "score", "score_train", "score_train"))
    dtype = "f32" if rng.random() < 0.25 else "bf16"
    if kind in ("lookup", "lookup_grad"):
        vocab, width = _spread(rng, 64, 131072), _spread(rng, 32, 8192)
        if rng.random() < 0.6:
            width = max(32, width // 64 * 64)
        vocab = min(vocab, 2 ** 27 // width)
        rows = _spread(rng, 1, min(65536, 2 ** 25 // width))
        case = {"kind": kind, "rows": rows, "vocab": vocab, "width": width, "dtype": dtype}
        return case if kind == "lookup" else {**case, "out": rng.choice(("f32", dtype))}
    if kind in ("conv", "conv_step"):
        channels = _spread(rng, 48, 8192)
        if rng.random() < 0.6:
            channels = max(64, channels // 64 * 64)
        case = {"kind": kind, "batch": _spread(rng, 1, 256 if kind == "conv_step" else 16), "channels": channels,
                "taps": rng.choice((2, 3, 4, 4, 4, 4, 5, 8)), "dtype": dtype}
        if kind == "conv":
            case["length"] = _spread(rng, 1, min(32768, 2 ** 26 // (channels * case["batch"])))
        return case
    if kind in ("scan", "scan_train", "scan_step"):
        states, groups = rng.choice((4, 8, 16, 16, 16, 16, 24, 32, 64)), rng.choice((1, 1, 1, 2, 4))
        channels = _spread(rng, 32, 8192)
        channels = max(groups, channels // groups * groups)
        if rng.random() < 0.6:
            channels = max(64, channels // 64 * 64)
        case = {"kind": kind, "batch": _spread(rng, 1, 256 if kind == "scan_step" else 16), "channels": channels,
                "states": states, "groups": groups, "dtype": dtype}
        if kind != "scan_step":
            most = (2 ** 30 if kind == "scan" else 2 ** 28) // (channels * states * case["batch"])
            case["length"] = _spread(rng, 1, max(2, min(16384, most)))
        if kind == "scan":
            case["ragged"] = rng.random() < 0.5
        return case
    vocab = _spread(rng, 64, 262144)
    rows = _spread(rng, 1, max(2, min(16384, 2 ** 28 // vocab)))
    case = {"kind": kind, "rows": rows, "vocab": vocab, "dtype": dtype}
    if kind == "score":
        rows = min(rows, max(1, 2 ** 26 // vocab))
        return {**case, "rows": rows, "top": rng.choice((0, 0, 1, 5, 20, 50))}
    return case


# ----------------------------------------------------------------------------
# Inputs
# ----------------------------------------------------------------------------


def _normal(g, shape, dtype, by=1.0):
    return (torch.randn(shape, generator=g, dtype=torch.float32, device="cuda") * by).to(dtype)


def _words(g, n, vocab):
    """Tokens whose frequencies fall off as words' do, the frequent ones anywhere
    in the vocabulary."""
    u = torch.rand((n,), generator=g, dtype=torch.float64, device="cuda")
    rank = torch.exp(u * math.log(vocab + 1)).floor().long().sub(1).clamp(0, vocab - 1)
    return torch.randperm(vocab, generator=g, device="cuda")[rank]


def _mixer(s, g, case, length):
    """A mixer's inputs: x and z as halves of one projection's rows, B and C as
    parts of another's, steps around a channel's own between 0.001 and 0.1."""
    dt, n, d, groups = _DTYPES[case["dtype"]], case["states"], case["channels"], case["groups"]
    rows = (case["batch"], length)
    both = _normal(g, (*rows, 2 * d), dt)
    s["x"], s["z"] = both[..., :d], both[..., d:]
    s["dt"] = _normal(g, (*rows, d), dt, 0.5)
    parts = _normal(g, (*rows, 2 * groups * n + 128), dt)
    s["B"] = parts[..., 128:128 + groups * n].unflatten(2, (groups, n))
    s["C"] = parts[..., 128 + groups * n:].unflatten(2, (groups, n))
    step = torch.exp(torch.rand((d,), generator=g, device="cuda") * math.log(100.0)) * 0.001
    s["bias"] = torch.log(torch.expm1(step))
    s["A"] = -(1.0 + torch.arange(n, device="cuda")) * torch.exp(0.1 * torch.randn((d, n), generator=g, device="cuda"))
    s["D"] = 1.0 + 0.1 * torch.randn((d,), generator=g, device="cuda")


def _lengths(case):
    """Lengths from a quarter of the longest to it."""
    n, most = case["batch"], case["length"]
    return [max(1, most - (most * 3 * i) // (4 * max(1, n - 1))) for i in range(n)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, s = case["kind"], {"case": case}
    dt = _DTYPES[case["dtype"]]
    if kind in ("lookup", "lookup_grad"):
        rows, vocab, width = case["rows"], case["vocab"], case["width"]
        s["tokens"], s["scale"] = _words(g, rows, vocab), math.sqrt(width)
        if kind == "lookup":
            s["table"] = _normal(g, (vocab, width), dt, width ** -0.5)
        else:
            s["tokens"][-1] = -1   # padding
            s["dy"] = _normal(g, (rows, width), dt)
    elif kind in ("conv", "conv_step"):
        d, k, rows = case["channels"], case["taps"], (case["batch"], case.get("length", 1))
        s["x"] = _normal(g, (*rows, 2 * d), dt)[..., :d]   # a part of a projection's rows
        s["w"], s["b"] = _normal(g, (d, k), dt, k ** -0.5), _normal(g, (d,), dt, 0.1)
        if kind == "conv":
            s["dy"] = _normal(g, (*rows, d), dt)
        else:
            s["x"], s["state"] = s["x"][:, 0], _normal(g, (case["batch"], k - 1, d), dt)
    elif kind in ("scan", "scan_train", "scan_step"):
        _mixer(s, g, case, case.get("length", 1))
        if kind == "scan":
            s["lengths"] = torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None
        elif kind == "scan_train":
            s["dy"] = _normal(g, s["x"].shape, dt)
        else:
            for name in ("x", "z", "dt", "B", "C"):
                s[name] = s[name][:, 0]
            s["h"] = torch.randn((case["batch"], case["channels"], case["states"]), generator=g, device="cuda")
    else:
        rows, vocab = case["rows"], case["vocab"]
        s["logits"] = _normal(g, (rows, vocab), dt, 3.0)
        s["tokens"] = torch.randint(vocab, (rows,), generator=g, device="cuda")
        if kind == "score_train":
            s["tokens"][::17] = -1   # not scored
            s["dlogp"] = torch.full((rows,), -1.0 / rows, device="cuda")
            s["dentropy"] = 0.01 * torch.randn((rows,), generator=g, device="cuda") / rows
    return s


# ----------------------------------------------------------------------------
# The plain forms
# ----------------------------------------------------------------------------


def _plain_lookup(tokens, table, scale):
    fine = (tokens >= 0) & (tokens < table.shape[0])
    y = table[torch.where(fine, tokens, 0)].float() * scale
    return torch.where(fine[:, None], y, 0.0).to(table.dtype)


def _plain_lookup_grad(tokens, dy, vocab, scale, out):
    fine = (tokens >= 0) & (tokens < vocab)
    d = torch.zeros((vocab + 1, dy.shape[1]), dtype=torch.float32, device=dy.device)
    d.index_add_(0, torch.where(fine, tokens, vocab), dy.float() * scale)
    return d[:vocab].to(out)


def _plain_taps(x, w, b):
    """The convolution's sums from windows x [.., channels, taps]."""
    return (x * w.float()).sum(-1) + b.float()


def _plain_conv(x, w, b, dy):
    k = w.shape[1]
    window = torch.nn.functional.pad(x.float(), (0, 0, k - 1, 0)).unfold(1, k, 1)
    pre = _plain_taps(window, w, b)
    gate = torch.sigmoid(pre)
    g = dy.float() * gate * (1.0 + pre * (1.0 - gate))
    after = torch.nn.functional.pad(g, (0, 0, 0, k - 1)).unfold(1, k, 1)
    dx = (after * w.float().flip(1)).sum(-1)
    dw = (window * g[..., None]).sum((0, 1))
    return {"y": (pre * gate).to(x.dtype), "dx": dx.to(x.dtype), "dw": dw, "db": g.sum((0, 1))}


def _plain_conv_step(x, w, b, state):
    window = torch.cat([state, x[:, None]], 1)
    pre = _plain_taps(window.float().transpose(1, 2), w, b)
    state.copy_(window[:, 1:])
    return {"y": (pre * torch.sigmoid(pre)).to(x.dtype), "state": state}


def _plain_softplus(v):
    return torch.log1p(torch.exp(-v.abs())) + v.clamp(min=0.0)


def _plain_recurrence(a, b):
    """h_t = a_t h_(t-1) + b_t along dimension 1, by doubling; both are overwritten, b by h."""
    reach = 1
    while reach < a.shape[1]:
        b[:, reach:] += a[:, reach:] * b[:, :-reach]
        a[:, reach:] = a[:, reach:] * a[:, :-reach]
        reach *= 2
    return b


def _plain_terms(s, lengths=None):
    """Steps, and each token's decay and input of the states [.., channels, N]."""
    x, shared = s["x"].float(), s["x"].shape[-1] // s["B"].shape[-2]
    step = _plain_softplus(s["dt"].float() + s["bias"])
    if lengths is not None:
        step = torch.where(torch.arange(x.shape[1], device=x.device)[:, None] < lengths[:, None, None], step, 0.0)
    a = torch.exp(step[..., None] * s["A"])
    b = (step * x)[..., None] * s["B"].float().repeat_interleave(shared, -2)
    return x, step, a, b, s["C"].float().repeat_interleave(shared, -2)


def _plain_gate(z):
    z = z.float()
    return z * torch.sigmoid(z)


def _plain_scan(s, lengths):
    x, _, a, b, c = _plain_terms(s, lengths)
    h = _plain_recurrence(a, b)
    del a
    last = h[:, -1].clone()
    y = h.mul_(c).sum(-1)
    y = (y + s["D"] * x) * _plain_gate(s["z"])
    if lengths is not None:
        y = torch.where(torch.arange(x.shape[1], device=x.device)[:, None] < lengths[:, None, None], y, 0.0)
    return {"y": y.to(s["x"].dtype), "h": last}


def _plain_scan_train(s):
    x, step, a, b, c = _plain_terms(s)
    shape, dtype, groups = s["x"].shape, s["x"].dtype, s["B"].shape[-2]
    h = _plain_recurrence(a.clone(), b)
    y = (h * c).sum(-1) + s["D"] * x
    z, dy = s["z"].float(), s["dy"].float()
    gate = torch.sigmoid(z)
    dz = dy * y * gate * (1.0 + z * (1.0 - gate))
    inner = dy * z * gate
    # The states' gradients, by the same recurrence from the end.
    later = torch.nn.functional.pad(a[:, 1:], (0, 0, 0, 0, 0, 1)).flip(1)
    g = _plain_recurrence(later, (inner[..., None] * c).flip(1)).flip(1)
    del later
    dc = (h * inner[..., None]).unflatten(2, (groups, -1)).sum(3)
    db = (g * (step * x)[..., None]).unflatten(2, (groups, -1)).sum(3)
    along = (g * s["B"].float().repeat_interleave(shape[-1] // groups, -2)).sum(-1)
    past = g * a * torch.nn.functional.pad(h[:, :-1], (0, 0, 0, 0, 1, 0))
    del a, h, g
    dstep = along * x + (past * s["A"]).sum(-1)
    ddt = dstep * torch.sigmoid(s["dt"].float() + s["bias"])
    return {"y": (y * z * gate).to(dtype), "dx": (along * step + inner * s["D"]).to(dtype), "ddt": ddt.to(dtype),
            "dA": (past * step[..., None]).sum((0, 1)), "dB": db.to(dtype), "dC": dc.to(dtype),
            "dD": (inner * x).sum((0, 1)), "dz": dz.to(dtype), "dbias": ddt.sum((0, 1))}


def _plain_scan_step(s):
    x, _, a, b, c = _plain_terms(s)
    h = s["h"]
    h.mul_(a).add_(b)
    y = ((h * c).sum(-1) + s["D"] * x) * _plain_gate(s["z"])
    return {"y": y.to(s["x"].dtype), "h": h}


def _plain_scores(logits, tokens):
    z = logits.float()
    low = z.amax(-1, keepdim=True)
    e = torch.exp(z - low)
    total = e.sum(-1)
    lse = torch.log(total) + low[:, 0]
    entropy = torch.log(total) - (e * (z - low)).sum(-1) / total
    fine = tokens >= 0
    picked = torch.gather(z, 1, torch.where(fine, tokens, 0)[:, None])[:, 0]
    return z, {"logp": torch.where(fine, picked - lse, 0.0), "lse": lse, "entropy": entropy}


def _plain_score(logits, tokens, top):
    z, out = _plain_scores(logits, tokens)
    if top:
        best, at = torch.sort(z, dim=-1, descending=True, stable=True)
        out["top_logp"], out["top_tokens"] = best[:, :top] - out["lse"][:, None], at[:, :top].contiguous()
    return out


def _plain_score_train(logits, tokens, dlogp, dentropy):
    z, out = _plain_scores(logits, tokens)
    fine = tokens >= 0
    dlogp = torch.where(fine, dlogp, 0.0)
    logs = z - out["lse"][:, None]
    d = torch.exp(logs) * -(dlogp[:, None] + dentropy[:, None] * (logs + out["entropy"][:, None]))
    d.scatter_add_(1, torch.where(fine, tokens, 0)[:, None], dlogp[:, None])
    return {**out, "dlogits": d.to(logits.dtype)}


# ----------------------------------------------------------------------------
# One pass
# ----------------------------------------------------------------------------


def run(state):
    if own:
        return _run_own(state)
    s, case = state, state["case"]
    kind = case["kind"]
    if kind == "lookup":
        return {"y": _plain_lookup(s["tokens"], s["table"], s["scale"])}
    if kind == "lookup_grad":
        return {"d": _plain_lookup_grad(s["tokens"], s["dy"], case["vocab"], s["scale"], _DTYPES[case["out"]])}
    if kind == "conv":
        return _plain_conv(s["x"], s["w"], s["b"], s["dy"])
    if kind == "conv_step":
        return _plain_conv_step(s["x"], s["w"], s["b"], s["state"])
    if kind == "scan":
        return _plain_scan(s, s["lengths"])
    if kind == "scan_train":
        return _plain_scan_train(s)
    if kind == "scan_step":
        return _plain_scan_step(s)
    if kind == "score":
        return _plain_score(s["logits"], s["tokens"], case["top"])
    return _plain_score_train(s["logits"], s["tokens"], s["dlogp"], s["dentropy"])


def _run_own(s):
    import paper_2512_13921_amd as swr
    case = s["case"]
    kind = case["kind"]
    if kind == "lookup":
        return {"y": swr.swr_embedding(s["tokens"], s["table"], scale=s["scale"])}
    if kind == "lookup_grad":
        return {"d": swr.swr_embedding_backward(s["tokens"], s["dy"], case["vocab"], scale=s["scale"],
                                                dtype=_DTYPES[case["out"]])}
    if kind == "conv":
        y, _ = swr.swr_causal_conv(s["x"], s["w"], s["b"])
        dx, dw, db = swr.swr_causal_conv_backward(s["x"], s["w"], s["dy"], s["b"])
        return {"y": y, "dx": dx, "dw": dw, "db": db}
    if kind == "conv_step":
        y = swr.swr_causal_conv_step(s["x"], s["w"], s["state"], s["b"])
        return {"y": y, "state": s["state"]}
    if kind in ("scan", "scan_train", "scan_step"):
        args, more = (s["x"], s["dt"], s["A"], s["B"], s["C"]), dict(D=s["D"], z=s["z"], dt_bias=s["bias"])
        if kind == "scan":
            y, _, h = swr.swr_selective_scan(*args, **more, lengths=s["lengths"], want_state=True)
            return {"y": y, "h": h}
        if kind == "scan_step":
            return {"y": swr.swr_selective_step(*args, s["h"], **more), "h": s["h"]}
        y, carriers, _ = swr.swr_selective_scan(*args, **more, save_carriers=True)
        dx, ddt, dA, dB, dC, dD, dz, dbias, _ = swr.swr_selective_scan_backward(*args, s["dy"], carriers, **more)
        return {"y": y, "dx": dx, "ddt": ddt, "dA": dA, "dB": dB, "dC": dC, "dD": dD, "dz": dz, "dbias": dbias}
    if kind == "score":
        r = swr.swr_log_probs(s["logits"], s["tokens"], top=case["top"])
        return dict(zip(("logp", "lse", "entropy", "top_logp", "top_tokens"), r))
    logp, lse, entropy = swr.swr_log_probs(s["logits"], s["tokens"])
    d = swr.swr_log_probs_backward(s["logits"], s["tokens"], lse, entropy, s["dlogp"], s["dentropy"])
    return {"logp": logp, "lse": lse, "entropy": entropy, "dlogits": d}


# ----------------------------------------------------------------------------
# Work, and the values in 64 bits
# ----------------------------------------------------------------------------


def work(case):
    """Bytes and operations of one pass: each call's inputs read once and its
    outputs written once (a forward and a backward are two calls).  Of the scan's
    states a step is a decay's product and exponential, the input's product, the
    update and the readout: 7 operations; its backward 17 more, the states' own
    values among them."""
    kind, es = case["kind"], _BYTES[case["dtype"]]
    if kind == "lookup":
        n = case["rows"] * case["width"]
        return {"bytes": 2 * n * es + 8 * case["rows"], "flops": n}
    if kind == "lookup_grad":
        n = case["rows"] * case["width"]
        return {"bytes": n * es + 8 * case["rows"] + case["vocab"] * case["width"] * _BYTES[case["out"]], "flops": 2 * n}
    if kind in ("conv", "conv_step"):
        n, d, k = case["batch"] * case.get("length", 1) * case["channels"], case["channels"], case["taps"]
        if kind == "conv_step":
            return {"bytes": (2 * n + 2 * (k - 1) * n + (k + 1) * d) * es, "flops": n * (2 * k + 5)}
        return {"bytes": 5 * n * es + 2 * (k + 1) * d * es + 4 * (k + 1) * d, "flops": n * (8 * k + 15)}
    if kind in ("scan", "scan_train", "scan_step"):
        d, n, groups = case["channels"], case["states"], case["groups"]
        tokens = sum(_lengths(case)) if case.get("ragged") else case["batch"] * case.get("length", 1)
        once = 4 * (d * n + 2 * d)
        h = 4 * case["batch"] * d * n
        if kind == "scan":
            return {"bytes": tokens * (4 * d + 2 * groups * n) * es + once + h, "flops": tokens * d * (7 * n + 20)}
        if kind == "scan_step":
            return {"bytes": tokens * (4 * d + 2 * groups * n) * es + once + 2 * h, "flops": tokens * d * (7 * n + 20)}
        return {"bytes": tokens * (11 * d + 6 * groups * n) * es + 3 * once, "flops": tokens * d * (24 * n + 60)}
    rows, vocab = case["rows"], case["vocab"]
    n = rows * vocab
    if kind == "score":
        return {"bytes": n * es + rows * (20 + 12 * case["top"]), "flops": 6 * n}
    return {"bytes": 3 * n * es + rows * 44, "flops": 12 * n}


def _exact_step(s, h, at):
    """One token of the scan in 64 bits: the states after it, and what it used of them."""
    f64 = torch.float64
    x = s["x"][:, at].to(f64)
    step = torch.logaddexp(s["dt"][:, at].to(f64) + s["bias"].to(f64), torch.zeros((), dtype=f64, device="cuda"))
    wide = x.shape[-1] // s["B"].shape[-2]
    b = s["B"][:, at].to(f64).repeat_interleave(wide, 1)
    c = s["C"][:, at].to(f64).repeat_interleave(wide, 1)
    decay = torch.exp(step[..., None] * s["A"].to(f64))
    return decay * h + (step * x)[..., None] * b, x, step, decay, b, c


def _exact_silu(v):
    return v / (1 + torch.exp(-v))


def _exact_scan(s, case):
    f64, length = torch.float64, case["length"]
    h = torch.zeros((case["batch"], case["channels"], case["states"]), dtype=f64, device="cuda")
    out, skip = torch.zeros(s["x"].shape, dtype=f64, device="cuda"), s["D"].to(f64)
    for at in range(length):
        new, x, _, _, _, c = _exact_step(s, h, at)
        y = ((new * c).sum(-1) + skip * x) * _exact_silu(s["z"][:, at].to(f64))
        if s["lengths"] is not None:
            live = at < s["lengths"]
            new, y = torch.where(live[:, None, None], new, h), torch.where(live[:, None], y, 0)
        h, out[:, at] = new, y
    return {"y": out, "h": h}


def _exact_scan_train(s, case):
    f64, length, wide = torch.float64, case["length"], case["channels"] // case["groups"]
    skip, rate = s["D"].to(f64), s["A"].to(f64)
    h = torch.zeros((case["batch"], case["channels"], case["states"]), dtype=f64, device="cuda")
    held = torch.empty((length + 1, *h.shape), dtype=f64, device="cuda")
    held[0] = h
    for at in range(length):
        held[at + 1] = _exact_step(s, held[at], at)[0]
    out = {n: torch.zeros(s[k].shape, dtype=f64, device="cuda") for n, k in (
        ("y", "x"), ("dx", "x"), ("ddt", "x"), ("dA", "A"), ("dB", "B"), ("dC", "C"), ("dD", "D"), ("dz", "x"),
        ("dbias", "D"))}
    back = torch.zeros_like(h)   # the gradient that reaches a token's states from later ones
    for at in reversed(range(length)):
        _, x, step, decay, b, c = _exact_step(s, held[at], at)
        y = (held[at + 1] * c).sum(-1) + skip * x
        z, dy = s["z"][:, at].to(f64), s["dy"][:, at].to(f64)
        gate = 1 / (1 + torch.exp(-z))
        out["y"][:, at], out["dz"][:, at] = y * z * gate, dy * y * (gate + z * gate * (1 - gate))
        inner = dy * z * gate
        back = back + inner[..., None] * c
        out["dC"][:, at] = (held[at + 1] * inner[..., None]).unflatten(1, (-1, wide)).sum(2)
        out["dB"][:, at] = (back * (step * x)[..., None]).unflatten(1, (-1, wide)).sum(2)
        along = (back * b).sum(-1)
        back = back * decay
        past = back * held[at]
        dstep = along * x + (past * rate).sum(-1)
        out["dx"][:, at] = along * step + skip * inner
        ddt = dstep / (1 + torch.exp(-(s["dt"][:, at].to(f64) + s["bias"].to(f64))))
        out["ddt"][:, at] = ddt
        out["dA"] += (past * step[..., None]).sum(0)
        out["dD"] += (inner * x).sum(0)
        out["dbias"] += ddt.sum(0)
    return out


def _exact_conv(s, case):
    """The definition tap by tap: the tap j of k has the token k - 1 - j back."""
    f64, k, length = torch.float64, case["taps"], case["length"]
    x, w, dy = s["x"].to(f64), s["w"].to(f64), s["dy"].to(f64)
    pre = s["b"].to(f64).expand(x.shape).clone()
    for j in range(k):
        lag = k - 1 - j
        if lag < length:
            pre[:, lag:] += w[:, j] * x[:, :length - lag]
    gate = 1 / (1 + torch.exp(-pre))
    g = dy * (gate + pre * gate * (1 - gate))
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    for j in range(k):
        lag = k - 1 - j
        if lag < length:
            dx[:, :length - lag] += w[:, j] * g[:, lag:]
            dw[:, j] = (g[:, lag:] * x[:, :length - lag]).sum((0, 1))
    return {"y": pre * gate, "dx": dx, "dw": dw, "db": g.sum((0, 1))}


def _exact_scores(s, case):
    """Row by row in 64 bits (a few at a time)."""
    f64, vocab, out = torch.float64, case["vocab"], {}
    parts = []
    for low in range(0, case["rows"], max(1, 2 ** 26 // vocab)):
        rows = slice(low, low + max(1, 2 ** 26 // vocab))
        z, tokens = s["logits"][rows].to(f64), s["tokens"][rows]
        lse = torch.logsumexp(z, -1)
        logs = z - lse[:, None]
        p = torch.exp(logs)
        entropy = -(p * logs).sum(-1)
        scored = tokens >= 0
        at = (torch.arange(len(tokens), device="cuda"), tokens.clamp(min=0))
        part = {"logp": logs[at] * scored, "lse": lse, "entropy": entropy}
        if case.get("top"):
            order = torch.argsort(-z, dim=-1, stable=True)[:, :case["top"]]
            part["top_logp"], part["top_tokens"] = torch.gather(logs, 1, order), order
        if case["kind"] == "score_train":
            dlogp, dentropy = s["dlogp"][rows].to(f64) * scored, s["dentropy"][rows].to(f64)
            d = -p * dlogp[:, None] - dentropy[:, None] * p * (logs + entropy[:, None])
            d[at] += dlogp
            part["dlogits"] = d
        parts.append(part)
    for name in parts[0]:
        out[name] = torch.cat([part[name] for part in parts])
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind == "lookup":
        return {"y": s["table"][s["tokens"]].to(f64) * s["scale"]}
    if kind == "lookup_grad":
        d = torch.zeros((case["vocab"], case["width"]), dtype=f64, device="cuda")
        kept = s["tokens"] >= 0
        d.index_add_(0, s["tokens"][kept], s["dy"][kept].to(f64))
        return {"d": d.mul_(s["scale"])}
    if kind == "conv":
        return _exact_conv(s, case)
    if kind == "conv_step":
        past = torch.cat([s["state"].to(f64), s["x"].to(f64)[:, None]], 1)
        pre = s["b"].to(f64) + sum(s["w"][:, j].to(f64) * past[:, j] for j in range(case["taps"]))
        return {"y": _exact_silu(pre), "state": past[:, 1:]}
    if kind == "scan":
        return _exact_scan(s, case)
    if kind == "scan_train":
        return _exact_scan_train(s, case)
    if kind == "scan_step":
        for name in ("x", "z", "dt", "B", "C"):
            s[name] = s[name][:, None]
        h, x, _, _, _, c = _exact_step(s, s["h"].to(f64), 0)
        y = ((h * c).sum(-1) + s["D"].to(f64) * x) * _exact_silu(s["z"][:, 0].to(f64))
        return {"y": y, "h": h}
    return _exact_scores(s, case)
