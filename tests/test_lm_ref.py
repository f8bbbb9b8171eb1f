"""The 64-bit definitions of a recurrent language model's operators against each other: their
gradients against differences of their values.

A central difference of step e is off by e^2 / 6 of the third derivative and by 2^-52 / e of the
value: with e = 2^-17 both stay below 1e-9 of values and derivatives of size 10, and sums of
a few hundred of them below 1e-6."""
import pytest
import torch

import lm_ref as ref

STEP = 2.0 ** -17


def rand(seed, *shape):
    return ref.rand(seed, shape, torch.float64)


def along(f, t, seed):
    """The derivative of f along a random direction from t by differences, and the direction."""
    way = rand(seed, *t.shape)
    return (f(t + STEP * way) - f(t - STEP * way)) / (2 * STEP), way


@pytest.mark.parametrize("with_silu", [False, True])
@pytest.mark.parametrize("lengths", [None, [0, 5, 9]])
def test_convolution(with_silu, lengths):
    n = None if lengths is None else torch.tensor(lengths)
    x, w, b, dy = rand(1, 3, 9, 4), rand(2, 4, 3), rand(3, 4), rand(4, 3, 9, 4)
    dx, dw, db = ref.conv_backward(x, w, b, with_silu, n, dy)[:3]

    def loss(x=x, w=w, b=b):
        return float((ref.conv(x, w, b, with_silu, None, n)[0] * dy).sum())

    for got, t, f in ((dx, x, lambda t: loss(x=t)), (dw, w, lambda t: loss(w=t)), (db, b, lambda t: loss(b=t))):
        d, way = along(f, t, 7)
        assert abs(d - float((got * way).sum())) < 1e-6


@pytest.mark.parametrize("softplus", [False, True])
@pytest.mark.parametrize("lengths", [None, [0, 6]])
def test_scan(softplus, lengths):
    n = None if lengths is None else torch.tensor(lengths)
    s = dict(x=rand(1, 2, 7, 4), dt=rand(2, 2, 7, 4) * 0.3, A=-torch.exp(rand(3, 4, 3) * 0.5), B=rand(4, 2, 7, 2, 3),
             C=rand(5, 2, 7, 2, 3), D=rand(6, 4), z=rand(7, 2, 7, 4), dt_bias=rand(8, 4) * 0.3, h0=rand(9, 2, 4, 3))
    dy, dh = rand(10, 2, 7, 4), rand(11, 2, 4, 3)

    def run(**kw):
        r = ref.Scan(use_softplus=softplus, lengths=n, **{**s, **kw})
        r.forward()
        return r

    def loss(**kw):
        r = run(**kw)
        return float((r.y * dy).sum() + (r.h[:, -1] * dh).sum())

    got = run().backward(dy, dh)
    for i, name in enumerate(s):
        d, way = along(lambda t: loss(**{name: t}), s[name], 20 + i)
        g = got["dt_bias" if name == "dt_bias" else "d" + name][0]
        assert abs(d - float((g * way).sum())) < 1e-6, name


def test_log_probs():
    z, tokens = rand(1, 5, 11), torch.tensor([0, 10, -1, 11, 4])
    weights = [rand(i, 5) for i in (2, 3, 4)]

    def loss(t):
        return float(sum((v * w).sum() for v, w in zip(ref.log_probs(t, tokens, 1.7)[:3], weights)))

    got, _ = ref.log_probs_backward(z, tokens, 1.7, weights[0], weights[1], weights[2])
    d, way = along(loss, z, 9)
    assert abs(d - float((got * way).sum())) < 1e-6


def test_embedding():
    table, tokens, dy = rand(1, 6, 3), torch.tensor([[0, 5, 5], [-1, 6, 2]]), rand(2, 2, 3, 3)
    got, _, most = ref.embedding_backward(tokens, dy, 6, 0.7)
    d, way = along(lambda t: float((ref.embedding(tokens, t, 0.7) * dy).sum()), table, 3)
    assert most == 2 and abs(d - float((got * way).sum())) < 1e-6
