"""Outputs that lie between the inputs' elements, as parts of one larger tensor do: taken, and the same as apart."""
import pytest

from lm_ref import rand
from test_lm_scan_gpu import make as make_scan

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


def _is_alias(swr, f):
    with pytest.raises(swr.SwrError) as e:
        f()
    assert e.value.code == -6


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_convolution(swr, dtype):
    """y beside x in a projection's rows; the gradients beside both, batch by batch and token by token."""
    B, T, C = 3, 37, 24
    w, bias = rand(1, (C, 4), dtype).cuda(), rand(2, (C,), dtype).cuda()
    rows = rand(3, (B, T, 5 * C), dtype).cuda()
    for wide in (rows, rows.transpose(0, 1).contiguous().transpose(0, 1)):   # (a batch, or a token, after the other)
        before = wide.clone()
        x, y, dy, dx = (wide[..., i * C:(i + 1) * C] for i in range(4))
        apart, _ = swr.swr_causal_conv(x.contiguous(), w, bias)
        out, _ = swr.swr_causal_conv(x, w, bias, y=y)
        assert torch.equal(out, apart) and torch.equal(y, apart)
        want = swr.swr_causal_conv_backward(x.contiguous(), w, dy.contiguous(), bias)
        got = swr.swr_causal_conv_backward(x, w, dy, bias, dx=dx)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(dx, want[0])
        for i in (0, 2, 4):
            assert torch.equal(wide[..., i * C:(i + 1) * C], before[..., i * C:(i + 1) * C])
        one = wide[..., C - 1:2 * C - 1]   # (its first column is x's last)
        _is_alias(swr, lambda: swr.swr_causal_conv(x, w, bias, y=one))
        _is_alias(swr, lambda: swr.swr_causal_conv_backward(x, w, dy, bias, dx=one))
        _is_alias(swr, lambda: swr.swr_causal_conv_backward(x, w, dy, bias, dx=dy))
        _is_alias(swr, lambda: swr.swr_causal_conv(x, w, bias, y=x))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [5, 40])
def test_scan(swr, dtype, T):
    """y in the rows that x, dt, z, B and C are parts of."""
    B, D, N, G = 2, 20, 16, 2
    width = 4 * D + 2 * G * N
    s = make_scan(1, B, T, D, N, G, dtype)
    for turned in (False, True):
        wide = torch.zeros((T, B, width) if turned else (B, T, width), dtype=dtype, device="cuda")
        if turned:
            wide = wide.transpose(0, 1)
        parts = {"x": wide[..., :D], "dt": wide[..., D:2 * D], "z": wide[..., 3 * D:4 * D],
                 "B": wide[..., 4 * D:4 * D + G * N].unflatten(2, (G, N)), "C": wide[..., 4 * D + G * N:].unflatten(2, (G, N))}
        for k, t in parts.items():
            t.copy_(s[k])
        want, _, _ = swr.swr_selective_scan(**s)
        y, _, _ = swr.swr_selective_scan(**{**s, **parts}, y=wide[..., 2 * D:3 * D])
        assert torch.equal(y, want)
        for k, t in parts.items():
            assert torch.equal(t, s[k])
        for at in (2 * D - 1, 2 * D + 1, 4 * D + G * N - 1, width - D):
            _is_alias(swr, lambda: swr.swr_selective_scan(**{**s, **parts}, y=wide[..., at:at + D]))
        if T == 5:   # a token alone, between the states' and the other tokens'
            x, dt, z, b, c = (parts[k][:, 1] for k in ("x", "dt", "z", "B", "C"))
            state = torch.zeros(B, D, N, device="cuda")
            apart = swr.swr_selective_step(x, dt, s["A"], b, c, state.clone(), s["D"], z, s["dt_bias"])
            y = swr.swr_selective_step(x, dt, s["A"], b, c, state, s["D"], z, s["dt_bias"], y=wide[:, 1, 2 * D:3 * D])
            assert torch.equal(y, apart)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_logits_gradient(swr, dtype):
    """dlogits beside the logits, row by row."""
    rows, V = 7, 300
    wide = rand(4, (rows, 2 * V), dtype).cuda()
    logits, tokens = wide[:, :V], torch.randint(V, (rows,), generator=torch.Generator().manual_seed(5)).cuda()
    before = logits.clone()
    _, lse, entropy = swr.swr_log_probs(logits, tokens)
    g = rand(6, (rows,), F32).cuda()
    want = swr.swr_log_probs_backward(before, tokens, lse, entropy, g)
    got = swr.swr_log_probs_backward(logits, tokens, lse, entropy, g, dlogits=wide[:, V:])
    assert torch.equal(got, want) and torch.equal(logits, before)
    _is_alias(swr, lambda: swr.swr_log_probs_backward(logits, tokens, lse, entropy, g, dlogits=wide[:, V - 1:2 * V - 1]))
    _is_alias(swr, lambda: swr.swr_log_probs_backward(logits[1:], tokens[1:], lse[1:], entropy[1:], g[1:],
                                                      dlogits=wide[:-1, :V]))
