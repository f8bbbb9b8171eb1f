"""Outputs that meet an input within a larger tensor's rows are refused, wherever in them (those that lie between its
elements are taken: test_lm_parts_gpu)."""
import pytest

from test_lm_abi import ADDRESS, E_ALIAS, _conv, _convolve, _convolve_back, _logp, _run, _scan, _score_back

X = ADDRESS[0]   # (bf16 elements of 2 bytes)


@pytest.mark.parametrize("turned", [False, True])
@pytest.mark.parametrize("at", [0, 1, 63, -1, -63, 128 - 63, 128 - 1, 128, 128 + 1, 50 * 128 - 1, 50 * 128, 50 * 128 + 63,
                                7 * 128 + 5, -7 * 128 - 5])
def test_convolution(at, turned):
    """Rows of 64 in rows of 128, a batch after the other or a token after the other."""
    sb, st = (128, 256) if turned else (6400, 128)
    p = _conv(**{f"s{n}_{d}": v for n in "xyd" for d, v in (("b", sb), ("t", st))})
    assert _convolve(p, y=X + 2 * at) == E_ALIAS
    assert _convolve_back(p, dx=X + 2 * at) == E_ALIAS
    assert _convolve_back(p, dx=ADDRESS[3] + 2 * at) == E_ALIAS
    # Rows of other strides are taken to meet where the tensors do.
    q = _conv(**{**{f"s{n}_{d}": v for n in "xd" for d, v in (("b", sb), ("t", st))}, "sy_b": 1 << 14, "sy_t": 256})
    assert _convolve(q, y=X + 2 * 64) == E_ALIAS


@pytest.mark.parametrize("name,width", [("x", 64), ("dt", 64), ("z", 64), ("B", 32), ("C", 32)])
def test_scan(name, width):
    strides = {f"s{n}_{d}": v for n in ("x", "dt", "z", "y", "B", "C") for d, v in (("b", 50 * 512), ("t", 512))}
    p, own = _scan(**strides), ADDRESS[("x", "dt", "A", "B", "C", "bias", "skip", "z").index(name)]
    for at in (0, width - 1, -63, 512 - 63, 512 + width - 1, 50 * 512, 49 * 512 + 3, -512 - 1, -50 * 512 - 63):
        assert _run(p, y=own + 2 * at) == E_ALIAS, at
    # (a token's groups count as one, with what lies between them)
    if name in "BC":
        far = _scan(**{**strides, f"s{name}_g": 200})
        assert _run(far, y=own + 2 * 100) == E_ALIAS


def test_logits():
    p = _logp(sl=256, sd=256)   # float32 rows of 100
    for at in (1, 99, -99, 256 - 99, 256, 256 + 5, 9 * 256 + 99, -256, -9 * 256 - 99):
        assert _score_back(p, dlogits=X + 4 * at) == E_ALIAS, at
