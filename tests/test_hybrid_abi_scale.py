"""Scales of attention whose product with log2 e is no float32 are refused (CPU only)."""
import ctypes

import pytest

from test_hybrid_abi import ADDRESS, E_ALIGN, E_UNSUP, _attention, _paged, hybrid


@pytest.mark.parametrize("scale", [2.4e38, -2.4e38, 3.4028234663852886e38, float("inf"), float("nan")])
def test_refused(scale):
    assert _attention(_paged(scale=scale)) == E_UNSUP
    assert hybrid._lib().swr_paged_workspace_bytes(ctypes.byref(_paged(scale=scale))) == E_UNSUP


@pytest.mark.parametrize("scale", [2.3e38, -2.3e38, 0.0, 1e-45])
def test_taken(scale):
    assert _attention(_paged(scale=scale), q=ADDRESS[11] + 8) == E_ALIGN     # (what is checked next)
