"""Few tokens of batches that are empty: nothing of theirs counts, their first token neither (the library's loads
for them go to A, which every call has), and their states stay as they are."""
import pytest

from test_lm_scan_gpu import check_forward, definition, make, swr  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T", [1, 5, 8])
@pytest.mark.parametrize("D,N,G,options", [(1, 1, 1, False), (130, 16, 1, True), (24, 6, 4, True), (9, 64, 9, False)])
@pytest.mark.parametrize("lengths", [[0], [0, 0], [0, 2, 0], [-4, 8, 0, 1, 0]])
def test_empty_batches(swr, dtype, T, D, N, G, options, lengths):  # noqa: F811
    B = len(lengths)
    s = make(60, B, T, D, N, G, dtype, options, options, options, True, lengths)
    for i, n in enumerate(lengths):
        for k, t in enumerate((s["x"], s["dt"], s["B"], s["C"], s["z"])):
            if t is not None:
                t[i, max(n, 0):] = (float("nan"), float("inf"))[(i + k) % 2]
    y, carriers, h = swr.swr_selective_scan(**s, save_carriers=True, want_state=True)
    check_forward(definition(s), y, h, carriers)
    for i, n in enumerate(lengths):
        if n <= 0:
            assert (y[i] == 0).all() and torch.equal(h[i], s["h0"][i])
    state = s["h0"].clone()
    swr.swr_selective_scan(**{**s, "h0": state}, h_last=state)
    assert torch.equal(state, h)
    _, _, h = swr.swr_selective_scan(**{**s, "h0": None}, want_state=True)
    assert all((h[i] == 0).all() for i, n in enumerate(lengths) if n <= 0)
