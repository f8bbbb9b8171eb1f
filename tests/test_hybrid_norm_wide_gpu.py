"""The norm's backward of rows so wide that one launch's blocks take several ranges of
columns each (more than 2^26 columns: 2^22 blocks of 1024 threads are a launch's limit)."""
import pytest

import hybrid_ref as ref
from hybrid_ref import ROUND, TINY, U
from test_hybrid_norm_gpu import _terms

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_backward_of_very_wide_rows(dtype):
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2512_13921_amd as swr
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("needs 8 GB of device memory")
    width = (1 << 26) + 1000003
    g = torch.Generator(device="cuda").manual_seed(1)
    h, dy, dh, w = (torch.randn((n, width) if n else (width,), generator=g, device="cuda").to(dtype) for n in (1, 1, 1, 0))
    dx, dw = swr.swr_rms_norm_backward(h, w, dy, dh=dh)
    again = swr.swr_rms_norm_backward(h, w, dy, dh=dh, dx=dh.clone())
    torch.cuda.synchronize()
    assert torch.equal(dx, again[0]) and torch.equal(dw, again[1])
    want_x, want_w, size_x, size_w = ref.norm_backward(h, w, dy, dh, 1e-6)
    ref.close(dx, want_x, want_x.abs() * ROUND[dtype] + size_x * U * (2 * _terms(width) + 16) + TINY, "dx")
    ref.close(dw, want_w, size_w * U * (_terms(width) + 64) + TINY, "dw")
