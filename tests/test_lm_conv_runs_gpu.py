"""The convolution's gradient where runs of 16, 32 and 48 tokens end inside a sequence, of data that is
dense there."""
import pytest

import lm_ref as ref
from lm_ref import ROUND, TINY, U, rand
from test_lm_conv_gpu import make, swr  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("B,T,C,K,adds", [
    # Runs: 48 tokens from 8192 waves of 32 on, 32 from 1024 on.  `adds`: additions in a row of a sum of dw, which a
    # wave makes over the runs of its own, the block over its four, and the last kernel over a quarter of 1024 rows.
    (2100, 100, 8, 4, 2 * 48 + 4 + 256 + 2), (1400, 200, 7, 8, 2 * 48 + 4 + 256 + 2), (300, 130, 12, 3, 32 + 4 + 256 + 2),
    (3, 75, 260, 5, 16 + 4 + 5 + 2)])
def test_runs(swr, dtype, B, T, C, K, adds):  # noqa: F811
    x, w, bias = make(31, B, T, C, K, dtype)
    dy = rand(32, (B, T, C), dtype).cuda()
    lengths = torch.randint(0, T + 1, (B,), generator=torch.Generator().manual_seed(33)).int()
    lengths[: B // 2] = T
    n = lengths.cuda()
    for silu, b, lens in ((True, bias, n), (False, None, None)):
        got = swr.swr_causal_conv_backward(x, w, dy, b, silu, lens)
        dx, dw, db, sx, sw, sb = ref.conv_backward(x, w, b, silu, lens, dy)
        ref.close(got[0], dx, dx.abs() * ROUND[dtype] + sx * U * (2 * K + 12) * (1 + ROUND[dtype]) + TINY, "dx")
        ref.close(got[1], dw, dw.abs() * ROUND[F32] + sw * U * (2 * K + 12 + adds) + TINY, "dw")
        if b is not None:
            ref.close(got[2], db, db.abs() * ROUND[F32] + sb * U * (2 * K + 12 + adds) + TINY, "db")
