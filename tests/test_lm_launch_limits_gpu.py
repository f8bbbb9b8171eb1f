"""A scan whose blocks would pass a launch's 2^32 threads."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
F32 = torch.float32


@pytest.fixture()
def swr():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    if torch.cuda.mem_get_info()[0] < 90 << 30:
        pytest.skip("needs 90 GB of device memory")
    import paper_2512_13921_amd as lib
    lib.load()
    return lib


def test_single_tokens_of_more_channels_than_a_launch_has_threads_for(swr):
    # 2^28 channels of 33 states, 16 lanes each: 2^32 threads.
    D, N = 1 << 28, 33
    x = torch.full((1, D), 0.5, dtype=torch.bfloat16, device="cuda")
    x[0, ::3] = -2.0
    dt = torch.full_like(x, 0.25)
    A = torch.full((D, N), -1.0, device="cuda")
    A[::7] = -2.0
    state = torch.full((1, D, N), 2.0, device="cuda")
    state[:, ::5] = -1.0
    b, c = (torch.full((1, N), v, dtype=torch.bfloat16, device="cuda") for v in (1.0, 0.5))
    y = swr.swr_selective_step(x, dt, A, b, c, state, softplus=False)
    torch.cuda.synchronize()
    step = 1 << 24
    for first in range(0, D, step):
        d = torch.arange(first, first + step, device="cuda")
        decay = torch.exp(-0.25 * torch.where(d % 7 == 0, 2.0, 1.0).double())
        h = decay * torch.where(d % 5 == 0, -1.0, 2.0).double() + 0.25 * torch.where(d % 3 == 0, -2.0, 0.5).double()
        got = state[0, first:first + step]
        # exp's argument and value, a product and a sum, of values of at most 2.5: some halves of a step of 2
        assert float((got.double() - h[:, None]).abs().max()) < 8 * 2.0 ** -23, first
        want = 0.5 * N * h
        assert float(((y[0, first:first + step].double() - want).abs() - want.abs() * 2.0 ** -8).max()) < 1e-4, first
