"""Products of few channels: rows of every number of 16-byte chunks, and calls with so many positions that one workgroup makes all channels."""
import pytest
import torch

from test_gpu_linear import DTYPES, _act_id, _case, _check_forward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("chunks", range(1, 17))
def test_rows_of_every_number_of_chunks(lp, chunks, dtype):
    each = 4 if dtype == torch.float32 else 8
    for i, (k, n) in enumerate(((chunks * each, 128), (chunks * each, 40), (chunks * each - each // 2, 97), (chunks * each - each + 1, 64))):
        for p in (9, 200):
            t = _case(p, k, n, dtype, 31 * chunks + i + p, ["", "even", "odd", "odd"][i])
            lin = lp.Linear(t["w"], t["b"], _act_id(lp, "silu"))
            y, pre = lp.linear_fwd(lin, t["x"], t["r"], keep=True)
            _check_forward(t, "silu", dtype, y, pre)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bytes_in", [64, 128, 160, 192, 256])
@pytest.mark.parametrize("n", [97, 128])
def test_many_positions_and_few_come_out_alike(lp, n, bytes_in, dtype):
    """A position's result does not depend on the others: a call of more positions than 1024 for each compute unit, and calls of some of them."""
    p, k = 1024 * torch.cuda.get_device_properties(0).multi_processor_count + 77, bytes_in // (4 if dtype == torch.float32 else 2)
    gen = torch.Generator(device="cuda").manual_seed(bytes_in + n)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    x, r = rand(p, k).to(dtype), rand(p, n).to(dtype)
    lin = lp.Linear((rand(n, k) / k ** 0.5).to(dtype), rand(n), lp.LP_ACT_GELU)
    y, pre = lp.linear_fwd(lin, x, r, keep=True)
    for at in (0, p // 2, p - 1500):
        want = lp.linear_fwd(lin, x[at:at + 1500], r[at:at + 1500], keep=True)
        assert torch.equal(y[at:at + 1500], want[0]) and torch.equal(pre[at:at + 1500], want[1])
