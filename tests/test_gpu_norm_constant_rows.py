"""Layer norm of rows whose spread is small next to their offset: the mean is the sum divided by the number of columns."""
import numpy as np
import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TORCH = {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("cols", [7, 15, 100, 300, 1001, 1300, 2900, 5001, 9000, 20001])
def test_constant_rows_have_no_spread(cols, dtype, off, packed):
    """Sums of 1000, 9984 (both with seven significant bits) and their negatives: multiples of 8 and of 256 below 2^28, so that they are exact in
    any order, and so is the mean: the distances are zero, y is beta and the variance zero."""
    values = [1000.0, 9984.0, -1000.0, -9984.0, 0.0]
    ld = cols + off
    x = torch.tensor(values, device="cuda").to(TORCH[dtype])[:, None].expand(-1, ld).contiguous()[:, :cols]
    beta = torch.from_numpy(np.linspace(-1, 1, cols).astype(np.float32)).cuda()
    gamma = torch.full((cols,), 1.5, device="cuda")
    y, mean, rstd = torch.empty(len(values), ld, dtype=TORCH[dtype], device="cuda"), *(torch.empty(len(values), device="cuda") for _ in range(2))
    buf = torch.empty(api.mx_bytes(len(values), cols, mx.B32), dtype=torch.uint8, device="cuda") if packed else None
    d = api.norm_desc(len(values), cols, dtype, ldx=ld, ldy=ld)
    assert api.fh_layer_norm(d, x, gamma, beta, y, mean, rstd, buf, api.mx_params() if packed else None) == api.FH_OK
    assert mean.tolist() == values
    assert torch.equal(y[:, :cols], beta.to(TORCH[dtype]).expand(len(values), -1))
    # eps = rn(1e-5), its root's reciprocal and one rounding
    want = 1 / np.sqrt(float(np.float32(1e-5)))
    assert (np.abs(rstd.double().cpu().numpy() - want) <= 2.0 ** -23 * want).all()


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("cols", [1, 3, 33, 127, 255, 1000, 4095, 8191, 16385, 28671])
def test_the_mean_of_an_exact_sum_is_rounded_once(cols, dtype):
    """Whole numbers of up to eight bits: their sums are exact in any order.  (A quotient by fewer than 2^15 columns is never so near to the
    middle of two fp32 numbers that rounding it by way of 64 bits would differ.)"""
    rows = 64
    x = np.random.default_rng(cols).integers(-255, 256, size=(rows, cols)).astype(np.float32)
    t, mean = torch.from_numpy(x).cuda().to(TORCH[dtype]), torch.empty(rows, device="cuda")
    assert api.fh_layer_norm(api.norm_desc(rows, cols, dtype), t, None, None, torch.empty_like(t), mean) == api.FH_OK
    assert np.array_equal(mean.cpu().numpy(), (x.astype(np.float64).sum(axis=1) / cols).astype(np.float32))


def test_a_sum_beyond_fp32():
    """An infinite sum: the mean is what it was, y has no value."""
    x = torch.full((2, 40), 3e38, device="cuda")
    x[1] = -3e38
    y, mean = torch.empty_like(x), torch.empty(2, device="cuda")
    assert api.fh_layer_norm(api.norm_desc(2, 40), x, None, None, y, mean) == api.FH_OK
    assert mean.tolist() == [float("inf"), float("-inf")] and not torch.isfinite(y).any()
