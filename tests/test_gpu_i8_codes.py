"""Codes of bf16 matrices for every magnitude and every element below it, and matrices on either side of the rules by which kernels are chosen."""
import numpy as np
import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def containers(x, dtype):
    """(by rows, by columns) of fp32 values that the type holds."""
    rows, cols = x.shape
    t = torch.from_numpy(x).cuda().to(torch.float32 if dtype == api.FH_F32 else torch.bfloat16)
    r, c = (torch.full((api.i8_bytes(*s),), 0xA5, dtype=torch.uint8, device="cuda") for s in ((rows, cols), (cols, rows)))
    assert api.fh_i8_compress(api.matrix(rows, cols, dtype), t, r, c) == api.FH_OK
    return r.cpu().numpy(), c.cpu().numpy()


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("exponent", [0, -37, 100, -119, -126])
def test_every_element_below_every_magnitude(exponent, dtype):
    """Rows of magnitude M 2^q for all M of eight bits, with all X 2^(q - e) up to it: X of eight bits and e up to 10, beyond which a quotient is below a
    quarter.  Half of the magnitude, where the quotient is next to 63.5, and M = 254, where quotients are middles exactly, are among them."""
    m = np.arange(128, 256)
    elements = np.array([x * 2.0 ** -e for e in range(11) for x in range(128, 256)])
    x = np.where(elements[None, :] <= m[:, None], elements[None, :], 0.0)
    x[:, ::2] *= -1
    x = np.concatenate([m[:, None], x], axis=1)
    x = (x * 2.0 ** (exponent - 7)).astype(np.float32)              # (below the normal numbers: fewer bits, which bf16 then rounds)
    if dtype == api.FH_BF16:
        x = torch.from_numpy(x).bfloat16().float().numpy()
    by_rows, _ = containers(x, dtype)
    assert np.array_equal(by_rows, i8.compress(x))
    _, by_cols = containers(np.ascontiguousarray(x.T), dtype)
    assert np.array_equal(by_cols, i8.compress(x))


# one kernel or three by columns: 1024 rows; up to 4096 where the device has several CTAs an SM
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("shape", [(1024, 40), (1025, 40), (1100, 9500), (4096, 4800), (4097, 100), (2000, 520)])
def test_either_side_of_the_rules(shape, dtype):
    rng = np.random.default_rng([1, *shape])
    x = (rng.standard_normal(shape) * np.exp(rng.standard_normal((1, shape[1])))).astype(np.float32)
    x[:, shape[1] // 2] = 0
    x[shape[0] // 3, 1] = np.nan
    x[shape[0] - 1, 2] = -np.inf
    x = torch.from_numpy(x).to(torch.float32 if dtype == api.FH_F32 else torch.bfloat16).float().numpy()
    by_rows, by_cols = containers(x, dtype)
    assert np.array_equal(by_rows, i8.compress(x))
    assert np.array_equal(by_cols, i8.compress(np.ascontiguousarray(x.T)))


def test_captured_by_columns_and_replayed_on_smaller_values():
    """The maxima of a replay are its own."""
    x = torch.randn(1500, 200, device="cuda") * 8
    c = torch.empty(api.i8_bytes(200, 1500), dtype=torch.uint8, device="cuda")
    m = api.matrix(1500, 200)
    assert api.fh_i8_compress(m, x, None, c) == api.FH_OK
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        assert api.fh_i8_compress(m, x, None, c) == api.FH_OK
    for scale in (4.0, 0.01):
        x.copy_(torch.randn(1500, 200, device="cuda") * scale)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(c.cpu().numpy(), i8.compress(np.ascontiguousarray(x.cpu().numpy().T)))
