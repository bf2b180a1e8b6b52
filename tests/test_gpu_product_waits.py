"""Products whose waits run out: the status says so, nothing beyond C is written, and the library goes on as before.  The failure is made on
the host: a short limit of the waits, and a stage that is not loaded."""
import numpy as np
import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


@pytest.fixture
def limits():
    """Sets (limit, silent stage); the defaults come back at the end."""
    def put(polls, silent):
        assert api.debug_set(api.FH_DEBUG_WAIT_POLLS, polls) == api.FH_OK
        assert api.debug_set(api.FH_DEBUG_SILENT_TILE, silent) == api.FH_OK
    yield put
    put(1 << 22, 2 ** 64 - 1)


def operand(rows, k, fmt, seed):
    x = np.random.default_rng([seed, rows, k]).integers(-6, 7, size=(rows, k)).astype(np.float32)
    x[:, ::mx.BLOCK[fmt]] = 6.0
    buf = mx.compress(x, fmt)
    return torch.from_numpy(buf).cuda(), mx.restore(buf, rows, k, fmt)


# one row; a cluster of parts; few tiles of pairs, their parts in one cluster; several tiles to a pair
SHAPES = [(1, 200, 512), (40, 300, 8192), (128, 1000, 6000), (300, 260, 9000), (2500, 2700, 2560)]


@pytest.mark.parametrize("polls,silent", [(1, 2 ** 64 - 1), (200, 0), (200, 1), (200, 7)])
@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("shape", SHAPES)
def test_a_wait_that_runs_out(shape, fmt, polls, silent, limits):
    m, n, k = shape
    (a, x), (b, y) = operand(m, k, fmt, 1), operand(n, k, fmt, 2)
    d = api.mx_product_desc(m, n, k, fmt)
    flat, status = torch.full((m * n + 512,), 7.0, device="cuda"), torch.full((1,), 99, dtype=torch.int64, device="cuda")
    limits(polls, silent)
    assert api.fh_mx_product(d, a, b, flat, status) == api.FH_OK
    torch.cuda.synchronize()
    ended = int(status.item())
    assert (flat[m * n:] == 7.0).all()
    want = torch.from_numpy(x).cuda() @ torch.from_numpy(y).cuda().T
    # A stage that nobody loads is never there.  (It is counted in each CTA, whose part may be shorter.)  Sixteen polls may or may not last until a
    # stage is.  Whoever is told OK has the result.
    if silent < 2 or (shape == SHAPES[-1] and silent == 7):
        assert ended == api.FH_ERR_TIMEOUT
    else:
        assert ended in (api.FH_OK, api.FH_ERR_TIMEOUT)
    if ended == api.FH_OK:
        assert torch.equal(flat[:m * n].view(m, n).double(), want)
    # a following call, on the same stream, of the same tensor memory and barriers, is exact: sums of integers below 2^24
    limits(1 << 22, 2 ** 64 - 1)
    assert api.fh_mx_product(d, a, b, flat, status) == api.FH_OK
    torch.cuda.synchronize()
    assert int(status.item()) == api.FH_OK
    assert torch.equal(flat[:m * n].view(m, n).double(), want)
