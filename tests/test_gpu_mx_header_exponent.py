"""A container of blocks of 32 has no exponent: another one in its header is refused by every reader."""
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


@pytest.mark.parametrize("exponent", [1, -1, 64])
@pytest.mark.parametrize("rows", [5, 200])
def test_an_exponent_in_a_container_of_blocks_of_32(rows, exponent):
    cols = 300
    x = np.random.default_rng(rows).standard_normal((rows, cols)).astype(np.float32)
    good = torch.from_numpy(mx.compress(x, mx.B32)).cuda()
    bad = good.clone()
    bad[16:20] = torch.from_numpy(np.array([exponent], dtype=np.int32).view(np.uint8)).cuda()
    status = torch.zeros(1, dtype=torch.int64, device="cuda")
    d = api.norm_desc(rows, cols)
    ones, dy = torch.ones(rows, device="cuda"), torch.from_numpy(x).cuda()
    work = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda")
    for buf, want in ((bad, api.FH_ERR_CORRUPT), (good, api.FH_OK)):
        for call in (lambda out: api.fh_mx_decompress(buf, api.matrix(rows, cols), mx.B32, out, status),
                     lambda out: api.fh_mx_product(api.mx_product_desc(rows, rows, cols), buf, good, out, status),
                     lambda out: api.fh_mx_product(api.mx_product_desc(rows, rows, cols), good, buf, out, status),
                     lambda out: api.fh_layer_norm_backward(d, dy, buf, None, ones, ones, out, None, None, None, mx.B32, status),
                     lambda out: api.fh_layer_norm_backward(d, dy, buf, None, ones, ones, None, out, None, work, mx.B32, status)):
            out = torch.full((rows, max(rows, cols)), 7.0, device="cuda")
            assert call(out) == api.FH_OK
            assert int(status.item()) == want
            assert bool((out == 7.0).all()) == (want != api.FH_OK)
