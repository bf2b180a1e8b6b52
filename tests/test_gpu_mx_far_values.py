"""Values far beyond what a scale of blocks of 16 holds: they are stored as the largest code with their own sign."""
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


@pytest.mark.parametrize("rounding", [0, 1])
@pytest.mark.parametrize("fmt,exponent", [(mx.B16, e) for e in (0, -12, -40, -64, 64)] + [(mx.B32, 0)])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
def test_every_binade_beyond_the_largest_code(dtype, fmt, exponent, rounding):
    """Blocks of one binade each, of both signs and four mantissas, from within the range up to the largest fp32 number; and blocks that mix
    a far value with near ones."""
    rows = []
    for e in range(max(exponent + 5, -126), 128):
        v = np.array([1.0, 1.25, 1.75, 1.9921875]) * 2.0 ** e
        rows.append(np.concatenate([-v, v, -v, v] * 2))
        rows.append(np.concatenate([[-v[3]], np.linspace(-6, 6, 15) * 2.0 ** exponent, [v[0]], np.linspace(-2688, 2688, 15) * 2.0 ** exponent]))
    t = torch.from_numpy(np.array(rows).astype(np.float32)).cuda()
    t = t if dtype == api.FH_F32 else t.to(torch.bfloat16)
    x = t.float().cpu().numpy()
    kw = dict(rounding=rounding, seed=5, tensor_id=6)
    bufs = [torch.empty(api.mx_bytes(*s, fmt), dtype=torch.uint8, device="cuda") for s in (x.shape, x.T.shape)]
    assert api.fh_mx_compress(api.matrix(*x.shape, dtype), api.mx_params(fmt, exponent, **kw), t, *bufs) == api.FH_OK
    for buf, a in zip(bufs, (x, x.T)):
        assert np.array_equal(buf.cpu().numpy(), mx.compress(a, fmt, exponent, **kw))
