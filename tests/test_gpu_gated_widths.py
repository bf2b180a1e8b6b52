"""The gated block's backward pass on rows of any width: gradients' codes put together in shared memory, byte by byte, or in whole pieces."""
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


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("extra", [0, 1])
@pytest.mark.parametrize("width", [8, 24, 511, 513, 4104, 8191, 8200, 15001, 15360, 15361, 15368, 16001, 20001, 20470, 25001, 25000, 33000, 40001])
def test_any_width(width, extra, dtype):
    """relu, whose products are one rounding from the formula's, then one for the type."""
    t, half = (torch.float32, 2.0 ** -24) if dtype == api.FH_F32 else (torch.bfloat16, 2.0 ** -8)
    rows, ldh, ldp = 3, width + extra, 2 * width + extra
    g = torch.Generator(device="cuda")
    g.manual_seed(width)
    pre, dh = (torch.randn(rows, ld, device="cuda", generator=g).to(t) for ld in (ldp, ldh))
    out = torch.full((rows, ldp), 7.0, dtype=t, device="cuda")
    n = api.i8_bytes(rows, 2 * width)
    both, alone = (torch.full((n + 32,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2))
    d = api.gated_desc(rows, width, 1, api.FH_RELU, dtype, ldh, ldp)
    x, y, z = pre[:, :2 * width], dh[:, :width], out[:, :2 * width]
    assert api.fh_gated_backward(d, y, x, z, both[:n]) == api.FH_OK
    assert api.fh_gated_backward(d, y, x, None, alone[:n]) == api.FH_OK
    torch.cuda.synchronize()
    got, p, q = (v.double().cpu().numpy() for v in (z, x, y))
    want = i8.gated_backward(q, p[:, :width], p[:, width:], i8.RELU)
    assert (np.abs(got - want) <= (2.0 ** -24 + half * (1 + 1e-6)) * np.abs(want)).all()
    assert (out[:, 2 * width:] == 7.0).all() and (both[n:] == 0xA5).all() and torch.equal(both, alone)
    assert np.array_equal(both[:n].cpu().numpy(), i8.compress(got.astype(np.float32)))
