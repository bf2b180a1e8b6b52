"""Layer norm of more rows than the device works on at once, so that every team takes several: the rings, the reductions' places and the four
rows whose codes are written together come round.  Against the formulas in 64 bits, on the device; containers against those of the dense output."""
import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
TORCH = {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16}
U = 2.0 ** -24                                   # half a step of fp32
HALF = {api.FH_F32: U, api.FH_BF16: 2.0 ** -8}   # half a step of a result


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def inputs(rows, cols, dtype, ldx, ldy, seed):
    """x and dy as slices of wider matrices of NaN, the weights in fp32."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    def apart(t, ld):
        wide = torch.full((rows, ld), float("nan"), dtype=TORCH[dtype], device="cuda")
        wide[:, :cols] = t
        return wide[:, :cols]

    x = apart(normal(rows, cols) * torch.exp(0.5 * normal(cols)) + 0.7, ldx)
    return x, apart(normal(rows, cols), ldy), 1 + 0.3 * normal(cols), 0.3 * normal(cols)


def adds(cols):
    """Additions one after the other in a sum over a row, at most: a lane's own, then five and eight across lanes and warps."""
    return cols / 32 + 16


def norm(x, gamma, beta, eps):
    x = x.double()
    mean = x.mean(dim=1)
    rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(dim=1) + eps)
    return (x - mean[:, None]) * rstd[:, None] * gamma.double() + beta.double(), mean, rstd


def check_forward(x, gamma, beta, y, mean, rstd, dtype):
    cols = x.shape[1]
    want, wmean, wrstd = norm(x, gamma, beta, 1e-5)
    emean = (adds(cols) + 2) * U * x.double().abs().mean(dim=1)
    evar = (adds(cols) + 6) * U + (emean * wrstd) ** 2
    ey = want.abs() * (evar + 6 * U)[:, None] + (emean * wrstd)[:, None] * gamma.double().abs() + 2 * U * beta.double().abs() * (1 + evar[:, None])
    ey += HALF[dtype] * (want.abs() + ey)
    assert bool(((mean.double() - wmean).abs() <= emean).all()) and bool(((rstd.double() - wrstd).abs() <= wrstd * (evar + 4 * U)).all())
    assert bool(((y.double() - want).abs() <= ey).all())


def check_backward(x, dy, gamma, mean, rstd, dx, dgamma, dbeta, dtype):
    rows, cols = dy.shape
    x, dy, mean, rstd, gamma = (t.double() for t in (x, dy, mean[:, None], rstd[:, None], gamma))
    xhat, g = (x - mean) * rstd, dy * gamma
    m1, m2 = g.mean(dim=1, keepdim=True), (g * xhat).mean(dim=1, keepdim=True)
    want = rstd * (g - m1 - xhat * m2)
    n = adds(cols) + 6
    b1, b2 = g.abs().mean(dim=1, keepdim=True), (g * xhat).abs().mean(dim=1, keepdim=True)
    e = rstd * (8 * U * (g.abs() + b1 + xhat.abs() * b2) + n * U * b1 + xhat.abs() * n * U * b2)
    assert bool(((dx.double() - want).abs() <= e + HALF[dtype] * (want.abs() + e)).all())
    for got, w, size in ((dgamma, (dy * xhat).sum(dim=0), (dy * xhat).abs()), (dbeta, dy.sum(dim=0), dy.abs())):
        e = (rows + 44) * U * size.sum(dim=0)
        assert bool(((got.double() - w).abs() <= e + U * (w.abs() + e)).all())


# rows and columns: for each number of threads that share a row, and of vectors to a thread, three rows or more to a team and an uneven
# split; the last two are read again for every sweep
FORWARD = [(20011, 200), (15007, 400), (15011, 900), (5003, 2047), (3001, 4095), (2503, 8191), (2507, 8200), (2501, 16384)]
BACKWARD = [(20011, 200), (6007, 900), (5003, 2047), (5001, 4095), (2503, 8191), (1003, 12011), (707, 20000)]


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("rows,cols", FORWARD)
def test_forward(rows, cols, dtype, off):
    ld = (cols + 7) // 8 * 8 + off                    # on the 16-byte grid, and off it
    x, _, gamma, beta = inputs(rows, cols, dtype, ld, ld, 1)
    d = api.norm_desc(rows, cols, dtype, ldx=ld, ldy=ld)
    wide = torch.full((rows + 1, ld), 7.0, dtype=TORCH[dtype], device="cuda")
    y, mean, rstd = wide[:rows, :cols], torch.full((rows + 8,), 7.0, device="cuda"), torch.full((rows + 8,), 7.0, device="cuda")
    assert api.fh_layer_norm(d, x, gamma, beta, y, mean, rstd) == api.FH_OK
    check_forward(x, gamma, beta, y, mean[:rows], rstd[:rows], dtype)
    assert bool((mean[rows:] == 7).all()) and bool((rstd[rows:] == 7).all()) and bool((wide[:, cols:] == 7).all()) and bool((wide[rows] == 7).all())
    # into containers: the bytes that compressing y gives, and y itself as it was
    for fmt, exponent in ((mx.B32, 0), (mx.B16, -2)):
        p, n = api.mx_params(fmt, exponent), api.mx_bytes(rows, cols, fmt)
        bufs = [torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(3)]
        again = torch.zeros(rows, ld, dtype=TORCH[dtype], device="cuda")[:, :cols]
        assert api.fh_layer_norm(d, x, gamma, beta, again, packed=bufs[0][:n], params=p) == api.FH_OK
        assert api.fh_layer_norm(d, x, gamma, beta, None, packed=bufs[1][:n], params=p) == api.FH_OK
        check_forward(x, gamma, beta, again, mean[:rows], rstd[:rows], dtype)
        assert api.fh_mx_compress(api.matrix(rows, cols, dtype, ld), p, again, bufs[2][:n]) == api.FH_OK
        assert torch.equal(bufs[0], bufs[2]) and torch.equal(bufs[1], bufs[2]) and bool((bufs[2][n:] == 0xA5).all())
    # in place
    assert api.fh_layer_norm(d, x, gamma, beta, x) == api.FH_OK and torch.equal(x, y)


@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("packed", [None, mx.B32, mx.B16])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("rows,cols", BACKWARD)
def test_backward(rows, cols, dtype, packed, off):
    ld = (cols + 7) // 8 * 8 + off
    x, dy, gamma, _ = inputs(rows, cols, dtype, ld, ld, 2)
    _, mean, rstd = norm(x, gamma, gamma, 1e-5)
    mean, rstd, source = mean.float(), rstd.float(), x
    if packed is not None:
        source, values = torch.empty(api.mx_bytes(rows, cols, packed), dtype=torch.uint8, device="cuda"), torch.empty(rows, cols, device="cuda")
        assert api.fh_mx_compress(api.matrix(rows, cols, dtype, ld), api.mx_params(packed, -3 if packed == mx.B16 else 0), x, source) == api.FH_OK
        assert api.fh_mx_decompress(source, api.matrix(rows, cols), packed, values) == api.FH_OK
        x = values
    d = api.norm_desc(rows, cols, dtype, ldx=ld, ldy=ld)
    wide, work = torch.full((rows + 1, ld), 7.0, dtype=TORCH[dtype], device="cuda"), torch.full((api.norm_work_bytes(d),), 0x7F, dtype=torch.uint8, device="cuda")
    dx, dgamma, dbeta = wide[:rows, :cols], torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    status = torch.full((1,), 9, dtype=torch.int64, device="cuda")
    assert api.fh_layer_norm_backward(d, dy, source, gamma, mean, rstd, dx, dgamma, dbeta, work, packed, status) == api.FH_OK
    assert int(status.item()) == api.FH_OK
    check_backward(x, dy, gamma, mean, rstd, dx, dgamma, dbeta, dtype)
    assert bool((wide[:, cols:] == 7).all()) and bool((wide[rows] == 7).all())
    # without the input's gradient, and without the weights': the same bits; over dy
    two, three = torch.empty_like(dgamma), torch.empty_like(dbeta)
    assert api.fh_layer_norm_backward(d, dy, source, gamma, mean, rstd, None, two, three, work, packed) == api.FH_OK
    assert torch.equal(two, dgamma) and torch.equal(three, dbeta)
    assert api.fh_layer_norm_backward(d, dy, source, gamma, mean, rstd, dy, packed=packed) == api.FH_OK and torch.equal(dy, dx)
