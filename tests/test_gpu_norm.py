"""Layer norm on the GPU, forward into dense and 4-bit outputs and backward from dense and 4-bit inputs, against the formulas in 64 bits;
and a linear block's training step of all the operators on 4-bit matrices together."""
import numpy as np
import pytest

from oracle import mx
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24                                   # half a step of fp32
TORCH = {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16}
HALF = {api.FH_F32: U, api.FH_BF16: 2.0 ** -8}   # half a step of a result


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def held(a, dtype):
    """(on the GPU in `dtype`, the values it holds in 64 bits)."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32)).cuda().to(TORCH[dtype])
    return t, t.double().cpu().numpy()


def apart(t, ld, offset=0):
    """The matrix at rows `ld` apart in a buffer of sevens."""
    rows, cols = t.shape
    flat = torch.full((offset + rows * ld + 64,), 7.0, dtype=t.dtype, device="cuda")
    view = flat.as_strided((rows, cols), (ld, 1), offset)
    view.copy_(t)
    return flat, view


def around(flat, view):
    keep = view.clone()
    view.fill_(7.0)
    ok = bool((flat == 7.0).all())
    view.copy_(keep)
    return ok


def num(t):
    return t.double().cpu().numpy()


def adds(cols):
    """Additions one after the other in a sum over a row, at most: a lane's own, then five and eight across lanes and warps, and the
    rounding of the factor 1 / cols."""
    return cols / 32 + 16


def forward_bounds(x, y, gamma, beta, rstd, cols, dtype):
    # the mean is off by its additions, relative to the mean magnitude; the variance by its own, twice the rounding of the
    # distances, and the square of the mean's error; rstd by half of that
    emean = (adds(cols) + 2) * U * np.abs(x).mean(axis=1)
    evar = (adds(cols) + 6) * U + (emean * rstd) ** 2
    scale = 1.0 if gamma is None else np.abs(gamma)
    ey = np.abs(y) * (evar + 6 * U)[:, None] + (emean * rstd)[:, None] * scale + 2 * U * (0.0 if beta is None else np.abs(beta)) * (1 + evar[:, None])
    return emean, rstd * (evar + 4 * U), ey + HALF[dtype] * (np.abs(y) + ey)


SHAPES = [(1, 1), (3, 7), (5, 32), (9, 100), (130, 64), (40, 256), (33, 257), (17, 1000), (300, 512), (6, 1024), (7, 1025), (20, 2048), (5, 4096), (3, 5000),
          (4, 8192), (2, 8193), (3, 16384), (2, 20000), (2, 28672)]


def inputs(rows, cols, dtype, wdtype, seed=0, affine=True):
    rng = np.random.default_rng([seed, rows, cols])
    x = held(rng.standard_normal((rows, cols)) * np.exp(0.5 * rng.standard_normal(cols)) + 0.7, dtype)
    gamma = held(1 + 0.3 * rng.standard_normal(cols), wdtype) if affine else (None, None)
    beta = held(0.3 * rng.standard_normal(cols), wdtype) if affine else (None, None)
    return x, gamma, beta, held(rng.standard_normal((rows, cols)), dtype)


@pytest.mark.parametrize("dtype,wdtype,affine", [(api.FH_F32, api.FH_F32, True), (api.FH_BF16, api.FH_F32, True), (api.FH_BF16, api.FH_BF16, True),
                                                 (api.FH_F32, api.FH_BF16, True), (api.FH_F32, api.FH_F32, False)])
@pytest.mark.parametrize("shape", SHAPES)
def test_forward(shape, dtype, wdtype, affine):
    rows, cols = shape
    (tx, x), (tg, g), (tb, b), _ = inputs(rows, cols, dtype, wdtype, 1, affine)
    want, mean, rstd = mx.layer_norm(x, g, b, 1e-5)
    flat, y = apart(torch.zeros_like(tx), cols)
    tmean, trstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    assert api.fh_layer_norm(api.norm_desc(rows, cols, dtype, wdtype, 1e-5), tx, tg, tb, y, tmean, trstd) == api.FH_OK
    emean, erstd, ey = forward_bounds(x, want, g, b, rstd, cols, dtype)
    assert (np.abs(num(tmean) - mean) <= emean).all() and (np.abs(num(trstd) - rstd) <= erstd).all()
    assert (np.abs(num(y) - want) <= ey).all()
    assert around(flat, y)


@pytest.mark.parametrize("fmt,exponent", [(mx.B32, 0), (mx.B16, 0), (mx.B16, -4)])
@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("shape", SHAPES)
def test_the_packed_output_is_what_compressing_the_dense_one_gives(shape, dtype, fmt, exponent):
    rows, cols = shape
    (tx, _), (tg, _), (tb, _), _ = inputs(rows, cols, dtype, api.FH_F32, 2)
    d, p = api.norm_desc(rows, cols, dtype), api.mx_params(fmt, exponent, tensor_id=77)
    n = api.mx_bytes(rows, cols, fmt)
    packed = [torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(3)]
    y = torch.empty_like(tx)
    assert api.fh_layer_norm(d, tx, tg, tb, y, packed=packed[0][:n], params=p) == api.FH_OK
    assert api.fh_layer_norm(d, tx, tg, tb, None, packed=packed[1][:n], params=p) == api.FH_OK
    assert api.fh_mx_compress(api.matrix(rows, cols, dtype), p, y, packed[2][:n]) == api.FH_OK
    for t in packed:
        assert torch.equal(t, packed[2]) and (t[n:] == 0xA5).all()


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("cols,ldx,ldy,offset", [(100, 101, 104, 0), (100, 104, 103, 0), (1000, 1008, 1016, 1), (1000, 1008, 1016, 8), (1001, 1008, 1008, 0),
                                                 (8200, 8208, 8201, 0)])
def test_strides_alignments_and_in_place(cols, ldx, ldy, offset, dtype):
    rows = 37
    (tx, x), (tg, g), (tb, b), (tdy, dy) = inputs(rows, cols, dtype, api.FH_F32, 3)
    d = api.norm_desc(rows, cols, dtype, api.FH_F32, 1e-5, ldx, ldy)
    want, mean, rstd = mx.layer_norm(x, g, b, 1e-5)
    _, _, ey = forward_bounds(x, want, g, b, rstd, cols, dtype)
    _, vx = apart(tx, ldx, offset)
    flat, vy = apart(torch.zeros_like(tx), ldy, offset)
    tmean, trstd = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    assert api.fh_layer_norm(d, vx, tg, tb, vy, tmean, trstd) == api.FH_OK
    assert (np.abs(num(vy) - want) <= ey).all() and around(flat, vy)
    fdx, vdx = apart(torch.zeros_like(tx), ldx, offset)
    _, vdy = apart(tdy, ldy, offset)
    work = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda")
    dgamma, dbeta = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    assert api.fh_layer_norm_backward(d, vdy, vx, tg, tmean, trstd, vdx, dgamma, dbeta, work) == api.FH_OK
    check_backward(num(vdx), num(dgamma), num(dbeta), dy, x, g, num(tmean), num(trstd), dtype, api.FH_F32)
    assert around(fdx, vdx)
    # in place: y over x, dx over dy, dx over x (of equal strides): what the same call gives out of place
    d = api.norm_desc(rows, cols, dtype, api.FH_F32, 1e-5, ldx, ldx)
    (_, vdy), (_, vdx), (_, vy) = apart(tdy, ldx, offset), apart(torch.zeros_like(tx), ldx, offset), apart(torch.zeros_like(tx), ldx, offset)
    assert api.fh_layer_norm_backward(d, vdy, vx, tg, tmean, trstd, vdx) == api.FH_OK and api.fh_layer_norm(d, vx, tg, tb, vy) == api.FH_OK
    check_backward(num(vdx), None, None, dy, x, g, num(tmean), num(trstd), dtype, api.FH_F32)
    _, over = apart(tx, ldx, offset)
    assert api.fh_layer_norm_backward(d, vdy, over, tg, tmean, trstd, over) == api.FH_OK and torch.equal(over, vdx)
    assert api.fh_layer_norm_backward(d, vdy, vx, tg, tmean, trstd, vdy) == api.FH_OK and torch.equal(vdy, vdx)
    assert api.fh_layer_norm(d, vx, tg, tb, vx) == api.FH_OK and torch.equal(vx, vy)


def check_backward(dx, dgamma, dbeta, dy, x, g, mean, rstd, dtype, wdtype):
    rows, cols = dy.shape
    want = mx.layer_norm_backward(dy, x, g, mean, rstd)
    xhat = np.abs((x - mean[:, None]) * rstd[:, None])
    gg = np.abs(dy * (1.0 if g is None else g))
    n = adds(cols) + 6                                  # (four more roundings in a product and its factors, two in the factor 1 / cols)
    e1, e2 = n * U * gg.mean(axis=1), n * U * (gg * xhat).mean(axis=1)
    m1, m2 = gg.mean(axis=1), (gg * xhat).mean(axis=1)  # (bounds of the means' magnitudes)
    edx = rstd[:, None] * (8 * U * (gg + m1[:, None] + xhat * m2[:, None]) + e1[:, None] + xhat * e2[:, None])
    # (results near the smallest normal numbers do not occur here)
    if dx is not None:
        assert (np.abs(dx - want[0]) <= edx + HALF[dtype] * (np.abs(want[0]) + edx)).all()
    # a column's sum: at most rows + 40 additions, in teams, CTAs and the last kernel
    for got, w, size in ((dgamma, want[1], np.abs(dy) * xhat), (dbeta, want[2], np.abs(dy))):
        if got is not None:
            e = (rows + 44) * U * size.sum(axis=0)
            assert (np.abs(got - w) <= e + HALF[wdtype] * (np.abs(w) + e)).all()


@pytest.mark.parametrize("dtype,wdtype,affine", [(api.FH_F32, api.FH_F32, True), (api.FH_BF16, api.FH_F32, True), (api.FH_BF16, api.FH_BF16, True),
                                                 (api.FH_F32, api.FH_BF16, False)])
@pytest.mark.parametrize("packed", [None, mx.B32, mx.B16])
@pytest.mark.parametrize("shape", SHAPES + [(700, 96), (1500, 1300)])
def test_backward(shape, packed, dtype, wdtype, affine):
    rows, cols = shape
    (tx, x), (tg, g), _, (tdy, dy) = inputs(rows, cols, dtype, wdtype, 4, affine)
    _, mean, rstd = mx.layer_norm(x, None, None, 1e-5)
    (tmean, mean), (trstd, rstd) = held(mean, api.FH_F32), held(rstd, api.FH_F32)
    if packed is not None:
        buf = mx.compress(x, packed, -3 if packed == mx.B16 else 0)
        x, tx = mx.restore(buf, rows, cols, packed), torch.from_numpy(buf).cuda()
    d = api.norm_desc(rows, cols, dtype, wdtype)
    fdx, dx = apart(torch.zeros_like(tdy), cols)
    dgamma, dbeta = (torch.full((cols + 8,), 7.0, dtype=TORCH[wdtype], device="cuda") for _ in range(2))
    n = api.norm_work_bytes(d)
    work, status = torch.full((n + 64,), 0x7F, dtype=torch.uint8, device="cuda"), torch.full((1,), 9, dtype=torch.int64, device="cuda")
    args = (d, tdy, tx, tg, tmean, trstd)
    assert api.fh_layer_norm_backward(*args, dx, dgamma, dbeta, work[:n], packed, status) == api.FH_OK
    assert int(status.item()) == api.FH_OK
    check_backward(num(dx), num(dgamma[:cols]), num(dbeta[:cols]), dy, x, g, mean, rstd, dtype, wdtype)
    assert (dgamma[cols:] == 7).all() and (dbeta[cols:] == 7).all() and (work[n:] == 0x7F).all() and around(fdx, dx)
    # each output alone, bit for bit
    one, two, three = torch.empty_like(dx), torch.empty_like(dgamma), torch.empty_like(dbeta)
    assert api.fh_layer_norm_backward(*args, one, packed=packed) == api.FH_OK and torch.equal(one, dx)
    assert api.fh_layer_norm_backward(*args, None, two, None, work, packed) == api.FH_OK and torch.equal(two[:cols], dgamma[:cols])
    assert api.fh_layer_norm_backward(*args, None, None, three, work, packed) == api.FH_OK and torch.equal(three[:cols], dbeta[:cols])


def test_constant_far_and_non_finite_rows():
    x = np.zeros((6, 300), dtype=np.float32)
    x[0] = 5.0
    x[1] = 1000.0 + np.random.default_rng(1).standard_normal(300) * 0.01
    x[2, 7], x[3, 8] = np.nan, np.inf
    x[4] = np.linspace(-1, 1, 300) * 1e18
    x[5, 3] = 1e-20
    tx, x = held(x, api.FH_F32)
    y, mean, rstd = torch.empty_like(tx), torch.empty(6, device="cuda"), torch.empty(6, device="cuda")
    packed = torch.empty(api.mx_bytes(6, 300, mx.B32), dtype=torch.uint8, device="cuda")
    assert api.fh_layer_norm(api.norm_desc(6, 300), tx, None, None, y, mean, rstd, packed, api.mx_params()) == api.FH_OK
    fine = [0, 1, 4, 5]
    want, wmean, wrstd = mx.layer_norm(x[fine], None, None, 1e-5)
    emean, erstd, ey = forward_bounds(x[fine], want, None, None, wrstd, 300, api.FH_F32)
    assert (np.abs(num(mean)[fine] - wmean) <= emean).all() and (np.abs(num(rstd)[fine] - wrstd) <= erstd).all()
    assert (np.abs(num(y)[fine] - want) <= ey).all() and torch.isnan(y[2:4]).all()
    assert np.array_equal(packed.cpu().numpy(), mx.compress(y.cpu().numpy(), mx.B32))


@pytest.mark.parametrize("change", [0, 8, 12, None])
def test_another_header_is_reported_and_nothing_written(change):
    (_, x), (tg, _), _, (tdy, _) = inputs(20, 300, api.FH_F32, api.FH_F32, 5)
    buf = torch.from_numpy(mx.compress(x, mx.B32)).cuda()
    if change is None:
        buf = buf[:-16]
    else:
        buf[change] += 1
    d = api.norm_desc(20, 300)
    mean, dx, dgamma, dbeta = torch.ones(20, device="cuda"), *(torch.full(s, 7.0, device="cuda") for s in ((20, 300), (300,), (300,)))
    work, status = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int64, device="cuda")
    assert api.fh_layer_norm_backward(d, tdy, buf, tg, mean, mean, dx, dgamma, dbeta, work, mx.B32, status) == api.FH_OK
    assert int(status.item()) == api.FH_ERR_CORRUPT and (dx == 7).all() and (dgamma == 7).all() and (dbeta == 7).all()


def test_gradients_against_differences():
    """dx, dgamma and dbeta of sum(dy * y) against central differences of the forward kernel, summed in 64 bits."""
    rows, cols = 3, 40
    (tx, x), (tg, g), (tb, b), (tdy, dy) = inputs(rows, cols, api.FH_F32, api.FH_F32, 6)
    d = api.norm_desc(rows, cols)
    y, mean, rstd = torch.empty_like(tx), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    assert api.fh_layer_norm(d, tx, tg, tb, y, mean, rstd) == api.FH_OK
    dx, dgamma, dbeta = torch.empty_like(tx), torch.empty_like(tg), torch.empty_like(tb)
    work = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda")
    assert api.fh_layer_norm_backward(d, tdy, tx, tg, mean, rstd, dx, dgamma, dbeta, work) == api.FH_OK
    h = 2.0 ** -7

    def loss():
        assert api.fh_layer_norm(d, tx, tg, tb, y) == api.FH_OK
        return float((tdy.double() * y.double()).sum())

    # the forward kernel's outputs, 120 of magnitude below 8, are off by at most 40 U each times |dy| < 4: a difference by 2 * 120 * 8 * 4 *
    # 40 U / (2 h) < 1.2, were the errors all of one sign; the step's own error is h^2 / 6 times a third derivative.  Errors of random sign
    # leave a sixteenth of that at ten standard deviations
    for t, grad in ((tx, dx), (tg, dgamma), (tb, dbeta)):
        flat, gr = t.view(-1), grad.view(-1)
        for i in range(0, flat.numel(), 7):
            keep = float(flat[i])
            flat[i] = keep + h
            up = loss()
            hi = float(flat[i])
            flat[i] = keep - h
            down = loss()
            lo = float(flat[i])
            flat[i] = keep
            assert abs((up - down) / (hi - lo) - float(gr[i])) < 0.075


def test_captured_backward_on_two_streams_at_once():
    """Graphs of forward and backward pass on two streams, replayed side by side with a workspace each."""
    runs = []
    for seed in (7, 8):
        (tx, x), (tg, g), (tb, _), (tdy, dy) = inputs(900, 700, api.FH_BF16, api.FH_F32, seed)
        d = api.norm_desc(900, 700, api.FH_BF16)
        y, mean, rstd, dx, dgamma, dbeta = torch.empty_like(tx), *(torch.empty(900, device="cuda") for _ in range(2)), torch.empty_like(tx), \
            torch.empty_like(tg), torch.empty_like(tb)
        work = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda")
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            assert api.fh_layer_norm(d, tx, tg, tb, y, mean, rstd) == api.FH_OK
            assert api.fh_layer_norm_backward(d, tdy, tx, tg, mean, rstd, dx, dgamma, dbeta, work) == api.FH_OK
        runs.append((stream, graph, (tx, tg, tb, tdy, y, work), dx, dgamma, dbeta, dy, x, g, mean, rstd))
    for _ in range(3):
        for stream, graph, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, _, dx, dgamma, dbeta, dy, x, g, mean, rstd in runs:
        check_backward(num(dx), num(dgamma), num(dbeta), dy, x, g, num(mean), num(rstd), api.FH_BF16, api.FH_F32)


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("tokens", [1, 77, 256])
def test_a_linear_block_trains_on_what_it_kept_in_4_bits(tokens, fmt):
    """y = norm(x) in 4 bits, z = y W^T, and back: what is kept between the passes is x and y in 4 bits.  Every step against the plain
    definition of that step on the inputs it got."""
    width, out, bf = 320, 200, api.FH_BF16
    (tx, x), (tg, g), (tb, b), _ = inputs(tokens, width, bf, bf, 9)
    rng = np.random.default_rng(10)
    (tw, w), (tdz, dz) = held(rng.standard_normal((out, width)) * 0.05, bf), held(rng.standard_normal((tokens, out)) * 0.01, bf)
    ew, edz = (-6, -8) if fmt == mx.B16 else (0, 0)

    def room(rows, cols):
        return torch.empty(api.mx_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda")

    def values(buf, rows, cols):
        return mx.restore(buf.cpu().numpy(), rows, cols, fmt)

    def agree(got, want, size, k, dtype):
        assert (np.abs(num(got) - want) <= (k + 8) * 2.0 ** -23 * size + HALF[dtype] * np.abs(want)).all()

    w_rows, w_cols = room(out, width), room(width, out)
    assert api.fh_mx_compress(api.matrix(out, width, bf), api.mx_params(fmt, ew), tw, w_rows, w_cols) == api.FH_OK
    # forward
    d = api.norm_desc(tokens, width, bf, bf)
    y, mean, rstd, y_rows = torch.empty_like(tx), torch.empty(tokens, device="cuda"), torch.empty(tokens, device="cuda"), room(tokens, width)
    assert api.fh_layer_norm(d, tx, tg, tb, y, mean, rstd, y_rows, api.mx_params(fmt)) == api.FH_OK
    x_kept, y_kept = room(tokens, width), room(width, tokens)
    assert api.fh_mx_compress(api.matrix(tokens, width, bf), api.mx_params(fmt), tx, x_kept) == api.FH_OK
    assert api.fh_mx_compress(api.matrix(tokens, width, bf), api.mx_params(fmt), y, None, y_kept) == api.FH_OK
    z = torch.empty(tokens, out, dtype=torch.bfloat16, device="cuda")
    assert api.fh_mx_product(api.mx_product_desc(tokens, out, width, fmt, bf), y_rows, w_rows, z) == api.FH_OK
    want, _, wrstd = mx.layer_norm(x, g, b, 1e-5)
    assert (np.abs(num(y) - want) <= forward_bounds(x, want, g, b, wrstd, width, bf)[2]).all()
    yv, wv = values(y_rows, tokens, width), values(w_rows, out, width)
    assert np.array_equal(yv, mx.restore(mx.compress(num(y), fmt), tokens, width, fmt)) and np.array_equal(wv, mx.restore(mx.compress(w, fmt, ew), out, width, fmt))
    agree(z, yv @ wv.T, np.abs(yv) @ np.abs(wv).T, width, bf)
    # backward: the gradient by rows and by columns, at random
    dz_rows, dz_cols = room(tokens, out), room(out, tokens)
    p = api.mx_params(fmt, edz, 1, seed=5, tensor_id=6)
    assert api.fh_mx_compress(api.matrix(tokens, out, bf), p, tdz, dz_rows, dz_cols) == api.FH_OK
    dy, dw = torch.empty_like(tx), torch.ones(out, width, device="cuda")
    assert api.fh_mx_product(api.mx_product_desc(tokens, width, out, fmt, bf), dz_rows, w_cols, dy) == api.FH_OK
    assert api.fh_mx_product(api.mx_product_desc(out, width, tokens, fmt, accumulate=True), dz_cols, y_kept, dw) == api.FH_OK
    a, c = values(dz_rows, tokens, out), values(w_cols, width, out)
    assert np.array_equal(a, mx.restore(mx.compress(dz, fmt, edz, 1, 5, 6), tokens, out, fmt))
    agree(dy, a @ c.T, np.abs(a) @ np.abs(c).T, out, bf)
    a, c = values(dz_cols, out, tokens), values(y_kept, width, tokens)
    agree(dw, 1 + a @ c.T, 1 + np.abs(a) @ np.abs(c).T, tokens, api.FH_F32)
    dx, dgamma, dbeta = torch.empty_like(tx), torch.empty_like(tg), torch.empty_like(tb)
    work = torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda")
    assert api.fh_layer_norm_backward(d, dy, x_kept, tg, mean, rstd, dx, dgamma, dbeta, work, fmt) == api.FH_OK
    check_backward(num(dx), num(dgamma), num(dbeta), num(dy), values(x_kept, tokens, width), g, num(mean), num(rstd), bf, bf)
