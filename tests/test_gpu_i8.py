"""Matrices in 8 bits, their products and the gated feed-forward block against the plain definition: containers byte for byte, results within what their
roundings allow."""
import numpy as np
import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24                                                       # half a step of fp32, relative
HALF = {api.FH_F32: U, api.FH_BF16: 2.0 ** -8}
TYPES = {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16}


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def values(rows, cols, seed, dtype=api.FH_F32):
    """fp32 values that the type holds, rows of different sizes."""
    rng = np.random.default_rng([seed, rows, cols])
    x = (rng.standard_normal((rows, cols)) * np.exp(2 * rng.standard_normal((rows, 1)))).astype(np.float32)
    return torch.from_numpy(x).to(TYPES[dtype]).float().numpy()


def watched(rows, cols, ld, dtype, offset=0):
    """(the buffer, a matrix in it): everything is 7."""
    flat = torch.full((rows * ld + offset + 128,), 7.0, dtype=TYPES[dtype], device="cuda")
    return flat, flat[offset:].as_strided((rows, cols), (ld, 1), offset)


def read(flat, view):
    """The matrix's values; nothing around it was written."""
    torch.cuda.synchronize()
    got = view.float().cpu().numpy().copy()
    view.fill_(7.0)
    assert (flat == 7.0).all()
    return got


def room(rows, cols):
    """A container's place with a border, full of bytes that nothing may be left of."""
    n = api.i8_bytes(rows, cols)
    buf = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    return buf, buf[:n]


def container(buf, part):
    torch.cuda.synchronize()
    assert (buf[part.numel():] == 0xA5).all()
    return part.cpu().numpy()


SHAPES = [(1, 1), (1, 16), (1, 4096), (2, 33), (3, 5000), (7, 31), (8, 32), (9, 1025), (16, 40000), (40, 70), (129, 300), (1200, 64), (1201, 130), (1300, 2100),
          (300, 9000), (5000, 17), (1190, 4608)]


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("extra,offset", [(0, 0), (8, 0), (1, 3), (2, 2)])
@pytest.mark.parametrize("shape", SHAPES)
def test_containers_and_restored_values(shape, extra, offset, dtype):
    rows, cols = shape
    x = values(rows, cols, 1, dtype)
    flat, view = watched(rows, cols, cols + extra, dtype, offset)
    view.copy_(torch.from_numpy(x))
    (br, r), (bc, c) = room(rows, cols), room(cols, rows)
    m = api.matrix(rows, cols, dtype, cols + extra)
    assert api.fh_i8_compress(m, view, r, c) == api.FH_OK
    by_rows, by_cols = container(br, r), container(bc, c)
    assert np.array_equal(by_rows, i8.compress(x)) and np.array_equal(by_cols, i8.compress(np.ascontiguousarray(x.T)))
    for only in (dict(rows=True), dict(cols=True)):                  # each alone
        b1, p1 = room(rows, cols) if "rows" in only else room(cols, rows)
        assert api.fh_i8_compress(m, view, p1 if "rows" in only else None, p1 if "cols" in only else None) == api.FH_OK
        assert np.array_equal(container(b1, p1), by_rows if "rows" in only else by_cols)
    out, ov = watched(rows, cols, cols + extra, dtype, offset)
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    assert api.fh_i8_decompress(r, m, ov, status) == api.FH_OK
    got = read(out, ov)
    assert int(status.item()) == api.FH_OK
    s = i8.scales(i8.magnitudes(x))[:, None]
    want = torch.from_numpy((i8.quantise(x)[0].astype(np.float32) * s)).to(TYPES[dtype]).float().numpy()
    assert np.array_equal(got, want)


@pytest.mark.parametrize("shape", [(1, 64), (64, 1), (24, 200), (1300, 2100)])
def test_values_at_the_edges(shape):
    """Ties between whole numbers, the smallest and largest numbers, zeros, NaN and infinities."""
    rows, cols = shape
    rng = np.random.default_rng(5)
    x = rng.integers(-254, 255, size=shape).astype(np.float32) * np.float32(0.5)
    x *= np.exp2(rng.integers(-140, 120, size=(rows, 1))).astype(np.float32)
    flat = x.reshape(-1)
    pick = rng.permutation(flat.size)
    for i, v in enumerate([np.nan, np.inf, -np.inf, 1e-45, -1e-45, 3.4028235e38, -0.0, 1.1754944e-38]):
        flat[pick[i * 3 % flat.size]] = v
    x[rows // 2] = 0
    x[0, cols // 2] = 3.0e38
    t = torch.from_numpy(x).cuda()
    (br, r), (bc, c) = room(rows, cols), room(cols, rows)
    assert api.fh_i8_compress(api.matrix(rows, cols), t, r, c) == api.FH_OK
    assert np.array_equal(container(br, r), i8.compress(x)) and np.array_equal(container(bc, c), i8.compress(np.ascontiguousarray(x.T)))
    back = torch.empty_like(t)
    assert api.fh_i8_decompress(r, api.matrix(rows, cols), back) == api.FH_OK
    bad = ~np.isfinite(x).all(axis=1)
    got = back.cpu().numpy()
    assert np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()


def test_near_ties_go_to_the_nearer_whole_number():
    """Elements next to the middle of two codes, to the last place on either side, under scales of 24 bits."""
    rng = np.random.default_rng(6)
    rows, k = 64, rng.integers(-126, 126, size=(64, 160))
    a = (1 + rng.random((rows, 1))).astype(np.float32)
    s = i8.scales(a)
    x = ((k + 0.5) * s.astype(np.float64)).astype(np.float32)
    for i in range(160):
        for _ in range(abs(i % 7 - 3)):
            x[:, i] = np.nextafter(x[:, i], np.float32(9 if i % 7 > 3 else -9))
    x = np.concatenate([a, x], axis=1)
    (br, r), (bc, c) = room(64, 161), room(64, 161)
    assert api.fh_i8_compress(api.matrix(64, 161), torch.from_numpy(x).cuda(), r, None) == api.FH_OK
    assert api.fh_i8_compress(api.matrix(161, 64), torch.from_numpy(np.ascontiguousarray(x.T)).cuda(), None, c) == api.FH_OK
    assert np.array_equal(container(br, r), i8.compress(x)) and np.array_equal(container(bc, c), i8.compress(x))


def operand(rows, k, seed):
    """(container on the GPU, codes, scales)."""
    x = values(rows, k, seed)
    return torch.from_numpy(i8.compress(x)).cuda(), *(lambda q, a: (q, i8.scales(a).astype(np.float64)))(*i8.quantise(x))


def sums(qa, qb):
    """Exact: below 2^53."""
    return (torch.from_numpy(qa.astype(np.float64)).cuda() @ torch.from_numpy(qb.astype(np.float64)).cuda().T).cpu().numpy()


PRODUCTS = [(1, 1, 1), (1, 8, 32), (1, 128, 64), (3, 40, 100), (8, 200, 256), (16, 128, 512), (17, 129, 300), (33, 500, 1000), (64, 96, 2048), (65, 256, 320),
            (128, 128, 128), (129, 127, 96), (200, 300, 777), (256, 512, 1024), (300, 260, 4096), (200, 8, 64), (257, 5, 40), (130, 1000, 256), (1, 4096, 4096),
            (5, 1000, 8192), (385, 513, 130), (1000, 777, 3000), (2100, 2300, 200)]


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_products(shape, dtype):
    m, n, k = shape
    (a, qa, sa), (b, qb, sb) = operand(m, k, 1), operand(n, k, 2)
    exact = sums(qa, qb) * sa[:, None] * sb[None, :]
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    for extra, alpha, accumulate in ((0, 1.0, False), (5, -0.37, True)):
        flat, c = watched(m, n, n + extra, dtype)
        c0 = values(m, n, 3, dtype)
        c.copy_(torch.from_numpy(c0))
        d = api.i8_product_desc(m, n, k, dtype, n + extra, alpha, accumulate)
        assert api.fh_i8_product(d, a, b, c, status) == api.FH_OK
        got = read(flat, c)
        assert int(status.item()) == api.FH_OK
        part = np.float64(np.float32(alpha)) * exact
        want = part + (c0 if accumulate else 0)
        # the sum, two factors and their product are rounded once each, then what is added, then the result
        assert (np.abs(got - want) <= 4.001 * U * np.abs(part) + U * np.abs(want) * accumulate + HALF[dtype] * (1 + 1e-6) * np.abs(want)).all()


def test_the_longest_axis():
    """Sums of the largest codes next to 2^31."""
    k = api.FH_I8_MAX_K
    for m in (2, 130):
        a, b = np.full((m, k), 3.0, dtype=np.float32), np.full((5, k), -2.0, dtype=np.float32)
        b[1] *= -1
        c = torch.empty(m, 5, device="cuda")
        assert api.fh_i8_product(api.i8_product_desc(m, 5, k), *(torch.from_numpy(i8.compress(x)).cuda() for x in (a, b)), c) == api.FH_OK
        want = np.tile(np.array([-6.0, 6, -6, -6, -6]) * k, (m, 1))
        assert (np.abs(c.cpu().numpy() - want) <= 8 * U * np.abs(want)).all()


@pytest.mark.parametrize("m", [2, 40, 300])
def test_factors_that_leave_fp32s_range_on_the_way(m):
    """Rows next to 2^127 times columns next to 2^-126, and alphas: what the result holds comes out."""
    n, k = 70, 64
    rng = np.random.default_rng(8)
    x, w = rng.standard_normal((m, k)).astype(np.float32), rng.standard_normal((n, k)).astype(np.float32)
    x[0] *= np.float32(2.0 ** 120)
    x[1] = 0
    w[1] *= np.float32(2.0 ** -118)
    w[2] = np.nan
    w[3] *= np.float32(2.0 ** 60)
    w[4] = 0
    a, b = (torch.from_numpy(i8.compress(v)).cuda() for v in (x, w))
    (qa, ma), (qb, mb) = i8.quantise(x), i8.quantise(w)
    for alpha in (1.0, 1e-30, 1e30, 0.0):
        c = torch.empty(m, n, device="cuda")
        assert api.fh_i8_product(api.i8_product_desc(m, n, k, alpha=alpha), a, b, c) == api.FH_OK
        want = sums(qa, qb) * i8.scales(ma).astype(np.float64)[:, None] * i8.scales(mb).astype(np.float64) * np.float64(np.float32(alpha))
        got = c.cpu().numpy().astype(np.float64)
        assert np.isnan(got[:, 2]).all()
        got, want = np.delete(got, 2, axis=1), np.delete(want, 2, axis=1)
        over = np.abs(want) > 3.5e38
        assert np.isinf(got[over]).all()
        small = np.abs(want) < 3.4e38
        assert (np.abs(got - want)[small] <= 5 * U * np.abs(want[small]) + 2.0 ** -149).all()


def pre_of(x, gate, up, m, f, k):
    (qx, sx), (qg, sg), (qu, su) = ((i8.quantise(v)[0], i8.scales(i8.magnitudes(v)).astype(np.float64)) for v in (x, gate, up))
    return sums(qx, qg) * sx[:, None] * sg, sums(qx, qu) * sx[:, None] * su


def act_slack(g, a, kind):
    """How far the kernel's activation may be from that of the same g: the fast exponential is within (2 + 1.2 |x|) steps, the fast quotient
    within two, erf within two of one; gelu's exponents are rounded four times ahead of that."""
    step = 2 * U
    if kind == i8.SILU:
        return np.abs(a) * ((2 + 1.2 * np.abs(g)) * step + 3 * step)
    if kind == i8.GELU:
        return np.abs(g) * 3 * step
    if kind == i8.GELU_TANH:
        w = 2 * np.sqrt(2 / np.pi) * np.abs(g + 0.044715 * g ** 3)
        return np.abs(a) * ((2 + 1.2 * w) * step + 4 * U * w + 3 * step)
    return 0 * a


GATED = [(1, 1, 1), (1, 128, 64), (1, 1000, 4096), (3, 40, 100), (16, 260, 512), (17, 129, 300), (64, 96, 2048), (70, 256, 320), (128, 130, 5000), (129, 127, 96),
         (130, 300, 8192), (300, 513, 777), (700, 1030, 256)]


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("kind", [api.FH_SILU, api.FH_GELU, api.FH_GELU_TANH, api.FH_RELU])
@pytest.mark.parametrize("shape", GATED)
def test_gated(shape, kind, dtype):
    m, f, k = shape
    rng = np.random.default_rng([9, m, f, k])
    x, gate, up = (rng.standard_normal((r, k)).astype(np.float32) * np.float32(s) for r, s in ((m, 1.0), (f, 1.5 * k ** -0.5), (f, k ** -0.5)))
    g, u = pre_of(x, gate, up, m, f, k)
    a, slope = i8.act(g, kind)
    c8, g8, u8 = (torch.from_numpy(i8.compress(v)).cuda() for v in (x, gate, up))
    fh, h = watched(m, f, f + 3, dtype)
    fp, pre = watched(m, 2 * f, 2 * f + 5, dtype)
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    d = api.gated_desc(m, f, k, kind, dtype, f + 3, 2 * f + 5)
    assert api.fh_i8_gated(d, c8, g8, u8, h, pre, status) == api.FH_OK
    got_h, got_p = read(fh, h), read(fp, pre)
    assert int(status.item()) == api.FH_OK
    both = np.concatenate([g, u], axis=1)
    assert (np.abs(got_p - both) <= (4.001 * U + HALF[dtype] * (1 + 1e-6)) * np.abs(both)).all()
    want = a * u
    # (a slope is at most 1.13 next to where it is taken)
    slack = np.abs(u) * (1.2 * 4.001 * U * np.abs(g) + act_slack(g, a, kind) + 1e-35) + 6 * U * np.abs(want)
    assert (np.abs(got_h - want) <= slack + HALF[dtype] * (1 + 1e-6) * np.abs(want)).all()
    for only in ("h", "pre"):                                        # each alone: the same bits
        flat, one = watched(m, f if only == "h" else 2 * f, f + 3 if only == "h" else 2 * f + 5, dtype)
        assert api.fh_i8_gated(d, c8, g8, u8, **{only: one}) == api.FH_OK
        assert np.array_equal(read(flat, one), got_h if only == "h" else got_p)


def slope_slack(g, kind):
    """(of the activation, of its derivative): functions within two steps, every product and sum within half of one."""
    a, slope = (np.abs(v) for v in i8.act(g, kind))
    step = 2 * U
    with np.errstate(over="ignore"):
        p = 1 / (1 + np.exp(-g))
        if kind == i8.SILU:
            return 4 * step * a, 6 * step * p * (1 + np.abs(g))
        if kind == i8.GELU:
            return 3 * step * np.abs(g), 3 * step + np.abs(g) * np.exp(-0.5 * g * g) * 0.4 * (4 + 0.5 * g * g) * step
        if kind == i8.GELU_TANH:
            w = 2 * np.sqrt(2 / np.pi) * np.abs(g + 0.044715 * g ** 3)
            e = 3 * U * w + 2 * step                                  # of the exponential
            p = 1 / (1 + np.exp(np.where(g > 0, -w, w)))
            t = 2 * np.abs(g) * p * (1 - p) * 0.8 * (1 + 0.135 * g * g)
            # (1e-36: beyond exp(88.7) the exponential is infinite and p 0 instead of less than 3e-39; |g| and the slope's factor are below 13 and 40)
            return a * (e + 3 * step) + 1e-36, p * (1 - p) * e + t * (2 * e + 8 * step) + 3 * step * p + 1e-36
    return 0 * a, 0 * a


BACKWARD = [(1, 1), (1, 16), (2, 100), (3, 8192), (9, 33), (1200, 48), (1201, 37), (1300, 1111), (1190, 2080), (40, 20000)]


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("kind", [api.FH_SILU, api.FH_GELU, api.FH_GELU_TANH, api.FH_RELU])
@pytest.mark.parametrize("shape", BACKWARD)
def test_gated_backward(shape, kind, dtype):
    m, f = shape
    rng = np.random.default_rng([10, m, f])
    pre, dh = (torch.from_numpy((rng.standard_normal(s) * 2).astype(np.float32)).to(TYPES[dtype]) for s in ((m, 2 * f), (m, f)))
    g, u, d64 = pre[:, :f].double().numpy(), pre[:, f:].double().numpy(), dh.double().numpy()
    want = i8.gated_backward(d64, g, u, kind)
    sa, ss = slope_slack(g, kind)
    slack = np.concatenate([np.abs(d64 * u) * ss, np.abs(d64) * sa], axis=1) + 3 * U * np.abs(want)
    for extra in (0, 3):
        fp, p = watched(m, 2 * f, 2 * f + extra, dtype)
        fd, dd = watched(m, f, f + extra, dtype)
        p.copy_(pre)
        dd.copy_(dh)
        fo, out = watched(m, 2 * f, 2 * f + extra, dtype)
        buf, packed = room(m, 2 * f)
        d = api.gated_desc(m, f, 1, kind, dtype, f + extra, 2 * f + extra)
        assert api.fh_gated_backward(d, dd, p, out, packed) == api.FH_OK
        held = container(buf, packed)
        got = read(fo, out)
        assert (np.abs(got - want) <= slack + HALF[dtype] * (1 + 1e-6) * np.abs(want) + 1e-44).all()
        assert np.array_equal(held, i8.compress(got))
        buf, packed = room(m, 2 * f)                                  # the container alone, the dense gradient alone, and over pre
        assert api.fh_gated_backward(d, dd, p, None, packed) == api.FH_OK
        assert np.array_equal(container(buf, packed), held)
        assert api.fh_gated_backward(d, dd, p, out) == api.FH_OK
        assert np.array_equal(read(fo, out), got)
        buf, packed = room(m, 2 * f)
        assert api.fh_gated_backward(d, dd, p, p, packed) == api.FH_OK
        assert np.array_equal(container(buf, packed), held)
        assert np.array_equal(read(fp, p), got)


def test_headers_that_are_not_expected():
    x = values(20, 70, 1)
    good = torch.from_numpy(i8.compress(x)).cuda()
    w = torch.from_numpy(i8.compress(values(30, 70, 2))).cuda()

    def calls(a, b, u):
        c, back = torch.full((20, 30), 7.0, device="cuda"), torch.full((20, 70), 7.0, device="cuda")
        st = torch.full((3,), 99, dtype=torch.int64, device="cuda")
        assert api.fh_i8_product(api.i8_product_desc(20, 30, 70), a, b, c, st[0:1]) == api.FH_OK
        assert api.fh_i8_gated(api.gated_desc(20, 30, 70), a, b, u, c, status=st[1:2]) == api.FH_OK
        assert api.fh_i8_decompress(a, api.matrix(20, 70), back, st[2:3]) == api.FH_OK
        return st.tolist(), bool((c == 7.0).all()), bool((back == 7.0).all())

    assert calls(good, w, w) == ([0, 0, 0], False, False)
    E = api.FH_ERR_CORRUPT
    for at in (0, 4, 8, 12, 16, 24):
        bad, badw = good.clone(), w.clone()
        bad[at] ^= 1
        badw[at] ^= 1
        assert calls(bad, w, w) == ([E, E, E], True, True)
        assert calls(good, badw, w)[0] == [E, E, 0] and calls(good, w, badw)[0] == [0, E, 0]
    assert calls(good[:-16], w, w) == ([E, E, E], True, True)
    for m in (200, 2000):                                             # a pair of CTAs
        big, c = torch.from_numpy(i8.compress(values(m, 70, 3))).cuda(), torch.full((m, 30), 7.0, device="cuda")
        st = torch.full((2,), 99, dtype=torch.int64, device="cuda")
        big[9] ^= 1
        assert api.fh_i8_product(api.i8_product_desc(m, 30, 70), big, w, c, st[0:1]) == api.FH_OK
        assert api.fh_i8_gated(api.gated_desc(m, 30, 70), big, w, w, c, status=st[1:2]) == api.FH_OK
        assert st.tolist() == [E, E] and (c == 7.0).all()


@pytest.fixture
def limits():
    """Sets (limit, silent stage); the defaults come back at the end."""
    def put(polls, silent):
        assert api.debug_set(api.FH_DEBUG_WAIT_POLLS, polls) == api.FH_OK
        assert api.debug_set(api.FH_DEBUG_SILENT_TILE, silent) == api.FH_OK
    yield put
    put(1 << 22, 2 ** 64 - 1)


@pytest.mark.parametrize("polls,silent", [(1, 2 ** 64 - 1), (200, 0), (200, 1), (200, 7)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("shape", [(1, 200, 512), (40, 300, 8192), (128, 1000, 6000), (300, 260, 9000), (2500, 2700, 2560)])
def test_a_wait_that_runs_out(shape, gated, polls, silent, limits):
    m, n, k = shape
    (a, qa, sa), (b, qb, sb) = operand(m, k, 1), operand(n, k, 2)
    want = sums(qa, qb) * sa[:, None] * sb
    flat, status = torch.full((m * n * (1 + gated) + 512,), 7.0, device="cuda"), torch.full((1,), 99, dtype=torch.int64, device="cuda")

    def call():
        if gated:                                                     # (both weights the same: what is kept is the product twice)
            return api.fh_i8_gated(api.gated_desc(m, n, k), a, b, b, None, flat, status)
        return api.fh_i8_product(api.i8_product_desc(m, n, k), a, b, flat, status)

    def right():
        got = flat[:-512].view(m, -1).cpu().numpy()
        return all((np.abs(got[:, i * n:(i + 1) * n] - want) <= 6 * U * np.abs(want)).all() for i in range(1 + gated))

    limits(polls, silent)
    assert call() == api.FH_OK
    torch.cuda.synchronize()
    ended = int(status.item())
    assert (flat[-512:] == 7.0).all()
    assert ended in (api.FH_OK, api.FH_ERR_TIMEOUT) and (silent > 1 or ended == api.FH_ERR_TIMEOUT)
    if ended == api.FH_OK:
        assert right()
    limits(1 << 22, 2 ** 64 - 1)                                      # a following call is right
    assert call() == api.FH_OK
    torch.cuda.synchronize()
    assert int(status.item()) == api.FH_OK and right()


def test_a_block_trains_on_what_it_kept_in_8_bits():
    """x -> gated block -> projection, and back: every product on containers, against the same in 64 bits on the values they hold.  Captured and
    replayed on other inputs; and on a stream of its own."""
    m, d, f = 272, 200, 328
    rng = np.random.default_rng(11)
    make = lambda *s, scale=1.0: torch.from_numpy((rng.standard_normal(s) * scale).astype(np.float32)).cuda()  # noqa: E731
    wg, wu, wd = make(f, d, scale=0.1), make(f, d, scale=0.1), make(d, f, scale=0.1)
    new = lambda r, c: torch.empty(api.i8_bytes(r, c), dtype=torch.uint8, device="cuda")  # noqa: E731
    g8, u8, d8, w8c, d8c = new(f, d), new(f, d), new(d, f), new(d, 2 * f), new(f, d)
    stacked = torch.cat([wg, wu])
    for mat, r, c in ((wg, g8, None), (wu, u8, None), (stacked, None, w8c), (wd, d8, d8c)):
        assert api.fh_i8_compress(api.matrix(*mat.shape), mat, r, c) == api.FH_OK
    x, dy = make(m, d), make(m, d)
    x8, x8c, h, pre, h8, h8c, y = new(m, d), new(d, m), *(torch.empty(s, device="cuda") for s in ((m, f), (m, 2 * f))), new(m, f), new(f, m), torch.empty(m, d, device="cuda")
    dy8, dy8c, dh, dpre, dp8, dp8c = new(m, d), new(d, m), torch.empty(m, f, device="cuda"), torch.empty(m, 2 * f, device="cuda"), new(m, 2 * f), new(2 * f, m)
    dx, dw, dwd = torch.empty(m, d, device="cuda"), torch.zeros(2 * f, d, device="cuda"), torch.zeros(d, f, device="cuda")
    gd = api.gated_desc(m, f, d)

    def step(stream=None):
        rcs = [api.fh_i8_compress(api.matrix(m, d), x, x8, x8c, stream), api.fh_i8_gated(gd, x8, g8, u8, h, pre, stream=stream),
               api.fh_i8_compress(api.matrix(m, f), h, h8, h8c, stream), api.fh_i8_product(api.i8_product_desc(m, d, f), h8, d8, y, stream=stream),
               api.fh_i8_compress(api.matrix(m, d), dy, dy8, dy8c, stream), api.fh_i8_product(api.i8_product_desc(m, f, d), dy8, d8c, dh, stream=stream),
               api.fh_i8_product(api.i8_product_desc(d, f, m), dy8c, h8c, dwd, stream=stream),
               api.fh_gated_backward(gd, dh, pre, dpre, dp8, stream), api.fh_i8_compress(api.matrix(m, 2 * f), dpre, None, dp8c, stream),
               api.fh_i8_product(api.i8_product_desc(m, d, 2 * f), dp8, w8c, dx, stream=stream),
               api.fh_i8_product(api.i8_product_desc(2 * f, d, m), dp8c, x8c, dw, stream=stream)]
        assert rcs == [api.FH_OK] * len(rcs)

    def product(a, b, rows, cols, k):
        """Of what two containers hold: the sums of the codes' products, exact, times both scales."""
        (qa, ma), (qb, mb) = i8.unpack(a.cpu().numpy(), rows, k), i8.unpack(b.cpu().numpy(), cols, k)
        return sums(qa, qb) * i8.scales(ma).astype(np.float64)[:, None] * i8.scales(mb).astype(np.float64)

    def check():
        torch.cuda.synchronize()
        n = lambda t: t.cpu().numpy().astype(np.float64)  # noqa: E731

        def near(got, want):
            # four roundings of each sum, and one of what was read back
            assert (np.abs(n(got) - want) <= 8 * U * np.abs(want)).all()
        p, g, u = n(pre), product(x8, g8, m, f, d), product(x8, u8, m, f, d)
        assert np.array_equal(x8.cpu().numpy(), i8.compress(x.cpu().numpy()))
        near(pre, np.concatenate([g, u], axis=1))
        want = i8.act(g, i8.SILU)[0] * u
        assert (np.abs(n(h) - want) <= 1e-5 * (1 + np.abs(want))).all()
        assert np.array_equal(h8.cpu().numpy(), i8.compress(h.cpu().numpy())) and np.array_equal(h8c.cpu().numpy(), i8.compress(h.cpu().numpy().T.copy()))
        near(y, product(h8, d8, m, d, f))
        near(dh, product(dy8, d8c, m, f, d))
        near(dwd, product(dy8c, h8c, d, f, m))
        near(dx, product(dp8, w8c, m, d, 2 * f))
        near(dw, product(dp8c, x8c, 2 * f, d, m))
        back = i8.gated_backward(n(dh), p[:, :f], p[:, f:], i8.SILU)
        assert (np.abs(n(dpre) - back) <= 64 * U * (np.abs(back) + np.abs(np.tile(n(dh), 2)) * (1 + np.abs(p)) * (1 + np.abs(np.roll(p, f, axis=1))))).all()
        assert np.array_equal(dp8.cpu().numpy(), i8.compress(dpre.cpu().numpy())) and np.array_equal(dp8c.cpu().numpy(), i8.compress(dpre.cpu().numpy().T.copy()))

    step()
    check()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    step(side)
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in range(2):
        x.copy_(make(m, d, scale=0.5 + seed))
        dy.copy_(make(m, d))
        graph.replay()
        check()


def test_large_products_are_those_of_their_parts():
    """Many tiles to a pair, from two streams at once: equal bits to products of slices."""
    m, n, k = 3000, 2900, 1111
    (a, _, _), (b, _, _) = operand(m, k, 1), operand(n, k, 2)
    xa = values(m, k, 1)
    whole, other = torch.empty(m, n, device="cuda"), torch.empty(m, n, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        assert api.fh_i8_product(api.i8_product_desc(m, n, k), a, b, whole) == api.FH_OK
        assert api.fh_i8_product(api.i8_product_desc(m, n, k), a, b, other, stream=s) == api.FH_OK
    torch.cuda.synchronize()
    assert torch.equal(whole, other)
    for lo, hi in ((0, 16), (1000, 1100), (2800, 3000)):
        part, one = torch.from_numpy(i8.compress(xa[lo:hi])).cuda(), torch.empty(hi - lo, n, device="cuda")
        assert api.fh_i8_product(api.i8_product_desc(hi - lo, n, k), part, b, one) == api.FH_OK
        assert torch.equal(one, whole[lo:hi])
