"""Products of microscaled 4-bit matrices against the plain definition's values multiplied in 64 bits."""
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


def operand(rows, k, fmt, exponent=0, seed=0):
    """(container on the GPU, the values it holds)."""
    rng = np.random.default_rng([seed, rows, k, fmt])
    x = (rng.standard_normal((rows, k)) * np.exp(rng.standard_normal((rows, 1))) * 2.0 ** exponent).astype(np.float32)
    buf = mx.compress(x, fmt, exponent)
    return torch.from_numpy(buf).cuda(), mx.restore(buf, rows, k, fmt)


def product(d, a, b, c0=None):
    """The result with its surroundings watched."""
    t = torch.float32 if d.dtype == api.FH_F32 else torch.bfloat16
    flat = torch.full((d.m * d.ldc + 128,), 7.0, dtype=t, device="cuda")
    view = flat.as_strided((d.m, d.n), (d.ldc, 1))
    if c0 is not None:
        view.copy_(c0)
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    assert api.fh_mx_product(d, a, b, flat, status) == api.FH_OK
    torch.cuda.synchronize()
    got = view.float().cpu().numpy()
    view.fill_(7.0)
    assert (flat == 7.0).all()
    return int(status.item()), got


def agree(got, want, size, k, dtype):
    """`size`: the products' magnitudes summed up.  The products of codes are exact; each of at most k + 8 fp32 additions and scalings is
    off by at most a last place of what has been summed, 2^-23 of `size`; one rounding of the result."""
    half = 2.0 ** -24 if dtype == api.FH_F32 else 2.0 ** -8
    assert np.isfinite(got).all()
    assert (np.abs(got - want) <= (k + 8) * 2.0 ** -23 * size + half * np.abs(want)).all()


SHAPES = [(1, 1, 1), (1, 8, 32), (1, 128, 64), (3, 40, 100), (8, 200, 256), (16, 128, 512), (17, 129, 300), (33, 500, 1000), (64, 96, 2048), (65, 256, 320),
          (128, 128, 128), (129, 127, 96), (200, 300, 777), (256, 512, 1024), (300, 260, 4096), (200, 8, 64), (257, 5, 40), (130, 1000, 256), (1, 4096, 4096), (5, 1000, 8192)]


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("fmt,ea,eb", [(mx.B32, 0, 0), (mx.B16, 0, 0), (mx.B16, -5, 3)])
@pytest.mark.parametrize("shape", SHAPES)
def test_products(shape, fmt, ea, eb, dtype):
    m, n, k = shape
    (a, x), (b, y) = operand(m, k, fmt, ea, 1), operand(n, k, fmt, eb, 2)
    st, got = product(api.mx_product_desc(m, n, k, fmt, dtype), a, b)
    assert st == api.FH_OK
    agree(got, x @ y.T, np.abs(x) @ np.abs(y).T, k, dtype)


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("m", [1, 20, 130])
def test_every_element_of_the_operands_counts_once(m, fmt):
    """Small integers: the sums are exact, so that a misplaced code or scale shows."""
    n, k = 136, 448
    rng = np.random.default_rng(m)
    xs, ys = [], []
    for rows, seed, out in ((m, 1, xs), (n, 2, ys)):
        v = rng.choice([-3.0, -2.0, -1.0, 0.0, 1.0, 2.0, 3.0], size=(rows, k))
        s = 2.0 ** rng.integers(0, 5, size=(rows, k // mx.BLOCK[fmt]))
        v[:, ::mx.BLOCK[fmt]] = 6.0                                  # (its block's scale is then the power of two)
        v *= np.repeat(s, mx.BLOCK[fmt], axis=1)
        buf = mx.compress(v, fmt)
        assert np.array_equal(mx.restore(buf, rows, k, fmt), v)
        out += [torch.from_numpy(buf).cuda(), v]
    st, got = product(api.mx_product_desc(m, n, k, fmt), xs[0], ys[0])
    assert st == api.FH_OK and np.array_equal(got, xs[1] @ ys[1].T)   # (below 448 * 96^2 < 2^24)


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("m,n,k,ldc", [(4, 50, 640, 50), (4, 50, 640, 77), (150, 140, 1500, 141)])
def test_alpha_strides_and_adding(m, n, k, ldc, dtype):
    (a, x), (b, y) = operand(m, k, mx.B32, 0, 3), operand(n, k, mx.B32, 0, 4)
    t = torch.float32 if dtype == api.FH_F32 else torch.bfloat16
    c0 = torch.from_numpy(np.random.default_rng(5).standard_normal((m, n))).to(t).cuda()
    for alpha in (1.0, -0.37, 0.0):
        for add in (False, True):
            al = float(np.float32(alpha))
            st, got = product(api.mx_product_desc(m, n, k, mx.B32, dtype, ldc, alpha, add), a, b, c0 if add else None)
            want = al * (x @ y.T) + (c0.double().cpu().numpy() if add else 0.0)
            size = abs(al) * (np.abs(x) @ np.abs(y).T) + (c0.double().abs().cpu().numpy() if add else 0.0)
            assert st == api.FH_OK
            agree(got, want, size, k, dtype)


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("dtype,add", [(api.FH_F32, False), (api.FH_F32, True), (api.FH_BF16, False)])
def test_more_tiles_than_the_device_holds_at_once(dtype, add, fmt):
    """10 x 11 tiles of 256 x 256, in a band of eight rows of tiles and one of two, the last row and column of tiles in part."""
    m, n, k = 2500, 2700, 700
    (a, x), (b, y) = operand(m, k, fmt, 0, 13), operand(n, k, fmt, 0, 14)
    c0 = torch.from_numpy(np.random.default_rng(15).standard_normal((m, n)).astype(np.float32)).cuda() if add else None
    st, got = product(api.mx_product_desc(m, n, k, fmt, dtype, n + 3, 0.75, add), a, b, c0)
    want, size = 0.75 * (x @ y.T), 0.75 * (np.abs(x) @ np.abs(y).T)
    if add:
        want, size = want + c0.double().cpu().numpy(), size + c0.double().abs().cpu().numpy()
    assert st == api.FH_OK
    agree(got, want, size, k, dtype)


def test_two_host_threads_at_once():
    """Calls from two threads, a stream each: large and small products, layer norms and containers in turn."""
    import threading
    found = []

    def work(seed):
        try:
            (a, x), (b, y) = operand(260, 900, mx.B16, 0, seed), operand(300, 900, mx.B16, 0, seed + 50)
            rows = np.random.default_rng(seed).standard_normal((40, 900)).astype(np.float32)
            want = mx.compress(rows, mx.B32)
            with torch.cuda.stream(torch.cuda.Stream()):
                t, c, c1 = torch.from_numpy(rows).cuda(), torch.empty(260, 300, device="cuda"), torch.empty(1, 300, device="cuda")
                one = mx.compress(x[:1], mx.B16)
                first, x1 = torch.from_numpy(one).cuda(), mx.restore(one, 1, 900, mx.B16)
                for _ in range(20):
                    buf = torch.zeros(api.mx_bytes(40, 900, mx.B32), dtype=torch.uint8, device="cuda")
                    assert api.fh_mx_product(api.mx_product_desc(260, 300, 900, mx.B16), a, b, c) == api.FH_OK
                    assert api.fh_mx_compress(api.matrix(40, 900), api.mx_params(), t, buf) == api.FH_OK
                    assert api.fh_mx_product(api.mx_product_desc(1, 300, 900, mx.B16), first, b, c1) == api.FH_OK
                    torch.cuda.current_stream().synchronize()
                    assert np.array_equal(buf.cpu().numpy(), want)
                    agree(c.cpu().numpy(), x @ y.T, np.abs(x) @ np.abs(y).T, 900, api.FH_F32)
                    agree(c1.cpu().numpy(), x1 @ y.T, np.abs(x1) @ np.abs(y).T, 900, api.FH_F32)
            found.append("ok")
        except BaseException as e:    # noqa: BLE001 (told to the test)
            found.append(repr(e))
    threads = [threading.Thread(target=work, args=(s,)) for s in (100, 200)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert found == ["ok", "ok"]


def test_equal_inputs_give_equal_bits():
    (a, _), (b, _) = operand(40, 8192, mx.B16, 0, 5), operand(200, 8192, mx.B16, 0, 6)
    d = api.mx_product_desc(40, 200, 8192, mx.B16)
    first = product(d, a, b)[1]
    for _ in range(5):
        assert np.array_equal(product(d, a, b)[1], first)


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
def test_nan_scales_stay_in_their_rows(fmt):
    rng = np.random.default_rng(8)
    x, y = rng.standard_normal((5, 600)), rng.standard_normal((200, 600))
    x[2, 100], y[150, 599] = np.nan, np.inf
    st, got = product(api.mx_product_desc(5, 200, 600, fmt), *(torch.from_numpy(mx.compress(v, fmt)).cuda() for v in (x, y)))
    want = np.zeros((5, 200), dtype=bool)
    want[2], want[:, 150] = True, True
    assert st == api.FH_OK and np.array_equal(np.isnan(got), want)


def test_far_exponents():
    """Exponents whose sum passes what one fp32 factor holds: what fits comes out, what is beyond fp32 (2^124 times the largest of the
    sums, a few hundred) is infinite."""
    for ea, eb in ((64, 60), (-64, -60), (64, -64)):
        (a, x), (b, y) = operand(4, 64, mx.B16, ea, 9), operand(8, 64, mx.B16, eb, 10)
        st, got = product(api.mx_product_desc(4, 8, 64, mx.B16), a, b)
        assert st == api.FH_OK
        want = x @ y.T
        beyond = np.abs(want) > float(np.finfo(np.float32).max)
        assert np.array_equal(got[beyond], np.where(want[beyond] > 0, np.inf, -np.inf)) and beyond.any() == (ea + eb == 124)
        # (numbers below 2^-126 have a step of 2^-149)
        off = np.abs(np.where(beyond, 0, got - want))
        assert (off <= 72 * 2.0 ** -23 * (np.abs(x) @ np.abs(y).T) + 2.0 ** -149).all()
        # with a factor that brings them back, or that is zero
        for alpha in (2.0 ** -(ea + eb) * 1.25, 0.0, -(2.0 ** -149) if ea + eb == 124 else 2.0 ** 100):
            st, got = product(api.mx_product_desc(4, 8, 64, mx.B16, alpha=alpha), a, b)
            assert st == api.FH_OK and (np.abs(got - alpha * want) <= 72 * 2.0 ** -23 * abs(alpha) * (np.abs(x) @ np.abs(y).T) + 2.0 ** -149).all()


@pytest.mark.parametrize("which", ["a", "b"])
@pytest.mark.parametrize("m", [3, 130])
def test_another_header_is_reported_and_nothing_written(m, which):
    (a, _), (b, _) = operand(m, 900, mx.B32, 0, 11), operand(130, 900, mx.B32, 0, 12)
    for change in (0, 8, 12, None):
        x, y = a.clone(), b.clone()
        t = x if which == "a" else y
        if change is None:
            x, y = (x[:-16], y) if which == "a" else (x, y[:-16])
        else:
            t[change] += 1
        st, got = product(api.mx_product_desc(m, 130, 900), x, y)
        assert st == api.FH_ERR_CORRUPT and (got == 7.0).all()
    st, got = product(api.mx_product_desc(m, 130, 900), a, b)
    assert st == api.FH_OK and (got != 7.0).any()


def test_captured_on_two_streams_at_once():
    """Two graphs on two streams, replayed side by side: no workspace is shared."""
    runs = []
    for seed in (1, 2):
        (a, x), (b, y) = operand(30, 4096, mx.B16, 0, seed), operand(600, 4096, mx.B16, 0, 20 + seed)
        c = torch.zeros(30, 600, device="cuda")
        d = api.mx_product_desc(30, 600, 4096, mx.B16)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            assert api.fh_mx_product(d, a, b, c) == api.FH_OK
        runs.append((stream, graph, a, b, c, x, y))
    for _ in range(3):
        for stream, graph, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, _, _, c, x, y in runs:
        agree(c.cpu().numpy(), x @ y.T, np.abs(x) @ np.abs(y).T, 4096, api.FH_F32)
