"""Products whose rings of stages come round several times, and what small products alone were tested on, for more than 128 rows: NaN scales, far
exponents, factors, two graphs side by side, equal bits, offsets beyond 2^31.  Operands are compressed on the device; the sums are in 64 bits."""
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


def operand(rows, k, fmt, exponent=0, seed=0, x=None):
    """(container, the values it holds in 64 bits), both on the device."""
    if x is None:
        g = torch.Generator(device="cuda").manual_seed(1000 * seed + rows + k)
        x = torch.randn(rows, k, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda")) * 2.0 ** exponent
    buf, values = torch.empty(api.mx_bytes(rows, k, fmt), dtype=torch.uint8, device="cuda"), torch.empty(rows, k, device="cuda")
    assert api.fh_mx_compress(api.matrix(rows, k), api.mx_params(fmt, exponent), x, buf) == api.FH_OK
    assert api.fh_mx_decompress(buf, api.matrix(rows, k), fmt, values) == api.FH_OK
    return buf, values.double()


def product(d, a, b, c0=None):
    """(status, C); what lies around C is watched."""
    flat = torch.full((d.m * d.ldc + 128,), 7.0, dtype=TORCH[d.dtype], device="cuda")
    view = flat.as_strided((d.m, d.n), (d.ldc, 1))
    if c0 is not None:
        view.copy_(c0)
    status = torch.full((1,), 99, dtype=torch.int64, device="cuda")
    assert api.fh_mx_product(d, a, b, flat, status) == api.FH_OK
    got = view.clone()
    view.fill_(7.0)
    assert bool((flat == 7.0).all())
    return int(status.item()), got


def agree(got, want, size, k, dtype):
    """`size`: the products' magnitudes summed up.  The products of codes are exact; each of at most k + 8 fp32 additions and scalings is
    off by at most a last place of what has been summed, 2^-23 of `size`; one rounding of the result."""
    half = 2.0 ** -24 if dtype == api.FH_F32 else 2.0 ** -8
    assert bool(torch.isfinite(got).all())
    assert bool(((got.double() - want).abs() <= (k + 8) * 2.0 ** -23 * size + half * want.abs()).all())


# more stages of 256 to a part than a ring has: one row to 128, and pairs with one tile, with parts, and with several tiles each
ROUNDS = [(1, 40, 40000), (16, 1000, 20011), (30, 3000, 12000), (64, 20000, 4100), (128, 500, 30000), (129, 200, 16400), (300, 260, 24000), (1000, 777, 16384),
          (2500, 2700, 3000), (2049, 4100, 1800)]


@pytest.mark.parametrize("dtype,add", [(api.FH_F32, False), (api.FH_BF16, False), (api.FH_F32, True)])
@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
@pytest.mark.parametrize("shape", ROUNDS)
def test_rings_come_round(shape, fmt, dtype, add):
    m, n, k = shape
    (a, x), (b, y) = operand(m, k, fmt, 0, 1), operand(n, k, fmt, 0, 2)
    c0 = torch.randn(m, n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda") if add else None
    d = api.mx_product_desc(m, n, k, fmt, dtype, n + 1, -0.75, add)
    st, got = product(d, a, b, c0)
    want, size = -0.75 * (x @ y.T), 0.75 * (x.abs() @ y.abs().T)
    if add:
        want, size = want + c0.double(), size + c0.double().abs()
    assert st == api.FH_OK
    agree(got, want, size, k, dtype)
    assert torch.equal(product(d, a, b, c0)[1], got)    # equal inputs, equal bits


@pytest.mark.parametrize("m,n,k", [(20, 300, 20000), (300, 260, 12000), (2500, 2700, 1600)])
@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
def test_every_element_counts_once_in_every_round(fmt, m, n, k):
    """Whole numbers: the sums are exact, so that a misplaced or repeated stage shows."""
    out = []
    for rows, seed in ((m, 1), (n, 2)):
        g = torch.Generator(device="cuda").manual_seed(seed)
        v = torch.randint(-3, 4, (rows, k), generator=g, device="cuda").float()
        v[:, ::mx.BLOCK[fmt]] = 6.0                       # (its block's scale is then one)
        buf, values = operand(rows, k, fmt, x=v)
        assert torch.equal(values, v.double())
        out += [buf, values]
    st, got = product(api.mx_product_desc(m, n, k, fmt), out[0], out[2])
    assert st == api.FH_OK and torch.equal(got.double(), out[1] @ out[3].T)    # (below 36 * 20000 < 2^24)


@pytest.mark.parametrize("m,n,k", [(300, 500, 900), (130, 256, 9000), (2500, 2700, 300)])
@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
def test_nan_scales_stay_in_their_rows(fmt, m, n, k):
    g = torch.Generator(device="cuda").manual_seed(8)
    x, y = torch.randn(m, k, generator=g, device="cuda"), torch.randn(n, k, generator=g, device="cuda")
    x[2, 100], x[m - 1, 0], y[150, k - 1], y[n - 1, 5] = float("nan"), float("inf"), -float("inf"), float("nan")
    st, got = product(api.mx_product_desc(m, n, k, fmt), operand(m, k, fmt, x=x)[0], operand(n, k, fmt, x=y)[0])
    want = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    want[[2, m - 1]], want[:, [150, n - 1]] = True, True
    assert st == api.FH_OK and torch.equal(torch.isnan(got), want)


@pytest.mark.parametrize("m,n,k", [(200, 300, 64), (300, 260, 5000)])
def test_far_exponents_and_factors(m, n, k):
    """Exponents and factors whose product passes what one fp32 factor holds: what fits comes out, what is beyond fp32 is infinite."""
    top = float(np.finfo(np.float32).max)
    for ea, eb in ((64, 60), (-64, -60), (64, -64), (40, -3)):
        (a, x), (b, y) = operand(m, k, mx.B16, ea, 9), operand(n, k, mx.B16, eb, 10)
        want, size = x @ y.T, x.abs() @ y.abs().T
        for alpha in (1.0, 2.0 ** -(ea + eb) * 1.25, 0.0, -(2.0 ** -149) if ea + eb == 124 else 2.0 ** 100, -0.3 * 2.0 ** -70):
            alpha = float(np.float32(alpha))
            st, got = product(api.mx_product_desc(m, n, k, mx.B16, alpha=alpha), a, b)
            assert st == api.FH_OK
            err = (k + 8) * 2.0 ** -23 * size * abs(alpha) + 2.0 ** -149       # (numbers below 2^-126 have a step of 2^-149)
            w = alpha * want
            inside, beyond = w.abs() + err <= top, w.abs() - err > top
            assert bool(((got.double() - w).abs() <= err)[inside].all())
            assert torch.equal(got[beyond], torch.where(w[beyond] > 0, float("inf"), -float("inf")).float())


def test_two_graphs_of_pairs_side_by_side():
    runs = []
    for seed in (1, 2):
        (a, x), (b, y) = operand(300, 9000, mx.B16, 0, seed), operand(700, 9000, mx.B16, 0, 20 + seed)
        c, d = torch.zeros(300, 700, device="cuda"), api.mx_product_desc(300, 700, 9000, mx.B16)
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                assert api.fh_mx_product(d, a, b, c) == api.FH_OK
        runs.append((stream, graph, a, b, c, x, y))
    torch.cuda.synchronize()
    for _ in range(5):
        for stream, graph, *_ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    for _, _, _, _, c, x, y in runs:
        agree(c, x @ y.T, x.abs() @ y.abs().T, 9000, api.FH_F32)


@pytest.mark.parametrize("m,ldc", [(100, 24_000_001), (70_000, 33_000)])
def test_c_beyond_2_to_the_31_elements(m, ldc):
    """Few rows far apart, and many: the last rows are where they belong, and nothing lies between."""
    n, k = 48, 300
    (a, x), (b, y) = operand(m, k, mx.B32, 0, 1), operand(n, k, mx.B32, 0, 2)
    flat = torch.full(((m - 1) * ldc + n + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    assert flat.numel() > 2 ** 31
    assert api.fh_mx_product(api.mx_product_desc(m, n, k, mx.B32, api.FH_BF16, ldc), a, b, flat) == api.FH_OK
    view = flat.as_strided((m, n), (ldc, 1))
    agree(view, x @ y.T, x.abs() @ y.abs().T, k, api.FH_BF16)
    view.fill_(7.0)
    assert bool((flat == 7.0).all())


def test_two_host_threads_with_norms_products_and_containers():
    """Calls of every operator from two threads, a stream and a workspace each."""
    import threading
    found = []

    def work(seed):
        try:
            rows, cols, n = 700, 1000, 300
            with torch.cuda.stream(torch.cuda.Stream()):
                g = torch.Generator(device="cuda").manual_seed(seed)
                x, dy = torch.randn(rows, cols, generator=g, device="cuda"), torch.randn(rows, cols, generator=g, device="cuda")
                gamma, beta = 1 + 0.1 * torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
                w4, _ = operand(n, cols, mx.B16, 0, seed)
                d, p, fmt = api.norm_desc(rows, cols), api.mx_params(mx.B16), mx.B16

                def step():
                    y, dx = torch.empty_like(x), torch.empty_like(x)
                    mean, rstd, dgamma, dbeta = (torch.empty(s, device="cuda") for s in (rows, rows, cols, cols))
                    y4, x4 = (torch.empty(api.mx_bytes(rows, cols, fmt), dtype=torch.uint8, device="cuda") for _ in range(2))
                    z, scratch = torch.empty(rows, n, device="cuda"), torch.empty(api.norm_work_bytes(d), dtype=torch.uint8, device="cuda")
                    assert api.fh_mx_compress(api.matrix(rows, cols), p, x, x4) == api.FH_OK
                    assert api.fh_layer_norm(d, x, gamma, beta, y, mean, rstd, y4, p) == api.FH_OK
                    assert api.fh_mx_product(api.mx_product_desc(rows, n, cols, fmt), y4, w4, z) == api.FH_OK
                    assert api.fh_layer_norm_backward(d, dy, x4, gamma, mean, rstd, dx, dgamma, dbeta, scratch, fmt) == api.FH_OK
                    return y, mean, rstd, y4, x4, z, dx, dgamma, dbeta

                first = step()
                torch.cuda.current_stream().synchronize()
                alone.setdefault(seed, first)
                for _ in range(30):
                    again = step()
                    torch.cuda.current_stream().synchronize()
                    assert all(torch.equal(s, t) for s, t in zip(again, alone[seed]))
            found.append("ok")
        except BaseException as e:    # noqa: BLE001 (told to the test)
            found.append(repr(e))

    alone = {}
    for seed in (1, 2):               # what each gives alone; its parts are held to the definitions elsewhere
        work(seed)
    threads = [threading.Thread(target=work, args=(s,)) for s in (1, 2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert found == ["ok"] * 4
