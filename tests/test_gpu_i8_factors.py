"""Products and gated blocks whose factors have to be multiplied in 64 bits, whose rows are not finite, or whose weights are not what they should be, on common
axes that are worked on in parts and on those that are not."""
import numpy as np
import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build
from tests.test_gpu_i8 import HALF, TYPES, U, act_slack, read, sums, watched

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
N = 70


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def held(x):
    """(container on the GPU, codes, scales)."""
    q, a = i8.quantise(x)
    return torch.from_numpy(i8.compress(x)).cuda(), q, i8.scales(a).astype(np.float64)


def rows(m, k, rng):
    """Tokens: a very large one, a NaN, an infinity, a very small one, zeros, then ordinary ones (as many as there are)."""
    x = rng.standard_normal((m, k)).astype(np.float32)
    for i, make in enumerate((lambda r: r * np.float32(2.0 ** 100), lambda r: np.where(np.arange(k) == k // 2, np.float32("nan"), r),
                              lambda r: np.where(np.arange(k) == k - 1, np.float32("-inf"), r), lambda r: r * np.float32(2.0 ** -110), lambda r: 0 * r)):
        at = i * 7 % m if m > 5 else i
        if at < m:
            x[at] = make(x[at])
    return x


def weights(k, rng):
    w = rng.standard_normal((N, k)).astype(np.float32)
    w[1] *= np.float32(2.0 ** -106)
    w[2] = np.nan
    w[3] *= np.float32(2.0 ** 100)
    w[4] = 0
    return w


def product(a, b):
    with np.errstate(invalid="ignore"):
        return sums(a[1], b[1]) * a[2][:, None] * b[2][None, :]


def near(got, want, bound, nan):
    """NaN where `nan`, infinite beyond the range, within the bound elsewhere (next to the range's end both are right)."""
    assert np.array_equal(np.isnan(got), nan)
    with np.errstate(invalid="ignore"):
        over, fine = np.abs(want) > 3.42e38, np.abs(want) < 3.38e38
        assert (np.isinf(got) & (np.sign(got) == np.sign(want)))[over & ~nan].all()
        assert (np.abs(got - want) <= bound)[fine & ~nan].all()


SHAPES = [(m, k) for m in (2, 5, 40, 128, 300) for k in (64, 8192)]


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("m,k", SHAPES)
def test_products(m, k, dtype):
    rng = np.random.default_rng([1, m, k])
    x, w = rows(m, k, rng), weights(k, rng)
    a, b = held(x), held(w)
    nan = np.isnan(a[2])[:, None] | np.isnan(b[2])[None, :]
    for alpha in (1.0, 1e-30, -1e30):
        flat, c = watched(m, N, N + 2, dtype)
        assert api.fh_i8_product(api.i8_product_desc(m, N, k, dtype, N + 2, alpha), a[0], b[0], c) == api.FH_OK
        want = product(a, b) * np.float64(np.float32(alpha))
        near(read(flat, c).astype(np.float64), want, (5 * U + HALF[dtype] * (1 + 1e-6)) * np.abs(want) + 2.0 ** (-149 if dtype == api.FH_F32 else -133), nan)


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("kind", [api.FH_SILU, api.FH_GELU, api.FH_GELU_TANH, api.FH_RELU])
@pytest.mark.parametrize("m,k", SHAPES)
def test_gated(m, k, kind, dtype):
    rng = np.random.default_rng([2, m, k])
    x, gate, up = rows(m, k, rng), weights(k, rng), np.roll(weights(k, rng), 9, axis=0)
    up[1] *= np.float32(2.0 ** -106)                                  # (so that a large token has an ordinary h)
    up[0] = gate[5] = np.inf
    a, b, c = held(x), held(gate), held(up)
    flat_h, h = watched(m, N, N + 1, dtype)
    flat_p, pre = watched(m, 2 * N, 2 * N + 1, dtype)
    assert api.fh_i8_gated(api.gated_desc(m, N, k, kind, dtype, N + 1, 2 * N + 1), a[0], b[0], c[0], h, pre) == api.FH_OK
    got_h, got_p = read(flat_h, h).astype(np.float64), read(flat_p, pre).astype(np.float64)
    g, u = product(a, b), product(a, c)
    nan_g, nan_u = (np.isnan(a[2])[:, None] | np.isnan(v[2])[None, :] for v in (b, c))
    least = 2.0 ** (-149 if dtype == api.FH_F32 else -133)
    both = np.concatenate([g, u], axis=1)
    near(got_p, both, (4.001 * U + HALF[dtype] * (1 + 1e-6)) * np.abs(both) + least, np.concatenate([nan_g, nan_u], axis=1))
    # h, where both of what it is made of are numbers of fp32, and the fast quotient's denominator is
    safe = np.where(nan_g | nan_u, 0.0, g)
    plain = ~(nan_g | nan_u) & (np.abs(g) < 3.38e38) & (np.abs(u) < 3.38e38)
    with np.errstate(over="ignore", invalid="ignore"):
        act = i8.act(np.clip(safe, -1e3, 1e3), kind)[0]
        act = np.where(safe > 1e3, safe, np.where(safe < -1e3, 0.0, act))
        want = act * np.where(nan_u, 0.0, u)
        bound = np.abs(u) * (1.2 * 4.001 * U * np.abs(safe) + act_slack(np.clip(safe, -1e3, 1e3), act, kind) + 1e-35) + (6 * U + HALF[dtype] * (1 + 1e-6)) * np.abs(want) + least
    assert np.isnan(got_h[nan_g | nan_u]).all()
    near(np.where(plain, got_h, 0.0), np.where(plain, want, 0.0), np.where(plain, bound, 1.0), np.zeros_like(plain))


@pytest.mark.parametrize("m", [1, 40, 300, 2000])
def test_headers_of_weights(m):
    """Of the only weight, of the gate and of the other one: nothing is written."""
    rng = np.random.default_rng(3)
    a, b = held(rng.standard_normal((m, 96)).astype(np.float32)), held(rng.standard_normal((N, 96)).astype(np.float32))
    for at in (0, 8, 12, 24):
        bad = b[0].clone()
        bad[at] ^= 1
        for call in (lambda c, p, s: api.fh_i8_product(api.i8_product_desc(m, N, 96), a[0], bad, c, s), lambda c, p, s: api.fh_i8_gated(api.gated_desc(m, N, 96), a[0], bad, b[0], c, p, s),
                     lambda c, p, s: api.fh_i8_gated(api.gated_desc(m, N, 96), a[0], b[0], bad, c, p, s)):
            c, p, status = torch.full((m, N), 7.0, device="cuda"), torch.full((m, 2 * N), 7.0, device="cuda"), torch.full((1,), 99, dtype=torch.int64, device="cuda")
            assert call(c, p, status) == api.FH_OK
            assert int(status.item()) == api.FH_ERR_CORRUPT and (c == 7.0).all() and (p == 7.0).all()
