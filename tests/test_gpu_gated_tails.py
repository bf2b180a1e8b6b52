"""The gated block's activations and their derivatives far from zero, where they are next to nothing or next to their argument: relative to their own
size, not to the largest of a row."""
import math

import numpy as np
import pytest

from oracle import i8
from paper_2510_11400_b200 import api, build

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")
U = 2.0 ** -24                                                       # half a step of fp32, relative
HALF = {api.FH_F32: U, api.FH_BF16: 2.0 ** -8}
TYPES = {api.FH_F32: torch.float32, api.FH_BF16: torch.bfloat16}
KINDS = [api.FH_SILU, api.FH_GELU, api.FH_GELU_TANH, api.FH_RELU]


@pytest.fixture(scope="module", autouse=True)
def library():
    build.build()
    api.lib()


def exact(g, kind):
    """(activation, derivative, 1 - p) in 64 bits, for any finite g."""
    g = np.asarray(g, dtype=np.float64)
    with np.errstate(all="ignore"):
        c = np.clip(g, -1e3, 1e3)                                    # (beyond, p is 0 or 1 and the density 0)
        if kind == i8.SILU:
            p, q = 1 / (1 + np.exp(-c)), 1 / (1 + np.exp(c))
            return g * p, p * (1 + g * q)
        if kind == i8.GELU:
            p = 0.5 * np.vectorize(math.erfc)(-c * math.sqrt(0.5))
            return g * p, p + c * np.exp(-0.5 * c * c) / math.sqrt(2 * math.pi)
        if kind == i8.GELU_TANH:
            v = 2 * math.sqrt(2 / math.pi) * (c + 0.044715 * c ** 3)
            p, q = 1 / (1 + np.exp(-v)), 1 / (1 + np.exp(v))
            return g * p, p + c * p * q * 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * c * c)
    return np.maximum(g, 0), (g > 0).astype(np.float64)


def slack(g, kind, dtype=api.FH_F32):
    """How far the activation and its derivative may be off in fp32.  Functions: exponential and quotient within two steps (4 U), complementary error function within four
    (8 U), the normal distribution of bf16 results within 16 U besides its exponential; every product and sum rounds once.  A rounded argument moves an
    exponential by the argument's error: 4 U of it for gelu_tanh's g (A + B g^2), A and B rounded, 1.5 U for the error function's (whose logarithm has a slope of at most 2 x + 1.2), U for the density's square.  Where an exponential is below the normal
    numbers it is a multiple of 2^-149."""
    a, d = (np.abs(v) for v in exact(g, kind))
    c = np.clip(np.abs(g), 0, 1e3)
    least = (np.minimum(np.abs(g), 200.0) + 4) * 2.0 ** -149
    with np.errstate(all="ignore"):
        if kind == i8.SILU:
            p, q = 1 / (1 + np.exp(-np.clip(g, -1e3, 1e3))), 1 / (1 + np.exp(np.clip(g, -1e3, 1e3)))
            return 11 * U * a + least, 8 * U * p + 18 * U * p * np.minimum(np.abs(g), 1e3) * q + 12 * U * d + least
        if kind == i8.GELU:
            x = c * math.sqrt(0.5)
            arg = np.where(g < 0, (2 * x + 1.2) * 1.5 * U * x, 1.5 * U * x * np.exp(-x * x) * 1.2)
            p = a / np.where(c == 0, 1, np.abs(g))
            dens = c * np.exp(-0.5 * c * c) * 0.4
            phi = 8 * U if dtype == api.FH_F32 else 20 * U
            return (phi + 4 * U + arg) * a + least, (phi + 2 * U + arg) * p + (8 * U + 0.5 * c * c * 2 * U) * dens + U * d + 40 * least
        if kind == i8.GELU_TANH:
            v = 2 * math.sqrt(2 / math.pi) * (c + 0.044715 * c ** 3)
            e = 4 * U + np.minimum(v, 110.0) * 4 * U                 # of exp(-|v|)
            s = np.exp(-v)
            p = np.where(g < 0, s, 1) / (1 + s)
            off = np.where(g < 0, e, e * s / (1 + s))                # of p
            t = c * s / (1 + s) ** 2 * 1.6 * (1 + 0.135 * c * c)
            return (off + 7 * U) * a + least, (off + 5 * U) * p + (2 * e + 13 * U) * t + 2 * U * d + 200 * least
    return 0 * a, 0 * a


def grid():
    """Both signs, dense where activations change and on to where nothing is left of them."""
    near = np.concatenate([np.linspace(0.0, 6.0, 701), np.linspace(6.0, 30.0, 601), np.linspace(30.0, 110.0, 701)])
    return np.concatenate([near, -near]).astype(np.float32)


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows", [1, 40, 200])
def test_forward(rows, kind, dtype):
    """A common axis of one element: every g is a weight, and so is every u, whatever the token."""
    g = grid()
    f = g.size
    rng = np.random.default_rng(kind)
    x = np.full((rows, 1), 127.0, dtype=np.float32)
    gate, up = (g / 127).astype(np.float32).reshape(-1, 1), rng.uniform(0.5, 2.0, size=(f, 1)).astype(np.float32)
    parts = [torch.from_numpy(i8.compress(v)).cuda() for v in (x, gate, up)]
    h, pre = torch.empty(rows, f, dtype=TYPES[dtype], device="cuda"), torch.empty(rows, 2 * f, dtype=TYPES[dtype], device="cuda")
    assert api.fh_i8_gated(api.gated_desc(rows, f, 1, kind, dtype), *parts, h, pre) == api.FH_OK
    got, kept = h.double().cpu().numpy(), pre.double().cpu().numpy()
    if dtype == api.FH_F32:                                           # what the kernel made h of
        eg, eu = kept[:, :f], kept[:, f:]
        want = exact(eg, kind)[0]
        bound = np.abs(eu) * slack(eg, kind)[0] + U * np.abs(want * eu) + 2.0 ** -149
    else:                                                             # three roundings from the containers; the fast exponential 1.2 |g| steps more
        (qg, mg), (qu, mu) = i8.quantise(gate), i8.quantise(up)
        eg, eu = (np.broadcast_to((127 * q[:, 0] * i8.scales(m).astype(np.float64))[None, :], (rows, f)) for q, m in ((qg, mg), (qu, mu)))
        want = exact(eg, kind)[0]
        wide = np.minimum(np.abs(eg), 110.0) ** (3 if kind == i8.GELU_TANH else 2 if kind == i8.GELU else 1) + 1
        bound = np.abs(want * eu) * (HALF[dtype] * (1 + 1e-6) + 40 * U * np.minimum(wide, 200.0)) + np.abs(eu) * slack(eg, kind, dtype)[0] + 2.0 ** -133
    assert np.isfinite(got).all()
    assert (np.abs(got - want * eu) <= bound).all()


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("extra", [0, 1])
def test_backward(extra, kind, dtype):
    """dh = u = 1: the derivative, and the activation.  On to the largest numbers."""
    far = np.exp2(np.arange(7, 128)).astype(np.float32) * np.float32(1.3)
    g = torch.from_numpy(np.concatenate([grid(), far, -far])).to(TYPES[dtype])
    f = g.numel()
    pre = torch.ones(2, 2 * f + extra, dtype=TYPES[dtype], device="cuda")
    pre[:, :f] = g.cuda()
    dh, out = torch.ones(2, f, dtype=TYPES[dtype], device="cuda"), torch.empty_like(pre)
    d = api.gated_desc(2, f, 1, kind, dtype, f, 2 * f + extra)
    assert api.fh_gated_backward(d, dh, pre[:, :2 * f], out[:, :2 * f]) == api.FH_OK
    v = g.double().numpy()
    (a, slope), (ea, es) = exact(v, kind), slack(v, kind, dtype)
    for row in out.double().cpu().numpy():
        for got, want, e in ((row[:f], slope, es), (row[f:2 * f], a, ea)):
            assert np.isfinite(got).all()
            assert (np.abs(got - want) <= e + HALF[dtype] * (1 + 1e-6) * np.abs(want) + 2.0 ** -133 * (dtype == api.FH_BF16)).all()


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
@pytest.mark.parametrize("kind", KINDS)
def test_nan_stays_in_its_place(kind, dtype):
    pre, dh, out = (torch.ones(3, n, dtype=TYPES[dtype], device="cuda") for n in (64, 32, 64))
    pre[1, 5] = float("nan")
    assert api.fh_gated_backward(api.gated_desc(3, 32, 1, kind, dtype), dh, pre, out) == api.FH_OK
    bad = out.isnan().nonzero().tolist()
    assert [1, 32 + 5] in bad and ([1, 5] in bad or kind == api.FH_RELU) and len(bad) <= 2    # (relu's derivative: not above zero)


@pytest.mark.parametrize("dtype", [api.FH_F32, api.FH_BF16])
def test_what_relu_takes_out_is_zero(dtype):
    """dh u is beyond the largest number there."""
    pre, dh, out = torch.full((2, 64), 1e30, dtype=TYPES[dtype], device="cuda"), torch.full((2, 32), 1e30, dtype=TYPES[dtype], device="cuda"), torch.empty(2, 64, dtype=TYPES[dtype], device="cuda")
    pre[:, :32] = -1.0
    assert api.fh_gated_backward(api.gated_desc(2, 32, 1, api.FH_RELU, dtype), dh, pre, out) == api.FH_OK
    assert (out == 0).all()
