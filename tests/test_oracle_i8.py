"""Pins of the plain definition of 8-bit matrices, the gated block and the norms of heads: hand cases, exact rational arithmetic, gradients against
differences."""
from fractions import Fraction

import numpy as np
import pytest

from oracle import i8


def test_hand_cases():
    x = np.array([[127.0, -1.0, 0.5, 1.5, -2.5, 126.5], [0, 0, 0, 0, 0, -0.0], [1e-45, 0, 0, 0, 0, -1e-45], [1, np.nan, 0, 0, 0, 0],
                  [np.inf, 1, 0, 0, 0, 0], [-254, 1, 3, 5, 2, 253]], dtype=np.float32)
    q, a = i8.quantise(x)
    assert q.tolist() == [[127, -1, 0, 2, -2, 126], [0] * 6, [0] * 6, [0] * 6, [0] * 6, [-127, 0, 2, 2, 1, 126]]
    assert a[0] == 127 and a[1] == 0 and a[2] == np.float32(1e-45) and np.isnan(a[3]) and np.isnan(a[4]) and a[5] == 254
    s = i8.scales(a)
    assert s[0] == 1 and s[1] == 0 and s[2] == np.float32(2.0 ** -126) and np.isnan(s[3]) and s[5] == 2


def test_codes_are_the_nearest_whole_numbers():
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((40, 50)) * np.exp(8 * rng.standard_normal((40, 1)))).astype(np.float32)
    x[:, 7] = (x[:, 0] * np.float32(0.5))
    q, a = i8.quantise(x)
    for r in range(40):
        s = Fraction(float(i8.scales(a)[r]))
        for c in range(50):
            t = Fraction(float(x[r, c])) / s
            assert q[r, c] == round(t)                              # (Python rounds a tie to the even neighbour)
        assert abs(q[r]).max() == 127


@pytest.mark.parametrize("shape", [(1, 1), (8, 32), (9, 33), (128, 64), (130, 17), (300, 100)])
def test_containers_hold_what_was_put_in(shape):
    rng = np.random.default_rng(2)
    x = rng.standard_normal(shape).astype(np.float32)
    buf = i8.compress(x)
    assert buf.size == i8.sizes(*shape)[2]
    q, a = i8.unpack(buf, *shape)
    assert np.array_equal(q, i8.quantise(x)[0]) and np.array_equal(a, np.abs(x).max(axis=1))
    assert (np.abs(i8.restore(buf, *shape) - x) <= (0.5 + 1e-6) * i8.scales(a)[:, None]).all()


def test_a_rows_16_bytes_are_where_the_description_says():
    x = np.zeros((140, 70), dtype=np.float32)
    x[:, 0] = 127
    x[131, 37] = 5
    buf = i8.compress(x)
    assert buf[128 + 128 * 96 + (2 * 16 + 3) * 16 + 5] == 5     # second block: 16 rows (140 - 128, padded to 8); chunk 2, row 3 of it, byte 5
    x[131, 37], x[127, 69] = 0, 6
    assert i8.compress(x)[128 + (4 * 128 + 127) * 16 + 5] == 6


def differences(f, x, h):
    out = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        up, down = x.copy(), x.copy()
        up[i] += h
        down[i] -= h
        out[i] = (f(up) - f(down)) / (2 * h)
    return out


@pytest.mark.parametrize("kind", [i8.SILU, i8.GELU, i8.GELU_TANH, i8.RELU])
def test_the_gated_blocks_gradient_against_differences(kind):
    rng = np.random.default_rng(3)
    g, u, dh = (rng.standard_normal((3, 5)) + 0.1 for _ in range(3))
    f = lambda p: (dh * i8.act(p[:, :5], kind)[0] * p[:, 5:]).sum()  # noqa: E731
    want = differences(f, np.concatenate([g, u], axis=1), 1e-5)
    assert np.abs(i8.gated_backward(dh, g, u, kind) - want).max() < 1e-8      # (h^2 times a third derivative, and 1e-16 / h)


@pytest.mark.parametrize("kind", [i8.RMS, i8.LAYER])
@pytest.mark.parametrize("pairs", [i8.HALVES, i8.NEIGHBOURS])
@pytest.mark.parametrize("rotary", [0, 4, 6])
def test_the_heads_gradient_against_differences(kind, pairs, rotary):
    rng = np.random.default_rng(4)
    x, dy, gamma = rng.standard_normal((2, 3, 6)), rng.standard_normal((2, 3, 6)), 1 + 0.3 * rng.standard_normal(6)
    cs = i8.table(9, max(rotary, 2))[[7, 2]]
    f = lambda v, w: (dy * i8.head_norm(v, w, cs, rotary, kind, pairs, 1e-3)).sum()  # noqa: E731
    dx, dgamma = i8.head_norm_backward(dy, x, gamma, cs, rotary, kind, pairs, 1e-3)
    assert np.abs(dx - differences(lambda v: f(v, gamma), x, 1e-5)).max() < 1e-8
    assert np.abs(dgamma - differences(lambda w: f(x, w), gamma, 1e-5)).max() < 1e-8


def test_the_rotation_keeps_lengths_and_adds_up():
    rng = np.random.default_rng(5)
    z = rng.standard_normal((4, 2, 10))
    t = i8.table(50, 8)
    for pairs in (i8.HALVES, i8.NEIGHBOURS):
        turned = i8._turned(i8._turned(z, t[[3, 5, 7, 9]], 8, pairs, False), t[[30, 20, 10, 0]], 8, pairs, False)
        assert np.abs(turned - i8._turned(z, t[[33, 25, 17, 9]], 8, pairs, False)).max() < 1e-12
        assert np.abs((turned ** 2).sum(axis=-1) - (z ** 2).sum(axis=-1)).max() < 1e-12
