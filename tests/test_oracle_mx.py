"""Pins of the plain definition of microscaled 4-bit matrices: values worked out by hand, and laws that any such quantiser has."""
import numpy as np
import pytest

from oracle import mx


def held(x, fmt, **kw):
    x = np.asarray(x, dtype=np.float64).reshape(1, -1)
    return mx.restore(mx.compress(x, fmt, **kw), 1, x.shape[1], fmt)[0]


def test_levels_and_ties_by_hand():
    # largest 6: the scale is 1 in either format, so values round to 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code
    x = [6, 0.25, 0.2500001, 0.75, 1.25, 1.75, 2.5, 3.5, 5, -5, 0.7499999, -0.1, 5.0001]
    want = [6, 0, 0.5, 1, 1, 2, 2, 4, 4, -4, 0.5, -0.0, 6]
    for fmt in (mx.B32, mx.B16):
        assert held(x, fmt).tolist() == want


def test_scales_by_hand():
    # the smallest scale with 6 * scale >= the largest magnitude
    for top, byte in ((6.0, 127), (6.0001, 128), (12.0, 128), (3.0, 126), (3.1, 127), (0.0, 0), (2.0 ** -149, 0), (3.4e38, 252)):
        assert mx.quantise(np.array([[top]]), mx.B32)[1][0, 0] == byte, top
    # E4M3: 1 = 0x38, 1.125 = 0x39; 2^-9 is byte 1, 448 byte 126
    for top, byte in ((6.0, 0x38), (6.01, 0x39), (6.75, 0x39), (6.76, 0x3A), (0.0, 1), (1e-9, 1), (6 * 2.0 ** -9, 1), (6.1 * 2.0 ** -9, 2),
                      (2688.0, 126), (1e9, 126)):
        assert mx.quantise(np.array([[top]]), mx.B16)[1][0, 0] == byte, top
    assert mx.quantise(np.array([[6.0 * 2 ** 10]]), mx.B16, exponent=10)[1][0, 0] == 0x38


def test_container_by_hand():
    # one row of 64 columns: header, 8 rows of codes (two chunks of 8 x 16 bytes), one group of scales
    x = np.zeros((1, 64))
    x[0, 0], x[0, 1], x[0, 33], x[0, 63] = 6.0, -3.0, 1.0, 12.0
    buf = mx.compress(x, mx.B32, tensor_id=7)
    assert buf.size == 128 + 8 * 32 + 512 and bytes(buf[:4]) == b"FHM4" and buf[32] == 7
    assert buf[128] == 0x7 | 0xD << 4 and buf[128 + 128 + 0] == 0x1 << 4 and buf[128 + 128 + 15] == 0x7 << 4
    assert buf[384:388].tolist() == [127, 128, 0, 0]
    # row 40 of 41: its scales are the second word of lane 8
    x = np.zeros((41, 32))
    x[40, 0] = 6.0
    buf = mx.compress(x, mx.B32)
    assert buf.size == 128 + 48 * 32 + 512 and buf[128 + 40 * 16] == 7 and buf[128 + 48 * 32 + 8 * 16 + 4] == 127


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
def test_error_is_within_half_a_step_and_holding_twice_in_b32_changes_nothing(fmt):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal((40, 100)) * np.exp(3 * rng.standard_normal((40, 1)))).astype(np.float32).astype(np.float64)
    y = mx.restore(mx.compress(x, fmt), 40, 100, fmt)
    bs = mx.BLOCK[fmt]
    top = np.repeat(np.abs(np.pad(x, ((0, 0), (0, -100 % bs)))).reshape(40, -1, bs).max(axis=2), bs, axis=1)[:, :100]
    # the widest step is 2 scales.  A power of two is less than a third of the largest magnitude; an E4M3 scale is at most the distance
    # to its lower neighbour beyond a sixth t of it, and neighbours around t are max(t / 8, 2^-9) apart.  Beyond 6 * 448 nothing is said.
    scale = top / 3 if fmt == mx.B32 else top / 6 + np.maximum(top / 48, 2.0 ** -9)
    assert (np.abs(x - y) <= np.where((fmt == mx.B16) & (top > 2688), np.inf, scale)).all()
    # (not so for B16: with the scale 3 * 2^-9 a largest magnitude may become 4 scales, and 12 * 2^-9 is 6 of 2 * 2^-9)
    assert fmt == mx.B16 or np.array_equal(mx.restore(mx.compress(y, fmt), 40, 100, fmt), y)


def test_non_finite_blocks_are_nan_and_alone():
    x = np.ones((2, 64))
    x[0, 5], x[1, 40] = np.nan, -np.inf
    for fmt in (mx.B32, mx.B16):
        bs = mx.BLOCK[fmt]
        y = mx.restore(mx.compress(x, fmt), 2, 64, fmt)
        assert np.isnan(y[0, :bs]).all() and np.isnan(y[1, 40 // bs * bs:40 // bs * bs + bs]).all() and np.isnan(y).sum() == 2 * bs


@pytest.mark.parametrize("fmt", [mx.B32, mx.B16])
def test_random_rounding_is_unbiased_and_takes_neighbours(fmt):
    x = np.tile(np.array([6.0, 0.1, 0.6, 1.3, 2.2, 3.9, 4.5, -5.5, 1.0, 0.0, 0.4, 1.9, 2.9, 3.1, -0.3, 5.0]), (4096, 2))
    y = mx.restore(mx.compress(x, fmt, rounding=1, seed=11, tensor_id=2), 4096, 32, fmt)
    for c in range(32):
        lo = mx.LEVELS[mx.LEVELS <= abs(x[0, c])].max()
        hi = mx.LEVELS[mx.LEVELS >= abs(x[0, c])].min()
        assert set(np.abs(y[:, c])) <= {lo, hi}
        # the mean of 4096 draws between neighbours: five standard deviations are 5 (hi - lo) / 2 / 64
        assert abs(np.abs(y[:, c]).mean() - abs(x[0, c])) <= 5 * (hi - lo) / 128


def test_draws_by_hand():
    # Philox-4x32-10 of counter 0, key 0 (known answer of the generator's authors)
    assert mx.draws(1, 8, 0, 0)[0].tolist() == [v for w in (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8) for v in (w & 0xFFFF, w >> 16)]


def test_layer_norm_gradients_against_differences():
    rng = np.random.default_rng(1)
    x, gamma, beta, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    _, mean, rstd = mx.layer_norm(x, gamma, beta, 1e-3)
    dx, dgamma, dbeta = mx.layer_norm_backward(dy, x, gamma, mean, rstd)
    h = 1e-6
    loss = lambda a, g, b: (dy * mx.layer_norm(a, g, b, 1e-3)[0]).sum()  # noqa: E731
    for i in range(3):
        for j in range(7):
            e = np.zeros((3, 7))
            e[i, j] = h
            # central differences: truncation h^2, rounding 2^-53 * |loss| / h, both below 1e-8
            assert abs((loss(x + e, gamma, beta) - loss(x - e, gamma, beta)) / (2 * h) - dx[i, j]) < 1e-7
    for j in range(7):
        e = np.zeros(7)
        e[j] = h
        assert abs((loss(x, gamma + e, beta) - loss(x, gamma - e, beta)) / (2 * h) - dgamma[j]) < 1e-7
        assert abs((loss(x, gamma, beta + e) - loss(x, gamma, beta - e)) / (2 * h) - dbeta[j]) < 1e-7
