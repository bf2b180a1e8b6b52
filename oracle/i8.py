"""Plain definition of matrices in 8-bit integers (include/fh.h describes format and container), of the gated feed-forward block and of the norms of heads
with the rotation by position, in NumPy and 64 bits.  Test infrastructure only."""
from __future__ import annotations

import math

import numpy as np

SILU, GELU, GELU_TANH, RELU = 0, 1, 2, 3
RMS, LAYER = 0, 1
HALVES, NEIGHBOURS = 0, 1


def sizes(rows: int, cols: int):
    """(padded rows, padded columns, total bytes)."""
    r8, kp = -(-rows // 8) * 8, -(-cols // 32) * 32
    return r8, kp, 128 + r8 * kp + 4 * r8


def magnitudes(x) -> np.ndarray:
    x = np.asarray(x, dtype=np.float32)
    a = np.abs(x).max(axis=1)
    return np.where(np.isfinite(x).all(axis=1), a, np.float32("nan")).astype(np.float32)


def scales(a) -> np.ndarray:
    """fp32 scales of fp32 magnitudes."""
    a = np.asarray(a, dtype=np.float32)
    s = np.maximum(a * (np.float32(1) / np.float32(127)), np.float32(2.0 ** -126))
    return np.where(a == 0, np.float32(0), np.where(np.isnan(a), a, s)).astype(np.float32)


def quantise(x):
    """(codes as int64, magnitudes): the quotient's nearest whole number, a tie to the even one.  (Quotients of two 24-bit numbers are no nearer than
    2^-31 to a tie that they are not, which 53 bits tell.)"""
    x = np.asarray(x, dtype=np.float32)
    a = magnitudes(x)
    s = scales(a).astype(np.float64)
    live = np.isfinite(s) & (s > 0)
    q = np.rint(np.where(live[:, None], x, 0).astype(np.float64) / np.where(live, s, 1.0)[:, None])
    return q.astype(np.int64), a


def compress(x) -> np.ndarray:
    """The container's bytes."""
    rows, cols = x.shape
    r8, kp, total = sizes(rows, cols)
    q, a = quantise(x)
    codes = np.zeros((r8, kp), dtype=np.int8)
    codes[:rows, :cols] = q
    out = np.zeros(total, dtype=np.uint8)
    out[:4] = np.frombuffer(b"FHI8", dtype=np.uint8)
    out[4] = 1
    out[8:16] = np.array([rows, cols], dtype=np.int32).view(np.uint8)
    out[24:32] = np.array([total], dtype=np.uint64).view(np.uint8)
    at = 128
    for b in range(0, r8, 128):
        block = codes[b:b + 128].view(np.uint8).reshape(min(128, r8 - b), kp // 16, 16).transpose(1, 0, 2)
        out[at:at + block.size] = block.reshape(-1)
        at += block.size
    m = np.zeros(r8, dtype=np.float32)
    m[:rows] = a
    bits = m.view(np.uint32)
    bits[np.isnan(m)] = 0x7FC00000
    out[at:] = bits.view(np.uint8)
    return out


def unpack(buf, rows: int, cols: int):
    """(codes, magnitudes) of a container."""
    r8, kp, total = sizes(rows, cols)
    codes, at = np.zeros((r8, kp), dtype=np.int8), 128
    for b in range(0, r8, 128):
        n = min(128, r8 - b)
        codes[b:b + n] = buf[at:at + n * kp].reshape(kp // 16, n, 16).transpose(1, 0, 2).reshape(n, kp).view(np.int8)
        at += n * kp
    return codes[:rows, :cols].astype(np.int64), np.ascontiguousarray(buf[at:total]).view(np.float32)[:rows]


def restore(buf, rows: int, cols: int) -> np.ndarray:
    """The values in 64 bits."""
    q, a = unpack(buf, rows, cols)
    return q * scales(a).astype(np.float64)[:, None]


def act(g, kind: int):
    """(activation, its derivative), element by element in 64 bits."""
    g = np.asarray(g, dtype=np.float64)
    with np.errstate(over="ignore"):
        if kind == SILU:
            p = 1 / (1 + np.exp(-g))
            return g * p, p * (1 + g * (1 - p))
        if kind == GELU:
            p = 0.5 * np.vectorize(math.erfc)(-g * math.sqrt(0.5))
            return g * p, p + g * np.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
        if kind == GELU_TANH:
            c = math.sqrt(2 / math.pi)
            w = c * (g + 0.044715 * g ** 3)
            p, q = 1 / (1 + np.exp(-2 * w)), 1 / (1 + np.exp(2 * w))    # (1 +- tanh w) / 2, which in itself would leave nothing of far values
            return g * p, p + 2 * g * p * q * c * (1 + 3 * 0.044715 * g * g)
    return np.maximum(g, 0), (g > 0).astype(np.float64)


def gated_backward(dh, g, u, kind: int) -> np.ndarray:
    a, slope = act(g, kind)
    return np.concatenate([dh * u * slope, dh * a], axis=1)


def table(positions: int, rotary: int, base: float = 10000.0, scale: float = 1.0) -> np.ndarray:
    angle = np.arange(positions, dtype=np.float64)[:, None] * base ** (-np.arange(0, rotary, 2, dtype=np.float64) / rotary) * scale
    return np.stack([np.cos(angle), np.sin(angle)], axis=-1)


def _turned(z, cs, rotary: int, pairs: int, back: bool):
    """z [tokens, heads, dim] turned by cs [tokens, rotary / 2, 2], or back."""
    c, n = cs[:, None, :, 0], cs[:, None, :, 1] * (-1 if back else 1)
    first = slice(0, rotary // 2) if pairs == HALVES else slice(0, rotary, 2)
    second = slice(rotary // 2, rotary) if pairs == HALVES else slice(1, rotary, 2)
    out = z.copy()
    out[..., first] = z[..., first] * c - z[..., second] * n
    out[..., second] = z[..., second] * c + z[..., first] * n
    return out


def _unit(x, kind: int, eps: float):
    x = np.asarray(x, dtype=np.float64)
    if kind == LAYER:
        x = x - x.mean(axis=-1, keepdims=True)
    rstd = 1 / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps)
    return x * rstd, rstd


def head_norm(x, gamma, cs, rotary: int, kind: int, pairs: int, eps: float) -> np.ndarray:
    """x [tokens, heads, dim], gamma [dim] or None, cs [tokens, rotary / 2, 2]."""
    z = _unit(x, kind, eps)[0] * (1.0 if gamma is None else np.asarray(gamma, dtype=np.float64))
    return _turned(z, cs, rotary, pairs, False) if rotary else z


def head_norm_backward(dy, x, gamma, cs, rotary: int, kind: int, pairs: int, eps: float):
    """(dx, dgamma)."""
    xhat, rstd = _unit(x, kind, eps)
    dz = np.asarray(dy, dtype=np.float64)
    if rotary:
        dz = _turned(dz, cs, rotary, pairs, True)
    g = dz * (1.0 if gamma is None else np.asarray(gamma, dtype=np.float64))
    dx = g - xhat * (g * xhat).mean(axis=-1, keepdims=True)
    if kind == LAYER:
        dx = dx - g.mean(axis=-1, keepdims=True)
    return dx * rstd, (dz * xhat).sum(axis=(0, 1))
