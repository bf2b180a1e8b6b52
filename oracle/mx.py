"""Plain definition of matrices in microscaled 4-bit floating point (include/fh.h describes format and container), of their
products and of the layer norm, in NumPy and 64 bits.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

B32, B16 = 0, 1
BLOCK = (32, 16)
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDS = (LEVELS[1:] + LEVELS[:-1]) / 2
# every scale of a format, ascending, at its byte (B16: without the factor 2^exponent; byte 0 is no scale that compressing gives)
SCALES = (np.array([2.0 ** k for k in range(-127, 126)]),
          np.array([m * 2.0 ** -9 for m in range(8)] + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)])[:127])


def bf16(bits) -> np.ndarray:
    return (np.ascontiguousarray(bits).view(np.uint16).astype(np.uint32) << 16).view(np.float32)


def to_bf16(x) -> np.ndarray:
    """Bit patterns of fp32 values rounded to bf16 (to nearest, ties to even); finite values only."""
    u = np.asarray(x, dtype=np.float32).view(np.uint32)
    return ((u + 0x7FFF + (u >> 16 & 1)) >> 16).astype(np.uint16)


def draws(rows: int, cols: int, seed: int, tensor_id: int) -> np.ndarray:
    """16 bits for each element: Philox-4x32-10 (Salmon et al., SC'11), eight a call."""
    g, m32 = -(-cols // 8), np.uint64(0xFFFFFFFF)
    c = [np.broadcast_to(np.arange(g, dtype=np.uint64), (rows, g)).copy(), np.broadcast_to(np.arange(rows, dtype=np.uint64)[:, None], (rows, g)).copy(),
         np.full((rows, g), tensor_id & 0xFFFFFFFF, dtype=np.uint64), np.full((rows, g), tensor_id >> 32, dtype=np.uint64)]
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), q & m32, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p & m32]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    out = np.stack([part for w in c for part in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1)
    return out.reshape(rows, 8 * g)[:, :cols].astype(np.int64)


def quantise(x, fmt: int, exponent: int = 0, rounding: int = 0, seed: int = 0, tensor_id: int = 0):
    """(codes [rows, cols], scale bytes [rows, blocks]) of a float matrix."""
    rows, cols = x.shape
    bs = BLOCK[fmt]
    pad = -cols % bs
    v = np.pad(np.asarray(x, dtype=np.float64), ((0, 0), (0, pad))).reshape(rows, -1, bs)
    bad = ~np.isfinite(v).all(axis=2)
    v = np.where(bad[:, :, None], 0.0, v) * 2.0 ** -exponent
    mag = np.abs(v)
    table = SCALES[fmt]
    least = 1 if fmt == B16 else 0
    byte = np.clip(np.searchsorted(6 * table, mag.max(axis=2)), least, len(table) - 1)
    s = table[byte][:, :, None]
    if rounding == 0:
        code = np.zeros(mag.shape, dtype=np.int64)
        for i, m in enumerate(MIDS):
            code += (mag >= m * s) if i % 2 else (mag > m * s)      # a tie goes to the even code
    else:
        low = np.zeros(mag.shape, dtype=np.int64)
        for lv in LEVELS[1:]:
            low += mag >= lv * s
        step = np.append(LEVELS[1:] - LEVELS[:-1], 0.0)[low] * s
        r = np.pad(draws(rows, cols, seed, tensor_id), ((0, 0), (0, pad))).reshape(mag.shape)
        code = low + ((low < 7) & ((mag - LEVELS[low] * s) * 65536 > step * (r + 0.5)))
    code |= np.signbit(v).astype(np.int64) << 3
    code[bad] = 0
    byte = np.where(bad, 255 if fmt == B32 else 127, byte)
    return code.reshape(rows, -1)[:, :cols], byte


def sizes(rows: int, cols: int, fmt: int):
    r8, kp = -(-rows // 8) * 8, -(-cols // 64) * 64
    atoms = -(-kp // (4 * BLOCK[fmt]))
    return r8, kp, atoms, 128 + r8 * kp // 2 + -(-rows // 128) * atoms * 512


def code_offsets(rows: int, cols: int, fmt: int) -> np.ndarray:
    """Byte of the container that holds columns 2i, 2i + 1 of a row: [r8, kp / 2]."""
    r8, kp, _, _ = sizes(rows, cols, fmt)
    r, i = np.arange(r8)[:, None], np.arange(kp // 2)[None, :]
    rb = np.minimum(128, r8 - r // 128 * 128)
    return 128 + r // 128 * 128 * (kp // 2) + (i // 16 * rb + r % 128) * 16 + i % 16


def scale_offsets(rows: int, cols: int, fmt: int) -> np.ndarray:
    r8, kp, atoms, _ = sizes(rows, cols, fmt)
    r, b = np.arange(rows)[:, None], np.arange(-(-cols // BLOCK[fmt]))[None, :]
    return 128 + r8 * kp // 2 + (r // 128 * atoms + b // 4) * 512 + r % 32 * 16 + r % 128 // 32 * 4 + b % 4


def compress(x, fmt: int, exponent: int = 0, rounding: int = 0, seed: int = 0, tensor_id: int = 0) -> np.ndarray:
    rows, cols = x.shape
    r8, kp, _, total = sizes(rows, cols, fmt)
    code, byte = quantise(x, fmt, exponent, rounding, seed, tensor_id)
    code = np.pad(code, ((0, r8 - rows), (0, kp - cols)))
    buf = np.zeros(total, dtype=np.uint8)
    buf[code_offsets(rows, cols, fmt)] = code[:, 0::2] | code[:, 1::2] << 4
    buf[scale_offsets(rows, cols, fmt)] = byte
    buf[:4] = np.frombuffer(b"FHM4", dtype=np.uint8)
    buf[4:8] = [1, 0, fmt, rounding]
    buf[8:20] = np.array([rows, cols, exponent], dtype=np.int32).view(np.uint8)
    buf[24:40] = np.array([total, tensor_id], dtype=np.uint64).view(np.uint8)
    return buf


def restore(buf, rows: int, cols: int, fmt: int) -> np.ndarray:
    exponent = int(np.ascontiguousarray(buf[16:20]).view(np.int32)[0])
    pair = buf[code_offsets(rows, cols, fmt)[:rows]].astype(np.int64)
    code = np.stack([pair & 15, pair >> 4], axis=-1).reshape(rows, -1)[:, :cols]
    byte = buf[scale_offsets(rows, cols, fmt)].astype(np.int64)
    s = np.where(byte == (255 if fmt == B32 else 127), np.nan, SCALES[fmt][np.minimum(byte, len(SCALES[fmt]) - 1)]) * 2.0 ** exponent
    v = LEVELS[code & 7] * np.where(code & 8, -1.0, 1.0)
    return v * np.repeat(s, BLOCK[fmt], axis=1)[:, :cols]


def layer_norm(x, gamma, beta, eps: float):
    """(y, mean, rstd)."""
    x = np.asarray(x, dtype=np.float64)
    mean = x.mean(axis=1)
    rstd = 1 / np.sqrt(((x - mean[:, None]) ** 2).mean(axis=1) + eps)
    y = (x - mean[:, None]) * rstd[:, None]
    return y * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta), mean, rstd


def layer_norm_backward(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta)."""
    dy, rstd = np.asarray(dy, dtype=np.float64), np.asarray(rstd, dtype=np.float64)[:, None]
    xhat = (x - np.asarray(mean, dtype=np.float64)[:, None]) * rstd
    g = dy * (1.0 if gamma is None else gamma)
    dx = rstd * (g - g.mean(axis=1, keepdims=True) - xhat * (g * xhat).mean(axis=1, keepdims=True))
    return dx, (dy * xhat).sum(axis=0), dy.sum(axis=0)
