"""Weights in 4-bit floats with a scale of a power of two per 32, and the products
with them, plainly. NumPy on the CPU, in 64 bits."""
import math

import numpy as np

GROUP = 32
MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
VALUES = np.concatenate([MAGNITUDES, -MAGNITUDES])
LEAST = 2.0 ** -96


def scale_byte(top):
    """The smallest e with top <= 7 * 2^e, as a byte; NaN where top is not finite."""
    if not np.isfinite(top):
        return 255
    top, e = max(float(top), LEAST), -127
    while top > 7 * 2.0 ** e:
        e += 1
    return e + 127


def nearest_code(v):
    """Codes of the nearest magnitudes, ties to the even code, beyond 6 to 6; the sign by its bit."""
    v = np.asarray(v, np.float64)
    a = np.minimum(np.abs(v), 6.0)
    far = np.abs(a[..., None] - MAGNITUDES)
    near = far == far.min(-1, keepdims=True)
    low = near.argmax(-1)
    code = np.where(near.sum(-1) == 2, low + low % 2, low)
    return (code + 8 * np.signbit(v)).astype(np.uint8)


def quantize(x):
    """Codes [n][ceil(k/32)*32] and scales [ceil(k/128)][n][4]."""
    x = np.asarray(x, np.float64)
    n, k = x.shape
    codes = np.zeros((n, -(-k // GROUP) * GROUP), np.uint8)
    scales = np.full((-(-k // 128), n, 4), scale_byte(0.0), np.uint8)
    for i in range(n):
        for c in range(0, k, GROUP):
            part = x[i, c:c + GROUP]
            byte = scale_byte(np.abs(part).max())
            scales[c // 128, i, c % 128 // GROUP] = byte
            if byte != 255:
                codes[i, c:c + len(part)] = nearest_code(part / 2.0 ** (byte - 127))
    return codes, scales


def pack(codes):
    return codes[:, 0::2] | codes[:, 1::2] << 4


def unpack(held):
    return np.stack([held & 15, held >> 4], -1).reshape(held.shape[0], -1)


def values(codes, scales, k):
    """What codes and scales stand for, [n][k]."""
    s = scales.astype(np.float64).transpose(1, 0, 2).reshape(scales.shape[1], -1)
    s = np.where(s == 255, np.nan, 2.0 ** (s - 127))
    return VALUES[codes[:, :k]] * np.repeat(s, GROUP, 1)[:, :k]


def activate(g, kind):
    """kind as in the header: 1, 2, 3."""
    if kind == 1:
        with np.errstate(over="ignore"):
            return g / (1 + np.exp(-g))
    if kind == 2:
        return g * np.vectorize(math.erfc, otypes=[np.float64])(-g / math.sqrt(2)) / 2
    with np.errstate(over="ignore"):
        return g / (1 + np.exp(-2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)))
