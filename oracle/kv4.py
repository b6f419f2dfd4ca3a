"""Tokens that enter a cache, and rows in 4 bits, in float64 (test oracle; see package header).

The paper takes the cache as given (Sec. 2.1) and names quantisation of the key/value vectors as its next step
(Appendix C); the scheme here is this build's reading, in the E2M1 / E8M0 formats of the OCP microscaling specification:
a row of 128 values is cut into blocks of 32; a block's scale is the least power of two 2^k, k >= -125, with which no
magnitude exceeds 6; a value over the scale becomes the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6 with its sign, ties to the even
code; the scale byte is k + 127. A block with a value that is not finite, or of 2^127 or more, has scale byte 255 and
codes of zero, and reads as NaN. Even dimensions are the low halves of the bytes.

A token's query and key heads are normed, x / sqrt(mean(x^2) + eps) * weight, and rotated: a pair (a, b) at position p becomes
(a cos - b sin, b cos + a sin) of the angle p * inv_freq[i]; pairs are (i, i + rot / 2) or, interleaved, (2 i, 2 i + 1).
"""
import numpy as np

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize_rows(X):
    """X [..., 128] (float32 values) -> (codes uint8 [..., 64], scale uint8 [..., 4])."""
    X = np.asarray(X, np.float32).astype(np.float64)
    B = X.reshape(-1, 32)
    codes = np.zeros(B.shape, np.uint8)
    scale = np.zeros(len(B), np.uint8)
    for i, b in enumerate(B):
        top = np.abs(b).max() if np.all(np.isfinite(b)) else np.inf
        if not top < 2.0 ** 127:
            scale[i] = 255
            continue
        k = -125
        while top > 6.0 * 2.0 ** k:
            k += 1
        scale[i] = k + 127
        y = np.abs(b) / 2.0 ** k
        far = np.abs(y[:, None] - GRID[None, :])
        # nearest; of two equally near ones the even code
        order = far + np.where(np.arange(8) % 2 == 1, 1e-9, 0.0)[None, :] * (far == far.min(axis=1, keepdims=True))
        codes[i] = order.argmin(axis=1) + 8 * np.signbit(b)
    codes = codes.reshape(*X.shape[:-1], 64, 2)
    return codes[..., 0] | (codes[..., 1] << 4), scale.reshape(*X.shape[:-1], 4)


def dequantize_rows(codes, scale):
    """-> float64 [..., 128], the values they stand for."""
    codes, scale = np.asarray(codes), np.asarray(scale)
    c = np.stack((codes & 15, codes >> 4), axis=-1).reshape(*codes.shape[:-1], 128)
    v = np.where(c >= 8, -1.0, 1.0) * GRID[c & 7]
    unit = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127.0))
    return v * np.repeat(unit, 32, axis=-1)


def head_rows(x, pos, weight=None, eps=1e-6, inv_freq=None, interleaved=False):
    """Norm and rotation of rows x [T][heads][128] of the tokens at positions pos [T] -> (float64 rows, for every
    value the sum of the magnitudes it is made of, which bounds its rounding)."""
    x = np.asarray(x, np.float64)
    if weight is not None:
        x = x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    out, size = x.copy(), np.abs(x)
    if inv_freq is not None:
        rot = 2 * len(inv_freq)
        i = np.arange(rot // 2)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        ang = np.asarray(pos, np.float64)[:, None, None] * np.asarray(inv_freq, np.float64)
        c, s = np.cos(ang), np.sin(ang)
        out[..., a], out[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a], size[..., b] = np.abs(x[..., a]) + np.abs(x[..., b]), np.abs(x[..., a]) + np.abs(x[..., b])
    return out, size
