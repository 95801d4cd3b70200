"""Microscaled 4-bit floating point: the definitions written out in numpy.
Blocks of 32 along a row share a power of two; a value is one of 0, 0.5, 1, 1.5,
2, 3, 4, 6 and a sign, times it."""
import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def ld(cols):
    return (cols + 255) // 256 * 256


def quantise(x):
    """(codes [rows, ld] of 0 .. 15 one by one, exponent bytes [rows, ld / 32]) of rows x."""
    with np.errstate(over="ignore"):
        x = np.asarray(x, np.float64).astype(np.float32).astype(np.float64)
    n, K = x.shape
    v = np.zeros((n, ld(K)))
    v[:, :K] = x
    v = v.reshape(n, -1, 32)
    a = np.abs(v).max(2)
    bad = ~np.isfinite(a)
    live = ~bad & (a >= 2.0 ** -100)
    m, e = np.frexp(np.where(live, a, 1.0))                  # a = m 2^e with m in [0.5, 1)
    exponent = e - 1 + (m >= 0.875) - 2
    u = np.abs(np.where(live[:, :, None], v, 0.0)) / 2.0 ** exponent[:, :, None]
    low = np.clip(np.searchsorted(VALUES, u, side="right") - 1, 0, 6)
    lo, hi = VALUES[low], VALUES[low + 1]
    up = (u - lo > hi - u) | ((u - lo == hi - u) & (low % 2 == 1))
    q = low + up
    q = np.where(np.signbit(v) & live[:, :, None], q + 8, q)
    return q.reshape(n, -1), np.where(live, exponent + 127, np.where(bad, 255, 0))


def values(q, e):
    """[rows, ld] float64 of codes and exponent bytes; NaN for byte 255."""
    v = np.where(q & 8, -1.0, 1.0) * VALUES[q & 7]
    scale = np.where(e == 255, np.nan, 2.0 ** (np.asarray(e, np.float64) - 127))
    with np.errstate(invalid="ignore"):
        return (v.reshape(len(q), -1, 32) * scale[:, :, None]).reshape(len(q), -1)


def pack(q, e):
    """Codes [rows, ld / 2] and scales [ld / 256, rows, 8] as the library holds them."""
    codes = (q[:, 0::2] + 16 * q[:, 1::2]).astype(np.uint8)
    return codes, np.ascontiguousarray(np.asarray(e, np.uint8).reshape(len(q), -1, 8).transpose(1, 0, 2))


def product(x, w, bias=None):
    """(x w^T + bias, sum of the terms' magnitudes) of values."""
    y, mag = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y, mag = y + bias, mag + np.abs(bias)
    return y, mag
