"""fp64 definitions of the 8-bit rows, the root-mean-square norm and the products
of 8-bit rows. Plain numpy, test infrastructure only.

An e4m3 code is sign, 4 exponent bits (bias 7), 3 fraction bits; exponent 0 holds
multiples of 2^-9, code 0x7F is NaN. A scale byte b stands for 2^(b - 127), 255
for NaN."""
from __future__ import annotations

import numpy as np

GROUP = 128
LARGEST = 448.0


def _table():
    t = np.empty(256)
    for code in range(256):
        e, f = (code >> 3) & 15, code & 7
        v = f * 2.0 ** -9 if e == 0 else (8 + f) * 2.0 ** (e - 10)
        t[code] = np.nan if code & 127 == 127 else -v if code & 128 else v
    return t


E4M3 = _table()


def scale_cols(n):
    return (n + 511) // 512 * 4


def scale_bytes(x):
    """The scale bytes of the groups of each row of x, padded with 127."""
    x = np.asarray(x, np.float64)
    rows, n = x.shape
    out = np.full((rows, scale_cols(n)), 127, np.uint8)
    for g in range((n + GROUP - 1) // GROUP):
        v = np.abs(x[:, g * GROUP:(g + 1) * GROUP])
        top = np.where(np.isfinite(v), v, 0.0).max(axis=1)
        f, q = np.frexp(top)   # top = f 2^q, 448 = 0.875 2^9
        e = np.where(top > 0, q - 9 + (f > 0.875), -127)
        out[:, g] = np.clip(e, -127, 127) + 127
    return out


def spread(scale, n):
    """2^(byte - 127) (NaN for 255) of every value of rows of n."""
    s = np.asarray(scale, np.int64)
    f = np.where(s == 255, np.nan, np.ldexp(1.0, s - 127))
    return np.repeat(f, GROUP, axis=1)[:, :n]


def codes(x, scale):
    """The e4m3 codes of x under the scale bytes: rounded to nearest even, NaN for
    what is not finite."""
    v = np.asarray(x, np.float64) / spread(scale, np.asarray(x).shape[1])
    mag = np.minimum(np.abs(np.where(np.isfinite(v), v, 0.0)), LARGEST)
    grid = E4M3[:127]
    lo = np.searchsorted(grid, mag, side="right") - 1
    hi = np.minimum(lo + 1, 126)
    below, above = mag - grid[lo], grid[hi] - mag
    code = np.where((above < below) | ((above == below) & (hi % 2 == 0)), hi, lo)
    code = np.where(np.isfinite(v), code, 127)
    return (code | np.where(np.signbit(v), 128, 0)).astype(np.uint8)


def quant(x):
    s = scale_bytes(x)
    return codes(x, s), s


def values(code, scale):
    return E4M3[np.asarray(code)] * spread(scale, np.asarray(code).shape[1])


def rms_forward(h, gamma, eps):
    """(y, rstd) of the stream h as it is stored."""
    h = np.asarray(h, np.float64)
    rstd = 1.0 / np.sqrt(np.square(h).mean(axis=1) + eps)
    y = h * rstd[:, None]
    return (y if gamma is None else y * gamma), rstd


def rms_backward(dy, h, gamma, rstd, dh=None):
    """(dx, dgamma) with the row statistics as given."""
    dy, hh = np.asarray(dy, np.float64), np.asarray(h, np.float64) * np.asarray(rstd, np.float64)[:, None]
    a = dy if gamma is None else dy * gamma
    dx = np.asarray(rstd, np.float64)[:, None] * (a - hh * (a * hh).mean(axis=1, keepdims=True))
    return (dx if dh is None else dx + dh), (dy * hh).sum(axis=0)


def product(a, a_scale, w, w_scale):
    return values(a, a_scale) @ values(w, w_scale).T


def weight_grad(dY, x, x_scale):
    return np.asarray(dY, np.float64).T @ values(x, x_scale)
