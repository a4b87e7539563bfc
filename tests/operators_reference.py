"""The residual blocks' operators in 64 bits on the CPU, for tests: from the definitions, one element's sums as numpy takes
them, nothing shared with the library."""
import math

import numpy as np

GROUP = 32


def e4m3_table():
    """value of each of the 256 codes: 4 exponent bits (bias 7), 3 mantissa bits, no infinity, 0x7f and 0xff NaN."""
    out = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v = math.nan if e == 15 and m == 7 else (m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
        out[c] = -v if c & 0x80 else v
    return out


TABLE = e4m3_table()


def nearest_code(v):
    """Code of the e4m3 number nearest to each v (|v| <= 448), ties to the even code."""
    positive = TABLE[:0x7f]                                  # ascending
    a = np.abs(v)
    hi = np.clip(np.searchsorted(positive, a), 0, 0x7e)
    lo = np.maximum(hi - 1, 0)
    dl, dh = a - positive[lo], positive[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    code = np.where(positive[hi] == a, hi, code)
    return (code | np.where(np.signbit(v), 0x80, 0)).astype(np.uint8)


def to_eight(x):
    """(codes [rows][cols], scale bytes [rows][groups]) of a matrix."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, groups), np.uint8)
    for r in range(rows):
        for g in range(groups):
            v = x[r, g * GROUP:(g + 1) * GROUP]
            finite = np.abs(v[np.isfinite(v)])
            top = float(finite.max()) if finite.size else 0.0
            e = -117
            while top > 448 * 2.0 ** e:
                e += 1
            most = 240.0 if e == 120 else 448.0
            s = np.clip(np.where(np.isfinite(v), v, 0.0) / 2.0 ** e, -most, most)
            c = nearest_code(s)
            codes[r, g * GROUP:(g + 1) * GROUP] = np.where(np.isfinite(v), c, 0x7f)
            scales[r, g] = e + 127
    return codes, scales


def from_eight(codes, scales):
    wide = np.repeat(scales.astype(np.float64), GROUP, axis=1)[:, :codes.shape[1]]
    return TABLE[codes] * 2.0 ** (wide - 127)


def norm_forward(x, branch, gain, eps):
    s = x if branch is None else x + branch
    rstd = 1 / np.sqrt((s * s).mean(axis=1) + eps)
    return s, rstd, s * rstd[:, None] * gain


def norm_backward(dy, s, gain, rstd, dsum):
    h, t = s * rstd[:, None], dy * gain
    dx = rstd[:, None] * (t - h * (t * h).mean(axis=1, keepdims=True))
    return dx + (0 if dsum is None else dsum), (dy * h).sum(axis=0)


def _normal(z):
    """Phi(z); by erfc, which keeps the left tail's digits."""
    return 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-z / math.sqrt(2))


def act(z, name):
    with np.errstate(over="ignore"):
        sig = 1 / (1 + np.exp(-z))
    return {"none": lambda: z, "sigmoid": lambda: sig, "relu": lambda: np.maximum(z, 0), "silu": lambda: z * sig,
            "gelu": lambda: z * _normal(z)}[name]()


def slope(z, name):
    with np.errstate(over="ignore"):
        sig = 1 / (1 + np.exp(-z))
    return {"none": lambda: np.ones_like(z), "sigmoid": lambda: sig * (1 - sig), "relu": lambda: (z > 0) * 1.0,
            "silu": lambda: sig * (1 + z * (1 - sig)),
            "gelu": lambda: _normal(z) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[name]()


def linear_forward(x, w, b, name, residual):
    z = x @ w.T + (0 if b is None else b)
    return z, act(z, name) + (0 if residual is None else residual)


def linear_backward(dy, z, name, x, w):
    dz = dy if name == "none" else dy * slope(z, name)
    return dz, dz @ w, dz.T @ x, dz.sum(axis=0)
