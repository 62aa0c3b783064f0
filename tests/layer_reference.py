"""The layer calls in 64 bits, on the CPU, from their definitions: what the GPU tests compare with."""
import math

import numpy as np

BLOCK = 128


def code_values():
    """Values of the 256 e4m3 codes."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        x = m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = math.nan if (c & 127) == 127 else (-x if c & 128 else x)
    return v


CODE_VALUES = code_values()
_GRID = CODE_VALUES[:127]                       # the magnitudes, ascending


def encode(y):
    """Codes of values of magnitude <= 448: nearest, ties to the even code; what is not finite gets 0xff."""
    fine = np.isfinite(y)
    a = np.where(fine, np.abs(y), 0.0)
    assert a.max(initial=0.0) <= 448.0
    hi = np.searchsorted(_GRID, a)              # first magnitude >= a
    lo = np.maximum(hi - 1, 0)
    below, above = a - _GRID[lo], _GRID[hi] - a
    pick = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(fine, pick | np.where(np.signbit(y), 128, 0), 0xFF).astype(np.uint8)


def exponent(top):
    """Stored exponent for a block's largest finite magnitude."""
    if top == 0.0:
        return 0
    e = math.frexp(top)[1] - 9                  # top < 2^(e + 9), so e or e + 1
    return max(0, 127 + (e if top <= 448.0 * 2.0 ** e else e + 1))


def pack(x, tiles=False):
    """(codes padded with zeros to whole blocks, scales) of a 2-D array."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    nb = -(-cols // BLOCK)
    codes = np.zeros((rows, nb * BLOCK), np.uint8)
    scales = np.zeros((rows, nb), np.uint8)
    deep = BLOCK if tiles else 1
    for r in range(0, rows, deep):
        for b in range(nb):
            v = x[r:r + deep, b * BLOCK:(b + 1) * BLOCK]
            s = exponent(np.abs(v[np.isfinite(v)]).max(initial=0.0))
            scales[r:r + deep, b] = s
            codes[r:r + deep, b * BLOCK:b * BLOCK + v.shape[1]] = encode(v * 2.0 ** (127 - s))
    return codes, scales


def values(codes, scales, cols):
    f = np.exp2(scales.astype(np.float64) - 127.0)
    f[scales == 255] = math.nan
    return CODE_VALUES[codes[:, :cols]] * np.repeat(f, BLOCK, axis=1)[:, :cols]


_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _logistic(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


def act(name, x):
    if name == "relu":
        return np.where(x < 0, 0.0, x)
    if name == "tanh":
        return np.tanh(x)
    if name == "sigmoid":
        return _logistic(x)
    if name == "silu":
        return x * _logistic(x)
    if name == "gelu":
        return x * 0.5 * _erfc(-x * math.sqrt(0.5))
    return x


def slope(name, x):
    if name == "relu":
        return np.where(np.isnan(x), x, (x > 0) * 1.0)
    if name == "tanh":
        return 4.0 * np.exp(-2 * np.abs(x)) / (1.0 + np.exp(-2 * np.abs(x))) ** 2
    if name == "sigmoid":
        return _logistic(x) * _logistic(-x)
    if name == "silu":
        return _logistic(x) + x * _logistic(x) * _logistic(-x)
    if name == "gelu":
        return 0.5 * _erfc(-x * math.sqrt(0.5)) + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    return np.where(np.isnan(x), x, 1.0)


def weight_grad(dy, x, begin):
    return np.stack([dy[a:b].T @ x[a:b] for a, b in zip(begin[:-1], begin[1:])])
