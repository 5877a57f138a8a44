"""Oracle of the 8-bit operators: numpy, 64 bits, from the definitions (e4m3 values with a power-of-two scale for each run of 128
values of a row, or each 128 x 128 block of a weight).  Shares nothing with the GPU path."""
import math

import numpy as np

BLOCK = 128


def e4m3_values():
    """What the 256 bytes stand for."""
    out = np.empty(256)
    for b in range(256):
        sign, exp, man = -1.0 if b & 0x80 else 1.0, (b >> 3) & 15, b & 7
        if exp == 15 and man == 7:
            out[b] = np.nan
        elif exp == 0:
            out[b] = sign * man * 2.0 ** -9
        else:
            out[b] = sign * (1 + man / 8) * 2.0 ** (exp - 7)
    return out


def round_e4m3(x):
    """Nearest e4m3 value, ties to even, for |x| <= 448."""
    a = np.abs(x)
    _, k = np.frexp(a)                                   # a = m 2^k, m in [1/2, 1)
    step = np.ldexp(1.0, np.maximum(k - 1, -6) - 3)
    return np.copysign(np.rint(a / step) * step, x)


def _blocks(W):
    return -(-W // BLOCK)


def _spread(e, shape, rows):
    return np.repeat(np.repeat(e, rows, 0), BLOCK, 1)[:shape[0], :shape[1]]


def scale_exponents(x, rows=1):
    """e of each block: the smallest with max |finite x| <= 448 * 2^e, at least -126."""
    n, W = x.shape
    e = np.empty((-(-n // rows), _blocks(W)), dtype=np.int64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    for i in range(e.shape[0]):
        for j in range(e.shape[1]):
            top = a[i * rows:(i + 1) * rows, j * BLOCK:(j + 1) * BLOCK].max()
            k = -126
            if top > 0:
                k = max(math.frexp(top / 448.0)[1], -126)     # 2^(k-1) <= top / 448 < 2^k
                if k > -126 and top <= math.ldexp(448.0, k - 1):
                    k -= 1
            e[i, j] = k
    return e


def store(x, rows=1):
    """(values of the stored bytes, exponents of the scales)."""
    x = np.asarray(x, dtype=np.float64)
    e = scale_exponents(x, rows)
    y = x * np.ldexp(1.0, -_spread(e, x.shape, rows))
    fine = np.isfinite(x)
    return np.where(fine, round_e4m3(np.where(fine, y, 0.0)), np.nan), e


def values(q, e, rows=1):
    return q * np.ldexp(1.0, _spread(e, q.shape, rows))


def gelu(h):
    """GeLU(h) and its derivative."""
    from scipy.special import erfc
    cdf = 0.5 * erfc(-h / math.sqrt(2.0))
    return h * cdf, cdf + h * np.exp(-0.5 * h * h) / math.sqrt(2.0 * math.pi)
