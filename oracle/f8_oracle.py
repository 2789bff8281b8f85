"""Plain 64-bit statements of the operators of a residual block: 8-bit floating-point codes with a scale for each block of
128, their product, the join of two blocks and its gradients, and dropout.  Written from the definitions in include/qbp.h
with numpy; it shares no code with the GPU path (test infrastructure)."""
from __future__ import annotations

import numpy as np

MAX = {0: 448.0, 1: 57344.0}                    # largest value of e4m3 and e5m2
MANTISSA = {0: 3, 1: 2}
LOWEST = {0: -6, 1: -14}                        # exponent of the smallest normal value


# --------------------------------------------------------------- the formats
def table(fmt):
    """The value of each of the 256 codes."""
    out = np.empty(256)
    for code in range(256):
        sign, rest = -1.0 if code & 128 else 1.0, code & 127
        m, e = rest & ((1 << MANTISSA[fmt]) - 1), rest >> MANTISSA[fmt]
        if fmt == 0 and rest == 127:
            v = np.nan
        elif fmt == 1 and e == 31:
            v = np.inf if m == 0 else np.nan
        elif e == 0:
            v = m * 2.0 ** (LOWEST[fmt] - MANTISSA[fmt])
        else:
            v = (1 + m / (1 << MANTISSA[fmt])) * 2.0 ** (e - 1 + LOWEST[fmt])
        out[code] = sign * v
    return out


def encode(v, fmt):
    """Codes of finite values within the format's range: nearest, ties to the even code; -0.0 keeps its sign."""
    t = table(fmt)[:128]
    finite = t[np.isfinite(t)]                   # ascending, code by code
    a = np.abs(np.asarray(v, np.float64))
    hi = np.clip(np.searchsorted(finite, a), 1, len(finite) - 1)
    lo = hi - 1
    dl, dh = a - finite[lo], finite[hi] - a
    code = np.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi).astype(np.uint8)
    return code | (np.signbit(v).astype(np.uint8) << 7)


# --------------------------------------------------------------- the quantiser
def exponent(amax, fmt):
    """The smallest e >= -127 with amax <= MAX * 2^e; 0 for zero, 128 for what is not finite."""
    if not np.isfinite(amax):
        return 128
    if amax == 0:
        return 0
    e = -127
    m, k = np.frexp(float(amax) / MAX[fmt])
    e = max(e, int(k) - (1 if m == 0.5 else 0))
    return e


def quantize(x, fmt, high=1, wide=128):
    """Codes [rows, cols] and exponents per block of high x wide elements."""
    x = np.asarray(x, np.float64)
    rows, cols = x.shape
    rb, cb = -(-rows // high), -(-cols // wide)
    q, ex = np.zeros((rows, cols), np.uint8), np.zeros((rb, cb), np.int64)
    for i in range(rb):
        for j in range(cb):
            at = np.s_[i * high:(i + 1) * high, j * wide:(j + 1) * wide]
            b = x[at]
            e = exponent(np.abs(b).max() if np.isfinite(b).all() else np.inf, fmt)
            ex[i, j] = e
            q[at] = 0x7F if e == 128 else encode(b * 2.0 ** -e, fmt)
    return q, ex


def pack(ex, outer):
    """The stored scales of exponents [outer, blocks]."""
    blocks = ex.shape[1]
    groups = -(-blocks // 4)
    out = np.full((-(-outer // 128), groups, 512), 127, np.uint8)
    for r in range(outer):
        for b in range(blocks):
            out[r // 128, b // 4, (r % 32) * 16 + (r // 32 % 4) * 4 + b % 4] = ex[r, b] + 127
    return out.reshape(-1)


def values(q, fmt, ex_full):
    """What codes with the exponent of each element stand for."""
    return table(fmt)[q] * np.where(ex_full == 128, np.nan, 2.0 ** np.asarray(ex_full, np.float64))


def spread(ex, n, axis=1):
    """Exponents of blocks of 128 along `axis`, one for each of n elements."""
    return np.take(np.repeat(ex, 128, axis), np.arange(n), axis)
