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


# --------------------------------------------------------------- dropout
def philox(counter, key):
    """Philox4x32-10 of counters [n, 4] (uint32 values) and a 64-bit key."""
    low = np.uint64(0xFFFFFFFF)
    c = [counter[:, k].astype(np.uint64) for k in range(4)]
    k0, k1 = key & 0xFFFFFFFF, key >> 32
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return np.stack(c, 1).astype(np.uint32)


def draws(first, count, seed, tensor_id):
    """The 16-bit draws of elements first .. first + count - 1."""
    i = np.arange(first, first + count, dtype=np.uint64)
    block = i >> np.uint64(3)
    counter = np.stack([block & np.uint64(0xFFFFFFFF), block >> np.uint64(32), np.full_like(i, tensor_id), np.full_like(i, 0xFFFFFFFF)], 1)
    w = philox(counter, seed)
    k = (i % np.uint64(8)).astype(np.int64)
    return (w[np.arange(count), k // 2] >> (16 * (k % 2)).astype(np.uint32)) & np.uint32(0xFFFF)


def keep(shape, p, seed, tensor_id, index_base=0):
    """The factor of each element: 1 / (1 - p) with p in steps of 2^-16, or 0."""
    t = int(np.floor(float(np.float32(p)) * 65536 + 0.5))
    n = int(np.prod(shape))
    if t == 65536:
        return np.zeros(shape)
    return np.where(draws(index_base, n, seed, tensor_id) >= t, 65536.0 / (65536 - t), 0.0).reshape(shape)


# --------------------------------------------------------------- the join of two blocks
def join(x, b, w_post, gate, w_pre, alpha, eps, gate_rows, mask, store, post=True, pre=True):
    """r (before and after `store` rounds it), h and both 1 / RMS, in 64 bits."""
    rows, c = x.shape
    ones = np.ones(c)
    g = np.ones((rows, c)) if gate is None else gate[np.arange(rows) // gate_rows if gate_rows else np.zeros(rows, int)]
    w1, w2 = ones if w_post is None else w_post, ones if w_pre is None else w_pre
    q1 = 1 / np.sqrt((b * b).mean(1) + eps) if post else np.ones(rows)
    n = b * q1[:, None] * w1 if post else b
    exact = alpha * x + g * np.where(mask != 0, n * mask, 0.0)
    r = store(exact)
    q2 = 1 / np.sqrt((r * r).mean(1) + eps)
    return exact, r, r * q2[:, None] * w2 if pre else None, q1, q2


def join_gradients(dr, dh, b, r, q1, q2, w_post, gate, w_pre, alpha, gate_rows, mask, post=True, pre=True):
    """(dx, db, dw_post, dgate, dw_pre) by the chain rule, in 64 bits."""
    rows, c = b.shape
    ones = np.ones(c)
    at = np.arange(rows) // gate_rows if gate_rows else np.zeros(rows, int)
    g = np.ones((rows, c)) if gate is None else gate[at]
    w1, w2 = ones if w_post is None or not post else w_post, ones if w_pre is None else w_pre
    R = np.zeros_like(b) if dr is None else dr.copy()
    dw2 = None
    if pre:
        rh = r * q2[:, None]
        u = dh * w2
        R = R + q2[:, None] * (u - rh * (u * rh).mean(1, keepdims=True))
        dw2 = (dh * rh).sum(0)
    bh = b * q1[:, None] if post else b
    live = np.where(mask != 0, R, 0.0)
    v = live * g * mask
    dg = np.zeros((at.max() + 1, c))
    np.add.at(dg, at, live * mask * bh * w1)
    z = v * w1
    db = q1[:, None] * (z - bh * (z * bh).mean(1, keepdims=True)) if post else v
    return alpha * R, db, (v * bh).sum(0) if post else None, dg, dw2
