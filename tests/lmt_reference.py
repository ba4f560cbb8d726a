"""The operators of lmt.h from their formulas, in 64 bits on the host (numpy).  Shares nothing with the kernels.

Bounds say how far a correct implementation may be away, from the number of fp32 roundings a result takes: a sum of n terms in
any order is off by at most (n - 1) u times the sum of their magnitudes (first order in u = 2^-24)."""
from __future__ import annotations

import numpy as np

U32 = 2.0 ** -24
UNIT = {"f32": 2.0 ** -24, "f16": 2.0 ** -11, "bf16": 2.0 ** -8}          # half the distance of neighbours, relative
TINY = {"f32": 2.0 ** -149, "f16": 2.0 ** -24, "bf16": 2.0 ** -133}        # distance of the smallest values
E4M3, E5M2 = "e4m3", "e5m2"
_FORM = {E4M3: (4, 3, 7), E5M2: (5, 2, 15)}                                # exponent bits, mantissa bits, bias
LARGEST = {E4M3: 448.0, E5M2: 57344.0}


def embed(table, tokens, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    there = (tokens >= 0) & (tokens < table.shape[0])
    out[there] = table[tokens[there]].astype(np.float64) * scale
    return out


def rounded(x, kind):
    """Bound for one rounding of fp32 results x to `kind`."""
    return UNIT[kind] * np.abs(x) + TINY[kind]


def embed_grad(grad_out, tokens, vocab, scale, skip, old=None):
    """The table's gradient and the bound of its fp32 sums."""
    g = grad_out.astype(np.float64)
    total, size, count = np.zeros((vocab, g.shape[1])), np.zeros((vocab, g.shape[1])), np.zeros(vocab)
    for t, v in enumerate(tokens):
        if v != skip and 0 <= v < vocab:
            total[v] += g[t]
            size[v] += np.abs(g[t])
            count[v] += 1
    total, bound = total * scale, U32 * (count[:, None] + 2) * size * abs(scale)   # sums, times scale, plus what was there
    if old is not None:
        total = total + old.astype(np.float64)
        bound = bound + U32 * (np.abs(total) + np.abs(old))
    return total, bound


def decode(codes, form):
    """Values of 8-bit codes."""
    e_bits, m_bits, bias = _FORM[form]
    c = codes.astype(np.int64)
    sign = np.where(c >> 7, -1.0, 1.0)
    e, m = (c >> m_bits) & ((1 << e_bits) - 1), c & ((1 << m_bits) - 1)
    v = np.where(e > 0, (1 + m / 2.0 ** m_bits) * 2.0 ** (e - bias), m / 2.0 ** m_bits * 2.0 ** (1 - bias))
    if form == E4M3:
        v = np.where((c & 127) == 127, np.nan, v)
    else:
        v = np.where(e == 31, np.where(m == 0, np.inf, np.nan), v)
    return sign * v


def _encode(y, form):
    """Codes of the values nearest to y (|y| <= the largest), ties to the even mantissa; NaN where y is not finite."""
    codes = np.arange(128)
    values = decode(codes, form)
    keep = np.isfinite(values)
    codes, values = codes[keep], values[keep]                     # in rising order
    a = np.abs(np.where(np.isfinite(y), y, 0.0))
    hi = np.clip(np.searchsorted(values, a), 1, len(values) - 1)
    lo = hi - 1
    d_lo, d_hi = a - values[lo], values[hi] - a
    up = (d_hi < d_lo) | ((d_hi == d_lo) & (codes[hi] % 2 == 0))
    c = np.where(up, codes[hi], codes[lo]) | np.where(np.signbit(y), 128, 0)
    return np.where(np.isfinite(y), c, 127).astype(np.uint8)


def quantize(x, form, tile):
    """Codes [rows, 128 * blocks] and scales [rows, 4 * ceil(blocks / 4)] of x."""
    x = x.astype(np.float64)
    rows, cols = x.shape
    nb, nr = -(-cols // 128), -(-rows // 128)
    z = np.zeros((128 * nr, 128 * nb))
    z[:rows, :cols] = x
    size = np.where(np.isfinite(z), np.abs(z), 0.0).reshape(nr, 128, nb, 128)
    size = np.broadcast_to(size.max((1, 3), keepdims=True), (nr, 128, nb, 1)) if tile else size.max(3, keepdims=True)
    size = size.reshape(128 * nr, nb)
    e = np.full(size.shape, -126)
    while True:                                                    # the smallest power that is enough
        low = size / 2.0 ** e > LARGEST[form]
        if not low.any():
            break
        e = e + low
    with np.errstate(invalid="ignore"):
        q = _encode(z / np.repeat(2.0 ** e, 128, 1), form)
    scales = np.full((rows, 4 * -(-nb // 4)), 127, np.uint8)
    scales[:, :nb] = (e + 127)[:rows]
    return q[:rows], scales


def values(codes, scales, form):
    return decode(codes, form) * np.repeat(2.0 ** (scales[:, :codes.shape[1] // 128].astype(np.float64) - 127), 128, 1)


def cross_entropy(x, targets, weights, ignore):
    """loss, lse, gradient; and their bounds."""
    x = x.astype(np.float64)
    n, V = x.shape
    loss, lse, grad = np.zeros(n), np.zeros(n), np.zeros((n, V))
    b_loss, b_lse, b_grad = np.zeros(n), np.zeros(n), np.zeros((n, V))
    for i in range(n):
        w = 1.0 if weights is None else float(weights[i])
        t = int(targets[i])
        counted = t != ignore and 0 <= t < V
        r = x[i]
        if np.isnan(r).any() or np.isposinf(r).any():
            lse[i] = np.nan
            if counted:
                loss[i], grad[i] = np.nan, np.nan
            continue
        top = r.max()
        if np.isneginf(top):
            lse[i] = -np.inf
            if counted:
                loss[i] = np.inf
            continue
        e = np.exp(r - top)
        total = e.sum()
        lse[i] = top + np.log(total)
        p = e / total
        # A term: its argument x log2(e) - max log2(e) takes the rounded constant (relative 2^-25 of the difference), the rounded product with the
        # maximum and one rounding, then exp2 to 2 ulp.  The sum: V roundings at most.  The logarithm and the last sum: 4 ulp.
        size = (np.abs(np.where(np.isfinite(r), r, top)) + abs(top)) * 1.45
        term = (2 * size * U32 + 4 * U32)
        rel = (p * term).sum() + V * U32
        b_lse[i] = rel + 4 * U32 * (abs(np.log(total)) + abs(lse[i]) + 1)
        if counted:
            loss[i] = w * (lse[i] - r[t])
            b_loss[i] = abs(w) * (b_lse[i] + 2 * U32 * (abs(lse[i]) + abs(np.where(np.isfinite(r[t]), r[t], 0)))) + 2 * U32 * abs(np.where(np.isfinite(loss[i]), loss[i], 0))
            grad[i] = w * p
            b_grad[i] = abs(w) * p * (term + rel + 4 * U32)
            grad[i, t] -= w
            b_grad[i, t] += abs(w) * 2 * U32
    return (loss, lse, grad), (b_loss, b_lse, b_grad)
