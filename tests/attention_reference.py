"""Rotary positions, attention, its gradient and the loss of a product from their formulas, in 64 bits on the host (numpy).  Shares
nothing with the kernels.

Bounds count the roundings of an implementation that keeps scores, exponentials and sums in fp32 (u = 2^-24; an exponential or a
logarithm is off by 2 u of its value, a sum of n terms by n u of the sum of their magnitudes) and rounds what it multiplies next to
`kind` (half a step: UNIT).  First order; the 1.01 pays for the second.  FLUSH: an exponential, a product or a sum below the smallest
normal fp32 number may be 0 (exp2 and the matrix instructions do not make smaller ones)."""
from __future__ import annotations

import numpy as np

from lmt_reference import TINY, U32, UNIT

FLUSH = 2.0 ** -126


def rotary(x, positions, frequencies, magnitude=1.0, neighbours=False, inverse=False):
    """x: [rows, heads, size].  Returns the result and the bound in fp32."""
    F = len(frequencies)
    z = positions.astype(np.float64)[:, None] * frequencies.astype(np.float64)[None]
    c, s = np.cos(z)[:, None] * magnitude, np.sin(-z if inverse else z)[:, None] * magnitude
    lo, hi = (slice(0, 2 * F, 2), slice(1, 2 * F, 2)) if neighbours else (slice(0, F), slice(F, 2 * F))
    out, bound = x.astype(np.float64).copy(), np.zeros(x.shape)
    a, b = x[..., lo].astype(np.float64), x[..., hi].astype(np.float64)
    out[..., lo], out[..., hi] = a * c - b * s, a * s + b * c
    # a quarter turn's part in fp32 (2^-26 of it), sine and cosine (2 u), the magnitude (2 u), product and sum (2 u); 64-bit angles: 2^-52 of them
    off = 8 * U32 + 2.0 ** -51 * np.abs(z)[:, None]
    bound[..., lo] = bound[..., hi] = (np.abs(a) + np.abs(b)) * abs(magnitude) * off
    return out, bound


def spans(rows, starts, lengths=None):
    """[(first row, end)] of the sequences."""
    return [(int(a), int(a) + int(lengths[s]) if lengths is not None else int(starts[s + 1])) for s, a in enumerate(starts[:-1])]


def _seen(n, causal, prefix):
    i = np.arange(n)
    return (i[None, :] <= i[:, None]) | (i[None, :] < prefix) if causal else np.ones((n, n), bool)


def _scores(q, k, scale, cap, slope):
    """Scores, what the cap multiplies derivatives by, and how far scores are off in fp32."""
    n, D = q.shape
    with np.errstate(invalid="ignore", over="ignore"):
        raw, size = q @ k.T * scale, np.abs(q) @ np.abs(k).T * abs(scale)
        apart = np.abs(np.arange(n)[None, :] - np.arange(n)[:, None])
        off = U32 * (D + 4) * size
        bend = np.ones_like(raw)
        s = raw
        if cap:
            t = np.tanh(raw / cap)
            s, bend = cap * t, 1 - t * t
            off = off + 8 * U32 * np.minimum(np.abs(raw), cap)     # the series or the exponential: 4 u of the tanh, the products
        if slope:
            s = s - slope * apart
            off = off + 3 * U32 * (np.abs(s) + abs(slope) * apart)
        return s, bend, off + 3 * U32 * np.abs(s)


def attention(q, k, v, starts, kind, lengths=None, prefixes=None, slopes=None, scale=1.0, cap=0.0, causal=False):
    """q: [rows, heads, size], k, v: [rows, kv_heads, size].  ((out, its bound), (lse [heads, rows], its bound))."""
    T, H, D = q.shape
    group = H // k.shape[1]
    out, lse = np.zeros((T, H, D)), np.full((H, T), -np.inf)
    b_out, b_lse = np.zeros((T, H, D)), np.zeros((H, T))
    for s, (a, e) in enumerate(spans(T, starts, lengths)):
        n = e - a
        if n <= 0:
            continue
        sees = _seen(n, causal, 0 if prefixes is None else int(prefixes[s]))
        for h in range(H):
            x, _, off = _scores(q[a:e, h], k[a:e, h // group], scale, cap, 0.0 if slopes is None else float(slopes[h]))
            vv = v[a:e, h // group]
            for i in range(n):
                at = np.nonzero(sees[i])[0]
                si = x[i, at]
                with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
                    if np.all(si == -np.inf):
                        continue
                    top = np.max(si) if not np.isnan(si).any() else np.nan
                    w = np.exp(si - top)
                    total = w.sum()
                    p = w / total
                    out[a + i, h] = p @ vv[at]
                    lse[h, a + i] = top + np.log(total)
                    worst = np.max(np.where(np.isfinite(off[i, at]), off[i, at], 0)) + U32 * (len(at) + 8 + 4 * np.abs(top))
                    b_out[a + i, h] = 1.01 * (p @ np.abs(vv[at]) * (UNIT[kind] + 2 * worst) + 2.0 ** -31 * np.abs(vv[at]).sum(0) * (kind == "f16") + UNIT[kind] * np.abs(out[a + i, h]) + TINY[kind] + FLUSH * (np.abs(vv[at]).sum(0) + n))
                    b_lse[h, a + i] = 1.01 * (worst + 4 * U32 * np.abs(lse[h, a + i])) + 2 * U32
    return (out, b_out), (lse, b_lse)


def attention_grad(go, q, k, v, out, lse, starts, kind, lengths=None, prefixes=None, slopes=None, scale=1.0, cap=0.0, causal=False):
    """((grad_q, bound), (grad_k, bound), (grad_v, bound)) from the given out and lse."""
    T, H, D = q.shape
    G = k.shape[1]
    group = H // G
    unit = UNIT[kind]
    grads = [np.zeros((T, n, D)) for n in (H, G, G)]
    bounds = [np.zeros((T, n, D)) for n in (H, G, G)]
    for s, (a, e) in enumerate(spans(T, starts, lengths)):
        n = e - a
        if n <= 0:
            continue
        sees = _seen(n, causal, 0 if prefixes is None else int(prefixes[s]))
        for h in range(H):
            g = h // group
            Q, K, V, GO, O = q[a:e, h], k[a:e, g], v[a:e, g], go[a:e, h], out[a:e, h]
            x, bend, off = _scores(Q, K, scale, cap, 0.0 if slopes is None else float(slopes[h]))
            L = lse[h, a:e][:, None]
            p = np.where(sees, np.exp(np.where(sees, x - np.where(np.isfinite(L), L, 0), -np.inf)), 0.0) * np.isfinite(L)
            rel = np.where(sees, off + U32 * (6 + 4 * np.abs(np.where(np.isfinite(L), L, 0))), 0)              # of p
            dp, delta = GO @ V.T, (GO * O).sum(1, keepdims=True)
            e_dp = U32 * (D + 3) * (np.abs(GO) @ np.abs(V).T + (np.abs(GO) * np.abs(O)).sum(1, keepdims=True))
            d = p * (dp - delta) * bend
            # a bend of 1 - t^2 is off by 4 u of 1, where t is near 1 of more than itself
            e_d = np.abs(d) * (rel + 6 * U32) + p * bend * e_dp + p * np.abs(dp - delta) * (12 * U32 if cap else 0.0) + FLUSH * (np.abs(dp - delta) + 2) * sees
            r_d = unit * (np.abs(d) + e_d) + (2.0 ** -38 * np.abs(d).max() if kind == "f16" else 0.0)           # rounded in front of the next product
            e_p = p * (rel + unit) + ((2.0 ** -38 if kind == "f16" else 0.0) + FLUSH) * sees
            sums = (n * group + 4) * U32
            grads[0][a:e, h] += scale * (d @ K)
            bounds[0][a:e, h] += abs(scale) * ((e_d + r_d + sums * np.abs(d)) @ np.abs(K))
            grads[1][a:e, g] += scale * (d.T @ Q)
            bounds[1][a:e, g] += abs(scale) * ((e_d + r_d + sums * np.abs(d)).T @ np.abs(Q))
            grads[2][a:e, g] += p.T @ GO
            bounds[2][a:e, g] += (e_p + sums * p).T @ np.abs(GO)
    return [(x, 1.01 * (b + unit * np.abs(x)) + TINY[kind] + FLUSH * (T * group * abs(scale) + 1)) for x, b in zip(grads, bounds)]


def linear_loss(x, table, targets, weights, ignore, kind, grad_table_kind=None, old=None):
    """{"loss", "lse", "grad_x", "grad_table"}: (value, bound)."""
    n, W = x.shape
    V = table.shape[0]
    unit = UNIT[kind]
    counted = (targets != ignore) & (targets >= 0) & (targets < V)
    w = np.where(counted, 1.0 if weights is None else weights.astype(np.float64), 0.0)
    logits, size = x @ table.T, np.abs(x) @ np.abs(table).T
    top = logits.max(1)
    e = np.exp(logits - top[:, None])
    total = e.sum(1)
    lse = top + np.log(total)
    off = U32 * (W + 2) * size                                                     # of a logit
    worst = off.max(1) + U32 * (V + 12 + 4 * (top - logits.min(1)))                # of the sum's logarithm
    t = np.where(counted, targets, 0)
    at = logits[np.arange(n), t]
    loss = w * (lse - at)
    b_loss = np.abs(w) * (worst + off[np.arange(n), t] + U32 * (4 * np.abs(top - at) + 4 * np.abs(lse - at) + 2)) * 1.01
    b_lse = (worst + 3 * U32 * (np.abs(lse) + np.abs(top))) * 1.01
    p = e / total[:, None]
    hot = np.zeros((n, V))
    hot[np.arange(n), t] = 1.0
    g = np.where(counted[:, None], p - hot, 0.0)
    e_g = np.where(counted[:, None], p * (off + worst[:, None] + U32 * (8 + 4 * np.abs(logits - top[:, None]))) + U32 * np.abs(g) + FLUSH, 0.0)
    r_g = unit * (np.abs(g) + e_g) + (2.0 ** -38 if kind == "f16" else 0.0) * counted[:, None]  # rounded in front of the products
    grad_x = w[:, None] * (g @ table)
    b_x = np.abs(w)[:, None] * ((e_g + r_g + U32 * (V + 8) * np.abs(g)) @ np.abs(table))
    gw, largest = w[:, None] * g, np.abs(w).max() if n else 0.0
    r_w = unit * np.abs(w)[:, None] * (np.abs(g) + e_g) + (2.0 ** -38 * largest if kind == "f16" else 0.0) * counted[:, None]
    grad_t = gw.T @ np.where(counted[:, None], x, 0.0)
    b_t = (np.abs(w)[:, None] * e_g + r_w + U32 * (n + 8) * np.abs(gw)).T @ np.abs(np.where(counted[:, None], x, 0.0))
    kt = grad_table_kind or kind
    b_x, b_t = b_x + FLUSH * V * (np.abs(w)[:, None] + 1), b_t + FLUSH * n * (largest + 1)
    if old is not None:
        grad_t = grad_t + old
        b_t = b_t + 2 * U32 * (np.abs(old) + np.abs(grad_t))
    return {"loss": (loss, b_loss), "lse": (lse, b_lse), "grad_x": (grad_x, 1.01 * (b_x + unit * np.abs(grad_x)) + TINY[kind]),
            "grad_table": (grad_t, 1.01 * (b_t + UNIT[kt] * np.abs(grad_t)) + TINY[kt])}
