"""Plain CPU implementation, in 64 bits, of the 8-bit expert products and of the
gate's balance loss (test infrastructure; shares no code with the GPU path).

8-bit values are handled as the numbers they stand for.  ``quantize`` follows
the stated recipe in its stated precision (one fp32 rounding per quotient and
product), so its results are the recipe's to the bit; everything behind it is
in fp64.
"""

from __future__ import annotations

import numpy as np

BLOCK = 128


def e4m3_round(x):
    """Nearest e4m3 value, ties to even: steps of 2^(e - 3) in [2^e, 2^(e + 1)), of 2^-9 below 2^-6, at most 448."""
    x = np.asarray(x, np.float64)
    _, e = np.frexp(np.where(np.isfinite(x), x, 0.0))
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    with np.errstate(invalid="ignore"):
        return np.clip(np.rint(x / step) * step, -448.0, 448.0)


def e4m3_decode(bits):
    """Values of e4m3 bytes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    b = np.asarray(bits, np.uint8).astype(np.int64)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, np.ldexp(m / 8.0, -6), np.ldexp(1.0 + m / 8.0, e - 7))
    v = np.where((b & 127) == 127, np.nan, v)
    return np.where(b & 128, -v, v)


def quantize(x, block_rows=1):
    """(values [rows, cols], fp32 scales [row blocks, column blocks]) of one matrix."""
    x = np.asarray(x, np.float32)
    rows, cols = x.shape
    nr, nc = -(-rows // block_rows), -(-cols // BLOCK)
    q = np.empty((rows, cols))
    s = np.empty((nr, nc), np.float32)
    for i in range(nr):
        for j in range(nc):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * BLOCK:(j + 1) * BLOCK]
            part = np.abs(x[at][~np.isnan(x[at])])
            a = np.float32(max(np.float32(2.0 ** -96), part.max() if part.size else np.float32(0)))
            with np.errstate(invalid="ignore", over="ignore"):
                s[i, j] = a / np.float32(448)
                q[at] = e4m3_round(x[at] * (np.float32(448) / a))
    return q, s


def widen(q, s, block_rows=1):
    """Stored values times their scales."""
    rows, cols = q.shape
    full = np.repeat(np.repeat(np.asarray(s, np.float64), block_rows, 0)[:rows], BLOCK, 1)[:, :cols]
    return np.asarray(q, np.float64) * full


def gelu(u):
    from scipy.special import erf
    return 0.5 * u * (1.0 + erf(u / np.sqrt(2.0)))


def silu(u):
    return u / (1.0 + np.exp(-u))


def experts(x, offsets, W1, W3, W2, topk_w, perm, requantize=True):
    """slot [n, d] of widened rows x in expert order and widened weights (W3 None: GELU).

    requantize rounds the hidden rows to e4m3 as the layer does."""
    n, d = x.shape
    slot = np.zeros((n, d))
    w = np.asarray(topk_w, np.float64).reshape(-1)
    for e in range(len(offsets) - 1):
        lo, hi = offsets[e], offsets[e + 1]
        if hi <= lo:
            continue
        u = x[lo:hi] @ W1[e].T
        h = gelu(u) if W3 is None else silu(u) * (x[lo:hi] @ W3[e].T)
        if requantize:
            h = widen(*quantize(h))
        slot[perm[lo:hi]] = (h @ W2[e].T) * w[perm[lo:hi], None]
    return slot


def gate_probabilities(logits, mask, n_groups, top_groups=0):
    """g [T, E] of Eq. 5-7 from the logits [T, E + K], with top-group pruning."""
    T = logits.shape[0]
    E = len(mask)
    K = n_groups
    mask = np.asarray(mask, bool)
    gs = E // K
    g = np.zeros((T, E))
    live = mask.reshape(K, gs).any(1)
    for t in range(T):
        kept = [j for j in range(K) if live[j]]
        if K > 1 and 0 < top_groups < len(kept):
            kept = sorted(kept, key=lambda j: (-logits[t, E + j], j))[:top_groups]
        pg = np.array([np.exp(logits[t, E + j] - max(logits[t, E + i] for i in kept)) if K > 1 else 1.0 for j in kept],
                      np.float64)
        pg /= pg.sum()
        for p, j in zip(pg, kept):
            ids = [i for i in range(j * gs, (j + 1) * gs) if mask[i]]
            z = logits[t, ids].astype(np.float64)
            e = np.exp(z - z.max())
            g[t, ids] = p * e / e.sum()
    return g


def balance(logits, mask, topk_idx, n_groups, coef, valid=None, seg_offsets=None, top_groups=0, d_loss=1.0):
    """(loss, counts [S, E], d_logits, d_bias)."""
    logits = np.asarray(logits, np.float64)
    T, O = logits.shape
    E, K = len(mask), n_groups
    gs = E // K
    k = topk_idx.shape[1]
    A = int(np.asarray(mask, bool).sum())
    g = gate_probabilities(logits, mask, K, top_groups)
    ok = np.ones(T, bool) if valid is None else np.asarray(valid, bool)
    seg = [0, T] if seg_offsets is None else list(seg_offsets)
    S = len(seg) - 1
    counts = np.zeros((S, E), np.int64)
    tokens = [[t for t in range(seg[s], seg[s + 1]) if ok[t]] for s in range(S)]
    S_live = sum(1 for ts in tokens if ts)
    loss = 0.0
    w = np.zeros((T, E))
    for s, ts in enumerate(tokens):
        if not ts:
            continue
        for t in ts:
            for e in topk_idx[t]:
                counts[s, e] += 1
        n = len(ts)
        f = counts[s] / (k * n)
        loss += coef / S_live * A * float((f * g[ts].mean(0)).sum())
        w[ts] = coef * A * f / (S_live * n)
    d = np.zeros((T, O))
    for j in range(K):
        ids = slice(j * gs, (j + 1) * gs)
        pj = g[:, ids].sum(1, keepdims=True)
        wbar = np.where(pj > 0, (g[:, ids] * w[:, ids]).sum(1, keepdims=True) / np.where(pj > 0, pj, 1.0), 0.0)
        d[:, ids] = g[:, ids] * (w[:, ids] - wbar)
        if K > 1:
            d[:, E + j] = (pj * (wbar - (g * w).sum(1, keepdims=True)))[:, 0]
    d *= d_loss
    return loss, counts, d, d.sum(0)
