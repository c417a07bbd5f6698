"""Plain 64-bit forms of a step that takes several tokens of a sequence: norms and rotation, attention of many rows, verification of drafts, pages taken
back.  numpy, sequence by sequence, written from the formulas in ``include/chess.h``."""
from __future__ import annotations

import numpy as np

D = 128
HALF_STEP = 2.0 ** -8            # of a bf16 value, relative to it


def rotated(x, positions, inv_freq, axis, interleaved=False, norm=None, eps=0.0, scale=1.0):
    """x: [rows, heads, 128]; positions: [axes, rows]; norm: [128], [heads, 128] or None."""
    x = x.astype(np.float64)
    if norm is not None:
        x = x / np.sqrt((x ** 2).mean(-1, keepdims=True) + eps) * norm
    n = 2 * len(inv_freq)
    angle = positions.astype(np.float64)[np.asarray(axis)].T * inv_freq.astype(np.float64)        # [rows, pairs]
    c, s = np.cos(angle)[:, None] * scale, np.sin(angle)[:, None] * scale
    y = x.copy()
    first, second = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    y[..., first], y[..., second] = x[..., first] * c - x[..., second] * s, x[..., first] * s + x[..., second] * c
    return y, x


def rotation_error(y, x, inv_freq, interleaved, scale=1.0):
    """How far a result may be off: half a step of bf16, and what fp32 loses on the way: per dim a norm (a sum of 128 squares: 64.5 half steps of fp32, a root, two
    products: 68 in all), sine and cosine to 2^-18 of 1 (and the fraction of a turn), two products and a sum: under 2^-16 of the pair's magnitude."""
    n = 2 * len(inv_freq)
    size = np.abs(x).copy()
    first, second = (slice(0, n, 2), slice(1, n, 2)) if interleaved else (slice(0, n // 2), slice(n // 2, n))
    size[..., first] = size[..., second] = (np.abs(x[..., first]) + np.abs(x[..., second])) * abs(scale)
    return HALF_STEP * np.abs(y) + 2.0 ** -16 * size + 2.0 ** -133


def interval(p, length, window=0, prefix=0, first=0):
    """First and last key that the token at position p sees."""
    lo, hi = max(first, 0), max(p, prefix - 1)
    if window > 0:
        lo = max(lo, p - window + 1)
    return lo, min(hi, length - 1)


def attend(q, k, v, positions, intervals, sm_scale, cap=0.0, slopes=None, keys=None):
    """One sequence and KV head.  q: [rows, G, 128]; k, v: [tokens, 128]; keys: which tokens there are (None: all).  -> out, sum of weights times |v|,
    how far a score may be off, each [rows, G, ...]."""
    rows, G, _ = q.shape
    keys = np.arange(len(k)) if keys is None else np.asarray(keys)
    out, size, off = np.zeros((rows, G, D)), np.zeros((rows, G, D)), np.zeros((rows, G, 1))
    for r in range(rows):
        lo, hi = intervals[r]
        t = keys[(keys >= lo) & (keys <= hi)]
        if len(t) == 0:
            continue
        for g in range(G):
            s = sm_scale * (k[t] @ q[r, g])
            # fp32: 128 products summed (in any order), the scale, the cap (tanh to 2^-21 of the cap), bias and maximum: three roundings of a number that large
            e = 2.0 ** -24 * (130 * sm_scale * (np.abs(k[t]) @ np.abs(q[r, g])).max() + 3 * np.abs(s).max())
            z = s
            if cap:
                z = cap * np.tanh(s / cap)
                e += cap * 2.0 ** -21
            if slopes is not None:
                bias = slopes[g] * np.abs(positions[r] - t)
                z = z - bias
                e += 2.0 ** -22 * np.abs(bias).max()
            w = np.exp(z - z.max())
            w /= w.sum()
            out[r, g], size[r, g], off[r, g] = w @ v[t], w @ np.abs(v[t]), e
    return out, size, off


def attention_error(out, size, off, n_keys, weight_step=2.0 ** -16):
    """Half a step of bf16; each weight off by its score (numerator and denominator), by its own rounding, the exponential (2^-22) and the fp32 sums."""
    return HALF_STEP * np.abs(out) + size * (2 * off + weight_step + 2.0 ** -20 + 2 * n_keys * 2.0 ** -24) + 1e-30


def verify(target, draft, tokens, starts, uniforms, lens):
    """target [rows, V], draft [batch, most, V] or None, uniforms [batch, most + 1]: fp32 values in fp64 arrays."""
    batch, most = len(lens), uniforms.shape[1] - 1
    accepted, out, after = np.zeros(batch, int), -np.ones((batch, most + 1), int), np.array(lens)
    V = target.shape[1]
    for b in range(batch):
        start, n_new = starts[b], starts[b + 1] - starts[b]
        if n_new <= 0 or start < 0 or start + n_new > len(target):
            continue
        n = min(n_new - 1, most)
        j = 0
        while j < n:
            x = tokens[start + 1 + j]
            p, q = (target[start + j, x], 1.0 if draft is None else draft[b, j, x]) if 0 <= x < V else (0.0, 1.0)
            if not uniforms[b, j] * q < p:
                break
            j += 1
        p = target[start + j]
        positive = lambda w: np.where(w > 0, w, 0.0)  # noqa: E731  (NaN too)
        w = positive(p)
        if j < n:
            if draft is not None:
                w = positive(p - draft[b, j])
            else:
                x = tokens[start + 1 + j]
                if 0 <= x < V:
                    w[x] = 0.0
            if not (0 < w.sum() < np.inf):
                w = positive(p)
        token = -1
        if 0 < w.sum() < np.inf:
            upto = w.cumsum()
            above = np.nonzero((upto > uniforms[b, most] * upto[-1]) & (w > 0))[0]
            token = above[0] if len(above) else np.nonzero(w > 0)[0][-1]
        accepted[b], after[b] = j, lens[b] - (n_new - 1 - j)
        out[b, :j], out[b, j] = tokens[start + 1:start + 1 + j], token
    return accepted, out, after


def trim(lens, keep, table, free, n_free, capacity, B):
    free = list(free)
    for b, (n, k) in enumerate(zip(lens, keep)):
        had, kept = -(-max(n, 0) // B), -(-max(k, 0) // B)
        pages = list(table[b][kept:had])
        if n_free + len(pages) > capacity:
            break
        free[n_free:n_free + len(pages)] = pages
        n_free += len(pages)
    return free, n_free
