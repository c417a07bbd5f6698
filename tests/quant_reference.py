"""The 8-bit paged cache and the dealing of pages from their definitions, in fp64 and whole numbers (numpy; nothing of the product): what the tests
of the kernels compare with."""
from __future__ import annotations

import numpy as np

E_MIN, E_MAX = -64, 119


def _e4m3_table():
    """Values of the 256 bytes: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN, no infinities."""
    t = np.empty(256)
    for byte in range(256):
        e, m = (byte >> 3) & 15, byte & 7
        v = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if byte & 127 == 127:
            v = np.nan
        t[byte] = -v if byte & 128 else v
    return t


TABLE = _e4m3_table()
_POSITIVE = TABLE[:127]                                          # ascending, 0 .. 448


def decode(b):
    return TABLE[np.asarray(b, dtype=np.uint8)]


def encode(y):
    """fp64 -> nearest e4m3 byte, ties to even, saturated at 448; NaN and infinities -> NaN."""
    y = np.asarray(y, dtype=np.float64)
    a = np.minimum(np.abs(np.where(np.isfinite(y), y, 0.0)), 448.0)
    hi = np.minimum(np.searchsorted(_POSITIVE, a), 126)
    lo = np.maximum(hi - 1, 0)
    d_hi, d_lo = _POSITIVE[hi] - a, a - _POSITIVE[lo]
    code = np.where((d_lo < d_hi) | ((d_lo == d_hi) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isfinite(y), code, 127)
    return (code | (np.signbit(y).astype(int) << 7)).astype(np.uint8)


def exponent(largest):
    """The smallest e with largest <= 448 * 2^e, within what a scale can have."""
    e = E_MIN
    while e < E_MAX and largest > 448 * 2.0 ** e:
        e += 1
    return e


def same_bytes(a, b):
    """Equal bytes; NaN of either sign is one value."""
    a, b = np.asarray(a), np.asarray(b)
    return bool(np.all((a == b) | ((a & 127 == 127) & (b & 127 == 127))))


def store(k, v, scales, k_new, v_new, writes):
    """quant_store in place: k [phys][H][B][d], v [phys][H][d][B] bytes, scales [phys][H][2]; k_new / v_new fp64 [token][H][d]."""
    H = k.shape[1]
    for phys, row, first, count in writes:
        for h in range(H):
            for which, page, rows in ((0, k[phys, h], k_new), (1, v[phys, h].T, v_new)):
                x = rows[row:row + count, h]
                finite = np.abs(x[np.isfinite(x)])
                e = exponent(finite.max() if finite.size else 0.0)
                if first > 0:
                    old = scales[phys, h, which]
                    e = max(e, int(np.log2(old)))
                    if 2.0 ** e != old:
                        page[:first] = encode(decode(page[:first]) * (np.float64(old) / 2.0 ** e))
                page[first:first + count] = encode(x / 2.0 ** e)
                scales[phys, h, which] = 2.0 ** e


def rows_of(pool, scales, which, bt_row, h, length):
    """The fp64 rows [length, d] that a sequence's pages stand for."""
    out = []
    B = pool.shape[2] if which == 0 else pool.shape[3]
    for p in range(-(-length // B)):
        page = decode(pool[bt_row[p], h]) * np.float64(scales[bt_row[p], h, which])
        out.append(page if which == 0 else page.T)
    return np.concatenate(out)[:length] if out else np.zeros((0, 128))


def attention(q, kl, vl, scale):
    """(outputs [G, d] of softmax attention, how far fp32 may be off), q [G, d], kl / vl [n, d], all fp64.

    With u = 2^-24: a score is a sum of 128 products that are exact, so it is off by at most 128 u sum |q k|, and 4 u of itself more by the two
    products with the scales; a weight relative to the largest one is then off by twice that, and by 2^-21 for the exponential, the rounding
    of its argument (at most 2^-24 of what is below 150 and counts) and the split into parts; sums of n terms, merged over waves and splits, by
    (n + 200) u of the sum of absolute terms, in the numerator and in the denominator."""
    u = 2.0 ** -24
    z = q @ kl.T * scale
    p = np.exp(z - z.max(1, keepdims=True))
    p /= p.sum(1, keepdims=True)
    off = ((128 * np.abs(q) @ np.abs(kl).T * scale + 4 * np.abs(z)) * u).max(1, keepdims=True)
    n = kl.shape[0]
    return p @ vl, 2 * (2 * off + 2.0 ** -21 + 150 * u + (n + 200) * u) * (p @ np.abs(vl)) + 1e-30


def release(lens, done, table, free, n_free, capacity, B):
    """(lens after, free list, its length)."""
    lens, free = list(lens), list(free)
    out, fits = list(lens), True
    for b, n in enumerate(lens):
        if not done[b]:
            continue
        pages = [int(table[b][j]) for j in range(-(-max(n, 0) // B))]
        fits = fits and n_free + len(pages) <= capacity
        if fits:
            free[n_free:n_free + len(pages)] = pages
            n_free += len(pages)
            out[b] = 0
    return out, free, n_free


def map_tokens(lens, new, table, free, n_free, max_tokens, max_pages, B):
    """What chess_map_tokens defines, sequence by sequence: a dict of its outputs, the table among them."""
    table = [list(r) for r in table]
    left, after, starts, slots, writes, refused, stop = n_free, [], [0], [], [], 0, False
    for b, (L, n) in enumerate(zip(lens, new)):
        got = n if n > 0 and L >= 0 and L + n <= max_pages * B else 0
        need = -(-(L + got) // B) - (-(-L // B)) if got else 0
        stop = stop or (got > 0 and (len(slots) + got > max_tokens or need > left))
        if stop:
            got = 0
        refused += n > 0 and got == 0
        for t in range(L, L + got):
            if t % B == 0:
                left -= 1
                table[b][t // B] = free[left]
            page = table[b][t // B]
            if t == L or t % B == 0:
                writes.append([page, len(slots), t % B, 0])
            writes[-1][3] += 1
            slots.append(page * B + t % B)
        after.append(L + got)
        starts.append(len(slots))
    return {"table": table, "lens_after": after, "n_left": left, "starts": starts, "slots": slots, "writes": writes,
            "counts": [len(slots), len(writes), n_free - left, refused]}
