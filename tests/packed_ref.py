"""Rows held in 4 bits, attention with first tokens that stay visible and the
handling of shared pages, by their definitions (numpy, one row, block or page
at a time), and the bounds that tests allow."""
import math

import numpy as np

from cache_ref import E32, INVALID, TINY, UNIT

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
EXPONENTS = {"bf16": (-125, 125), "f16": (-23, 13)}


def pack(x, dtype):
    """x (..., dim) float64: (codes, scales), uint8."""
    lo, hi = EXPONENTS[dtype]
    d = x.shape[-1]
    blocks = -(-d // 32)
    x = np.concatenate([x, np.zeros(x.shape[:-1] + (blocks * 32 - d,))], -1).reshape(*x.shape[:-1], blocks, 32)
    odd = ~np.isfinite(x).all(-1)
    x = np.where(odd[..., None], 0, x)
    top = np.abs(x).max(-1)
    e = np.full(top.shape, lo)
    for power in range(lo, hi):
        e[top >= 7 * 2.0 ** power] = power + 1
    y = np.abs(x) / 2.0 ** e[..., None]
    code = np.zeros(y.shape, np.uint8)
    for i in range(1, 8):
        border = (LEVELS[i - 1] + LEVELS[i]) / 2
        code[(y > border) | ((y == border) & (i % 2 == 0))] = i
    code[np.signbit(x)] |= 8
    code[odd] = 0
    code = code.reshape(*code.shape[:-2], blocks * 32)
    return code[..., 0::2] | code[..., 1::2] << 4, np.where(odd, 255, e + 127).astype(np.uint8)


def unpack(codes, scales, dim, dtype):
    n = np.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], 2 * codes.shape[-1])
    v = np.where(n >= 8, -1.0, 1.0) * LEVELS[n & 7]
    f = np.where(scales > EXPONENTS[dtype][1] + 127, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (v * np.repeat(f, 32, -1))[..., :dim]


def visible(p, length, causal, window, sinks):
    j = np.arange(length)
    see = j <= p if causal else np.ones(length, bool)
    if window:
        see &= (j > p - window) | (j < sinks)
    return see


def attend_ref(q, keys, vals, p0, scale, causal=True, window=0, sinks=0):
    """As cache_ref's, with first tokens that every row sees: out, lse,
    weights, the bound of out by type, and those of lse and weights."""
    n, hq, d = q.shape
    length, hk = keys.shape[:2]
    g = hq // hk
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -math.inf)
    spread, lse_err = np.zeros((n, hq, d)), np.zeros((n, hq))
    weights, w_err = np.zeros((hk, length)), np.zeros((hk, length))
    top = np.zeros((n, hq, d))
    for i in range(n):
        see = np.flatnonzero(visible(p0 + i, length, causal, window, sinks))
        if not len(see):
            continue
        for h in range(hq):
            k, v = keys[see, h // g], vals[see, h // g]
            s = scale * (k @ q[i, h])
            m = s.max()
            e = np.exp(s - m)
            w = e / e.sum()
            out[i, h], lse[i, h] = w @ v, m + math.log(e.sum())
            spread[i, h] = w @ np.abs(v)
            top[i, h] = np.abs(v).max(0) * len(see)
            # scores: a dot product of d terms and a scaling, in 32 bits;
            # the sum: a rounding a tile of 16 keys at most, exponentials to 2^-22
            size = scale * (np.abs(k) @ np.abs(q[i, h])).max()
            lse_err[i, h] = E32 * ((d + 8) * size + len(see) / 16 + 64 + 4 * abs(lse[i, h]))
            weights[h // g, see] += w
            w_err[h // g, see] += w * (2 * lse_err[i, h] + 8 * E32)

    def out_bound(dtype):
        # (the probabilities and the result are rounded to the 16-bit type)
        u = UNIT[dtype]
        return 1.05 * u * (np.abs(out) + spread) + 2 * lse_err[..., None] * spread + TINY[dtype] * (1 + top) + 1e-30

    return out, lse, weights, out_bound, lse_err, w_err


# ------------------------------------------------------------------ pages
def names(table, lens, page, n_pages):
    """refs by counting."""
    refs = np.zeros(n_pages, np.int64)
    for row, n in zip(table, lens):
        for p in row[:-(-int(n) // page)]:
            refs[p] += 1
    return refs


def fork_ref(table, lens, page, parents, refs, drop):
    refs = refs.copy()
    new, new_lens = np.full((len(parents), table.shape[1]), INVALID, np.uint32), np.zeros(len(parents), np.uint32)
    for i, p in enumerate(parents):
        if p == INVALID:
            continue
        n = -(-int(lens[p]) // page)
        new[i, :n], new_lens[i] = table[p, :n], lens[p]
        np.add.at(refs, table[p, :n], 1)
    if drop:
        refs -= names(table, lens, page, len(refs))
    return new, new_lens, refs


def grow_ref(table, lens, page, n_new, refs):
    """One sequence after the other; whether a page is shared is asked before any is given."""
    table, lens, refs, shared = table.copy(), lens.copy(), refs.copy(), refs > 1
    free = [p for p in range(len(refs)) if refs[p] == 0]
    src, dst = np.full(len(lens), INVALID, np.uint32), np.full(len(lens), INVALID, np.uint32)
    short, wanted = [], 0
    for b, n in enumerate(n_new):
        n0, n1 = -(-int(lens[b]) // page), -(-(int(lens[b]) + int(n)) // page)
        if n1 > table.shape[1]:
            short.append(b)
            continue
        copy = bool(n and lens[b] % page and shared[table[b, n0 - 1]])
        need = n1 - n0 + copy
        wanted += need
        if need and wanted > len(free):
            short.append(b)
            continue
        got = free[wanted - need:wanted]
        if copy:
            src[b], dst[b] = table[b, n0 - 1], got[0]
            refs[src[b]] -= 1
            n0 -= 1
        table[b, n0:n1] = got
        refs[got] = 1
        lens[b] += n
    return table, lens, refs, src, dst, short


def release_ref(ids, counts, refs):
    refs = refs.copy()
    gone = np.zeros_like(refs)
    for i, row in enumerate(ids):
        for p in row[:len(row) if counts is None else int(counts[i])]:
            if p != INVALID:
                gone[p] += 1
    freed = np.flatnonzero((refs > 0) & (gone >= refs))
    res = np.full(min(len(refs), ids.size), INVALID, np.uint32)
    res[:len(freed)] = freed
    return np.maximum(refs - gone, 0), res, len(freed)


def compact_ref(table, lens, page, refs):
    refs, n = refs.copy(), int((refs > 0).sum())
    src = [p for p in range(n, len(refs)) if refs[p]]
    dst = [p for p in range(n) if not refs[p]]
    to = np.arange(len(refs))
    to[src] = dst
    new = np.full_like(table, INVALID)
    for b, length in enumerate(lens):
        k = -(-int(length) // page)
        new[b, :k] = to[table[b, :k]]
    refs[dst] = refs[src]
    refs[src] = 0
    lists = [np.concatenate([np.array(x, np.uint32), np.full(len(refs) - len(x), INVALID, np.uint32)]) for x in (src, dst)]
    return new, refs, *lists, len(src)
