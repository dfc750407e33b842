"""The cache operators' definitions in 64 bits (numpy, one row at a time), the
bounds that their tests allow, and small random caches."""
import math

import numpy as np

INVALID = 0xFFFFFFFF
UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}   # unit roundoff: 8 and 11 significant bits
TINY = {"bf16": 0.0, "f16": 2.0 ** -25}         # and their absolute error below the normal range
E32 = 2.0 ** -24


def attend_ref(q, keys, vals, p0, scale, causal=True, window=0):
    """One sequence: q rows x heads x dim, keys / vals len x kv_heads x dim
    (float64).  Returns out, lse, weights (kv_heads x len) and the bounds of
    out, lse and weights for a computation that rounds the probabilities and
    the result to the 16-bit type and keeps everything else in 32 bits
    (bounds are functions of the type: out_bound(type))."""
    n, hq, d = q.shape
    length, hk = keys.shape[:2]
    g = hq // hk
    out, lse = np.zeros((n, hq, d)), np.full((n, hq), -math.inf)
    spread, lse_err = np.zeros((n, hq, d)), np.zeros((n, hq))
    weights, w_err = np.zeros((hk, length)), np.zeros((hk, length))
    top = np.zeros((n, hq, d))
    for i in range(n):
        hi = min(length, p0 + i + 1) if causal else length
        lo = max(0, p0 + i - window + 1) if window else 0
        if hi <= lo:
            continue
        for h in range(hq):
            k, v = keys[lo:hi, h // g], vals[lo:hi, h // g]
            s = scale * (k @ q[i, h])
            m = s.max()
            e = np.exp(s - m)
            w = e / e.sum()
            seen = w @ v
            out[i, h], lse[i, h] = seen, m + math.log(e.sum())
            spread[i, h] = w @ np.abs(v)
            top[i, h] = np.abs(v).max(0) * (hi - lo)
            # scores: a dot product of d terms and a scaling, in 32 bits;
            # the sum: a rounding a tile of 16 keys at most, exponentials to 2^-22
            size = scale * (np.abs(k) @ np.abs(q[i, h])).max()
            lse_err[i, h] = E32 * ((d + 8) * size + (hi - lo) / 16 + 64 + 4 * abs(lse[i, h]))
            weights[h // g, lo:hi] += w
            w_err[h // g, lo:hi] += w * (2 * lse_err[i, h] + 8 * E32)

    def out_bound(dtype):
        u = UNIT[dtype]
        return (1.05 * u * (np.abs(out) + spread) + 2 * lse_err[..., None] * spread + TINY[dtype] * (1 + top) + 1e-30)

    return out, lse, weights, out_bound, lse_err, w_err


def ids_ref(q, k_slots, v_slots, ids, scale, prior=None):
    """q seqs x heads x dim, k_slots / v_slots slots x kv_heads x dim."""
    b, hq, d = q.shape
    g = hq // k_slots.shape[1]
    out, lse = np.zeros((b, hq, d)), np.full((b, hq), -math.inf)
    spread, lse_err = np.zeros((b, hq, d)), np.zeros((b, hq))
    for i in range(b):
        for h in range(hq):
            x = [j for j in ids[i, h] if j != INVALID]
            parts = []
            if x:
                k, v = k_slots[x, h // g], v_slots[x, h // g]
                s = scale * (k @ q[i, h])
                parts = [(s[j], v[j]) for j in range(len(x))]
                size = scale * (np.abs(k) @ np.abs(q[i, h])).max()
                lse_err[i, h] = E32 * ((d + 8) * size + len(x) + 64)
            if prior is not None and prior[1][i, h] > -math.inf:
                parts.append((prior[1][i, h], prior[0][i, h]))
                lse_err[i, h] += E32 * 4 * abs(prior[1][i, h])
            if not parts:
                continue
            s, v = np.array([p[0] for p in parts]), np.stack([p[1] for p in parts])
            m = s.max()
            e = np.exp(s - m)
            out[i, h], lse[i, h] = e @ v / e.sum(), m + math.log(e.sum())
            spread[i, h] = e @ np.abs(v) / e.sum()
            lse_err[i, h] += E32 * 4 * abs(lse[i, h])

    def out_bound(dtype):
        return 1.05 * UNIT[dtype] * np.abs(out) + (2 * lse_err + E32 * 64)[..., None] * spread + TINY[dtype] + 1e-30

    return out, lse, out_bound, lse_err


def evict_ref(table, lens, weights, budget, page, sinks, recent):
    """numpy, one sequence and page at a time; scores are 32-bit sums head by
    head and token by token."""
    n_seq, max_pages = table.shape
    heads, cap = weights.shape[1:]
    new_table, freed = np.full_like(table, INVALID), np.full_like(table, INVALID)
    new_w = np.zeros_like(weights)
    new_lens, n_freed = np.zeros(n_seq, np.uint32), np.zeros(n_seq, np.uint32)
    for b in range(n_seq):
        length = int(lens[b])
        n = -(-length // page)
        tail = min(n, max(recent, 1 if length % page else 0))
        fixed = {p for p in range(n) if p < sinks or p >= n - tail}
        score = {}
        for p in range(n):
            s = np.float32(0)
            for h in range(heads):
                for t in range(p * page, min(length, (p + 1) * page)):
                    s = np.float32(s + weights[b, h, t])
            score[p] = -math.inf if np.isnan(s) else float(s)
        rest = sorted((p for p in range(n) if p not in fixed), key=lambda p: (-score[p], p))
        room = max(0, min(n, int(budget[b])) - len(fixed))
        keep = sorted(fixed | set(rest[:room]))
        gone = sorted(set(range(n)) - set(keep))
        new_table[b, :len(keep)] = table[b, keep]
        freed[b, :len(gone)] = table[b, gone]
        tokens = [t for p in keep for t in range(p * page, min(length, (p + 1) * page))]
        new_w[b, :, :len(tokens)] = weights[b][:, tokens]
        new_lens[b], n_freed[b] = len(tokens), len(gone)
    return new_table, new_w, new_lens, freed, n_freed
