"""Plain NumPy statements (64 bits) of caches in 4 or 8 bits, of the scores of their tokens and of eviction, for their tests."""
import numpy as np

import serving_ref as ref

E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def values(codes, scales, bits):
    """[pages, heads, page, D] fp64 values of page arrays; scale byte 255 is NaN."""
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127)).transpose(0, 1, 3, 2)
    if bits == 8:
        with np.errstate(invalid="ignore"):
            return np.where(np.isnan(np.repeat(s, 32, -1)), np.nan, ref.cache_values(codes, np.minimum(scales, 254)))
    v = np.stack([E2M1[codes & 15], E2M1[codes >> 4]], -1).reshape(*codes.shape[:-1], -1)
    return v * np.repeat(s, 32, -1)


def random_arrays(rng, pages, page, heads, D, bits):
    """Codes and scales of keys and of values, of the order of 1."""
    out = []
    for _ in range(2):
        codes, scales = ref.random_cache(rng, pages, page, heads, D)
        if bits == 4:
            codes, scales = rng.integers(0, 256, (pages, heads, page, D // 2), dtype=np.uint8), scales + np.uint8(3)
        out += [codes, scales]
    return out


def batch_case(rng, lens, qs, hq, hkv, D, page, bits, spare=0, more_pages=2):
    """(arrays, q as bf16 bits [T, hq D], q [T, hq, D], cu, lens, table, T): what no token was written to holds NaN."""
    lens, qs = np.array(lens), np.array(qs)
    per = -(-lens // page)
    pages = int(per.sum()) + more_pages
    arrays = random_arrays(rng, pages, page, hkv, D, bits)
    order = rng.permutation(pages)
    table = np.full((len(lens), max(1, int(per.max()))), -7, np.int32)
    filled, at = np.zeros(pages, np.int64), 0
    for b in range(len(lens)):
        mine = order[at: at + per[b]]
        at += per[b]
        table[b, : per[b]] = mine
        filled[mine] = np.minimum(page, lens[b] - page * np.arange(per[b]))
    empty = np.arange(page)[None] >= filled[:, None]
    for n in (0, 2):
        arrays[n][np.broadcast_to(empty[:, None, :, None], arrays[n].shape)] = 0x7F
        arrays[n + 1][np.broadcast_to(empty[:, None, None, :], arrays[n + 1].shape)] = 255
    cu = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
    T = int(cu[-1]) + spare
    qbits, q = ref.bf16_values(rng, T, hq * D)
    return arrays, qbits, q.reshape(T, hq, D).astype(np.float64), cu, lens.astype(np.int32), table, T


def score(kv, q, lse, had, cu, lens, table, page, scale, causal, window, add, max_q=None):
    """fp64 scores [pages, heads, page] after a call on `had`, and how far an fp32 computation may be off them (-1: not touched):
    a score is off by (D + 8) 2^-24 of sum |q k| scale (fp32 sums of exact products); it and lse are multiplied with a rounded
    log2 e and subtracted, 2^-24 of each four times at most; exp2 to 2^-23; sums of positive numbers, at most N + 8 additions
    for N rows (those of masked rows are exact); a weight below 2^-126 may be zero."""
    pages, heads, _, D = kv.shape
    hq = q.shape[1]
    group = hq // heads
    want, tol = had.astype(np.float64), np.full(had.shape, -1.0)
    for b, L in enumerate(lens):
        true_n = cu[b + 1] - cu[b]
        n = true_n if max_q is None else min(true_n, max_q)
        t = np.arange(L)
        ids = table[b][t // page] if L else np.zeros(0, np.int64)
        known = (ids >= 0) & (ids < pages)
        t, ids = t[known], ids[known]
        pos = (L - true_n + np.arange(n))[:, None]
        see = np.broadcast_to(t <= pos if causal else t < L, (n, len(t))).copy()
        if window:
            see &= t > pos.astype(np.int64) - window
        for h in range(heads):
            K = kv[ids, h, t % page]
            w, off = np.zeros(len(t)), np.zeros(len(t))
            for g in range(h * group, (h + 1) * group):
                rows = q[cu[b]: cu[b] + n, g]
                s, mag = rows @ K.T * scale, np.abs(rows) @ np.abs(K).T * scale
                ls = lse[cu[b]: cu[b] + n, g].astype(np.float64)[:, None]
                dead = ls == -np.inf
                with np.errstate(invalid="ignore"):
                    p = np.where(see & ~dead, np.exp(s - np.where(dead, 0.0, ls)), 0.0)
                    drift = np.where(see & ~dead, 2.0 ** -24 * ((D + 12) * mag + 4 * np.abs(np.where(dead, 0.0, ls)) + 4), 0.0)
                w += p.sum(0)
                off += (p * (drift * 1.01 + 2.0 ** -23)).sum(0) + n * 2.0 ** -126
            old = np.where(add & (t < L - true_n), had[ids, h, t % page].astype(np.float64), 0.0)
            want[ids, h, t % page] = w + old
            tol[ids, h, t % page] = off + (n * group + 8) * 2.0 ** -24 * (w + np.abs(old))
    return want, tol


def assert_score(got, want_tol, had):
    want, tol = want_tol
    untouched = tol == -1
    bad = ~(np.abs(got - want) <= tol) & ~(np.isnan(got) & np.isnan(want)) & ~untouched
    assert not bad.any(), (np.argwhere(bad)[:4], got[bad][:4], want[bad][:4], tol[bad][:4])
    assert np.array_equal(got[untouched], had[untouched])


def evict(arrays, score_, lens, table, out_table, budget, first, last):
    """(arrays, score, keep, new_len) after an eviction; lens as the call takes them."""
    pages, heads, page = score_.shape
    got, sc = [a.copy() for a in arrays], score_.copy()
    keep, new_len = np.full((len(lens), heads, budget), -1, np.int32), np.zeros(len(lens), np.int32)
    for b, L in enumerate(lens):
        t = np.arange(L)
        new_len[b] = n = min(L, budget)
        ids = table[b][t // page] if L else np.zeros(0, np.int64)
        known = (ids >= 0) & (ids < pages)
        for h in range(heads):
            x = np.where(known, score_[np.where(known, ids, 0), h, t % page], np.nan).astype(np.float64)
            rank = np.where(np.isnan(x), -1, np.searchsorted(np.unique(x[~np.isnan(x)]), np.where(np.isnan(x), 0, x)))
            rank[(t < first) | (t >= L - last)] = L + 1
            kept = np.sort(np.argsort(-rank, kind="stable")[:n])
            keep[b, h, :n] = kept
            j = np.arange(n)
            dst = out_table[b][j // page] if n else j
            moved = known[kept] & (dst >= 0) & (dst < pages)
            j, src, dst = j[moved], kept[moved], dst[moved]
            for i in (0, 2):
                got[i][dst, h, j % page] = arrays[i][ids[src], h, src % page]
                got[i + 1][dst, h, :, j % page] = arrays[i + 1][ids[src], h, :, src % page]
            sc[dst, h, j % page] = score_[ids[src], h, src % page]
    return got, sc, keep, new_len
