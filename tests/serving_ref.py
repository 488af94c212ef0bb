"""Plain NumPy statements (64 bits) of the paged cache, the attention over it and the adapters, for their tests."""
import numpy as np

import batq_inputs as bi
from oracle import batq_oracle as o


def rope_table(positions, rot, base=10000.0):
    """fp32 [positions, rot]: cosines of the angles, then sines (angles in 64 bits)."""
    ang = np.arange(positions, dtype=np.float64)[:, None] * base ** (-np.arange(0, rot, 2) / rot)
    return np.concatenate([np.cos(ang), np.sin(ang)], 1).astype(np.float32)


def rotate(x, table, positions, rot, interleaved):
    """x fp32 [M, heads, D]: the definition's fp32 products and sums, each rounded."""
    x = np.array(x, dtype=np.float32)
    c, s = table[positions][:, None, : rot // 2], table[positions][:, None, rot // 2:]
    i, j = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i].copy(), x[..., j].copy()
    x[..., i] = (a * c).astype(np.float32) - (b * s).astype(np.float32)
    x[..., j] = (b * c).astype(np.float32) + (a * s).astype(np.float32)
    return x


def scatter(codes, scales, slots, page, kv_heads, D, row_codes, row_scales):
    """Rows of codes [M, kv_heads * D] and scales [M, kv_heads * D / 32] into the page arrays, in place."""
    pages = codes.shape[0]
    for m, slot in enumerate(slots):
        if 0 <= slot < pages * page:
            codes[slot // page, :, slot % page] = row_codes[m].reshape(kv_heads, D)
            scales[slot // page, :, :, slot % page] = row_scales[m].reshape(kv_heads, D // 32)


def cache_values(codes, scales):
    """[pages, heads, page, D] fp64 values of page arrays (NaN codes give NaN)."""
    s = np.exp2(scales.astype(np.float64) - 127).transpose(0, 1, 3, 2)
    return o.e4m3_value(codes) * np.repeat(s, 32, axis=-1)


def random_cache(rng, pages, page, heads, D, spread=2):
    """Codes without NaN and scales around 1 / 16, so that values are of the order of 1."""
    codes = rng.integers(0, 256, (pages, heads, page, D), dtype=np.uint8)
    codes[(codes & 0x7F) == 0x7F] = 0x31
    codes[(codes & 0x7F) > 0x50] &= 0x8F                    # most magnitudes are small
    scales = rng.integers(121 - spread, 122 + spread, (pages, heads, D // 32, page), dtype=np.uint8)
    return codes, scales


def attention(kv, vv, q, cu, lens, table, page, scale, causal, window, total_q):
    """fp64 attention over cache values kv, vv [pages, heads, page, D]; q [total_q, q_heads, D].
    Returns (out, lse, sum of p |v|, largest sum of |q k| scale) per row and head; rows of no sequence are NaN."""
    pages, heads, _, D = kv.shape
    hq = q.shape[1]
    group = hq // heads
    out, mag = np.full((total_q, hq, D), np.nan), np.full((total_q, hq, D), np.nan)
    lse, smax = np.full((total_q, hq), np.nan), np.zeros((total_q, hq))
    for b, L in enumerate(lens):
        n = cu[b + 1] - cu[b]
        t = np.arange(L)
        ids = table[b][t // page] if L else np.zeros(0, np.int64)
        known = (ids >= 0) & (ids < pages)
        K = np.where(known[:, None, None], kv[np.where(known, ids, 0), :, t % page], 0.0)       # [L, heads, D]
        V = np.where(known[:, None, None], vv[np.where(known, ids, 0), :, t % page], 0.0)
        for i in range(n):
            pos = L - n + i
            see = known & ((t <= pos) if causal else (t < L))
            if window:
                see &= t > pos - window
            for h in range(hq):
                row = cu[b] + i
                if not see.any():
                    out[row, h], mag[row, h], lse[row, h] = 0.0, 0.0, -np.inf
                    continue
                s = (K[see, h // group] @ q[row, h]) * scale
                smax[row, h] = (np.abs(K[see, h // group]) @ np.abs(q[row, h])).max() * scale
                m = s.max()
                p = np.exp(s - m)
                lse[row, h] = m + np.log(p.sum())
                p /= p.sum()
                out[row, h] = p @ V[see, h // group]
                mag[row, h] = p @ np.abs(V[see, h // group])
    return out, lse, mag, smax


def assert_attention(got, lse, ref, terms=1):
    """Bounds: a score is off by at most (D + 8) 2^-24 of sum |q k| scale (fp32 sums of exact products), which moves p by
    that factor; p is rounded to bf16 (`terms` 1: 2^-8 each, 2: 2^-16), the sums are fp32 and the output bf16 (2^-8)."""
    out, ref_lse, mag, smax = ref
    rows = ~np.isnan(ref_lse)
    drift = (136 * 2.0 ** -24 * smax + 2.0 ** -18)[..., None]
    tol = 2.0 ** -8 * np.abs(out) + (2.0 ** (-8 * terms) + 2 * drift) * mag * (1 + 2.0 ** -8) + 1e-30
    bad = np.abs(got - out) > tol
    assert not bad[rows].any(), (np.argwhere(bad & rows[..., None])[:4], np.abs(got - out)[bad & rows[..., None]][:4])
    assert np.isfinite(got[rows]).all()
    if lse is not None:
        live = rows & np.isfinite(ref_lse)
        assert np.all(np.abs(lse[live] - ref_lse[live]) <= drift[..., 0][live] + 2.0 ** -22 * (1 + np.abs(ref_lse[live])))
        assert np.all(lse[rows & ~np.isfinite(ref_lse)] == -np.inf)


def bf16_values(rng, *shape, scale=1.0):
    """(bf16 bits uint16, the values as fp32)."""
    bits = bi.f32_to_bf16_bits((scale * rng.standard_normal(shape)).astype(np.float32))
    return bits, bi.bf16_bits_to_f32(bits)
