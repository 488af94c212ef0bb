"""The paged cache in 4 bits: batq_kv_paged_append and batq_paged_attention on it, against plain 64-bit statements."""
import numpy as np
import pytest

import batq_inputs as bi
from oracle import batq_oracle as o
from gpu_util import require_gpu, to_dev, y_to_f32
import budget_ref as br
import serving_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    require_gpu()
    import paper_2603_16590_amd as b
    return b


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def make_cache(B, arrays, bits=4):
    pages, heads, page, D = arrays[0].shape
    return B.PagedCache(pages, page, heads, D * 8 // bits, tensors=[dev(a) for a in arrays], bits=bits)


def host(cache):
    return [t.cpu().numpy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


# ---------------------------------------------------------------------------------------- append
APPEND = [
    # M, q heads, kv heads, D, page, rot, interleaved, dtype
    (1, 4, 4, 64, 16, 64, False, "bf16"),
    (1, 32, 8, 128, 16, 128, False, "bf16"),
    (31, 7, 1, 128, 32, 64, True, "f32"),
    (33, 0, 3, 64, 256, 16, False, "f32"),
    (65, 8, 2, 64, 16, 32, True, "bf16"),
    (200, 28, 4, 128, 16, 0, False, "bf16"),
    (311, 12, 3, 64, 128, 64, False, "f32"),
]
# more than 16 D units of 32 tokens x 32 channels: the kernel for many tokens, in every layout (head width, element size), pair
# distance and direction that it takes; 15 heads leave a wave of the last workgroup without one, the last tile is ragged
MANY = [(4489, 9, 3, D, 64, rot, inter, dtype) for D, rot, inter, dtype in (
    (64, 64, False, "bf16"), (64, 64, False, "f32"), (64, 16, True, "bf16"), (64, 0, False, "f32"), (128, 64, False, "bf16"),
    (128, 128, False, "bf16"), (128, 128, False, "f32"), (128, 48, True, "f32"), (128, 0, False, "bf16"))]


def append_case(rng, M, hq, hkv, D, page, dtype):
    """q, k, v as fp32 [M, heads, D] and on the device, positions, slots, pages: slots scattered, some unused."""
    X = rng.standard_normal((M, (hq + 2 * hkv) * D + 8)).astype(np.float32)
    X[:, ::37] *= 30.0
    X[M // 2, :64] = 0.0                                    # zero blocks
    X[M // 3, -72:-8] *= 0.0 if M % 2 else -0.0             # and of -0
    if dtype == "bf16":
        bits = bi.f32_to_bf16_bits(X)
        X, Xd = bi.bf16_bits_to_f32(bits), to_dev(bits, "bf16")
    else:
        Xd = to_dev(X, "f32")
    cut = np.cumsum([0, hq * D, hkv * D, hkv * D])
    parts = [X[:, cut[i]: cut[i + 1]].reshape(M, -1, D) for i in range(3)]
    dparts = [Xd[:, cut[i]: cut[i + 1]] for i in range(3)]
    pages = -(-M // page) + 3
    slots = rng.permutation(pages * page)[:M].astype(np.int64)
    positions = rng.integers(0, 1000, M).astype(np.int32)
    if M > 4:
        slots[[1, M // 2]] = -1, pages * page               # unused and past the end
        positions[[2, 3]] = -1, 1000                        # outside the table
    return parts, dparts, positions, slots, pages


def scatter(arrays, n, slots, page, row_codes, row_scales):
    pages, heads, _, width = arrays[n].shape
    for m, slot in enumerate(slots):
        if 0 <= slot < pages * page:
            arrays[n][slot // page, :, slot % page] = row_codes[m].reshape(heads, width)
            arrays[n + 1][slot // page, :, :, slot % page] = row_scales[m].reshape(heads, -1)


@pytest.mark.parametrize("M,hq,hkv,D,page,rot,inter,dtype", APPEND + MANY)
def test_append_without_transforms_is_bit_exact(B, M, hq, hkv, D, page, rot, inter, dtype):
    import torch
    rng = np.random.default_rng(M + hq + D + rot)
    (q, k, v), (qd, kd, vd), positions, slots, pages = append_case(rng, M, hq, hkv, D, page, dtype)
    arrays = br.random_arrays(rng, pages, page, hkv, D, 4)
    cache = make_cache(B, arrays)
    table = ref.rope_table(1000, rot) if rot else None
    q_out = torch.full((M, hq * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    B.batq_kv_paged_append(cache, kd, vd, dev(slots), positions=dev(positions) if rot else None, q=qd if hq else None,
                           q_out=q_out[:, : hq * D] if hq else None, rope=dev(table) if rot else None, interleaved=inter)
    torch.cuda.synchronize()
    left_out = np.zeros(M, bool)
    if rot:
        left_out = (positions < 0) | (positions >= 1000)
        at = np.where(left_out, 0, positions)
        q, k = ref.rotate(q, table, at, rot, inter), ref.rotate(k, table, at, rot, inter)
    used = np.where(left_out, -1, slots)
    want = [a.copy() for a in arrays]
    for n, x in ((0, k), (2, v)):
        scatter(want, n, used, page, *o.mxfp4_quantize(x.reshape(M, -1)))
    for got, w, name in zip(host(cache), want, ("k codes", "k scales", "v codes", "v scales")):
        assert np.array_equal(got, w), name
    if hq:
        got = y_to_f32(q_out)
        assert np.array_equal(got[~left_out, : hq * D], o.bf16_round(q.reshape(M, -1))[~left_out])
        assert np.all(got[left_out] == 7.0) and np.all(got[:, hq * D:] == 7.0)


def transforms(B, rng, width, form):
    G = (np.eye(4) + 0.05 * rng.standard_normal((4, 4))).astype(np.float32)
    P = (np.eye(8) + 0.05 * rng.standard_normal((width // 32, 8, 8))).astype(np.float32)
    c = rng.uniform(0.85, 1.0, width // 32).astype(np.float32)
    T = o.kron_blocks(G, P)
    if form == "kron":
        return B.Transform(width, G, P, c), T, c
    return B.Transform.general(width, dense=T.astype(np.float32), clip=c), T.astype(np.float32).astype(np.float64), c


@pytest.mark.parametrize("M,hq,hkv,D,page,rot,inter,dtype", [c for c in APPEND if c[0] > 1] + [MANY[0], MANY[3], MANY[5], MANY[7]])
@pytest.mark.parametrize("form", ["kron", "dense"])
def test_append_with_transforms(B, M, hq, hkv, D, page, rot, inter, dtype, form):
    """Codes against the 64-bit transform: an element may sit on the other side of a rounding border only if the
    exact value is within the transform's accuracy (2^-19 of the block's largest sum |x| |T|) of it."""
    import torch
    rng = np.random.default_rng(M + hq + D + rot + 1)
    (q, k, v), (qd, kd, vd), positions, slots, pages = append_case(rng, M, hq, hkv, D, page, dtype)
    arrays = br.random_arrays(rng, pages, page, hkv, D, 4)
    cache = make_cache(B, arrays)
    tk, Tk, ck = transforms(B, rng, hkv * D, form)
    tv, Tv, cv = transforms(B, rng, hkv * D, form)
    table = ref.rope_table(1000, rot) if rot else None
    B.batq_kv_paged_append(cache, kd, vd, dev(slots), positions=dev(positions) if rot else None, q=qd if hq else None,
                           rope=dev(table) if rot else None, interleaved=inter, tk=tk, tv=tv)
    torch.cuda.synchronize()
    left_out = ((positions < 0) | (positions >= 1000)) if rot else np.zeros(M, bool)
    if rot:
        k = ref.rotate(k, table, np.where(left_out, 0, positions), rot, inter)
    live = ~left_out & (slots >= 0) & (slots < pages * page)
    got = host(cache)
    for n, x, T, c in ((0, k, Tk, ck), (2, v, Tv, cv)):
        x = x.reshape(M, -1).astype(np.float64)
        y, absy = o.apply_blocks(x, T), o.apply_blocks(np.abs(x), np.abs(T))
        want_c, want_s = o.mxfp4_quantize(y.astype(np.float32), c)
        gc = got[n][slots[live] // page, :, slots[live] % page].reshape(live.sum(), -1)
        gs = got[n + 1][slots[live] // page, :, :, slots[live] % page].reshape(live.sum(), -1)
        assert np.mean(gc != want_c[live]) <= 1e-3 and np.mean(gs != want_s[live]) <= 1e-3
        val = o.dequantize(gc, gs)
        y, absy = y[live], absy[live]
        lim = np.repeat(np.abs(y).reshape(len(y), -1, 32).max(-1) * c, 32, 1)
        unit = np.repeat(np.exp2(gs.astype(np.float64) - 127), 32, 1)
        clipped = np.clip(np.clip(y, -lim, lim), -6 * unit, 6 * unit)
        step = unit * np.where(np.abs(clipped) < 2 * unit, 0.5, np.where(np.abs(clipped) < 4 * unit, 1.0, 2.0))
        assert np.all(np.abs(val - clipped) <= step / 2 + 2.0 ** -19 * np.repeat(absy.reshape(len(y), -1, 32).max(-1), 32, 1))
        mask = np.ones(got[n].shape, bool)                  # nothing else was touched
        mask[slots[live] // page, :, slots[live] % page] = False
        assert np.array_equal(got[n][mask], arrays[n][mask])


@pytest.mark.parametrize("kind", ["kron", "minmax", "clip only"])
@pytest.mark.parametrize("D,M,hkv", [(128, 150, 2), (64, 90, 3), (128, 4700, 4)])
def test_append_without_rotation_writes_the_bytes_of_batq_kv_append(B, kind, D, M, hkv):
    """One sequence in page order, few tokens in pieces of any size or many at once: the pages hold what the row-window cache
    holds, byte for byte."""
    import torch
    rng = np.random.default_rng(5)
    page, width = 32, hkv * D
    X = to_dev(ref.bf16_values(rng, M, width)[0], "bf16")
    if kind == "kron":
        t = transforms(B, rng, width, "kron")[0]
    elif kind == "clip only":
        t = B.Transform(width, None, None, rng.uniform(0.7, 1.0, width // 32).astype(np.float32))
    else:
        lo, hi = (rng.uniform(0.7, 1.0, width // 32).astype(np.float32) for _ in range(2))
        t = B.Transform.general(width, outer=np.eye(4, dtype=np.float32) * 1.25,
                                inner=(np.eye(8) + 0.05 * rng.standard_normal((width // 32, 8, 8))), clip_min=lo, clip_max=hi)
    cache = B.PagedCache(-(-M // page), page, hkv, D, bits=4)
    for lo, hi in ((0, 1), (1, 40), (40, M)) if M < 1000 else ((0, M),):
        B.batq_kv_paged_append(cache, X[lo:hi], X[lo:hi], torch.arange(lo, hi, device="cuda"), tk=t, tv=t)
    codes = torch.zeros(B.batq_code_bytes(M, width), dtype=torch.uint8, device="cuda")
    scales = torch.zeros(B.batq_scale_bytes(M, width), dtype=torch.uint8, device="cuda")
    B.batq_kv_append(t, X, codes, scales, 0, M, bits=4)
    rc, rs = B.batq_codes_to_rowmajor(codes, M, width), B.batq_scales_to_rowmajor(scales, M, width)
    torch.cuda.synchronize()
    for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
        assert torch.equal(c.permute(0, 2, 1, 3).reshape(-1, width // 2)[:M], rc)
        assert torch.equal(s.permute(0, 3, 1, 2).reshape(-1, width // 32)[:M], rs)


@pytest.mark.parametrize("D,rot,inter,dtype", [(128, 128, False, "bf16"), (64, 64, False, "f32"), (128, 64, True, "f32")])
def test_append_of_many_tokens_equals_single_ones(B, D, rot, inter, dtype):
    """A long call, calls of 96 tokens (another kernel) and single tokens of neighbouring places leave the same bytes."""
    import torch
    rng = np.random.default_rng(D + rot)
    M, hq, hkv, page = 4489, 9, 3, 128
    X = torch.randn((M, (hq + 2 * hkv) * D), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, k, v = X.split((hq * D, hkv * D, hkv * D), 1)
    tk, tv = transforms(B, rng, hkv * D, "kron")[0], transforms(B, rng, hkv * D, "dense")[0]
    table = dev(ref.rope_table(4000, rot))
    slots, pos = torch.randperm(40 * page, device="cuda")[:M], torch.randint(0, 4000, (M,), device="cuda", dtype=torch.int32)
    slots[:60] = torch.arange(60, device="cuda")
    slots[60:] = torch.randperm(40 * page - 60, device="cuda")[: M - 60] + 60
    slots[[99, M - 1]], slots[4000], pos[133] = -1, 40 * page, -5
    a, b = B.PagedCache(40, page, hkv, D, bits=4), B.PagedCache(40, page, hkv, D, bits=4)
    qa = torch.full((M, hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
    qb = qa.clone()
    B.batq_kv_paged_append(a, k, v, slots, pos, q=q, q_out=qa, rope=table, interleaved=inter, tk=tk, tv=tv)
    for lo, hi in [(i, i + 1) for i in range(60)] + [(i, min(M, i + 96)) for i in range(60, M, 96)]:
        s = slice(lo, hi)
        B.batq_kv_paged_append(b, k[s], v[s], slots[s], pos[s], q=q[s], q_out=qb[s], rope=table, interleaved=inter, tk=tk, tv=tv)
    torch.cuda.synchronize()
    assert torch.equal(qa, qb)
    for x, y in zip(host(a), host(b)):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("D,M,rot,dtype", [(64, 40, 64, "bf16"), (128, 33, 0, "f32"), (128, 4489, 128, "bf16"), (64, 4489, 0, "f32")])
@pytest.mark.parametrize("bits", [4, 8])
def test_append_never_writes_scale_byte_255(B, D, M, rot, dtype, bits):
    """Not for NaN and infinite elements either (their blocks' codes are nobody's promise); all other blocks are as without them."""
    import torch
    rng = np.random.default_rng(91 + M + D)
    hkv, page = 3, 64
    X = rng.standard_normal((M, 2 * hkv * D)).astype(np.float32)
    if dtype == "bf16":
        X = bi.bf16_bits_to_f32(bi.f32_to_bf16_bits(X))
    odd = X.copy()
    hit = np.zeros((M, 2 * hkv * D // 32), bool)
    for i, x in enumerate((np.nan, -np.nan, np.inf, -np.inf, "all")):
        m = (7 * i + 3) % M
        if x == "all":
            odd[m, : D] = np.nan
            hit[m, : D // 32] = True
        else:
            odd[m, 5 + 32 * i], odd[m, hkv * D + 9] = x, x
            hit[m, (5 + 32 * i) // 32] = hit[m, (hkv * D + 9) // 32] = True
    if rot:                                                 # a rotated channel's partner is half of the rotation away
        hit |= hit.reshape(M, 2, hkv, D // 32).any(3, keepdims=True).repeat(D // 32, 3).reshape(M, -1)
    caches = []
    for x in (X, odd):
        xd = to_dev(bi.f32_to_bf16_bits(x), "bf16") if dtype == "bf16" else to_dev(x, "f32")
        cache = B.PagedCache(-(-M // page), page, hkv, D, bits=bits)
        B.batq_kv_paged_append(cache, xd[:, : hkv * D], xd[:, hkv * D:], torch.arange(M, device="cuda"),
                               positions=torch.arange(M, dtype=torch.int32, device="cuda") if rot else None, rope=dev(ref.rope_table(M, rot)) if rot else None)
        torch.cuda.synchronize()
        caches.append(host(cache))
    fine = ~hit.reshape(M, 2, hkv, D // 32)
    for n in range(4):
        a, b = (c[n].transpose(0, 2, 1, 3).reshape(-1, hkv, D // 32, 4 * bits) if n % 2 == 0 else c[n].transpose(0, 3, 1, 2).reshape(-1, hkv, D // 32, 1)
                for c in caches)
        assert np.array_equal(a[:M][fine[:, n // 2]], b[:M][fine[:, n // 2]])
        assert n % 2 == 0 or not (b == 255).any()


# ---------------------------------------------------------------------------------------- attention
def run_attention(B, cache, qd, cu, lens, table, T, hq, max_q=None, max_kv=None, **kw):
    import torch
    D = cache.head_dim
    out = torch.full((T, hq * D + 8), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, hq), 7.0, dtype=torch.float32, device="cuda")
    max_q = int(np.diff(cu).max()) if max_q is None else max_q
    max_kv = int(max(lens)) if max_kv is None else max_kv
    B.batq_paged_attention(cache, qd, dev(cu), dev(lens), dev(table), max_q, max_kv, out=out[:, : hq * D], lse=lse, **kw)
    torch.cuda.synchronize()
    got = y_to_f32(out).astype(np.float64)
    assert np.all(got[:, hq * D:] == 7.0)
    assert np.all(got[cu[-1]:, : hq * D] == 7.0) and bool((lse[int(cu[-1]):] == 7.0).all())
    return got[:, : hq * D].reshape(T, hq, D), lse.cpu().numpy().astype(np.float64)


ATTEND = [
    # lens, query counts, q heads, kv heads, D, page, window
    ([1], [1], 1, 1, 64, 16, 0),
    ([64], [1], 4, 1, 128, 16, 0),
    ([1, 15, 16, 17, 63, 64, 65, 129], [1] * 8, 8, 2, 128, 16, 0),
    ([0, 5, 0, 300], [1, 1, 2, 1], 7, 1, 128, 32, 0),
    ([700, 3, 1025], [1, 1, 1], 28, 4, 64, 64, 0),
    ([513, 40], [3, 2], 8, 4, 64, 256, 0),
    ([200, 90], [5, 7], 6, 2, 128, 16, 33),
    ([300, 20], [10, 20], 32, 1, 64, 16, 0),
    ([1000], [1], 16, 1, 128, 128, 64),
    ([333], [333], 3, 3, 64, 32, 0),
    ([290], [290], 8, 1, 128, 16, 0),
    ([130, 64, 257, 1], [130, 1, 100, 1], 14, 2, 128, 64, 0),
    ([200, 140], [70, 140], 4, 4, 128, 32, 1),
    ([500], [129], 2, 1, 64, 16, 100),
    ([77], [40], 40, 1, 128, 16, 0),
    ([5, 9], [9, 20], 4, 2, 64, 16, 0),                     # more queries than tokens: the first ones see nothing
]


@pytest.mark.parametrize("lens,qs,hq,hkv,D,page,window", ATTEND)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(B, lens, qs, hq, hkv, D, page, window, causal):
    rng = np.random.default_rng(sum(lens) + sum(qs) + hq)
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 4, spare=3)
    got, lse = run_attention(B, make_cache(B, arrays), to_dev(qbits, "bf16"), cu, lens, table, T, hq, causal=causal, window=window)
    want = ref.attention(br.values(*arrays[:2], 4), br.values(*arrays[2:], 4), q, cu, lens, table, page, D ** -0.5, causal, window, T)
    ref.assert_attention(got, lse, want, terms=2 if max(qs) * (hq // hkv) <= 32 else 1)


@pytest.mark.parametrize("lens,qs,hq,hkv,D,page,window", [
    ([20000, 9, 7001, 1, 15000], [1, 1, 4, 1, 2], 8, 2, 128, 64, 0), ([9000, 300], [1, 2], 4, 1, 64, 16, 1000),
    ([3000, 1500, 2500], [70, 1, 300], 4, 1, 64, 16, 700), ([4000], [200], 2, 1, 128, 64, 0)])
def test_attention_of_long_sequences(B, lens, qs, hq, hkv, D, page, window):
    """Cut into parts that are joined, with and without a window."""
    rng = np.random.default_rng(3 + hq)
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 4)
    got, lse = run_attention(B, make_cache(B, arrays), to_dev(qbits, "bf16"), cu, lens, table, T, hq, window=window)
    ref.assert_attention(got, lse, ref.attention(br.values(*arrays[:2], 4), br.values(*arrays[2:], 4), q, cu, lens, table, page, D ** -0.5, True, window, T))


def test_attention_does_not_trust_its_lists(B):
    rng = np.random.default_rng(6)
    hq, hkv, D, page = 4, 2, 128, 16
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [100, 40, 64, 90], [1, 3, 20, 1], hq, hkv, D, page, 4, spare=2)
    table[0, 2], table[2, 0], table[2, 3], table[1, 0] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1
    table[3, :] = -1                                        # a sequence without any page
    got, lse = run_attention(B, make_cache(B, arrays), to_dev(qbits, "bf16"), cu, lens, table, T, hq, max_kv=128)
    kv, vv = br.values(*arrays[:2], 4), br.values(*arrays[2:], 4)
    ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, 0, T))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("byte", [255, 253])
def test_blocks_that_are_not_finite(B, D, byte):
    """Scale byte 255 is NaN whatever the codes are; 6 x 2^(253 - 127) is infinite in bf16.  A key makes the rows that see it NaN (255),
    a value its block of 32 channels, or those of them that are not finite; where nobody looks it does nothing."""
    rng = np.random.default_rng(22 + D)
    page = 16
    for hq, hkv, lens, qs, window in ((4, 2, [200, 90], [1, 1], 0), (4, 2, [200], [200], 50), (6, 2, [300, 70], [3, 2], 0), (2, 1, [1000], [130], 0)):
        arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 4)
        for what in (1, 3) if byte == 255 else (3,):
            a = [x.copy() for x in arrays]
            for tok in (int(lens[0]) - 1, int(lens[0]) - 1 - min(60, qs[0])):
                a[what][table[0, tok // page], hkv - 1, D // 32 - 1, tok % page] = byte
                if byte == 253:                             # every second channel 6, the others 1
                    a[2][table[0, tok // page], hkv - 1, tok % page, (D - 32) // 2:] = 0x27
            kv, vv = br.values(*a[:2], 4), br.values(*a[2:], 4)
            vv = np.where(np.abs(vv) >= 2.0 ** 128, np.nan, vv)
            with np.errstate(invalid="ignore", over="ignore"):
                want = ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, window, T)
            got, lse = run_attention(B, make_cache(B, a), to_dev(qbits, "bf16"), cu, lens, table, T, hq, window=window)
            assert np.isnan(want[0]).any() and not np.isnan(want[0]).all()
            # a row that sees an infinite value has an infinity there, or NaN
            assert np.array_equal(~np.isfinite(got), np.isnan(want[0])) and np.array_equal(np.isnan(lse), np.isnan(want[1]))


def test_attention_past_four_gigabytes(B):
    """Offsets into the code arrays beyond 32 bits: pages at either end of a pool of 4.2 GB per array."""
    import torch
    rng = np.random.default_rng(10)
    hq, hkv, D, page, L = 4, 1, 128, 256, 300
    pages = (1 << 32) // (page * D // 2) + 1000
    cache = B.PagedCache(pages, page, hkv, D, bits=4)
    ids = np.array([[pages - 1, 3]], np.int32)
    X = to_dev(ref.bf16_values(rng, L, 2 * D)[0], "bf16")
    t = np.arange(L)
    B.batq_kv_paged_append(cache, X[:, :D], X[:, D:], dev(ids[0].astype(np.int64)[t // page] * page + t % page))
    bits, q = ref.bf16_values(rng, 40, hq * D)
    lens = np.array([L], np.int32)
    at = torch.tensor(ids[0].astype(np.int64), device="cuda")
    small = [a[at].cpu().numpy() for a in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    kv, vv = br.values(*small[:2], 4), br.values(*small[2:], 4)
    codes, scales = o.mxfp4_quantize(X[:, :D].float().cpu().numpy())
    assert np.array_equal(small[0][:, 0].reshape(-1, D // 2)[:L], codes)
    for n in (1, 2, 40):
        cu = np.array([0, n], np.int32)
        got, lse = run_attention(B, cache, to_dev(bits[:n], "bf16"), cu, lens, ids, n, hq)
        ref.assert_attention(got, lse, ref.attention(kv, vv, q[:n].reshape(n, hq, D).astype(np.float64), cu, lens, np.array([[0, 1]]), page, D ** -0.5, True, 0, n))


def test_one_workspace_serves_both_widths_on_streams_and_in_graphs(B):
    """The same bits on another stream and from replays of two graphs, one of each width, that share a workspace, with eager
    work and other lengths in between."""
    import torch
    rng = np.random.default_rng(11)
    hq, hkv, D, page = 8, 2, 128, 16
    calls = []                                              # a cache of each width, with its own queries and page table
    dlens = dev(np.array([5000, 333, 1], np.int32))
    for bits in (4, 8):
        arrays, qbits, _, cu, lens, table, T = br.batch_case(rng, [5000, 333, 1], [1, 1, 1], hq, hkv, D, page, bits)
        calls.append((make_cache(B, arrays, bits), to_dev(qbits, "bf16"), dev(cu), dlens, dev(table), 1, 5000))
    ws = torch.full((B.batq_paged_attention_workspace(calls[0][0], hq, 3, T, 1, 5000),), 0xFF, dtype=torch.uint8, device="cuda")
    want = [B.batq_paged_attention(*c, workspace=ws) for c in calls]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = [B.batq_paged_attention(*c, workspace=ws) for c in calls]
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want)) and not torch.equal(*want)
    outs, graphs = [torch.zeros_like(want[0]) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, oo, c in zip(graphs, outs, calls):
        with torch.cuda.graph(g, stream=side):
            B.batq_paged_attention(*c, out=oo, workspace=ws)
    for rep in range(3):
        dlens.copy_(torch.tensor([5000 - 1000 * rep, 333 - rep, 1], dtype=torch.int32))
        want = [B.batq_paged_attention(*c) for c in calls]
        for oo in outs:
            oo.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), rep
