"""The paged 8-bit cache: batq_kv_paged_append (rotation, transforms, MXFP8, scatter) and batq_paged_attention
against plain 64-bit statements, separately and together as a serving step uses them."""
import numpy as np
import pytest

import batq_inputs as bi
from oracle import batq_oracle as o
from gpu_util import require_gpu, to_dev, y_to_f32
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


def make_cache(B, rng, pages, page, heads, D):
    arrays = ref.random_cache(rng, pages, page, heads, D) + ref.random_cache(rng, pages, page, heads, D)
    return arrays, B.PagedCache(pages, page, heads, D, tensors=[dev(a) for a in arrays])


def host(cache):
    return [t.cpu().numpy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


APPEND = [
    # M, q heads, kv heads, D, page, rot, interleaved, dtype
    (1, 4, 4, 64, 16, 64, False, "bf16"),
    (1, 32, 8, 128, 16, 128, False, "bf16"),
    (31, 7, 1, 128, 32, 64, True, "f32"),
    (33, 0, 3, 64, 256, 16, False, "f32"),
    (33, 6, 2, 128, 64, 48, False, "bf16"),
    (65, 8, 2, 64, 16, 32, True, "bf16"),
    (200, 28, 4, 128, 16, 0, False, "bf16"),
    (311, 12, 3, 64, 128, 64, False, "f32"),
]


def append_case(rng, M, hq, hkv, D, page, rot, dtype):
    """(X storage, q, k, v as fp32 [M, heads, D], positions, slots, pages): slots scattered, some unused."""
    X = rng.standard_normal((M, (hq + 2 * hkv) * D + 8)).astype(np.float32)
    X[:, ::37] *= 30.0
    X[M // 2, :64] = 0.0                                    # zero blocks
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


@pytest.mark.parametrize("M,hq,hkv,D,page,rot,inter,dtype", APPEND)
def test_append_without_transforms_is_bit_exact(B, M, hq, hkv, D, page, rot, inter, dtype):
    import torch
    rng = np.random.default_rng(M + hq + D + rot)
    (q, k, v), (qd, kd, vd), positions, slots, pages = append_case(rng, M, hq, hkv, D, page, rot, dtype)
    arrays, cache = make_cache(B, rng, pages, page, hkv, D)
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
        ref.scatter(want[n], want[n + 1], used, page, hkv, D, *o.mxfp8_quantize(x.reshape(M, -1)))
    for got, w, old, name in zip(host(cache), want, arrays, ("k codes", "k scales", "v codes", "v scales")):
        assert np.array_equal(got, w), name
    if hq:
        got = y_to_f32(q_out)
        assert np.array_equal(got[~left_out, : hq * D], o.bf16_round(q.reshape(M, -1))[~left_out])
        assert np.all(got[left_out] == 7.0) and np.all(got[:, hq * D:] == 7.0)


def _transforms(B, rng, hkv, D, form, clip=True):
    width = hkv * D
    G = (np.eye(4) + 0.05 * rng.standard_normal((4, 4))).astype(np.float32)
    P = (np.eye(8) + 0.05 * rng.standard_normal((width // 32, 8, 8))).astype(np.float32)
    c = rng.uniform(0.85, 1.0, width // 32).astype(np.float32) if clip else None
    T = o.kron_blocks(G, P)
    if form == "kron":
        return B.Transform(width, G, P, c), T, c
    return B.Transform.general(width, dense=T.astype(np.float32), clip=c), T.astype(np.float32).astype(np.float64), c


@pytest.mark.parametrize("M,hq,hkv,D,page,rot,inter,dtype", [c for c in APPEND if c[0] > 1])
@pytest.mark.parametrize("form", ["kron", "dense"])
def test_append_with_transforms(B, M, hq, hkv, D, page, rot, inter, dtype, form):
    """Codes against the 64-bit transform: an element may sit on the other side of a rounding border only if the
    exact value is within the transform's accuracy (2^-20 sum |x| |T|) of it."""
    import torch
    rng = np.random.default_rng(M + hq + D + rot + 1)
    (q, k, v), (qd, kd, vd), positions, slots, pages = append_case(rng, M, hq, hkv, D, page, rot, dtype)
    arrays, cache = make_cache(B, rng, pages, page, hkv, D)
    tk, Tk, ck = _transforms(B, rng, hkv, D, form)
    tv, Tv, cv = _transforms(B, rng, hkv, D, form)
    table = ref.rope_table(1000, rot) if rot else None
    q_out = B.batq_kv_paged_append(cache, kd, vd, dev(slots), positions=dev(positions) if rot else None, q=qd if hq else None,
                                   rope=dev(table) if rot else None, interleaved=inter, tk=tk, tv=tv)
    torch.cuda.synchronize()
    left_out = ((positions < 0) | (positions >= 1000)) if rot else np.zeros(M, bool)
    if rot:
        at = np.where(left_out, 0, positions)
        q, k = ref.rotate(q, table, at, rot, inter), ref.rotate(k, table, at, rot, inter)
    live = ~left_out & (slots >= 0) & (slots < pages * page)
    got = host(cache)
    for n, x, T, c in ((0, k, Tk, ck), (2, v, Tv, cv)):
        x = x.reshape(M, -1).astype(np.float64)
        y, absy = o.apply_blocks(x, T), o.apply_blocks(np.abs(x), np.abs(T))
        want_c, want_s = o.mxfp8_quantize(y.astype(np.float32), c)
        gc = got[n][slots[live] // page, :, slots[live] % page].reshape(live.sum(), -1)
        gs = got[n + 1][slots[live] // page, :, :, slots[live] % page].reshape(live.sum(), -1)
        assert np.mean(gc != want_c[live]) <= 1e-3 and np.mean(gs != want_s[live]) <= 1e-3
        val = o.dequantize_fp8(gc, gs)
        y, absy = y[live], absy[live]
        lim = np.repeat(np.abs(y).reshape(len(y), -1, 32).max(-1) * c, 32, 1)
        unit = np.repeat(np.exp2(gs.astype(np.float64) - 127), 32, 1)
        clipped = np.clip(np.clip(y, -lim, lim), -448 * unit, 448 * unit)
        step = np.maximum(np.exp2(np.floor(np.log2(np.maximum(np.abs(clipped), 1e-300))) - 3), unit * 2.0 ** -9)
        assert np.all(np.abs(val - clipped) <= step / 2 + 2.0 ** -19 * np.repeat(absy.reshape(len(y), -1, 32).max(-1), 32, 1))
        # nothing else was touched
        mask = np.ones(got[n].shape, bool)
        mask[slots[live] // page, :, slots[live] % page] = False
        assert np.array_equal(got[n][mask], arrays[n][mask])
    if hq:
        Tq = np.repeat(o.inverse_transpose_blocks(Tk).reshape(hkv, -1, 32, 32), hq // hkv, 0).reshape(-1, 32, 32)
        x = q.reshape(M, -1).astype(np.float64)
        y, absy = o.apply_blocks(x, Tq), o.apply_blocks(np.abs(x), np.abs(Tq))
        d = np.abs(y_to_f32(q_out).astype(np.float64) - y)
        assert np.all((d <= 2.0 ** -8 * np.abs(y) + 2.0 ** -19 * absy)[~left_out])


@pytest.mark.parametrize("kind", ["kron", "minmax", "clip only"])
def test_append_without_rotation_writes_the_bytes_of_batq_kv_append(B, kind):
    """One sequence in page order: the rows of the paged cache hold what the row-window cache holds, byte for byte."""
    import torch
    rng = np.random.default_rng(5)
    M, hkv, D, page = 150, 2, 128, 32
    width = hkv * D
    bits, _ = ref.bf16_values(rng, M, width)
    X = to_dev(bits, "bf16")
    if kind == "kron":
        t, _, _ = _transforms(B, rng, hkv, D, "kron")
    elif kind == "clip only":
        t = B.Transform(width, None, None, rng.uniform(0.7, 1.0, width // 32).astype(np.float32))
    else:
        lo, hi = (rng.uniform(0.7, 1.0, width // 32).astype(np.float32) for _ in range(2))
        t = B.Transform.general(width, outer=np.eye(4, dtype=np.float32) * 1.25,
                                inner=(np.eye(8) + 0.05 * rng.standard_normal((width // 32, 8, 8))), clip_min=lo, clip_max=hi)
    cache = B.PagedCache(-(-M // page), page, hkv, D)
    for lo, hi in ((0, 1), (1, 40), (40, M)):               # in pieces of any size
        B.batq_kv_paged_append(cache, X[lo:hi], X[lo:hi], torch.arange(lo, hi, device="cuda"), tk=t, tv=t)
    codes = torch.zeros(B.batq_code8_bytes(M, width), dtype=torch.uint8, device="cuda")
    scales = torch.zeros(B.batq_scale_bytes(M, width), dtype=torch.uint8, device="cuda")
    B.batq_kv_append(t, X, codes, scales, 0, M, bits=8)
    rc, rs = B.batq_codes8_to_rowmajor(codes, M, width), B.batq_scales_to_rowmajor(scales, M, width)
    torch.cuda.synchronize()
    for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
        assert torch.equal(c.permute(0, 2, 1, 3).reshape(-1, width)[:M], rc)
        assert torch.equal(s.permute(0, 3, 1, 2).reshape(-1, width // 32)[:M], rs)


def test_append_token_by_token_equals_one_call(B):
    import torch
    rng = np.random.default_rng(8)
    M, hq, hkv, D, page = 70, 4, 2, 128, 16
    X = to_dev(ref.bf16_values(rng, M, (hq + 2 * hkv) * D)[0], "bf16")
    q, k, v = X.split((hq * D, hkv * D, hkv * D), 1)
    tk, _, _ = _transforms(B, rng, hkv, D, "kron")
    table, slots = dev(ref.rope_table(4000, D)), torch.randperm(6 * page, device="cuda")[:M]
    pos = torch.arange(M, device="cuda", dtype=torch.int32) + 3900
    a, b = B.PagedCache(6, page, hkv, D), B.PagedCache(6, page, hkv, D)
    qa = B.batq_kv_paged_append(a, k, v, slots, pos, q=q, rope=table, tk=tk)
    qb = torch.zeros_like(qa)
    for m in range(M):
        B.batq_kv_paged_append(b, k[m:m + 1], v[m:m + 1], slots[m:m + 1], pos[m:m + 1], q=q[m:m + 1], q_out=qb[m:m + 1],
                               rope=table, tk=tk)
    torch.cuda.synchronize()
    assert torch.equal(qa, qb)
    for x, y in zip(host(a), host(b)):
        assert np.array_equal(x, y)


@pytest.mark.parametrize("dtype,D,rot,inter", [("bf16", 128, 128, False), ("bf16", 64, 48, False), ("f32", 128, 64, True), ("f32", 64, 32, False)])
def test_append_of_many_tokens_equals_pieces(B, dtype, D, rot, inter):
    """A long call and its pieces (other kernels, other tiles) leave the same bytes and the same queries."""
    import torch
    rng = np.random.default_rng(13)
    M, hq, hkv, page = 2100, 6, 3, 64
    X = torch.randn((M, (hq + 2 * hkv) * D), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, k, v = X.split((hq * D, hkv * D, hkv * D), 1)
    tk, _, _ = _transforms(B, rng, hkv, D, "kron")
    tv, _, _ = _transforms(B, rng, hkv, D, "dense")
    table, slots = dev(ref.rope_table(4000, rot)), torch.randperm(40 * page, device="cuda")[:M]
    slots[5], slots[1000] = -1, 10 ** 12
    pos = torch.randint(0, 4000, (M,), device="cuda", dtype=torch.int32)
    pos[7], pos[2000] = -1, 4000
    for t in ((tk, tv), (None, None)):
        a, b = B.PagedCache(40, page, hkv, D), B.PagedCache(40, page, hkv, D)
        qa = torch.full((M, hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
        qb = qa.clone()
        B.batq_kv_paged_append(a, k, v, slots, pos, q=q, q_out=qa, rope=table, interleaved=inter, tk=t[0], tv=t[1])
        for lo in range(0, M, 111):
            s = slice(lo, min(M, lo + 111))
            B.batq_kv_paged_append(b, k[s], v[s], slots[s], pos[s], q=q[s], q_out=qb[s], rope=table, interleaved=inter, tk=t[0], tv=t[1])
        torch.cuda.synchronize()
        assert torch.equal(qa, qb) and bool((qa[7] == 7.0).all()) and bool((qa[2000] == 7.0).all())
        for x, y in zip(host(a), host(b)):
            assert np.array_equal(x, y)


# Calls past 16 D units of 32 tokens x 32 channels, whose rotations the kernel for many tokens takes: every layout of it (head
# width, element size), pair distance and direction; 15 heads leave a wave of the last workgroup without one, and 141 tiles of
# 32 tokens are two for some workgroups, the last one ragged.
MANY = [
    # D, rot, interleaved, dtype
    (64, 64, False, "bf16"), (64, 64, False, "f32"), (64, 32, True, "f32"), (64, 16, True, "bf16"), (64, 0, False, "bf16"), (64, 0, False, "f32"),
    (128, 64, False, "bf16"), (128, 64, False, "f32"), (128, 128, False, "bf16"), (128, 128, False, "f32"), (128, 128, True, "bf16"),
    (128, 48, True, "f32"), (128, 0, False, "bf16"), (128, 0, False, "f32"),
]
MANY_M, MANY_HQ, MANY_HKV = 4489, 9, 3


def many_tokens(D, rot, inter):
    """Whether the kernel for many tokens takes the call."""
    return -(-MANY_M // 32) * (MANY_HQ + 2 * MANY_HKV) * (D // 32) > 16 * D and (rot % 64 == 0 or inter)


@pytest.mark.parametrize("D,rot,inter,dtype", MANY)
def test_append_of_many_tokens_is_bit_exact(B, D, rot, inter, dtype):
    assert many_tokens(D, rot, inter)
    test_append_without_transforms_is_bit_exact(B, MANY_M, MANY_HQ, MANY_HKV, D, 64, rot, inter, dtype)


@pytest.mark.parametrize("D,rot,inter,dtype,form", [(64, 64, False, "bf16", "kron"), (64, 32, True, "f32", "dense"), (64, 0, False, "f32", "kron"), (64, 0, False, "bf16", "dense"),
                                                    (128, 64, False, "bf16", "dense"), (128, 128, False, "f32", "kron"), (128, 128, True, "bf16", "kron"), (128, 0, False, "bf16", "kron")])
def test_append_of_many_tokens_with_transforms(B, D, rot, inter, dtype, form):
    assert many_tokens(D, rot, inter)
    test_append_with_transforms(B, MANY_M, MANY_HQ, MANY_HKV, D, 32, rot, inter, dtype, form)


def other_transforms(B, rng, width):
    """Clipping alone, and the two-ratio form (minimum and maximum of a block) with dense blocks."""
    lo, hi = (rng.uniform(0.7, 1.0, width // 32).astype(np.float32) for _ in range(2))
    blocks = (np.eye(32) + 0.03 * rng.standard_normal((width // 32, 32, 32))).astype(np.float32)
    return B.Transform(width, None, None, rng.uniform(0.7, 1.0, width // 32).astype(np.float32)), B.Transform.general(width, dense=blocks, clip_min=lo, clip_max=hi)


@pytest.mark.parametrize("D,rot,inter,dtype", MANY)
def test_append_of_many_tokens_equals_short_calls(B, D, rot, inter, dtype):
    """Calls of 96 tokens go to the kernel for few: the same bytes and queries, with one clip ratio for the keys and two for the values,
    and the other way round."""
    import torch
    assert many_tokens(D, rot, inter)
    rng = np.random.default_rng(D + rot)
    M, hq, hkv, page = MANY_M, MANY_HQ, MANY_HKV, 128
    X = torch.randn((M, (hq + 2 * hkv) * D), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, k, v = X.split((hq * D, hkv * D, hkv * D), 1)
    clip, minmax = other_transforms(B, rng, hkv * D)
    table = dev(ref.rope_table(4000, rot)) if rot else None
    slots, pos = torch.randperm(40 * page, device="cuda")[:M], torch.randint(0, 4000, (M,), device="cuda", dtype=torch.int32)
    slots[[9, M - 1]], slots[4000] = -1, 40 * page
    if rot:
        pos[33], pos[M - 2] = -5, 4000
    for tk, tv in ((clip, minmax), (minmax, clip)):
        a, b = B.PagedCache(40, page, hkv, D), B.PagedCache(40, page, hkv, D)
        qa = torch.full((M, hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
        qb = qa.clone()
        B.batq_kv_paged_append(a, k, v, slots, pos, q=q, q_out=qa, rope=table, interleaved=inter, tk=tk, tv=tv)
        for lo in range(0, M, 96):
            s = slice(lo, min(M, lo + 96))
            B.batq_kv_paged_append(b, k[s], v[s], slots[s], pos[s], q=q[s], q_out=qb[s], rope=table, interleaved=inter, tk=tk, tv=tv)
        torch.cuda.synchronize()
        assert torch.equal(qa, qb)
        for x, y in zip(host(a), host(b)):
            assert np.array_equal(x, y)


@pytest.mark.parametrize("D,dtype", [(64, "bf16"), (64, "f32"), (128, "bf16")])
def test_append_of_many_tokens_writes_the_bytes_of_batq_kv_append(B, D, dtype):
    """Without rotation, one sequence in page order: what the row-window cache holds, with each kind of clipping.  Transformed fp32
    rows are summed in another order there: 32 products in fp32 are within 32 x 2^-24 of S = sum |x| |T|.  The columns of |T| and
    |T^-1| add up to less than 3 here and clip ratios are at least 0.7, so S < 9 max |y| < 16 b for a block's bound b < 2^9 units
    (2^scale): the two sums of an element are less than 2 x 2^-19 x 16 x 2^9 = 2^-5 units apart, and what they are rounded to a step more."""
    import torch
    rng = np.random.default_rng(23)
    M, hkv, page = 10240 if D == 64 else 4700, 4, 16
    width = hkv * D
    assert -(-M // 32) * 2 * hkv * (D // 32) > 16 * D
    X = torch.randn((M, width), device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32)

    def values(codes, scales):
        return codes.view(torch.float8_e4m3fn).double().view(M, -1, 32) * torch.exp2(scales.double() - 127).unsqueeze(-1)

    for n, t in enumerate(other_transforms(B, rng, width) + (_transforms(B, rng, hkv, D, "kron")[0],)):
        cache = B.PagedCache(-(-M // page), page, hkv, D)
        B.batq_kv_paged_append(cache, X, X, torch.arange(M, device="cuda"), tk=t, tv=t)
        codes = torch.zeros(B.batq_code8_bytes(M, width), dtype=torch.uint8, device="cuda")
        scales = torch.zeros(B.batq_scale_bytes(M, width), dtype=torch.uint8, device="cuda")
        B.batq_kv_append(t, X, codes, scales, 0, M, bits=8)
        rc, rs = B.batq_codes8_to_rowmajor(codes, M, width), B.batq_scales_to_rowmajor(scales, M, width)
        torch.cuda.synchronize()
        for c, s in ((cache.k_codes, cache.k_scales), (cache.v_codes, cache.v_scales)):
            c, s = c.permute(0, 2, 1, 3).reshape(-1, width)[:M], s.permute(0, 3, 1, 2).reshape(-1, width // 32)[:M]
            if dtype == "bf16" or n == 0:                   # (the first one has no blocks)
                assert torch.equal(c, rc) and torch.equal(s, rs)
                continue
            a, b, unit = values(c, s), values(rc, rs), torch.exp2(torch.maximum(s, rs).double() - 127).unsqueeze(-1)
            step = torch.clamp(torch.exp2(torch.floor(torch.log2(torch.maximum(a.abs(), b.abs()).clamp_min(1e-300))) - 3), min=unit * 2.0 ** -9)
            assert bool(((a - b).abs() <= step + unit * 2.0 ** -5).all())


# ---------------------------------------------------------------------------------------- attention
def attend_case(rng, B, lens, qs, hq, hkv, D, page, spare=0):
    lens, qs = np.array(lens), np.array(qs)
    per = -(-lens // page)
    pages = int(per.sum()) + 2
    arrays, cache = make_cache(B, rng, pages, page, hkv, D)
    order = rng.permutation(pages)
    table = np.full((len(lens), max(1, int(per.max()))), -7, np.int32)
    filled = np.zeros(pages, np.int64)
    at = 0
    for b in range(len(lens)):
        mine = order[at: at + per[b]]
        at += per[b]
        table[b, : per[b]] = mine
        filled[mine] = np.minimum(page, lens[b] - page * np.arange(per[b]))
    # what no token was written to holds NaN codes and NaN scales
    empty = np.arange(page)[None] >= filled[:, None]
    for n in (0, 2):
        arrays[n][np.broadcast_to(empty[:, None, :, None], arrays[n].shape)] = 0x7F
        arrays[n + 1][np.broadcast_to(empty[:, None, None, :], arrays[n + 1].shape)] = 255
    cache = B.PagedCache(pages, page, hkv, D, tensors=[dev(a) for a in arrays])
    cu = np.concatenate([[0], np.cumsum(qs)]).astype(np.int32)
    T = int(cu[-1]) + spare
    bits, q = ref.bf16_values(rng, T, hq * D)
    with np.errstate(invalid="ignore"):
        kv, vv = ref.cache_values(arrays[0], arrays[1]), ref.cache_values(arrays[2], arrays[3])
    return cache, (kv, vv), to_dev(bits, "bf16"), q.reshape(T, hq, D).astype(np.float64), cu, lens.astype(np.int32), table, T


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
    ([1000], [1], 16, 1, 128, 128, 64),
    ([333], [333], 3, 3, 64, 32, 0),
    ([290], [290], 8, 1, 128, 16, 0),
    ([130, 64, 257, 1], [130, 1, 100, 1], 14, 2, 128, 64, 0),
    ([200, 140], [70, 140], 4, 4, 128, 32, 1),
    ([500], [129], 2, 1, 64, 16, 100),
    ([300, 20], [10, 20], 32, 1, 64, 16, 0),
    ([77], [40], 40, 1, 128, 16, 0),
    ([5, 9], [9, 20], 4, 2, 64, 16, 0),                     # more queries than tokens: the first ones see nothing
]


@pytest.mark.parametrize("lens,qs,hq,hkv,D,page,window", ATTEND)
@pytest.mark.parametrize("causal", [True, False])
def test_attention(B, lens, qs, hq, hkv, D, page, window, causal):
    rng = np.random.default_rng(sum(lens) + sum(qs) + hq)
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page, spare=3)
    got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, causal=causal, window=window)
    want = ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, causal, window, T)
    ref.assert_attention(got, lse, want)


def test_attention_of_long_sequences(B):
    """Long enough for every way of cutting a sequence into parts: one against the reference, and each against a
    batch of which it is a part."""
    import torch
    rng = np.random.default_rng(3)
    hq, hkv, D, page = 8, 2, 128, 64
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [20000, 9, 7001, 1, 15000], [1, 1, 4, 1, 2], hq, hkv, D, page)
    got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq)
    ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, 0, T))
    for b in range(5):
        one = np.array([0, cu[b + 1] - cu[b]], np.int32)
        alone, _ = run_attention(B, cache, qd[cu[b]: cu[b + 1]], one, lens[b: b + 1], table[b: b + 1], int(one[1]), hq)
        ref.assert_attention(alone, None, tuple(x[cu[b]: cu[b + 1]] for x in ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, 0, T)))


def test_attention_of_a_long_chunk(B):
    """A prompt's later chunk: many queries over a long context, next to decoding sequences."""
    rng = np.random.default_rng(4)
    hq, hkv, D, page = 4, 1, 64, 16
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [3000, 1500, 2500], [70, 1, 300], hq, hkv, D, page)
    for window in (0, 700):
        got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, window=window)
        ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, window, T))


def test_attention_does_not_trust_its_lists(B):
    """Pages outside the cache, lengths past the table or max_kv, rows outside q: none of it takes part."""
    rng = np.random.default_rng(6)
    hq, hkv, D, page = 4, 2, 128, 16
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [100, 40, 64, 90], [1, 3, 20, 1], hq, hkv, D, page, spare=2)
    table[0, 2], table[2, 0], table[2, 3], table[1, 0] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1
    table[3, :] = -1                                        # a sequence without any page
    got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, max_kv=128)
    ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, 0, T))
    # lengths: past the table's width, negative
    longer = lens.copy()
    longer[0], longer[1] = 10 ** 9, -5
    eff = np.array([table.shape[1] * page, 0, 64, 90])
    got, lse = run_attention(B, cache, qd, cu, longer, table, T, hq, max_kv=10 ** 6)
    full = np.nan_to_num(kv), np.nan_to_num(vv)
    t2 = table.copy()
    t2[0] = np.where((table[0] >= 0), table[0], -1)
    want = ref.attention(*full, q, cu, eff, t2, page, D ** -0.5, True, 0, T)
    rows = slice(int(cu[1]), int(cu[4]))                    # (sequence 0 now reads places that nothing was written to)
    ref.assert_attention(got[rows], lse[rows], tuple(x[rows] for x in want))
    # row lists: a decreasing one and one past the end leave their rows alone
    for broken in ([0, 1, 4, 24, 10 ** 6], [0, 1, 4, 24, 3], [0, -1, 4, 24, 25]):
        broken = np.array(broken, np.int32)
        import torch
        out = torch.full((T, hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
        B.batq_paged_attention(cache, qd, dev(broken), dev(lens), dev(table), 20, 128, out=out)
        torch.cuda.synchronize()
        got = y_to_f32(out).astype(np.float64).reshape(T, hq, D)
        assert np.all(got[25:] == 7.0)
        sel = slice(4, 24)
        ref.assert_attention(got[sel], None, tuple(x[sel] for x in ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, 0, T)))


@pytest.mark.parametrize("max_q,max_kv", [(1, 64), (3, 50), (64, 0)])
def test_attention_bounds_cut_a_sequence(B, max_q, max_kv):
    import torch
    rng = np.random.default_rng(7)
    hq, hkv, D, page = 4, 2, 64, 16
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [64, 50], [5, 6], hq, hkv, D, page)
    out = torch.full((T, hq * D), 7.0, dtype=torch.bfloat16, device="cuda")
    B.batq_paged_attention(cache, qd, dev(cu), dev(lens), dev(table), max_q, max_kv, out=out)
    torch.cuda.synchronize()
    got = y_to_f32(out).astype(np.float64).reshape(T, hq, D)
    want = ref.attention(np.nan_to_num(kv), np.nan_to_num(vv), q, cu, np.minimum(lens, max_kv), table, page, D ** -0.5, True, 0, T)
    for b in range(2):
        n = min(max_q, int(cu[b + 1] - cu[b]))
        sel = slice(int(cu[b]), int(cu[b]) + n)
        ref.assert_attention(got[sel], None, tuple(x[sel] for x in want))
        assert np.all(got[int(cu[b]) + n: int(cu[b + 1])] == 7.0)


def test_attention_with_extreme_scores(B):
    """One key that carries everything, scores of +-1000, equal keys, and a scale of its own."""
    import torch
    rng = np.random.default_rng(9)
    hq, hkv, D, page = 2, 1, 64, 16
    for n, qn in ((200, 1), (200, 100)):
        cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [n], [qn], hq, hkv, D, page)
        kc, ks = cache.k_codes.cpu().numpy(), cache.k_scales.cpu().numpy()
        ks[...] = np.where(ks == 255, 255, ks + 6)
        kc[table[0, 3], 0, 5] = 0x38
        ks[table[0, 3], 0, :, 5] = 133
        cache = B.PagedCache(cache.num_pages, page, hkv, D, tensors=[dev(kc), dev(ks), cache.v_codes, cache.v_scales])
        with np.errstate(invalid="ignore"):
            kv = ref.cache_values(kc, ks)
        for scale in (D ** -0.5, 1.0, 1e-3):
            got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, scale=scale)
            ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, scale, True, 0, T))


def test_attention_past_four_gigabytes(B):
    """Offsets into the code arrays beyond 32 bits: two pages at either end of a pool of 4.3 GB per array."""
    import torch
    rng = np.random.default_rng(10)
    hq, hkv, D, page = 4, 1, 128, 256
    pages = (1 << 32) // (page * D) + 2000
    cache = B.PagedCache(pages, page, hkv, D)
    L = 300
    ids = np.array([[pages - 1, 3]], np.int32)
    X = to_dev(ref.bf16_values(rng, L, 2 * D)[0], "bf16")
    t = np.arange(L)
    slots = ids[0].astype(np.int64)[t // page] * page + t % page
    B.batq_kv_paged_append(cache, X[:, :D], X[:, D:], dev(slots))
    bits, q = ref.bf16_values(rng, 2, hq * D)
    lens, cu = np.array([L], np.int32), np.array([0, 2], np.int32)
    got, lse = run_attention(B, cache, to_dev(bits, "bf16"), cu, lens, ids, 2, hq)
    small = [a[torch.tensor(ids[0].astype(np.int64), device="cuda")].cpu().numpy() for a in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    kv, vv = ref.cache_values(small[0], small[1]), ref.cache_values(small[2], small[3])
    x = X[:, :D].float().cpu().numpy()
    # the keys are there: half a step of 3 mantissa bits is |x| / 16; of a block whose maximum is a = (1.75 .. 2) 2^f the
    # elements above 448 2^(f - 8) = 1.75 2^f saturate, which takes at most (2 - 1.75) / 2 = 1 / 8 of them; the smallest
    # step of a block with a < 8 is 2^(2 - 8 - 9)
    assert bool(np.all(np.abs(kv[:, 0].reshape(-1, D)[:L] - x) <= np.abs(x) / 8 + 2.0 ** -15))
    ref.assert_attention(got, lse, ref.attention(kv, vv, q.reshape(2, hq, D).astype(np.float64), cu, lens, np.array([[0, 1]]), page, D ** -0.5, True, 0, 2))


def test_attention_is_repeatable_and_runs_on_a_side_stream_and_in_graphs(B):
    """Same bits on another stream and from replays of two graphs that share one workspace, with eager work and a
    moved cache state in between (lengths live on the device)."""
    import torch
    rng = np.random.default_rng(11)
    hq, hkv, D, page = 8, 2, 128, 16
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [5000, 333, 1], [1, 1, 1], hq, hkv, D, page)
    dcu, dlens, dtable = dev(cu), dev(lens), dev(table)
    n = B.batq_paged_attention_workspace(cache, hq, 3, T, 1, 5000)
    ws = torch.full((max(n, 16),), 0xFF, dtype=torch.uint8, device="cuda")
    args = (dcu, dlens, dtable, 1, 5000)
    want = B.batq_paged_attention(cache, qd, *args, workspace=ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        o2 = B.batq_paged_attention(cache, qd, *args, workspace=ws)
    side.synchronize()
    assert torch.equal(o2, want)
    outs, graphs = [torch.zeros_like(want) for _ in range(2)], [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, oo in zip(graphs, outs):
        with torch.cuda.graph(g, stream=side):
            B.batq_paged_attention(cache, qd, *args, out=oo, workspace=ws)
    for rep in range(3):
        dlens.copy_(torch.tensor([5000 - 1000 * rep, 333 - rep, 1], dtype=torch.int32))
        want = B.batq_paged_attention(cache, qd, *args)
        junk = torch.randn(300, 300, device="cuda") @ torch.randn(300, 300, device="cuda")
        for oo in outs:
            oo.zero_()
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(oo, want) for oo in outs), rep
        assert bool(torch.isfinite(junk).all())


def test_attention_of_a_large_ragged_batch(B):
    """More sequences than a wave has lanes: chunks and single tokens in any order, empty ones among them."""
    rng = np.random.default_rng(14)
    hq, hkv, D, page = 6, 2, 64, 16
    n = 150
    lens = rng.integers(0, 90, n)
    qs = np.where(rng.random(n) < 0.2, rng.integers(0, 60, n), 1)
    qs[[0, 70, 149]] = 0, 120, 95
    lens[[70, 149]] = 300, 95
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page, spare=1)
    for window in (0, 40):
        got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, window=window)
        ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, window, T))


def test_attention_cut_into_parts_with_a_window(B):
    """Windows that start and end inside parts, for single tokens and for chunks of long sequences."""
    rng = np.random.default_rng(15)
    for hq, hkv, D, page, lens, qs in ((4, 1, 128, 16, [5000, 900], [1, 2]), (2, 1, 64, 64, [4000], [200])):
        cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
        for window in (1, 255, 1000, 3777):
            got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, window=window)
            ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, window, T))


def test_pages_behind_a_window_may_be_gone(B):
    """A server frees pages that no query sees any more: their table entries may be anything, and reused pages may hold
    another sequence's tokens or none."""
    rng = np.random.default_rng(16)
    hq, hkv, D, page, window = 4, 2, 128, 16, 50
    for qn in (1, 3, 70):
        L = 500
        cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, [L, 33], [qn, 1], hq, hkv, D, page)
        first = max(0, L - qn - window + 1) // page          # pages before this one are seen by nobody
        want = ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, window, T)
        for filler in (-1, 2 ** 30, int(table[1, 2])):       # gone, nonsense, a page with unwritten places
            broken = table.copy()
            broken[0, :first] = filler
            got, lse = run_attention(B, cache, qd, cu, lens, broken, T, hq, window=window)
            ref.assert_attention(got, lse, want)


@pytest.mark.parametrize("D", [64, 128])
def test_values_that_are_not_finite(B, D):
    """NaN codes where some rows look and others do not: in a causal prompt, short drafts and windows; a key of NaN makes the
    rows that see it NaN, a value its channel of them, nothing else changes."""
    rng = np.random.default_rng(18 + D)
    page = 16
    for hq, hkv, lens, qs, window, causal in ((2, 1, [200, 90], [200, 3], 0, True), (4, 4, [333], [333], 40, True), (12, 2, [150, 700], [2, 5], 0, True),
                                              (8, 2, [300], [4], 6, True), (4, 1, [64, 1000], [1, 120], 100, True), (3, 1, [129], [100], 60, False),
                                              (6, 2, [77, 500], [1, 2], 0, False)):
        cache, _, qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
        arrays = host(cache)
        for what, count in ((2, 5), (2, 1), (0, 1)):        # values, one value, one key
            a = [x.copy() for x in arrays]
            for _ in range(count):
                b = int(rng.integers(len(lens)))
                tok = int(lens[b]) - 1 - int(rng.integers(0, min(int(lens[b]), qs[b] + 4)))
                a[what][table[b, tok // page], rng.integers(hkv), tok % page, rng.integers(D)] = rng.choice([0x7F, 0xFF])
            broken = B.PagedCache(cache.num_pages, page, hkv, D, tensors=[dev(x) for x in a])
            with np.errstate(invalid="ignore"):
                kv, vv = ref.cache_values(a[0], a[1]), ref.cache_values(a[2], a[3])
                want = ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, causal, window, T)
            got, lse = run_attention(B, broken, qd, cu, lens, table, T, hq, window=window, causal=causal)
            assert np.array_equal(np.isnan(got), np.isnan(want[0]))
            assert np.array_equal(np.isnan(lse), np.isnan(want[1]))
            clean = [np.where(np.isnan(want[0]), 0.0, x) for x in (want[0], want[2])]
            smax, seen = np.where(np.isnan(want[3]), 0.0, want[3]), np.where(np.isnan(want[1]), 0.0, want[1])
            ref.assert_attention(np.where(np.isnan(got), 0.0, got), np.where(np.isnan(lse), 0.0, lse), (clean[0], seen, clean[1], smax))


def test_windows_without_causal_and_of_any_size(B):
    """A window without causal ends nowhere above: rows of long sequences see more than a window; windows up to the largest
    number beside sequences with more queries than tokens; fewer queries served than there are."""
    rng = np.random.default_rng(19)
    hq, hkv, D, page = 4, 2, 64, 16
    cases = (([3000], [2500], 20, False, None), ([2100, 900], [1, 2], 7, False, None), ([40, 9], [60, 12], 2 ** 31 - 1, True, None),
             ([2600], [2600], 30, False, 5), ([2600, 30], [1300, 1], 30, False, 3), ([2600, 30], [1300, 1], 30, True, 1), ([1500], [1400], 2 ** 31 - 1, False, 300))
    for lens, qs, window, causal, max_q in cases:
        cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
        got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, window=window, causal=causal, max_q=max_q)
        want = ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, causal, window, T)
        if max_q:
            rest = np.concatenate([np.arange(cu[b] + min(max_q, cu[b + 1] - cu[b]), cu[b + 1]) for b in range(len(lens))])
            assert np.all(got[rest] == 7.0) and np.all(lse[rest] == 7.0)
            want[1][rest] = np.nan
        ref.assert_attention(got, lse, want)


def test_two_attentions_at_once(B):
    """Calls on two streams with a workspace each do not meet."""
    import torch
    rng = np.random.default_rng(17)
    hq, hkv, D, page = 8, 2, 128, 16
    cases = [attend_case(rng, B, lens, qs, hq, hkv, D, page) for lens, qs in (([3000, 10], [1, 1]), ([2500], [60]), ([64] * 20, [1] * 20))]
    args = [(c[0], c[2], dev(c[4]), dev(c[5]), dev(c[6]), int(np.diff(c[4]).max()), int(c[5].max())) for c in cases]
    want = [B.batq_paged_attention(*a) for a in args]
    ws = [torch.empty(max(16, B.batq_paged_attention_workspace(a[0], hq, a[3].shape[0], a[1].shape[0], a[5], a[6])), dtype=torch.uint8, device="cuda") for a in args]
    streams = [torch.cuda.Stream() for _ in args]
    torch.cuda.synchronize()
    for rep in range(3):
        outs = [torch.zeros_like(w) for w in want]
        torch.cuda.synchronize()
        for _ in range(4):
            for a, w, o_, s in zip(args, ws, outs, streams):
                with torch.cuda.stream(s):
                    B.batq_paged_attention(*a, out=o_, workspace=w)
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(outs, want)), rep


def weights_rounded_once(kv, vv, q, cu, lens, table, page, scale, rows):
    """What attention of these rows (b, i) would give if its weights lost their second bf16 term: [row, head, channel] in 64 bits."""
    hkv, D = kv.shape[1], kv.shape[3]
    hq, out = q.shape[1], []
    for b, i in rows:
        t = np.arange(lens[b] - (cu[b + 1] - cu[b]) + i + 1)
        ids = table[b][t // page]
        for h in range(hq):
            s = kv[ids, h * hkv // hq, t % page] @ q[cu[b] + i, h] * scale
            p = np.exp(s - s.max())
            out.append(o.bf16_round(p.astype(np.float32)).astype(np.float64) @ vv[ids, h * hkv // hq, t % page] / p.sum())
    return np.array(out).reshape(len(rows), hq, D)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("hq,hkv,lens,qs", [(8, 2, [64, 63, 40, 5], [1] * 4), (8, 2, [70, 64], [3, 4]), (8, 2, [50, 64], [8, 5]), (6, 2, [60, 33, 400], [1, 2, 60]),
                                            (8, 1, [3000, 61], [1, 1]), (16, 1, [64, 900], [1, 40])])
def test_weights_of_few_rows_have_two_terms(B, D, hq, hkv, lens, qs):
    """Sequences of few rows multiply their weights as two bf16 terms.  The bound for that is only tight where the sum nearly cancels
    (else the rounding of the output hides the second term) and scores are small, so the scale is; among the channels of contexts of
    up to 70 tokens there are enough of those: the same sums with weights rounded once are outside it."""
    rng = np.random.default_rng(24 + D + hq + sum(lens))
    page, scale = 16, D ** -0.5 / 16
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
    got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, scale=scale)
    want = ref.attention(kv, vv, q, cu, lens, table, page, scale, True, 0, T)
    group = hq // hkv
    most = 32 if max(qs) * group <= 32 else 16              # beside a sequence of more than 32 rows only those of up to 16
    rows = [(b, i) for b in range(len(qs)) if qs[b] * group <= most for i in range(qs[b])]
    assert rows
    sel = np.array([cu[b] + i for b, i in rows])
    picked = tuple(x[sel] for x in want)
    ref.assert_attention(got[sel], lse[sel], picked, terms=2)
    if max(lens[b] for b, _ in rows) <= 70:
        with pytest.raises(AssertionError):
            ref.assert_attention(weights_rounded_once(kv, vv, q, cu, lens, table, page, scale, rows), None, picked, terms=2)


@pytest.mark.parametrize("lens,qs,hq,hkv,D,page,window", [c for c in ATTEND if max(c[1]) * (c[2] // c[3]) <= 32])
@pytest.mark.parametrize("causal", [True, False])
def test_attention_of_few_rows_to_two_terms(B, lens, qs, hq, hkv, D, page, window, causal):
    rng = np.random.default_rng(25 + sum(lens) + hq)
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
    got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, causal=causal, window=window)
    ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, causal, window, T), terms=2)


def test_workspace_of_long_contexts_stays_in_bounds(B):
    """Partial results are a tradeoff of a few blocks of tokens against writing them: never more than 2^20 rows x parts of a call's
    sequences of many rows, and 32 rows x a part for 1024 tokens (at least four to a compute unit) of those of few."""
    for D, hq, hkv in ((128, 32, 8), (64, 16, 2), (128, 128, 1)):
        cache = B.PagedCache(2, 16, hkv, D)
        for max_kv in (8192, 131072, 1 << 20, 1 << 24):
            few = 32 * (max(hkv * max_kv // 1024, 5 * 256) + 2 * hkv)
            assert B.batq_paged_attention_workspace(cache, hq, 1, 8192, 8192, max_kv) <= ((1 << 20) + few) * (D + 2) * 4


@pytest.mark.parametrize("D", [64, 128])
def test_scale_byte_255_is_nan(B, D):
    """E8M0 255 is NaN whatever the block's codes are: a key makes the rows that see it NaN, a value its block of 32 channels;
    where nobody looks it does nothing."""
    rng = np.random.default_rng(22 + D)
    page = 16
    for hq, hkv, lens, qs, window in ((4, 2, [200, 90], [1, 1], 0), (4, 2, [200], [200], 50), (6, 2, [300, 70], [3, 2], 0), (2, 1, [1000], [130], 0)):
        cache, _, qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
        arrays = host(cache)
        for what in (1, 3):
            a = [x.copy() for x in arrays]
            for tok in (int(lens[0]) - 1, int(lens[0]) - 1 - min(60, qs[0])):
                a[what][table[0, tok // page], hkv - 1, D // 32 - 1, tok % page] = 255
            broken = B.PagedCache(cache.num_pages, page, hkv, D, tensors=[dev(x) for x in a])
            with np.errstate(invalid="ignore"):
                kv, vv = (np.where(np.repeat(x[1].transpose(0, 1, 3, 2), 32, -1) == 255, np.nan, ref.cache_values(*x)) for x in (a[:2], a[2:]))
                want = ref.attention(kv, vv, q, cu, lens, table, page, D ** -0.5, True, window, T)
            got, lse = run_attention(B, broken, qd, cu, lens, table, T, hq, window=window)
            assert np.isnan(want[0]).any() and not np.isnan(want[0]).all()
            assert np.array_equal(np.isnan(got), np.isnan(want[0])) and np.array_equal(np.isnan(lse), np.isnan(want[1]))


@pytest.mark.parametrize("hq,hkv,lens,qs,window", [(128, 1, [300, 40, 1], [1, 3, 1], 0), (100, 1, [200, 1030], [1, 9], 0), (128, 1, [700], [30], 64),
                                                   (384, 3, [90, 33], [2, 1], 5), (33, 1, [2100], [1], 0)])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_of_many_heads_to_a_key_head(B, hq, hkv, lens, qs, window, D):
    """Groups of 33 to 128 query heads: one token alone is more rows than a tile of the few-row kernel."""
    rng = np.random.default_rng(hq + sum(lens))
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, 32, spare=1)
    got, lse = run_attention(B, cache, qd, cu, lens, table, T, hq, window=window)
    ref.assert_attention(got, lse, ref.attention(kv, vv, q, cu, lens, table, 32, D ** -0.5, True, window, T))


def test_workspace_sizes_grow_with_every_bound(B):
    """A server sizes its workspace once, for its largest batch: no smaller call may ask for more."""
    rng = np.random.default_rng(20)
    for D, hq, hkv in ((128, 32, 8), (128, 28, 4), (64, 16, 2), (64, 1, 1), (128, 128, 1), (64, 24, 24)):
        cache = B.PagedCache(2, 16, hkv, D)
        size = lambda *a: B.batq_paged_attention_workspace(cache, hq, *a)
        assert size(1, 8192, 8192, 8192) >= size(1, 1, 1, 8192) and size(5, 5, 1, 8192) >= size(4, 4, 1, 8192)
        for _ in range(400):
            big = [int(np.exp(rng.uniform(0, np.log(n)))) for n in (200, 8192, 8192, 200000)]
            small = [int(rng.integers(1, n + 1)) if rng.random() < 0.7 else n for n in big]
            assert size(*small) <= size(*big), (small, big)


def test_one_workspace_serves_every_smaller_attention(B):
    """Calls of every kind (a prompt, chunks cut into parts, drafts, single tokens, windows) share the workspace of their bounds."""
    import torch
    rng = np.random.default_rng(21)
    hq, hkv, D, page = 4, 2, 64, 16
    lens, qs = [6000, 2500, 1700, 900, 300], [1, 40, 3, 9, 300]
    cache, (kv, vv), qd, q, cu, lens, table, T = attend_case(rng, B, lens, qs, hq, hkv, D, page)
    ws = torch.full((B.batq_paged_attention_workspace(cache, hq, 5, T, 2500, 8192),), 0xFF, dtype=torch.uint8, device="cuda")
    for rows, window in (([0, 1, 2, 3, 4], 0), ([0], 0), ([1], 0), ([1], 700), ([2, 3], 0), ([0, 3], 100), ([4], 0), ([1, 4], 0)):
        sel = np.concatenate([np.arange(cu[b], cu[b + 1]) for b in rows])
        c = np.concatenate([[0], np.cumsum([cu[b + 1] - cu[b] for b in rows])]).astype(np.int32)
        part = qd[torch.from_numpy(sel).cuda()].contiguous()
        got, lse = run_attention(B, cache, part, c, lens[rows], table[rows], len(sel), hq, window=window, workspace=ws)
        ref.assert_attention(got, lse, ref.attention(kv, vv, q[sel], c, lens[rows], table[rows], page, D ** -0.5, True, window, len(sel)))


def test_binding_refuses_what_does_not_fit(B):
    import torch
    cache = B.PagedCache(4, 16, 2, 64)
    q = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    good = (cache, q, i32(0, 3), i32(5), i32(0, 1).view(1, 2), 3, 5)
    B.batq_paged_attention(*good)
    for k, bad in ((1, q.float()), (1, q[:, ::2]), (2, i32(0, 3).long()), (2, i32(0, 2, 3)), (3, i32(5).cpu()), (4, i32(0, 1)), (1, q.cpu())):
        with pytest.raises(ValueError):
            B.batq_paged_attention(*good[:k], bad, *good[k + 1:])
    with pytest.raises(B.BatqError):
        B.batq_paged_attention(*good, workspace=torch.empty(100, dtype=torch.uint8, device="cuda")[1:])   # alignment
    long = (cache, q, i32(0, 3), i32(5), i32(0, 1).view(1, 2), 3, 100000)
    with pytest.raises(B.BatqError):
        B.batq_paged_attention(*long, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    k = torch.zeros((2, 128), dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros(2, dtype=torch.int64, device="cuda")
    B.batq_kv_paged_append(cache, k, k, slots)
    for bad in (dict(k=k.cpu()), dict(v=k[:1]), dict(slots=slots.int()), dict(rope=torch.zeros((4, 64), device="cuda")),
                dict(q=k[:1]), dict(v=k.float())):
        with pytest.raises(ValueError):
            B.batq_kv_paged_append(**{**dict(cache=cache, k=k, v=k, slots=slots), **bad})
    with pytest.raises(B.BatqError):
        B.batq_kv_paged_append(cache, k, k, slots, tk=B.Transform(64, None, None, None))


# ---------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("transforms", [False, True])
def test_a_serving_step_end_to_end(B, transforms):
    """Fused projection (W4A8) with adapters, append, attention, the way back through T_v^-1: two sequences are
    prefilled and then decoded in a captured step that is replayed at moving positions (they live on the device)."""
    import torch
    rng = np.random.default_rng(12)
    K, hq, hkv, D, page = 256, 4, 2, 64, 16
    N = (hq + 2 * hkv) * D
    w = bi.make_small(8, K, N, seed=2, dtype="bf16")
    t = B.Transform(K, w.G, w.P, w.clip)
    wh = B.batq_prepare_weight(t, to_dev(w.W, "bf16"))
    A = to_dev(ref.bf16_values(rng, 2, 8, K, scale=K ** -0.5)[0], "bf16")
    Bm = to_dev(ref.bf16_values(rng, 2, N, 8, scale=8 ** -0.5)[0], "bf16")
    tk = tv = to = None
    if transforms:
        tk, tv = _transforms(B, rng, hkv, D, "kron", clip=False)[0], None
        G = (np.eye(4) + 0.05 * rng.standard_normal((4, 4))).astype(np.float32)
        P = (np.eye(8) + 0.05 * rng.standard_normal((hkv, D // 32, 8, 8))).astype(np.float32)
        tv = B.Transform(hkv * D, G, P.reshape(-1, 8, 8), None)
        to = B.Transform(hq * D, G, np.repeat(P, hq // hkv, 0).reshape(-1, 8, 8), None)
    cache = B.PagedCache(12, page, hkv, D)
    rope = dev(ref.rope_table(200, D))
    order = rng.permutation(12)
    table = np.stack([order[:6], order[6:]]).astype(np.int32)
    dtable = dev(table)
    lens0, steps = np.array([37, 20]), 14
    tokens = to_dev(ref.bf16_values(rng, 2, 80, K)[0], "bf16")       # inputs of both sequences

    def slots_of(b, p):
        return table[b][p // page].astype(np.int64) * page + p % page

    def layer(X, index, slots, pos, cu, lens, max_q, out=None, work=None):
        Y = B.batq_linear_a8w4(t, wh, X, torch.bfloat16)
        Y = B.batq_lora_add(X, A, Bm, index, Y, out=Y)
        q, k, v = Y.split((hq * D, hkv * D, hkv * D), 1)
        qr = B.batq_kv_paged_append(cache, k, v, slots, pos, q=q, rope=rope, tk=tk, tv=tv)
        oo = B.batq_paged_attention(cache, qr, cu, lens, dtable, max_q, 96, out=out)
        return Y, (oo if to is None else B.batq_transform_apply(to, oo, B.APPLY_INVERSE))

    # what the cache should stand for, kept on the side in fp32 from the same projection outputs
    kept = [[], []]

    def check(Y, out, rows):
        Yf, got = y_to_f32(Y), y_to_f32(out).astype(np.float64).reshape(len(rows), hq, D)
        tab = ref.rope_table(200, D)
        for r, (b, p) in enumerate(rows):
            q, k, v = np.split(Yf[r], [hq * D, (hq + hkv) * D])
            kept[b].append((ref.rotate(k.reshape(1, hkv, D), tab, [p], D, False)[0], v.reshape(hkv, D)))
        for r, (b, p) in enumerate(rows):
            q = ref.rotate(Yf[r, : hq * D].reshape(1, hq, D), tab, [p], D, False)[0].astype(np.float64)
            kk = np.stack([x for x, _ in kept[b][: p + 1]]).astype(np.float64)
            vv = np.stack([x for _, x in kept[b][: p + 1]]).astype(np.float64)
            for h in range(hq):
                s = kk[:, h // 2] @ q[h] / np.sqrt(D)
                pr = np.exp(s - s.max())
                pr /= pr.sum()
                want = pr @ vv[:, h // 2]
                # keys and values carry 4 significant bits (2^-4 of an element, more of small ones in a block): scores
                # move by about 2^-4 |q| |k| / sqrt(D) and outputs with them; a wrong rotation, page or head is off by 1
                bound = 0.35 * np.sqrt((vv[:, h // 2] ** 2).mean())
                assert np.sqrt(((got[r, h] - want) ** 2).mean()) <= bound, (r, b, p, h)

    rows = [(b, p) for b in range(2) for p in range(lens0[b])]
    X = torch.cat([tokens[b, : lens0[b]] for b in range(2)])
    Y, out = layer(X, dev(np.array([b for b, _ in rows], np.int32)), dev(np.array([slots_of(b, p) for b, p in rows])),
                   dev(np.array([p for _, p in rows], np.int32)), dev(np.array([0, lens0[0], lens0.sum()], np.int32)),
                   dev(lens0.astype(np.int32)), int(lens0.max()))
    torch.cuda.synchronize()
    check(Y, out, rows)
    # the decode step, captured once
    sX = torch.zeros((2, K), dtype=torch.bfloat16, device="cuda")
    index, cu = dev(np.array([0, 1], np.int32)), dev(np.array([0, 1, 2], np.int32))
    slots, pos, lens = dev(np.zeros(2, np.int64) - 1), dev(np.zeros(2, np.int32)), dev(np.ones(2, np.int32))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        layer(sX, index, slots, pos, cu, lens, 1)           # first calls outside the capture (slots -1: nothing is written)
    side.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        gY, gout = layer(sX, index, slots, pos, cu, lens, 1)
    for step in range(steps):
        p = lens0 + step
        sX.copy_(torch.stack([tokens[b, int(p[b])] for b in range(2)]))
        slots.copy_(dev(np.array([slots_of(b, p[b]) for b in range(2)])))
        pos.copy_(dev(p.astype(np.int32)))
        lens.copy_(dev((p + 1).astype(np.int32)))
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        check(gY, gout, [(b, int(p[b])) for b in range(2)])
