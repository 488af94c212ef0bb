"""The serving operators around a paged cache that is held in 4 bits and kept to a budget, with a plain form of each.

  append   rotation by position, the block transforms and MXFP4 of new tokens, scattered into the pages
           (batq_kv_paged_append on a 4-bit cache)
  attend   attention of a ragged batch over the 4-bit cache (batq_paged_attention on it)
  score    what each cached token has received of the attention: the softmax weights of a batch's queries, summed over
           queries and the query heads of a key head (batq_kv_paged_score)
  evict    the tokens of each key head with the largest scores, beside the first and the last ones, move to fresh pages
           (batq_kv_paged_evict)

The shapes are the repository's own (an 8B-class decoder with 32 query and 8 key heads of 128 channels; a multimodal
model with 28 query and 4 key heads) or generic.
"""
import math

import numpy as np
import torch

own = False

ROT_BASE = 500000.0
MOST_APPEND = 8192 * 48 * 128              # elements of the largest listed case, likewise below
MOST_SCORES = 32 * 4096 * 16384
MOST_CACHE = 4 * 131072 * 4 * 128
MOST_KEPT = 64 * 2048 * 8 * 128


def listed():
    def append(name, M, hq, hkv, D, page, transform, rot, inter=False, x="bf16", pad=0):
        return {"name": name, "op": "append", "bits": 4, "M": M, "hq": hq, "hkv": hkv, "D": D, "page": page,
                "transform": transform, "rot": rot, "inter": inter, "x": x, "pad": pad}

    def batch(name, op, bits, B, q, kv, hq, hkv, D, page, spread, window=0, **more):
        return {"name": name, "op": op, "bits": bits, "B": B, "q": q, "kv": kv, "hq": hq, "hkv": hkv, "D": D, "page": page,
                "spread": spread, "window": window, **more}

    def evict(name, bits, B, kv, hkv, D, page, spread, budget, first, last):
        return {"name": name, "op": "evict", "bits": bits, "B": B, "kv": kv, "hkv": hkv, "D": D, "page": page,
                "spread": spread, "budget": budget, "first": first, "last": last}

    return [
        # a decode step of one user at a far position, keys and values transformed: launch and latency
        append("append-one", 1, 32, 8, 128, 16, True, 128),
        # a batch of odd prompts in fp32 with a partial, interleaved rotation, small heads, no transforms, unused slots
        append("append-ragged", 777, 28, 4, 64, 32, False, 32, inter=True, x="f32", pad=3),
        # prefill of 8192 tokens, keys, values and queries transformed
        append("append-prefill", 8192, 32, 8, 128, 64, True, 128),
        # attention of a decode step: one user with a context of 8192 tokens
        batch("attend-one", "attend", 4, 1, 1, 8192, 32, 8, 128, 16, 0.0),
        # four very long contexts, seven query heads to a key head: what a cache of 4 bits is for
        batch("attend-long", "attend", 4, 4, 1, 131072, 28, 4, 128, 64, 0.2),
        # chunked prefill beside decoding sequences: query lengths 1 to 500, small heads, a sliding window
        batch("attend-chunk", "attend", 4, 9, 500, 10000, 16, 2, 64, 32, 1.0, window=4096),
        # a chunk of 4096 tokens of a prompt behind 12288 tokens of it
        batch("attend-prefill", "attend", 4, 1, 4096, 16384, 32, 8, 128, 64, 0.0),
        # scores of a decode step of 64 sequences of very different lengths, added to what the tokens have
        batch("score-decode", "score", 4, 64, 1, 8192, 32, 8, 128, 16, 1.0, add=True),
        # what the last 64 queries of four prompts look at, from an 8-bit cache: a prompt's cache is cut down after it
        batch("score-observe", "score", 8, 4, 64, 32768, 28, 4, 128, 64, 0.1, add=False),
        # scores of a whole prompt
        batch("score-prefill", "score", 4, 1, 8192, 8192, 32, 8, 128, 64, 0.0, add=True),
        # a prompt's cache cut down from 32768 to 2048 tokens in each key head
        evict("evict-prompt", 4, 4, 32768, 8, 128, 64, 0.0, 2048, 4, 64),
        # 64 sequences that have grown by a few pages beyond their budget while decoding, in 8 bits
        evict("evict-step", 8, 64, 2112, 8, 128, 16, 0.01, 2048, 4, 256),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "score", "evict"])
    hkv = rng.choice([1, 2, 4, 8])
    D, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    hq = hkv * rng.choice([1, 2, 3, 4, 7, 8])
    if op == "append":
        M = max(1, min(_log(rng, 1, 8192), MOST_APPEND // ((hq + 2 * hkv) * D)))
        return {"op": op, "bits": 4, "M": M, "hq": hq, "hkv": hkv, "D": D, "page": page, "transform": rng.choice([True, False]),
                "rot": rng.choice([0, D // 2, D, D]), "inter": rng.choice([False, False, True]), "x": rng.choice(["bf16", "bf16", "f32"]),
                "pad": rng.choice([0, min(3, M - 1)])}
    spread = rng.choice([0.0, 0.3, 1.0])
    if op == "evict":
        budget = _log(rng, 16, 8192)
        kv = min(131072, max(1, int(budget * math.exp(rng.uniform(-0.3, 3.0)))))
        B = max(1, min(_log(rng, 1, 64), MOST_KEPT // (min(kv, budget) * hkv * D), 8 * MOST_CACHE // (kv * hkv * D)))
        return {"op": op, "bits": rng.choice([4, 4, 8]), "B": B, "kv": kv, "hkv": hkv, "D": D, "page": page, "spread": spread,
                "budget": budget, "first": rng.randint(0, 4), "last": rng.randint(0, budget // 4)}
    B = _log(rng, 1, 64)
    kv = max(1, min(_log(rng, 1, 131072), MOST_CACHE // (B * hkv * D)))
    q = min(kv, rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 4096)]), max(1, MOST_SCORES // (B * hq * kv)))
    case = {"op": op, "bits": 4, "B": B, "q": q, "kv": kv, "hq": hq, "hkv": hkv, "D": D, "page": page, "spread": spread,
            "window": rng.choice([0, 0, 0, max(1, kv // 3)])}
    if op == "score":
        case.update(bits=rng.choice([4, 4, 8]), add=rng.choice([True, False]))
    return case


_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0])


def _factors(rng, width):
    """Global-and-private Kronecker factors near the identity and learned clip ratios."""
    G = (np.eye(4) + 0.05 * rng.standard_normal((4, 4))).astype(np.float32)
    P = (np.eye(8) + 0.05 * rng.standard_normal((width // 32, 8, 8))).astype(np.float32)
    return G, P, rng.uniform(0.85, 1.0, width // 32).astype(np.float32)


def _blocks(G, P):
    return np.stack([np.kron(G.astype(np.float64), p.astype(np.float64)) for p in P])


def _quantise(y, clip, bits):
    """MXFP4 or MXFP8 of y [..., blocks, 32] in fp32: (bytes of the codes [..., blocks, 4 bits], scale bytes [..., blocks])."""
    bound = y.abs().amax(-1)
    if clip is not None:
        bound = bound * clip
    e = (torch.frexp(bound).exponent - (3 if bits == 4 else 9)).clamp(-127, 127)
    e = torch.where(bound > 0, e, -127)
    b = bound.unsqueeze(-1)
    scaled = torch.ldexp(torch.minimum(torch.maximum(y, -b), b), -e.unsqueeze(-1))
    if bits == 8:
        return scaled.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)
    a = scaled.abs()                                        # ties to the code with an even mantissa bit
    code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0)
    code = code + 8 * torch.signbit(y).to(torch.uint8)
    return code[..., 0::2] + 16 * code[..., 1::2], (e + 127).to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    # how a batch is cut into sequences belongs to the case: outputs of another seed have the same shapes
    shape = np.random.default_rng([v for k, v in sorted(case.items()) if isinstance(v, int)])
    s = dict(case)
    hkv, D, page, bits = (case[k] for k in ("hkv", "D", "page", "bits"))
    pair = np.stack([_E2M1[np.arange(256) & 15], _E2M1[np.arange(256) >> 4]], 1)     # a byte's two values
    s["pair"] = torch.from_numpy(pair).float().cuda()

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    def dev(a, dtype=None):
        t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
        return t if dtype is None else t.to(dtype)

    def lengths(n, top):                                    # the first is the largest, the others spread below it
        x = np.maximum(1, np.round(top * np.exp(-case["spread"] * shape.random(n) * math.log(top + 1))).astype(np.int64))
        x[0] = top
        return x

    if case["op"] == "append":
        M, hq, rot = (case[k] for k in ("M", "hq", "rot"))
        # one projection gives all three: q, k and v are column ranges of its output
        X = normal(M, (hq + 2 * hkv) * D)
        X[:, :: 97] *= 8.0                                  # outlier channels
        X = X.to(_DTYPE[case["x"]])
        s["q"], s["k"], s["v"] = X.split((hq * D, hkv * D, hkv * D), 1)
        # runs of tokens continue sequences: consecutive positions, consecutive slots up to the end of a page
        far = 131072
        starts = np.zeros(M, np.int64)
        runs = max(1, M // 300) if M > 64 else M
        cut = np.sort(shape.choice(M, runs, replace=False))
        cut[0] = 0
        starts[cut] = 1
        run = np.cumsum(starts) - 1
        within = np.arange(M) - cut[run]
        s["positions"] = dev((rng.integers(0, far - M, runs)[run] + within).astype(np.int32))
        length = np.diff(np.append(cut, M))
        lead = shape.integers(0, page, runs)                # the run's first offset in its page
        pages = -(-(lead + length) // page)
        first = np.cumsum(pages) - pages
        total = int(pages.sum())
        order = rng.permutation(total)
        at = lead[run] + within
        slots = order[first[run] + at // page] * page + at % page
        if case["pad"]:
            slots[rng.choice(M, case["pad"], replace=False)] = -1
        s["slots"] = dev(slots.astype(np.int64))
        s["codes"] = torch.zeros((2, total, hkv, page, D // 2), dtype=torch.uint8, device="cuda")
        s["k_codes"], s["v_codes"] = s["codes"]
        s["k_scales"], s["v_scales"] = (torch.full((total, hkv, D // 32, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
        # a byte's two values as two bytes of 8-bit floating point, which holds them exactly
        s["pair8"] = s["pair"].to(torch.float8_e4m3fn).view(torch.int16).view(-1)
        s["table"] = None
        if rot:
            freq = ROT_BASE ** (-np.arange(0, rot, 2, dtype=np.float64) / rot)
            angle = torch.arange(far, dtype=torch.float64, device="cuda")[:, None] * dev(freq)[None]
            s["table"] = torch.cat([angle.cos(), angle.sin()], 1).float()      # angles in 64 bits, the table in 32
        s["q_out"] = torch.empty((M, hq * D), dtype=torch.bfloat16, device="cuda")
        if case["transform"]:
            fk, fv = _factors(rng, hkv * D), _factors(rng, hkv * D)
            Tk, Tv = _blocks(*fk[:2]), _blocks(*fv[:2])
            s["T_k"], s["T_v"], s["T_q"] = dev(Tk), dev(Tv), dev(np.linalg.inv(Tk).transpose(0, 2, 1))
            s["clip_k"], s["clip_v"] = dev(fk[2]), dev(fv[2])
        if own:                                             # the handles that a program keeps for its lifetime
            import paper_2603_16590_amd as B
            s["cache"] = B.PagedCache(total, page, hkv, D, tensors=tuple(s[k] for k in ("k_codes", "k_scales", "v_codes", "v_scales")), bits=4)
            s["tk"] = B.Transform(hkv * D, *fk) if case["transform"] else None
            s["tv"] = B.Transform(hkv * D, *fv) if case["transform"] else None
        return s

    # the other operators work on caches of a ragged batch
    nB, kv = case["B"], case["kv"]
    lens = lengths(nB, kv)
    pages = -(-lens // page)
    fresh = -(-np.minimum(lens, case.get("budget", 0)) // page)        # pages that the kept tokens move to
    total = int(pages.sum() + fresh.sum()) + 3
    order = rng.permutation(total)
    table, out_table = np.full((nB, int(pages.max())), -1, np.int32), np.full((nB, max(1, int(fresh.max()))), -1, np.int32)
    written = np.zeros((total,), np.int64)                  # tokens of each page
    first, first_out = np.cumsum(pages) - pages, int(pages.sum()) + np.cumsum(fresh) - fresh
    for b in range(nB):
        mine = order[first[b]: first[b] + pages[b]]
        table[b, : pages[b]] = mine
        written[mine] = np.minimum(page, lens[b] - page * np.arange(pages[b]))
        out_table[b, : fresh[b]] = order[first_out[b]: first_out[b] + fresh[b]]
    unwritten = (torch.arange(page, device="cuda")[None] >= dev(written)[:, None])[:, None, :, None]
    for name in ("k", "v"):
        x = normal(total, hkv, page, D).to(torch.bfloat16)
        x[..., 5] *= 6.0                                    # an outlier channel of each head
        codes, scales = _quantise(x.float().view(total, hkv, page, D // 32, 32), None, bits)
        # places that no token has been written to hold whatever was there: here NaN
        s[name + "_codes"] = torch.where(unwritten, 0x7F, codes.view(total, hkv, page, -1))
        s[name + "_scales"] = torch.where(unwritten, 255, scales).transpose(2, 3).contiguous()
        del x, codes, scales
    s["kv_len"], s["page_table"], s["max_kv"] = dev(lens.astype(np.int32)), dev(table), int(lens.max())
    if own:
        import paper_2603_16590_amd as B
        s["cache"] = B.PagedCache(total, page, hkv, D, tensors=tuple(s[k] for k in ("k_codes", "k_scales", "v_codes", "v_scales")), bits=bits)

    if case["op"] == "evict":
        # sums of weights: few tokens have much, many next to nothing, some exactly the same
        score = (3.0 * normal(total, hkv, page) - 4.0).exp()
        s["score"] = torch.where(score < 1e-3, 0.0, score)
        s["out_table"] = dev(out_table)
        s["keep"] = torch.empty((nB, hkv, case["budget"]), dtype=torch.int32, device="cuda")
        s["new_len"] = torch.empty((nB,), dtype=torch.int32, device="cuda")
        if own:
            s["ws"] = torch.empty(max(16, B.batq_kv_paged_evict_workspace(s["cache"], nB, s["max_kv"], case["budget"])),
                                  dtype=torch.uint8, device="cuda")
        return s

    q, hq = case["q"], case["hq"]
    qs = np.minimum(lens, lengths(nB, q))
    qs[0] = min(q, kv)
    cu = np.concatenate([[0], np.cumsum(qs)])
    T = int(cu[-1])
    s["queries"] = normal(T, hq * D).to(torch.bfloat16)
    s["cu_q"], s["max_q"] = dev(cu.astype(np.int32)), int(qs.max())
    s["lse"] = torch.empty((T, hq), dtype=torch.float32, device="cuda")
    s["seq"] = dev(np.repeat(np.arange(nB), qs))            # the plain form's gather indices
    s["within"] = dev(np.arange(T) - np.repeat(cu[:-1], qs))
    s["rows"] = torch.minimum(dev(cu[:-1])[:, None] + torch.arange(s["max_q"], device="cuda")[None], dev(cu[1:])[:, None] - 1)
    if case["op"] == "attend":
        s["out"] = torch.empty_like(s["queries"])
    else:
        s["lse"].copy_(_of_rows(s, torch.logsumexp(_scores(s), -1)))          # what the attention before it has returned
        s["score"] = normal(total, hkv, page).abs()
    if own:
        size = B.batq_paged_attention_workspace if case["op"] == "attend" else B.batq_kv_paged_score_workspace
        s["ws"] = torch.empty(max(16, size(s["cache"], hq, nB, T, s["max_q"], s["max_kv"])), dtype=torch.uint8, device="cuda")
    return s


def _rotate(x, cos, sin, rot, inter):
    """x [M, heads, D] with its first `rot` channels rotated in pairs (j, j + rot/2), or (2j, 2j + 1)."""
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if inter else (x[..., : rot // 2], x[..., rot // 2: rot])
    cos, sin = cos[:, None], sin[:, None]
    a2, b2 = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a2, b2], -1).flatten(-2) if inter else torch.cat([a2, b2], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _by_blocks(x, T):
    """x [M, width] times the block-diagonal T [width / 32, 32, 32], in fp32."""
    return torch.matmul(x.reshape(x.shape[0], -1, 32).transpose(0, 1).contiguous(), T.float()).transpose(0, 1).reshape(x.shape[0], -1)


def _appended(s):
    """What an append leaves, as the numbers that it stands for: E2M1 codes, E8M0 scales."""
    codes = s["pair8"][s["codes"].int()].view(torch.float8_e4m3fn)
    return {"q": s["q_out"], "codes": codes, "k_scales": s["k_scales"].view(torch.float8_e8m0fnu), "v_scales": s["v_scales"].view(torch.float8_e8m0fnu)}


def _append(s):
    M, hq, hkv, D, page, rot = (s[k] for k in ("M", "hq", "hkv", "D", "page", "rot"))
    q, k, v = s["q"].float().view(M, hq, D), s["k"].float().view(M, hkv, D), s["v"].float()
    if rot:
        cos, sin = s["table"][s["positions"].long()].split(rot // 2, 1)
        q, k = _rotate(q, cos, sin, rot, s["inter"]), _rotate(k, cos, sin, rot, s["inter"])
    clip_k = clip_v = None
    if s["transform"]:
        of_head = torch.arange(hq, device="cuda") // (hq // hkv)
        q = _by_blocks(q.reshape(M, -1), s["T_q"].view(hkv, D // 32, 32, 32)[of_head].flatten(0, 1))
        k, v = _by_blocks(k.reshape(M, -1), s["T_k"]), _by_blocks(v, s["T_v"])
        clip_k, clip_v = s["clip_k"].view(hkv, -1), s["clip_v"].view(hkv, -1)
    s["q_out"].copy_(q.reshape(M, -1))
    # an unused slot is written where the last one goes that is used, with the same bytes
    live = torch.where(s["slots"] >= 0, torch.arange(M, device="cuda"), -1).amax()
    tok = torch.where(s["slots"] >= 0, torch.arange(M, device="cuda"), live)
    slot = s["slots"][tok]
    for x, clip, name in ((k, clip_k, "k"), (v, clip_v, "v")):
        codes, scales = _quantise(x.reshape(M, hkv, D // 32, 32), clip, 4)
        s[name + "_codes"][slot // page, :, slot % page] = codes.view(M, hkv, D // 2)[tok]
        s[name + "_scales"][slot // page, :, :, slot % page] = scales[tok]
    return _appended(s)


def _values(s, codes):
    """Bytes of codes as the values they stand for, in fp32."""
    return codes.view(torch.float8_e4m3fn).float() if s["bits"] == 8 else s["pair"][codes.int()].flatten(-2)


def _context(s, name, mask):
    """The batch's keys or values as fp32 [B, kv heads, length, D]; zeros where `mask` [B, length] is not set."""
    nB, page, hkv, D = s["B"], s["page"], s["hkv"], s["D"]
    pt = s["page_table"].clamp_min(0).long()
    codes = _values(s, s[name + "_codes"][pt])                                      # [B, pages, heads, page, D]
    scale = torch.exp2(s[name + "_scales"][pt].float() - 127.0).transpose(3, 4)     # [B, pages, heads, page, D / 32]
    x = codes.view(nB, -1, hkv, page, D // 32, 32) * scale.unsqueeze(-1)
    x = x.permute(0, 2, 1, 3, 4, 5).reshape(nB, hkv, -1, D)
    return torch.where(mask[:, None, :, None], x, 0.0)


def _scores(s):
    """q k / sqrt(D) of every query and token, -infinity where a query does not look: [B, kv heads, group, queries, length]."""
    nB, hq, hkv, D, Q = s["B"], s["hq"], s["hkv"], s["D"], s["max_q"]
    t = torch.arange(s["page_table"].shape[1] * s["page"], device="cuda")
    mask = t[None] < s["kv_len"][:, None]
    qs = s["cu_q"][1:] - s["cu_q"][:-1]
    pos = (s["kv_len"] - qs)[:, None] + torch.arange(Q, device="cuda")[None]        # [B, Q]
    seen = mask[:, None, :] & (t[None, None] <= pos[..., None])
    if s["window"]:
        seen = seen & (t[None, None] > pos[..., None] - s["window"])
    q = s["queries"][s["rows"]].float().view(nB, Q, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(nB, hkv, -1, D)
    S = torch.matmul(q * (1.0 / math.sqrt(D)), _context(s, "k", mask).transpose(2, 3))
    return S.view(nB, hkv, hq // hkv, Q, -1).masked_fill_(~seen[:, None, None], -math.inf)


def _of_rows(s, x):
    """x [B, kv heads, group, queries, ...] as rows of the batch: [rows, query heads * ...]."""
    return x[s["seq"], :, :, s["within"]].reshape(len(s["seq"]), -1)


def _attend(s):
    mask = torch.arange(s["page_table"].shape[1] * s["page"], device="cuda")[None] < s["kv_len"][:, None]
    S = _scores(s)
    m = S.amax(-1, keepdim=True).clamp_min(-3e38)
    S = S.sub_(m).exp_()
    total = S.sum(-1, keepdim=True)
    O = torch.matmul(S.view(s["B"], s["hkv"], -1, S.shape[-1]), _context(s, "v", mask)).view(*S.shape[:4], s["D"]) / total
    s["out"].copy_(_of_rows(s, O))
    s["lse"].copy_(_of_rows(s, (m + total.log()).squeeze(-1)))
    return {"out": s["out"], "lse": s["lse"]}


def _score(s):
    page, L = s["page"], s["page_table"].shape[1] * s["page"]
    S = _scores(s)
    lse = s["lse"][s["rows"]].view(s["B"], s["max_q"], s["hkv"], -1).permute(0, 2, 3, 1)       # [B, kv heads, group, queries]
    S = S.sub_(lse.unsqueeze(-1)).exp_()
    qs = s["cu_q"][1:] - s["cu_q"][:-1]
    S = S.masked_fill_((torch.arange(s["max_q"], device="cuda")[None] >= qs[:, None])[:, None, None, :, None], 0.0)
    mass = S.sum((2, 3)).transpose(1, 2)                    # [B, length, kv heads]
    t = torch.arange(L, device="cuda")[None].expand(s["B"], -1)
    t = torch.where(t < s["kv_len"][:, None], t, 0)         # places without a token: the first one's, again
    mass = torch.gather(mass, 1, t.unsqueeze(-1).expand_as(mass))
    at = torch.gather(s["page_table"].long(), 1, t // page)
    if s["add"]:                                            # the queries' own tokens are new
        old = (t < (s["kv_len"] - qs)[:, None]).unsqueeze(-1)
        mass = mass + torch.where(old, s["score"][at, :, t % page], 0.0)
    s["score"][at, :, t % page] = mass
    return s["score"]


def _evict(s):
    page, n, first, last = (s[k] for k in ("page", "budget", "first", "last"))
    L = max(s["page_table"].shape[1] * page, n)
    t = torch.arange(L, device="cuda")
    lens = s["kv_len"].long()
    table = torch.nn.functional.pad(s["page_table"].clamp_min(0), (0, max(0, -(-n // page) - s["page_table"].shape[1]))).long()
    key = s["score"][table].transpose(1, 2).flatten(2)[..., :L]                     # [B, kv heads, length]
    always = (t[None] < first) | (t[None] >= lens[:, None] - last)
    key = torch.where(always[:, None], math.inf, key)
    key = torch.where((t[None] < lens[:, None])[:, None], key, -math.inf)
    order = torch.sort(key, dim=-1, descending=True, stable=True).indices[..., :n]      # ties: the lowest index first
    count = lens.clamp_max(n)
    live = (torch.arange(n, device="cuda")[None] < count[:, None])[:, None].expand_as(order)
    kept = torch.sort(torch.where(live, order, L), -1).values
    s["keep"].copy_(torch.where(live, kept, -1))
    s["new_len"].copy_(count)
    # places behind the last kept token: the first one's, again
    src = torch.where(live, kept, kept[..., :1])
    dst = torch.where(live, torch.arange(n, device="cuda"), 0)
    b, h = torch.arange(s["B"], device="cuda")[:, None, None], torch.arange(s["hkv"], device="cuda")[None, :, None]
    sp, dp = table[b, src // page], s["out_table"].clamp_min(0).long()[b, dst // page]
    for name in ("k_codes", "v_codes", "score"):
        s[name][dp, h, dst % page] = s[name][sp, h, src % page]
    for name in ("k_scales", "v_scales"):
        s[name][dp, h, :, dst % page] = s[name][sp, h, :, src % page]
    return _moved(s)


def _moved(s):
    """What an eviction leaves.  The codes are moved as they are: their bytes, two values of 4 bits or one of 8 each."""
    return {k: s[k] for k in ("keep", "new_len", "score", "k_codes", "k_scales", "v_codes", "v_scales")}


def run(s):
    if not own:
        return {"append": _append, "attend": _attend, "score": _score, "evict": _evict}[s["op"]](s)
    import paper_2603_16590_amd as B
    if s["op"] == "append":
        B.batq_kv_paged_append(s["cache"], s["k"], s["v"], s["slots"], positions=s["positions"], q=s["q"], q_out=s["q_out"],
                               rope=s["table"], interleaved=s["inter"], tk=s["tk"], tv=s["tv"])
        return _appended(s)
    if s["op"] == "attend":
        B.batq_paged_attention(s["cache"], s["queries"], s["cu_q"], s["kv_len"], s["page_table"], s["max_q"], s["max_kv"],
                               window=s["window"], out=s["out"], lse=s["lse"], workspace=s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    if s["op"] == "score":
        return B.batq_kv_paged_score(s["cache"], s["queries"], s["lse"], s["score"], s["cu_q"], s["kv_len"], s["page_table"],
                                     s["max_q"], s["max_kv"], window=s["window"], add=s["add"], workspace=s["ws"])
    B.batq_kv_paged_evict(s["cache"], s["score"], s["kv_len"], s["page_table"], s["out_table"], s["max_kv"], s["budget"],
                          first=s["first"], last=s["last"], keep=s["keep"], new_len=s["new_len"], workspace=s["ws"])
    return _moved(s)


def _mean(top, spread):                                     # of top * exp(-spread * u * log(top + 1)), u uniform
    a = spread * math.log(top + 1)
    return top * (1.0 if a == 0 else (1.0 - math.exp(-a)) / a)


def _lengths(case):
    """Expected sums over a batch: (tokens of the caches that some query sees, query tokens, visible pairs of a query token and
    a key, tokens of the caches)."""
    B, q, kv, spread, window = case["B"], case["q"], case["kv"], case["spread"], case["window"] or case["kv"]
    all_kv, T = kv + (B - 1) * _mean(kv, spread), q + (B - 1) * _mean(q, spread)

    def pairs(n, length):                                   # the last n queries of `length` tokens
        return n * min(window, max(1.0, length - (n - 1) / 2.0))

    seen = pairs(min(q, kv), kv) + (B - 1) * pairs(_mean(q, spread), _mean(kv, spread))
    reach = min(kv, window + q) + (B - 1) * min(_mean(kv, spread), window + _mean(q, spread))
    return min(all_kv, reach), T, seen, all_kv


def work(case):
    hkv, D = case["hkv"], case["D"]
    token = D * (case["bits"] / 8 + 1 / 32)                 # bytes of a token's keys, or values, in a head
    if case["op"] == "append":
        M, hq, rot = (case[k] for k in ("M", "hq", "rot"))
        size = {"bf16": 2, "f32": 4}[case["x"]]
        per = (hq + 2 * hkv) * D * size + hq * D * 2 + 2 * hkv * token + rot * 4 + 12
        # a block's Kronecker product takes 12 multiply-adds per element, a rotation 3 operations
        return {"bytes": M * per, "flops": M * D * (24.0 * (hq + 2 * hkv) * case["transform"] + 3.0 * (hq + hkv))}
    if case["op"] == "evict":
        B, kv, n = case["B"], case["kv"], case["budget"]
        tokens = kv + (B - 1) * _mean(kv, case["spread"])
        kept = min(n, kv) + (B - 1) * min(n, _mean(kv, case["spread"]))
        # every score once, a kept token's bytes in and out, the list of the kept ones
        return {"bytes": hkv * (4 * tokens + kept * (4 * token + 8)), "flops": hkv * tokens}
    hq = case["hq"]
    L, T, seen, tokens = _lengths(case)
    if case["op"] == "attend":
        return {"bytes": L * hkv * 2 * token + T * hq * (4 * D + 4), "flops": 4.0 * seen * hq * D}
    return {"bytes": L * hkv * token + tokens * hkv * (8 if case["add"] else 4) + T * hq * (2 * D + 4), "flops": 2.0 * seen * hq * D}


def _exact_append(s):
    M, hq, hkv, D, page, rot = (s[k] for k in ("M", "hq", "hkv", "D", "page", "rot"))
    q, k, v = (s[n].cpu().double().numpy().reshape(M, -1, D) for n in ("q", "k", "v"))
    if rot:
        row = s["table"].cpu().double().numpy()[s["positions"].cpu().numpy()]
        turn = row[:, : rot // 2] + 1j * row[:, rot // 2:]
        first, second = (slice(0, rot, 2), slice(1, rot, 2)) if s["inter"] else (slice(0, rot // 2), slice(rot // 2, rot))
        for x in (q, k):
            z = (x[..., first] + 1j * x[..., second]) * turn[:, None]
            x[..., first], x[..., second] = z.real, z.imag
    if s["transform"]:
        # a code next to the border between two roundings has no value that 32 bits can be held to: queries alone
        Tq = s["T_q"].cpu().numpy().reshape(hkv, D // 32, 32, 32).repeat(hq // hkv, 0)
        q = np.einsum("mhbi,hbij->mhbj", q.reshape(M, hq, D // 32, 32), Tq)
        return {"q": q.reshape(M, -1), "codes": None, "k_scales": None, "v_scales": None}
    slots = s["slots"].cpu().numpy()
    used, pages = slots >= 0, s["codes"].shape[1]
    codes, out = np.zeros((2, pages, hkv, page, D)), {"q": q.reshape(M, -1)}
    for i, x in enumerate((k, v)):
        scales = np.ones((pages, hkv, D // 32, page))
        x = x.reshape(M, hkv, D // 32, 32)
        top = np.abs(x).max(-1, keepdims=True)
        e = np.where(top > 0, np.clip(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 2, -127, 127), -127)
        y = x * 2.0 ** -e
        step = 2.0 ** (np.clip(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -30))), 0, 2) - 1)
        y = np.clip(np.rint(y / step) * step, -6, 6)        # (rint: ties to even)
        codes[i, slots[used] // page, :, slots[used] % page] = y.reshape(M, hkv, D)[used]
        scales[slots[used] // page, :, :, slots[used] % page] = 2.0 ** e[used][..., 0]
        out["kv"[i] + "_scales"] = scales
    out["codes"] = codes
    return out


def _exact_batch(s):
    hq, hkv, D, page = (s[k] for k in ("hq", "hkv", "D", "page"))
    cu, lens = s["cu_q"].tolist(), s["kv_len"].tolist()
    e2m1 = torch.from_numpy(_E2M1).cuda()
    attend = s["op"] == "attend"
    out = torch.zeros(s["queries"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    score = None if attend else s["score"].double()
    for b, L in enumerate(lens):
        pages = s["page_table"][b, : -(-L // page)].long()
        n = cu[b + 1] - cu[b]
        at = torch.arange(L - n, L, device="cuda")[:, None]
        t = torch.arange(L, device="cuda")
        hidden = (t > at) | (t <= at - s["window"]) if s["window"] else t > at
        for h in range(hkv):
            kv = []
            for name in ("k", "v")[: 2 if attend else 1]:
                codes = s[name + "_codes"][pages, h]
                if s["bits"] == 4:
                    codes = e2m1[torch.stack([codes & 15, codes >> 4], -1).long()].reshape(-1, D)[:L]
                else:
                    codes = codes.reshape(-1, D)[:L].view(torch.float8_e4m3fn).double()
                scale = s[name + "_scales"][pages, h].transpose(1, 2).reshape(-1, D // 32)[:L].double()
                kv.append(codes * (2.0 ** (scale - 127)).repeat_interleave(32, 1))
            mass = 0.0
            for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                S = s["queries"][cu[b]: cu[b + 1], g * D: (g + 1) * D].double() @ kv[0].t() / math.sqrt(D)
                S.masked_fill_(hidden, -math.inf)
                if attend:
                    lse[cu[b]: cu[b + 1], g] = torch.logsumexp(S, 1)
                    out[cu[b]: cu[b + 1], g * D: (g + 1) * D] = torch.softmax(S, 1) @ kv[1]
                else:
                    mass = mass + (S - s["lse"][cu[b]: cu[b + 1], g, None].double()).exp().sum(0)
            if not attend:
                had = score[pages[t // page], h, t % page] if s["add"] else torch.zeros_like(mass)
                score[pages[t // page], h, t % page] = mass + torch.where(t < L - n, had, 0.0)
    return {"out": out.cpu().numpy(), "lse": lse.cpu().numpy()} if attend else score.cpu().numpy()


def _exact_evict(s):
    page, n = s["page"], s["budget"]
    got = {k: s[k].cpu().numpy() for k in ("score", "k_codes", "k_scales", "v_codes", "v_scales")}
    table, fresh = s["page_table"].cpu().numpy(), s["out_table"].cpu().numpy()
    keep, new_len = np.full((s["B"], s["hkv"], n), -1, np.int32), np.zeros(s["B"], np.int32)
    old = {k: v.copy() for k, v in got.items()}
    for b, L in enumerate(s["kv_len"].tolist()):
        t = np.arange(L)
        new_len[b] = m = min(L, n)
        for h in range(s["hkv"]):
            key = old["score"][table[b, t // page], h, t % page].astype(np.float64)
            key[(t < s["first"]) | (t >= L - s["last"])] = np.inf
            kept = np.sort(np.argsort(-key, kind="stable")[:m])
            keep[b, h, :m] = kept
            src, dst = (table[b, kept // page], kept % page), (fresh[b, t[:m] // page], t[:m] % page)
            for k in ("score", "k_codes", "v_codes"):
                got[k][dst[0], h, dst[1]] = old[k][src[0], h, src[1]]
            for k in ("k_scales", "v_scales"):
                got[k][dst[0], h, :, dst[1]] = old[k][src[0], h, :, src[1]]
    return {"keep": keep, "new_len": new_len, **got}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_batch, "score": _exact_batch, "evict": _exact_evict}[s["op"]](s)
