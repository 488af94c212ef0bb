"""The serving operators around the quantised projections, as measurable cases with a plain form of each.

  append   the new tokens' queries, keys and values between the fused projection and the attention: rotation by
           position, the block transforms of keys, values and queries, MXFP8, and the scatter into the pages of a
           paged cache (batq_kv_paged_append)
  attend   attention of a ragged batch over that cache: one token a sequence, a few, or whole prompts
           (batq_paged_attention)
  lora     the low-rank adapters of many requests on top of a shared projection's output (batq_lora_add)

The shapes are the repository's own (an 8B-class decoder with 32 query and 8 key heads of 128 channels, hidden size
4096 and intermediate size 14336; a multimodal model with hidden size 3584, 28 query and 4 key heads) or generic.
"""
import math

import numpy as np
import torch

own = False

ROT_BASE = 500000.0
MOST_APPEND = 8192 * 48 * 128              # elements of the largest listed case, likewise below
MOST_SCORES = 32 * 8192 * 8192
MOST_CACHE = 4 * 131072 * 4 * 128
MOST_LORA = 4096 * 14336


def listed():
    def append(name, M, hq, hkv, D, page, transform, rot, inter=False, x="bf16", pad=0):
        return {"name": name, "op": "append", "M": M, "hq": hq, "hkv": hkv, "D": D, "page": page, "transform": transform,
                "rot": rot, "inter": inter, "x": x, "pad": pad}

    def attend(name, B, q, kv, hq, hkv, D, page, spread, window=0):
        return {"name": name, "op": "attend", "B": B, "q": q, "kv": kv, "hq": hq, "hkv": hkv, "D": D, "page": page,
                "spread": spread, "window": window}

    def lora(name, M, K, N, r, n, runs, y="bf16"):
        return {"name": name, "op": "lora", "M": M, "K": K, "N": N, "r": r, "n": n, "runs": runs, "y": y}

    return [
        # a decode step of one user at a far position, keys and values transformed: launch and latency
        append("append-one", 1, 32, 8, 128, 16, True, 128),
        # a decode step of 64 sequences without transforms, some slots of the captured batch unused
        append("append-decode", 64, 32, 8, 128, 16, False, 128, pad=5),
        # a batch of odd prompts in fp32 with a partial, interleaved rotation and small heads
        append("append-ragged", 777, 28, 4, 64, 32, False, 32, inter=True, x="f32"),
        # prefill of 8192 tokens, keys, values and queries transformed
        append("append-prefill", 8192, 32, 8, 128, 64, True, 128),
        # attention of a decode step: one user with a context of 8192 tokens
        attend("attend-one", 1, 1, 8192, 32, 8, 128, 16, 0.0),
        # 64 sequences of very different lengths
        attend("attend-decode", 64, 1, 8192, 32, 8, 128, 16, 1.0),
        # four very long contexts, seven query heads to a key head
        attend("attend-long", 4, 1, 131072, 28, 4, 128, 64, 0.2),
        # chunked prefill beside decoding sequences: query lengths 1 to 500, small heads, a sliding window
        attend("attend-chunk", 9, 500, 10000, 16, 2, 64, 32, 1.0, window=4096),
        # a prompt of 8192 tokens
        attend("attend-prefill", 1, 8192, 8192, 32, 8, 128, 64, 0.0),
        # a decode step of 32 requests with 16 adapters beside the query projection
        lora("lora-decode", 32, 4096, 4096, 16, 16, 1),
        # a batch of odd size, an odd rank and an odd width, added in fp32
        lora("lora-ragged", 333, 3616, 5000, 24, 7, 20, y="f32"),
        # prefill of four requests beside the up projection
        lora("lora-prefill", 4096, 4096, 14336, 32, 4, 1024),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attend", "attend", "lora"])
    hkv = rng.choice([1, 2, 4, 8])
    D, page = rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    hq = hkv * rng.choice([1, 2, 3, 4, 7, 8])
    if op == "append":
        M = max(1, min(_log(rng, 1, 8192), MOST_APPEND // ((hq + 2 * hkv) * D)))
        return {"op": op, "M": M, "hq": hq, "hkv": hkv, "D": D, "page": page, "transform": rng.choice([True, False]),
                "rot": rng.choice([0, D // 2, D, D]), "inter": rng.choice([False, False, True]), "x": rng.choice(["bf16", "bf16", "f32"]),
                "pad": rng.choice([0, min(3, M - 1)])}
    if op == "attend":
        B, spread = _log(rng, 1, 64), rng.choice([0.0, 0.3, 1.0])
        kv = max(1, min(_log(rng, 1, 131072), MOST_CACHE // (B * hkv * D)))
        q = min(kv, rng.choice([1, 1, rng.randint(2, 8), _log(rng, 9, 4096)]), max(1, MOST_SCORES // (B * hq * kv)))
        return {"op": op, "B": B, "q": q, "kv": kv, "hq": hq, "hkv": hkv, "D": D, "page": page, "spread": spread,
                "window": rng.choice([0, 0, 0, max(1, kv // 3)])}
    M = _log(rng, 1, 4096)
    K, N = 32 * rng.randint(16, 448), rng.choice([1, 8, 64]) * rng.randint(80, 224)
    return {"op": op, "M": M, "K": K, "N": min(N, MOST_LORA // M), "r": 8 * rng.randint(1, 8), "n": min(M, _log(rng, 1, 32)),
            "runs": _log(rng, 1, max(1, M // 2)), "y": rng.choice(["bf16", "bf16", "f32"])}


_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _factors(rng, width):
    """Global-and-private Kronecker factors near the identity and learned clip ratios."""
    G = (np.eye(4) + 0.05 * rng.standard_normal((4, 4))).astype(np.float32)
    P = (np.eye(8) + 0.05 * rng.standard_normal((width // 32, 8, 8))).astype(np.float32)
    return G, P, rng.uniform(0.85, 1.0, width // 32).astype(np.float32)


def _blocks(G, P):
    return np.stack([np.kron(G.astype(np.float64), p.astype(np.float64)) for p in P])


def _quantise(y, clip):
    """MXFP8 of y [..., blocks, 32] in fp32: (codes as E4M3 numbers, scale bytes [..., blocks])."""
    bound = y.abs().amax(-1)
    if clip is not None:
        bound = bound * clip
    e = (torch.frexp(bound).exponent - 9).clamp(-127, 127)
    e = torch.where(bound > 0, e, -127)
    scaled = torch.ldexp(torch.minimum(torch.maximum(y, -bound.unsqueeze(-1)), bound.unsqueeze(-1)), -e.unsqueeze(-1))
    return scaled.clamp(-448, 448).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    rng = np.random.default_rng(seed)
    # how a batch is cut into sequences belongs to the case: outputs of another seed have the same shapes
    shape = np.random.default_rng([v for k, v in sorted(case.items()) if isinstance(v, int)])
    s = dict(case)

    def normal(*shape):
        return torch.randn(shape, device="cuda", generator=gen)

    def dev(a, dtype=None):
        t = torch.from_numpy(np.ascontiguousarray(a)).cuda()
        return t if dtype is None else t.to(dtype)

    if case["op"] == "append":
        M, hq, hkv, D, page, rot = (case[k] for k in ("M", "hq", "hkv", "D", "page", "rot"))
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
        lead = shape.integers(0, page, runs)                  # the run's first offset in its page
        pages = -(-(lead + length) // page)
        first = np.cumsum(pages) - pages
        total = int(pages.sum())
        order = rng.permutation(total)
        at = lead[run] + within
        slots = order[first[run] + at // page] * page + at % page
        if case["pad"]:
            slots[rng.choice(M, case["pad"], replace=False)] = -1
        s["slots"] = dev(slots.astype(np.int64))
        nb = D // 32
        s["k_codes"], s["v_codes"] = (torch.zeros((total, hkv, page, D), dtype=torch.uint8, device="cuda") for _ in range(2))
        s["k_scales"], s["v_scales"] = (torch.full((total, hkv, nb, page), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
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
            s["cache"] = B.PagedCache(total, page, hkv, D, tensors=tuple(s[k] for k in ("k_codes", "k_scales", "v_codes", "v_scales")))
            s["tk"] = B.Transform(hkv * D, *fk) if case["transform"] else None
            s["tv"] = B.Transform(hkv * D, *fv) if case["transform"] else None
    elif case["op"] == "attend":
        nB, q, kv, hq, hkv, D, page = (case[k] for k in ("B", "q", "kv", "hq", "hkv", "D", "page"))
        # lengths: the first sequence has the largest, the others are spread below it over their logarithm
        lens = np.maximum(1, np.round(kv * np.exp(-case["spread"] * shape.random(nB) * math.log(kv + 1))).astype(np.int64))
        lens[0] = kv
        qs = np.minimum(lens, np.maximum(1, np.round(q * np.exp(-case["spread"] * shape.random(nB) * math.log(q + 1))).astype(np.int64)))
        qs[0] = min(q, kv)
        cu = np.concatenate([[0], np.cumsum(qs)])
        pages = -(-lens // page)
        total = int(pages.sum()) + 3
        order = rng.permutation(total)
        table = np.full((nB, int(pages.max())), -1, np.int32)
        owner_len = np.zeros((total,), np.int64)            # tokens that are written in each page
        first = np.cumsum(pages) - pages
        for b in range(nB):
            mine = order[first[b]: first[b] + pages[b]]
            table[b, : pages[b]] = mine
            owner_len[mine] = np.minimum(page, lens[b] - page * np.arange(pages[b]))
        unwritten = (torch.arange(page, device="cuda")[None] >= dev(owner_len)[:, None])[:, None, :, None]
        for name in ("k", "v"):
            x = normal(total, hkv, page, D).to(torch.bfloat16)
            x[..., 5] *= 6.0                                # an outlier channel of each head
            y = x.float()
            codes, scales = _quantise(y.view(total, hkv, page, D // 32, 32), None)
            codes = codes.view(torch.uint8).view(total, hkv, page, D)
            # places that no token has been written to hold whatever was there: here the codes of NaN
            s[name + "_codes"] = torch.where(unwritten, 0x7F, codes)
            s[name + "_scales"] = torch.where(unwritten, 255, scales).transpose(2, 3).contiguous()
            del x, y, codes, scales
        s["queries"] = normal(int(cu[-1]), hq * D).to(torch.bfloat16)
        s["cu_q"], s["kv_len"], s["page_table"] = dev(cu.astype(np.int32)), dev(lens.astype(np.int32)), dev(table)
        s["max_q"], s["max_kv"] = int(qs.max()), int(lens.max())
        s["out"] = torch.empty_like(s["queries"])
        s["lse"] = torch.empty((int(cu[-1]), hq), dtype=torch.float32, device="cuda")
        s["seq"] = dev(np.repeat(np.arange(nB), qs))        # the plain form's gather indices
        s["within"] = dev(np.arange(cu[-1]) - np.repeat(cu[:-1], qs))
        s["rows"] = torch.minimum(dev(cu[:-1])[:, None] + torch.arange(s["max_q"], device="cuda")[None], dev(cu[1:])[:, None] - 1)
        if own:
            import paper_2603_16590_amd as B
            s["cache"] = B.PagedCache(total, page, hkv, D, tensors=tuple(s[k] for k in ("k_codes", "k_scales", "v_codes", "v_scales")))
            s["ws"] = torch.empty(max(16, B.batq_paged_attention_workspace(s["cache"], hq, nB, int(cu[-1]), s["max_q"], s["max_kv"])),
                                  dtype=torch.uint8, device="cuda")
    else:
        M, K, N, r, n = (case[k] for k in ("M", "K", "N", "r", "n"))
        s["X"] = normal(M, K).to(torch.bfloat16)
        s["A"] = (normal(n, r, K) / math.sqrt(K)).to(torch.bfloat16)
        s["Bm"] = (normal(n, N, r) / math.sqrt(r)).to(torch.bfloat16)
        index = rng.integers(-1 if M > 4 else 0, n, M // case["runs"] + 1).repeat(case["runs"])[:M]     # -1: no adapter
        s["index"] = dev(index.astype(np.int32))
        s["scales"] = dev(rng.uniform(0.5, 2.0, n).astype(np.float32))
        s["base"] = normal(M, N).to(_DTYPE[case["y"]])
        s["out"] = torch.empty_like(s["base"])
        if own:
            import paper_2603_16590_amd as B
            s["ws"] = torch.empty(max(16, B.batq_lora_workspace(M, K, N, r, n)), dtype=torch.uint8, device="cuda")
    return s


def _cache_views(s):
    """The cache's buffers as the numbers that they stand for: E4M3 codes and E8M0 scales."""
    return {k: s[k].view(torch.float8_e4m3fn if k.endswith("codes") else torch.float8_e8m0fnu)
            for k in ("k_codes", "v_codes", "k_scales", "v_scales")}


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
        codes, scales = _quantise(x.reshape(M, hkv, D // 32, 32), clip)
        s[name + "_codes"][slot // page, :, slot % page] = codes.view(torch.uint8).view(M, hkv, D)[tok]
        s[name + "_scales"][slot // page, :, :, slot % page] = scales[tok]
    return {"q": s["q_out"], **_cache_views(s)}


def _context(s, name, mask):
    """The batch's keys or values as fp32 [B, kv heads, length, D]; zeros where `mask` [B, length] is not set."""
    nB, page, hkv, D = s["B"], s["page"], s["hkv"], s["D"]
    pt = s["page_table"].clamp_min(0).long()
    codes = s[name + "_codes"][pt].view(torch.float8_e4m3fn).float()                # [B, pages, heads, page, D]
    scale = torch.exp2(s[name + "_scales"][pt].float() - 127.0).transpose(3, 4)     # [B, pages, heads, page, D / 32]
    x = codes.view(nB, -1, hkv, page, D // 32, 32) * scale.unsqueeze(-1)
    x = x.permute(0, 2, 1, 3, 4, 5).reshape(nB, hkv, -1, D)
    return torch.where(mask[:, None, :, None], x, 0.0)


def _attend(s):
    nB, hq, hkv, D, Q = s["B"], s["hq"], s["hkv"], s["D"], s["max_q"]
    T = s["queries"].shape[0]
    L = s["page_table"].shape[1] * s["page"]
    t = torch.arange(L, device="cuda")
    mask = t[None] < s["kv_len"][:, None]
    qs = s["cu_q"][1:] - s["cu_q"][:-1]
    pos = (s["kv_len"] - qs)[:, None] + torch.arange(Q, device="cuda")[None]        # [B, Q]
    seen = mask[:, None, :] & (t[None, None] <= pos[..., None])
    if s["window"]:
        seen = seen & (t[None, None] > pos[..., None] - s["window"])
    q = s["queries"][s["rows"]].float().view(nB, Q, hkv, hq // hkv, D).permute(0, 2, 3, 1, 4).reshape(nB, hkv, -1, D)
    S = torch.matmul(q * (1.0 / math.sqrt(D)), _context(s, "k", mask).transpose(2, 3))
    S = S.view(nB, hkv, hq // hkv, Q, L).masked_fill_(~seen[:, None, None], -math.inf)
    m = S.amax(-1, keepdim=True).clamp_min(-3e38)
    S = S.sub_(m).exp_()
    total = S.sum(-1, keepdim=True)
    O = torch.matmul(S.view(nB, hkv, -1, L), _context(s, "v", mask)).view(nB, hkv, hq // hkv, Q, D) / total
    lse = (m + total.log()).squeeze(-1)
    s["out"].copy_(O[s["seq"], :, :, s["within"]].reshape(T, hq * D))
    s["lse"].copy_(lse[s["seq"], :, :, s["within"]].reshape(T, hq))
    return {"out": s["out"], "lse": s["lse"]}


def _lora(s):
    M, K, N, r, n = (s[k] for k in ("M", "K", "N", "r", "n"))
    H = torch.matmul(s["X"].float(), s["A"].float().view(n * r, K).t()).view(M, n, r)
    mine = (s["index"][:, None] == torch.arange(n, device="cuda")[None]) * s["scales"][None]
    delta = torch.matmul((H * mine[..., None]).view(M, n * r), s["Bm"].float().transpose(1, 2).reshape(n * r, N))
    s["out"].copy_(s["base"].float() + delta)
    return s["out"]


def run(s):
    if not own:
        return {"append": _append, "attend": _attend, "lora": _lora}[s["op"]](s)
    import paper_2603_16590_amd as B
    if s["op"] == "append":
        B.batq_kv_paged_append(s["cache"], s["k"], s["v"], s["slots"], positions=s["positions"], q=s["q"], q_out=s["q_out"],
                               rope=s["table"], interleaved=s["inter"], tk=s["tk"], tv=s["tv"])
        return {"q": s["q_out"], **_cache_views(s)}
    if s["op"] == "attend":
        B.batq_paged_attention(s["cache"], s["queries"], s["cu_q"], s["kv_len"], s["page_table"], s["max_q"], s["max_kv"],
                               window=s["window"], out=s["out"], lse=s["lse"], workspace=s["ws"])
        return {"out": s["out"], "lse": s["lse"]}
    return B.batq_lora_add(s["X"], s["A"], s["Bm"], s["index"], s["base"], scales=s["scales"], out=s["out"], workspace=s["ws"])


def _lengths(case):
    """Expected sums over a batch: (tokens of the caches, query tokens, visible pairs of a query token and a key)."""
    def mean(top, spread):                                  # of top * exp(-spread * u * log(top + 1)), u uniform
        a = spread * math.log(top + 1)
        return top * (1.0 if a == 0 else (1.0 - math.exp(-a)) / a)

    B, q, kv, spread, window = case["B"], case["q"], case["kv"], case["spread"], case["window"] or case["kv"]
    L, T = kv + (B - 1) * mean(kv, spread), q + (B - 1) * mean(q, spread)

    def pairs(n, length):                                   # the last n queries of `length` tokens
        return n * min(window, max(1.0, length - (n - 1) / 2.0))

    seen = pairs(min(q, kv), kv) + (B - 1) * pairs(mean(q, spread), mean(kv, spread))
    reach = min(kv, window + q) + (B - 1) * min(mean(kv, spread), window + mean(q, spread))
    return min(L, reach), T, seen


def work(case):
    if case["op"] == "append":
        M, hq, hkv, D, rot = (case[k] for k in ("M", "hq", "hkv", "D", "rot"))
        size = {"bf16": 2, "f32": 4}[case["x"]]
        per = (hq + 2 * hkv) * D * size + hq * D * 2 + 2 * hkv * D * 33 / 32 + rot * 4 + 12
        # a block's Kronecker product takes 12 multiply-adds per element, a rotation 3 operations
        return {"bytes": M * per, "flops": M * D * (24.0 * (hq + 2 * hkv) * case["transform"] + 3.0 * (hq + hkv))}
    if case["op"] == "attend":
        hq, hkv, D = case["hq"], case["hkv"], case["D"]
        L, T, seen = _lengths(case)
        return {"bytes": L * hkv * D * 2 * 33 / 32 + T * hq * (4 * D + 4), "flops": 4.0 * seen * hq * D}
    M, K, N, r, n = (case[k] for k in ("M", "K", "N", "r", "n"))
    used = min(n, M // case["runs"] + 1)
    return {"bytes": M * K * 2 + used * r * (K + N) * 2 + 2 * M * N * {"bf16": 2, "f32": 4}[case["y"]], "flops": 2.0 * M * r * (K + N)}


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
        return {"q": q.reshape(M, -1), "k_codes": None, "v_codes": None, "k_scales": None, "v_scales": None}
    out = {"q": q.reshape(M, -1)}
    slots = s["slots"].cpu().numpy()
    for name, x in (("k", k), ("v", v)):
        pages = s[name + "_codes"].shape[0]
        codes, scales = np.zeros((pages, hkv, page, D)), np.ones((pages, hkv, D // 32, page))
        x = x.reshape(M, hkv, D // 32, 32)
        top = np.abs(x).max(-1, keepdims=True)
        e = np.where(top > 0, np.clip(np.floor(np.log2(np.where(top > 0, top, 1.0))) - 8, -127, 127), -127)
        y = x * 2.0 ** -e
        step = 2.0 ** (np.clip(np.floor(np.log2(np.maximum(np.abs(y), 2.0 ** -30))), -6, 8) - 3)
        y = np.clip(np.rint(y / step) * step, -448, 448)    # (rint: ties to even)
        used = slots >= 0
        codes[slots[used] // page, :, slots[used] % page] = y.reshape(M, hkv, D)[used]
        scales[slots[used] // page, :, :, slots[used] % page] = 2.0 ** e[used][..., 0]
        out[name + "_codes"], out[name + "_scales"] = codes, scales
    return out


def _exact_attend(s):
    hq, hkv, D, page = (s[k] for k in ("hq", "hkv", "D", "page"))
    cu, lens = s["cu_q"].tolist(), s["kv_len"].tolist()
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["lse"].shape, dtype=torch.float64, device="cuda")
    for b, L in enumerate(lens):
        pages = s["page_table"][b, : -(-L // page)].long()
        n = cu[b + 1] - cu[b]
        at = torch.arange(L - n, L, device="cuda")[:, None]
        t = torch.arange(L, device="cuda")[None]
        hidden = (t > at) | (t <= at - s["window"]) if s["window"] else t > at
        for h in range(hkv):
            kv = []
            for name in ("k", "v"):
                codes = s[name + "_codes"][pages, h].reshape(-1, D)[:L].view(torch.float8_e4m3fn).double()
                scale = s[name + "_scales"][pages, h].transpose(1, 2).reshape(-1, D // 32)[:L].double()
                kv.append(codes * (2.0 ** (scale - 127)).repeat_interleave(32, 1))
            for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                S = s["queries"][cu[b]: cu[b + 1], g * D: (g + 1) * D].double() @ kv[0].t() / math.sqrt(D)
                S.masked_fill_(hidden, -math.inf)
                lse[cu[b]: cu[b + 1], g] = torch.logsumexp(S, 1)
                out[cu[b]: cu[b + 1], g * D: (g + 1) * D] = torch.softmax(S, 1) @ kv[1]
    return {"out": out.cpu().numpy(), "lse": lse.cpu().numpy()}


def _exact_lora(s):
    out = s["base"].double()
    index = s["index"].tolist()
    for a in sorted(set(index) - {-1}):
        rows = torch.tensor([m for m, i in enumerate(index) if i == a], device="cuda")
        out[rows] += float(s["scales"][a]) * ((s["X"][rows].double() @ s["A"][a].double().t()) @ s["Bm"][a].double().t())
    return out.cpu().numpy()


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attend": _exact_attend, "lora": _exact_lora}[s["op"]](s)
