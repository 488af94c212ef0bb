"""Scores of cached tokens and eviction by them (batq_kv_paged_score, batq_kv_paged_evict), against plain 64-bit statements, and a
decoder that lives within a budget of tokens."""
import numpy as np
import pytest

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


def make_cache(B, arrays, bits):
    pages, heads, page, D = arrays[0].shape
    return B.PagedCache(pages, page, heads, D * 8 // bits, tensors=[dev(a) for a in arrays], bits=bits)


def host(cache):
    return [t.cpu().numpy() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]


def lse_of(arrays, bits, q, cu, lens, table, page, causal, window, T):
    """fp32 lse of the attention, 7 in rows of no sequence."""
    kv = br.values(*arrays[:2], bits)
    x = ref.attention(kv, np.zeros_like(kv), q, cu, lens, table, page, kv.shape[-1] ** -0.5, causal, window, T)[1]
    return np.where(np.isnan(x) & (np.arange(T) >= cu[-1])[:, None], 7.0, x).astype(np.float32)


def run_score(B, cache, qd, lse, had, cu, lens, table, max_q=None, max_kv=None, **kw):
    import torch
    score = dev(had)
    B.batq_kv_paged_score(cache, qd, dev(lse), score, dev(cu), dev(lens), dev(table), int(np.diff(cu).max()) if max_q is None else max_q,
                          int(max(lens)) if max_kv is None else max_kv, **kw)
    torch.cuda.synchronize()
    return score.cpu().numpy()


SCORE = [
    # lens, query counts, q heads, kv heads, D, page, window
    ([1], [1], 1, 1, 64, 16, 0),
    ([1, 15, 16, 17, 63, 64, 65, 129], [1] * 8, 8, 2, 128, 16, 0),
    ([0, 5, 0, 300], [1, 1, 2, 1], 7, 1, 128, 32, 0),
    ([700, 3, 1025], [1, 1, 1], 28, 4, 64, 64, 0),
    ([513, 40], [3, 2], 8, 4, 64, 256, 0),
    ([200, 90], [5, 7], 6, 2, 128, 16, 33),
    ([333], [333], 3, 3, 64, 32, 0),
    ([290], [290], 8, 1, 128, 16, 0),
    ([130, 64, 257, 1], [130, 1, 100, 1], 14, 2, 128, 64, 0),
    ([200, 140], [70, 140], 4, 4, 128, 32, 1),
    ([500], [129], 2, 1, 64, 16, 100),
    ([700, 600], [0, 2], 128, 1, 128, 16, 0),               # a sequence without queries
    ([5, 9], [9, 20], 4, 2, 64, 16, 0),                     # more queries than tokens
    ([3000, 200], [64, 64], 4, 1, 128, 64, 0),
    ([900], [900], 16, 2, 64, 64, 301),
]


@pytest.mark.parametrize("lens,qs,hq,hkv,D,page,window", SCORE)
@pytest.mark.parametrize("bits,causal,add", [(4, True, False), (8, True, True), (4, False, True)])
def test_score(B, lens, qs, hq, hkv, D, page, window, bits, causal, add):
    rng = np.random.default_rng(sum(lens) + sum(qs) + hq)
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, bits, spare=2)
    lse = lse_of(arrays, bits, q, cu, lens, table, page, causal, window, T)
    had = rng.uniform(0, 3, (arrays[0].shape[0], hkv, page)).astype(np.float32)
    got = run_score(B, make_cache(B, arrays, bits), to_dev(qbits, "bf16"), lse, had, cu, lens, table, causal=causal, window=window, add=add)
    want = br.score(br.values(*arrays[:2], bits), q, lse, had, cu, lens, table, page, D ** -0.5, causal, window, add)
    br.assert_score(got, want, had)


def test_scores_add_up_to_the_number_of_rows(B):
    """The weights of a row that sees something add up to 1: with the library's own lse, over all tokens of a key head."""
    import torch
    rng = np.random.default_rng(1)
    hq, hkv, D, page = 12, 3, 128, 32
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [1200, 77, 300], [200, 77, 1], hq, hkv, D, page, 4)
    cache, qd = make_cache(B, arrays, 4), to_dev(qbits, "bf16")
    lse = torch.empty((T, hq), device="cuda")
    B.batq_paged_attention(cache, qd, dev(cu), dev(lens), dev(table), 200, 1200, lse=lse)
    score = torch.full((arrays[0].shape[0], hkv, page), -1.0, device="cuda")
    B.batq_kv_paged_score(cache, qd, lse, score, dev(cu), dev(lens), dev(table), 200, 1200)
    got = score.double().cpu().numpy()
    for b, n in enumerate(np.diff(cu)):
        t = np.arange(lens[b])
        total = got[table[b, t // page], :, t % page].sum(0)
        assert np.all(np.abs(total / (n * hq / hkv) - 1) < 1e-4)


def test_score_of_some_queries_and_other_scales(B):
    """The last queries of a prompt alone (their rows of q and lse), column ranges of wider tensors, a scale."""
    import torch
    rng = np.random.default_rng(2)
    hq, hkv, D, page, scale = 8, 2, 64, 16, 0.3
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [400, 90], [60, 32], hq, hkv, D, page, 8)
    kv = br.values(*arrays[:2], 8)
    lse = ref.attention(kv, np.zeros_like(kv), q, cu, lens, table, page, scale, True, 0, T)[1].astype(np.float32)
    rows = np.concatenate([np.arange(cu[b + 1] - 32, cu[b + 1]) for b in range(2)])
    cu2 = np.array([0, 32, 64], np.int32)
    wide = torch.zeros((64, hq * D + 64), dtype=torch.bfloat16, device="cuda")
    wide[:, : hq * D] = to_dev(qbits, "bf16")[torch.from_numpy(rows).cuda()]
    had = np.full((arrays[0].shape[0], hkv, page), 5.0, np.float32)
    got = run_score(B, make_cache(B, arrays, 8), wide[:, : hq * D], lse[rows], had, cu2, lens, table, scale=scale)
    br.assert_score(got, br.score(kv, q[rows], lse[rows], had, cu2, lens, table, page, scale, True, 0, False), had)


def test_score_does_not_trust_its_lists(B):
    """Pages outside the cache, lengths past the table, negative ones, bounds below what the lists say, rows outside q."""
    rng = np.random.default_rng(6)
    hq, hkv, D, page = 4, 2, 128, 16
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [100, 40, 64, 90], [1, 3, 20, 1], hq, hkv, D, page, 4, spare=2)
    kv, qd = br.values(*arrays[:2], 4), to_dev(qbits, "bf16")
    table[0, 2], table[2, 0], table[2, 3], table[1, 0] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1
    table[3, :] = -1
    cache = make_cache(B, arrays, 4)
    lse = np.nan_to_num(lse_of(arrays, 4, q, cu, lens, table, page, True, 0, T), neginf=-np.inf)
    had = rng.uniform(0, 3, (arrays[0].shape[0], hkv, page)).astype(np.float32)
    for add in (False, True):
        got = run_score(B, cache, qd, lse, had, cu, lens, table, max_kv=128, add=add)
        br.assert_score(got, br.score(kv, q, lse, had, cu, lens, table, page, D ** -0.5, True, 0, add), had)
        # the first two queries of each; tokens up to 50
        got = run_score(B, cache, qd, lse, had, cu, lens, table, max_q=2, max_kv=50, add=add)
        br.assert_score(got, br.score(kv, q, lse, had, cu, np.minimum(lens, 50), table, page, D ** -0.5, True, 0, add, max_q=2), had)
        longer = lens.copy()
        longer[1], longer[3] = -5, 10 ** 9
        got = run_score(B, cache, qd, lse, had, cu, longer, table, max_kv=10 ** 6, add=add)
        eff = np.array([100, 0, 64, table.shape[1] * page])
        br.assert_score(got, br.score(kv, q, lse, had, cu, eff, table, page, D ** -0.5, True, 0, add), had)
        for broken in ([0, 1, 4, 24, 10 ** 6], [0, -1, 4, 24, 25]):
            got = run_score(B, cache, qd, lse, had, np.array(broken, np.int32), lens, table, max_q=20, max_kv=128, add=add)
            t = np.arange(16, 64 - 20)                      # sequence 2 keeps its rows (0 and 3 are pages that do not exist)
            want = br.score(kv, q, lse, had, cu, lens, table, page, D ** -0.5, True, 0, add)
            t = t[(t // page == 1) | (t // page == 2)]
            at = (table[2, t // page], slice(None), t % page)
            assert np.all(np.abs(got[at] - want[0][at]) <= want[1][at])


def test_scores_of_a_large_ragged_batch(B):
    """More sequences than a wave has lanes: chunks and single tokens in any order, empty ones among them, sequences without queries; parts
    of rows in some."""
    rng = np.random.default_rng(15)
    hq, hkv, D, page, n = 8, 2, 64, 16, 150
    lens = rng.integers(0, 90, n)
    qs = np.where(rng.random(n) < 0.2, rng.integers(0, 60, n), 1)
    qs[[0, 70, 149]], lens[[0, 70, 149]] = [0, 420, 95], [400, 700, 95]
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 4, spare=1)
    kv = br.values(*arrays[:2], 4)
    for window, add in ((0, True), (40, False)):
        lse = lse_of(arrays, 4, q, cu, lens, table, page, True, window, T)
        had = rng.uniform(0, 3, (arrays[0].shape[0], hkv, page)).astype(np.float32)
        got = run_score(B, make_cache(B, arrays, 4), to_dev(qbits, "bf16"), lse, had, cu, lens, table, window=window, add=add)
        br.assert_score(got, br.score(kv, q, lse, had, cu, lens, table, page, D ** -0.5, True, window, add), had)


@pytest.mark.parametrize("qs,max_q", [([300, 2], None), ([40, 3, 500], 45)])
def test_few_rows_beside_many(B, qs, max_q):
    """Sequences of few rows beside one of many, also where the bound on queries hides some of them."""
    rng = np.random.default_rng(16)
    hq, hkv, D, page = 4, 1, 128, 32
    lens = [700, 900, 600][: len(qs)]
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 8)
    lse = lse_of(arrays, 8, q, cu, lens, table, page, True, 0, T)
    had = np.ones((arrays[0].shape[0], hkv, page), np.float32)
    got = run_score(B, make_cache(B, arrays, 8), to_dev(qbits, "bf16"), lse, had, cu, lens, table, max_q=max_q, add=True)
    br.assert_score(got, br.score(br.values(*arrays[:2], 8), q, lse, had, cu, lens, table, page, D ** -0.5, True, 0, True, max_q=max_q), had)


def test_score_arrays_at_any_word(B):
    """Scores that begin at a multiple of 4 bytes, no more: scoring and eviction."""
    import torch
    rng = np.random.default_rng(17)
    hq, hkv, D, page, budget = 4, 2, 64, 16, 70
    arrays, lens, table, out_table = evict_case(rng, [200, 90, 333], hkv, D, page, budget, 4)
    cu, T = np.array([0, 1, 2, 40], np.int32), 40
    qd = to_dev(ref.bf16_values(rng, T, hq * D)[0], "bf16")
    lse = dev(rng.uniform(3, 6, (T, hq)).astype(np.float32))
    had = scores_for(rng, "sums", (arrays[0].shape[0], hkv, page))
    results = []
    for shift in (0, 1, 2, 3):
        cache = make_cache(B, arrays, 4)
        store = torch.full((had.size + 8,), 9.0, device="cuda")
        score = store[shift: shift + had.size].view(had.shape)
        score.copy_(dev(had))
        B.batq_kv_paged_score(cache, qd, lse, score, dev(cu), dev(lens), dev(table), 38, 333, add=True)
        keep, new_len = B.batq_kv_paged_evict(cache, score, dev(lens), dev(table), dev(out_table), 333, budget, 2, 5)
        torch.cuda.synchronize()
        assert bool((store[:shift] == 9.0).all()) and bool((store[shift + had.size:] == 9.0).all())
        results.append([score.clone(), keep, new_len] + [t.clone() for t in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)])
    for r in results[1:]:
        assert all(torch.equal(x, y) for x, y in zip(r, results[0]))


def test_score_of_keys_and_rows_that_are_not_finite(B):
    """A NaN key makes the lse of the rows that see it NaN, and with it the scores of all tokens that they see; other tokens' stay."""
    rng = np.random.default_rng(7)
    hq, hkv, D, page = 4, 2, 64, 16
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [200, 90], [120, 1], hq, hkv, D, page, 4)
    arrays[1][table[0, 150 // page], 1, 0, 150 % page] = 255
    lse = lse_of(arrays, 4, q, cu, lens, table, page, True, 30, T)
    assert np.isnan(lse).any()
    had = np.ones((arrays[0].shape[0], hkv, page), np.float32)
    got = run_score(B, make_cache(B, arrays, 4), to_dev(qbits, "bf16"), lse, had, cu, lens, table, window=30)
    want, tol = br.score(br.values(*arrays[:2], 4), q, lse, had, cu, lens, table, page, D ** -0.5, True, 30, False)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).any() and not np.isnan(want).all()
    fine = ~np.isnan(want)
    br.assert_score(np.where(fine, got, 0.0), (np.where(fine, want, 0.0), np.where(fine, tol, 0.0)), np.where(fine, had, 0.0))


@pytest.mark.parametrize("hq,hkv,lens,qs", [(3, 1, [700, 300], [400, 300]), (14, 2, [500], [173]), (48, 1, [400], [77]), (65, 1, [300, 90], [50, 21]),
                                            (100, 1, [600], [64]), (254, 2, [270], [31]), (128, 1, [520], [70])])
def test_each_row_of_many_takes_its_own_lse(B, hq, hkv, lens, qs):
    """Groups that do not divide a stage of 64 rows, or are larger than one, with an lse that tells every query and head from all
    others: weights by another row's would be off by 2 % at least (neighbouring heads by e, neighbouring queries by e^0.02)."""
    rng = np.random.default_rng(hq + sum(qs))
    D, page = 64, 16
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 8)
    lse = (np.arange(T)[:, None] * 0.02 % 3 + np.arange(hq) % 5).astype(np.float32)
    had = rng.uniform(0, 3, (arrays[0].shape[0], hkv, page)).astype(np.float32)
    got = run_score(B, make_cache(B, arrays, 8), to_dev(qbits, "bf16"), lse, had, cu, lens, table)
    br.assert_score(got, br.score(br.values(*arrays[:2], 8), q, lse, had, cu, lens, table, page, D ** -0.5, True, 0, False), had)


def share_prefix(rng, arrays, table, lens, page, prefix, extra):
    """The first `prefix` tokens' pages of sequence 0 for all sequences, and score pages behind the cache's for those that share them.
    Returns (page table, score table, arrays with a copy of each shared page in its score page's place, number of pages of the cache)."""
    pages, n = arrays[0].shape[0], prefix // page
    table, score_table = table.copy(), table.copy()
    at = pages + rng.permutation(extra)[: n * (len(lens) - 1)]
    copies = [np.concatenate([a, a[rng.integers(0, pages, extra)]]) for a in arrays]
    for b in range(1, len(lens)):
        table[b, :n] = table[0, :n]
        score_table[b, :n] = at[(b - 1) * n: b * n]
        for c in copies:
            c[score_table[b, :n]] = c[table[0, :n]]
    return table, score_table, copies, pages


@pytest.mark.parametrize("add", [False, True])
@pytest.mark.parametrize("qs,hq,hkv,D,bits", [([1, 1, 1], 8, 2, 128, 4), ([2, 5, 1], 4, 1, 64, 8), ([40, 300, 1], 4, 2, 64, 4), ([200, 1, 130], 14, 2, 128, 8)])
def test_scores_of_a_shared_prefix(B, qs, hq, hkv, D, bits, add):
    """Three sequences share the pages of their first tokens and have score pages of their own for them: each place gets its own
    sequence's sum, the same bits whenever the call is repeated.  Entries without a page of either kind take no part."""
    rng = np.random.default_rng(31 + sum(qs))
    page = 16
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [1100, 700, 400], qs, hq, hkv, D, page, bits)
    table, score_table, copies, pages = share_prefix(rng, arrays, table, lens, page, 256, 40)
    lse = lse_of(arrays, bits, q, cu, lens, table, page, True, 0, T)
    lse[np.isnan(lse)] = 3.0
    score_table[1, 3], score_table[2, 5], table[0, 20], table[1, 18] = -1, pages + 40, -5, pages
    where = np.where((table < 0) | (table >= pages), -1, score_table)
    had = rng.uniform(0, 3, (pages + 40, hkv, page)).astype(np.float32)
    cache, qd = make_cache(B, arrays, bits), to_dev(qbits, "bf16")
    got = [run_score(B, cache, qd, lse, had, cu, lens, table, score_table=dev(score_table), add=add) for _ in range(3)]
    br.assert_score(got[0], br.score(br.values(*copies[:2], bits), q, lse, had, cu, lens, where, page, D ** -0.5, True, 0, add), had)
    assert all(np.array_equal(x.view(np.uint32), got[0].view(np.uint32)) for x in got[1:])
    own = run_score(B, cache, qd, lse, had[:pages], cu, lens, table, add=add)      # what is not shared is as without the table
    mine = np.setdiff1d(table[(table >= 0) & (table < pages)], table[0, :16])
    assert np.array_equal(own[mine].view(np.uint32), got[0][mine].view(np.uint32))


@pytest.mark.parametrize("lens,budget,kind", [([300, 500, 90], 100, "sums"), ([5000, 300, 4500], 700, "odd"), ([40000, 33000], 3000, "ties")])
def test_evict_by_scores_of_their_own(B, lens, budget, kind):
    """Sequences with a common prefix, evicted by score pages of their own; a token without one counts as the smallest and moves
    with a score of 0."""
    rng = np.random.default_rng(41 + budget)
    hkv, D, page, first, last = 2, 64, 16, 3, 20
    arrays, lens, table, out_table = evict_case(rng, lens, hkv, D, page, budget, 4)
    table, score_table, copies, pages = share_prefix(rng, arrays, table, lens, page, 64, 20)
    none = pages + 20                                       # a page of scores that is not there
    score = scores_for(rng, kind, (pages + 20, hkv, page))
    want_score = np.concatenate([score, np.full((1, hkv, page), np.nan, np.float32)])
    copies = [np.concatenate([c, c[table[0, 0]][None]]) for c in copies]
    told, where = score_table.copy(), score_table.copy()
    told[1, 0], where[1, 0] = -3, none                      # among the first tokens, which stay
    want = br.evict(copies, want_score, lens, where, out_table, budget, first, last)
    for h in range(hkv):
        j = np.arange(want[3][1])
        moved = want[2][1, h, j] < page
        want[1][out_table[1][j[moved] // page], h, j[moved] % page] = 0.0
    got = run_evict(B, make_cache(B, arrays, 4), score, lens, table, out_table, budget, first, last, score_table=dev(told))
    assert_evicted(got, ([w[:pages] for w in want[0]], want[1][:none], want[2], want[3]))


@pytest.mark.parametrize("lens,qs,hq,hkv,D,window", [([3000, 90], [1, 1], 8, 2, 128, 50), ([500, 700, 33], [3, 1, 0], 4, 2, 64, 100), ([900, 1500], [64, 100], 4, 1, 64, 200),
                                                     ([1000], [5], 2, 1, 64, 1), ([3000, 2500], [700, 1], 8, 1, 128, 33), ([400, 300], [0, 2], 4, 1, 64, 0)])
@pytest.mark.parametrize("causal", [True, False])
def test_tokens_that_no_query_sees(B, lens, qs, hq, hkv, D, window, causal):
    """With add their places keep their bits (-0 among them, which a sum with 0 would turn to 0); without it they become 0."""
    rng = np.random.default_rng(61 + sum(lens))
    page = 16
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 4)
    lse = lse_of(arrays, 4, q, cu, lens, table, page, causal, window, T)
    had = np.where(rng.random((arrays[0].shape[0], hkv, page)) < 0.5, -0.0, rng.uniform(0, 3, (arrays[0].shape[0], hkv, page))).astype(np.float32)
    cache, qd = make_cache(B, arrays, 4), to_dev(qbits, "bf16")
    unseen = []
    for b, L in enumerate(lens):
        first = L - qs[b]
        t = np.arange(max(0, first - window + 1) if window else 0) if qs[b] else np.arange(L)
        unseen.append((table[b, t // page], t % page))
    assert sum(len(x[0]) for x in unseen) > 100
    for add in (True, False):
        got = run_score(B, cache, qd, lse, had, cu, lens, table, causal=causal, window=window, add=add)
        br.assert_score(got, br.score(br.values(*arrays[:2], 4), q, lse, had, cu, lens, table, page, D ** -0.5, causal, window, add), had)
        for pg, off in unseen:
            want = had[pg, :, off] if add else np.zeros((len(pg), hkv), np.float32)
            assert np.array_equal(got[pg, :, off].view(np.uint32), want.view(np.uint32))


@pytest.mark.parametrize("qn", [1, 40])
def test_pages_given_back_behind_a_window(B, qn):
    """A sequence's table still names pages behind its window that are another sequence's by now: with add they get the other's sums."""
    rng = np.random.default_rng(71 + qn)
    hq, hkv, D, page, window = 4, 2, 128, 16, 60
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, [900, 400], [qn, qn], hq, hkv, D, page, 4)
    lse = lse_of(arrays, 4, q, cu, lens, table, page, True, window, T)
    had = rng.uniform(0, 3, (arrays[0].shape[0], hkv, page)).astype(np.float32)
    want = br.score(br.values(*arrays[:2], 4), q, lse, had, cu, lens, table, page, D ** -0.5, True, window, True)
    gone = (900 - qn - window + 1) // page                  # pages before this one are seen by nobody
    stale = table.copy()
    stale[0, :gone] = np.resize(table[1, : -(-400 // page)], gone)
    untouched = want[1].copy()
    untouched[table[0, :gone]] = -1.0
    cache, qd = make_cache(B, arrays, 4), to_dev(qbits, "bf16")
    got = [run_score(B, cache, qd, lse, had, cu, lens, stale, window=window, add=True) for _ in range(3)]
    br.assert_score(got[0], (want[0], untouched), had)
    assert all(np.array_equal(x.view(np.uint32), got[0].view(np.uint32)) for x in got[1:])


@pytest.mark.parametrize("first", ["whole prompt, added", "last queries, set", "last queries, added"])
def test_first_scores_in_pages_that_were_used_before(B, first):
    """Pages full of other sequences' scores: a first call over the whole prompt may add, one of its last queries must not; the steps behind
    it add.  (Added from the start, the last queries leave the old owners' scores in the earlier tokens' places.)"""
    rng = np.random.default_rng(81)
    hq, hkv, D, page, L = 4, 2, 64, 16, 210
    arrays, qbits, q, _, lens, table, T = br.batch_case(rng, [L + 2], [L + 2], hq, hkv, D, page, 8)
    kv, cache, qd = br.values(*arrays[:2], 8), make_cache(B, arrays, 8), to_dev(qbits, "bf16")
    lse = lse_of(arrays, 8, q, np.array([0, L + 2]), lens, table, page, True, 0, T)
    junk = np.full((arrays[0].shape[0], hkv, page), 1e3, np.float32)
    begin, add = (0 if "whole" in first else L - 20), "added" in first
    score, clean = junk, np.zeros_like(junk)
    want, tol = clean.astype(np.float64), clean.astype(np.float64)
    for lo, hi, a in ((begin, L, add), (L, L + 1, True), (L + 1, L + 2, True)):
        cu, n = np.array([0, hi - lo], np.int32), np.array([hi], np.int32)
        score = run_score(B, cache, qd[lo:hi], lse[lo:hi], score, cu, n, table, add=a)
        w, t = br.score(kv, q[lo:hi], lse[lo:hi], clean, cu, n, table, page, D ** -0.5, True, 0, True)
        want, tol = want + w, tol + np.maximum(t, 0) + 2.0 ** -24 * np.abs(want + w)
    at = np.arange(L + 2)
    at = (table[0, at // page], slice(None), at % page)
    if first != "last queries, added":
        assert np.all(np.abs(score[at] - want[at]) <= tol[at])
    else:                                                   # old tokens: fp32 sums upon the thousand, each off by half a step of 2^-14
        old = np.arange(L + 2)[:, None] < begin
        assert np.all(np.abs(score[at] - want[at] - 1e3 * old) <= tol[at] + 3 * 2.0 ** -14 * old)


# ---------------------------------------------------------------------------------------- eviction
EVICT = [
    # lens, kv heads, D, page, budget, first, last
    ([1], 1, 64, 16, 1, 0, 0),
    ([2], 1, 64, 16, 1, 0, 0),
    ([40, 17, 0, 16, 300], 2, 128, 16, 16, 1, 3),
    ([40, 17, 0, 16, 300], 3, 64, 32, 17, 0, 0),
    ([1000, 999, 5], 2, 64, 64, 333, 4, 100),
    ([100], 2, 128, 16, 64, 32, 32),                        # nothing left to choose
    ([100, 70], 1, 128, 256, 64, 64, 0),
    ([100, 70], 1, 64, 16, 64, 0, 64),
    ([2500, 2049], 2, 64, 16, 2048, 4, 64),
    ([70, 80], 2, 64, 16, 200, 4, 64),                      # all stay
    ([5000], 1, 64, 128, 1, 0, 0),
    ([9000, 4097], 1, 64, 32, 1025, 1, 1),
]


def evict_case(rng, lens, hkv, D, page, budget, bits):
    lens = np.array(lens)
    fresh = -(-np.minimum(lens, budget) // page)
    arrays, _, _, _, lens, table, _ = br.batch_case(rng, lens, np.zeros(len(lens), int), 1 * hkv, hkv, D, page, bits, more_pages=int(fresh.sum()) + 2)
    free = np.setdiff1d(np.arange(arrays[0].shape[0]), table)
    rng.shuffle(free)
    out_table = np.full((len(lens), max(1, int(fresh.max()))), -9, np.int32)
    at = 0
    for b, n in enumerate(fresh):
        out_table[b, :n] = free[at: at + n]
        at += n
    return arrays, lens, table, out_table


def scores_for(rng, kind, shape):
    x = rng.standard_normal(shape).astype(np.float32)
    if kind == "sums":                                      # what sums of weights look like
        x = np.exp(3 * x - 4).astype(np.float32)
    elif kind == "ties":
        x = np.round(2 * x).astype(np.float32) * np.float32(0.25)
        x[x == 0] *= np.float32(-1.0)                       # some zeros are -0
    elif kind == "same":
        x[...] = 0.5
    elif kind == "close":                                   # all bits but the last ones are the same
        x = (np.float32(1.0).view(np.uint32) + rng.integers(0, 40, shape, dtype=np.uint32)).astype(np.uint32).view(np.float32)
    elif kind == "odd":
        x[rng.random(shape) < 0.2] = np.nan
        x[rng.random(shape) < 0.1] = np.inf
        x[rng.random(shape) < 0.1] = -np.inf
        x[rng.random(shape) < 0.05] = -np.nan
        x[rng.random(shape) < 0.05] = np.float32(1e-42)
    return x


def run_evict(B, cache, score, lens, table, out_table, budget, first, last, max_kv=None, **kw):
    import torch
    ds = dev(score)
    keep, new_len = B.batq_kv_paged_evict(cache, ds, dev(lens), dev(table), dev(out_table), int(max(lens)) if max_kv is None else max_kv,
                                          budget, first, last, **kw)
    torch.cuda.synchronize()
    return host(cache), ds.cpu().numpy(), keep.cpu().numpy(), new_len.cpu().numpy()


def assert_evicted(got, want):
    assert np.array_equal(got[3], want[3]) and np.array_equal(got[2], want[2])
    for g, w, name in zip(got[0], want[0], ("k codes", "k scales", "v codes", "v scales")):
        assert np.array_equal(g, w), name
    assert np.array_equal(got[1].view(np.uint32), want[1].view(np.uint32))


@pytest.mark.parametrize("lens,hkv,D,page,budget,first,last", EVICT)
@pytest.mark.parametrize("kind,bits", [("sums", 4), ("ties", 8), ("same", 4), ("close", 8), ("odd", 4)])
def test_evict(B, lens, hkv, D, page, budget, first, last, kind, bits):
    rng = np.random.default_rng(sum(lens) + budget)
    arrays, lens, table, out_table = evict_case(rng, lens, hkv, D, page, budget, bits)
    score = scores_for(rng, kind, (arrays[0].shape[0], hkv, page))
    got = run_evict(B, make_cache(B, arrays, bits), score, lens, table, out_table, budget, first, last)
    assert_evicted(got, br.evict(arrays, score, lens, table, out_table, budget, first, last))


@pytest.mark.parametrize("lens,hkv,budget,first,last,kind", [
    ([20000, 33], 2, 5000, 3, 500, "ties"),                 # a workgroup's registers
    ([70000, 33, 40000], 2, 20000, 3, 500, "sums"),         # several workgroups to a (sequence, key head)
    ([70000, 100, 0], 1, 100, 0, 0, "same"), ([66000], 3, 8000, 4000, 4000, "close"), ([65537, 70000], 1, 33000, 1, 0, "odd")])
def test_evict_of_long_sequences(B, lens, hkv, budget, first, last, kind):
    rng = np.random.default_rng(3 + budget)
    arrays, lens, table, out_table = evict_case(rng, lens, hkv, 64, 256, budget, 4)
    score = scores_for(rng, kind, (arrays[0].shape[0], hkv, 256))
    got = run_evict(B, make_cache(B, arrays, 4), score, lens, table, out_table, budget, first, last)
    assert_evicted(got, br.evict(arrays, score, lens, table, out_table, budget, first, last))


def test_evict_of_many_long_sequences(B):
    """So many (sequence, key head) pairs of long sequences that a workgroup each fills the card: 260 that share their pages."""
    import torch
    rng = np.random.default_rng(18)
    hkv, D, page, L, budget, n = 4, 64, 256, 33000, 40, 260
    arrays, lens, table, out_table = evict_case(rng, [L] + [budget] * (n - 1), hkv, D, page, budget, 4)
    score = scores_for(rng, "ties", (arrays[0].shape[0], hkv, page))
    want = br.evict(arrays, score, lens[:1], table[:1], out_table[:1], budget, 1, 5)
    cache, ds = make_cache(B, arrays, 4), dev(score)
    keep, new_len = B.batq_kv_paged_evict(cache, ds, dev(np.full(n, L, np.int32)), dev(np.repeat(table[:1], n, 0)), dev(out_table), L, budget, 1, 5)
    torch.cuda.synchronize()
    assert bool((new_len == budget).all()) and np.array_equal(keep.cpu().numpy(), np.repeat(want[2], n, 0))
    first, rest = out_table[0, 0], torch.from_numpy(out_table[1:, 0].astype(np.int64)).cuda()
    for got, w in zip(host(cache), want[0]):
        assert np.array_equal(got[first], w[first])
    for t in (cache.k_codes, cache.v_codes, ds):
        assert bool((t[rest][:, :, :budget] == t[int(first)][None, :, :budget]).all())


def test_a_workspace_serves_every_smaller_call(B):
    """Sizes grow with every bound, and a call runs with what its bounds ask for, full of anything."""
    import torch
    rng = np.random.default_rng(14)
    for D, hq, hkv in ((128, 32, 8), (64, 16, 2), (128, 128, 1), (64, 3, 3)):
        cache = B.PagedCache(2, 16, hkv, D, bits=4)
        for _ in range(400):
            big = [int(np.exp(rng.uniform(0, np.log(n)))) for n in (200, 8192, 8192, 200000)]
            small = [int(rng.integers(1, n + 1)) if rng.random() < 0.7 else n for n in big]
            assert B.batq_kv_paged_score_workspace(cache, hq, *small) <= B.batq_kv_paged_score_workspace(cache, hq, *big), (small, big)
            e = [B.batq_kv_paged_evict_workspace(cache, x[0], x[3], x[1]) for x in (small, big)]
            assert e[0] <= e[1], (small, big)
    hq, hkv, D, page = 8, 2, 64, 16
    lens, qs = [3000, 2500, 300, 900], [1500, 40, 300, 1]
    arrays, qbits, q, cu, lens, table, T = br.batch_case(rng, lens, qs, hq, hkv, D, page, 4)
    kv, qd = br.values(*arrays[:2], 4), to_dev(qbits, "bf16")
    lse = lse_of(arrays, 4, q, cu, lens, table, page, True, 0, T)
    cache, had = make_cache(B, arrays, 4), np.ones((arrays[0].shape[0], hkv, page), np.float32)
    ws = torch.full((B.batq_kv_paged_score_workspace(cache, hq, 4, T, 1500, 3000),), 0xFF, dtype=torch.uint8, device="cuda")
    assert ws.numel()
    for rows in ([0, 1, 2, 3], [0], [1], [2, 3], [0, 3]):
        sel = np.concatenate([np.arange(cu[b], cu[b + 1]) for b in rows])
        c = np.concatenate([[0], np.cumsum([cu[b + 1] - cu[b] for b in rows])]).astype(np.int32)
        got = run_score(B, cache, qd[torch.from_numpy(sel).cuda()].contiguous(), lse[sel], had, c, lens[rows], table[rows], workspace=ws)
        br.assert_score(got, br.score(kv, q[sel], lse[sel], had, c, lens[rows], table[rows], page, D ** -0.5, True, 0, False), had)


def test_evict_does_not_trust_its_lists(B):
    """Pages outside the cache on either side, lengths past the table, past max_kv, negative ones."""
    rng = np.random.default_rng(4)
    hkv, D, page, budget = 2, 64, 16, 40
    arrays, lens, table, out_table = evict_case(rng, [100, 64, 90, 48], hkv, D, page, budget, 4)
    table[0, 1], table[0, 3], table[1, :], table[2, 5], out_table[2, 1], out_table[3, 0] = -1, 10 ** 6, -2 ** 31, 2 ** 31 - 1, -3, 10 ** 8
    score = scores_for(rng, "odd", (arrays[0].shape[0], hkv, page))
    got = run_evict(B, make_cache(B, arrays, 4), score, lens, table, out_table, budget, 2, 5)
    assert_evicted(got, br.evict(arrays, score, lens, table, out_table, budget, 2, 5))
    told = np.array([10 ** 9, 64, -7, 48], np.int32)
    eff = np.array([table.shape[1] * page, 64, 0, 48])
    got = run_evict(B, make_cache(B, arrays, 4), score, told, table, out_table, budget, 2, 5, max_kv=10 ** 6)
    assert_evicted(got, br.evict(arrays, score, eff, table, out_table, budget, 2, 5))
    for max_kv in (0, 10 ** 6):                             # no token at all
        empty = np.zeros(4, np.int32)
        got = run_evict(B, make_cache(B, arrays, 4), score, empty, table, out_table, budget, 2, 5, max_kv=max_kv)
        assert_evicted(got, br.evict(arrays, score, empty, table, out_table, budget, 2, 5))
    got = run_evict(B, make_cache(B, arrays, 4), score, lens, table, out_table, budget, 2, 5, max_kv=50)
    assert_evicted(got, br.evict(arrays, score, np.minimum(lens, 50), table, out_table, budget, 2, 5))


def test_evict_from_shared_pages(B):
    """Two sequences with a common prefix: its pages are read by both and stay as they are."""
    rng = np.random.default_rng(5)
    hkv, D, page, budget = 1, 128, 16, 20
    arrays, lens, table, out_table = evict_case(rng, [80, 60], hkv, D, page, budget, 8)
    table[1, :3] = table[0, :3]
    score = scores_for(rng, "sums", (arrays[0].shape[0], hkv, page))
    got = run_evict(B, make_cache(B, arrays, 8), score, lens, table, out_table, budget, 1, 2)
    assert_evicted(got, br.evict(arrays, score, lens, table, out_table, budget, 1, 2))


def test_offsets_past_four_gigabytes(B):
    """Codes and scores at either end of a pool of 4.3 GB per array."""
    import torch
    rng = np.random.default_rng(8)
    hq, hkv, D, page, L, budget = 4, 2, 128, 256, 500, 300
    pages = (1 << 32) // (page * D * hkv) + 1000
    cache = B.PagedCache(pages, page, hkv, D, bits=8)
    ids, out_ids = np.array([[pages - 1, 3]], np.int32), np.array([[5, pages - 2]], np.int32)
    X = to_dev(ref.bf16_values(rng, L, 2 * hkv * D)[0], "bf16")
    t = np.arange(L)
    B.batq_kv_paged_append(cache, X[:, : hkv * D], X[:, hkv * D:], dev(ids[0].astype(np.int64)[t // page] * page + t % page))
    both = torch.tensor(np.concatenate([ids[0], out_ids[0]]).astype(np.int64), device="cuda")
    score = torch.zeros((pages, hkv, page), device="cuda")
    qbits, q = ref.bf16_values(rng, 2, hq * D)
    lse, cu, lens = torch.empty((2, hq), device="cuda"), np.array([0, 2], np.int32), np.array([L], np.int32)
    small = [a[both].cpu().numpy() for a in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    B.batq_paged_attention(cache, to_dev(qbits, "bf16"), dev(cu), dev(lens), dev(ids), 2, L, lse=lse)
    B.batq_kv_paged_score(cache, to_dev(qbits, "bf16"), lse, score, dev(cu), dev(lens), dev(ids), 2, L)
    had = np.zeros((4, hkv, page), np.float32)
    got = score[both].cpu().numpy()
    br.assert_score(got, br.score(br.values(*small[:2], 8), q.reshape(2, hq, D).astype(np.float64), lse.cpu().numpy(), had, cu, lens,
                                  np.array([[0, 1]]), page, D ** -0.5, True, 0, False), had)
    keep, new_len = B.batq_kv_paged_evict(cache, score, dev(lens), dev(ids), dev(out_ids), L, budget, 4, 50)
    torch.cuda.synchronize()
    after = [a[both].cpu().numpy() for a in (cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales)]
    want = br.evict(small, got, lens, np.array([[0, 1]]), np.array([[2, 3]]), budget, 4, 50)
    assert_evicted((after, score[both].cpu().numpy(), keep.cpu().numpy(), new_len.cpu().numpy()), want)


def test_repeatable_on_streams_and_in_graphs(B):
    """Same bits on another stream with a workspace full of anything, and from replays of a graph of score and eviction with eager work
    and other lengths in between."""
    import torch
    rng = np.random.default_rng(9)
    hq, hkv, D, page, budget = 8, 2, 128, 16, 256
    lens0 = [3000, 700, 90]
    arrays, lens, table, out_table = evict_case(rng, lens0, hkv, D, page, budget, 4)
    cu, T = np.array([0, 300, 301, 303], np.int32), 303
    qd = to_dev(ref.bf16_values(rng, T, hq * D)[0], "bf16")
    dlens, dtable, dout, dcu = dev(lens), dev(table), dev(out_table), dev(cu)
    cache = make_cache(B, arrays, 4)
    had = dev(rng.uniform(0, 1, (arrays[0].shape[0], hkv, page)).astype(np.float32))
    lse = torch.empty((T, hq), device="cuda")
    ws1 = torch.full((max(256, B.batq_kv_paged_score_workspace(cache, hq, 3, T, 300, 3000)),), 0xFF, dtype=torch.uint8, device="cuda")
    ws2 = torch.full((max(256, B.batq_kv_paged_evict_workspace(cache, 3, 3000, budget)),), 0xFF, dtype=torch.uint8, device="cuda")

    def step(score, keep, new_len):
        B.batq_paged_attention(cache, qd, dcu, dlens, dtable, 300, 3000, lse=lse)
        B.batq_kv_paged_score(cache, qd, lse, score, dcu, dlens, dtable, 300, 3000, add=True, workspace=ws1)
        B.batq_kv_paged_evict(cache, score, dlens, dtable, dout, 3000, budget, 4, 16, keep=keep, new_len=new_len, workspace=ws2)

    def fresh():
        return had.clone(), torch.zeros((3, hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")

    want = fresh()
    step(*want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = fresh()
    with torch.cuda.stream(side):
        side.wait_stream(torch.cuda.default_stream())
        step(*got)
    side.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(got, want))
    g, held = torch.cuda.CUDAGraph(), fresh()
    with torch.cuda.graph(g, stream=side):
        step(*held)
    for rep in range(3):
        dlens.copy_(torch.tensor([3000 - 500 * rep, 700 - rep, 90 - rep], dtype=torch.int32))
        want = fresh()
        step(*want)
        codes = host(cache)
        junk = torch.randn(300, 300, device="cuda") @ torch.randn(300, 300, device="cuda")
        held[0].copy_(had)
        held[1].fill_(-5)
        ws1.fill_(0x7F), ws2.fill_(0x7F)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(held, want)), rep
        assert all(np.array_equal(x, y) for x, y in zip(codes, host(cache)))
        assert bool(torch.isfinite(junk).all())


def test_two_evictions_and_scores_at_once(B):
    """Calls on two streams with caches and workspaces of their own do not meet."""
    import torch
    rng = np.random.default_rng(10)
    hq, hkv, D, page, budget = 4, 1, 64, 16, 100
    sides = []
    for lens in ([4000, 50], [130, 2222, 700]):
        arrays, lens, table, out_table = evict_case(rng, lens, hkv, D, page, budget, 4)
        n = len(lens)
        cu = np.arange(0, 40 * n + 1, 40).astype(np.int32)
        score = scores_for(rng, "sums", (arrays[0].shape[0], hkv, page))
        sides.append((make_cache(B, arrays, 4), to_dev(ref.bf16_values(rng, 40 * n, hq * D)[0], "bf16"), torch.zeros((40 * n, hq), device="cuda"),
                      dev(score), dev(cu), dev(lens), dev(table), dev(out_table), int(max(lens)), torch.cuda.Stream()))

    def run(s):
        score = s[3].clone()
        B.batq_kv_paged_score(s[0], s[1], s[2], score, s[4], s[5], s[6], 40, s[8], add=True)
        return (score,) + B.batq_kv_paged_evict(s[0], score, s[5], s[6], s[7], s[8], budget, 1, 10)

    want = [run(s) for s in sides]
    torch.cuda.synchronize()
    for rep in range(3):
        got = []
        for s in sides:
            with torch.cuda.stream(s[9]):
                got.append([run(s) for _ in range(3)][-1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b)), rep


def test_binding_refuses_what_does_not_fit(B):
    import torch
    cache = B.PagedCache(6, 16, 2, 64, bits=4)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q, lse = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 4), device="cuda")
    score = torch.zeros((6, 2, 16), device="cuda")
    good = (cache, q, lse, score, i32(0, 3), i32(5), i32(0, 1).view(1, 2), 3, 5)
    B.batq_kv_paged_score(*good)
    for k, bad in ((1, q.float()), (1, q.cpu()), (2, lse[:2]), (2, lse.double()), (3, score[:5]), (3, score.half()), (3, score.cpu()),
                   (4, i32(0, 3).long()), (5, i32(5).cpu()), (6, i32(0, 1))):
        with pytest.raises(ValueError):
            B.batq_kv_paged_score(*good[:k], bad, *good[k + 1:])
    good = (cache, score, i32(25), i32(0, 1).view(1, 2), i32(2).view(1, 1), 32, 10)
    B.batq_kv_paged_evict(*good)
    for k, bad in ((1, score[:5]), (2, i32(5).long()), (3, i32(0, 1)), (4, i32(2))):
        with pytest.raises(ValueError):
            B.batq_kv_paged_evict(*good[:k], bad, *good[k + 1:])
    with pytest.raises(B.BatqError):
        B.batq_kv_paged_evict(*good, first=6, last=5)       # more than the budget
    with pytest.raises(B.BatqError):
        B.batq_kv_paged_evict(*good[:-1], 30)               # out_table has room for 16
    with pytest.raises(B.BatqError):
        B.batq_kv_paged_evict(*good, new_len=good[2])
    with pytest.raises(ValueError):
        B.batq_kv_paged_evict(*good, keep=torch.zeros((1, 2, 9), dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        B.PagedCache(6, 16, 2, 64, tensors=[cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales])    # 8 bits


# ---------------------------------------------------------------------------------------- together
@pytest.mark.parametrize("bits", [4, 8])
def test_decoding_within_a_budget(B, bits):
    """Two prompts are appended, attended and scored, cut down to a budget, and decoded on: append, attention, score a step, an
    eviction into fresh pages whenever a sequence has grown by half of the budget.  Every call is checked against its statement on what
    the cache holds then."""
    import torch
    rng = np.random.default_rng(12)
    hq, hkv, D, page, budget, first, last = 4, 2, 64, 16, 32, 2, 8
    pages, width = 24, 6
    cache = B.PagedCache(pages, page, hkv, D, bits=bits)
    score = torch.full((pages, hkv, page), 1e9, device="cuda")        # whatever the pages' last owners have left
    G, P = (np.eye(4) + 0.05 * rng.standard_normal((4, 4))).astype(np.float32), (np.eye(8) + 0.05 * rng.standard_normal((hkv * D // 32, 8, 8))).astype(np.float32)
    tk = B.Transform(hkv * D, G, P, None)
    rope = dev(ref.rope_table(400, D))
    free = list(rng.permutation(pages))
    table = np.full((2, width), -1, np.int32)
    lens, pos = np.zeros(2, np.int64), np.zeros(2, np.int64)

    def grow(n):
        for b in range(2):
            for i in range(-(-int(lens[b] + n[b]) // page)):
                if table[b, i] < 0:
                    table[b, i] = free.pop()

    def step(n):
        """n[b] new tokens of each sequence."""
        nonlocal lens, pos
        grow(n)
        M = int(sum(n))
        X = to_dev(ref.bf16_values(rng, M, (hq + 2 * hkv) * D)[0], "bf16")
        q, k, v = X.split((hq * D, hkv * D, hkv * D), 1)
        at = np.concatenate([lens[b] + np.arange(n[b]) for b in range(2)])
        owner = np.repeat([0, 1], n)
        slots = table[owner, at // page].astype(np.int64) * page + at % page
        p = np.concatenate([pos[b] + np.arange(n[b]) for b in range(2)]).astype(np.int32)
        qr = B.batq_kv_paged_append(cache, k, v, dev(slots), dev(p), q=q, rope=rope, tk=tk)
        lens, pos = lens + n, pos + n
        cu, l32 = np.array([0, n[0], M], np.int32), lens.astype(np.int32)
        lse = torch.empty((M, hq), device="cuda")
        had = score.cpu().numpy()
        out = B.batq_paged_attention(cache, qr, dev(cu), dev(l32), dev(table), max(n), width * page, lse=lse)
        B.batq_kv_paged_score(cache, qr, lse, score, dev(cu), dev(l32), dev(table), max(n), width * page, add=True)
        torch.cuda.synchronize()
        arrays = host(cache)
        kv, vv = br.values(*arrays[:2], bits), br.values(*arrays[2:], bits)
        qf = y_to_f32(qr).astype(np.float64).reshape(M, hq, D)
        want = ref.attention(kv, vv, qf, cu, l32, table, page, D ** -0.5, True, 0, M)
        ref.assert_attention(y_to_f32(out).astype(np.float64).reshape(M, hq, D), lse.cpu().numpy().astype(np.float64), want)
        got = score.cpu().numpy()
        br.assert_score(got, br.score(kv, qf, lse.cpu().numpy(), had, cu, l32, table, page, D ** -0.5, True, 0, True), had)

    def evict():
        nonlocal lens
        kept = np.minimum(lens, budget)
        out_table = np.full((2, budget // page), -1, np.int32)
        for b in range(2):
            out_table[b, : -(-int(kept[b]) // page)] = [free.pop() for _ in range(-(-int(kept[b]) // page))]
        before, had = host(cache), score.cpu().numpy()
        keep, new_len = B.batq_kv_paged_evict(cache, score, dev(lens.astype(np.int32)), dev(table), dev(out_table), width * page, budget, first, last)
        torch.cuda.synchronize()
        assert_evicted((host(cache), score.cpu().numpy(), keep.cpu().numpy(), new_len.cpu().numpy()),
                       br.evict(before, had, lens, table, out_table, budget, first, last))
        free.extend(int(x) for x in table[table >= 0])
        table[...] = -1
        table[:, : budget // page] = out_table
        lens = new_len.cpu().numpy().astype(np.int64)

    step([70, 25])
    evict()
    assert list(lens) == [32, 25]
    for i in range(40):
        step([1, 1])
        if max(lens) >= budget + 16:
            evict()
    assert list(pos) == [110, 65] and max(lens) < budget + 16


def test_a_prefix_that_is_shared_scored_and_evicted(B):
    """Two sequences decode behind one prompt whose pages they share, each with scores of its own, and are cut down to a budget: as two
    sequences with copies of those pages, bit for bit."""
    import torch
    rng = np.random.default_rng(51)
    hq, hkv, D, page, budget = 8, 2, 128, 16, 96
    L = [330, 300]
    arrays, lens, table, out_table = evict_case(rng, L, hkv, D, page, budget, 4)
    pages = arrays[0].shape[0]
    shared, n = table.copy(), 256 // page
    shared[1, :n] = table[0, :n]
    for a in arrays:
        a[table[1, :n]] = a[table[0, :n]]                   # (sequence 1's own pages hold the copies; their scores are its own in both runs)
    results = []
    for t, st in ((table, None), (shared, table)):
        cache, score = make_cache(B, arrays, 4), torch.zeros((pages, hkv, page), device="cuda")
        kw = {} if st is None else dict(score_table=dev(st))
        r = np.random.default_rng(52)
        for step, qn in enumerate([60, 1, 1, 1]):
            qd = to_dev(ref.bf16_values(r, 2 * qn, hq * D)[0], "bf16")
            cu, l32 = dev(np.array([0, qn, 2 * qn], np.int32)), dev(lens - 3 + step)
            lse = torch.empty((2 * qn, hq), device="cuda")
            B.batq_paged_attention(cache, qd, cu, l32, dev(t), qn, 330, lse=lse)
            B.batq_kv_paged_score(cache, qd, lse, score, cu, l32, dev(t), qn, 330, add=step > 0, **kw)
        keep, new_len = B.batq_kv_paged_evict(cache, score, l32, dev(t), dev(out_table), 330, budget, 2, 16, **kw)
        torch.cuda.synchronize()
        results.append([score, keep, new_len, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales])
    assert all(torch.equal(x, y) for x, y in zip(*results))
    assert not torch.equal(results[0][1][0], results[0][1][1])


def dirty(n, byte):
    import torch
    return torch.full((n,), byte, dtype=torch.uint8, device="cuda")


def test_long_sequences_in_graphs_with_workspaces_of_larger_calls(B):
    """Several workgroups to a (sequence, key head), whose histograms and counts are in the workspace: on another stream and replayed from
    a graph, with other scores and lengths, eager calls between the replays, and workspaces of larger calls full of anything; every
    replay against the statement."""
    import torch
    rng = np.random.default_rng(101)
    hkv, D, page, budget, first, last, most = 2, 64, 256, 1500, 3, 200, 40000
    arrays, lens, table, out_table = evict_case(rng, [most, 33000, 700], hkv, D, page, budget, 4)
    cache = make_cache(B, arrays, 4)
    need = B.batq_kv_paged_evict_workspace(cache, 3, most, budget)
    larger = B.batq_kv_paged_evict_workspace(cache, 5, 200000, budget)
    assert 0 < need < larger
    ws = dirty(larger, 0xFF)
    with pytest.raises(B.BatqError):                        # it is in use
        B.batq_kv_paged_evict(cache, dev(np.zeros((arrays[0].shape[0], hkv, page), np.float32)), dev(lens), dev(table), dev(out_table), most, budget,
                              workspace=dirty(256, 0))
    score, dlens = torch.zeros((arrays[0].shape[0], hkv, page), device="cuda"), dev(lens)
    keep, new_len = torch.zeros((3, hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    dtable, dout = dev(table), dev(out_table)

    def step(keep=keep, new_len=new_len):
        B.batq_kv_paged_evict(cache, score, dlens, dtable, dout, most, budget, first, last, keep=keep, new_len=new_len, workspace=ws)

    def restore(kind):
        x = scores_for(rng, kind, tuple(score.shape))
        for t, a in zip((cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales), arrays):
            t.copy_(dev(a))
        score.copy_(dev(x))
        keep.fill_(-5), new_len.fill_(-5)
        return x

    def result():
        return host(cache), score.cpu().numpy(), keep.cpu().numpy(), new_len.cpu().numpy()

    x = restore("sums")
    side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert_evicted(result(), br.evict(arrays, x, lens, table, out_table, budget, first, last))
    with torch.cuda.graph(g, stream=side):
        step()
    for rep, (kind, ls) in enumerate((("ties", [most, 33000, 700]), ("odd", [39000, 1499, 700]), ("same", [36000, 32768, 0]), ("sums", [33000, 8193, 1]))):
        x = restore(kind)
        dlens.copy_(torch.tensor(ls, dtype=torch.int32))
        ws.fill_(0x7F + rep)
        g.replay()
        torch.cuda.synchronize()
        got = result()
        assert_evicted(got, br.evict(arrays, x, np.array(ls), table, out_table, budget, first, last))
        score.copy_(dev(x))
        step(torch.empty_like(keep), torch.empty_like(new_len))      # eager, between the replays
        torch.cuda.synchronize()


def test_calls_at_once_that_use_their_workspaces(B):
    """Scores whose rows are cut into parts and evictions of long sequences, on two streams with dirty workspaces of their own."""
    import torch
    rng = np.random.default_rng(111)
    hq, hkv, D, page, budget = 8, 1, 64, 64, 600
    sides = []
    for lens, qn in (([40000, 50], 400), ([35000, 33100, 900], 300)):
        arrays, lens, table, out_table = evict_case(rng, lens, hkv, D, page, budget, 4)
        n, L = len(lens), int(max(lens))
        cu = np.arange(0, qn * n + 1, qn).astype(np.int32)
        cache = make_cache(B, arrays, 4)
        sizes = B.batq_kv_paged_score_workspace(cache, hq, n, qn * n, qn, L), B.batq_kv_paged_evict_workspace(cache, n, L, budget)
        assert min(sizes) > 0
        sides.append(dict(cache=cache, q=to_dev(ref.bf16_values(rng, qn * n, hq * D)[0], "bf16"), lse=torch.full((qn * n, hq), 9.0, device="cuda"),
                          had=dev(scores_for(rng, "sums", (arrays[0].shape[0], hkv, page))), cu=dev(cu), lens=dev(lens), table=dev(table), out=dev(out_table),
                          qn=qn, L=L, ws=[dirty(s, 0xFF) for s in sizes], stream=torch.cuda.Stream()))
    small = dirty(256, 0)

    def run(s, ws=None):
        score, ws = s["had"].clone(), ws or s["ws"]
        B.batq_kv_paged_score(s["cache"], s["q"], s["lse"], score, s["cu"], s["lens"], s["table"], s["qn"], s["L"], add=True, workspace=ws[0])
        return (score,) + B.batq_kv_paged_evict(s["cache"], score, s["lens"], s["table"], s["out"], s["L"], budget, 1, 10, workspace=ws[1])

    for s in sides:                                         # both calls take of their workspaces
        with pytest.raises(B.BatqError):
            run(s, [small, s["ws"][1]])
        with pytest.raises(B.BatqError):
            run(s, [s["ws"][0], small])
    torch.cuda.synchronize()
    want = [run(s) for s in sides]
    torch.cuda.synchronize()
    for rep in range(3):
        got = []
        for s in sides:
            for w in s["ws"]:
                w.fill_(0x55 + rep)
            s["stream"].wait_stream(torch.cuda.current_stream())
        for s in sides:
            with torch.cuda.stream(s["stream"]):
                got.append([run(s) for _ in range(3)][-1])
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for a, b in zip(got, want) for x, y in zip(a, b)), rep


def test_plain_entry_points_are_those_of_eight_bits(B):
    """batq_kv_paged_append and batq_paged_attention as a C program calls them (the binding takes the forms with a width), and
    batq_kv_paged_score and batq_kv_paged_evict without a table of score pages: the bits of the others."""
    import ctypes as C
    import torch
    from paper_2603_16590_amd.binding import _PagedBatch
    rng = np.random.default_rng(121)
    hq, hkv, D, page, budget = 4, 2, 128, 16, 50
    lens, qs = [300, 77], [40, 1]
    arrays, lens, table, out_table = evict_case(rng, lens, hkv, D, page, budget, 8)
    cu, T = np.array([0, 40, 41], np.int32), 41
    X = to_dev(ref.bf16_values(rng, T, (hq + 2 * hkv) * D)[0], "bf16")
    q, k, v = X.split((hq * D, hkv * D, hkv * D), 1)
    at = np.concatenate([lens[b] - qs[b] + np.arange(qs[b]) for b in range(2)])
    owner = np.repeat([0, 1], qs)
    slots = dev(table[owner, at // page].astype(np.int64) * page + at % page)
    dcu, dlens, dtable, dout = dev(cu), dev(lens), dev(table), dev(out_table)
    shape = (arrays[0].shape[0], hkv, page)
    stream = torch.cuda.current_stream().cuda_stream
    results = []
    for plain in (False, True):
        cache = make_cache(B, arrays, 8)
        q_out, out = (torch.zeros((T, hq * D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lse, score = torch.zeros((T, hq), device="cuda"), torch.zeros(shape, device="cuda")
        keep, new_len = torch.zeros((2, hkv, budget), dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
        n = [B.batq_paged_attention_workspace(cache, hq, 2, T, 40, 300), B.batq_kv_paged_score_workspace(cache, hq, 2, T, 40, 300),
             B.batq_kv_paged_evict_workspace(cache, 2, 300, budget)]
        ws = dirty(max(n) + 256, 0xFF)
        if plain:
            c, b = C.byref(cache._d), C.byref(_PagedBatch(dcu.data_ptr(), dlens.data_ptr(), dtable.data_ptr(), 2, table.shape[1], T, 40, 300))
            w = (ws.data_ptr(), ws.numel(), stream)
            assert B.lib.batq_kv_paged_append(c, None, None, None, q.data_ptr(), q.stride(0), hq, q_out.data_ptr(), hq * D, k.data_ptr(), k.stride(0),
                                              v.data_ptr(), v.stride(0), B.BF16, None, slots.data_ptr(), T, stream) == 0
            assert B.lib.batq_paged_attention(c, b, q_out.data_ptr(), hq * D, hq, D ** -0.5, 1, 0, out.data_ptr(), hq * D, lse.data_ptr(), *w) == 0
            assert B.lib.batq_kv_paged_score(c, 8, b, q_out.data_ptr(), hq * D, hq, D ** -0.5, 1, 0, lse.data_ptr(), score.data_ptr(), 0, *w) == 0
            assert B.lib.batq_kv_paged_evict(c, 8, score.data_ptr(), dlens.data_ptr(), dtable.data_ptr(), table.shape[1], dout.data_ptr(), out_table.shape[1],
                                             2, 300, budget, 2, 5, keep.data_ptr(), new_len.data_ptr(), *w) == 0
        else:
            B.batq_kv_paged_append(cache, k, v, slots, q=q, q_out=q_out)
            B.batq_paged_attention(cache, q_out, dcu, dlens, dtable, 40, 300, out=out, lse=lse, workspace=ws)
            B.batq_kv_paged_score(cache, q_out, lse, score, dcu, dlens, dtable, 40, 300, workspace=ws)
            B.batq_kv_paged_evict(cache, score, dlens, dtable, dout, 300, budget, 2, 5, keep=keep, new_len=new_len, workspace=ws)
        torch.cuda.synchronize()
        results.append([q_out, out, lse, score, keep, new_len, cache.k_codes, cache.k_scales, cache.v_codes, cache.v_scales])
    assert all(torch.equal(x, y) for x, y in zip(*results))
    assert bool((results[0][4] >= 0).any()) and bool((results[0][1] != 0).any())


@pytest.mark.parametrize("L,alias", [(500, "new_len"), (40000, "new_len"), (40000, "workspace"), (500, "score")])
def test_evict_stays_within_its_arrays(B, L, alias):
    """Lists, lengths, scores and workspace that lie on each other make what is kept unspecified; nothing but the pages of out_table, and
    what is handed over to be written, is written to."""
    import torch
    rng = np.random.default_rng(131 + L)
    hkv, D, page, budget = 2, 64, 64, 1024 if L > 1000 else 192
    arrays, lens, table, out_table = evict_case(rng, [L, L], hkv, D, page, budget, 4)
    cache, pages = make_cache(B, arrays, 4), arrays[0].shape[0]
    need = B.batq_kv_paged_evict_workspace(cache, 2, L, budget)
    size = 2 * hkv * budget
    words = max(pages * hkv * page, 4 * need, 8 * size)
    store = torch.full((words + 2048,), 12345678, dtype=torch.int32, device="cuda")
    at = 1024                                               # (4 KiB: the workspace's alignment)
    score = store[at: at + pages * hkv * page].view(torch.float32).view(pages, hkv, page)
    score.copy_(dev(scores_for(rng, "sums", tuple(score.shape))))
    keep = torch.full((size + 2048,), 12345678, dtype=torch.int32, device="cuda")
    kept = keep[1024: 1024 + size].view(2, hkv, budget)
    new_len, ws = torch.zeros(2, dtype=torch.int32, device="cuda"), dirty(max(need, 256), 0xFF)
    if alias == "new_len":
        new_len = kept.view(-1)[budget - 1: budget + 1]     # in the middle of the lists
    elif alias == "workspace":
        ws = store[at: at + need // 4].view(torch.uint8)
        assert need <= score.nbytes
    else:
        kept = store[at: at + size].view(2, hkv, budget)
    B.batq_kv_paged_evict(cache, score, dev(lens), dev(table), dev(out_table), L, budget, 2, 5, keep=kept, new_len=new_len, workspace=ws)
    torch.cuda.synchronize()
    assert bool((store[:at] == 12345678).all()) and bool((store[at + pages * hkv * page:] == 12345678).all())
    assert bool((keep[:1024] == 12345678).all()) and bool((keep[1024 + size:] == 12345678).all())
    rest = np.setdiff1d(np.arange(pages), out_table)
    for got, a in zip(host(cache), arrays):
        assert np.array_equal(got[rest], a[rest])
