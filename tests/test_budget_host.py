"""Refusals of the calls on caches of 4 bits, of scores and of eviction: every argument is looked at on the host, before any device is
touched."""
import ctypes as C

import numpy as np
import pytest

import budget_ref as br
from oracle import batq_oracle as o
from test_serving_host import Batch, P, cache


@pytest.fixture(scope="module")
def B():
    import paper_2603_16590_amd as b
    return b


def test_sizes(B):
    f = B.lib.batq_kv_paged_code_bytes_ex
    assert f(4, 16, 2, 64, 4) == 4 * 16 * 2 * 32 and f(4, 16, 2, 64, 8) == 4 * 16 * 2 * 64
    assert f(1 << 20, 256, 8, 128, 4) == 1 << 37
    for bad in ((4, 16, 2, 64, 5), (4, 16, 2, 64, 0), (4, 16, 2, 96, 4), (4, 24, 2, 64, 4), (0, 16, 2, 64, 4)):
        assert f(*bad) == 0


def test_widths_other_than_4_and_8_are_refused(B):
    c = cache()
    for bits in (0, 2, 6, 16, -4):
        assert B.lib.batq_kv_paged_append_ex(C.byref(c), bits, None, None, None, None, 0, 0, None, 0, P, 128, P, 128, 1, None, P, 4, None) == 4
        assert attend(B, c, bits) == 4 and score(B, c, bits=bits) == 4 and evict(B, c, bits=bits) == 4
    assert B.lib.batq_kv_paged_append_ex(C.byref(c), 4, None, None, None, None, 0, 0, None, 0, P, 120, P, 128, 1, None, P, 4, None) == 2
    assert B.lib.batq_kv_paged_append_ex(C.byref(c), 4, None, None, None, None, 0, 0, None, 0, None, 128, None, 128, 1, None, None, 0, None) == 0


def attend(B, c, bits):
    b = Batch(cu_q=P, kv_len=P, page_table=P, batch=2, table_width=3, total_q=5, max_q=4, max_kv=48)
    return B.lib.batq_paged_attention_ex(C.byref(c), bits, C.byref(b), P, 256, 4, 0.1, 1, 0, 2 * P, 256, None, None, 0, None)


def score(B, c, bits=4, q=P, ldq=256, q_heads=4, scale=0.1, window=0, lse=P, out=P, ws=None, wsb=0, **kw):
    b = Batch(**{**dict(cu_q=P, kv_len=P, page_table=P, batch=2, table_width=3, total_q=5, max_q=4, max_kv=48), **kw})
    return B.lib.batq_kv_paged_score(C.byref(c) if c is not None else None, bits, C.byref(b), q, ldq, q_heads, scale, 1, window, lse, out, 0,
                                     ws, wsb, None)


def test_score_refusals(B):
    ok = cache()
    assert score(B, None) == 1
    assert B.lib.batq_kv_paged_score(C.byref(ok), 4, None, P, 256, 4, 0.1, 1, 0, P, P, 0, None, 0, None) == 1
    assert score(B, cache(head_dim=32)) == 4 and score(B, cache(page_size=0)) == 2 and score(B, cache(k_codes=None)) == 1
    for kw, want in ((dict(q_heads=3), 2), (dict(q_heads=0), 2), (dict(q_heads=2 * 130), 2), (dict(ldq=255), 2), (dict(ldq=260), 2),
                     (dict(batch=-1), 2), (dict(total_q=-1), 2), (dict(max_q=-1), 2), (dict(max_kv=-1), 2), (dict(table_width=-1), 2),
                     (dict(window=-1), 2), (dict(scale=0.0), 2), (dict(scale=float("nan")), 2), (dict(scale=float("inf")), 2),
                     (dict(q=None), 1), (dict(lse=None), 1), (dict(out=None), 1), (dict(cu_q=None), 1), (dict(kv_len=None), 1),
                     (dict(page_table=None), 1), (dict(q=P + 2), 2), (dict(cu_q=P + 2), 2), (dict(lse=P + 1), 2), (dict(out=P + 2), 2),
                     (dict(ws=P + 16), 2), (dict(total_q=1 << 30), 2), (dict(batch=1 << 17, max_kv=1 << 15), 2)):
        assert score(B, ok, **kw) == want, kw
    for kw in (dict(batch=0), dict(max_kv=0), dict(table_width=0)):
        assert score(B, ok, **{**kw, "q": None, "lse": None, "out": None}) == 0
    assert B.lib.batq_kv_paged_score_workspace(None, 4, 1, 1, 1, 100) == 0


def evict(B, c, bits=4, score=P, kv_len=P, table=P, width=3, out=2 * P, out_width=2, batch=2, max_kv=48, budget=20, first=1, last=2, keep=P,
          new_len=2 * P, ws=None, wsb=0):
    return B.lib.batq_kv_paged_evict(C.byref(c) if c is not None else None, bits, score, kv_len, table, width, out, out_width, batch, max_kv,
                                     budget, first, last, keep, new_len, ws, wsb, None)


def test_evict_refusals(B):
    ok = cache()
    assert evict(B, None) == 1
    assert evict(B, cache(head_dim=32)) == 4 and evict(B, cache(page_size=0)) == 2 and evict(B, cache(v_scales=None)) == 1
    for kw, want in ((dict(batch=-1), 2), (dict(max_kv=-1), 2), (dict(budget=0), 2), (dict(first=-1), 2), (dict(last=-1), 2),
                     (dict(first=10, last=11), 2), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), 2), (dict(width=-1), 2), (dict(out_width=-1), 2),
                     (dict(out_width=1), 2), (dict(budget=40), 2), (dict(score=None), 1), (dict(kv_len=None), 1), (dict(table=None), 1),
                     (dict(out=None), 1), (dict(keep=None), 1), (dict(new_len=None), 1), (dict(score=P + 2), 2), (dict(kv_len=P + 1), 2),
                     (dict(table=P + 2), 2), (dict(out=P + 2), 2), (dict(keep=P + 2), 2), (dict(new_len=P + 2), 2), (dict(new_len=P), 2),
                     (dict(out=P), 2), (dict(new_len=P + 4), 2), (dict(new_len=P - 4), 2), (dict(ws=P + 128), 2), (dict(batch=1 << 20, max_kv=8192 * 2), 2), (dict(batch=1 << 20, max_kv=1 << 20, budget=1 << 20), 2)):
        assert evict(B, ok, **kw) == want, kw
    assert evict(B, ok, batch=0, score=None, kv_len=None, table=None, out=None, keep=None, new_len=None) == 0
    assert B.lib.batq_kv_paged_evict_workspace(None, 1, 100, 10) == 0


def test_statements_of_the_tests():
    """The helpers' values of 4-bit codes are the oracle's, and an eviction's statement keeps what a sort keeps."""
    rng = np.random.default_rng(0)
    codes, scales = br.random_arrays(rng, 3, 16, 2, 64, 4)[:2]
    v = br.values(codes, scales, 4)
    want = o.dequantize(codes.reshape(-1, 32), scales.transpose(0, 1, 3, 2).reshape(-1, 2))
    assert np.array_equal(v.reshape(-1, 64), want)
    arrays = br.random_arrays(rng, 6, 16, 1, 64, 8)
    s = rng.standard_normal((6, 1, 16)).astype(np.float32)
    table, out = np.array([[2, 0, 5]]), np.array([[1, 3]])
    _, sc, keep, n = br.evict(arrays, s, [40], table, out, 20, 2, 3)
    flat = s[table[0], 0].reshape(-1)[:40]
    chosen = set(np.argsort(-flat[2:37])[:15] + 2) | {0, 1, 37, 38, 39}
    assert n[0] == 20 and set(keep[0, 0]) == chosen and np.array_equal(sc[out[0], 0].reshape(-1)[:20], flat[keep[0, 0]])


def test_budgets_past_two_to_the_thirty_are_refused(B):
    """A list's places are counted in 32 bits, 1024 at a time: behind 2^31 - 1 - 1024 they would wrap to places before the list."""
    ok = cache()
    for budget in ((1 << 30) + 1, 2 ** 31 - 1024, 2 ** 31 - 1):
        assert evict(B, ok, budget=budget, out_width=3) == 2 and evict(B, ok, budget=budget, out_width=3, batch=0) == 2
        assert B.lib.batq_kv_paged_evict_workspace(C.byref(ok), 2, 1 << 20, budget) == 0
    assert evict(B, ok, budget=1 << 30, out_width=3, batch=0) == 0


def test_score_tables_are_looked_at(B):
    ok = cache()
    b = Batch(cu_q=P, kv_len=P, page_table=P, batch=2, table_width=3, total_q=5, max_q=4, max_kv=48)

    def score_ex(table, pages, **kw):
        bb = Batch(**{**{n: getattr(b, n) for n, _ in Batch._fields_}, **kw})
        return B.lib.batq_kv_paged_score_ex(C.byref(ok), 4, C.byref(bb), P, 256, 4, 0.1, 1, 0, P, P, table, pages, 0, None, 0, None)

    def evict_ex(table, pages, batch=2, out=2 * P):
        return B.lib.batq_kv_paged_evict_ex(C.byref(ok), 4, P, table, pages, P, P, 3, out, 2, batch, 48, 20, 1, 2, P, 2 * P, None, 0, None)

    for f in (score_ex, evict_ex):
        for table in (None, 3 * P):
            assert f(table, ok.num_pages - 1) == 2 and f(table, 0) == 2 and f(table, -1) == 2
            assert f(table, ok.num_pages, batch=0) == 0 and f(table, 2 ** 31 - 1, batch=0) == 0
        assert f(3 * P + 2, ok.num_pages) == 2
    assert evict_ex(2 * P, ok.num_pages) == 2               # the table that the tokens move to
    assert B.lib.batq_kv_paged_score_ex(None, 4, C.byref(b), P, 256, 4, 0.1, 1, 0, P, P, None, 4, 0, None, 0, None) == 1
    assert B.lib.batq_kv_paged_evict_ex(None, 4, P, None, 4, P, P, 3, 2 * P, 2, 2, 48, 20, 1, 2, P, 2 * P, None, 0, None) == 1


def test_numbers_past_32_bits_are_not_cut(B):
    """2^32 + 5 is no bound of 5, and a window of 2^32 is not none."""
    import torch
    q, table, far = torch.zeros((1, 64)), torch.zeros((1, 2), dtype=torch.int32), (1 << 32) + 5
    for kw in (dict(max_q=far, max_kv=5), dict(max_q=1, max_kv=far), dict(max_q=1, max_kv=5, window=1 << 32)):
        with pytest.raises(ValueError, match="2\\^31"):
            B.batq_paged_attention(None, q, None, None, table, **kw)
        with pytest.raises(ValueError, match="2\\^31"):
            B.batq_kv_paged_score(None, q, None, None, None, None, table, **kw)
    good = dict(max_kv=5, budget=4, first=1, last=1)
    for name in good:
        with pytest.raises(ValueError, match="2\\^31"):
            B.batq_kv_paged_evict(None, None, None, table, table, **{**good, name: far})
    for f, n in ((B.batq_paged_attention_workspace, 5), (B.batq_kv_paged_score_workspace, 5), (B.batq_kv_paged_evict_workspace, 3)):
        for i in range(n):
            with pytest.raises(ValueError, match="2\\^31"):
                f(None, *[far if k == i else 1 for k in range(n)])
