"""Refusals of the serving calls: every argument is looked at on the host, before any device is touched."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def B():
    import paper_2603_16590_amd as b
    return b


class Cache(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("num_pages", "page_size", "kv_heads", "head_dim")] + \
               [(n, C.c_void_p) for n in ("k_codes", "k_scales", "v_codes", "v_scales")]


class Rope(C.Structure):
    _fields_ = [("table", C.c_void_p)] + [(n, C.c_int) for n in ("positions", "rotary_dim", "interleaved")]


class Batch(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("cu_q", "kv_len", "page_table")] + \
               [(n, C.c_int) for n in ("batch", "table_width", "total_q", "max_q", "max_kv")]


P = 1 << 20                                                 # an aligned address that is never followed


def cache(**kw):
    return Cache(**{**dict(num_pages=4, page_size=16, kv_heads=2, head_dim=64, k_codes=P, k_scales=P, v_codes=P, v_scales=P), **kw})


def test_sizes(B):
    f, g = B.lib.batq_kv_paged_code_bytes, B.lib.batq_kv_paged_scale_bytes
    assert f(4, 16, 2, 64) == 4 * 16 * 2 * 64 and g(4, 16, 2, 64) == 4 * 16 * 2 * 2
    assert f(1 << 20, 256, 8, 128) == 1 << 38               # past 32 bits
    for bad in ((0, 16, 2, 64), (4, 8, 2, 64), (4, 24, 2, 64), (4, 512, 2, 64), (4, 16, 0, 64), (4, 16, 2, 96), (-1, 16, 2, 128)):
        assert f(*bad) == 0 and g(*bad) == 0
    w = B.lib.batq_lora_workspace
    assert w(4, 64, 64, 8, 1) % 4 == 0
    for bad in ((-1, 64, 64, 8, 1), (4, 48, 64, 8, 1), (4, 64, 0, 8, 1), (4, 64, 64, 12, 1), (4, 64, 64, 136, 1), (4, 64, 64, 8, 0)):
        assert w(*bad) == 0


def append(B, c, rope=None, q=None, ldq=0, q_heads=0, q_out=None, ldqo=0, k=P, ldk=128, v=P, ldv=128, dt=1, pos=P, slots=P, M=4, tk=None):
    return B.lib.batq_kv_paged_append(C.byref(c) if c is not None else None, tk, None, C.byref(rope) if rope is not None else None,
                                      q, ldq, q_heads, q_out, ldqo, k, ldk, v, ldv, dt, pos, slots, M, None)


def test_append_refusals(B):
    ok = cache()
    assert append(B, None) == 1
    for kw, want in ((dict(head_dim=96), 4), (dict(page_size=24), 2), (dict(num_pages=0), 2), (dict(kv_heads=0), 2),
                     (dict(k_codes=None), 1), (dict(v_scales=None), 1), (dict(k_scales=P + 8), 2)):
        assert append(B, cache(**kw)) == want, kw
    for kw, want in ((dict(dt=2), 3), (dict(M=-1), 2), (dict(ldk=127), 2), (dict(ldv=120), 2), (dict(k=None), 1), (dict(v=None), 1),
                     (dict(slots=None), 1), (dict(slots=P + 4), 2), (dict(k=P + 2), 2), (dict(ldk=132), 2),
                     (dict(q_heads=3), 2), (dict(q_heads=-2), 2), (dict(q=P, q_heads=0), 1),
                     (dict(q_heads=2, ldq=128, ldqo=128, q_out=P), 1), (dict(q_heads=2, ldq=128, ldqo=128, q=P), 1),
                     (dict(q_heads=2, ldq=120, ldqo=128, q=P, q_out=2 * P), 2), (dict(q_heads=2, ldq=128, ldqo=120, q=P, q_out=2 * P), 2),
                     (dict(q_heads=2, ldq=128, ldqo=128, q=P, q_out=P), 2), (dict(q_heads=2, ldq=128, ldqo=132, q=P, q_out=2 * P), 2)):
        assert append(B, ok, **kw) == want, kw
    for r, want in ((Rope(None, 10, 64, 0), 1), (Rope(P, 0, 64, 0), 2), (Rope(P, 10, 24, 0), 2), (Rope(P, 10, 80, 0), 2),
                    (Rope(P, 10, 0, 0), 2), (Rope(P + 4, 10, 64, 0), 2)):
        assert append(B, ok, rope=r) == want
    assert append(B, ok, rope=Rope(P, 10, 64, 0), pos=None) == 1
    assert append(B, ok, rope=Rope(P, 10, 64, 0), pos=P + 2) == 2
    assert append(B, ok, M=0, k=None, v=None, slots=None) == 0


def attend(B, c, q=P, ldq=256, q_heads=4, scale=0.1, window=0, out=2 * P, ldo=256, lse=None, ws=None, wsb=0, **kw):
    b = Batch(**{**dict(cu_q=P, kv_len=P, page_table=P, batch=2, table_width=3, total_q=5, max_q=4, max_kv=48), **kw})
    return B.lib.batq_paged_attention(C.byref(c) if c is not None else None, C.byref(b), q, ldq, q_heads, scale, 1, window, out, ldo,
                                      lse, ws, wsb, None)


def test_attention_refusals(B):
    ok = cache()
    assert attend(B, None) == 1
    assert B.lib.batq_paged_attention(C.byref(ok), None, P, 256, 4, 0.1, 1, 0, 2 * P, 256, None, None, 0, None) == 1
    assert attend(B, cache(head_dim=32)) == 4 and attend(B, cache(page_size=0)) == 2 and attend(B, cache(v_codes=None)) == 1
    for kw, want in ((dict(q_heads=3), 2), (dict(q_heads=0), 2), (dict(q_heads=2 * 130), 2), (dict(ldq=255), 2), (dict(ldo=200), 2),
                     (dict(ldq=260), 2), (dict(batch=-1), 2), (dict(total_q=-1), 2), (dict(max_q=-1), 2), (dict(max_kv=-1), 2),
                     (dict(table_width=-1), 2), (dict(window=-1), 2), (dict(scale=0.0), 2), (dict(scale=float("nan")), 2),
                     (dict(scale=float("inf")), 2), (dict(q=None), 1), (dict(out=None), 1), (dict(cu_q=None), 1), (dict(kv_len=None), 1),
                     (dict(page_table=None), 1), (dict(q=P + 2), 2), (dict(out=P), 2), (dict(cu_q=P + 2), 2), (dict(lse=P + 1), 2),
                     (dict(ws=P + 16), 2), (dict(total_q=1 << 30), 2)):
        assert attend(B, ok, **kw) == want, kw
    for kw in (dict(batch=0), dict(total_q=0), dict(max_q=0)):
        assert attend(B, ok, **{**kw, "q": None, "out": None}) == 0
    assert B.lib.batq_paged_attention_workspace(None, 4, 1, 1, 1, 100) == 0
    assert B.lib.batq_paged_attention_workspace(C.byref(ok), 3, 1, 1, 1, 100) == 0


def lora(B, X=P, xdt=1, M=4, K=64, ldx=64, A=P, Bm=P, N=40, rank=8, n=2, scales=P, index=P, base=P, ldb=40, out=2 * P, ldo=40, ydt=1, ws=P, wsb=1 << 20):
    return B.lib.batq_lora_add(X, xdt, M, K, ldx, A, Bm, N, rank, n, scales, index, base, ldb, out, ldo, ydt, ws, wsb, None)


def test_lora_refusals(B):
    for kw, want in ((dict(xdt=5), 3), (dict(ydt=-1), 3), (dict(M=-1), 2), (dict(K=48), 2), (dict(K=0), 2), (dict(N=0), 2), (dict(rank=4), 2),
                     (dict(rank=20), 2), (dict(rank=136), 2), (dict(n=0), 2), (dict(ldx=63), 2), (dict(ldx=68), 2), (dict(ldb=39), 2),
                     (dict(ldo=39), 2), (dict(X=None), 1), (dict(A=None), 1), (dict(Bm=None), 1), (dict(index=None), 1), (dict(out=None), 1),
                     (dict(X=P + 8), 2), (dict(A=P + 2), 2), (dict(Bm=P + 2), 2), (dict(index=P + 2), 2), (dict(scales=P + 2), 2),
                     (dict(out=P + 1), 2), (dict(base=P + 1), 2), (dict(ws=P + 64), 2), (dict(out=P), 2), (dict(base=2 * P, ldb=48), 2)):
        assert lora(B, **kw) == want, kw
    assert lora(B, M=0, X=None, A=None, Bm=None, index=None, out=None) == 0


def test_binding_refusals(B):
    torch = pytest.importorskip("torch")
    with pytest.raises(ValueError):
        B.PagedCache(4, 24, 2, 64)
    with pytest.raises(ValueError):
        B.batq_lora_add(torch.zeros(2, 64), torch.zeros(1, 8, 32).bfloat16(), torch.zeros(1, 4, 8).bfloat16(), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(ValueError):
        B.batq_lora_add(torch.zeros(2, 32), torch.zeros(1, 8, 32), torch.zeros(1, 4, 8).bfloat16(), torch.zeros(2, dtype=torch.int32))


def test_sizes_past_a_launch_are_refused(B):
    big = cache(kv_heads=4096)
    for kw in (dict(batch=128, q_heads=4096, ldq=1 << 18, ldo=1 << 18), dict(batch=100, q_heads=4096, ldq=1 << 18, ldo=1 << 18, max_kv=1 << 20),
               dict(batch=1, q_heads=4096, ldq=1 << 18, ldo=1 << 18, max_kv=1 << 30)):
        assert attend(B, big, **kw) == 2, kw
        assert B.lib.batq_paged_attention_workspace(C.byref(big), 4096, kw["batch"], 5, 4, kw.get("max_kv", 48)) == 0
    assert append(B, big, M=1 << 22, ldk=1 << 18, ldv=1 << 18) == 2
    for kw in (dict(M=(1 << 26) + 1), dict(K=(1 << 26) + 32, ldx=(1 << 26) + 32), dict(N=(1 << 26) + 1, ldb=(1 << 26) + 1, ldo=(1 << 26) + 1)):
        assert lora(B, **kw) == 2, kw
        assert B.lib.batq_lora_workspace(*[{**dict(M=4, K=64, N=40, rank=8, n=2), **kw}[k] for k in ("M", "K", "N", "rank", "n")]) == 0


def test_a_cache_does_not_keep_addresses_that_are_gone(B, monkeypatch):
    """Calls pass the addresses of a cache's arrays: it cannot be given others, and arrays whose memory has been moved or freed are refused."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(B.binding, "_device", lambda: -1)   # (the arrays are host memory here, which is device -1 to torch)
    shapes = ((4, 2, 16, 64), (4, 2, 2, 16)) * 2
    arrays = [torch.zeros(s, dtype=torch.uint8) for s in shapes]
    c = B.PagedCache(4, 16, 2, 64, tensors=arrays)
    assert c.k_codes is arrays[0] and c.v_scales is arrays[3] and (c.num_pages, c.page_size, c.kv_heads, c.head_dim) == (4, 16, 2, 64)
    d = c.desc(-1)._obj
    assert [d.k_codes, d.k_scales, d.v_codes, d.v_scales] == [t.data_ptr() for t in arrays]
    for name, value in (("k_codes", arrays[2]), ("k_scales", arrays[3]), ("v_codes", arrays[0]), ("v_scales", arrays[1]), ("num_pages", 8),
                        ("page_size", 32), ("kv_heads", 1), ("head_dim", 128), ("device", 0)):
        with pytest.raises(AttributeError):
            setattr(c, name, value)
    assert c.desc(-1)._obj.k_codes == arrays[0].data_ptr()
    for i in range(4):
        fresh = [torch.zeros(s, dtype=torch.uint8) for s in shapes]
        c = B.PagedCache(4, 16, 2, 64, tensors=fresh)
        c.desc(-1)
        if i % 2:
            fresh[i].untyped_storage().resize_(0)           # freed
        else:
            fresh[i].data = torch.zeros(shapes[i], dtype=torch.uint8)       # moved
        with pytest.raises(ValueError):
            c.desc(-1)


def test_scales_that_overflow_are_refused(B):
    """The kernels keep scores in units of ln 2: a scale whose product with log2 e is infinite would make a score of zero NaN."""
    for scale in (2.5e38, 2.9e38, 3.4e38):
        assert attend(B, cache(), scale=scale) == 2
    assert attend(B, cache(), scale=1.9e38, q=None) == 1    # (the next check)


def lora_parts(M, K, N):
    """Parts of K that a call of the adapters computes (each takes M x rank floats of its workspace)."""
    tiles, few = -(-M // 16), M <= 64
    least, most = (256, 8) if few else (4096 if N // 2 > K else 2048, 4)
    n = max(1, min(256 // tiles, -(-K // least), most))
    step = 256 if few and n > 1 else 512
    return -(-K // (-(-(-(-K // n)) // step) * step))


@pytest.mark.parametrize("K", [32, 256, 288, 608, 2048, 2080, 4096, 4128, 8192, 14336, 16384, 1 << 20])
def test_lora_workspace_of_the_largest_call_is_enough_for_smaller_ones(B, K):
    """A server sizes its workspace once: fewer rows, a shorter K or a smaller rank never ask for more."""
    w, before = B.lib.batq_lora_workspace, 0
    for M in sorted({m + d for m in [1, 16, 32, 48, 64, 128, 512, 1024, 1360, 1376, 2048, 4096, 8192] for d in (-1, 0, 1) if m + d > 0}):
        got = w(M, K, 64, 16, 2)
        for N in (64, 1 << 24):
            assert got == w(M, K, N, 16, 3) and got >= 4 * 16 * M * lora_parts(M, K, N)
        assert got >= before and w(M, K, 64, 24, 2) >= got and w(M, K + 32, 64, 16, 2) >= got and w(M, K + 2048, 64, 16, 2) >= got
        assert got <= 4 * 16 * max(M, min(M, 64) * 8, min(M, 1024) * 4, min(M, 1360) * 3, min(M, 2048) * 2)
        before = got


def test_queries_are_not_written_over_keys_or_values(B):
    """Other workgroups may still read them."""
    for kw in (dict(k=3 * P), dict(v=3 * P)):
        assert append(B, cache(), q=2 * P, q_heads=2, ldq=128, ldqo=128, q_out=3 * P, **kw) == 2


def test_a_cache_can_carry_what_a_program_attaches(B, monkeypatch):
    """Only the arrays and sizes are fixed."""
    torch = pytest.importorskip("torch")
    monkeypatch.setattr(B.binding, "_device", lambda: -1)
    c = B.PagedCache(4, 16, 2, 64, tensors=[torch.zeros(s, dtype=torch.uint8) for s in ((4, 2, 16, 64), (4, 2, 2, 16)) * 2])
    c.layer = 3
    c.layer += 1
    assert c.layer == 4
    with pytest.raises(AttributeError):
        c._at = []
