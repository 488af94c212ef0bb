"""batq_lora_add against the 64-bit statement of it."""
import numpy as np
import pytest

import batq_inputs as bi
from gpu_util import require_gpu, to_dev
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


def storage(rng, shape, dtype, scale=1.0):
    if dtype == "bf16":
        bits, val = ref.bf16_values(rng, *shape, scale=scale)
        return to_dev(bits, "bf16"), val.astype(np.float64)
    val = (scale * rng.standard_normal(shape)).astype(np.float32)
    return to_dev(val, "f32"), val.astype(np.float64)


def problem(rng, M, K, N, r, n, xdt, ydt, pattern, pad=0):
    X, Xv = storage(rng, (M, K + 8), xdt)
    A, Av = storage(rng, (n, r, K), "bf16", K ** -0.5)
    Bm, Bv = storage(rng, (n, N, r), "bf16", r ** -0.5)
    base, basev = storage(rng, (M, N + pad), ydt)
    scales = rng.uniform(0.5, 2.0, n).astype(np.float32)
    index = {"mixed": rng.integers(-1, n + 1, M), "runs": np.sort(rng.integers(0, n, M)), "one": np.full(M, n - 1),
             "none": np.full(M, -1), "each": np.arange(M) % n}[pattern].astype(np.int32)
    return X[:, :K], Xv[:, :K], A, Av, Bm, Bv, base[:, :N], basev[:, :N], scales, index


def check(got, Xv, Av, Bv, basev, scales, index, ydt):
    """Products of bf16 (or fp32) numbers summed in fp32 (K and then rank terms, at most 2^-24 each of the sums of
    magnitudes; a random walk of them stays far below K 2^-24), one rounding to the output type."""
    M, K = Xv.shape
    want, mag = basev.copy(), np.abs(basev)
    for m in range(M):
        a = index[m]
        if 0 <= a < len(scales):
            h, habs = Xv[m] @ Av[a].T, np.abs(Xv[m]) @ np.abs(Av[a]).T
            want[m] += scales[a].astype(np.float64) * (Bv[a] @ h)
            mag[m] += scales[a] * (np.abs(Bv[a]) @ habs)
    half = 2.0 ** -8 if ydt == "bf16" else 2.0 ** -24
    tol = half * np.abs(want) + (np.sqrt(K) + Av.shape[1]) * 2.0 ** -22 * mag
    assert np.all(np.abs(got - want) <= tol), (np.abs(got - want) / tol).max()
    untouched = (index < 0) | (index >= len(scales))
    assert np.array_equal(got[untouched], basev[untouched])


CASES = [
    # M, K, N, rank, adapters, index
    (1, 32, 1, 8, 1, "one"),
    (1, 4096, 4096, 16, 3, "one"),
    (5, 96, 33, 8, 2, "mixed"),
    (17, 256, 130, 24, 4, "each"),
    (32, 1024, 512, 16, 32, "each"),
    (33, 512, 700, 64, 3, "mixed"),
    (64, 2048, 96, 128, 2, "runs"),
    (130, 608, 1000, 40, 5, "mixed"),
    (257, 320, 257, 32, 2, "runs"),
    (300, 64, 64, 16, 1, "none"),
    (700, 1024, 640, 16, 3, "runs"),
    (513, 4096, 72, 72, 2, "one"),
]


@pytest.mark.parametrize("M,K,N,r,n,pattern", CASES)
@pytest.mark.parametrize("xdt,ydt", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
def test_lora_add(B, M, K, N, r, n, pattern, xdt, ydt):
    import torch
    rng = np.random.default_rng(M + K + N + r)
    X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, M, K, N, r, n, xdt, ydt, pattern, pad=3)
    full = torch.full((M, N + 5), 7.0, dtype=base.dtype, device="cuda")
    out = full[:, :N]                                       # odd row pitches: elements, not vectors, are aligned
    B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales), out=out)
    torch.cuda.synchronize()
    check(out.float().cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, scales, index, ydt)
    assert bool((full[:, N:] == 7.0).all())
    # in place, contiguous, and without scales
    out2 = base.clone()
    B.batq_lora_add(X, A, Bm, dev(index), out2, out=out2)
    torch.cuda.synchronize()
    check(out2.float().cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, np.ones(n, np.float32), index, ydt)
    # without a base
    out3 = B.batq_lora_add(X, A, Bm, dev(index), scales=dev(scales), out_dtype=base.dtype)
    torch.cuda.synchronize()
    check(out3.float().cpu().numpy().astype(np.float64), Xv, Av, Bv, 0 * basev, scales, index, ydt)


def test_rows_do_not_depend_on_the_batch(B):
    """The rows of a request give the same bits whatever else is in the batch of the same size class."""
    import torch
    rng = np.random.default_rng(2)
    X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, 200, 512, 320, 16, 4, "bf16", "f32", "mixed")
    a = B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales))
    again = B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales))
    other = index.copy()
    other[100:] = rng.integers(-1, 4, 100)
    b = B.batq_lora_add(X, A, Bm, dev(other), base, scales=dev(scales))
    torch.cuda.synchronize()
    assert torch.equal(a, again) and torch.equal(a[:100], b[:100])


def test_lora_beside_the_projection_on_streams_and_in_graphs(B):
    """batq_linear and the adapters as one captured step; two graphs share a workspace, replays follow new inputs."""
    import torch
    rng = np.random.default_rng(3)
    M, K, N, r, n = 40, 640, 320, 16, 3
    w = bi.make_small(M, K, N, seed=1, dtype="bf16")
    t = B.Transform(K, w.G, w.P, w.clip)
    wh = B.batq_prepare_weight(t, to_dev(w.W, "bf16"))
    X, A, Bm = to_dev(w.X, "bf16"), to_dev(ref.bf16_values(rng, n, r, K, scale=0.05)[0], "bf16"), to_dev(ref.bf16_values(rng, n, N, r, scale=0.2)[0], "bf16")
    index = dev(rng.integers(-1, n, M).astype(np.int32))
    ws = torch.full((max(16, B.batq_lora_workspace(M, K, N, r, n)),), 0xFF, dtype=torch.uint8, device="cuda")
    lw = torch.empty(B.batq_linear_workspace_for(wh, M), dtype=torch.uint8, device="cuda")

    def step(out):
        B.batq_linear(t, wh, X, Y=out, workspace=lw)
        B.batq_lora_add(X, A, Bm, index, out, out=out, workspace=ws)

    outs = [torch.zeros((M, N), dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    step(outs[2])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for g, oo in zip(graphs, outs):
        with torch.cuda.graph(g, stream=side):
            step(oo)
    for rep in range(3):
        X.copy_(torch.randn_like(X) * (rep + 1))
        index.copy_(dev(rng.integers(-1, n, M).astype(np.int32)))
        step(outs[2])
        torch.cuda.synchronize()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2]), rep


def test_sizes_at_the_edges(B):
    """Widths of one column, ranks at the ends, rows of every tile remainder, many rows with many adapters mixed."""
    import torch
    for M, K, N, r, n, pattern in ((1, 32, 1, 128, 1, "one"), (15, 64, 63, 8, 15, "each"), (16, 64, 65, 56, 2, "mixed"), (512, 96, 40, 104, 9, "mixed"),
                                   (600, 160, 130, 8, 40, "mixed"), (1025, 32, 257, 48, 3, "runs"), (2000, 512, 64, 16, 2, "none")):
        rng = np.random.default_rng(M * 7 + N)
        X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, M, K, N, r, n, "bf16", "f32", pattern)
        out = B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales))
        torch.cuda.synchronize()
        check(out.cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, scales, index, "f32")


def test_garbage_in_the_workspace_and_beside_the_rows_does_not_show(B):
    """NaN in the workspace, in rows of X behind M and in padding columns."""
    import torch
    rng = np.random.default_rng(8)
    for M, pattern in ((20, "mixed"), (700, "mixed")):
        X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, M, 96, 70, 24, 3, "bf16", "bf16", pattern)
        wide = torch.full((M + 40, 96 + 32), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:M, :96] = X
        ws = torch.full((B.batq_lora_workspace(M, 96, 70, 24, 3),), 0xFF, dtype=torch.uint8, device="cuda")
        out = B.batq_lora_add(wide[:M, :96], A, Bm, dev(index), base, scales=dev(scales), workspace=ws)
        torch.cuda.synchronize()
        check(out.float().cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, scales, index, "bf16")


def test_two_calls_at_once(B):
    import torch
    rng = np.random.default_rng(9)
    probs = [problem(rng, M, 512, 300, 16, 4, "bf16", "f32", "mixed") for M in (30, 700)]
    want, ws, streams = [], [], [torch.cuda.Stream() for _ in probs]
    for X, _, A, _, Bm, _, base, _, scales, index in probs:
        want.append(B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales)))
        ws.append(torch.empty(B.batq_lora_workspace(X.shape[0], 512, 300, 16, 4), dtype=torch.uint8, device="cuda"))
    devs = [(dev(p[9]), dev(p[8])) for p in probs]
    outs = [torch.zeros_like(w) for w in want]
    torch.cuda.synchronize()
    for _ in range(5):
        for (X, _, A, _, Bm, _, base, _, _, _), (index, scales), w, out, s in zip(probs, devs, ws, outs, streams):
            with torch.cuda.stream(s):
                B.batq_lora_add(X, A, Bm, index, base, scales=scales, out=out, workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(outs, want))


def test_binding_refuses_what_does_not_fit(B):
    import torch
    X, A, Bm = torch.zeros((2, 64), device="cuda"), torch.zeros((1, 8, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 40, 8), dtype=torch.bfloat16, device="cuda")
    index, base = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros((2, 40), device="cuda")
    B.batq_lora_add(X, A, Bm, index, base)
    for bad in (dict(X=X.cpu()), dict(X=X[:, ::2]), dict(A=A.float()), dict(B=Bm[:, :, :4]), dict(index=index.long()), dict(base=base[:1]),
                dict(base=base.t()), dict(out=base.bfloat16()), dict(scales=torch.zeros(2, device="cuda"))):
        with pytest.raises(ValueError):
            B.batq_lora_add(**{**dict(X=X, A=A, B=Bm, index=index, base=base), **bad})
    with pytest.raises(B.BatqError):
        B.batq_lora_add(X, A, Bm, index, base, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("M,K,N,r,n,pattern,xdt", [(100, 4128, 72, 24, 3, "mixed", "bf16"), (70, 8992, 50, 8, 70, "each", "f32"), (513, 4096, 65, 40, 5, "mixed", "bf16"),
                                                   (65, 2080, 300, 128, 4, "runs", "bf16"), (64, 2080, 300, 72, 4, "mixed", "f32"), (200, 16384, 33, 16, 2, "mixed", "bf16")])
def test_long_contractions(B, M, K, N, r, n, pattern, xdt):
    """K in two to eight parts, on both sides of 64 and of 512 rows."""
    import torch
    rng = np.random.default_rng(M + K)
    X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, M, K, N, r, n, xdt, "f32", pattern)
    out = B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales))
    torch.cuda.synchronize()
    check(out.cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, scales, index, "f32")


def test_one_workspace_serves_every_smaller_call(B):
    """A workspace sized for the largest call, full of NaN, with calls of fewer rows in more parts."""
    import torch
    K, N, r, n = 4096, 72, 16, 3
    ws = torch.full((B.batq_lora_workspace(3000, K, N, r, n),), 0xFF, dtype=torch.uint8, device="cuda")
    for M in (3000, 2048, 1024, 513, 65, 64, 17, 1):
        rng = np.random.default_rng(M)
        X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, M, K, N, r, n, "bf16", "f32", "mixed")
        out = B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales), workspace=ws)
        torch.cuda.synchronize()
        check(out.cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, scales, index, "f32")
    small = torch.full((B.batq_lora_workspace(64, 8192, N, r, n),), 0xFF, dtype=torch.uint8, device="cuda")
    for M, k in ((64, 8192), (64, 512), (9, 4096)):
        rng = np.random.default_rng(M + k)
        X, Xv, A, Av, Bm, Bv, base, basev, scales, index = problem(rng, M, k, N, r, n, "f32", "bf16", "mixed")
        out = B.batq_lora_add(X, A, Bm, dev(index), base, scales=dev(scales), workspace=small)
        torch.cuda.synchronize()
        check(out.float().cpu().numpy().astype(np.float64), Xv, Av, Bv, basev, scales, index, "bf16")
