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
