// Low-rank adapters of many requests beside a shared projection: out = base + s (X A^T) B^T with each row's own pair.
// gfx950 only.
//
// Two kernels: shrink_kernel leaves h = X A^T (fp32, in parts of K) in the workspace, expand_kernel adds s h B^T.  Both
// take tiles of rows and, within a tile, one adapter at a time in the order of first appearance: no sorting, no
// bookkeeping between calls, and a tile whose rows share an adapter (the tokens of a request stand side by side) is one
// matrix product.  A matrix instruction's columns are rows of X: rows of other adapters are computed and not stored.
#include "batq_internal.h"
#include "mxfp4_device.h"

namespace batq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct LoraArgs {
    const void* X;
    const uint16_t *A, *B;
    const float* scales;
    const int32_t* index;
    const void* base;
    void* out;
    float* h;                                               // [part of K][M][rank]
    int64_t ldx, ldb, ldo;
    int M, K, N, rank, adapters;
    int slots;                                              // workgroups that share a tile's adapters
    int parts, part_k;                                      // parts of K and their length (a multiple of 256)
    int blocks_n;                                           // columns of a workgroup of expand_kernel, in blocks of 256
    int vec;                                                // base and out rows allow 16-byte accesses
};

// The adapter that row m uses, -1 for none.
__device__ __forceinline__ int adapter_of(const LoraArgs& a, int m) {
    const int i = a.index[m];
    return i >= 0 && i < a.adapters ? i : -1;
}

// Calls f(adapter) for each `slot`-th, (slot + slots)-th, ... distinct value of the tile's rows [row0, row0 + count), in
// the order of first appearance; count <= 64.  Wave-uniform.
template <typename F>
__device__ __forceinline__ void for_adapters(const LoraArgs& a, int row0, int count, int slot, F f) {
    const int lane = threadIdx.x & 63;
    const int mine = lane < count ? adapter_of(a, row0 + lane) : -2;
    uint64_t left = __ballot(lane < count);
    for (int n = 0; left; ++n) {
        const int id = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
        left &= ~__ballot(mine == id);
        if (n % a.slots == slot) f(id);
    }
}

// Sixteen consecutive elements as bf16 operands (k-slots 0..7 and 8..15), in `Terms` terms whose sum is the element.
template <int Terms>
__device__ __forceinline__ void load16(const uint16_t* p, bf16x8 (&x)[Terms][2]) {
    x[0][0] = reinterpret_cast<const bf16x8*>(p)[0], x[0][1] = reinterpret_cast<const bf16x8*>(p)[1];
}
template <int Terms>
__device__ __forceinline__ void load16(const float* p, bf16x8 (&x)[Terms][2]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4 v = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float r = v[e];
#pragma unroll
            for (int t = 0; t < Terms; ++t) {
                const __bf16 b = (__bf16)r;
                x[t][i >> 1][4 * (i & 1) + e] = b;
                r -= (float)b;
            }
        }
    }
}

// h[m][j] = sum over a part of K of X[m][k] A_a[j][k].  A workgroup takes (row tile of 16 RG rows, adapters of a slot, part
// of K); its four waves split the part and are added through LDS in wave order.  Lane (i, g) = (l % 16, l / 16) loads
// k = 16g .. 16g + 15 of every 64 for its row of A (i: rank index) and of X: whole 128-byte lines over two instructions.
template <typename XT, int RG, int JT>
__global__ void __launch_bounds__(256)
shrink_kernel(const LoraArgs a) {
    constexpr int kTerms = sizeof(XT) == 4 ? 3 : 1;
    __shared__ f32x4 s_acc[3][RG * JT][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int slot = blockIdx.x % a.slots, tile = blockIdx.x / a.slots, part = blockIdx.y;
    const int row0 = tile * 16 * RG, count = min(16 * RG, a.M - row0);
    const int k0 = part * a.part_k, k1 = min(a.K, k0 + a.part_k);
    for_adapters(a, row0, count, slot, [&](int id) {
        if (id < 0) return;
        const uint16_t* ap[JT];
#pragma unroll
        for (int j = 0; j < JT; ++j) ap[j] = a.A + ((size_t)id * a.rank + min(16 * j + i, a.rank - 1)) * a.K + 16 * g;
        const XT* xp[RG];
#pragma unroll
        for (int r = 0; r < RG; ++r) xp[r] = static_cast<const XT*>(a.X) + (size_t)min(row0 + 16 * r + i, a.M - 1) * a.ldx + 16 * g;
        f32x4 acc[RG][JT];
#pragma unroll
        for (int r = 0; r < RG; ++r)
#pragma unroll
            for (int j = 0; j < JT; ++j) acc[r][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        auto step = [&](int k, bool inside) {               // K is a multiple of 32: the last 64 may be half there
            bf16x8 aw[JT][1][2];
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                load16<1>(ap[j] + (inside ? k : 0), aw[j]);
                if (!inside) aw[j][0][0] = bf16x8{}, aw[j][0][1] = bf16x8{};
            }
#pragma unroll
            for (int r = 0; r < RG; ++r) {
                bf16x8 x[kTerms][2];
                load16<kTerms>(xp[r] + (inside ? k : 0), x);
                if (!inside)
#pragma unroll
                    for (int t = 0; t < kTerms; ++t) x[t][0] = bf16x8{}, x[t][1] = bf16x8{};
#pragma unroll
                for (int j = 0; j < JT; ++j)
#pragma unroll
                    for (int t = kTerms - 1; t >= 0; --t)
#pragma unroll
                        for (int e = 0; e < 2; ++e) acc[r][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw[j][0][e], x[t][e], acc[r][j], 0, 0, 0);
            }
        };
        // (a lane whose 16 elements lie behind K reads the row's first ones instead and multiplies zeros)
        for (int k = k0 + 64 * wave; k < k1; k += 256) {
            if (k + 64 <= k1) step(k, true);
            else step(k, k + 16 * g < k1);
        }
        __syncthreads();                                    // (the previous adapter's sums have been read)
        if (wave > 0)
#pragma unroll
            for (int r = 0; r < RG; ++r)
#pragma unroll
                for (int j = 0; j < JT; ++j) s_acc[wave - 1][r * JT + j][lane] = acc[r][j];
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int r = 0; r < RG; ++r) {
            const int m = row0 + 16 * r + i;
            const bool live = 16 * r + i < count && adapter_of(a, min(m, a.M - 1)) == id;
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                f32x4 v = acc[r][j];
#pragma unroll
                for (int w = 0; w < 3; ++w) v += s_acc[w][r * JT + j][lane];
                const int at = 16 * j + 4 * g;              // the rank is a multiple of 8
                if (live && at < a.rank) *reinterpret_cast<f32x4*>(a.h + ((size_t)part * a.M + m) * a.rank + at) = v;
            }
        }
    });
}

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return bf16_bits_to_float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }
// Sixteen elements with 16-byte accesses.
__device__ __forceinline__ void read16(const float* p, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4 x = reinterpret_cast<const f32x4*>(p)[i];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * i + e] = x[e];
    }
}
__device__ __forceinline__ void read16(const uint16_t* p, float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const bf16x8 x = reinterpret_cast<const bf16x8*>(p)[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[8 * i + e] = (float)x[e];
    }
}
__device__ __forceinline__ void write16(float* p, const float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) reinterpret_cast<f32x4*>(p)[i] = f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]};
}
__device__ __forceinline__ void write16(uint16_t* p, const float (&v)[16]) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        bf16x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (__bf16)v[8 * i + e];
        reinterpret_cast<bf16x8*>(p)[i] = x;
    }
}

// Eight-element chunks of the contraction: the rank's chunks of h's first bf16 term, then of the second and the third
// (their sum is h to 24 bits), padded to whole instructions of four chunks with zeros.
__device__ __forceinline__ int chunk_steps(int rank) { return (3 * (rank / 8) + 3) / 4; }
__host__ __device__ inline int h_pitch(int rank) { return ((3 * (rank / 8) + 3) / 4) * 64 + 16; }   // bytes of a row in LDS

// out = base + s h B^T.  A workgroup takes (row tile of 16 RG rows, adapters of a slot, 256 blocks_n columns); a wave takes 64
// columns at a time.  Lane (i, g) ends with columns 16g .. 16g + 15 of row i (the columns of the four instructions of a
// step are numbered that way): 128 contiguous bytes of bf16 per row.
template <typename YT, int RG>
__global__ void __launch_bounds__(256)
expand_kernel(const LoraArgs a) {
    extern __shared__ __align__(16) uint8_t s_h[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int slot = blockIdx.x % a.slots, tile = blockIdx.x / a.slots;
    const int row0 = tile * 16 * RG, count = min(16 * RG, a.M - row0);
    const int n_begin = blockIdx.y * a.blocks_n * 256, n_end = (int)min((int64_t)a.N, (int64_t)n_begin + a.blocks_n * 256);
    const int chunks = a.rank / 8, steps = chunk_steps(a.rank), pitch = h_pitch(a.rank);
    for_adapters(a, row0, count, slot, [&](int id) {
        if (id < 0 && a.base == a.out) return;              // nothing to add, nothing to copy
        if (id >= 0) {
            const float s = a.scales ? a.scales[id] : 1.0f;
            __syncthreads();                                // (the previous adapter's h has been read)
            for (int c = threadIdx.x; c < 16 * RG * chunks; c += 256) {
                const int r = c / chunks, ch = c - r * chunks;
                const bool live = r < count && adapter_of(a, row0 + r) == id;       // other rows of h may hold anything
                float v[8] = {};
                if (live)
                    for (int p = 0; p < a.parts; ++p) {
                        const float* hp = a.h + ((size_t)p * a.M + row0 + r) * a.rank + 8 * ch;
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] += hp[e];
                    }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] *= s;
#pragma unroll
                for (int t = 0; t < 3; ++t) {
                    bf16x8 x;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        x[e] = (__bf16)v[e];
                        v[e] -= (float)x[e];
                    }
                    *reinterpret_cast<bf16x8*>(s_h + r * pitch + (t * chunks + ch) * 16) = x;
                }
            }
            for (int c = threadIdx.x; c < 16 * RG * (4 * steps - 3 * chunks); c += 256) {
                const int pad = 4 * steps - 3 * chunks, r = c / pad;
                *reinterpret_cast<bf16x8*>(s_h + r * pitch + (3 * chunks + c - r * pad) * 16) = bf16x8{};
            }
            __syncthreads();
        }
        for (int n0 = n_begin + 64 * wave; n0 < n_end; n0 += 256) {
            f32x4 acc[RG][4];
#pragma unroll
            for (int r = 0; r < RG; ++r)
#pragma unroll
                for (int t = 0; t < 4; ++t) acc[r][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
            if (id >= 0) {
                const uint16_t* bp[4];                      // instruction t's row 4q + e is column 16q + 4t + e
#pragma unroll
                for (int t = 0; t < 4; ++t) bp[t] = a.B + ((size_t)id * a.N + min(n0 + 16 * (i >> 2) + 4 * t + (i & 3), a.N - 1)) * a.rank;
                for (int st = steps - 1; st >= 0; --st) {   // smallest terms first
                    const int rc = (4 * st + g) % chunks;
                    bf16x8 bw[4];
#pragma unroll
                    for (int t = 0; t < 4; ++t) bw[t] = *reinterpret_cast<const bf16x8*>(bp[t] + 8 * rc);
#pragma unroll
                    for (int r = 0; r < RG; ++r) {
                        const bf16x8 hw = *reinterpret_cast<const bf16x8*>(s_h + (16 * r + i) * pitch + (4 * st + g) * 16);
#pragma unroll
                        for (int t = 0; t < 4; ++t) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bw[t], hw, acc[r][t], 0, 0, 0);
                    }
                }
            }
            const int n = n0 + 16 * g;
#pragma unroll
            for (int r = 0; r < RG; ++r) {
                const int m = row0 + 16 * r + i;
                if (16 * r + i >= count || adapter_of(a, m) != id || n >= a.N) continue;
                const YT* b = a.base ? static_cast<const YT*>(a.base) + (size_t)m * a.ldb + n : nullptr;
                YT* o = static_cast<YT*>(a.out) + (size_t)m * a.ldo + n;
                float v[16];
                if (a.vec && n + 16 <= a.N) {
                    if (b) read16(b, v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) v[e] = (b ? v[e] : 0.0f) + acc[r][e >> 2][e & 3];
                    write16(o, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (n + e < a.N) put(o + e, (b ? value(b[e]) : 0.0f) + acc[r][e >> 2][e & 3]);
                }
            }
        }
    });
}

// How a call is cut.  Row tiles: 16 rows where there are few (decoding: a tile's adapters are spread over workgroups), else
// 64 (32 of large ranks, whose sums fill the registers).  Parts of K: two workgroups to a compute unit if the rows of a tile
// share one or two adapters, at least 256 to a part.
struct Plan {
    int rg, tiles, slots, parts, part_k;
};
Plan plan(int M, int K, int rank, int adapters) {
    Plan p;
    p.rg = M <= 512 ? 1 : rank > 64 ? 2 : 4;
    p.tiles = (int)(((int64_t)M + 16 * p.rg - 1) / (16 * p.rg));
    p.slots = p.rg == 1 ? 16 : 4;
    if (p.slots > adapters + 1) p.slots = adapters + 1;     // (rows without an adapter count as one)
    int n = 512 / (p.rg == 1 ? 2 * p.tiles : p.tiles);
    if (n > (K + 255) / 256) n = (K + 255) / 256;
    if (n > 16) n = 16;
    if (n < 1) n = 1;
    p.part_k = ((K + n - 1) / n + 255) & ~255;
    p.parts = (K + p.part_k - 1) / p.part_k;
    return p;
}

template <typename XT>
void shrink(const LoraArgs& a, int rg, dim3 grid, hipStream_t stream) {
    if (a.rank > 64) rg == 1 ? shrink_kernel<XT, 1, 8><<<grid, 256, 0, stream>>>(a) : shrink_kernel<XT, 2, 8><<<grid, 256, 0, stream>>>(a);
    else if (a.rank > 32) rg == 1 ? shrink_kernel<XT, 1, 4><<<grid, 256, 0, stream>>>(a) : shrink_kernel<XT, 4, 4><<<grid, 256, 0, stream>>>(a);
    else if (a.rank > 16) rg == 1 ? shrink_kernel<XT, 1, 2><<<grid, 256, 0, stream>>>(a) : shrink_kernel<XT, 4, 2><<<grid, 256, 0, stream>>>(a);
    else rg == 1 ? shrink_kernel<XT, 1, 1><<<grid, 256, 0, stream>>>(a) : shrink_kernel<XT, 4, 1><<<grid, 256, 0, stream>>>(a);
}

template <typename YT>
void expand(const LoraArgs& a, int rg, dim3 grid, hipStream_t stream) {
    if (rg == 1) expand_kernel<YT, 1><<<grid, 256, 16 * h_pitch(a.rank), stream>>>(a);
    else if (rg == 2) expand_kernel<YT, 2><<<grid, 256, 32 * h_pitch(a.rank), stream>>>(a);
    else expand_kernel<YT, 4><<<grid, 256, 64 * h_pitch(a.rank), stream>>>(a);
}

}  // namespace

size_t lora_workspace_bytes(int M, int K, int, int rank, int adapters) {
    return M > 0 ? (size_t)plan(M, K, rank, adapters).parts * M * rank * 4 : 0;
}

hipError_t launch_lora_add(const void* X, batq_dtype xdtype, int M, int K, int64_t ldx, const void* A, const void* B,
                           int N, int rank, int adapters, const float* scales, const int32_t* index, const void* base,
                           int64_t ldb, void* out, int64_t ldo, batq_dtype ydtype, void* workspace, hipStream_t stream) {
    const Plan p = plan(M, K, rank, adapters);
    LoraArgs a = {};
    a.X = X, a.A = static_cast<const uint16_t*>(A), a.B = static_cast<const uint16_t*>(B), a.scales = scales, a.index = index;
    a.base = base, a.out = out, a.h = static_cast<float*>(workspace), a.ldx = ldx, a.ldb = ldb, a.ldo = ldo;
    a.M = M, a.K = K, a.N = N, a.rank = rank, a.adapters = adapters, a.slots = p.slots, a.parts = p.parts, a.part_k = p.part_k;
    const int64_t size = ydtype == BATQ_BF16 ? 2 : 4;
    a.vec = ((uintptr_t)out | (uintptr_t)base | (uintptr_t)(ldo * size) | (uintptr_t)(base ? ldb * size : 0)) % 16 == 0;
    const dim3 grid((unsigned)p.tiles * p.slots, p.parts);
    if (xdtype == BATQ_BF16) shrink<uint16_t>(a, p.rg, grid, stream);
    else shrink<float>(a, p.rg, grid, stream);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    // columns of a workgroup: h is read again for each of them, so as many as leave four workgroups to a compute unit
    const int blocks = (int)(((int64_t)N + 255) / 256);
    a.blocks_n = p.rg == 1 ? 1 : (int)(((int64_t)p.tiles * blocks + 1023) / 1024);
    if (a.blocks_n > blocks) a.blocks_n = blocks;
    if (a.blocks_n < (blocks + 65534) / 65535) a.blocks_n = (blocks + 65534) / 65535;      // grid.y
    const dim3 wide((unsigned)p.tiles * p.slots, (blocks + a.blocks_n - 1) / a.blocks_n);
    if (ydtype == BATQ_BF16) expand<uint16_t>(a, p.rg, wide, stream);
    else expand<float>(a, p.rg, wide, stream);
    return hipGetLastError();
}

}  // namespace batq
