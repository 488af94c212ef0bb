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

constexpr int kMaxParts = 8;                                // of K

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
    int tile_rows, groups_n;                                // row tiles of a workgroup of expand_kernel, workgroups beside each other
    int vec;                                                // base and out rows allow 16-byte accesses
    int past_cache;                                         // base and out together do not stay in the memory-side cache
};

// The adapter that row m uses, -1 for none.
__device__ __forceinline__ int adapter_of(const LoraArgs& a, int m) {
    const int i = a.index[m];
    return i >= 0 && i < a.adapters ? i : -1;
}

// Calls f(adapter) for each `slot`-th, (slot + slots)-th, ... distinct adapter of a tile of 16 rows, in the order of first
// appearance; lane l holds the adapter of row l % 16 (-1: none, -2: no such row).  Wave-uniform.
template <typename F>
__device__ __forceinline__ void for_adapters(const LoraArgs& a, int mine, int slot, F f) {
    uint64_t left = __ballot(mine != -2) & 0xFFFFu;
    for (int n = 0; left; ++n) {
        const int id = __builtin_amdgcn_readlane(mine, __builtin_ctzll(left));
        left &= ~__ballot(mine == id);
        if (n == slot || (n > slot && (n - slot) % a.slots == 0)) f(id);
    }
}

// Eight consecutive elements as bf16 operands in `Terms` terms whose sum is the element.
template <int Terms>
__device__ __forceinline__ void terms8(const uint16_t*, const f32x4* w, bf16x8 (&x)[Terms]) {
    x[0] = __builtin_bit_cast(bf16x8, w[0]);
}
template <int Terms>
__device__ __forceinline__ void terms8(const float*, const f32x4* w, bf16x8 (&x)[Terms]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float r = w[e >> 2][e & 3];
#pragma unroll
        for (int t = 0; t < Terms; ++t) {
            x[t][e] = (__bf16)r;
            r -= (float)x[t][e];
        }
    }
}

// A wave's piece of a matrix in LDS: Rows rows of 64 elements, requested with 16-byte loads whose neighbouring lanes take
// neighbouring 16 bytes of a row (operands loaded straight into registers would have every lane in another row: with
// rows 8 KiB apart, four times slower), the 16-byte chunks of a row XORed with the row's number so that 16 lanes
// that read a chunk of 16 rows reach all banks.
template <typename T, int Rows>
struct Piece {
    static constexpr int kChunks = 4 * (int)sizeof(T);      // of a row
    static constexpr int kRowsAtOnce = 64 / kChunks, kLoads = Rows / kRowsAtOnce, kBytes = Rows * kChunks * 16;
    f32x4 w[kLoads];
    __device__ static int place(int row, int chunk) { return row * kChunks + (kChunks == 16 ? chunk ^ (row & 15) : chunk ^ ((row >> 1) & 7)); }
    // element 64 of row r at rows(r) + k; lanes whose chunk lies behind `left` elements get zeros
    template <typename F>
    __device__ __forceinline__ void request(F rows, int k, int left) {
        const int lane = threadIdx.x & 63, c = lane % kChunks, e = c * (16 / (int)sizeof(T));
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const T* p = rows(i * kRowsAtOnce + lane / kChunks) + k;
            w[i] = e < left ? *reinterpret_cast<const f32x4*>(p + e) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        }
    }
    __device__ __forceinline__ void store(f32x4* lds) const {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) lds[place(i * kRowsAtOnce + lane / kChunks, lane % kChunks)] = w[i];
    }
    // elements 8 c .. 8 c + 7 of a row
    template <int Terms>
    __device__ static void operand(const f32x4* lds, int row, int c, bf16x8 (&x)[Terms]) {
        f32x4 v[kChunks / 8];
#pragma unroll
        for (int i = 0; i < kChunks / 8; ++i) v[i] = lds[place(row, c * (kChunks / 8) + i)];
        terms8<Terms>(static_cast<const T*>(nullptr), v, x);
    }
};

template <typename XT, int JT, int W>
constexpr int shrink_lds() { return W * (Piece<XT, 16>::kBytes + Piece<uint16_t, 16 * JT>::kBytes); }   // (the sums need less)

// h[m][j] = sum over a part of K of X[m][k] A_a[j][k].  A workgroup takes (16 rows, adapters of a slot, part of K); its W
// waves split the part into W ranges and are added through LDS in wave order.  A wave works on 64 k at a time, out of
// its own pieces of LDS, while the next 64 are on their way to registers.  Bound: the stream of X (many rows), the latency
// of index, loads and sums in a row (few).  Measured: 4096 rows of K 4096 in bf16, rank 32: 12 us (2.8 TB/s); 32 rows with 16
// adapters of rank 16: 4.5 us.
template <typename XT, int JT, int W>
__global__ void __launch_bounds__(64 * W)
shrink_kernel(const LoraArgs a) {
    constexpr int kTerms = sizeof(XT) == 4 ? 3 : 1;
    using PX = Piece<XT, 16>;
    using PA = Piece<uint16_t, 16 * JT>;
    extern __shared__ __align__(16) uint8_t s_raw[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int part = blockIdx.x % a.parts, ts = blockIdx.x / a.parts, slot = ts % a.slots, row0 = ts / a.slots * 16;
    const int share = a.part_k / W, k0 = part * a.part_k + wave * share, k1 = min(a.K, k0 + share);
    f32x4* const s_x = reinterpret_cast<f32x4*>(s_raw + wave * (PX::kBytes + PA::kBytes));
    f32x4* const s_a = s_x + PX::kBytes / 16;
    f32x4* const s_acc = reinterpret_cast<f32x4*>(s_raw);   // [W - 1][JT][64], when the pieces are used up
    auto x_row = [&](int r) { return static_cast<const XT*>(a.X) + (size_t)min(row0 + r, a.M - 1) * a.ldx; };
    const int mine = row0 + i < a.M ? adapter_of(a, row0 + i) : -2;
    for_adapters(a, mine, slot, [&](int id) {
        if (id < 0) return;
        auto a_row = [&](int j) { return a.A + ((size_t)id * a.rank + min(j, a.rank - 1)) * a.K; };
        f32x4 acc[JT];
#pragma unroll
        for (int j = 0; j < JT; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        PX px;
        PA pa;
        if (k0 < k1) px.request(x_row, k0, k1 - k0), pa.request(a_row, k0, k1 - k0);
        for (int k = k0; k < k1; k += 64) {
            // (a wave's LDS operations are carried out in order: the last step's reads come before these writes)
            px.store(s_x);
            pa.store(s_a);
            if (k + 64 < k1) px.request(x_row, k + 64, k1 - k - 64), pa.request(a_row, k + 64, k1 - k - 64);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                bf16x8 x[kTerms];
                PX::template operand<kTerms>(s_x, i, 4 * e + g, x);
#pragma unroll
                for (int j = 0; j < JT; ++j) {
                    bf16x8 aw[1];
                    PA::template operand<1>(s_a, 16 * j + i, 4 * e + g, aw);
#pragma unroll
                    for (int t = kTerms - 1; t >= 0; --t) acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(aw[0], x[t], acc[j], 0, 0, 0);
                }
            }
        }
        __syncthreads();                                    // every wave is done with its pieces
        if (wave > 0)
#pragma unroll
            for (int j = 0; j < JT; ++j) s_acc[((wave - 1) * JT + j) * 64 + lane] = acc[j];
        __syncthreads();
        if (wave == 0)
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                f32x4 v = acc[j];
#pragma unroll
                for (int w = 0; w < W - 1; ++w) v += s_acc[(w * JT + j) * 64 + lane];
                const int at = 16 * j + 4 * g;              // the rank is a multiple of 8
                if (mine == id && at < a.rank) *reinterpret_cast<f32x4*>(a.h + ((size_t)part * a.M + row0 + i) * a.rank + at) = v;
            }
        __syncthreads();                                    // the sums have been read: the pieces may be written again
    });
}

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return bf16_bits_to_float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *reinterpret_cast<__bf16*>(p) = (__bf16)x; }
// C neighbouring columns of a row (16 or 8 bytes) as they lie in memory.
template <typename T, int C>
struct Cols {
    typedef uint32_t words __attribute__((ext_vector_type(C * (int)sizeof(T) / 4)));
    words w;
    __device__ __forceinline__ float at(int c) const {
        if constexpr (sizeof(T) == 4) return __uint_as_float(w[c]);
        else return __uint_as_float(c & 1 ? w[c / 2] & 0xFFFF0000u : w[c / 2] << 16);
    }
    // (in assembly: the compiler would make one plain store of this and of the other branch's)
    __device__ __forceinline__ void store_nt(void* p) const {
        if constexpr (sizeof(words) == 16) asm volatile("global_store_dwordx4 %0, %1, off nt\n\ts_nop 1" :: "v"(p), "v"(w) : "memory");
        else asm volatile("global_store_dwordx2 %0, %1, off nt\n\ts_nop 1" :: "v"(p), "v"(w) : "memory");
    }
    __device__ __forceinline__ void set(const float (&v)[C]) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int c = 0; c < C; ++c) w[c] = __float_as_uint(v[c]);
        } else {
            typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int c = 0; c < C; c += 2) w[c / 2] = __builtin_bit_cast(uint32_t, bf16x2{(__bf16)v[c], (__bf16)v[c + 1]});
        }
    }
};

// out = base + s h B^T.  A wave takes 16 C columns and tile_rows tiles of 16 rows, one after the other, and keeps the
// adapter's B for its columns in registers (G groups of 32 rank indexes) until a row wants another adapter.  Column t of the C
// instructions of a tile is column C i + t in lane (i, g) = (l % 16, l / 16): a lane ends with C neighbouring columns of
// rows 4g .. 4g + 3, 16 lanes with a contiguous piece of a row.  h is taken as three bf16 terms (24 bits).  The sums start
// from base, which is requested a tile ahead.  Bound: base in, out out.  Measured: 4096 x 14336 in bf16, rank 32: 62.6 us
// (3.8 TB/s in and out; with 8 columns to a lane the same in half the waves, 16 registers spilled and 78 us in three quarters);
// 32 x 4096 with 16 adapters: 7.6 us.
template <typename YT, int G, int P>
__global__ void __launch_bounds__(256, P > 1 ? (G == 4 ? 1 : 2) : G == 1 ? 4 : 2)
expand_kernel(const LoraArgs a) {
    constexpr int C = 4, kWide = 16 * C;                    // columns of a lane, of a wave
    typedef Cols<YT, C> V;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane & 15, g = lane >> 4;
    const int y = blockIdx.x % a.groups_n, ts = blockIdx.x / a.groups_n, slot = ts % a.slots, tile0 = ts / a.slots * a.tile_rows;
    const int n0 = (y * 4 + wave) * kWide, n = n0 + C * i;
    if (n0 >= a.N) return;
    const bool whole = a.vec && n0 + kWide <= a.N;          // wave-uniform
    const int chunks = a.rank / 8, tiles = (a.M + 15) / 16, tile1 = min(tiles, tile0 + a.tile_rows);
    auto base_row = [&](int m) { return static_cast<const YT*>(a.base) + (size_t)min(m, a.M - 1) * a.ldb; };   // (past the end: the last row again)
    auto request = [&](int tile, V (&v)[4]) {
        if (a.base && whole)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const V*>(base_row(tile * 16 + 4 * g + e) + n);
    };
    auto adapters = [&](int tile) { return tile * 16 + i < a.M ? adapter_of(a, tile * 16 + i) : -2; };
    bf16x8 bw[G][C];
    float s = 0.0f;
    int loaded = -1;
    V next[4];
    if (slot == 0) request(tile0, next);
    int mine_next = adapters(tile0);
    if (slot > 0) {                                         // (one tile, which may have fewer adapters than there are slots)
        bool any = false;
        for_adapters(a, mine_next, slot, [&](int) { any = true; });
        if (!any) return;
        request(tile0, next);
    }
    for (int tile = tile0; tile < tile1; ++tile) {
        const int row0 = tile * 16, mine = mine_next;
        V now[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) now[e] = next[e];
        if (tile + 1 < tile1) {
            request(tile + 1, next);
            mine_next = adapters(tile + 1);
        }
        for_adapters(a, mine, slot, [&](int id) {
            if (id < 0 && a.base == a.out) return;          // nothing to add, nothing to copy
            f32x4 acc[C];                                   // [column][row]
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int t = 0; t < C; ++t) acc[t][e] = a.base && whole ? now[e].at(t) : 0.0f;
            if (id >= 0) {
                if (id != loaded) {
                    loaded = id;
                    s = a.scales ? a.scales[id] : 1.0f;
#pragma unroll
                    for (int q = 0; q < G; ++q)
#pragma unroll
                        for (int t = 0; t < C; ++t)
                            bw[q][t] = *reinterpret_cast<const bf16x8*>(a.B + ((size_t)id * a.N + min(n + t, a.N - 1)) * a.rank + 8 * min(4 * q + g, chunks - 1));
                }
#pragma unroll
                for (int q = 0; q < G; ++q) {
                    float v[8] = {};
                    if (mine == id && 4 * q + g < chunks) { // (other rows of h may hold anything)
                        const float* hp = a.h + (size_t)(row0 + i) * a.rank + 8 * (4 * q + g);
                        const size_t step = (size_t)a.M * a.rank;
                        f32x4 h0[P], h1[P];                 // all parts in flight (past the last one: the last one again)
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            const f32x4* from = reinterpret_cast<const f32x4*>(hp + (P > 1 ? min(p, a.parts - 1) : 0) * step);
                            h0[p] = from[0], h1[p] = from[1];
                        }
#pragma unroll
                        for (int p = 0; p < P; ++p)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                v[e] += P == 1 || p < a.parts ? h0[p][e] : 0.0f;
                                v[4 + e] += P == 1 || p < a.parts ? h1[p][e] : 0.0f;
                            }
                    }
                    bf16x8 h[3];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        float r = v[e] * s;
#pragma unroll
                        for (int t = 0; t < 3; ++t) {
                            h[t][e] = (__bf16)r;
                            r -= (float)h[t][e];
                        }
                    }
#pragma unroll
                    for (int e = 2; e >= 0; --e)
#pragma unroll
                        for (int t = 0; t < C; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(h[e], bw[q][t], acc[t], 0, 0, 0);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (__shfl(mine, 4 * g + e) != id) continue;
                YT* o = static_cast<YT*>(a.out) + (size_t)(row0 + 4 * g + e) * a.ldo + n;
                float v[C];
#pragma unroll
                for (int t = 0; t < C; ++t) v[t] = acc[t][e];
                if (whole) {
                    V w;
                    w.set(v);
                    if (a.past_cache) w.store_nt(o);
                    else *reinterpret_cast<V*>(o) = w;
                } else {
#pragma unroll
                    for (int t = 0; t < C; ++t)
                        if (n + t < a.N) put(o + t, (a.base ? value(base_row(row0 + 4 * g + e)[n + t]) : 0.0f) + v[t]);
                }
            }
        });
    }
}

// How a call is cut.  Up to 512 rows a tile's adapters are spread over workgroups, 64 / tiles at most.  Up to 64 rows, K is cut
// into parts so that there are about two workgroups of four waves to a compute unit if the rows of a tile share one or two
// adapters, at least 256 to a part.  More rows: workgroups of eight waves, and parts only as long as there is a compute unit
// for each, of 2048, or of 4096 where N is wide (each part of h is read again for every 256 columns): K 14336 with 16 x 4096
// at 256 rows 14.6 us in one part, 9.3 in four, 12.2 in eight of the small kind; K 4096 with 32 x 14336 at 256 rows
// 14.1 in one part, 15.9 in two, 26 in eight; at 64 rows the small kind 15.5 (K 14336, rank 64) beside 24.9.
struct Plan {
    int tiles, slots, parts, part_k;
    bool few;
};
Plan plan(int M, int K, int N, int adapters) {
    Plan p;
    p.few = M <= 64;
    p.tiles = (int)(((int64_t)M + 15) / 16);
    p.slots = M <= 512 ? 64 / p.tiles : 1;
    if (p.slots > 16) p.slots = 16;
    if (p.slots - 1 > adapters) p.slots = adapters + 1;     // (rows without an adapter count as one)
    const int least = p.few ? 256 : N / 2 > K ? 4096 : 2048, most = p.few ? kMaxParts : 4;
    int n = 256 / p.tiles;
    if (n > (K + least - 1) / least) n = (K + least - 1) / least;
    if (n > most) n = most;
    if (n < 1) n = 1;
    // whole steps of 64 for each of a workgroup's waves
    const int step = p.few && n > 1 ? 256 : 512;
    p.part_k = ((K + n - 1) / n + step - 1) / step * step;
    p.parts = (K + p.part_k - 1) / p.part_k;
    return p;
}

template <typename XT, int JT, int W>
hipError_t launch_shrink(const LoraArgs& a, unsigned grid, int dev, hipStream_t stream) {
    constexpr int lds = shrink_lds<XT, JT, W>();
    if constexpr (lds > 65536)
        if (hipError_t e = ensure_dynamic_lds<&shrink_kernel<XT, JT, W>>(dev, lds); e != hipSuccess) return e;
    shrink_kernel<XT, JT, W><<<grid, 64 * W, lds, stream>>>(a);
    return hipGetLastError();
}
template <typename XT>
hipError_t shrink(const LoraArgs& a, bool few, unsigned grid, int dev, hipStream_t stream) {
    if (a.rank > 64) return launch_shrink<XT, 8, 4>(a, grid, dev, stream);
    if (a.rank > 32) return few ? launch_shrink<XT, 4, 4>(a, grid, dev, stream) : launch_shrink<XT, 4, 8>(a, grid, dev, stream);
    if (a.rank > 16) return few ? launch_shrink<XT, 2, 4>(a, grid, dev, stream) : launch_shrink<XT, 2, 8>(a, grid, dev, stream);
    return few ? launch_shrink<XT, 1, 4>(a, grid, dev, stream) : launch_shrink<XT, 1, 8>(a, grid, dev, stream);
}

template <typename YT, int G>
hipError_t launch_expand(LoraArgs& a, const Plan& p, hipStream_t stream) {
    a.groups_n = (int)(((int64_t)a.N + 255) / 256);
    // a tile's adapters: spread over workgroups while there are fewer than four to a compute unit (333 rows in runs of 20
    // beside 3616 x 5000: 14.4 us with two to a tile, 16.9 with one; those that find no adapter are not free: 128 rows with
    // one adapter to a tile beside 4096 x 4096, this kernel 7.5 us with eight to a tile, 4.8 with one)
    const int64_t wide = (int64_t)p.tiles * a.groups_n;
    a.slots = wide >= 1024 ? 1 : (int)(1024 / wide < p.slots ? 1024 / wide : p.slots);
    // tiles of a workgroup: as many as leave eight workgroups to a compute unit, within 2^23 workgroups
    int64_t t = a.slots > 1 ? 1 : wide / 2048;
    if (t > 32) t = 32;
    if (t < wide / (1 << 22) + 1) t = wide / (1 << 22) + 1;
    a.tile_rows = (int)t;
    const unsigned grid = (unsigned)((p.tiles + t - 1) / t * a.slots * a.groups_n);
    if (p.parts > 4) expand_kernel<YT, G, kMaxParts><<<grid, 256, 0, stream>>>(a);
    else if (p.parts > 1) expand_kernel<YT, G, 4><<<grid, 256, 0, stream>>>(a);
    else expand_kernel<YT, G, 1><<<grid, 256, 0, stream>>>(a);
    return hipGetLastError();
}
template <typename YT>
hipError_t expand(LoraArgs& a, const Plan& p, hipStream_t stream) {
    if (a.rank <= 32) return launch_expand<YT, 1>(a, p, stream);
    if (a.rank <= 64) return launch_expand<YT, 2>(a, p, stream);
    return launch_expand<YT, 4>(a, p, stream);
}

}  // namespace

size_t lora_parts_bytes(int M, int K, int N, int rank, int adapters) {
    return M > 0 ? (size_t)plan(M, K, N, adapters).parts * M * rank * 4 : 0;
}

// Fewer rows can take more room, in more parts: the most that any call of at most M rows over at most K with at most `rank`
// takes.  The number of parts (at most that of plan() in front of its rounding, with the shorter least length of wide and narrow
// N) falls with the number of 16-row tiles only, so the most rows for each number are looked at.
size_t lora_workspace_bytes(int M, int K, int rank) {
    auto most = [&](int rows, int least, int parts) {
        const int n = (int)(((int64_t)K + least - 1) / least);
        return (size_t)(n < parts ? n : parts) * (rows < M ? rows : M);
    };
    size_t h = most(64, 256, kMaxParts);
    if (M > 64)
        for (int n = 4; n >= 1; --n) {
            const size_t x = most(n == 1 ? M : 256 / n * 16, 2048, n);
            if (x > h) h = x;
        }
    return M > 0 ? h * rank * 4 : 0;
}

hipError_t launch_lora_add(const void* X, batq_dtype xdtype, int M, int K, int64_t ldx, const void* A, const void* B,
                           int N, int rank, int adapters, const float* scales, const int32_t* index, const void* base,
                           int64_t ldb, void* out, int64_t ldo, batq_dtype ydtype, void* workspace, hipStream_t stream) {
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    const Plan p = plan(M, K, N, adapters);
    LoraArgs a = {};
    a.X = X, a.A = static_cast<const uint16_t*>(A), a.B = static_cast<const uint16_t*>(B), a.scales = scales, a.index = index;
    a.base = base, a.out = out, a.h = static_cast<float*>(workspace), a.ldx = ldx, a.ldb = ldb, a.ldo = ldo;
    a.M = M, a.K = K, a.N = N, a.rank = rank, a.adapters = adapters, a.slots = p.slots, a.parts = p.parts, a.part_k = p.part_k;
    const int64_t size = ydtype == BATQ_BF16 ? 2 : 4;
    a.vec = ((uintptr_t)out | (uintptr_t)base | (uintptr_t)(ldo * size) | (uintptr_t)(base ? ldb * size : 0)) % 16 == 0;
    // Non-temporal stores from 192 MiB of base and out on (three quarters of the memory-side cache): 4096 x 14336 in bf16
    // 69 -> 57 us and together with a reader of out right behind it 98 -> 97; at 8192 x 4096 (128 MiB) the reader pays for
    // them, 72 -> 79 together, and in place (112 MiB for 4096 x 14336) they change nothing.
    a.past_cache = (size_t)M * N * size * (base && base != out ? 2 : 1) > (size_t)192 << 20;
    const unsigned grid = (unsigned)p.tiles * p.slots * p.parts;
    if (hipError_t e = xdtype == BATQ_BF16 ? shrink<uint16_t>(a, p.few, grid, dev, stream) : shrink<float>(a, p.few, grid, dev, stream); e != hipSuccess)
        return e;
    return ydtype == BATQ_BF16 ? expand<uint16_t>(a, p, stream) : expand<float>(a, p, stream);
}

}  // namespace batq
