// Eviction from the paged cache: per sequence and key head the first tokens, the last ones and those with the largest scores
// between them stay, and move to fresh pages in their order.  gfx950 only.
#include "batq_internal.h"
#include "paged_device.h"

namespace batq {
namespace {

struct EvictArgs {
    const int32_t *kv_len, *page_table, *out_table;
    int batch, table_width, out_width, max_kv, num_pages, page_shift, kv_heads;
    int budget, first, last, chunks;
    float* score;
    int32_t *keep, *new_len;
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
};

__device__ __forceinline__ int tokens_of(const EvictArgs& a, int b) {
    return (int)min((int64_t)max(0, min(a.kv_len[b], a.max_kv)), (int64_t)a.table_width << a.page_shift);
}

// A score as an unsigned number of the same order; the smallest for NaN and for tokens of pages that do not exist.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);           // (-0 becomes 0)
    if (x != x) return 0u;
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

constexpr int kWaves = 16;

// A workgroup to a (sequence, key head): the k-th largest key by its bytes from the highest, each from a histogram of the
// keys that share the bytes above it, then one pass in order that lists what stays.
__global__ void __launch_bounds__(64 * kWaves)
select_kernel(const EvictArgs a) {
    __shared__ uint32_t s_hist[kWaves][256];
    __shared__ uint32_t s_prefix, s_left;
    __shared__ int s_gt[kWaves], s_eq[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int h = blockIdx.x % a.kv_heads, b = blockIdx.x / a.kv_heads;
    const int len = tokens_of(a, b), n = min(len, a.budget);
    int32_t* const keep = a.keep + (size_t)blockIdx.x * a.budget;
    if (h == 0 && tid == 0) a.new_len[b] = n;
    for (int j = n + tid; j < a.budget; j += 64 * kWaves) keep[j] = -1;
    if (n == len) {
        for (int j = tid; j < n; j += 64 * kWaves) keep[j] = j;
        return;
    }
    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1;
    auto key = [&](int t) -> uint32_t {
        const int page = table[t >> a.page_shift];
        if ((uint32_t)page >= (uint32_t)a.num_pages) return 0u;
        return order_of(a.score[(((int64_t)page * a.kv_heads + h) << a.page_shift) + (t & page_mask)]);
    };
    const int lo = a.first, hi = len - a.last;              // the tokens between them are chosen from: more than are kept
    uint32_t prefix = 0, left = a.budget - a.first - a.last;     // of the keys that begin with prefix, `left` stay
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = tid; i < kWaves * 256; i += 64 * kWaves) (&s_hist[0][0])[i] = 0u;
        __syncthreads();
        for (int t = lo + tid; t < hi; t += 64 * kWaves) {
            const uint32_t u = key(t);
            if (shift == 24 || (u >> (shift + 8)) == prefix) atomicAdd(&s_hist[wave][(u >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            uint32_t c[4] = {}, sum = 0;                    // lane's bins, from the largest: 255 - 4 lane ..
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                for (int w = 0; w < kWaves; ++w) c[i] += s_hist[w][255 - 4 * lane - i];
                sum += c[i];
            }
            uint32_t before = sum;                          // keys in larger bins than this lane's
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t v = __shfl_up(before, d);
                if (lane >= d) before += v;
            }
            before -= sum;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (before < left && before + c[i] >= left) s_prefix = prefix << 8 | (uint32_t)(255 - 4 * lane - i), s_left = left - before;
                before += c[i];
            }
            if (left == 0 && lane == 0) s_prefix = 0xFFFFFFFFu >> shift, s_left = 0;    // nothing is above it
        }
        __syncthreads();
        prefix = s_prefix, left = s_left;
    }
    const uint32_t border = prefix;                         // `left` of the keys that are equal to it stay, the first ones
    int at = 0, equal = 0;                                  // kept and equal ones so far
    for (int t0 = 0; t0 < len; t0 += 64 * kWaves) {
        const int t = t0 + tid;
        bool sure = t < len && (t < lo || t >= hi), eq = false;
        if (t < len && !sure) {
            const uint32_t u = key(t);
            sure = u > border, eq = u == border;
        }
        const uint64_t m_sure = __ballot(sure), m_eq = __ballot(eq);
        __syncthreads();
        if (lane == 0) s_gt[wave] = __builtin_popcountll(m_sure), s_eq[wave] = __builtin_popcountll(m_eq);
        __syncthreads();
        int mine = 0, mine_eq = 0;
        for (int w = 0; w < kWaves; ++w) {
            const int taken = max(0, min(s_eq[w], (int)left - equal));
            if (w == wave) mine = at, mine_eq = equal;
            at += s_gt[w] + taken, equal += s_eq[w];
        }
        const uint64_t below = (1ull << lane) - 1;
        const bool stays_eq = eq && mine_eq + __builtin_popcountll(m_eq & below) < (int)left;
        const uint64_t m = m_sure | __ballot(stays_eq);
        if (sure || stays_eq) keep[mine + __builtin_popcountll(m & below)] = t;
    }
}

constexpr int kMove = 64;                                   // tokens of a workgroup of the move

// Moves the listed tokens: keys, values, scales and score.
template <int D, int BITS>
__global__ void __launch_bounds__(256)
move_kernel(const EvictArgs a) {
    constexpr int kToken = D * BITS / 8, kCh = kToken / 16, kNb = D / 32;
    __shared__ int s_from[kMove], s_from_off[kMove], s_to[kMove], s_to_off[kMove];      // page, place in it
    const int tid = threadIdx.x;
    const int bh = blockIdx.x / a.chunks, j0 = (blockIdx.x % a.chunks) * kMove;
    const int h = bh % a.kv_heads, b = bh / a.kv_heads;
    const int n = min(tokens_of(a, b), a.budget);
    if (j0 >= n) return;
    const int page_mask = (1 << a.page_shift) - 1;
    if (tid < kMove) {
        const int j = j0 + tid;
        int from = -1, to = -1;
        if (j < n) {
            const int t = a.keep[(size_t)bh * a.budget + j];
            from = a.page_table[(size_t)b * a.table_width + (t >> a.page_shift)];
            to = a.out_table[(size_t)b * a.out_width + (j >> a.page_shift)];
            if ((uint32_t)from >= (uint32_t)a.num_pages || (uint32_t)to >= (uint32_t)a.num_pages) from = -1;
            s_from_off[tid] = t & page_mask, s_to_off[tid] = j & page_mask;
        }
        s_from[tid] = from, s_to[tid] = to;
    }
    __syncthreads();
    auto place = [&](int page, int off) { return (((int64_t)page * a.kv_heads + h) << a.page_shift) + off; };
    for (int i = tid; i < kMove * kCh; i += 256) {
        const int j = i / kCh, c = i % kCh;
        if (s_from[j] < 0) continue;
        const int64_t from = place(s_from[j], s_from_off[j]) * kToken + c * 16, to = place(s_to[j], s_to_off[j]) * kToken + c * 16;
        const u32x4 k = *reinterpret_cast<const u32x4*>(a.k_codes + from), v = *reinterpret_cast<const u32x4*>(a.v_codes + from);
        *reinterpret_cast<u32x4*>(a.k_codes + to) = k;
        *reinterpret_cast<u32x4*>(a.v_codes + to) = v;
    }
    for (int i = tid; i < kMove * kNb; i += 256) {
        const int j = i % kMove, blk = i / kMove;
        if (s_from[j] < 0) continue;
        const int64_t from = ((((int64_t)s_from[j] * a.kv_heads + h) * kNb + blk) << a.page_shift) + s_from_off[j];
        const int64_t to = ((((int64_t)s_to[j] * a.kv_heads + h) * kNb + blk) << a.page_shift) + s_to_off[j];
        const uint8_t k = a.k_scales[from], v = a.v_scales[from];
        a.k_scales[to] = k, a.v_scales[to] = v;
    }
    if (tid < kMove && s_from[tid] >= 0) a.score[place(s_to[tid], s_to_off[tid])] = a.score[place(s_from[tid], s_from_off[tid])];
}

template <int D, int BITS>
hipError_t launch_move(const EvictArgs& a, hipStream_t stream) {
    move_kernel<D, BITS><<<(unsigned)a.batch * a.kv_heads * a.chunks, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t paged_evict_workspace_bytes(const batq_paged_cache& c, int batch, int max_kv, int budget, int compute_units) { return 0; }

hipError_t launch_kv_paged_evict(const batq_paged_cache& c, int bits, float* score, const int32_t* kv_len, const int32_t* page_table,
                                 int table_width, const int32_t* out_table, int out_width, int batch, int max_kv, int budget,
                                 int first, int last, int32_t* keep, int32_t* new_len, void* workspace, hipStream_t stream) {
    EvictArgs a = {};
    a.kv_len = kv_len, a.page_table = page_table, a.out_table = out_table, a.batch = batch, a.table_width = table_width;
    a.out_width = out_width, a.max_kv = max_kv, a.num_pages = c.num_pages, a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.kv_heads = c.kv_heads, a.budget = budget, a.first = first, a.last = last;
    a.chunks = ((budget < max_kv ? budget : max_kv) + kMove - 1) / kMove;
    a.score = score, a.keep = keep, a.new_len = new_len;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales, a.v_codes = c.v_codes, a.v_scales = c.v_scales;
    select_kernel<<<(unsigned)batch * c.kv_heads, 64 * kWaves, 0, stream>>>(a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess || a.chunks == 0) return e;
    if (bits == 8) return c.head_dim == 64 ? launch_move<64, 8>(a, stream) : launch_move<128, 8>(a, stream);
    return c.head_dim == 64 ? launch_move<64, 4>(a, stream) : launch_move<128, 4>(a, stream);
}

}  // namespace batq
