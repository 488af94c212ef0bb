// Eviction from the paged cache: per sequence and key head the first tokens, the last ones and those with the largest scores
// between them stay, and move to fresh pages in their order.  gfx950 only.
#include "batq_internal.h"
#include "paged_device.h"

namespace batq {
namespace {

struct EvictArgs {
    const int32_t *kv_len, *page_table, *out_table;
    const int32_t* score_table;                             // pages of the scores; page_table where they are those of the keys
    int batch, table_width, out_width, max_kv, num_pages, score_pages, page_shift, kv_heads;
    int budget, first, last, chunks;
    float* score;
    int32_t *keep, *new_len;
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    int team_chunks;                                        // of a (sequence, key head), where several workgroups choose
    uint32_t* team;                                         // [sequence][key head][3][kBins] histograms
    int2* team_counts;                                      // [sequence][key head][chunk] keys above the border, on it
};

__device__ __forceinline__ int tokens_of(const EvictArgs& a, int b) {
    return (int)min((int64_t)max(0, min(a.kv_len[b], a.max_kv)), (int64_t)a.table_width << a.page_shift);
}

// A score as an unsigned number of the same order; the smallest for NaN and for tokens whose page, or page of scores, does not exist.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);           // (-0 becomes 0)
    if (x != x) return 0u;
    return u ^ ((u >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

// The border between what stays and what goes is the k-th largest key, found eleven bits at a time from the highest: a histogram
// of the keys that begin with the bits found so far, and the bin in which the k-th is.  Equal keys stay in the order of their tokens.
constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048, kCopies = 8;
__device__ __forceinline__ int shift_of(int pass) { return pass == 0 ? 21 : pass == 1 ? 10 : 0; }
__device__ __forceinline__ uint32_t bin_of(uint32_t key, int pass) { return (key >> shift_of(pass)) & (pass == 2 ? 1023u : 2047u); }
// Whether a key begins with the bits found before the pass.
__device__ __forceinline__ bool begins(uint32_t key, uint32_t found, int pass) { return pass == 0 || ((key ^ found) >> shift_of(pass - 1)) == 0; }

// The bits found so far and how many of the keys that begin with them stay, of how many there are.
struct Found {
    uint32_t bits, left, all;
};

// Sum of the waves' numbers before this one's.
__device__ __forceinline__ int waves_before(const int* x, int wave) {
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kWaves / 4; ++i) {
        const int4 v = reinterpret_cast<const int4*>(x)[i];
        sum += (4 * i < wave ? v.x : 0) + (4 * i + 1 < wave ? v.y : 0) + (4 * i + 2 < wave ? v.z : 0) + (4 * i + 3 < wave ? v.w : 0);
    }
    return sum;
}

// Of the bins' counts (thread i: bins 2047 - 2i and 2046 - 2i in c) the one with the left-th key from the largest, by a workgroup.
__device__ __forceinline__ Found pick_bin(uint32_t c0, uint32_t c1, Found f, int pass) {
    __shared__ __align__(16) int s_sum[kWaves];
    __shared__ Found s_found;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    uint32_t upto = c0 + c1;                                // keys in this thread's bins and larger ones of the wave
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t v = __shfl_up(upto, d);
        if (lane >= d) upto += v;
    }
    if (lane == 63) s_sum[wave] = (int)upto;
    __syncthreads();
    uint32_t before = upto - c0 - c1 + (uint32_t)waves_before(s_sum, wave);
    const uint32_t top = kBins - 1 - 2 * tid;
    if (before < f.left && before + c0 >= f.left) s_found = Found{f.bits | top << shift_of(pass), f.left - before, c0};
    before += c0;
    if (before < f.left && before + c1 >= f.left) s_found = Found{f.bits | (top - 1) << shift_of(pass), f.left - before, c1};
    __syncthreads();
    return s_found;
}

// A (sequence, key head)'s tokens and their keys, four neighbours at a time (a page holds a multiple of them): the order of the scores,
// with the largest key of all for the first and the last tokens, which stay in any case.
struct Tokens {
    const int32_t *table, *score_table;
    const float* score;
    int len, first, hi;                                     // tokens [first, hi) are chosen from
    int h, num_pages, score_pages, kv_heads, page_shift;
    // Behind the last token come the smallest keys: there are more tokens than stay, so that none of them is reached.
    __device__ __forceinline__ u32x4 keys(int t) const {
        typedef float f32x4 __attribute__((ext_vector_type(4), aligned(4)));
        u32x4 u = {0u, 0u, 0u, 0u};
        if (t >= len) return u;
        const int page = score_table[t >> page_shift];
        bool there = (uint32_t)page < (uint32_t)score_pages;
        if (score_table != table) there = there && (uint32_t)table[t >> page_shift] < (uint32_t)num_pages;      // (always looked at: 1.5 us of 28)
        const f32x4 v = *reinterpret_cast<const f32x4*>(score + (((int64_t)(there ? page : 0) * kv_heads + h) << page_shift) + (t & ((1 << page_shift) - 1)));
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = there ? order_of(v[e]) : 0u;
        if (t < first || t + 4 > hi)
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = t + e >= len ? 0u : t + e < first || t + e >= hi ? 0xFFFFFFFFu : u[e];
        return u;
    }
};
__device__ __forceinline__ Tokens tokens_of_pair(const EvictArgs& a, int pair) {
    const int h = pair % a.kv_heads, b = pair / a.kv_heads, len = tokens_of(a, b);
    const size_t row = (size_t)b * a.table_width;
    const bool same = a.score_table == a.page_table;        // (pages below num_pages alone then have tokens)
    return Tokens{a.page_table + row, a.score_table + row, a.score, len, a.first, len - a.last, h, a.num_pages, same ? a.num_pages : a.score_pages, a.kv_heads, a.page_shift};
}

// The length, the end of the list, and all of it for a sequence that stays whole, by one workgroup of a pair.  Returns whether that is all.
__device__ __forceinline__ bool list_whole(const EvictArgs& a, const Tokens& x, int pair) {
    int32_t* const keep = a.keep + (size_t)pair * a.budget;
    const int n = min(x.len, a.budget);
    if (x.h == 0 && threadIdx.x == 0) a.new_len[pair / a.kv_heads] = n;
    for (int j = n + threadIdx.x; j < a.budget; j += kThreads) keep[j] = -1;
    if (n < x.len) return false;
    for (int j = threadIdx.x; j < n; j += kThreads) keep[j] = j;
    return true;
}

__device__ __forceinline__ void count_bins(const u32x4& u, uint32_t found, int pass, uint32_t* hist) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (begins(u[e], found, pass)) atomicAdd(&hist[bin_of(u[e], pass) * kCopies + (threadIdx.x & (kCopies - 1))], 1u);
}
__device__ __forceinline__ void clear_bins(uint32_t* hist) {
    for (int i = threadIdx.x; i < kBins * kCopies / 4; i += kThreads) reinterpret_cast<u32x4*>(hist)[i] = u32x4{0u, 0u, 0u, 0u};
}
__device__ __forceinline__ uint32_t bin_count(const uint32_t* hist, int bin) {
    const u32x4* p = reinterpret_cast<const u32x4*>(hist + bin * kCopies);
    const u32x4 v = p[0] + p[1];
    return v[0] + v[1] + v[2] + v[3];
}

// A lane's keys above the border, and on it.
__device__ __forceinline__ void count_keys(const u32x4& u, uint32_t border, int* gt, int* eq) {
#pragma unroll
    for (int e = 0; e < 4; ++e) *gt += u[e] > border, *eq += u[e] == border;
}
__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}
// The sum of a number of 0 to 4 over the lanes before this one; over all of them in *all.
__device__ __forceinline__ int sum_before(int c, int* all) {
    int before = 0;
    *all = 0;
#pragma unroll
    for (int bit = 0; bit < 3; ++bit) {
        const uint64_t m = __ballot((c >> bit) & 1);
        before += (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u)) << bit;
        *all += __builtin_popcountll(m) << bit;
    }
    return before;
}
// 256 keys of a wave in order (lane l has tokens t .. t + 3): lists those above the border and, of those on it, the ones with fewer than
// `left` before them.  (More than `budget` only if scores or workspace are written to meanwhile: not behind the list then either.)
__device__ __forceinline__ void list_keys(const u32x4& u, int t, uint32_t border, int left, int* at, int* equal, int32_t* keep, int budget) {
    bool stays[4], on = false;
    int c = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) stays[e] = u[e] > border, on = on || u[e] == border;
    if (*equal < left && __ballot(on)) {
        int ties = 0, all;
#pragma unroll
        for (int e = 0; e < 4; ++e) ties += u[e] == border;
        int rank = *equal + sum_before(ties, &all);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (u[e] == border) stays[e] = rank++ < left;
        *equal += all;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) c += stays[e];
    int all;
    const int before = sum_before(c, &all), begin = __builtin_amdgcn_readfirstlane(*at);
    *at += all;
    if (begin < 0 || begin > budget - all) return;
    int32_t* to = keep + begin + before;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (stays[e]) *to++ = t + e;
}

// A workgroup to a (sequence, key head): latencies and the vector instructions of one compute unit (32 pairs of 32768 tokens 23 us, 512 of 2112
// 16.6 us; read in every pass, key by key, 99 us).  KEYS > 0: up to KEYS keys a thread, read once and held in registers; 0: read in every pass.
// A wave has a run of neighbouring tokens.  Copies of the histogram keep lanes with equal bits apart (most scores share their exponent).
template <int KEYS>
__global__ void __launch_bounds__(kThreads)
select_kernel(const EvictArgs a) {
    __shared__ uint32_t s_hist[kBins * kCopies];
    __shared__ __align__(16) int s_gt[kWaves], s_eq[kWaves];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pair = blockIdx.x;
    const Tokens x = tokens_of_pair(a, pair);
    const int run = KEYS ? KEYS / 4 : (x.len + 4 * kThreads - 1) / (4 * kThreads), t0 = wave * run * 256 + 4 * lane;      // of 256 tokens
    u32x4 held[KEYS ? KEYS / 4 : 1];
    if constexpr (KEYS > 0)
#pragma unroll
        for (int k = 0; k < KEYS / 4; ++k) held[k] = x.keys(t0 + 256 * k);
    if (list_whole(a, x, pair)) return;
    auto each = [&](auto f) {                               // f(keys, token)
        if constexpr (KEYS > 0) {
#pragma unroll
            for (int k = 0; k < KEYS / 4; ++k) f(held[k], t0 + 256 * k);
        } else {
            for (int k = 0; k < run; ++k) f(x.keys(t0 + 256 * k), t0 + 256 * k);
        }
    };
    Found f = {0u, (uint32_t)a.budget, 0u};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        if (f.left == f.all) break;                         // (all of them stay: the border is right below their bits)
        clear_bins(s_hist);
        __syncthreads();
        each([&](const u32x4& u, int) { count_bins(u, f.bits, pass, s_hist); });
        __syncthreads();
        f = pick_bin(bin_count(s_hist, kBins - 1 - 2 * tid), bin_count(s_hist, kBins - 2 - 2 * tid), f, pass);
    }
    if (f.left == f.all) f = Found{f.bits - 1, 0u, 0u};      // (not 0: below the largest `budget` keys there are others)
    const int left = (int)f.left;
    int gt = 0, eq = 0;
    each([&](const u32x4& u, int) { count_keys(u, f.bits, &gt, &eq); });
    gt = wave_sum(gt), eq = wave_sum(eq);
    if (lane == 0) s_gt[wave] = gt, s_eq[wave] = eq;
    __syncthreads();
    int equal = waves_before(s_eq, wave), at = waves_before(s_gt, wave) + min(equal, left);
    int32_t* const keep = a.keep + (size_t)pair * a.budget;
    each([&](const u32x4& u, int t) { list_keys(u, t, f.bits, left, &at, &equal, keep, a.budget); });
}

// Long sequences of few pairs: a workgroup to a chunk of tokens, with a launch for every pass.  The histograms of all passes and the
// chunks' counts are in the workspace; every workgroup picks the passes' bins again.  8 pairs of 131072 tokens: 30 us of six launches (one
// workgroup each: 360); 32 pairs of 32768 are as fast with one workgroup each.
constexpr int kChunkKeys = 8, kChunk = kThreads * kChunkKeys, kTeamWords = 3 * kBins;

__device__ __forceinline__ Found found_before(const EvictArgs& a, int pair, int passes) {
    Found f = {0u, (uint32_t)a.budget, 0u};
    uint2 c[3];
#pragma unroll
    for (int p = 0; p < 3; ++p)                             // (bins 2046 - 2i and 2047 - 2i)
        if (p < passes) c[p] = *reinterpret_cast<const uint2*>(a.team + (size_t)pair * kTeamWords + p * kBins + kBins - 2 - 2 * threadIdx.x);
#pragma unroll
    for (int p = 0; p < 3; ++p)
        if (p < passes) f = pick_bin(c[p].y, c[p].x, f, p);
    return f;
}

__global__ void __launch_bounds__(256)
team_clear(const EvictArgs a) {
    const size_t n = (size_t)a.batch * a.kv_heads * kTeamWords / 4;
    for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256)
        reinterpret_cast<u32x4*>(a.team)[i] = u32x4{0u, 0u, 0u, 0u};
}

__global__ void __launch_bounds__(kThreads)
team_histogram(const EvictArgs a, int pass) {
    __shared__ uint32_t s_hist[kBins * kCopies];
    const int tid = threadIdx.x, pair = blockIdx.x / a.team_chunks, chunk = blockIdx.x % a.team_chunks;
    const Tokens x = tokens_of_pair(a, pair);
    if (pass == 0 && chunk == 0) list_whole(a, x, pair);
    const int t0 = chunk * kChunk + (tid >> 6) * kChunkKeys * 64 + 4 * (tid & 63);
    if (x.len <= a.budget || chunk * kChunk >= x.len) return;
    u32x4 u[kChunkKeys / 4];
#pragma unroll
    for (int k = 0; k < kChunkKeys / 4; ++k) u[k] = x.keys(t0 + 256 * k);
    clear_bins(s_hist);
    const Found f = found_before(a, pair, pass);
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kChunkKeys / 4; ++k) count_bins(u[k], f.bits, pass, s_hist);
    __syncthreads();
    uint32_t* const hist = a.team + (size_t)pair * kTeamWords + pass * kBins;
#pragma unroll
    for (int e = 0; e < 2; ++e)
        if (const uint32_t c = bin_count(s_hist, tid + e * kThreads)) atomicAdd(&hist[tid + e * kThreads], c);
}

// LIST false: counts each chunk's keys above the border and on it; true: lists what stays.
template <bool LIST>
__global__ void __launch_bounds__(kThreads)
team_list(const EvictArgs a) {
    __shared__ __align__(16) int s_gt[kWaves], s_eq[kWaves], s_before[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pair = blockIdx.x / a.team_chunks, chunk = blockIdx.x % a.team_chunks;
    const Tokens x = tokens_of_pair(a, pair);
    if (x.len <= a.budget || chunk * kChunk >= x.len) return;
    const int t0 = chunk * kChunk + wave * kChunkKeys * 64 + 4 * lane;
    u32x4 u[kChunkKeys / 4];
#pragma unroll
    for (int k = 0; k < kChunkKeys / 4; ++k) u[k] = x.keys(t0 + 256 * k);
    int2* const counts = a.team_counts + (size_t)pair * a.team_chunks;
    int g = 0, e = 0;
    if (LIST && wave == 0)
        for (int c = lane; c < chunk; c += 64) g += counts[c].x, e += counts[c].y;
    const Found f = found_before(a, pair, 3);
    const int left = (int)f.left;
    int gt = 0, eq = 0;
#pragma unroll
    for (int k = 0; k < kChunkKeys / 4; ++k) count_keys(u[k], f.bits, &gt, &eq);
    gt = wave_sum(gt), eq = wave_sum(eq);
    if (lane == 0) s_gt[wave] = gt, s_eq[wave] = eq;
    if (LIST && wave == 0) {                                // of the chunks before this one
#pragma unroll
        for (int d = 32; d; d >>= 1) g += __shfl_xor(g, d), e += __shfl_xor(e, d);
        if (lane == 0) s_before[0] = g, s_before[1] = e;
    }
    __syncthreads();
    if constexpr (!LIST) {
        if (tid == 0) {
            int2 c = {0, 0};
            for (int w = 0; w < kWaves; ++w) c.x += s_gt[w], c.y += s_eq[w];
            counts[chunk] = c;
        }
    } else {
        int equal = s_before[1] + waves_before(s_eq, wave), at = s_before[0] + waves_before(s_gt, wave) + min(equal, left);
        int32_t* const keep = a.keep + (size_t)pair * a.budget;
#pragma unroll
        for (int k = 0; k < kChunkKeys / 4; ++k) list_keys(u[k], t0 + 256 * k, f.bits, left, &at, &equal, keep, a.budget);
    }
}

constexpr int kMove = 64;                                   // tokens of a workgroup of the move

// Moves the listed tokens: keys, values, scales and score (0 for one without a page of scores).  Bound by the copy: 64 x 8 x 2048 tokens of 128 channels in 8 bits 116 us (562 MB in and
// out, 4.9 TB/s, a large copy's rate).
template <int D, int BITS>
__global__ void __launch_bounds__(256)
move_kernel(const EvictArgs a) {
    constexpr int kToken = D * BITS / 8, kCh = kToken / 16, kNb = D / 32;
    __shared__ int s_from[kMove], s_from_off[kMove], s_to[kMove], s_to_off[kMove], s_score[kMove];      // page, place in it; page of the score
    const int tid = threadIdx.x;
    const int bh = blockIdx.x / a.chunks, j0 = (blockIdx.x % a.chunks) * kMove;
    const int h = bh % a.kv_heads, b = bh / a.kv_heads;
    const int len = tokens_of(a, b), n = min(len, a.budget);
    if (j0 >= n) return;
    const int page_mask = (1 << a.page_shift) - 1;
    if (tid < kMove) {
        const int j = j0 + tid;
        int from = -1, to = -1;
        if (j < n) {
            const int t = min((uint32_t)a.keep[(size_t)bh * a.budget + j], (uint32_t)len - 1);      // (the caller's memory: not trusted)
            const size_t entry = (size_t)b * a.table_width + (t >> a.page_shift);
            from = a.page_table[entry];
            s_score[tid] = a.score_table[entry];
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
    if (tid < kMove && s_from[tid] >= 0)
        a.score[place(s_to[tid], s_to_off[tid])] = (uint32_t)s_score[tid] < (uint32_t)a.score_pages ? a.score[place(s_score[tid], s_from_off[tid])] : 0.0f;
}

template <int D, int BITS>
hipError_t launch_move(const EvictArgs& a, hipStream_t stream) {
    move_kernel<D, BITS><<<(unsigned)a.batch * a.kv_heads * a.chunks, 256, 0, stream>>>(a);
    return hipGetLastError();
}

// Whether several workgroups choose for a (sequence, key head): where a workgroup's registers do not hold its keys and there are
// too few pairs to fill the card.
constexpr int kHeldKeys = 32;
bool teams(int64_t pairs, int max_kv, int compute_units) { return max_kv > kHeldKeys * kThreads && pairs < 4 * compute_units; }

int64_t team_bytes(int64_t pairs, int max_kv) {
    return pairs * (kTeamWords * 4 + (int64_t)((max_kv + kChunk - 1) / kChunk) * 8);
}

hipError_t launch_select(const EvictArgs& a, bool team, hipStream_t stream) {
    const unsigned pairs = (unsigned)a.batch * a.kv_heads;
    if (team) {
        team_clear<<<(unsigned)((size_t)pairs * kTeamWords / 4 / 256), 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        for (int pass = 0; pass < 3; ++pass) {
            team_histogram<<<pairs * a.team_chunks, kThreads, 0, stream>>>(a, pass);
            if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        }
        team_list<false><<<pairs * a.team_chunks, kThreads, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
        team_list<true><<<pairs * a.team_chunks, kThreads, 0, stream>>>(a);
    } else if (a.max_kv <= 4 * kThreads) {
        select_kernel<4><<<pairs, kThreads, 0, stream>>>(a);
    } else if (a.max_kv <= 16 * kThreads) {
        select_kernel<16><<<pairs, kThreads, 0, stream>>>(a);
    } else if (a.max_kv <= kHeldKeys * kThreads) {
        select_kernel<kHeldKeys><<<pairs, kThreads, 0, stream>>>(a);
    } else {
        select_kernel<0><<<pairs, kThreads, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace

size_t paged_evict_part_bytes(const batq_paged_cache& c, int batch, int max_kv, int compute_units) {
    const int64_t pairs = (int64_t)batch * c.kv_heads;
    return teams(pairs, max_kv, compute_units) ? (size_t)team_bytes(pairs, max_kv) : 0;
}

// At least the former for every smaller call: of up to as many pairs as teams are used for.
size_t paged_evict_workspace_bytes(const batq_paged_cache& c, int batch, int max_kv, int compute_units) {
    int64_t pairs = (int64_t)batch * c.kv_heads;
    if (pairs >= 4 * compute_units) pairs = 4 * compute_units - 1;
    return teams(pairs, max_kv, compute_units) ? (size_t)team_bytes(pairs, max_kv) : 0;
}

hipError_t launch_kv_paged_evict(const batq_paged_cache& c, int bits, float* score, const int32_t* score_table, int score_pages,
                                 const int32_t* kv_len, const int32_t* page_table, int table_width, const int32_t* out_table, int out_width, int batch, int max_kv, int budget,
                                 int first, int last, int32_t* keep, int32_t* new_len, void* workspace, hipStream_t stream) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const int cus = e == hipSuccess ? device_compute_units(dev, &e) : 0;
    if (e != hipSuccess) return e;
    EvictArgs a = {};
    a.kv_len = kv_len, a.page_table = page_table, a.out_table = out_table, a.batch = batch, a.table_width = table_width;
    a.out_width = out_width, a.max_kv = max_kv, a.num_pages = c.num_pages, a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.kv_heads = c.kv_heads, a.budget = budget, a.first = first, a.last = last;
    a.chunks = ((budget < max_kv ? budget : max_kv) + kMove - 1) / kMove;
    a.score_table = score_table ? score_table : page_table, a.score_pages = score_pages;
    a.score = score, a.keep = keep, a.new_len = new_len;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales, a.v_codes = c.v_codes, a.v_scales = c.v_scales;
    const int64_t pairs = (int64_t)batch * c.kv_heads;
    a.team_chunks = (max_kv + kChunk - 1) / kChunk;
    a.team = static_cast<uint32_t*>(workspace), a.team_counts = reinterpret_cast<int2*>(a.team + pairs * kTeamWords);
    if (e = launch_select(a, teams(pairs, max_kv, cus), stream); e != hipSuccess || a.chunks == 0) return e;
    if (bits == 8) return c.head_dim == 64 ? launch_move<64, 8>(a, stream) : launch_move<128, 8>(a, stream);
    return c.head_dim == 64 ? launch_move<64, 4>(a, stream) : launch_move<128, 4>(a, stream);
}

}  // namespace batq
