// What the cached tokens have received of the attention: for each key head and token t the softmax weights
// exp(scale q_i k_t - lse_i) of the batch's queries, summed over the queries i that see t and the query heads that read the
// key head.  gfx950 only.
//
// Sums belong to tokens, so a workgroup has tokens and walks rows (row = query token * group + head of the group): no two
// workgroups add to the same place where every sequence has score pages of its own, and the order of a sum follows from the
// call's sizes alone.
#include <math.h>

#include <type_traits>

#include "batq_internal.h"
#include "mxfp4_device.h"
#include "paged_device.h"

namespace batq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

struct ScoreArgs : PagedLists {
    const uint16_t* q;
    int64_t ldq;
    const float* lse;
    const uint8_t *k_codes, *k_scales;
    float* score;
    const int32_t* score_table;                             // pages of the scores; page_table where they are those of the keys
    int score_pages;
    float scale;                                            // times log2 e
    int add;
    // sequences of at most few_rows rows belong to score_few, in parts of few_len tokens, the others to score_many
    int few_rows, few_len, few_parts;
    int key_tiles, chunk, parts;                            // tiles of kTileTokens; parts of `chunk` rows
    float* part;                                            // [sequence][key head][key tile][part][token of the tile]
};

// The subtrahend of a row's exponents; a row that has seen nothing has no weights.
__device__ __forceinline__ float ref_of(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f; }

// Places of tokens before this one are not written: with `add`, those of old tokens that no query sees (pages that a sequence has
// given back behind its window may be another one's).
__device__ __forceinline__ int kept_below(const ScoreArgs& a, const Seq& s) { return !a.add ? 0 : s.n ? s.t_lo : s.first_pos; }

// Stores a sum: `v` for token t of the sequence.
__device__ __forceinline__ void store_score(const ScoreArgs& a, const Seq& s, int b, int h, int t, float v) {
    if (t < kept_below(a, s) || t >= s.len) return;
    const size_t entry = (size_t)b * a.table_width + (t >> a.page_shift);
    const int page = a.score_table[entry];
    if ((uint32_t)page >= (uint32_t)a.score_pages || (uint32_t)a.page_table[entry] >= (uint32_t)a.num_pages) return;
    float* to = a.score + ((((int64_t)page * a.kv_heads + h) << a.page_shift) + (t & ((1 << a.page_shift) - 1)));
    if (a.add && t < s.first_pos) v += *to;
    *to = v;
}

// Few rows to a key head (decoding): bound by the stream of key codes, read once (64 x 8192 tokens of 8 heads of 128 channels in 4 bits:
// 302 MB in 60 us, 5.0 TB/s), and for ragged sequences by a part's chain of loads (64 of up to 8192 tokens: 35 MB in 21 us; parts of 256, 512
// tokens 26, 22 us there, but 86, 69 us for 64 x 8192; tokens shared out evenly over all workgroups 23 and 90: more registers, fewer waves;
// requested one, two, three blocks ahead 24, 21.7, 22.9).  A workgroup takes a part of one (sequence, key
// head), its four waves blocks of 32 tokens in turn.  S = Q K^T with the queries' operands in registers: lane (n, g) =
// (l % 16, l / 16) loads channels [g D/4, (g + 1) D/4) of tokens 2n and 2n + 1 (the order in which a product runs over channels is
// free), and element r of its results of tile x is row 16x + 4g + r: a token's sum is one over elements and four lanes.
// Blocks that no row sees are left out (64 x 8192 tokens behind a window of 1024: 17 us beside 65; 1 x 131072: 9.6 beside 19).
// OWN: with a table of the scores' pages (ragged batch 19.8 us beside 19.5 in a graph; looked at in one kernel for both, calls without one
// took 22.8 instead of 20.6).
template <int D, int NT, int BITS, bool OWN>
__global__ void __launch_bounds__(256)
score_few(const ScoreArgs a) {
    constexpr int kC = D / 4, kU = D / 32, kToken = D * BITS / 8, kKw = kC * BITS / 32, kStages = 2;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    // the first parts of all sequences, then the second ones ..: short sequences have few, and workgroups go to the dies in turn
    const int pairs = a.batch * a.kv_heads, part = blockIdx.x / pairs, bh = blockIdx.x - part * pairs;
    const int h = bh % a.kv_heads, b = bh / a.kv_heads;
    const Seq s = sequence(a, b);
    const int rows = s.n * a.group;
    const int t_begin = part * a.few_len, t_end = min(s.len, t_begin + a.few_len);
    if (rows > a.few_rows || t_begin >= t_end) return;
    // blocks of 32 tokens with one that some row sees: [b_lo, b_hi); the others' sums are zero
    const int b_lo = min(t_end, t_begin + (max(0, s.t_lo - t_begin) & ~31)), b_hi = s.n ? max(b_lo, min(t_end, s.t_hi)) : b_lo;
    for (int t = t_begin + threadIdx.x; t < b_lo; t += 256) store_score(a, s, b, h, t, 0.0f);
    for (int t = b_lo + ((b_hi - b_lo + 31) & ~31) + threadIdx.x; t < t_end; t += 256) store_score(a, s, b, h, t, 0.0f);
    if (b_lo == b_hi) return;

    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1, last_page = (s.len - 1) >> a.page_shift;
    // lane i holds the page of tokens t_begin + 16 i .. + 15 (a part is at most 1024 long)
    const int entry = min((t_begin + 16 * lane) >> a.page_shift, last_page), pages = table[entry];
    const int score_pages = OWN ? a.score_table[(size_t)b * a.table_width + entry] : 0;
    // blocks t, t + 128, .. are requested kStages ahead
    uint32_t kw[kStages][2][kKw];
    uint32_t ks[kStages];
    f32x2 old[kStages];
    float* to[kStages];
    bool there[kStages];
    auto request = [&](int t, int st) {
        t += 2 * n;
        int page = __shfl(pages, (t - t_begin) >> 4);
        there[st] = (uint32_t)page < (uint32_t)a.num_pages;
        page = there[st] ? page : 0;
        const int off = t & page_mask;
        const int64_t ph = (int64_t)page * a.kv_heads + h;
        const uint8_t* p = a.k_codes + ((ph << a.page_shift) + off) * kToken + g * (kToken / 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) load_words<kKw>(kw[st][i], p + i * kToken);
        ks[st] = *reinterpret_cast<const uint16_t*>(a.k_scales + ((ph * (D / 32) + g * kC / 32) << a.page_shift) + off);
        int64_t score_ph = ph;
        if constexpr (OWN) {
            const int score_page = __shfl(score_pages, (t - t_begin) >> 4);
            const bool known = (uint32_t)score_page < (uint32_t)a.score_pages;
            there[st] = there[st] && known;
            score_ph = (int64_t)(known ? score_page : 0) * a.kv_heads + h;
        }
        to[st] = a.score + (score_ph << a.page_shift) + off;
        if (a.add) old[st][0] = to[st][0], old[st][1] = to[st][1];      // (a page holds an even number of tokens)
    };
    int t = b_lo + wave * 32;
#pragma unroll
    for (int st = 0; st < kStages; ++st)
        if (t + 128 * st < b_hi) request(t + 128 * st, st);

    bf16x8 qf[NT][kU];
    float ref[NT][4];
    int lo[NT][4], hi[NT][4];                               // tokens [lo, hi) are visible to row 16x + 4g + r
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        const int row = min(x * 16 + n, rows - 1), i = row / a.group;
        const uint16_t* p = a.q + (size_t)(s.begin + i) * a.ldq + (size_t)(h * a.group + row - i * a.group) * D + g * kC;
#pragma unroll
        for (int u = 0; u < kU; ++u) qf[x][u] = *reinterpret_cast<const bf16x8*>(p + 8 * u);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int rr = x * 16 + 4 * g + r, ii = rr / a.group, pos = s.first_pos + ii;
            const bool live = rr < rows;
            ref[x][r] = live ? ref_of(a.lse[(size_t)(s.begin + ii) * a.q_heads + h * a.group + rr - ii * a.group]) : INFINITY;
            hi[x][r] = !live ? 0 : a.causal ? min(s.len, pos + 1) : s.len;
            lo[x][r] = first_seen(a, pos);
        }
    }
    // blocks in [all_lo, all_hi) are seen whole by every row
    const bool full = rows == NT * 16;
    const int all_hi = !full ? 0 : a.causal ? min(s.len, s.first_pos + 1) : s.len;
    const int all_lo = first_seen(a, s.first_pos + s.n - 1);
    const int kept = kept_below(a, s);                      // (below t_end, or no row would see a token of the part)
    const uint32_t places = (uint32_t)(t_end - kept);
    while (t < b_hi)
#pragma unroll
    for (int st = 0; st < kStages; ++st) {
        if (st > 0 && t >= b_hi) break;
        f32x4 sc[NT][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float kscale = scale_operand((ks[st] >> (8 * i)) & 0xFFu);
            bf16x8 kf[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) kf[u] = cvt_eight<BITS>(kw[st][i] + u * BITS / 4, kscale);
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                sc[x][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < kU; ++u) sc[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[x][u], kf[u], sc[x][i], 0, 0, 0);
            }
        }
        float* const at = to[st];
        const f32x2 had = old[st];
        const bool stored = there[st];
        if (t + 128 * kStages < b_hi) request(t + 128 * kStages, st);
        const bool whole = t >= all_lo && t + 32 <= all_hi;
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int x = 0; x < NT; ++x)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    float w = exp2_(__builtin_fmaf(sc[x][i][r], a.scale, -ref[x][r]));
                    if (!whole) {
                        const int tok = t + 2 * n + i;
                        const int hide = ((tok - lo[x][r]) | (hi[x][r] - 1 - tok)) >> 31;
                        w = __uint_as_float(__float_as_uint(w) & ~(uint32_t)hide);
                    }
                    sum[i] += w;
                }
            sum[i] = total(across32(total(across16(sum[i]))));
        }
        if (g == 0 && stored) {
            const int tok = t + 2 * n;
            const f32x2 v = {sum[0] + (a.add && tok < s.first_pos ? had[0] : 0.0f), sum[1] + (a.add && tok + 1 < s.first_pos ? had[1] : 0.0f)};
            if ((uint32_t)(tok - kept) < places) at[0] = v[0];
            if ((uint32_t)(tok + 1 - kept) < places) at[1] = v[1];
        }
        t += 128;
    }
}

// Many rows (prompts, their last queries): bound by the vector instructions around the exponentials (32 exponentials at half rate, 64 others: 512
// clocks of a SIMD for 32 rows x 64 tokens, as many as the products take), with the products beside them: a prompt of 8192 tokens of 32 and 8 heads
// of 128 channels 340 us (800 TFLOP/s; 1000 without causal), the last 64 queries of four of 32768 tokens, 28 and 4 heads, 53 us.  Weights formed
// behind their own products instead of between the next ones: 400 and 57 us; three waves per SIMD instead of two spill (429).  A
// workgroup has 256 tokens, 64 to a wave, whose keys stay in registers as operands, and walks its part of the rows that may see
// them 64 at a time; they go through LDS, two buffers, requested a stage ahead.  S^T = K Q^T, so that a lane adds the weights
// of its rows up token by token; the lanes' sums are added at the end.  Lane (n, h) = (l % 32, l / 32) holds channels
// [h D/2, (h + 1) D/2) of token n of either half and of row n; result element e of half x is token 32x + 8 (e / 4) + 4h + e % 4.
// A chunk of 8 channels has its place in a row of LDS XORed with the row's number, so that 16 lanes reach all banks.
constexpr int kTileTokens = 256, kStageRows = 64, kDeep = 4;

template <int D>
__device__ __forceinline__ int q_place(int row, int chunk) { return D == 128 ? chunk ^ (row & 15) : chunk ^ ((row >> 1) & 7); }

// Rows of a sequence that may see a token of a key tile: [lo, hi), and the parts among them: those that begin below hi and end
// behind lo.
struct RowRange {
    int lo, hi;
};
__device__ __forceinline__ RowRange tile_rows(const ScoreArgs& a, const Seq& s, int t0) {
    const int last = min(t0 + kTileTokens, s.len) - 1;
    const int64_t i_lo = a.causal ? max(0, t0 - s.first_pos) : 0;
    const int64_t i_hi = a.window ? max((int64_t)0, min((int64_t)s.n, (int64_t)last + a.window - s.first_pos)) : s.n;
    return RowRange{(int)i_lo * a.group, (int)i_hi * a.group};
}

// The sequence and key tile of number `x` among those of the sequences with many rows; b < 0: none.
__device__ __forceinline__ void find_key_tile(const ScoreArgs& a, int x, int* b, int* tile) {
    const int lane = threadIdx.x & 63;
    *b = -1, *tile = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        int c = 0;
        if (b0 + lane < a.batch) {
            const Seq s = sequence(a, b0 + lane);
            if (s.n * a.group > a.few_rows) c = (s.len + kTileTokens - 1) / kTileTokens;
        }
        int sum = c;                                        // inclusive prefix sum over the lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        const uint64_t past = __ballot(sum > x);
        if (past) {
            const int l = __builtin_ctzll(past);
            *b = __builtin_amdgcn_readfirstlane(b0 + l);
            *tile = __builtin_amdgcn_readfirstlane(x - __shfl(sum - c, l));
            return;
        }
        x -= __shfl(sum, 63);
    }
}

template <int D, int BITS>
__global__ void __launch_bounds__(256, 2)
score_many(const ScoreArgs a) {
    constexpr int kU = D / 16, kToken = D * BITS / 8, kWords = kToken / 8, kNb = D / 32;
    constexpr int kCh = D / 8, kPer = 256 / kCh, kLoads = kStageRows / kPer;        // chunks of a row, rows a load, loads of a thread
    __shared__ __align__(16) uint8_t s_q[2][kStageRows * D * 2];
    __shared__ float s_ref[2][kStageRows];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    // Parts of the last rows first, of a part the key tiles in order, of a tile its heads.  What has nothing to do (tiles that a
    // causal part does not reach, more than there are) then comes in long runs: workgroups go to the dies and their shader engines in
    // turn, and tile by tile the idle ones would always meet the same engines (prompt of 8192 tokens then 619 us, so 397).
    const unsigned all_tiles = (unsigned)a.batch * a.key_tiles, unit = blockIdx.x / a.kv_heads;
    const int h = blockIdx.x - unit * a.kv_heads, part = a.parts - 1 - (int)(unit / all_tiles);
    int b = 0, tile = (int)(unit % all_tiles);
    if (a.batch > 1) find_key_tile(a, tile, &b, &tile);
    if (b < 0) return;
    const int bh = b * a.kv_heads + h;
    const Seq s = sequence(a, b);
    const int tile0 = tile * kTileTokens, t0 = tile0 + wave * 64;
    if (tile0 >= s.len || s.n * a.group <= a.few_rows) return;
    const RowRange range = tile_rows(a, s, tile0);
    int row_lo = range.lo, row_hi = range.hi;
    if (a.parts > 1) {
        row_lo = max(row_lo, part * a.chunk);
        row_hi = min(row_hi, (int)min((int64_t)0x7FFFFFFF, (int64_t)(part + 1) * a.chunk));
    }
    if (row_lo >= row_hi) {                                 // (a part's sum is then not read)
        if (a.parts == 1) store_score(a, s, b, h, tile0 + tid, 0.0f);
        return;
    }

    // staging: a thread moves chunk tid % kCh of rows tid / kCh + kPer k of a stage, the first 64 threads a row's lse each.  A row's
    // address is advanced by a stage of rows: tokens and heads, one token more where the heads pass the group's last one
    const int step_i = kStageRows / a.group, step_j = kStageRows % a.group, end = s.n * a.group, q_c = tid % kCh;
    const int64_t q_step = step_i * a.ldq + (int64_t)step_j * D, q_wrap = q_step + a.ldq - (int64_t)a.group * D;
    const int64_t l_step = (int64_t)step_i * a.q_heads + step_j, l_wrap = l_step + a.q_heads - a.group;
    const uint16_t* const q_first = a.q + (size_t)s.begin * a.ldq + (size_t)h * a.group * D + 8 * q_c;
    const float* const l_first = a.lse + (size_t)s.begin * a.q_heads + h * a.group;
    const uint16_t* q_at[kLoads];
    int q_j[kLoads];
    struct TokenHead {
        int token, head;
    };
    auto of_row = [&](int r) { return TokenHead{r / a.group, r % a.group}; };
#pragma unroll
    for (int k = 0; k < kLoads; ++k) {
        const TokenHead at = of_row(row_lo + tid / kCh + kPer * k);
        q_j[k] = at.head;
        q_at[k] = q_first + at.token * a.ldq + at.head * D;
    }
    const TokenHead l_row = of_row(row_lo + lane);
    int l_j = l_row.head;
    const float* l_at = l_first + l_row.token * (int64_t)a.q_heads + l_row.head;
    u32x4 qw[kLoads];
    float lw = 0.0f;
    auto request = [&](int r0) {                            // (rows past the end repeat the first one: they have no weights)
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            qw[k] = *reinterpret_cast<const u32x4*>(r0 + tid / kCh + kPer * k < end ? q_at[k] : q_first);
            q_j[k] += step_j;
            q_at[k] += q_j[k] >= a.group ? q_wrap : q_step;
            q_j[k] -= q_j[k] >= a.group ? a.group : 0;
        }
        if (wave == 0) {
            lw = *(r0 + lane < end ? l_at : l_first);
            l_j += step_j;
            l_at += l_j >= a.group ? l_wrap : l_step;
            l_j -= l_j >= a.group ? a.group : 0;
        }
    };
    auto stage = [&](int r0, int buf) {                     // what was requested: rows r0 ..
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            const int r = tid / kCh + kPer * k;
            *reinterpret_cast<u32x4*>(s_q[buf] + r * (D * 2) + q_place<D>(r, q_c) * 16) = qw[k];
        }
        if (wave == 0) s_ref[buf][lane] = r0 + lane < row_hi ? ref_of(lw) : INFINITY;
    };
    request(row_lo);
    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    bf16x8 kf[2][kU];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int t = min(t0 + 32 * x + n, s.len - 1);      // (tokens past the end are not stored)
        int page = table[t >> a.page_shift];
        page = (uint32_t)page < (uint32_t)a.num_pages ? page : 0;
        const int off = t & ((1 << a.page_shift) - 1);
        const int64_t ph = (int64_t)page * a.kv_heads + h;
        uint32_t w[kWords];
        load_words<kWords>(w, a.k_codes + ((ph << a.page_shift) + off) * kToken + hh * (kToken / 2));
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const float sc = scale_operand(a.k_scales[((ph * kNb + hh * (kNb / 2) + u / 4) << a.page_shift) + off]);
            kf[x][u] = cvt_eight<BITS>(w + u * BITS / 4, sc);
        }
    }

    float acc[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) acc[i] = 0.0f;
    stage(row_lo, 0);
    __syncthreads();
    // 32 rows' scores: chunk u of a lane's row is at (its chunk 0) ^ 16 u
    auto product = [&](v16f (&sc)[2], int buf, int sub) {
        uint32_t at = (uint32_t)((32 * sub + n) * (D * 2) + q_place<D>(n, hh * kU) * 16);
        asm volatile("" : "+v"(at));                        // (opaque, or every address is kept in a register of its own)
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            const bf16x8 qf = *reinterpret_cast<const bf16x8*>(s_q[buf] + (at ^ (uint32_t)(16 * u)));
#pragma unroll
            for (int x = 0; x < 2; ++x) sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x][u], qf, u ? sc[x] : v16f{}, 0, 0, 0);
        }
    };
    auto weigh = [&](const v16f (&sc)[2], float ref, int i) { acc[i] += exp2_(__builtin_fmaf(sc[i / 16][i % 16], a.scale, -ref)); };
    // the scores of 32 rows, and between their products the weights of the 32 rows before them: the matrix pipe and the vector
    // instructions of a wave then run at once
    auto both = [&](v16f (&sc)[2], int buf, int sub, const v16f (&last)[2], float ref) {
        constexpr int kEach = 32 / (2 * kU);                // weights to a product
        uint32_t at = (uint32_t)((32 * sub + n) * (D * 2) + q_place<D>(n, hh * kU) * 16);
        asm volatile("" : "+v"(at));
        bf16x8 qf[kDeep];
        float w[kEach];
#pragma unroll
        for (int u = 0; u < kDeep - 1; ++u) qf[u] = *reinterpret_cast<const bf16x8*>(s_q[buf] + (at ^ (uint32_t)(16 * u)));
#pragma unroll
        for (int u = 0; u < kU; ++u) {
            constexpr int kNext = kDeep - 1;
            if (u + kNext < kU) qf[(u + kNext) % kDeep] = *reinterpret_cast<const bf16x8*>(s_q[buf] + (at ^ (uint32_t)(16 * (u + kNext))));
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                __builtin_amdgcn_sched_barrier(0);
                sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x][u], qf[u % kDeep], u ? sc[x] : v16f{}, 0, 0, 0);
                // (the last product's weights are added before this one's are formed: nothing waits for an exponential)
                const int i0 = (2 * u + x) * kEach;
                float y[kEach];
#pragma unroll
                for (int k = 0; k < kEach; ++k) y[k] = __builtin_fmaf(last[(i0 + k) / 16][(i0 + k) % 16], a.scale, -ref);
#pragma unroll
                for (int k = 0; k < kEach && i0 > 0; ++k) {
                    acc[i0 - kEach + k] += w[k];
                    asm volatile("" : "+v"(acc[i0 - kEach + k]));      // (here, and not where the sum is used)
                }
#pragma unroll
                for (int k = 0; k < kEach; ++k) {
                    w[k] = exp2_(y[k]);
                    asm volatile("" : "+v"(w[k]));
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int k = 0; k < kEach; ++k) acc[32 - kEach + k] += w[k];
    };
    int r0 = row_lo, buf = 0;
    v16f even[2], odd[2] = {v16f{}, v16f{}};
    float ref_odd = INFINITY;                               // (weights of zero)
    // a stage's rows, the next stage's on their way meanwhile
    auto turn = [&](auto whole) {
        const bool more = r0 + kStageRows < row_hi;
        if (more) request(r0 + kStageRows);
        if constexpr (whole) {
            both(even, buf, 0, odd, ref_odd);
            const float ref_even = s_ref[buf][n];
            ref_odd = s_ref[buf][32 + n];
            both(odd, buf, 1, even, ref_even);
        } else {
#pragma unroll 1
            for (int sub = 0; sub < kStageRows / 32; ++sub) {
                const int rs = r0 + 32 * sub;
                const int first = s.first_pos + rs / a.group, last = s.first_pos + (rs + 31) / a.group;
                if (rs < row_hi && !(a.causal && last < t0) && !(a.window && (int64_t)first - a.window >= t0 + 63)) {
                    v16f sc[2];
                    product(sc, buf, sub);
                    const float ref = s_ref[buf][32 * sub + n];
                    const int pos = s.first_pos + (rs + n) / a.group;
                    const int lo = first_seen(a, pos) - t0 - 4 * hh, hi = (rs + n >= row_hi ? -1 : a.causal ? pos : 0x3FFFFFFF) - t0 - 4 * hh;
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int at = 32 * (i / 16) + 8 * (i % 16 / 4) + i % 4;
                        const float w = exp2_(__builtin_fmaf(sc[i / 16][i % 16], a.scale, -ref));
                        acc[i] += at >= lo && at <= hi ? w : 0.0f;
                    }
                }
            }
        }
        r0 += kStageRows, buf ^= 1;
        if (more) stage(r0, buf);
        __syncthreads();
    };
    // rows [whole_lo, whole_hi) see all tokens of the wave (the bounds are each wave's own, the stages and barriers are the same)
    const int64_t first_whole = a.causal ? max((int64_t)0, (int64_t)t0 + 63 - s.first_pos) * a.group : 0;
    const int64_t end_whole = a.window ? max((int64_t)0, (int64_t)t0 + a.window - s.first_pos) * a.group : row_hi;
    const int whole_lo = (int)min(first_whole, (int64_t)row_hi), whole_hi = (int)min(end_whole, (int64_t)row_hi) - kStageRows;
    auto whole_stage = [&]() { return r0 >= whole_lo && r0 <= whole_hi; };
    while (r0 < row_hi && !whole_stage()) turn(std::false_type());
    while (r0 < row_hi && whole_stage()) turn(std::true_type());
#pragma unroll
    for (int i = 0; i < 32; ++i) weigh(odd, ref_odd, i);
    while (r0 < row_hi) turn(std::false_type());
    // sums over the 32 lanes of a half: each step halves the values that a lane has; lane n is left with value n
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        // (exchanged by bits: a choice between two of them would become an index into all of them)
        const uint32_t up = n & d ? 0xFFFFFFFFu : 0u;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const uint32_t x = __float_as_uint(acc[i]), y = __float_as_uint(acc[i + d]), swap = (x ^ y) & up;
            acc[i] = __uint_as_float(x ^ swap) + __shfl_xor(__uint_as_float(y ^ swap), d);
        }
    }
    const int tok = wave * 64 + 32 * (n >> 4) + 8 * ((n & 15) >> 2) + 4 * hh + (n & 3);
    if (a.parts == 1) store_score(a, s, b, h, tile0 + tok, acc[0]);
    else a.part[(((size_t)bh * a.key_tiles + tile) * a.parts + part) * kTileTokens + tok] = acc[0];
}

// Adds the parts of a tile, in order.
__global__ void __launch_bounds__(256)
join_scores(const ScoreArgs a) {
    const int tile = blockIdx.x % a.key_tiles, bh = blockIdx.x / a.key_tiles;
    const int h = bh % a.kv_heads, b = bh / a.kv_heads;
    const Seq s = sequence(a, b);
    if (tile * kTileTokens >= s.len || s.n * a.group <= a.few_rows) return;
    const RowRange range = tile_rows(a, s, tile * kTileTokens);
    const float* p = a.part + (size_t)blockIdx.x * a.parts * kTileTokens + threadIdx.x;
    float v = 0.0f;
    if (range.lo < range.hi)
        for (int i = range.lo / a.chunk; i <= (range.hi - 1) / a.chunk; ++i) v += p[(size_t)i * kTileTokens];
    store_score(a, s, b, h, tile * kTileTokens + threadIdx.x, v);
}

struct ScorePlan {
    bool few, many;
    int few_rows, few_len, few_parts, key_tiles, chunk, parts;
};

// Parts of score_many: as many (key tile, part) units as make sixteen to a compute unit, a KiB of partial sums each, with parts of at
// least 512 rows; or two to a compute unit with parts of at least 256 (prompt of 8192 tokens of 32 and 8 heads of 128: 8, 16 and 32 units 382, 368
// and 383 us, of 16384 1211, 1106, 1072; prompt of 512 in parts of 1024, 512, 256 rows 44, 26, 18 us, of 2048 55, 46, 50).
constexpr int kUnits = 16, kLeastRows = 512;

ScorePlan score_plan(int group, int kv_heads, int batch, int total_q, int max_q, int max_kv, int compute_units) {
    ScorePlan p = {};
    const int64_t rows = (int64_t)max_q * group, pairs = (int64_t)batch * kv_heads;
    p.many = rows > 32;
    // (where one sequence of few rows would leave more queries than the others may have, there is none)
    p.few = !p.many || (int64_t)total_q <= (int64_t)(batch - 1) * max_q + 32 / group;
    p.few_rows = !p.few ? -1 : rows > 16 ? 32 : 16;
    int64_t len = (pairs * max_kv / (4 * compute_units) + 255) & ~int64_t(255);
    len = len < 256 ? 256 : len > 1024 ? 1024 : len;
    p.few_len = (int)len;
    p.few_parts = (int)((max_kv + len - 1) / len);
    p.key_tiles = (max_kv + kTileTokens - 1) / kTileTokens;
    p.parts = 1, p.chunk = 1 << 30;
    if (p.many) {
        const int64_t units = pairs * p.key_tiles > 0 ? pairs * p.key_tiles : 1;
        auto parts_of = [&](int64_t per_unit, int64_t least) {
            const int64_t wanted = per_unit * compute_units / units, most = (rows + least - 1) / least;
            return wanted < most ? wanted : most;
        };
        const int64_t many = parts_of(kUnits, kLeastRows), idle = parts_of(2, kLeastRows / 2), parts = many > idle ? many : idle;
        if (parts > 1) {
            p.chunk = (int)(((rows + parts - 1) / parts + kStageRows - 1) / kStageRows * kStageRows);
            p.parts = (int)((rows + p.chunk - 1) / p.chunk);
        }
    }
    return p;
}

template <int D, int BITS>
hipError_t launch_score(const ScoreArgs& a, const ScorePlan& p, hipStream_t stream) {
    const unsigned pairs = (unsigned)a.batch * a.kv_heads;
    if (p.many) {
        score_many<D, BITS><<<pairs * p.key_tiles * p.parts, 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (p.few) {
        const unsigned units = pairs * p.few_parts;
        if (a.score_table != a.page_table) {
            if (p.few_rows == 16) score_few<D, 1, BITS, true><<<units, 256, 0, stream>>>(a);
            else score_few<D, 2, BITS, true><<<units, 256, 0, stream>>>(a);
        } else {
            if (p.few_rows == 16) score_few<D, 1, BITS, false><<<units, 256, 0, stream>>>(a);
            else score_few<D, 2, BITS, false><<<units, 256, 0, stream>>>(a);
        }
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (p.parts > 1) join_scores<<<pairs * p.key_tiles, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t paged_score_part_bytes(const batq_paged_cache& c, int q_heads, int batch, int total_q, int max_q, int max_kv, int compute_units) {
    const ScorePlan p = score_plan(q_heads / c.kv_heads, c.kv_heads, batch, total_q, max_q, max_kv, compute_units);
    return p.parts > 1 ? (size_t)batch * c.kv_heads * p.key_tiles * p.parts * kTileTokens * 4 : 0;
}

// At least the former for every smaller call: tiles times parts are at most both of these, which grow with the arguments.
size_t paged_score_workspace_bytes(const batq_paged_cache& c, int q_heads, int batch, int total_q, int max_q, int max_kv, int compute_units) {
    const int64_t rows = (int64_t)max_q * (q_heads / c.kv_heads), most = (int64_t)kUnits * compute_units;
    const int64_t units = (int64_t)batch * c.kv_heads * ((max_kv + kTileTokens - 1) / kTileTokens) * ((rows + kLeastRows / 2 - 1) / (kLeastRows / 2));
    return rows <= kLeastRows / 2 ? 0 : (size_t)(units < most ? units : most) * kTileTokens * 4;
}

hipError_t launch_kv_paged_score(const batq_paged_cache& c, int bits, const batq_paged_batch& b, const void* q, int64_t ldq,
                                 int q_heads, float scale, bool causal, int window, const float* lse, float* score,
                                 const int32_t* score_table, int score_pages, bool add, void* workspace, hipStream_t stream) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const int cus = e == hipSuccess ? device_compute_units(dev, &e) : 0;
    if (e != hipSuccess) return e;
    const ScorePlan p = score_plan(q_heads / c.kv_heads, c.kv_heads, b.batch, b.total_q, b.max_q, b.max_kv, cus);
    ScoreArgs a = {};
    set_lists(a, c, b, q_heads, causal, window);
    a.q = static_cast<const uint16_t*>(q), a.ldq = ldq, a.lse = lse, a.score = score, a.add = add;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales;
    a.score_table = score_table ? score_table : b.page_table, a.score_pages = score_pages;
    a.scale = scale * 1.4426950408889634f;
    a.few_rows = p.few_rows, a.few_len = p.few_len, a.few_parts = p.few_parts;
    a.key_tiles = p.key_tiles, a.chunk = p.chunk, a.parts = p.parts, a.part = static_cast<float*>(workspace);
    if (bits == 8) return c.head_dim == 64 ? launch_score<64, 8>(a, p, stream) : launch_score<128, 8>(a, p, stream);
    return c.head_dim == 64 ? launch_score<64, 4>(a, p, stream) : launch_score<128, 4>(a, p, stream);
}

}  // namespace batq
