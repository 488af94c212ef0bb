// What the cached tokens have received of the attention: for each key head and token t the softmax weights
// exp(scale q_i k_t - lse_i) of the batch's queries, summed over the queries i that see t and the query heads that read the
// key head.  gfx950 only.
#include "batq_internal.h"
#include "mxfp4_device.h"
#include "paged_device.h"

namespace batq {
namespace {

struct ScoreArgs : PagedLists {
    const uint16_t* q;
    int64_t ldq;
    const float* lse;
    const uint8_t *k_codes, *k_scales;
    float* score;
    float scale;                                            // times log2 e
    int add, key_tiles;
};

constexpr int kTileTokens = 256;                            // of a workgroup, 64 to a wave

// A wave has 64 tokens, whose keys stay in registers as operands, and walks the rows that may see them 32 at a time:
// S^T = K Q^T, so that a lane holds scores of one row and adds its weights up token by token; the lanes' sums are added at
// the end.  Lane (n, h) = (l % 32, l / 32) holds channels [h D/2, (h + 1) D/2) of token n of either half (the order in which
// a product runs over channels is free) and of row n; result element e of half x is token 32x + 8 (e / 4) + 4h + e % 4.
template <int D, int BITS>
__global__ void __launch_bounds__(256)
score_kernel(const ScoreArgs a) {
    constexpr int kU = D / 16, kToken = D * BITS / 8, kWords = kToken / 8, kNb = D / 32;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int tile = blockIdx.x % a.key_tiles, bh = blockIdx.x / a.key_tiles;
    const int h = bh % a.kv_heads, b = bh / a.kv_heads;
    const Seq s = sequence(a, b);
    const int t0 = tile * kTileTokens + wave * 64;
    if (t0 >= s.len) return;
    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1;

    bf16x8 kf[2][kU];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
        const int t = min(t0 + 32 * x + n, s.len - 1);      // (tokens past the end are not stored)
        int page = table[t >> a.page_shift];
        page = (uint32_t)page < (uint32_t)a.num_pages ? page : 0;
        const int off = t & page_mask;
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
    const int i_lo = a.causal ? max(0, t0 - s.first_pos) : 0;
    const int i_hi = a.window ? (int)max((int64_t)0, min((int64_t)s.n, (int64_t)t0 + 63 + a.window - s.first_pos)) : s.n;
    const int row_end = i_hi * a.group;
    for (int r0 = i_lo * a.group; r0 < row_end; r0 += 32) {
        const int r = r0 + n, i = r / a.group;
        const bool live = r < row_end;
        const size_t row = (size_t)(s.begin + (live ? i : 0));
        const int head = h * a.group + (live ? r - i * a.group : 0);
        const uint16_t* p = a.q + row * a.ldq + (size_t)head * D + hh * (D / 2);
        bf16x8 qf[kU];
#pragma unroll
        for (int u = 0; u < kU; ++u) qf[u] = *reinterpret_cast<const bf16x8*>(p + 8 * u);
        const float lse = a.lse[row * a.q_heads + head];
        // a row that has seen nothing has no weights
        const float ref = lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f;
        v16f sc[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            sc[x] = v16f{};
#pragma unroll
            for (int u = 0; u < kU; ++u) sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[x][u], qf[u], sc[x], 0, 0, 0);
        }
        const int pos = s.first_pos + i;
        const int lo = first_seen(a, pos), hi = !live ? 0 : a.causal ? pos + 1 : 0x7FFFFFFF;
        const bool whole = __ballot(!(lo <= t0 && hi >= t0 + 64)) == 0;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int t = t0 + 32 * x + 8 * (e >> 2) + 4 * hh + (e & 3);
                float w = exp2_(__builtin_fmaf(sc[x][e], a.scale, -ref));
                if (!whole && !(t >= lo && t < hi)) w = 0.0f;
                acc[16 * x + e] += w;
            }
    }
    // sums over the 32 lanes of a half: each step halves the values that a lane has; lane n is left with value n
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        const bool up = n & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float give = up ? acc[i] : acc[i + d], own = up ? acc[i + d] : acc[i];
            acc[i] = own + __shfl_xor(give, d);
        }
    }
    const int t = t0 + 32 * (n >> 4) + 8 * ((n & 15) >> 2) + 4 * hh + (n & 3);
    if (t >= s.len) return;
    const int page = table[t >> a.page_shift];
    if ((uint32_t)page >= (uint32_t)a.num_pages) return;
    float* to = a.score + ((((int64_t)page * a.kv_heads + h) << a.page_shift) + (t & page_mask));
    float v = acc[0];
    if (a.add && t < s.first_pos) v += *to;
    *to = v;
}

template <int D, int BITS>
hipError_t launch_score(const ScoreArgs& a, hipStream_t stream) {
    score_kernel<D, BITS><<<(unsigned)a.batch * a.kv_heads * a.key_tiles, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace

size_t paged_score_part_bytes(const batq_paged_cache& c, int q_heads, int batch, int total_q, int max_q, int max_kv, int compute_units) {
    return 0;
}
size_t paged_score_workspace_bytes(const batq_paged_cache& c, int q_heads, int batch, int total_q, int max_q, int max_kv, int compute_units) {
    return 0;
}

hipError_t launch_kv_paged_score(const batq_paged_cache& c, int bits, const batq_paged_batch& b, const void* q, int64_t ldq,
                                 int q_heads, float scale, bool causal, int window, const float* lse, float* score, bool add,
                                 void* workspace, hipStream_t stream) {
    ScoreArgs a = {};
    set_lists(a, c, b, q_heads, causal, window);
    a.q = static_cast<const uint16_t*>(q), a.ldq = ldq, a.lse = lse, a.score = score, a.add = add;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales;
    a.scale = scale * 1.4426950408889634f;
    a.key_tiles = (b.max_kv + kTileTokens - 1) / kTileTokens;
    if (bits == 8) return c.head_dim == 64 ? launch_score<64, 8>(a, stream) : launch_score<128, 8>(a, stream);
    return c.head_dim == 64 ? launch_score<64, 4>(a, stream) : launch_score<128, 4>(a, stream);
}

}  // namespace batq
