// Attention over the paged MXFP8 cache: one pass over a sequence's keys and values with the running maximum and sum
// of the softmax.  gfx950 only.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T: the instruction's result layout then has a lane hold scores of one
// query row, and with the tokens of a tile numbered as below, exactly the tokens that the same lane has to supply as
// the second product's operand.  Probabilities never leave their lane.
#include <math.h>

#include "batq_internal.h"
#include "mxfp4_device.h"

namespace batq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs {
    const uint16_t* q;
    int64_t ldq, ldo;
    uint16_t* out;
    float* lse;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t *cu_q, *kv_len, *page_table;
    int batch, table_width, total_q, max_q, max_kv, num_pages, page_shift, q_heads, kv_heads, group;
    int causal, window;
    float scale;                                            // times log2 e: scores are kept in units of ln 2
    // sequences of at most few_rows rows (query tokens x heads of a group) belong to attend_few, the others to
    // attend_rows; parts of few_len tokens
    int few_rows, few_len, max_parts;
    int part_rows;                                          // rows of a (sequence, key head) that partial results have room for
    float* part_o;                                          // [sequence][key head][row][part][D]: sums with the part's own maximum
    float* part_ml;                                         // [sequence][key head][row][part][2]: maximum, sum of the weights
};

// Sequence b as the kernels take it: nothing in the lists is trusted.
struct Seq {
    int begin, n, len;                                      // first row, queries served, tokens
    int first_pos;                                          // position of the first query
    int t_lo, t_hi;                                         // tokens that some query may see
};

__device__ __forceinline__ Seq sequence(const AttnArgs& a, int b) {
    Seq s;
    s.begin = a.cu_q[b];
    const int end = a.cu_q[b + 1];
    const int n = (s.begin < 0 || end > a.total_q || end < s.begin) ? 0 : end - s.begin;
    s.n = min(n, a.max_q);
    s.len = (int)min((int64_t)max(0, min(a.kv_len[b], a.max_kv)), (int64_t)a.table_width << a.page_shift);
    s.first_pos = s.len - n;
    s.t_hi = a.causal ? max(0, min(s.len, s.first_pos + s.n)) : s.len;
    s.t_lo = a.window ? min(s.t_hi, max(0, s.first_pos - a.window + 1)) : 0;
    return s;
}

// Parts of part_len tokens that a sequence is cut into (counted from its first visible token's block of 64; at least one,
// which writes the zeros of rows that see nothing).
__device__ __forceinline__ int live_parts(const Seq& s, int part_len) {
    return max(1, (s.t_hi - (s.t_lo & ~63) + part_len - 1) / part_len);
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t cvt_lo(uint32_t w, float sc) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, false));
}
__device__ __forceinline__ uint32_t cvt_hi(uint32_t w, float sc) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, true));
}
// The low (high) halves of x and y: transposes a 2 x 2 tile of 16-bit numbers.
__device__ __forceinline__ uint32_t low_halves(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }
__device__ __forceinline__ float scale_byte(uint32_t w, int i) { return scale_operand((w >> (8 * i)) & 0xFFu); }
__device__ __forceinline__ float shuffle_xor(float x, int d) { return __shfl_xor(x, d); }

// Few query rows to a key head (decoding, short drafts): bound by the stream of codes.  A workgroup takes one part of one
// (sequence, key head); its four waves take blocks of 64 tokens in turn, each with its own running maximum, and are
// joined at the end.  Rows: query token i and head j of the group are row i * group + j of NT tiles of 16.
//   keys     lane (m, g) = (l % 16, l / 16) loads channels [g D/4, (g + 1) D/4) of tokens 4m .. 4m + 3 straight into the
//            operand of S^T's tile t = 0..3 (tokens 4m + t): the order in which a product runs over channels is free, so a
//            lane's 16 bytes are contiguous, and its scales of the four tokens are one dword.
//   scores   result element r of tile t in lane (n, g) is row n and token 16g + 4r + t
//   values   lane (m, g) loads channels [m D/16, (m + 1) D/16) of tokens 16g .. 16g + 15, converts them with their tokens'
//            scales and turns pairs of tokens by 2 x 2; tile j of O^T has channels m D/16 + j
// Loads of the next block's keys are issued when this block's are used up, likewise the values, and page numbers one
// block further ahead: nothing passes through LDS before the end.
template <int D, int NT>
__global__ void __launch_bounds__(256, 2)
attend_few(const AttnArgs a) {
    constexpr int kC = D / 4, kV = D / 16, kU = D / 32;      // channels of a key lane, of a value lane, products per tile
    constexpr int kRow = D + 4;                             // floats of a row in LDS (spread over the banks)
    __shared__ float s_o[4][16][kRow];
    __shared__ float s_m[4][NT * 16], s_l[4][NT * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n = lane & 15, g = lane >> 4;
    const int part = blockIdx.x % a.max_parts, bh = blockIdx.x / a.max_parts;
    const int h = bh % a.kv_heads, b = bh / a.kv_heads;
    const Seq s = sequence(a, b);
    const int rows = s.n * a.group;
    if (rows == 0 || rows > a.few_rows || part >= live_parts(s, a.few_len)) return;
    const int t_begin = (s.t_lo & ~63) + part * a.few_len, t_end = min(s.t_hi, t_begin + a.few_len);

    bf16x8 qf[NT][kU];
    int row_lo[NT], row_hi[NT];                             // tokens [lo, hi) are visible to this lane's row
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        const int r = x * 16 + n, i = r / a.group;
        const bool live = r < rows;
        const uint16_t* p = a.q + (size_t)(s.begin + (live ? i : 0)) * a.ldq + (size_t)(h * a.group + (live ? r - i * a.group : 0)) * D + g * kC;
#pragma unroll
        for (int u = 0; u < kU; ++u) qf[x][u] = *reinterpret_cast<const bf16x8*>(p + 8 * u);
        const int pos = s.first_pos + i;
        row_hi[x] = !live ? 0 : a.causal ? min(s.len, pos + 1) : s.len;
        row_lo[x] = a.window ? max(0, pos - a.window + 1) : 0;
    }
    // blocks in [all_lo, all_hi) are seen whole by every row
    const int all_hi = a.causal ? min(s.len, s.first_pos + 1) : s.len;
    const int all_lo = a.window ? max(0, s.first_pos + s.n - a.window) : 0;

    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1;
    const int last_page = max(0, (s.len - 1) >> a.page_shift);      // entries behind it are not read
    auto entry = [&](int t) { return table[min(t >> a.page_shift, last_page)]; };
    const int k_group = 16 * (n >> 2), v_group = 16 * g;    // offset of the lane's 16 tokens in a block

    u32x4 kw[4][kC / 16];
    uint32_t ks;
    uint32_t vw[16][kV / 4];
    u32x4 vs;
    bool v_ok = false;
    auto load_k = [&](int t, int page) {
        page = (uint32_t)page < (uint32_t)a.num_pages ? page : 0;
        const int off = (t + 4 * n) & page_mask;
        const int64_t ph = (int64_t)page * a.kv_heads + h;
        const uint8_t* p = a.k_codes + ((ph << a.page_shift) + off) * D + g * kC;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int c = 0; c < kC / 16; ++c) kw[i][c] = *reinterpret_cast<const u32x4*>(p + i * D + c * 16);
        ks = *reinterpret_cast<const uint32_t*>(a.k_scales + ((ph * (D / 32) + g * kC / 32) << a.page_shift) + off);
    };
    auto load_v = [&](int t, int page) {
        v_ok = (uint32_t)page < (uint32_t)a.num_pages;
        page = v_ok ? page : 0;
        const int off = (t + v_group) & page_mask;
        const int64_t ph = (int64_t)page * a.kv_heads + h;
        const uint8_t* p = a.v_codes + ((ph << a.page_shift) + off) * D + n * kV;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (kV == 8) {
                const u32x2 w = *reinterpret_cast<const u32x2*>(p + i * D);
                vw[i][0] = w[0], vw[i][kV / 4 - 1] = w[1];
            } else {
                vw[i][0] = *reinterpret_cast<const uint32_t*>(p + i * D);
            }
        }
        vs = *reinterpret_cast<const u32x4*>(a.v_scales + ((ph * (D / 32) + n * kV / 32) << a.page_shift) + off);
    };

    float m[NT], l[NT];
    f32x4 o[NT][kV];
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        m[x] = -INFINITY, l[x] = 0.0f;
#pragma unroll
        for (int j = 0; j < kV; ++j) o[x][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    int t = t_begin + wave * 64;
    int kp = 0, vp = 0;
    if (t < t_end) {
        const int k0 = entry(t + k_group), v0 = entry(t + v_group);
        kp = entry(t + 256 + k_group), vp = entry(t + 256 + v_group);
        load_k(t, k0);
        load_v(t, v0);
    }
    for (; t < t_end; t += 256) {
        const bool more = t + 256 < t_end;
        f32x4 sc[NT][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float kscale = scale_byte(ks, i);
            bf16x8 kf[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) {
                const uint32_t w0 = kw[i][u / 2][2 * (u & 1)], w1 = kw[i][u / 2][2 * (u & 1) + 1];
                kf[u] = __builtin_bit_cast(bf16x8, u32x4{cvt_lo(w0, kscale), cvt_hi(w0, kscale), cvt_lo(w1, kscale), cvt_hi(w1, kscale)});
            }
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                sc[x][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < kU; ++u) sc[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u], qf[x][u], sc[x][i], 0, 0, 0);
            }
        }
        if (more) load_k(t + 256, kp);
        const bool whole = t >= all_lo && t + 64 <= all_hi && __ballot(!v_ok) == 0;
        if (!whole) {
            // masked places may hold anything (unwritten codes, pages that are gone): their scores are replaced, their
            // values and scales become zeros and ones, so that a weight of zero stays a product of zero
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int tok = t + v_group + 4 * r + i;
#pragma unroll
                    for (int x = 0; x < NT; ++x)
                        if (!(v_ok && tok >= row_lo[x] && tok < row_hi[x])) sc[x][i][r] = -INFINITY;
                }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int tok = t + v_group + i;
                if (!(v_ok && tok >= s.t_lo && tok < s.len)) {
#pragma unroll
                    for (int c = 0; c < kV / 4; ++c) vw[i][c] = 0u;
                    vs[i / 4] = (vs[i / 4] & ~(0xFFu << (8 * (i & 3)))) | (127u << (8 * (i & 3)));
                }
            }
        }
        bf16x8 ph[NT][2], pl[NT][2];                        // the weights as two bf16 terms
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            float mx = sc[x][0][0];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx = __builtin_fmaxf(mx, sc[x][i][r]);
            mx = __builtin_fmaxf(mx, shuffle_xor(mx, 16));
            mx = __builtin_fmaxf(mx, shuffle_xor(mx, 32));
            const float m2 = __builtin_fmaxf(m[x], mx * a.scale);
            const float ref = m2 == -INFINITY ? 0.0f : m2;
            if (__ballot(m2 > m[x])) {
                const float f = exp2_(m[x] - ref);
                l[x] *= f;
#pragma unroll
                for (int j = 0; j < kV; ++j) o[x][j] *= f;
            }
            m[x] = m2;
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float p = exp2_(__builtin_fmaf(sc[x][e & 3][2 * u + (e >> 2)], a.scale, -ref));
                    l[x] += p;
                    ph[x][u][e] = (__bf16)p;
                    pl[x][u][e] = (__bf16)(p - (float)ph[x][u][e]);
                }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int c = 0; c < kV / 4; ++c) {              // four channels of eight tokens
                uint32_t f[4][4];                           // [channel][token pair]
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int i0 = 8 * u + 2 * e, i1 = i0 + 1;
                    const float s0 = scale_byte(vs[i0 / 4], i0 & 3), s1 = scale_byte(vs[i1 / 4], i1 & 3);
                    const uint32_t a0 = cvt_lo(vw[i0][c], s0), b0 = cvt_lo(vw[i1][c], s1);
                    const uint32_t a1 = cvt_hi(vw[i0][c], s0), b1 = cvt_hi(vw[i1][c], s1);
                    f[0][e] = low_halves(a0, b0), f[1][e] = high_halves(a0, b0);
                    f[2][e] = low_halves(a1, b1), f[3][e] = high_halves(a1, b1);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{f[j][0], f[j][1], f[j][2], f[j][3]});
#pragma unroll
                    for (int x = 0; x < NT; ++x) {
                        f32x4& acc = o[x][4 * c + j];
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pl[x][u], acc, 0, 0, 0);
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, ph[x][u], acc, 0, 0, 0);
                    }
                }
            }
        if (more) {
            load_v(t + 256, vp);
            if (t + 512 < t_end) kp = entry(t + 512 + k_group), vp = entry(t + 512 + v_group);
        }
    }

    // join the waves: element r of tile j is channel (4g + r) D/16 + j of row n
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        l[x] += shuffle_xor(l[x], 16);
        l[x] += shuffle_xor(l[x], 32);
        if (g == 0) s_m[wave][x * 16 + n] = m[x], s_l[wave][x * 16 + n] = l[x];
    }
    const bool only = live_parts(s, a.few_len) == 1;
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        __syncthreads();                                    // (also: the last tile's rows have been read)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int j = 0; j < kV; j += 4)
                *reinterpret_cast<f32x4*>(&s_o[wave][n][(4 * g + r) * kV + j]) = f32x4{o[x][j][r], o[x][j + 1][r], o[x][j + 2][r], o[x][j + 3][r]};
        __syncthreads();
        const int rr = threadIdx.x >> 4, c0 = (threadIdx.x & 15) * kV, r = x * 16 + rr;
        if (r >= rows) continue;                            // (every thread of the workgroup reaches the barriers above)
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < 4; ++w) top = __builtin_fmaxf(top, s_m[w][r]);
        float sum = 0.0f, v[kV] = {};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = top == -INFINITY ? 0.0f : exp2_(s_m[w][r] - top);
            sum += f * s_l[w][r];
#pragma unroll
            for (int j = 0; j < kV; ++j) v[j] = __builtin_fmaf(f, s_o[w][rr][c0 + j], v[j]);
        }
        const int i = r / a.group, head = h * a.group + r - i * a.group;
        const size_t row = (size_t)(s.begin + i);
        if (only) {
            const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
            uint16_t* p = a.out + row * a.ldo + (size_t)head * D + c0;
#pragma unroll
            for (int j = 0; j < kV; j += 4) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<bf16x4*>(p + j) = bf16x4{(__bf16)(v[j] * inv), (__bf16)(v[j + 1] * inv), (__bf16)(v[j + 2] * inv), (__bf16)(v[j + 3] * inv)};
            }
            if (a.lse && c0 == 0) a.lse[row * a.q_heads + head] = sum > 0.0f ? (top + __log2f(sum)) * 0.69314718055994531f : -INFINITY;
        } else {
            const size_t at = ((size_t)bh * a.part_rows + r) * a.max_parts + part;
#pragma unroll
            for (int j = 0; j < kV; j += 4) *reinterpret_cast<f32x4*>(a.part_o + at * D + c0 + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
            if (c0 == 0) a.part_ml[2 * at] = top, a.part_ml[2 * at + 1] = sum;
        }
    }
}

// Joins the parts of sequences that were cut, in part order: one wave per row of a (sequence, key head).
template <int D>
__global__ void __launch_bounds__(256)
join_parts(const AttnArgs a) {
    const int lane = threadIdx.x & 63;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t bh = unit / a.part_rows;
    const int r = (int)(unit - bh * a.part_rows), h = (int)(bh % a.kv_heads), b = (int)(bh / a.kv_heads);
    if (b >= a.batch) return;
    const Seq s = sequence(a, b);
    const int rows = s.n * a.group;
    if (r >= rows || rows > a.few_rows) return;
    const size_t row = (size_t)s.begin + r / a.group;
    const int head = h * a.group + r % a.group;
    const int parts = live_parts(s, a.few_len);
    if (parts == 1) return;
    const size_t at = (size_t)unit * a.max_parts;
    float top = -INFINITY;
    for (int p = lane; p < parts; p += 64) top = __builtin_fmaxf(top, a.part_ml[2 * (at + p)]);
#pragma unroll
    for (int d = 32; d; d >>= 1) top = __builtin_fmaxf(top, shuffle_xor(top, d));
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, v[D / 64] = {};
    for (int p0 = 0; p0 < parts; p0 += 64) {
        const int p = p0 + lane;
        const float f = p < parts ? exp2_(a.part_ml[2 * (at + p)] - ref) : 0.0f;
        const float w = p < parts ? f * a.part_ml[2 * (at + p) + 1] : 0.0f;
        sum += w;
        const int count = min(64, parts - p0);
#pragma unroll 8
        for (int j = 0; j < count; ++j) {
            const float fj = __shfl(f, j);
#pragma unroll
            for (int c = 0; c < D / 64; ++c) v[c] = __builtin_fmaf(fj, a.part_o[(at + p0 + j) * D + lane * (D / 64) + c], v[c]);
        }
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += shuffle_xor(sum, d);
    const float inv = sum > 0.0f ? 1.0f / sum : 0.0f;
    uint16_t* o = a.out + row * a.ldo + (size_t)head * D + lane * (D / 64);
#pragma unroll
    for (int c = 0; c < D / 64; ++c) reinterpret_cast<__bf16*>(o)[c] = (__bf16)(v[c] * inv);
    if (a.lse && lane == 0) a.lse[row * a.q_heads + head] = sum > 0.0f ? (top + __log2f(sum)) * 0.69314718055994531f : -INFINITY;
}

// One wave per (row of q, query head): a lane takes a key of 64 at a time, then a channel (or two) of the values.
template <int D>
__global__ void __launch_bounds__(64)
attend_rows(const AttnArgs a) {
    __shared__ float sq[D];
    const int lane = threadIdx.x, row = blockIdx.x, head = blockIdx.y, kvh = head / a.group;
    int b = 0, begin = 0, end = 0;
    for (; b < a.batch; ++b) {
        begin = a.cu_q[b], end = a.cu_q[b + 1];
        if (begin >= 0 && row >= begin && row < end && end <= a.total_q) break;
    }
    if (b == a.batch || row - begin >= a.max_q || min(end - begin, a.max_q) * a.group <= a.few_rows) return;
    int64_t width = (int64_t)a.table_width << a.page_shift;
    const int len = (int)min((int64_t)max(0, min(a.kv_len[b], a.max_kv)), width);
    const int pos = len - (end - begin) + (row - begin);
    const int t1 = a.causal ? min(len, pos + 1) : len;
    const int t0 = a.window ? max(0, pos - a.window + 1) : 0;
    for (int i = lane; i < D; i += 64) sq[i] = bf16_bits_to_float(a.q[(size_t)row * a.ldq + (size_t)head * D + i]);
    __syncthreads();
    float m = -INFINITY, l = 0.0f, o[D / 64] = {};
    const int page_mask = (1 << a.page_shift) - 1;
    for (int t = t0 & ~63; t < t1; t += 64) {
        const int tt = t + lane;
        float s = -INFINITY;
        if (tt >= t0 && tt < t1) {
            const int page = a.page_table[(size_t)b * a.table_width + (tt >> a.page_shift)];
            if (page >= 0 && page < a.num_pages) {
                const int64_t ph = (int64_t)page * a.kv_heads + kvh;
                const uint8_t* kc = a.k_codes + (((ph << a.page_shift) + (tt & page_mask)) * D);
                s = 0.0f;
                for (int blk = 0; blk < D / 32; ++blk) {
                    const float sc = scale_operand(a.k_scales[((ph * (D / 32) + blk) << a.page_shift) + (tt & page_mask)]);
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t w = reinterpret_cast<const uint32_t*>(kc + blk * 32)[i];
                        const auto lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, false);
                        const auto hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, true);
                        const float* qq = sq + blk * 32 + 4 * i;
                        s += lo[0] * qq[0] + lo[1] * qq[1] + hi[0] * qq[2] + hi[1] * qq[3];
                    }
                }
                s *= a.scale * 0.69314718055994531f;
            }
        }
        float mx = s;
        for (int d = 32; d; d >>= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
        if (mx == -INFINITY) continue;
        const float m2 = fmaxf(m, mx), f = expf(m - m2), p = expf(s - m2);
        float sum = p;
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        l = l * f + sum;
        m = m2;
        for (int i = 0; i < D / 64; ++i) o[i] *= f;
        for (int j = 0; j < 64; ++j) {
            const float pj = __shfl(p, j);
            const int u = t + j;
            if (pj == 0.0f) continue;                       // (places that take no part may hold anything)
            const int page = a.page_table[(size_t)b * a.table_width + (u >> a.page_shift)];
            const int64_t ph = (int64_t)page * a.kv_heads + kvh;
            for (int i = 0; i < D / 64; ++i) {
                const int c = i * 64 + lane;
                const uint32_t w = a.v_codes[((ph << a.page_shift) + (u & page_mask)) * D + c];
                const float sc = scale_operand(a.v_scales[((ph * (D / 32) + c / 32) << a.page_shift) + (u & page_mask)]);
                o[i] += pj * __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, sc, false)[0];
            }
        }
    }
    for (int i = 0; i < D / 64; ++i)
        a.out[(size_t)row * a.ldo + (size_t)head * D + i * 64 + lane] = (uint16_t)float_to_bf16_bits(l > 0.0f ? o[i] / l : 0.0f);
    if (a.lse && lane == 0) a.lse[(size_t)row * a.q_heads + head] = l > 0.0f ? m + logf(l) : -INFINITY;
}

}  // namespace

namespace {

struct Plan {
    int few_rows, few_len, max_parts, part_rows;
    bool few, rows;                                         // which kernels run
};

// Part length: enough workgroups for two to a compute unit (four where a sequence is long), at least 256 tokens (a
// block for each wave) and at most 1024, so that the longest of ragged sequences does not outlast the others.
Plan plan(int group, int kv_heads, int batch, int max_q, int max_kv, int compute_units) {
    Plan p = {};
    const int64_t rows = (int64_t)max_q * group;
    p.rows = rows > 32;
    p.few = !p.rows || batch > 1;
    p.few_rows = !p.few ? 0 : p.rows ? 16 : rows > 16 ? 32 : 16;
    p.part_rows = (int)(rows < p.few_rows ? rows : p.few_rows);
    const int64_t tokens = (int64_t)batch * kv_heads * max_kv;
    int64_t len = (tokens / (4 * compute_units) + 255) & ~int64_t(255);
    if (len < 256) len = 256;
    if (len > 1024) len = 1024;
    p.few_len = (int)len;
    p.max_parts = p.few ? (int)((max_kv + 63 + len - 1) / len) : 1;
    if (p.max_parts < 1) p.max_parts = 1;
    return p;
}

int64_t part_units(const Plan& p, int batch, int kv_heads) { return p.max_parts > 1 ? (int64_t)batch * kv_heads * p.part_rows : 0; }

template <int D>
hipError_t launch_attention(const AttnArgs& a, const Plan& p, hipStream_t stream) {
    if (p.few) {
        const unsigned units = (unsigned)a.batch * a.kv_heads * p.max_parts;
        if (p.few_rows == 16) attend_few<D, 1><<<units, 256, 0, stream>>>(a);
        else attend_few<D, 2><<<units, 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (p.rows) {
        attend_rows<D><<<dim3(a.total_q, a.q_heads), 64, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (const int64_t units = part_units(p, a.batch, a.kv_heads)) {
        join_parts<D><<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    return hipSuccess;
}

}  // namespace

size_t paged_attention_workspace_bytes(const batq_paged_cache& c, int q_heads, int batch, int, int max_q, int max_kv,
                                       int compute_units) {
    const Plan p = plan(q_heads / c.kv_heads, c.kv_heads, batch, max_q, max_kv, compute_units);
    return (size_t)part_units(p, batch, c.kv_heads) * p.max_parts * (c.head_dim + 2) * 4;
}

hipError_t launch_paged_attention(const batq_paged_cache& c, const batq_paged_batch& b, const void* q, int64_t ldq,
                                  int q_heads, float scale, bool causal, int window, void* out, int64_t ldo, float* lse,
                                  void* workspace, hipStream_t stream) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const int cus = e == hipSuccess ? device_compute_units(dev, &e) : 0;
    if (e != hipSuccess) return e;
    const Plan p = plan(q_heads / c.kv_heads, c.kv_heads, b.batch, b.max_q, b.max_kv, cus);
    AttnArgs a = {};
    a.q = static_cast<const uint16_t*>(q), a.ldq = ldq, a.ldo = ldo, a.out = static_cast<uint16_t*>(out), a.lse = lse;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales, a.v_codes = c.v_codes, a.v_scales = c.v_scales;
    a.cu_q = b.cu_q, a.kv_len = b.kv_len, a.page_table = b.page_table, a.batch = b.batch, a.table_width = b.table_width;
    a.total_q = b.total_q, a.max_q = b.max_q, a.max_kv = b.max_kv, a.num_pages = c.num_pages;
    a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.q_heads = q_heads, a.kv_heads = c.kv_heads, a.group = q_heads / c.kv_heads;
    a.causal = causal, a.window = window, a.scale = scale * 1.4426950408889634f;
    a.few_rows = p.few_rows, a.few_len = p.few_len, a.max_parts = p.max_parts, a.part_rows = p.part_rows;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o ? a.part_o + (size_t)part_units(p, b.batch, c.kv_heads) * p.max_parts * c.head_dim : nullptr;
    return c.head_dim == 64 ? launch_attention<64>(a, p, stream) : launch_attention<128>(a, p, stream);
}

}  // namespace batq
