// Attention over the paged cache of MXFP8 or MXFP4 (BITS 8 or 4): one pass over a sequence's keys and values with the running maximum and sum
// of the softmax.  gfx950 only.
//
// Both kernels compute S^T = K Q^T and O^T = V^T P^T: the instruction's result layout then has a lane hold scores of one
// query row, and with the tokens of a tile numbered as below, exactly the tokens that the same lane has to supply as
// the second product's operand.  Probabilities never leave their lane.
#include <math.h>

#include "batq_internal.h"
#include "mxfp4_device.h"
#include "paged_device.h"

namespace batq {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

struct AttnArgs : PagedLists {
    const uint16_t* q;
    int64_t ldq, ldo;
    uint16_t* out;
    float* lse;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    float scale;                                            // times log2 e: scores are kept in units of ln 2
    // sequences of at most few_rows rows (query tokens x heads of a group) belong to attend_few, the others to
    // attend_many; parts of few_len and many_len tokens
    int few_rows, few_len, max_parts;
    int part_rows;                                          // rows of a (sequence, key head) that partial results have room for
    float* part_o;                                          // [sequence][key head][row][part][D]: sums with the part's own maximum
    float* part_ml;                                         // [sequence][key head][row][part][2]: maximum, sum of the weights
    int many_len, many_parts;
    float *many_o, *many_ml;                                // likewise [row of q][query head][part]
};

// Tokens [lo, hi) that some row of a workgroup sees, and the parts of part_len tokens that they are cut into (counted
// from the block of 64 with the first of them; at least one, which writes the zeros of rows that see nothing).
struct TokenRange {
    int lo, hi;
};
__device__ __forceinline__ int range_parts(const TokenRange& t, int part_len) {
    return max(1, (t.hi - (t.lo & ~63) + part_len - 1) / part_len);
}
__device__ __forceinline__ int live_parts(const Seq& s, int part_len) { return range_parts(TokenRange{s.t_lo, s.t_hi}, part_len); }

// The low (high) halves of x and y: transposes a 2 x 2 tile of 16-bit numbers.
__device__ __forceinline__ uint32_t low_halves(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t x, uint32_t y) { return __builtin_amdgcn_perm(y, x, 0x07060302u); }
__device__ __forceinline__ float scale_byte(uint32_t w, int i) { return scale_operand((w >> (8 * i)) & 0xFFu); }

// A weight of zero times a value that is not finite is not zero, and a matrix product has no mask: where a block's tokens are
// seen by some rows only and such a value may be among them, it is taken as zero, and the sums of the rows that do see it
// become NaN by themselves.
// Whether four codes with their scale may give one: NaN codes; scales from 2^120 on (448 x 2^120 is past bf16).
__device__ __forceinline__ uint32_t odd_codes(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u; }
__device__ __forceinline__ uint32_t odd_scales(uint32_t w) { return ((w & 0x7F7F7F7Fu) + 0x09090909u) & w & 0x80808080u; }
// All bits of the bf16 halves that are not finite.
__device__ __forceinline__ uint32_t odd_halves(uint32_t w) {
    return ((w & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((w & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
}

__device__ __forceinline__ float shuffle_xor(float x, int d) { return __shfl_xor(x, d); }

// Few query rows to a key head (decoding, short drafts): bound by the stream of codes.  A workgroup takes one part of one
// (sequence, key head); its four waves take blocks of 32 tokens in turn, each with its own running maximum, and are
// joined at the end.  Rows: query token i and head j of the group are row i * group + j of NT tiles of 16.
//   keys     lane (m, g) = (l % 16, l / 16) loads channels [g D/4, (g + 1) D/4) of tokens 2m and 2m + 1 straight into the
//            operands of S^T's tiles 0 and 1: the order in which a product runs over channels is free, so a lane's
//            16 bytes are contiguous, and its scales of the two tokens are one 16-bit word
//   scores   result element r of tile t in lane (n, g) is row n and token 8g + 2r + t
//   values   lane (m, g) loads channels [m D/16, (m + 1) D/16) of tokens 8g .. 8g + 7, converts them with their tokens'
//            scales and turns pairs of tokens by 2 x 2; tile j of O^T has channels m D/16 + j
// Loads of the next block's keys are issued when this block's are used up, likewise the values: nothing passes through LDS
// before the end.  The reference of the exponentials moves only when a row's maximum has grown by more than 2^8.
// The weights go in as two bf16 terms (2^-16): the products are not the bound here.  Measured: 4 sequences of about 131072 tokens, 28 query
// and 4 key heads of 128: 73 us (367 MB, 5.0 TB/s, a large copy's rate); 64 sequences of up to 8192, 32 and 8 heads: 36 us.
// Blocks of 64 tokens at two waves per SIMD: 40 us instead of 36; four waves per SIMD spill: 50 us.
// Codes of 4 bits are half the bytes for the same vector instructions, and those with the waves' waits are the bound: 64 x 8192 tokens of 32 and 8
// heads of 128 channels 145 us (570 MB, 3.9 TB/s; 8 bits 202 us, 5.5 TB/s), 4 of about 131072 under 28 and 4 heads 46 us.  Not better: keys and
// values requested two blocks ahead, which leaves two waves per SIMD (163 us), each sum's two products apart (148), parts of 512 to 896
// tokens (151 to 141 beside 140), four waves per SIMD (spills, 285), first parts of all sequences first (ragged ones 37 us instead of 33).
template <int D, int NT, int BITS>
__global__ void __launch_bounds__(256, NT == 1 ? 3 : 2)
attend_few(const AttnArgs a) {
    constexpr int kC = D / 4, kV = D / 16, kU = D / 32;      // channels of a key lane, of a value lane, products per tile
    constexpr int kToken = D * BITS / 8;                    // bytes of a token's codes
    constexpr int kKw = kC * BITS / 32, kVw = kV * BITS >= 32 ? kV * BITS / 32 : 1;      // words of a lane's key, of its values
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

    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1;
    const int last_page = max(0, (s.len - 1) >> a.page_shift);      // entries behind it are not read
    // lane i holds the page of tokens t_begin + 16 i .. + 15 (a part is at most 1024 long): page numbers are not loaded in
    // the loop, where waiting for them would wait for the codes requested before them
    const int pages = t_begin < t_end ? table[min((t_begin + 16 * lane) >> a.page_shift, last_page)] : 0;
    auto entry = [&](int t) { return __shfl(pages, (t - t_begin) >> 4); };

    uint32_t kw[2][kKw];
    uint32_t ks;
    uint32_t vw[8][kVw];
    u32x2 vs;
    bool v_ok = false;
    auto load_k = [&](int t) {
        t += 2 * n;
        int page = entry(t);
        page = (uint32_t)page < (uint32_t)a.num_pages ? page : 0;
        const int off = t & page_mask;
        const int64_t ph = (int64_t)page * a.kv_heads + h;
        const uint8_t* p = a.k_codes + ((ph << a.page_shift) + off) * kToken + g * (kToken / 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) load_words<kKw>(kw[i], p + i * kToken);
        ks = *reinterpret_cast<const uint16_t*>(a.k_scales + ((ph * (D / 32) + g * kC / 32) << a.page_shift) + off);
    };
    auto load_v = [&](int t) {
        t += 8 * g;
        int page = entry(t);
        v_ok = (uint32_t)page < (uint32_t)a.num_pages;
        page = v_ok ? page : 0;
        const int off = t & page_mask;
        const int64_t ph = (int64_t)page * a.kv_heads + h;
        const uint8_t* p = a.v_codes + ((ph << a.page_shift) + off) * kToken + n * (kToken / 16);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if constexpr (kV * BITS >= 32) load_words<kVw>(vw[i], p + i * kToken);
            else vw[i][0] = *reinterpret_cast<const uint16_t*>(p + i * kToken);
        }
        vs = *reinterpret_cast<const u32x2*>(a.v_scales + ((ph * (D / 32) + n * kV / 32) << a.page_shift) + off);
    };
    int t = t_begin + wave * 32;
    if (t < t_end) {
        load_k(t);
        load_v(t);
    }

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
        row_lo[x] = first_seen(a, pos);
    }
    // blocks in [all_lo, all_hi) are seen whole by every row
    const int all_hi = a.causal ? min(s.len, s.first_pos + 1) : s.len;
    const int all_lo = first_seen(a, s.first_pos + s.n - 1);

    float m[NT], l[NT];
    f32x4 o[NT][kV];
#pragma unroll
    for (int x = 0; x < NT; ++x) {
        m[x] = -INFINITY, l[x] = 0.0f;
#pragma unroll
        for (int j = 0; j < kV; ++j) o[x][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    }
    for (; t < t_end; t += 128) {
        const bool more = t + 128 < t_end;
        f32x4 sc[NT][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float kscale = scale_byte(ks, i);
            bf16x8 kf[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u) kf[u] = cvt_eight<BITS>(kw[i] + u * BITS / 4, kscale);
#pragma unroll
            for (int x = 0; x < NT; ++x) {
                sc[x][i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                for (int u = 0; u < kU; ++u) sc[x][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[u], qf[x][u], sc[x][i], 0, 0, 0);
            }
        }
        if (more) load_k(t + 128);
        const bool whole = t >= all_lo && t + 32 <= all_hi && __ballot(!v_ok) == 0;
        bool odd = false;                                   // wave-uniform
        if (!whole) {
            // masked places may hold anything (unwritten codes, pages that are gone): their scores are replaced, their
            // values and scales become zeros and ones, so that a weight of zero stays a product of zero
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int tok = t + 8 * g + 2 * r + i;
#pragma unroll
                    for (int x = 0; x < NT; ++x)
                        if (!(v_ok && tok >= row_lo[x] && tok < row_hi[x])) sc[x][i][r] = -INFINITY;
                }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int tok = t + 8 * g + i;
                if (!(v_ok && tok >= s.t_lo && tok < s.t_hi)) {
#pragma unroll
                    for (int c = 0; c < kVw; ++c) vw[i][c] = 0u;
                    vs[i / 4] = (vs[i / 4] & ~(0xFFu << (8 * (i & 3)))) | (127u << (8 * (i & 3)));
                }
            }
            if (s.n > 1) {                                  // (one query: the tokens left are seen by all rows)
                uint32_t any = odd_scales(vs[0]) | odd_scales(vs[1]);
                if constexpr (BITS == 8)                    // (no code of 4 bits is NaN)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int c = 0; c < kVw; ++c) any |= odd_codes(vw[i][c]);
                odd = __ballot(any != 0) != 0;
            }
        }
        bf16x8 ph[NT], pl[NT];                              // the weights as two bf16 terms
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            float mx = sc[x][0][0];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) mx = __builtin_fmaxf(mx, sc[x][i][r]);
            mx = larger(across32(larger(across16(mx)))) * a.scale;
            if (__ballot(mx > m[x] + 8.0f)) {
                const float m2 = __builtin_fmaxf(m[x], mx);
                const float f = m2 == -INFINITY ? 0.0f : exp2_(m[x] - m2);
                l[x] *= f;
#pragma unroll
                for (int j = 0; j < kV; ++j) o[x][j] *= f;
                m[x] = m2;
            }
            const float ref = m[x] == -INFINITY ? 0.0f : m[x];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float p = exp2_(__builtin_fmaf(sc[x][e & 1][e >> 1], a.scale, -ref));
                l[x] += p;
                ph[x][e] = (__bf16)p;
                pl[x][e] = (__bf16)(p - (float)ph[x][e]);
            }
        }
#pragma unroll
        for (int c = 0; c < kV / 4; ++c) {                  // four channels of eight tokens
            uint32_t f[4][4];                               // [channel][token pair]
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int i0 = 2 * e, i1 = i0 + 1;
                const float s0 = scale_byte(vs[i0 / 4], i0 & 3), s1 = scale_byte(vs[i1 / 4], i1 & 3);
                const uint32_t a0 = cvt_pair<BITS>(vw[i0], 2 * c, s0), b0 = cvt_pair<BITS>(vw[i1], 2 * c, s1);
                const uint32_t a1 = cvt_pair<BITS>(vw[i0], 2 * c + 1, s0), b1 = cvt_pair<BITS>(vw[i1], 2 * c + 1, s1);
                f[0][e] = low_halves(a0, b0), f[1][e] = high_halves(a0, b0);
                f[2][e] = low_halves(a1, b1), f[3][e] = high_halves(a1, b1);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 vf = __builtin_bit_cast(bf16x8, u32x4{f[j][0], f[j][1], f[j][2], f[j][3]});
#pragma unroll
                for (int x = 0; x < NT; ++x) {
                    f32x4& acc = o[x][4 * c + j];
                    bf16x8 vx = vf;
                    if (odd) {
                        // a product of ones in their places with ones in the places that a row sees counts what each sum meets
                        u32x4 w = __builtin_bit_cast(u32x4, vf), ones;
#pragma unroll
                        for (int e = 0; e < 4; ++e) ones[e] = odd_halves(w[e]) & 0x3F803F80u, w[e] &= ~odd_halves(w[e]);
                        vx = __builtin_bit_cast(bf16x8, w);
                        bf16x8 sees;
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const int tok = t + 8 * g + e;
                            sees[e] = (__bf16)(v_ok && tok >= row_lo[x] && tok < row_hi[x] ? 1.0f : 0.0f);
                        }
                        const f32x4 z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ones), sees, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
                        for (int r = 0; r < 4; ++r) acc[r] += z[r] > 0.0f ? __builtin_nanf("") : 0.0f;
                    }
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vx, pl[x], acc, 0, 0, 0);
                    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vx, ph[x], acc, 0, 0, 0);
                }
            }
        }
        if (more) load_v(t + 128);
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
            const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
            uint16_t* p = a.out + row * a.ldo + (size_t)head * D + c0;
#pragma unroll
            for (int j = 0; j < kV; j += 4) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<bf16x4*>(p + j) = bf16x4{(__bf16)(v[j] * inv), (__bf16)(v[j + 1] * inv), (__bf16)(v[j + 2] * inv), (__bf16)(v[j + 3] * inv)};
            }
            if (a.lse && c0 == 0) a.lse[row * a.q_heads + head] = sum != 0.0f ? (top + __log2f(sum)) * 0.69314718055994531f : -INFINITY;
        } else {
            const size_t at = ((size_t)bh * a.part_rows + r) * a.max_parts + part;
#pragma unroll
            for (int j = 0; j < kV; j += 4) *reinterpret_cast<f32x4*>(a.part_o + at * D + c0 + j) = f32x4{v[j], v[j + 1], v[j + 2], v[j + 3]};
            if (c0 == 0) a.part_ml[2 * at] = top, a.part_ml[2 * at + 1] = sum;
        }
    }
}

// Joins the parts of a row: W waves take the parts in turn, or for W = 0 half a wave takes them all, eight in flight each, and
// they are added in wave order; `at` is the row's first part.  Every wave of the workgroup takes part (W = 0: `parts` is 0 where there is
// nothing to join).
template <int D, int W>
__device__ __forceinline__ void join_row(const AttnArgs& a, const float* part_o, const float* part_ml, size_t at, int parts,
                                         size_t row, int head) {
    constexpr int kLanes = W == 0 ? 32 : 64, kC = D / kLanes, kStep = W == 0 ? 1 : W;
    __shared__ float s_v[W ? W : 1][D], s_sum[W ? W : 1];
    const int lane = threadIdx.x & (kLanes - 1), wave = W <= 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    float top = -INFINITY;
    for (int p = lane; p < parts; p += kLanes) top = __builtin_fmaxf(top, part_ml[2 * (at + p)]);
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) top = __builtin_fmaxf(top, shuffle_xor(top, d));
    const float ref = top == -INFINITY ? 0.0f : top;
    float sum = 0.0f, v[kC] = {};
    for (int p0 = wave; p0 < parts; p0 += 8 * kStep) {      // parts p0, p0 + W, .. p0 + 7 W; past the end: the last one, weight 0
        float x[8][kC], m[8], l[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const size_t p = at + min(p0 + kStep * j, parts - 1);
            m[j] = part_ml[2 * p], l[j] = part_ml[2 * p + 1];
#pragma unroll
            for (int c = 0; c < kC; ++c) x[j][c] = part_o[p * D + lane * kC + c];
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float f = p0 + kStep * j < parts ? exp2_(m[j] - ref) : 0.0f;
            sum = __builtin_fmaf(f, l[j], sum);
#pragma unroll
            for (int c = 0; c < kC; ++c) v[c] = __builtin_fmaf(f, x[j][c], v[c]);
        }
    }
    if constexpr (W > 1) {
#pragma unroll
        for (int c = 0; c < kC; ++c) s_v[wave][lane * kC + c] = v[c];
        if (lane == 0) s_sum[wave] = sum;
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 1; w < W; ++w) {
            sum += s_sum[w];
#pragma unroll
            for (int c = 0; c < kC; ++c) v[c] += s_v[w][lane * kC + c];
        }
    }
    if (W == 0 && parts == 0) return;
    const float inv = sum != 0.0f ? 1.0f / sum : 0.0f;
    __bf16* o = reinterpret_cast<__bf16*>(a.out + row * a.ldo + (size_t)head * D + lane * kC);
#pragma unroll
    for (int c = 0; c < kC; ++c) o[c] = (__bf16)(v[c] * inv);
    if (a.lse && lane == 0) a.lse[row * a.q_heads + head] = sum != 0.0f ? (top + __log2f(sum)) * 0.69314718055994531f : -INFINITY;
}

// Many query rows to a key head (prompts, chunks of prompts): bound by the matrix pipe and the vector instructions around the
// exponentials, which add up where the two waves of a SIMD run in step.  A causal prompt of 8192 tokens with 32 query and 8 key
// heads of 128: 598 us = 920 TFLOP/s.  Not better: two groups of waves a phase apart with a barrier for each (744), half of
// the waves a tile behind (980, spills), 128 rows to a workgroup (835), raw codes through LDS (964), two or four operands
// less or more read ahead (676 to 703 beside 676, profiled).  Codes of 4 bits take as long: 4096 queries behind 12288 tokens 955 us, 975 in 8 bits.
// A workgroup of eight waves takes 256 rows (row = query token * group + head of the group) of one (sequence, key head), 32
// to a wave, and walks the visible tokens in tiles of 64.  The codes of the next tile are requested while this one is
// worked on, converted once for all eight waves and written to LDS as bf16:
//   keys    [64][D] in chunks of 8 channels, values transposed, [D][64] in chunks of 8 tokens (chunk 2j + h of tokens
//           16j + 4h .. + 3 and 16j + 8 + 4h .. + 3: those whose weights lane half h holds); a chunk's place in its row is
//           XORed with the row's number so that 16 lanes that read a chunk of 16 rows reach all banks
//   scores  result element r of 32-token tile x in lane (n, h) = (l % 32, l / 32) is row n, token 32x + 8 (r / 4) + 4h + r % 4
// The weights are rounded to bf16 once (2^-8 at most): two terms would add half of the products again.  Against 64 bits the
// prompt is 0.0020 off (root of squares, relative), of which rounding the output to bf16 is 0.0015.  The reference
// of the exponentials moves only when a row's maximum has grown by more than 2^8, which spares most rescalings of O.
// Up to 32 rows attend_few is the faster one: 16 x 4096 tokens, 32 rows of 4 heads of 128: 50 us beside 81; 64-channel heads 15
// beside 30.  In a call with sequences of more rows it takes those of up to 16 only: 64 sequences of 2048 tokens beside a chunk of 256
// queries (32 and 8 heads of 128) 150 us with 16 rows each, which attend_few takes, 197 with 32, which attend_many takes (alone
// 66 and 94).
constexpr int kManyRows = 256;

template <int D>
__device__ __forceinline__ int k_place(int row, int chunk) { return D == 128 ? chunk ^ (row & 15) : chunk ^ ((row >> 1) & 7); }
__device__ __forceinline__ int v_place(int row, int chunk) { return chunk ^ (((row >> 1) ^ (row >> 4 & 1)) & 7); }

template <int D>
constexpr int many_lds() { return 4 * 64 * D * 2 + 2 * 16; }   // two buffers of keys and values, marks

// Tokens that some row of a sequence's 256-row tile sees.
__device__ __forceinline__ TokenRange tile_tokens(const AttnArgs& a, const Seq& s, int tile) {
    const int i0 = tile * kManyRows / a.group, i1 = (min(s.n * a.group, (tile + 1) * kManyRows) - 1) / a.group;
    TokenRange t;
    t.hi = a.causal ? max(0, min(s.len, s.first_pos + i1 + 1)) : s.len;
    t.lo = min(t.hi, first_seen(a, s.first_pos + i0));
    return t;
}

// The sequence and 256-row tile of workgroup tile `x`, last ones first (they see the most tokens); b < 0: none.
__device__ __forceinline__ void find_tile(const AttnArgs& a, int x, int* b, int* tile) {
    const int lane = threadIdx.x & 63;
    auto tiles_of = [&](int i) {
        if (i >= a.batch) return 0;
        const Seq s = sequence(a, i);
        const int rows = s.n * a.group;
        return rows > a.few_rows ? (rows + kManyRows - 1) / kManyRows : 0;
    };
    int total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        int c = tiles_of(b0 + lane);
#pragma unroll
        for (int d = 32; d; d >>= 1) c += __shfl_xor(c, d);
        total += c;
    }
    *b = -1, *tile = 0;
    int left = total - 1 - x;                               // the tile's number from the front
    if (left < 0) return;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const int c = tiles_of(b0 + lane);
        int sum = c;                                        // inclusive prefix sum over the lanes
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(sum, d);
            if (lane >= d) sum += v;
        }
        const uint64_t past = __ballot(sum > left);
        if (past) {
            const int l = __builtin_ctzll(past);
            *b = __builtin_amdgcn_readfirstlane(b0 + l);
            *tile = __builtin_amdgcn_readfirstlane(left - __shfl(sum - c, l));
            return;
        }
        left -= __shfl(sum, 63);
    }
}

constexpr int kDeep = 6;                                    // operands that are read ahead of their product

template <int D, int BITS>
__global__ void __launch_bounds__(512, 2)
attend_many(const AttnArgs a) {
    constexpr int kU = D / 16, kCb = D / 32, kHalf = 64 * D * 2;
    constexpr int kToken = D * BITS / 8;                    // bytes of a token's codes
    extern __shared__ __align__(16) uint8_t lds[];
    uint8_t* const s_k = lds;                               // [2][64][D] bf16
    uint8_t* const s_v = lds + 2 * kHalf;                   // [2][D][64] bf16
    uint8_t* const s_ok = lds + 4 * kHalf;                  // [2][4]: whether the page of 16 tokens exists
    uint8_t* const s_odd = s_ok + 16;                       // [8]: whether a wave took values as zero
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, hh = lane >> 5;
    const int h = blockIdx.x % a.kv_heads, xp = blockIdx.x / a.kv_heads;
    const int part = xp % a.many_parts;
    int b, tile;
    find_tile(a, xp / a.many_parts, &b, &tile);
    b = __builtin_amdgcn_readfirstlane(b), tile = __builtin_amdgcn_readfirstlane(tile);
    if (b < 0) return;
    const Seq s = sequence(a, b);
    const int rows = s.n * a.group, row0 = tile * kManyRows;
    const TokenRange range = tile_tokens(a, s, tile);
    const int parts = range_parts(range, a.many_len);
    if (part >= parts) return;
    const int t_begin = (range.lo & ~63) + part * a.many_len, t_end = min(range.hi, t_begin + a.many_len);

    // this lane's row
    const int r = row0 + wave * 32 + n, i = r / a.group;
    const bool live = r < rows;
    const int head = h * a.group + (live ? r - i * a.group : 0);
    const size_t row = (size_t)(s.begin + (live ? i : 0));
    bf16x8 qf[kU];
    {
        const uint16_t* p = a.q + row * a.ldq + (size_t)head * D + 8 * hh;
#pragma unroll
        for (int u = 0; u < kU; ++u) qf[u] = *reinterpret_cast<const bf16x8*>(p + 16 * u);
    }
    const int pos = s.first_pos + i;
    const int row_hi = !live ? 0 : a.causal ? min(s.len, pos + 1) : s.len;
    const int row_lo = first_seen(a, pos);
    // the wave's rows: [some_lo, some_hi) is seen by some, [all_lo, all_hi) by all of them
    const int wr0 = row0 + wave * 32, wr1 = min(rows, wr0 + 32) - 1;
    const bool wave_live = wr0 < rows;
    const int wp0 = s.first_pos + wr0 / a.group, wp1 = s.first_pos + wr1 / a.group;
    const int some_hi = !wave_live ? 0 : a.causal ? min(s.len, wp1 + 1) : s.len, some_lo = first_seen(a, wp0);
    const int all_hi = a.causal ? min(s.len, wp0 + 1) : s.len, all_lo = first_seen(a, wp1);
    // likewise of the workgroup's rows
    const int last_pos = s.first_pos + (min(rows, row0 + kManyRows) - 1) / a.group;
    const int tile_all_hi = a.causal ? min(s.len, s.first_pos + row0 / a.group + 1) : s.len, tile_all_lo = first_seen(a, last_pos);

    // staging: a thread has a piece of 16 channels of a key and a 4 x 4 piece of values (D = 64: one or the other).  A wave's 8
    // (16) tokens lie in one page: pages and addresses are scalars, what a lane adds to them stays the same
    const int32_t* table = a.page_table + (size_t)b * a.table_width;
    const int page_mask = (1 << a.page_shift) - 1, last_page = max(0, (s.len - 1) >> a.page_shift);
    const bool do_k = D == 128 || wave < 4, do_v = D == 128 || wave >= 4;
    constexpr int kKc = D / 16, kVc = D / 4;                // pieces of a key, of four values' tokens
    const int tok0 = D == 128 ? wave * 8 : (wave & 3) * 16; // the wave's first token of the tile
    const int k_tok = lane / kKc, k_c = lane % kKc;         // from there: this lane's key, its 16 channels
    const int v_tok = lane / kVc * 4, v_c = lane % kVc;     // tokens v_tok .. + 3, channels 4 v_c .. + 3
    const uint32_t k_lane = lane * (2 * BITS), ks_lane = ((uint32_t)(k_c / 2) << a.page_shift) + k_tok;
    const uint32_t v_lane = v_tok * kToken + v_c * (BITS / 2), vs_lane = ((uint32_t)(v_c / 8) << a.page_shift) + v_tok;
    auto entry = [&](int t) {                               // page of the wave's tokens of the tile that starts with t
        return __builtin_amdgcn_readfirstlane(table[min((t + tok0) >> a.page_shift, last_page)]);
    };
    uint32_t kw[BITS / 2] = {};
    uint32_t kscale = 0, vw[4] = {}, vscale = 0;
    bool there = false;
    auto request = [&](int t, int page) {
        there = (uint32_t)page < (uint32_t)a.num_pages;
        const int64_t ph = (int64_t)(there ? page : 0) * a.kv_heads + h;
        const int off = (t + tok0) & page_mask;
        const int64_t codes = ((ph << a.page_shift) + off) * kToken, scales = ((ph * (D / 32)) << a.page_shift) + off;
        if (do_k) {
            load_words<BITS / 2>(kw, a.k_codes + codes + k_lane);
            kscale = a.k_scales[scales + ks_lane];
        }
        if (do_v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) vw[e] = load_four<BITS>(a.v_codes + codes + v_lane + e * kToken);
            vscale = *reinterpret_cast<const uint32_t*>(a.v_scales + scales + vs_lane);
        }
    };
    uint32_t k_to[2], v_to[4];                              // where the piece goes in a buffer
#pragma unroll
    for (int e = 0; e < 2; ++e) k_to[e] = (tok0 + k_tok) * (D * 2) + k_place<D>(tok0 + k_tok, 2 * k_c + e) * 16;
    {
        const int quad = (tok0 + v_tok) / 4, chunk = 2 * (quad >> 2) + (quad & 1), half = (quad >> 1) & 1;
#pragma unroll
        for (int c = 0; c < 4; ++c) v_to[c] = (4 * v_c + c) * 128 + v_place(4 * v_c + c, chunk) * 16 + half * 8;
    }
    auto partly_seen = [&](int t) { return t < tile_all_lo || t + 64 > tile_all_hi; };
    bool odd = false;                                       // wave-uniform
    auto stage = [&](int t, int buf) {                      // the requested tile (first token t) into LDS
        if (do_k) {
            const float sc = scale_operand(kscale);
#pragma unroll
            for (int e = 0; e < 2; ++e)
                *reinterpret_cast<bf16x8*>(s_k + buf * kHalf + k_to[e]) = cvt_eight<BITS>(kw + e * (BITS / 4), sc);
            if (k_c == 0 && ((tok0 + k_tok) & 15) == 0) s_ok[buf * 4 + (tok0 + k_tok) / 16] = there;
        }
        if (do_v) {
            // places that nobody sees may hold anything: a weight of zero must stay a product of zero
            if (!there || t < range.lo || t + 64 > range.hi) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int tok = t + tok0 + v_tok + e;
                    if (!(there && tok >= range.lo && tok < range.hi)) {
                        vw[e] = 0u;
                        vscale = (vscale & ~(0xFFu << (8 * e))) | (127u << (8 * e));
                    }
                }
            }
            uint32_t lo[4], hi[4];                          // [token] channels 0, 1 and 2, 3
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float sc = scale_byte(vscale, e);
                lo[e] = cvt_pair<BITS>(vw + e, 0, sc), hi[e] = cvt_pair<BITS>(vw + e, 1, sc);
            }
            if (partly_seen(t) && __ballot((odd_scales(vscale) | (BITS == 8 ? odd_codes(vw[0]) | odd_codes(vw[1]) | odd_codes(vw[2]) | odd_codes(vw[3]) : 0u)) != 0)) {
                odd = true;
#pragma unroll
                for (int e = 0; e < 4; ++e) lo[e] &= ~odd_halves(lo[e]), hi[e] &= ~odd_halves(hi[e]);
            }
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const uint32_t* w = c < 2 ? lo : hi;
                *reinterpret_cast<u32x2*>(s_v + buf * kHalf + v_to[c]) =
                    c & 1 ? u32x2{high_halves(w[0], w[1]), high_halves(w[2], w[3])} : u32x2{low_halves(w[0], w[1]), low_halves(w[2], w[3])};
            }
        }
    };

    float m = -INFINITY, l = 0.0f;
    v16f o[kCb];
#pragma unroll
    for (int c = 0; c < kCb; ++c) o[c] = v16f{};

    int page = 0;                                           // of the tile after the one that is requested next
    if (t_begin < t_end) {
        request(t_begin, entry(t_begin));
        page = entry(t_begin + 64);
        stage(t_begin, 0);
    }
    __syncthreads();
    int buf = 0;
    for (int t = t_begin; t < t_end; t += 64, buf ^= 1) {
        const bool more = t + 64 < t_end;
        if (more) {
            request(t + 64, page);
            page = entry(t + 128);
        }
        if (t < some_hi && t + 64 > some_lo) {              // wave-uniform
            // chunk 2 j + h of a lane's row is at (the row's address with chunk h) ^ 32 j; opaque, or every address of a tile
            // would be kept in a register of its own
            uint32_t at_v = (uint32_t)(n * 128 + v_place(n, hh) * 16), at_k = (uint32_t)(n * (D * 2) + k_place<D>(n, hh) * 16);
            asm volatile("" : "+v"(at_v), "+v"(at_k));
            const uint32_t ok = *reinterpret_cast<const uint32_t*>(s_ok + buf * 4);
            // operand i of the keys: tile half i % 2, step i / 2; of the values: channel block i % kCb, step i / kCb (neighbouring
            // products go to different sums).  They are read kDeep products ahead, the first values before the softmax
            auto read_k = [&](int i) { return *reinterpret_cast<const bf16x8*>(s_k + buf * kHalf + (at_k ^ (uint32_t)(i / 2 * 32)) + i % 2 * 32 * (D * 2)); };
            auto read_v = [&](int i) { return *reinterpret_cast<const bf16x8*>(s_v + buf * kHalf + (at_v ^ (uint32_t)(i / kCb * 32)) + i % kCb * 32 * 128); };
            v16f sc[2];
            bf16x8 ring[kDeep];
#pragma unroll
            for (int i = 0; i < kDeep; ++i) ring[i] = read_k(i);
#pragma unroll
            for (int i = 0; i < 2 * kU; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                sc[i % 2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % kDeep], qf[i / 2], i < 2 ? v16f{} : sc[i % 2], 0, 0, 0);
                if (i + kDeep < 2 * kU) ring[i % kDeep] = read_k(i + kDeep);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kDeep; ++i) ring[i] = read_v(i);
            if (t < all_lo || t + 64 > all_hi || ok != 0x01010101u) {
                // (in integer arithmetic: conditions would take two scalar registers for each element)
                const int first = row_lo - t - 4 * hh, last = row_hi - 1 - t - 4 * hh;
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int at = 32 * x + 8 * (e >> 2) + (e & 3);
                        const int hide = ((at - first) | (last - at) | ((int)((ok >> (8 * (2 * x + (e >> 3)))) & 1u) - 1)) >> 31;
                        sc[x][e] = __uint_as_float((__float_as_uint(sc[x][e]) & ~(uint32_t)hide) | (0xFF800000u & (uint32_t)hide));
                    }
            }
            float mx = sc[0][0];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) mx = __builtin_fmaxf(mx, sc[x][e]);
            if (__ballot(mx * a.scale > m + 8.0f)) {        // (the two halves of a row are compared only then)
                mx = __builtin_fmaxf(mx, shuffle_xor(mx, 32)) * a.scale;
                const float m2 = __builtin_fmaxf(m, mx);
                const float f = m2 == -INFINITY ? 0.0f : exp2_(m - m2);
                l *= f;
#pragma unroll
                for (int c = 0; c < kCb; ++c) o[c] *= f;
                m = m2;
            }
            const float ref = m == -INFINITY ? 0.0f : m;
            bf16x8 pf[4];
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float p = exp2_(__builtin_fmaf(sc[x][e], a.scale, -ref));
                    l += p;
                    pf[2 * x + (e >> 3)][e & 7] = (__bf16)p;
                }
#pragma unroll
            for (int i = 0; i < 4 * kCb; ++i) {
                __builtin_amdgcn_sched_barrier(0);
                o[i % kCb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ring[i % kDeep], pf[i / kCb], o[i % kCb], 0, 0, 0);
                if (i + kDeep < 4 * kCb) ring[i % kDeep] = read_v(i + kDeep);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (more) stage(t + 64, buf ^ 1);
        __syncthreads();
    }
    if (lane == 0) s_odd[wave] = odd;
    __syncthreads();
    const u32x2 odds = *reinterpret_cast<const u32x2*>(s_odd);
    if (odds[0] | odds[1]) {                                // (rare: as slow as it likes)
        for (int tok = t_begin; tok < t_end; ++tok) {
            const int pg = table[min(tok >> a.page_shift, last_page)];
            if (!partly_seen(tok & ~63) || tok < range.lo || (uint32_t)pg >= (uint32_t)a.num_pages) continue;
            const bool sees = tok >= row_lo && tok < row_hi;
            const int64_t ph = (int64_t)pg * a.kv_heads + h;
            const uint8_t* p = a.v_codes + ((ph << a.page_shift) + (tok & page_mask)) * kToken + hh * (BITS / 2);
#pragma unroll
            for (int c = 0; c < kCb; ++c) {
                const float sc = scale_operand(a.v_scales[((ph * (D / 32) + c) << a.page_shift) + (tok & page_mask)]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t w = load_four<BITS>(p + (32 * c + 8 * e) * BITS / 8);
                    const uint32_t x = odd_halves(cvt_pair<BITS>(&w, 0, sc)), y = odd_halves(cvt_pair<BITS>(&w, 1, sc));
                    const uint32_t hit[4] = {x & 0xFFFFu, x >> 16, y & 0xFFFFu, y >> 16};
#pragma unroll
                    for (int k = 0; k < 4; ++k) o[c][4 * e + k] += sees && hit[k] ? __builtin_nanf("") : 0.0f;
                }
            }
        }
    }
    if (!live || i >= s.n) return;
    l += shuffle_xor(l, 32);
    // element e of o[c] is channel 32c + 8 (e / 4) + 4h + e % 4
    if (parts == 1) {
        const float inv = l != 0.0f ? 1.0f / l : 0.0f;
        uint16_t* p = a.out + row * a.ldo + (size_t)head * D + 4 * hh;
#pragma unroll
        for (int c = 0; c < kCb; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                *reinterpret_cast<bf16x4*>(p + 32 * c + 8 * e) =
                    bf16x4{(__bf16)(o[c][4 * e] * inv), (__bf16)(o[c][4 * e + 1] * inv), (__bf16)(o[c][4 * e + 2] * inv), (__bf16)(o[c][4 * e + 3] * inv)};
            }
        if (a.lse && hh == 0) a.lse[row * a.q_heads + head] = l != 0.0f ? (m + __log2f(l)) * 0.69314718055994531f : -INFINITY;
    } else {
        const size_t at = (row * a.q_heads + head) * a.many_parts + part;
        float* p = a.many_o + at * D + 4 * hh;
#pragma unroll
        for (int c = 0; c < kCb; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e) *reinterpret_cast<f32x4*>(p + 32 * c + 8 * e) = f32x4{o[c][4 * e], o[c][4 * e + 1], o[c][4 * e + 2], o[c][4 * e + 3]};
        if (hh == 0) a.many_ml[2 * at] = m, a.many_ml[2 * at + 1] = l;
    }
}

// A row of a (sequence, key head) of few rows: by a workgroup.
template <int D>
__device__ __forceinline__ void join_few(const AttnArgs& a, unsigned unit) {
    const unsigned bh = unit / (unsigned)a.part_rows;
    const int r = (int)(unit - bh * a.part_rows), h = (int)(bh % a.kv_heads), b = (int)(bh / a.kv_heads);
    const Seq s = sequence(a, b);
    const int rows = s.n * a.group;
    if (r >= rows || rows > a.few_rows) return;
    const int parts = live_parts(s, a.few_len);
    if (parts == 1) return;
    join_row<D, 4>(a, a.part_o, a.part_ml, (size_t)unit * a.max_parts, parts, (size_t)s.begin + r / a.group, h * a.group + r % a.group);
}

// Two (row of q, query head) pairs of sequences with many rows, by a wave's halves: there are many of them, of few parts.  The wave
// looks for the first one's sequence; the second one's is mostly the same, else it is looked for too.
template <int D>
__device__ __forceinline__ void join_many(const AttnArgs& a, unsigned pair) {
    const int lane = threadIdx.x & 63;
    const int64_t units = (int64_t)a.total_q * a.q_heads, unit = 2 * (int64_t)pair + (lane >> 5);
    const int row = (int)(unit / a.q_heads), head = (int)(unit - (int64_t)row * a.q_heads);
    int b = -1;                                             // the half's sequence
    for (int half = 0; half < 2; ++half) {
        const int r = __builtin_amdgcn_readfirstlane(__shfl(row, 32 * half));
        if (half == 1 && r == __builtin_amdgcn_readfirstlane(row)) break;
        int found = -1;
        for (int b0 = 0; b0 < a.batch && found < 0; b0 += 64) {      // lanes look at 64 sequences at a time
            bool mine = false;
            if (b0 + lane < a.batch) {
                const int begin = a.cu_q[b0 + lane], end = a.cu_q[b0 + lane + 1];
                mine = begin >= 0 && end <= a.total_q && r >= begin && r < end;
            }
            const uint64_t m = __ballot(mine);
            if (m) found = b0 + __builtin_ctzll(m);
        }
        if (half == 0 || lane >= 32) b = found;
    }
    int parts = 0;
    if (b >= 0 && unit < units) {
        const Seq s = sequence(a, b);
        const int rows = s.n * a.group, i = row - s.begin;
        if (i < s.n && rows > a.few_rows) {
            parts = range_parts(tile_tokens(a, s, (i * a.group + head % a.group) / kManyRows), a.many_len);
            if (parts == 1) parts = 0;                      // (it has been written)
        }
    }
    if (__ballot(parts != 0) == 0) return;
    join_row<D, 0>(a, a.many_o, a.many_ml, (size_t)unit * a.many_parts, parts, (size_t)row, head);
}

// Joins what both kernels have cut: the first `few` workgroups take a row each, the others eight.
template <int D>
__global__ void __launch_bounds__(256)
join_parts(const AttnArgs a, unsigned few) {
    if (blockIdx.x < few) join_few<D>(a, blockIdx.x);
    else join_many<D>(a, (blockIdx.x - few) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
}

}  // namespace

namespace {

struct Plan {
    int few_rows, few_len, max_parts, part_rows;
    int many_tiles, many_len, many_parts;
    bool few, many;                                         // which kernels run
};

// Rows x parts that attend_many may be cut into for calls of at most total_q queries and max_kv tokens: what the estimate below
// asks for, give or take.  It weighs tokens / 64 n blocks of a part against writing n rows' results, which makes n fall
// with the root of tokens / rows, and rows x parts grow with that of tokens x rows; rows are cut only while there are fewer
// tiles of them than compute units.  Never more than 2^20, sixteen tiles to a compute unit (thousands of rows over contexts from
// 131072 tokens on would be cut further: to 0.94 of the estimated time at best up to 2^20 tokens).  Grows with both arguments, so
// that a workspace serves smaller calls.
int64_t many_room(int head_dim, int q_heads, int kv_heads, int64_t total_q, int max_kv, int compute_units) {
    if (max_kv < 512) return 0;
    int64_t rows = (int64_t)kManyRows * (compute_units + kv_heads);
    if (rows > total_q * q_heads) rows = total_q * q_heads;
    const int64_t all = rows * ((max_kv < 64 * 256 ? max_kv / 256 : 64) + 1);
    const int64_t most = (int64_t)(sqrt((double)rows * (max_kv + 1024.0)) * (head_dim == 64 ? 22.6 : 16.0));
    const int64_t least = all < most ? all : most;
    return least < (1 << 20) ? least : 1 << 20;
}

// Part length of attend_few: enough workgroups for four to a compute unit where there are tokens for it, at least 256
// tokens (two blocks for each wave) and at most 1024, so that the longest of ragged sequences does not outlast the others
// (64 sequences of up to 8192 tokens: parts of 512 and 1024 tokens 35 us, of 256 45 us; 4 of up to 131072: 74 us, 80 us).
// A window bounds the tokens that matter: of a sequence of few rows, of a tile of many.
// Where row tiles fill the compute units attend_many does not cut the tokens, and a sequence much longer than the others is
// walked by one workgroup to a key head and tile (prompt of 8192 tokens 573 us, 16 queries over 131072 tokens 140, both in one call
// 3776): parts that only it has would be workgroups without work for all other tiles, and room for their rows.
// attend_many cuts the tokens only where its row tiles are fewer than the compute units (one workgroup to each at a time), into the
// number of parts with the least estimated time, in units of a block of 64 tokens (about 2 us): whole rounds over the card
// where the tiles are alike (1.1: a round of exactly all compute units has come out as two), half of that and a part at the
// end where they are not (lengths, the triangle of a prompt); 4 blocks for what a part begins and ends with, 4 for the
// join, 10 MB of partial results written and read to a block.  Beside parts that make one workgroup, or two, to a compute
// unit: 4 sequences of 256 queries and 8192 tokens, 32 and 8 heads of 128 channels 216 us (273, 216); 8 of 128 and 2048 79
// (80, 89); 2 of 512 and 4096, 8 heads and 1, 44 (43, 60); 9 ragged sequences of up to 500 queries and 10000 tokens with a
// window of 4096, 16 heads and 2 of 64, 37 (45, 37).
Plan plan(int head_dim, int group, int kv_heads, int batch, int total_q, int max_q, int max_kv, int window, int compute_units) {
    Plan p = {};
    const int64_t rows = (int64_t)max_q * group;
    p.many = rows > 32;
    p.few = !p.many || batch > 1;
    p.few_rows = !p.few ? 0 : p.many ? 16 : rows > 16 ? 32 : 16;
    p.part_rows = (int)(rows < p.few_rows ? rows : p.few_rows);
    auto span = [&](int queries) { return window > 0 && window < max_kv - queries ? window + queries : max_kv; };
    p.max_parts = 1, p.few_len = 256;
    if (p.few) {
        const int64_t tokens = span(p.few_rows);
        int64_t len = (batch * kv_heads * tokens / (4 * compute_units) + 255) & ~int64_t(255);
        if (len < 256) len = 256;
        if (len > 1024) len = 1024;
        p.few_len = (int)len;
        p.max_parts = (int)((tokens + 63 + len - 1) / len);
        if (p.max_parts < 1) p.max_parts = 1;
    }
    p.many_parts = 1, p.many_len = 1 << 30;
    if (p.many) {
        // sum of ceil(rows / 256) over sequences of more than few_rows rows, rows / (few_rows + 1) of them at most
        const int64_t all = (int64_t)total_q * group, longer = all / (p.few_rows + 1);
        p.many_tiles = (int)(all / kManyRows + (longer < batch ? longer : batch));
        const bool same = (int64_t)batch * max_q == total_q;   // every sequence has max_q queries
        const int64_t tiles = same ? batch * ((rows + kManyRows - 1) / kManyRows) : all / kManyRows + (longer < batch ? longer : batch) / 2;
        const int64_t units = (tiles < 1 ? 1 : tiles) * kv_heads, tokens = span(kManyRows / group + 1);
        const bool even = same && max_q <= max_kv / 4;
        const int64_t room = many_room(head_dim, group * kv_heads, kv_heads, total_q, max_kv, compute_units);
        double best = 0;
        for (int n = 1; n == 1 || (units < compute_units && n <= 64 && n * 256 <= tokens); ++n) {
            const int64_t len = ((tokens + n - 1) / n + 63) & ~int64_t(63), parts = n > 1 ? (tokens + 63 + len - 1) / len : 1;
            if (n > 1 && all * kv_heads * parts > room) continue;
            const double load = (double)units * n / compute_units;
            double cost = (even ? ceil(1.1 * load) : 0.5 * load + 1.0) * (double)(len / 64 + 4);
            if (n > 1) cost += 4.0 + (double)total_q * group * kv_heads * n * head_dim * 8e-7;
            if (n > 1 && cost >= best) continue;
            best = cost;
            p.many_len = n > 1 ? (int)len : 1 << 30;
            p.many_parts = (int)parts;
        }
    }
    return p;
}

// Partial results: rows x parts of attend_few, then of attend_many.
int64_t few_units(const Plan& p, int batch, int kv_heads) { return p.max_parts > 1 ? (int64_t)batch * kv_heads * p.part_rows * p.max_parts : 0; }
int64_t many_units(const Plan& p, int total_q, int q_heads) { return p.many_parts > 1 ? (int64_t)total_q * q_heads * p.many_parts : 0; }

template <int D, int BITS>
hipError_t launch_attention(const AttnArgs& a, const Plan& p, int dev, hipStream_t stream) {
    if (p.many) {
        if (hipError_t e = ensure_dynamic_lds<&attend_many<D, BITS>>(dev, many_lds<D>()); e != hipSuccess) return e;
        attend_many<D, BITS><<<(unsigned)p.many_tiles * p.many_parts * a.kv_heads, 512, many_lds<D>(), stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (p.few) {
        const unsigned units = (unsigned)a.batch * a.kv_heads * p.max_parts;
        if (p.few_rows == 16) attend_few<D, 1, BITS><<<units, 256, 0, stream>>>(a);
        else attend_few<D, 2, BITS><<<units, 256, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    const unsigned few = p.max_parts > 1 ? (unsigned)a.batch * a.kv_heads * p.part_rows : 0;
    const unsigned many = p.many_parts > 1 ? ((unsigned)a.total_q * a.q_heads + 7) / 8 : 0;
    if (few + many == 0) return hipSuccess;
    join_parts<D><<<few + many, 256, 0, stream>>>(a, few);
    return hipGetLastError();
}

}  // namespace

namespace {

size_t part_bytes(const Plan& p, const batq_paged_cache& c, int q_heads, int batch, int total_q) {
    return (size_t)(few_units(p, batch, c.kv_heads) + many_units(p, total_q, q_heads)) * (c.head_dim + 2) * 4;
}

}  // namespace

size_t paged_attention_part_bytes(const batq_paged_cache& c, int q_heads, int batch, int total_q, int max_q, int max_kv,
                                  int compute_units) {
    return part_bytes(plan(c.head_dim, q_heads / c.kv_heads, c.kv_heads, batch, total_q, max_q, max_kv, 0, compute_units), c, q_heads, batch, total_q);
}

// At least the former for every batch, total_q, max_q and max_kv up to the given ones (a few sequences are cut into more parts
// than many, few rows than a prompt).  attend_few: up to 32 rows of each pair of a sequence and a key head, one part to
// 256 tokens but at most four to a compute unit (a 64th more: the rounding of their length), or to 1024 tokens; each pair's
// last part and the one by which a range that starts inside a block can be longer, 1 + 62 / 256, on top.
size_t paged_attention_workspace_bytes(const batq_paged_cache& c, int q_heads, int batch, int total_q, int max_q, int max_kv,
                                       int compute_units) {
    const int64_t rows = (int64_t)max_q * (q_heads / c.kv_heads), pairs = (int64_t)batch * c.kv_heads;
    int64_t units = 0;
    if (max_kv > 256 - 63) {
        int64_t parts = (pairs * max_kv + 255) / 256;
        if (parts > 4 * compute_units + compute_units / 16 + 1) parts = 4 * compute_units + compute_units / 16 + 1;
        if (parts < (pairs * max_kv + 1023) / 1024) parts = (pairs * max_kv + 1023) / 1024;
        units = (parts + pairs + (pairs + 3) / 4) * (rows < 32 ? rows : 32);
    }
    if (rows > 32) units += many_room(c.head_dim, q_heads, c.kv_heads, total_q, max_kv, compute_units);
    return (size_t)units * (c.head_dim + 2) * 4;
}

hipError_t launch_paged_attention(const batq_paged_cache& c, int bits, const batq_paged_batch& b, const void* q, int64_t ldq,
                                  int q_heads, float scale, bool causal, int window, void* out, int64_t ldo, float* lse,
                                  void* workspace, hipStream_t stream) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    const int cus = e == hipSuccess ? device_compute_units(dev, &e) : 0;
    if (e != hipSuccess) return e;
    // a window's plan where it needs no more room than the plan without one, which is what the workspace is sized for
    const Plan full = plan(c.head_dim, q_heads / c.kv_heads, c.kv_heads, b.batch, b.total_q, b.max_q, b.max_kv, 0, cus);
    // (without causal a window has no upper end)
    Plan p = plan(c.head_dim, q_heads / c.kv_heads, c.kv_heads, b.batch, b.total_q, b.max_q, b.max_kv, causal ? window : 0, cus);
    if (part_bytes(p, c, q_heads, b.batch, b.total_q) > part_bytes(full, c, q_heads, b.batch, b.total_q)) p = full;
    AttnArgs a = {};
    set_lists(a, c, b, q_heads, causal, window);
    a.q = static_cast<const uint16_t*>(q), a.ldq = ldq, a.ldo = ldo, a.out = static_cast<uint16_t*>(out), a.lse = lse;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales, a.v_codes = c.v_codes, a.v_scales = c.v_scales;
    a.scale = scale * 1.4426950408889634f;
    a.few_rows = p.few_rows, a.few_len = p.few_len, a.max_parts = p.max_parts, a.part_rows = p.part_rows;
    a.many_len = p.many_len, a.many_parts = p.many_parts;
    const size_t few = (size_t)few_units(p, b.batch, c.kv_heads), many = (size_t)many_units(p, b.total_q, q_heads);
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.part_o + few * c.head_dim;
    a.many_o = a.part_ml + few * 2;
    a.many_ml = a.many_o + many * c.head_dim;
    if (bits == 8) return c.head_dim == 64 ? launch_attention<64, 8>(a, p, dev, stream) : launch_attention<128, 8>(a, p, dev, stream);
    return c.head_dim == 64 ? launch_attention<64, 4>(a, p, dev, stream) : launch_attention<128, 4>(a, p, dev, stream);
}

}  // namespace batq
