// Attention over the paged MXFP8 cache: one pass over a sequence's keys and values with the running maximum and sum
// of the softmax.  gfx950 only.
#include <math.h>

#include "batq_internal.h"
#include "mxfp4_device.h"

namespace batq {
namespace {

struct AttnArgs {
    const uint16_t* q;
    int64_t ldq, ldo;
    uint16_t* out;
    float* lse;
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t *cu_q, *kv_len, *page_table;
    int batch, table_width, total_q, max_q, max_kv, num_pages, page_shift, q_heads, kv_heads, group;
    int causal, window;
    float scale;
};

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
    if (b == a.batch || row - begin >= a.max_q) return;
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
                s *= a.scale;
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

size_t paged_attention_workspace_bytes(const batq_paged_cache&, int, int, int, int, int, int) { return 0; }

hipError_t launch_paged_attention(const batq_paged_cache& c, const batq_paged_batch& b, const void* q, int64_t ldq,
                                  int q_heads, float scale, bool causal, int window, void* out, int64_t ldo, float* lse,
                                  void*, hipStream_t stream) {
    AttnArgs a = {};
    a.q = static_cast<const uint16_t*>(q), a.ldq = ldq, a.ldo = ldo, a.out = static_cast<uint16_t*>(out), a.lse = lse;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales, a.v_codes = c.v_codes, a.v_scales = c.v_scales;
    a.cu_q = b.cu_q, a.kv_len = b.kv_len, a.page_table = b.page_table, a.batch = b.batch, a.table_width = b.table_width;
    a.total_q = b.total_q, a.max_q = b.max_q, a.max_kv = b.max_kv, a.num_pages = c.num_pages;
    a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.q_heads = q_heads, a.kv_heads = c.kv_heads, a.group = q_heads / c.kv_heads;
    a.causal = causal, a.window = window, a.scale = scale;
    const dim3 grid(b.total_q, q_heads), block(64);
    if (c.head_dim == 64) attend_rows<64><<<grid, block, 0, stream>>>(a);
    else attend_rows<128><<<grid, block, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace batq
