// What happens to the queries, keys and values of new tokens between the fused projection and the attention: rotation
// by position, the block transforms (Sec. 3.2: P_k and P_v transform the key and value cache head by head, queries
// take T_k^-T), MXFP8 (Sec. 2) and the scatter into the pages of the cache.  gfx950 only.
#include "batq_internal.h"
#include "mxfp4_device.h"

namespace batq {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct AppendArgs {
    const void *q, *k, *v;
    int64_t ldq, ldk, ldv;                                  // elements
    uint16_t* q_out;
    int64_t ldq_out;
    uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const uint4 *tq, *tk, *tv;                              // split operands (T_k^-T, T_k, T_v) or null
    const float *clip_k, *clip_k_max, *clip_v, *clip_v_max; // null: no clipping; *_max: the two-ratio form
    const float* table;                                     // null: no rotation
    const int32_t* positions;
    const int64_t* slots;
    int64_t num_slots;
    int table_rows, rotary_dim, interleaved;
    int M, q_heads, kv_heads, group, page_shift;
};

__device__ __forceinline__ void load8(const uint16_t* p, float (&x)[8]) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ void load8(const float* p, float (&x)[8]) {
    const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
    x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
}

// a c - b s and b c + a s with every product and sum rounded to fp32 (not contracted): the result is the same in every
// program that follows the definition, so a rotated key's code does not depend on how its kernel was compiled.
__device__ __forceinline__ float rot_first(float a, float b, float c, float s) {
#pragma clang fp contract(off)
    const float ac = a * c, bs = b * s;
    return ac - bs;
}
__device__ __forceinline__ float rot_second(float a, float b, float c, float s) {
#pragma clang fp contract(off)
    const float bc = b * c, as = a * s;
    return bc + as;
}

// Channels c0 .. c0 + 7 of a head whose row starts at `head`, rotated.  A group of 8 lies in one half of the rotated
// channels, whole (rotary_dim is a multiple of 16).
template <typename XT>
__device__ __forceinline__ void load_rotated8(const XT* head, int c0, const AppendArgs& a, const float* row, float (&x)[8]) {
    load8(head + c0, x);
    if (!row || c0 >= a.rotary_dim) return;
    const int half = a.rotary_dim >> 1;
    if (a.interleaved) {
        const float4 c = *reinterpret_cast<const float4*>(row + (c0 >> 1));
        const float4 s = *reinterpret_cast<const float4*>(row + half + (c0 >> 1));
        const float cv[4] = {c.x, c.y, c.z, c.w}, sv[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float p = x[2 * i], r = x[2 * i + 1];
            x[2 * i] = rot_first(p, r, cv[i], sv[i]);
            x[2 * i + 1] = rot_second(p, r, cv[i], sv[i]);
        }
        return;
    }
    const bool first = c0 < half;
    const int j0 = first ? c0 : c0 - half;
    float y[8], c[8], s[8];
    load8(head + (first ? c0 + half : j0), y);
    load8(row + j0, c);
    load8(row + half + j0, s);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = first ? rot_first(x[i], y[i], c[i], s[i]) : rot_second(y[i], x[i], c[i], s[i]);
}

__device__ __forceinline__ bf16x8 to_bf16(const float* x) {
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = (__bf16)x[i];
    return r;
}

// One wave per (32 tokens, MX block of a query, key or value head).  Lane l holds channels 16 (l / 32) .. + 15 of the
// block for token l % 32, before the transform and after it: the operand order of the 32x32x16 matrix instruction
// (the handle's split operands are stored so that its results come in the same order).
template <typename XT, int D>
__global__ void __launch_bounds__(256)
append_kernel(const AppendArgs a) {
    constexpr int kBlocks = D / 32;
    const int lane = threadIdx.x & 63, l32 = lane & 31, kg = lane >> 5;
    const int per_tile = (a.q_heads + 2 * a.kv_heads) * kBlocks;
    const int tiles = (a.M + 31) >> 5;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (int64_t)tiles * per_tile) return;          // wave-uniform
    const int tile = (int)(unit / per_tile);
    int hb = (int)(unit - (int64_t)tile * per_tile);        // head * kBlocks + block, queries first
    int kind = 0;                                           // 0 query, 1 key, 2 value
    if (hb >= a.q_heads * kBlocks) {
        hb -= a.q_heads * kBlocks;
        kind = 1;
        if (hb >= a.kv_heads * kBlocks) hb -= a.kv_heads * kBlocks, kind = 2;
    }
    const int head = hb / kBlocks, b = hb % kBlocks;
    const int m = tile * 32 + l32, mm = min(m, a.M - 1);    // rows past the end repeat the last one: computed, not stored
    bool live = m < a.M;
    const float* row = nullptr;
    if (a.table && kind != 2) {
        const int p = a.positions[mm];
        const bool inside = p >= 0 && p < a.table_rows;
        live = live && inside;
        row = a.table + (size_t)(inside ? p : 0) * a.rotary_dim;
    } else if (a.table) {
        const int p = a.positions[mm];
        live = live && p >= 0 && p < a.table_rows;
    }
    const XT* src = kind == 0 ? static_cast<const XT*>(a.q) + (size_t)mm * a.ldq
                  : kind == 1 ? static_cast<const XT*>(a.k) + (size_t)mm * a.ldk
                              : static_cast<const XT*>(a.v) + (size_t)mm * a.ldv;
    float y[16];
    load_rotated8<XT>(src + (size_t)head * D, b * 32 + 16 * kg, a, row, *reinterpret_cast<float(*)[8]>(y));
    load_rotated8<XT>(src + (size_t)head * D, b * 32 + 16 * kg + 8, a, row, *reinterpret_cast<float(*)[8]>(y + 8));

    const int blk = (kind == 0 ? head / a.group : head) * kBlocks + b;      // block of the transform
    const uint4* op = kind == 0 ? a.tq : kind == 1 ? a.tk : a.tv;
    if (op) {
        // y = h + m + l in bf16 terms, T = t0 + t1 + t2 likewise: the six products that matter at 24 bits are summed in
        // fp32, smallest first (bf16 input that was not rotated has m = l = 0: the quantiser's own three products)
        bf16x8 t[6];
#pragma unroll
        for (int i = 0; i < 6; ++i) t[i] = __builtin_bit_cast(bf16x8, op[(size_t)blk * 384 + i * 64 + lane]);
        const bool exact = sizeof(XT) == 2 && !row;         // wave-uniform
        bf16x8 xs[3][2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float r[8];
            xs[0][h] = to_bf16(y + 8 * h);
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = y[8 * h + i] - (float)xs[0][h][i];
            xs[1][h] = to_bf16(r);
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] -= (float)xs[1][h][i];
            xs[2][h] = to_bf16(r);
        }
        v16f acc = {};
        auto product = [&](int xt, int tt) {
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(t[tt * 2 + h], xs[xt][h], acc, 0, 0, 0);
        };
        if (!exact) {
            product(2, 0);
            product(1, 1);
        }
        product(0, 2);
        if (!exact) product(1, 0);
        product(0, 1);
        product(0, 0);
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = acc[r];
    }

    if (kind == 0) {
        if (!live) return;
        uint16_t* o = a.q_out + (size_t)m * a.ldq_out + (size_t)hb * 32 + 16 * kg;
        *reinterpret_cast<bf16x8*>(o) = to_bf16(y);
        *reinterpret_cast<bf16x8*>(o + 8) = to_bf16(y + 8);
        return;
    }
    const float* clip = kind == 1 ? a.clip_k : a.clip_v;
    const float* clip_max = kind == 1 ? a.clip_k_max : a.clip_v_max;
    auto other_half = [&](float x) -> float {
        return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute((lane ^ 32) << 2, __builtin_bit_cast(int, x)));
    };
    float bound;
    if (clip_max) {
        float mn = y[0], mx = y[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) {
            mn = __builtin_fminf(mn, y[r]);
            mx = __builtin_fmaxf(mx, y[r]);
        }
        mn = __builtin_fminf(mn, other_half(mn));
        mx = __builtin_fmaxf(mx, other_half(mx));
        const float lo = clip[blk] * mn, hi = clip_max[blk] * mx;
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = clamp_lo_hi(y[r], lo, hi);
        bound = __builtin_fmaxf(__builtin_fabsf(clamp_lo_hi(mn, lo, hi)), __builtin_fabsf(clamp_lo_hi(mx, lo, hi)));
    } else {
        float x = __builtin_fabsf(y[0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) x = __builtin_fmaxf(x, __builtin_fabsf(y[r]));
        bound = __builtin_fmaxf(x, other_half(x));
        if (clip) bound *= clip[blk];
    }
    const uint32_t sb = e8m0_of_bound_fp8(bound);
    const float sc = scale_operand(sb);
    const uint2 o0 = encode8_fp8(y, bound, sb, sc), o1 = encode8_fp8(y + 8, bound, sb, sc);
    const int64_t slot = a.slots[mm];
    if (!live || slot < 0 || slot >= a.num_slots) return;
    const int64_t page = slot >> a.page_shift, off = slot & ((1 << a.page_shift) - 1);
    uint8_t* codes = kind == 1 ? a.k_codes : a.v_codes;
    uint8_t* scales = kind == 1 ? a.k_scales : a.v_scales;
    const int64_t ph = page * a.kv_heads + head;
    *reinterpret_cast<uint4*>(codes + (((ph << a.page_shift) + off) * D + b * 32 + 16 * kg)) = uint4{o0.x, o0.y, o1.x, o1.y};
    if (kg == 0) scales[((ph * kBlocks + b) << a.page_shift) + off] = (uint8_t)sb;
}

}  // namespace

hipError_t launch_kv_paged_append(const batq_paged_cache& c, const batq_transform* tk, const batq_transform* tv,
                                  const batq_rope* rope, const void* q, int64_t ldq, int q_heads, void* q_out,
                                  int64_t ldq_out, const void* k, int64_t ldk, const void* v, int64_t ldv,
                                  batq_dtype xdtype, const int32_t* positions, const int64_t* slots, int M,
                                  hipStream_t stream) {
    AppendArgs a = {};
    a.q = q, a.k = k, a.v = v, a.ldq = ldq, a.ldk = ldk, a.ldv = ldv;
    a.q_out = static_cast<uint16_t*>(q_out), a.ldq_out = ldq_out;
    a.k_codes = c.k_codes, a.k_scales = c.k_scales, a.v_codes = c.v_codes, a.v_scales = c.v_scales;
    if (tk && tk->has_transform) {
        a.tk = reinterpret_cast<const uint4*>(tk->d_Tsplit);
        a.tq = reinterpret_cast<const uint4*>(tk->d_TinvTSplit);
    }
    if (tv && tv->has_transform) a.tv = reinterpret_cast<const uint4*>(tv->d_Tsplit);
    if (tk) a.clip_k = tk->d_clip, a.clip_k_max = tk->minmax ? tk->d_clip_max : nullptr;
    if (tv) a.clip_v = tv->d_clip, a.clip_v_max = tv->minmax ? tv->d_clip_max : nullptr;
    if (rope) a.table = rope->table, a.table_rows = rope->positions, a.rotary_dim = rope->rotary_dim, a.interleaved = rope->interleaved;
    a.positions = positions, a.slots = slots, a.M = M;
    a.num_slots = (int64_t)c.num_pages * c.page_size;
    a.q_heads = q_heads, a.kv_heads = c.kv_heads, a.group = q_heads ? q_heads / c.kv_heads : 1;
    a.page_shift = __builtin_ctz((unsigned)c.page_size);
    const int64_t units = (int64_t)((M + 31) / 32) * (q_heads + 2 * c.kv_heads) * (c.head_dim / 32);
    const dim3 grid((unsigned)((units + 3) / 4)), block(256);
    if (xdtype == BATQ_BF16) {
        if (c.head_dim == 64) append_kernel<uint16_t, 64><<<grid, block, 0, stream>>>(a);
        else append_kernel<uint16_t, 128><<<grid, block, 0, stream>>>(a);
    } else {
        if (c.head_dim == 64) append_kernel<float, 64><<<grid, block, 0, stream>>>(a);
        else append_kernel<float, 128><<<grid, block, 0, stream>>>(a);
    }
    return hipGetLastError();
}

}  // namespace batq
