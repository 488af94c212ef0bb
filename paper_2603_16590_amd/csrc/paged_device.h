// What the kernels on a paged cache share: the lists of a ragged batch, as nothing in them is trusted, and the codes of
// either width as bf16 matrix operands.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/batq.h"
#include "mxfp4_device.h"

namespace batq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float v16f __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct PagedLists {
    const int32_t *cu_q, *kv_len, *page_table;
    int batch, table_width, total_q, max_q, max_kv, num_pages, page_shift, q_heads, kv_heads, group;
    int causal, window;
};

// First token that the window leaves to a query at `pos`, which may be far below zero (more queries than tokens) beside a
// window of any size.
__device__ __forceinline__ int first_seen(const PagedLists& a, int pos) { return a.window && pos >= a.window ? pos - a.window + 1 : 0; }

// Sequence b as the kernels take it: nothing in the lists is trusted.
struct Seq {
    int begin, n, len;                                      // first row, queries served, tokens
    int first_pos;                                          // position of the first query
    int t_lo, t_hi;                                         // tokens that some query may see
};

__device__ __forceinline__ Seq sequence(const PagedLists& a, int b) {
    Seq s;
    s.begin = a.cu_q[b];
    const int end = a.cu_q[b + 1];
    const int n = (s.begin < 0 || end > a.total_q || end < s.begin) ? 0 : end - s.begin;
    s.n = min(n, a.max_q);
    s.len = (int)min((int64_t)max(0, min(a.kv_len[b], a.max_kv)), (int64_t)a.table_width << a.page_shift);
    s.first_pos = s.len - n;
    s.t_hi = a.causal ? max(0, min(s.len, s.first_pos + s.n)) : s.len;
    s.t_lo = min(s.t_hi, first_seen(a, s.first_pos));
    return s;
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// x of the lane and of the lane 16 (32) away, in one order for both, without LDS's latency.
struct Two {
    float a, b;
};
__device__ __forceinline__ Two across16(float x) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return Two{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ Two across32(float x) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return Two{__uint_as_float(r[0]), __uint_as_float(r[1])};
}
__device__ __forceinline__ float larger(const Two& t) { return __builtin_fmaxf(t.a, t.b); }
__device__ __forceinline__ float total(const Two& t) { return t.a + t.b; }

// Two values of a word of four E4M3 codes as bf16.
__device__ __forceinline__ uint32_t cvt_lo(uint32_t w, float sc) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, false));
}
__device__ __forceinline__ uint32_t cvt_hi(uint32_t w, float sc) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, sc, true));
}

// Two neighbouring values of codes of BITS bits as bf16: pair i (a constant once loops are unrolled) of the words at w.
template <int BITS>
__device__ __forceinline__ uint32_t cvt_pair(const uint32_t* w, int i, float sc) {
    if constexpr (BITS == 8) return i % 2 ? cvt_hi(w[i / 2], sc) : cvt_lo(w[i / 2], sc);
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    const bf16x2 v = i % 4 == 0   ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i / 4], sc, 0)
                     : i % 4 == 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i / 4], sc, 1)
                     : i % 4 == 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i / 4], sc, 2)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w[i / 4], sc, 3);
    return __builtin_bit_cast(uint32_t, v);
}
// Eight values: the words at w.
template <int BITS>
__device__ __forceinline__ bf16x8 cvt_eight(const uint32_t* w, float sc) {
    return __builtin_bit_cast(bf16x8, u32x4{cvt_pair<BITS>(w, 0, sc), cvt_pair<BITS>(w, 1, sc), cvt_pair<BITS>(w, 2, sc), cvt_pair<BITS>(w, 3, sc)});
}


// N consecutive words (1, 2 or a multiple of 4) in the widest loads.
template <int N>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* p) {
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const u32x4 v = reinterpret_cast<const u32x4*>(p)[i];
            w[4 * i] = v[0], w[4 * i + 1] = v[1], w[4 * i + 2] = v[2], w[4 * i + 3] = v[3];
        }
    } else if constexpr (N == 2) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(p);
        w[0] = v[0], w[1] = v[1];
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
}
// The codes of four channels.
template <int BITS>
__device__ __forceinline__ uint32_t load_four(const uint8_t* p) {
    if constexpr (BITS == 8) return *reinterpret_cast<const uint32_t*>(p);
    else return *reinterpret_cast<const uint16_t*>(p);
}

inline void set_lists(PagedLists& a, const batq_paged_cache& c, const batq_paged_batch& b, int q_heads, bool causal, int window) {
    a.cu_q = b.cu_q, a.kv_len = b.kv_len, a.page_table = b.page_table, a.batch = b.batch, a.table_width = b.table_width;
    a.total_q = b.total_q, a.max_q = b.max_q, a.max_kv = b.max_kv, a.num_pages = c.num_pages;
    a.page_shift = __builtin_ctz((unsigned)c.page_size);
    a.q_heads = q_heads, a.kv_heads = c.kv_heads, a.group = q_heads / c.kv_heads;
    a.causal = causal, a.window = window;
}

}  // namespace batq
