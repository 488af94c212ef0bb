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
    int tiles_wg;                                           // append_many: 32-token tiles of a workgroup
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

// What a wave works on: a block of a head.
enum Kind { kQuery, kKey, kValue };

// The transform of 16 channels a lane (operand order of the 32x32x16 matrix instruction, see below), in place.
// y = h + m + l in bf16 terms, T = t0 + t1 + t2 likewise: the six products that matter at 24 bits are summed in fp32,
// smallest first (bf16 input that was not rotated, `exact`, has m = l = 0: the quantiser's own three products).
__device__ __forceinline__ void transform16(float (&y)[16], const bf16x8 (&t)[6], bool exact) {
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

// Clips and quantises the lane's half of a block; returns the codes, and the scale byte in *scale.  `clip` is 1 for no clipping,
// or with `minmax` the ratio of the block's minimum beside clip_max of its maximum.
__device__ __forceinline__ uint4 quantise16(float (&y)[16], bool minmax, float clip, float clip_max, uint32_t* scale) {
    const int lane = threadIdx.x & 63;
    auto other_half = [&](float x) -> float {
        return __builtin_bit_cast(float, __builtin_amdgcn_ds_bpermute((lane ^ 32) << 2, __builtin_bit_cast(int, x)));
    };
    float bound;
    if (minmax) {
        float mn = y[0], mx = y[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) {
            mn = __builtin_fminf(mn, y[r]);
            mx = __builtin_fmaxf(mx, y[r]);
        }
        mn = __builtin_fminf(mn, other_half(mn));
        mx = __builtin_fmaxf(mx, other_half(mx));
        const float lo = clip * mn, hi = clip_max * mx;
#pragma unroll
        for (int r = 0; r < 16; ++r) y[r] = clamp_lo_hi(y[r], lo, hi);
        bound = __builtin_fmaxf(__builtin_fabsf(clamp_lo_hi(mn, lo, hi)), __builtin_fabsf(clamp_lo_hi(mx, lo, hi)));
    } else {
        float x = __builtin_fabsf(y[0]);
#pragma unroll
        for (int r = 1; r < 16; ++r) x = __builtin_fmaxf(x, __builtin_fabsf(y[r]));
        bound = __builtin_fmaxf(x, other_half(x)) * clip;
    }
    const uint32_t sb = e8m0_of_bound_fp8(bound);
    const float sc = scale_operand(sb);
    const uint2 o0 = encode8_fp8(y, bound, sb, sc), o1 = encode8_fp8(y + 8, bound, sb, sc);
    *scale = sb;
    return uint4{o0.x, o0.y, o1.x, o1.y};
}

// Head number `head` of a token's queries, keys and values, in that order.
__device__ __forceinline__ Kind kind_of(const AppendArgs& a, int* head) {
    if (*head < a.q_heads) return kQuery;
    *head -= a.q_heads;
    if (*head < a.kv_heads) return kKey;
    *head -= a.kv_heads;
    return kValue;
}

// Few tokens (decoding): a chain of latencies (one token of 32 + 2 x 8 heads, rotated and transformed, 4.4 us; 64 tokens
// 5.0).  One wave per (32 tokens, MX block of a head).  Lane l holds channels
// 16 (l / 32) .. + 15 of the block for token l % 32, before the transform and after it (the handle's split operands are
// stored so that the matrix instruction's results come in the order of its operands).
template <typename XT, int D>
__global__ void __launch_bounds__(256)
append_few(const AppendArgs a) {
    constexpr int kBlocks = D / 32;
    const int lane = threadIdx.x & 63, l32 = lane & 31, kg = lane >> 5;
    const int per_tile = (a.q_heads + 2 * a.kv_heads) * kBlocks;
    const int tiles = (a.M + 31) >> 5;
    const int64_t unit = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (unit >= (int64_t)tiles * per_tile) return;          // wave-uniform
    const int tile = (int)(unit / per_tile), hb = (int)(unit - (int64_t)tile * per_tile), b = hb % kBlocks;
    int head = hb / kBlocks;
    const Kind kind = kind_of(a, &head);
    const int m = tile * 32 + l32, mm = min(m, a.M - 1);    // rows past the end repeat the last one: computed, not stored
    bool live = m < a.M;
    const float* row = nullptr;
    if (a.table) {
        const int p = a.positions[mm];
        const bool inside = p >= 0 && p < a.table_rows;
        live = live && inside;
        if (kind != kValue) row = a.table + (size_t)(inside ? p : 0) * a.rotary_dim;
    }
    const int64_t slot = a.slots[mm];
    const XT* src = kind == kQuery ? static_cast<const XT*>(a.q) + (size_t)mm * a.ldq
                  : kind == kKey   ? static_cast<const XT*>(a.k) + (size_t)mm * a.ldk
                                   : static_cast<const XT*>(a.v) + (size_t)mm * a.ldv;
    const int blk = (kind == kQuery ? head / a.group : head) * kBlocks + b;     // block of the transform
    const uint4* op = kind == kQuery ? a.tq : kind == kKey ? a.tk : a.tv;
    const float* clips = kind == kKey ? a.clip_k : a.clip_v;
    const float* clips_max = kind == kKey ? a.clip_k_max : a.clip_v_max;
    float clip = 1.0f, clip_max = 1.0f;
    if (kind != kQuery && clips) clip = clips[blk];
    if (kind != kQuery && clips_max) clip_max = clips_max[blk];
    bf16x8 t[6];
    if (op)
#pragma unroll
        for (int i = 0; i < 6; ++i) t[i] = __builtin_bit_cast(bf16x8, op[(size_t)blk * 384 + i * 64 + lane]);
    float y[16];
    load_rotated8<XT>(src + (size_t)head * D, b * 32 + 16 * kg, a, row, *reinterpret_cast<float(*)[8]>(y));
    load_rotated8<XT>(src + (size_t)head * D, b * 32 + 16 * kg + 8, a, row, *reinterpret_cast<float(*)[8]>(y + 8));
    if (op) transform16(y, t, sizeof(XT) == 2 && !row);

    if (kind == kQuery) {
        if (!live) return;
        uint16_t* o = a.q_out + (size_t)m * a.ldq_out + (size_t)head * D + b * 32 + 16 * kg;
        *reinterpret_cast<bf16x8*>(o) = to_bf16(y);
        *reinterpret_cast<bf16x8*>(o + 8) = to_bf16(y + 8);
        return;
    }
    uint32_t sb;
    const uint4 codes = quantise16(y, clips_max, clip, clip_max, &sb);
    if (!live || slot < 0 || slot >= a.num_slots) return;
    const int64_t off = slot & ((1 << a.page_shift) - 1), ph = (slot >> a.page_shift) * a.kv_heads + head;
    *reinterpret_cast<uint4*>((kind == kKey ? a.k_codes : a.v_codes) + (((ph << a.page_shift) + off) * D + b * 32 + 16 * kg)) = codes;
    if (kg == 0) (kind == kKey ? a.k_scales : a.v_scales)[((ph * kBlocks + b) << a.page_shift) + off] = (uint8_t)sb;
}

// Orders a wave's own LDS accesses across its lanes (they are carried out in order; this keeps the compiler to it).
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename XT, int D>
constexpr int many_lds() { return 4 * 2 * 32 * D * (int)sizeof(XT) + 32 * 512; }    // two tiles a wave, a tile's rows of the table

// Many tokens (prompts): bound by the streams in and out, and close behind them the vector instructions.  One wave per
// head and range of 32-token tiles: the head's split operands stay in registers.  Rows go to LDS by LDS-direct loads, a
// tile ahead, with neighbouring lanes in the same row, and results leave from the places that their inputs have been read
// from.  A 16-byte chunk's place in its row is XORed with the row's number, so that a lane's address for chunk c is
// (its row's address) ^ 16 c.  The four waves of a workgroup share the tile's cosines and sines.  For rotations whose
// pairs a lane holds (interleaved, or whole blocks apart); arithmetic as in append_few, same bits.  Measured: 8192 tokens of
// 32 + 2 x 8 heads of 128 channels in bf16, all transformed: 53 us (184 MB in and out, 3.5 TB/s); a wait at the top of each
// tile, behind the last one's stores, 69 us; equal ranges of tiles over all workgroups instead of whole ones, the same 53.
template <typename XT, int D>
__global__ void __launch_bounds__(256, sizeof(XT) == 4 && D == 128 ? 1 : 2)
append_many(const AppendArgs a) {
    constexpr int kBlocks = D / 32, kSize = (int)sizeof(XT), kCh = D * kSize / 16, kRows = 64 / kCh, kLoads = 32 / kRows, kTile = 32 * kCh * 16;
    constexpr int kQCh = D / 8, kCCh = D / 16;              // 16-byte chunks of a row of queries out, of codes
    extern __shared__ __align__(16) uint8_t s_raw[];
    typedef __attribute__((address_space(3))) uint8_t lds_byte;
    int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint8_t* const s_x = s_raw + wave * 2 * kTile;
    uint8_t* const s_t = s_raw + 4 * 2 * kTile;             // [32][128] floats
    const uint32_t x_lds = (uint32_t)(uintptr_t)(lds_byte*)s_raw + wave * 2 * kTile;
    const int heads = a.q_heads + 2 * a.kv_heads, head_groups = (heads + 3) / 4;
    int head = blockIdx.x % head_groups * 4 + wave;
    const bool busy = head < heads;                         // (the others keep the workgroup's barriers)
    if (!busy) head = 0;
    const Kind kind = kind_of(a, &head);
    const int tiles = (a.M + 31) >> 5, tile0 = (int)(blockIdx.x / head_groups) * a.tiles_wg, tile1 = min(tiles, tile0 + a.tiles_wg);
    const uint4* op = kind == kQuery ? a.tq : kind == kKey ? a.tk : a.tv;
    const int blk0 = (kind == kQuery ? head / a.group : head) * kBlocks;
    const float* clips = kind == kKey ? a.clip_k : a.clip_v;
    const float* clips_max = kind == kKey ? a.clip_k_max : a.clip_v_max;
    float clip[kBlocks], clip_max[kBlocks];                 // scalars
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
        auto scalar = [&](const float* p) { return p && kind != kQuery ? __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(p[blk0 + b]))) : 1.0f; };
        clip[b] = scalar(clips), clip_max[b] = scalar(clips_max);
    }
    const XT* src = (kind == kQuery ? static_cast<const XT*>(a.q) : kind == kKey ? static_cast<const XT*>(a.k) : static_cast<const XT*>(a.v)) + (size_t)head * D;
    const int64_t ld = kind == kQuery ? a.ldq : kind == kKey ? a.ldk : a.ldv;
    const bool rotated = a.table && kind != kValue;
    const int rot = rotated ? a.rotary_dim : 0, half = rot >> 1;
    bf16x8 t[kBlocks][6];
    if (op)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 6; ++i) t[b][i] = __builtin_bit_cast(bf16x8, op[(size_t)(blk0 + b) * 384 + i * 64 + lane]);
    // byte address of row r's chunk 0 (XOR 16 c: chunk c) among rows of `ch` chunks
    auto at = [](int r, int ch) { return r * ch * 16 + (ch == 8 ? (r >> 1) & 7 : r & 15) * 16; };
    auto request = [&](int tile, int buf) {                 // (rows past the end repeat the last one)
        const uint8_t* from = reinterpret_cast<const uint8_t*>(src + (size_t)tile * 32 * ld);
        const int rows_left = a.M - 1 - tile * 32;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int r = i * kRows + lane / kCh;           // this lane's 16 bytes of LDS hold chunk (place) ^ (the row's XOR)
            const int c = (lane % kCh) ^ (at(r, kCh) / 16 % kCh);
            const uint32_t voff = (uint32_t)min(r, rows_left) * (uint32_t)(ld * kSize) + (uint32_t)c * 16;
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
                         :: "v"(voff), "s"(from), "s"(x_lds + (uint32_t)(buf * kTile + i * 1024)) : "memory");
        }
    };
    // the tile's rows of the table: thread i moves chunks i % 8, i % 8 + 8, ... of row i / 8
    const int t_chunks = a.table ? a.rotary_dim / 4 : 0, t_row = threadIdx.x >> 3, t_c = threadIdx.x & 7;
    u32x4 tw[4] = {};
    int pos = 0;
    auto positions = [&](int tile) { pos = a.positions[min(tile * 32 + t_row, a.M - 1)]; };
    auto request_table = [&]() {
        const u32x4* p = reinterpret_cast<const u32x4*>(a.table + (size_t)(pos >= 0 && pos < a.table_rows ? pos : 0) * a.rotary_dim) + t_c;
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (t_c + 8 * x < t_chunks) tw[x] = p[8 * x];
    };
    // (not __syncthreads, which would also wait for the loads and stores on their way)
    auto barrier = [&]() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); };
    // a tile's slots and positions are asked for a tile ahead (the table's positions two).  Loads and stores are counted
    // together, in order: the loop waits once, when a tile's results are ready and before they are stored, so that the next
    // tile's loads have had the arithmetic of this one to arrive and the stores have that of the next one to leave
    auto landed = [&]() {
        __builtin_amdgcn_s_waitcnt(0x0F70);                 // vmcnt(0)
        asm volatile("" ::: "memory");
    };
    auto slot_of = [&](int tile) { return kind == kQuery ? (int64_t)0 : a.slots[min(tile * 32 + (lane & 31), a.M - 1)]; };
    auto position_of = [&](int tile) { return a.table ? a.positions[min(tile * 32 + (lane & 31), a.M - 1)] : 0; };
    if (a.table) {
        positions(tile0);
        request_table();
        positions(min(tile0 + 1, tiles - 1));
    }
    int64_t next_slot = slot_of(tile0);                     // (every workgroup has a tile)
    int next_pos = position_of(tile0);
    if (busy) request(tile0, 0);
    landed();
    for (int tile = tile0, buf = 0; tile < tile1; ++tile, buf ^= 1) {
        // opaque here: otherwise every LDS address of a tile is kept in a register of its own across the tiles
        asm volatile("" : "+v"(lane));
        lane &= 63;                                         // (its range is not known behind that)
        const int l32 = lane & 31, kg = lane >> 5, m = tile * 32 + l32;
        const int64_t slot = next_slot;
        const bool there = m < a.M && (!a.table || (next_pos >= 0 && next_pos < a.table_rows));
        const bool live = there && slot >= 0 && slot < a.num_slots;
        if (a.table) {
            barrier();                                      // the last tile's angles have been used
#pragma unroll
            for (int x = 0; x < 4; ++x)
                if (t_c + 8 * x < t_chunks) *reinterpret_cast<u32x4*>(s_t + (at(t_row, 32) ^ ((t_c + 8 * x) * 16))) = tw[x];
            if (tile + 1 < tile1) {
                request_table();
                positions(min(tile + 2, tiles - 1));
            }
            barrier();
        }
        if (tile + 1 < tile1) {
            next_slot = slot_of(tile + 1), next_pos = position_of(tile + 1);
            if (busy) request(tile + 1, buf ^ 1);
        }
        if (!busy) continue;
        const int64_t off = slot & ((1 << a.page_shift) - 1), ph = (slot >> a.page_shift) * a.kv_heads + head;
        uint8_t* const x_at = s_x + buf * kTile;
        const int own = at(l32, kCh) ^ (kg * 16 * kSize), t_at = at(l32, 32);    // channels 16 kg ..: XOR 32 b kSize: of block b
        auto block16 = [&](int b, float (&x)[16]) {         // channels 16 kg .. + 15 of block b of this lane's token
#pragma unroll
            for (int i = 0; i < kSize; ++i) {
                const u32x4 v = *reinterpret_cast<const u32x4*>(x_at + (own ^ (32 * kSize * b + 16 * i)));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (kSize == 4) x[4 * i + e] = __uint_as_float(v[e]);
                    else x[8 * i + 2 * e] = __uint_as_float(v[e] << 16), x[8 * i + 2 * e + 1] = __uint_as_float(v[e] & 0xFFFF0000u);
                }
            }
        };
        auto angles4 = [&](int j, float (&x)[4]) {          // entries j .. j + 3 of this lane's row of the table
            const u32x4 v = *reinterpret_cast<const u32x4*>(s_t + (t_at ^ (4 * j)));
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
        };
        auto interleaved16 = [&](float (&y)[16], int b) {   // (rotary_dim is a multiple of 16)
            const int c0 = 32 * b + 16 * kg;
            if (c0 >= rot) return;
#pragma unroll
            for (int i = 0; i < 16; i += 8) {
                float c[4], s[4];
                angles4((c0 + i) >> 1, c);
                angles4(half + ((c0 + i) >> 1), s);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float p = y[i + 2 * e], r = y[i + 2 * e + 1];
                    y[i + 2 * e] = rot_first(p, r, c[e], s[e]);
                    y[i + 2 * e + 1] = rot_second(p, r, c[e], s[e]);
                }
            }
        };
        uint32_t scale_bytes = 0;
        auto finish = [&](float (&y)[16], const bf16x8 (&tb)[6], int b) {
            if (op) transform16(y, tb, kSize == 2 && !rotated);
            if (kind == kQuery) {
#pragma unroll
                for (int h = 0; h < 2; ++h) *reinterpret_cast<bf16x8*>(x_at + (own ^ (32 * kSize * b + 16 * h))) = to_bf16(y + 8 * h);
            } else {
                uint32_t sb;
                const uint4 codes = quantise16(y, clips_max, clip[b], clip_max[b], &sb);
                scale_bytes |= sb << (8 * b);
                *reinterpret_cast<uint4*>(x_at + (own ^ (32 * kSize * b))) = codes;
            }
            __builtin_amdgcn_sched_barrier(0);              // block by block: interleaved, they would not fit the registers
        };
        auto pair = [&](const bf16x8 (&t0)[6], const bf16x8 (&t1)[6], int b0, int b1) {     // two blocks
            float y0[16], y1[16];
            block16(b0, y0);
            if (!rotated || a.interleaved) {
                if (rotated) interleaved16(y0, b0);
                finish(y0, t0, b0);
                block16(b1, y1);
                if (rotated) interleaved16(y1, b1);
                finish(y1, t1, b1);
                return;
            }
            block16(b1, y1);
            if (32 * b0 < half)
#pragma unroll
                for (int i = 0; i < 16; i += 4) {
                    float c[4], s[4];
                    angles4(32 * b0 + 16 * kg + i, c);
                    angles4(half + 32 * b0 + 16 * kg + i, s);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float p = y0[i + e], r = y1[i + e];
                        y0[i + e] = rot_first(p, r, c[e], s[e]);
                        y1[i + e] = rot_second(p, r, c[e], s[e]);
                    }
                }
            finish(y0, t0, b0);
            finish(y1, t1, b1);
        };
        if constexpr (kBlocks == 2) {
            pair(t[0], t[1], 0, 1);
        } else if (half == 64) {
            pair(t[0], t[2], 0, 2);
            pair(t[1], t[3], 1, 3);
        } else {
            pair(t[0], t[1], 0, 1);
            pair(t[2], t[3], 2, 3);
        }
        wave_lds_order();
        landed();
        // (used here, or the compiler would wait for them behind the stores)
        asm volatile("" : "+v"(next_slot), "+v"(next_pos), "+v"(tw[0]), "+v"(tw[1]), "+v"(tw[2]), "+v"(tw[3]), "+v"(pos));
        // rows out: lane l moves chunk l % kQCh (kCCh) of row l / kQCh, from where its lane put it; what the row's own lane
        // knows about it is shuffled over
        if (kind == kQuery) {
#pragma unroll
            for (int i = 0; i < kQCh / 2; ++i) {
                const int r = i * (64 / kQCh) + lane / kQCh, c = lane % kQCh;
                const u32x4 v = *reinterpret_cast<const u32x4*>(x_at + (at(r, kCh) ^ ((c >> 1 & 1) * 16 * kSize) ^ ((c >> 2) * 32 * kSize + (c & 1) * 16)));
                if (__shfl((int)there, r)) store16_through(a.q_out + (size_t)(tile * 32 + r) * a.ldq_out + (size_t)head * D + c * 8, v);
            }
        } else {
            if (live && kg == 0)
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) (kind == kKey ? a.k_scales : a.v_scales)[((ph * kBlocks + b) << a.page_shift) + off] = (uint8_t)(scale_bytes >> (8 * b));
            const int64_t to = live ? ((ph << a.page_shift) + off) * D : -1;
#pragma unroll
            for (int i = 0; i < kCCh / 2; ++i) {
                const int r = i * (64 / kCCh) + lane / kCCh, c = lane % kCCh;
                const u32x4 v = *reinterpret_cast<const u32x4*>(x_at + (at(r, kCh) ^ ((c & 1) * 16 * kSize) ^ ((c >> 1) * 32 * kSize)));
                const int64_t from = (int64_t)(((uint64_t)(uint32_t)__shfl((int)(to >> 32), r) << 32) | (uint32_t)__shfl((int)to, r));
                if (from >= 0) *reinterpret_cast<u32x4*>((kind == kKey ? a.k_codes : a.v_codes) + from + c * 16) = v;
            }
        }
        wave_lds_order();
    }
}

template <typename XT, int D>
hipError_t launch_append(AppendArgs& a, hipStream_t stream) {
    const int tiles = (int)(((int64_t)a.M + 31) / 32), heads = a.q_heads + 2 * a.kv_heads;
    const int64_t units = (int64_t)tiles * heads * (D / 32);
    // append_many: pairs of a rotation in one lane, and rows of a tile within 32-bit offsets
    const int64_t ld = a.ldq > a.ldk ? (a.ldq > a.ldv ? a.ldq : a.ldv) : (a.ldk > a.ldv ? a.ldk : a.ldv);
    const bool fits = (!a.table || a.interleaved || a.rotary_dim % 64 == 0) && ld * (int64_t)sizeof(XT) < (int64_t(1) << 26);
    // append_few up to 2048 units of 32 tokens x 32 channels (head_dim 128: 256 tokens of 32 + 2 x 8 heads 6.7 us beside 7.9,
    // 384 tokens 8.6 beside 7.9) or 1024 (head_dim 64: 384 tokens of 28 + 2 x 4 heads 4.9 beside 5.5, 512 tokens 6.3 beside 5.5)
    if (units <= 16 * D || !fits) {
        append_few<XT, D><<<(unsigned)((units + 3) / 4), 256, 0, stream>>>(a);
        return hipGetLastError();
    }
    int dev = 0;
    if (hipError_t e = hipGetDevice(&dev); e != hipSuccess) return e;
    hipError_t e;
    const int cus = device_compute_units(dev, &e);
    if (e != hipSuccess) return e;
    constexpr int lds = many_lds<XT, D>();
    if constexpr (lds > 65536)
        if (e = ensure_dynamic_lds<&append_many<XT, D>>(dev, lds); e != hipSuccess) return e;
    // tiles of a workgroup: two workgroups to a compute unit at a time, in whole rounds
    const int groups = (heads + 3) / 4;
    int64_t n = ((int64_t)tiles * groups + 2 * cus - 1) / (2 * cus);
    while (n < 16 && (tiles + n - 1) / n * groups > 2 * cus) ++n;
    if (n > 16) n = 16;
    a.tiles_wg = (int)n;
    const int64_t grid = (tiles + n - 1) / n * groups;
    append_many<XT, D><<<(unsigned)grid, 256, lds, stream>>>(a);
    return hipGetLastError();
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
    if (xdtype == BATQ_BF16) return c.head_dim == 64 ? launch_append<uint16_t, 64>(a, stream) : launch_append<uint16_t, 128>(a, stream);
    return c.head_dim == 64 ? launch_append<float, 64>(a, stream) : launch_append<float, 128>(a, stream);
}

}  // namespace batq
