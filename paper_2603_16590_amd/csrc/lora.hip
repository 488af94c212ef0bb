// Low-rank adapters of many requests beside a shared projection: out = base + s (X A^T) B^T with each row's own pair.
// gfx950 only.
#include "batq_internal.h"
#include "mxfp4_device.h"

namespace batq {
namespace {

__device__ __forceinline__ float value(float x) { return x; }
__device__ __forceinline__ float value(uint16_t x) { return bf16_bits_to_float(x); }
__device__ __forceinline__ void put(float* p, float x) { *p = x; }
__device__ __forceinline__ void put(uint16_t* p, float x) { *p = (uint16_t)float_to_bf16_bits(x); }

// h[m][j] = s_a sum_k X[m][k] A_a[j][k]: a workgroup per row, a wave per j.
template <typename XT>
__global__ void __launch_bounds__(256)
shrink_kernel(const XT* X, int64_t ldx, int K, const uint16_t* A, int rank, int adapters, const float* scales, const int32_t* index,
              float* h) {
    const int m = blockIdx.x, lane = threadIdx.x & 63, a = index[m];
    if (a < 0 || a >= adapters) return;
    for (int j = threadIdx.x >> 6; j < rank; j += 4) {
        float sum = 0.0f;
        for (int k = lane; k < K; k += 64)
            sum = __builtin_fmaf(value(X[(size_t)m * ldx + k]), value(A[((size_t)a * rank + j) * K + k]), sum);
        for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
        if (lane == 0) h[(size_t)m * rank + j] = sum * (scales ? scales[a] : 1.0f);
    }
}

template <typename YT>
__global__ void __launch_bounds__(256)
expand_kernel(const float* h, const uint16_t* B, int N, int rank, int adapters, const int32_t* index, const YT* base, int64_t ldb,
              YT* out, int64_t ldo) {
    const int m = blockIdx.y, n = blockIdx.x * 256 + threadIdx.x, a = index[m];
    if (n >= N) return;
    float sum = 0.0f;
    if (a >= 0 && a < adapters)
        for (int j = 0; j < rank; ++j) sum = __builtin_fmaf(h[(size_t)m * rank + j], value(B[((size_t)a * N + n) * rank + j]), sum);
    put(out + (size_t)m * ldo + n, (base ? value(base[(size_t)m * ldb + n]) : 0.0f) + sum);
}

}  // namespace

size_t lora_workspace_bytes(int M, int, int, int rank, int) { return (size_t)M * rank * 4; }

hipError_t launch_lora_add(const void* X, batq_dtype xdtype, int M, int K, int64_t ldx, const void* A, const void* B,
                           int N, int rank, int adapters, const float* scales, const int32_t* index, const void* base,
                           int64_t ldb, void* out, int64_t ldo, batq_dtype ydtype, void* workspace, hipStream_t stream) {
    float* h = static_cast<float*>(workspace);
    auto a = static_cast<const uint16_t*>(A), b = static_cast<const uint16_t*>(B);
    if (xdtype == BATQ_BF16)
        shrink_kernel<<<M, 256, 0, stream>>>(static_cast<const uint16_t*>(X), ldx, K, a, rank, adapters, scales, index, h);
    else
        shrink_kernel<<<M, 256, 0, stream>>>(static_cast<const float*>(X), ldx, K, a, rank, adapters, scales, index, h);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    const dim3 grid((N + 255) / 256, M);
    if (ydtype == BATQ_BF16)
        expand_kernel<<<grid, 256, 0, stream>>>(h, b, N, rank, adapters, index, static_cast<const uint16_t*>(base), ldb, static_cast<uint16_t*>(out), ldo);
    else
        expand_kernel<<<grid, 256, 0, stream>>>(h, b, N, rank, adapters, index, static_cast<const float*>(base), ldb, static_cast<float*>(out), ldo);
    return hipGetLastError();
}

}  // namespace batq
