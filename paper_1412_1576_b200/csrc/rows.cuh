// Shared pieces of the operators on rows of logits or probabilities (toplogits.cu, distill.cu, verify.cu): element types,
// 2^x, keys that order values, reductions over a CTA.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/lda_b200.h"

namespace lda {

constexpr float LOG2E = 1.4426950408889634f;
constexpr double LN2 = 0.69314718055994531;

__device__ __forceinline__ float row_value(float x) { return x; }
__device__ __forceinline__ float row_value(__half x) { return __half2float(x); }
__device__ __forceinline__ float row_value(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T row_element(float x);
template <>
__device__ __forceinline__ float row_element<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half row_element<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 row_element<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

// 2^x by the multifunction unit (at most 2^-22 off, relative; results below 2^-126 are zero).
__device__ __forceinline__ float exp2_unit(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Whole numbers in the order of the values: NaN of either sign above +infinity, both zeros alike.
constexpr uint32_t KEY_NAN = 0xFFFFFFFFu, KEY_NEG_INF = 0x007FFFFFu;
__device__ __forceinline__ uint32_t order_key(float x)
{
    const uint32_t b = __float_as_uint(x + 0.0f);
    return x != x ? KEY_NAN : b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u);
}

__device__ __forceinline__ float warp_reduce_max(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Block-wide maximum; `smem` holds at least 32 floats; result returned to every thread.
__device__ __forceinline__ float block_reduce_max(float v, float* smem)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
    v = warp_reduce_max(v);
    __syncthreads();
    if (lane == 0) smem[warp] = v;
    __syncthreads();
    return warp_reduce_max(lane < nw ? smem[lane] : -INFINITY);
}

// Sizes that every one of the operators refuses.
inline int check_rows(const void* p, int dtype, int64_t rows, int32_t V, int64_t stride)
{
    if (dtype != LDA_F32 && dtype != LDA_F16 && dtype != LDA_BF16) return LDA_EINVAL;
    if (rows < 0 || V <= 0 || stride < 0) return LDA_EINVAL;
    if (rows > 0x7fffffffll || V > LDA_ROW_MAX_V) return LDA_ERANGE;
    // an element's offset in bytes stays inside 63 bits
    if (stride > (1ll << 31)) return LDA_ERANGE;
    if (rows > 0 && (!p || (uintptr_t)p % (dtype == LDA_F32 ? 4 : 2))) return LDA_EINVAL;
    return LDA_OK;
}

// Temperatures at which 1 / tau and log2(e) / tau are ordinary single-precision values.
inline bool temperature_ok(double tau) { return tau >= 1e-6 && tau <= 1e6; }

}  // namespace lda
