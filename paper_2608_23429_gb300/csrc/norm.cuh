// Internal: the RMS norm's arguments and kernels (norm.cu and the instantiations norm_lines_*.cu).
#pragma once

#include <cuda_bf16.h>

#include <algorithm>

#include "../../include/chebboost_block.h"
#include "cb_device.h"

namespace cbk {

struct NormArgs {
    int overlap;
    unsigned rows, tokens;
    int hidden;
    long long x_stride, branch_stride, x_out_stride, out_stride, line_stride;
    const void *x, *branch, *gate, *weight, *scale, *shift;
    void *x_out, *out;
    float* out_scale;
    float eps, inv_hidden;
    int x_bf16, branch_bf16, param_bf16, out_dtype;
    unsigned team_rows;  // consecutive rows of a CTA, or of a warp
};

// Rows reached by vectors of 8, with gate, weight, scale and shift in bf16 or in fp32.
cudaError_t launch_norm_bf16_lines(NormArgs& a, int sms, cudaStream_t s);
cudaError_t launch_norm_fp32_lines(NormArgs& a, int sms, cudaStream_t s);

#ifdef __CUDACC__
namespace {

constexpr float kNormTiny = 1.17549435e-38f;  // 2^-126, the smallest scale: its reciprocal is finite

// Pairs of fp32, for the units that take two together.
using Two = unsigned long long;
__device__ __forceinline__ Two two(float a, float b) {
    Two r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ __forceinline__ float2 both(Two v) {
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ __forceinline__ uint32_t norm_bf16x2(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t norm_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

// Sum over a row's W warps, or largest of magnitudes as bits; `slots` has one word per warp.
template <int W, bool MAX>
__device__ __forceinline__ uint32_t row_reduce(uint32_t v, uint32_t* slots) {
    auto join = [](uint32_t a, uint32_t b) {
        return MAX ? max(a, b) : __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    };
    if constexpr (MAX) {
        v = __reduce_max_sync(0xFFFFFFFFu, v);
    } else {
#pragma unroll
        for (int d = 16; d >= 1; d >>= 1) v = join(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    }
    if constexpr (W > 1) {
        if (threadIdx.x % 32 == 0) slots[threadIdx.x / 32] = v;
        __syncthreads();
        v = slots[0];
#pragma unroll
        for (int i = 1; i < W; ++i) v = join(v, slots[i]);
    }
    return v;
}

__device__ __forceinline__ float value_at(const void* p, long long e, int bf16) {
    return bf16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[e] << 16) : reinterpret_cast<const float*>(p)[e];
}
__device__ __forceinline__ void put(void* p, long long e, int dtype, float v) {
    if (dtype == CB_BF16)
        reinterpret_cast<__nv_bfloat16*>(p)[e] = __float2bfloat16_rn(v);
    else if (dtype == CB_FP32)
        reinterpret_cast<float*>(p)[e] = v;
    else
        reinterpret_cast<uint8_t*>(p)[e] = (uint8_t)norm_e4m3x2(v, 0.0f);
}

// Elements t, t + T, ... of a row from or to p (threads behind its end read its start and write nothing). The type is
// asked for once, so that all loads are in flight together.
template <int CH, int T>
__device__ __forceinline__ void load_all(const void* p, long long e, int bf16, int t, int hidden, float* v) {
    if (bf16) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + e;
        uint16_t w[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) w[c] = q[c * T + t < hidden ? c * T + t : 0];
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = __uint_as_float((uint32_t)w[c] << 16);
    } else {
        const float* q = reinterpret_cast<const float*>(p) + e;
#pragma unroll
        for (int c = 0; c < CH; ++c) v[c] = q[c * T + t < hidden ? c * T + t : 0];
    }
}
template <int CH, int T>
__device__ __forceinline__ void store_all(void* p, long long e, int dtype, int t, int hidden, const float* v) {
    if (dtype == CB_BF16) {
        __nv_bfloat16* q = reinterpret_cast<__nv_bfloat16*>(p) + e + t;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * T + t < hidden) q[c * T] = __float2bfloat16_rn(v[c]);
    } else if (dtype == CB_FP32) {
        float* q = reinterpret_cast<float*>(p) + e + t;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * T + t < hidden) q[c * T] = v[c];
    } else {
        uint8_t* q = reinterpret_cast<uint8_t*>(p) + e + t;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * T + t < hidden) q[c * T] = (uint8_t)norm_e4m3x2(v[c], 0.0f);
    }
}

// The larger magnitude; a NaN wins.
__device__ __forceinline__ float max_abs(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(fabsf(b)));
    return r;
}

// The row's scale from its largest magnitude as bits (NaN above infinity above all others).
__device__ __forceinline__ float norm_scale_of(uint32_t amax) {
    const float s = __uint_as_float(amax) * (1.0f / 448.0f);
    return amax >= 0x7F800000u ? s : fmaxf(s, kNormTiny);
}

}  // namespace
#endif

}  // namespace cbk
