// Internal: arguments and epilogue shared by the kernels of cb_linear_run.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/chebboost_block.h"
#include "cb_device.h"

namespace cbk {

struct LinearArgs {
    CUtensorMap x_map, w_map;  // where the operands come by TMA
    int overlap;
    int M, N;              // rows, output features
    int k_bytes;           // bytes of a row of x and of w
    int tiles_m, tiles_n, k_blocks, stages;
    int tile_n;            // output columns of a tile
    int act;
    unsigned tokens;       // rows of one sample
    int out_dtype, resid_bf16, bias_bf16, gate_bf16;
    int wide;              // four columns of every operand of the epilogue are one aligned vector
    long long out_stride, resid_stride, resid_out_stride, gate_stride;  // elements
    long long x_row, w_row;                                              // bytes from row to row
    const void *x, *w;
    const float *x_scale, *w_scale;
    const void *bias, *resid, *gate;
    void *out, *resid_out;
    int* status;
};

// The tensor-core kernels (linear_tc.cu): cg CTAs per tile of 128 cg rows; `words`: operands off the 16-byte grid
// (cg = 1 only). prepare_linear raises the kernels' shared-memory limit and tells how many pairs of CTAs run at once.
size_t linear_stage_bytes(int cg, int tile_n);
int linear_max_stages(size_t smem, size_t stage_bytes);
cudaError_t prepare_linear(size_t smem, int* pairs);
cudaError_t launch_linear(const LinearArgs& a, int cg, bool fp8, bool words, int grid, cudaStream_t s);

#ifdef __CUDACC__
namespace {

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

__device__ __forceinline__ float lin_value(const void* p, long long e, int bf16) {
    return bf16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[e] << 16)
                : reinterpret_cast<const float*>(p)[e];
}

// Four consecutive columns from element e, `n` of them within the row (vectors where `wide`, with n = 4).
__device__ __forceinline__ float4 lin_load4(const void* p, long long e, int bf16, int wide, int n) {
    if (wide) {
        if (n <= 0) return make_float4(0.f, 0.f, 0.f, 0.f);
        if (!bf16) return *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + e);
        const uint2 r = *reinterpret_cast<const uint2*>(reinterpret_cast<const uint16_t*>(p) + e);
        return make_float4(__uint_as_float(r.x << 16), __uint_as_float(r.x & 0xFFFF0000u), __uint_as_float(r.y << 16),
                           __uint_as_float(r.y & 0xFFFF0000u));
    }
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? lin_value(p, e + i, bf16) : 0.0f;
    return make_float4(v[0], v[1], v[2], v[3]);
}

__device__ __forceinline__ void lin_store4(void* p, long long e, int bf16, int wide, int n, float4 v) {
    if (wide) {
        if (n <= 0) return;
        if (bf16)
            *reinterpret_cast<uint2*>(reinterpret_cast<uint16_t*>(p) + e) = make_uint2(bf16x2(v.x, v.y), bf16x2(v.z, v.w));
        else
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + e) = v;
        return;
    }
    const float a[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= n) continue;
        if (bf16)
            reinterpret_cast<__nv_bfloat16*>(p)[e + i] = __float2bfloat16_rn(a[i]);
        else
            reinterpret_cast<float*>(p)[e + i] = a[i];
    }
}

// v / (1 + exp(-t)): SiLU with t = v, the tanh form of GELU with t = 2 sqrt(2/pi) (v + 0.044715 v^3), since
// (1 + tanh(t/2)) / 2 = 1 / (1 + exp(-t)).
__device__ __forceinline__ float lin_act(float v, int act) {
    const float t = act == CB_ACT_GELU ? v * fmaf(0.0713548163f, v * v, 1.59576912f) : v;
    return __fdividef(v, 1.0f + __expf(-t));
}

// Eight rows by four columns of a thread: v[i] belongs to row0 + step * i and the
// columns from col. Bias, activation, output and hidden state.
template <int ROWS>
__device__ __forceinline__ void lin_finish(const LinearArgs& A, int row0, int step, int col, float4* v) {
    const int n = A.N - col < 4 ? A.N - col : 4;  // columns of this thread (<= 0: none)
    const float4 none = make_float4(0.f, 0.f, 0.f, 0.f);
    float4 r[ROWS];
    if (A.resid_out)
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = row0 + step * i;
            r[i] = row < A.M ? lin_load4(A.resid, row * A.resid_stride + col, A.resid_bf16, A.wide, n) : none;
        }
    if (A.w_scale) {
        const float4 s = lin_load4(A.w_scale, col, 0, A.wide, n);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) v[i] = make_float4(v[i].x * s.x, v[i].y * s.y, v[i].z * s.z, v[i].w * s.w);
    }
    if (A.bias) {
        const float4 b = lin_load4(A.bias, col, A.bias_bf16, A.wide, n);
#pragma unroll
        for (int i = 0; i < ROWS; ++i) v[i] = make_float4(v[i].x + b.x, v[i].y + b.y, v[i].z + b.z, v[i].w + b.w);
    }
    if (A.act != CB_ACT_NONE)
#pragma unroll
        for (int i = 0; i < ROWS; ++i)
            v[i] = make_float4(lin_act(v[i].x, A.act), lin_act(v[i].y, A.act), lin_act(v[i].z, A.act), lin_act(v[i].w, A.act));
    if (A.out)
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = row0 + step * i;
            if (row < A.M) lin_store4(A.out, row * A.out_stride + col, A.out_dtype == CB_BF16, A.wide, n, v[i]);
        }
    if (A.resid_out)
#pragma unroll
        for (int i = 0; i < ROWS; ++i) {
            const int row = row0 + step * i;
            if (row >= A.M) continue;
            float4 g = make_float4(1.f, 1.f, 1.f, 1.f);
            if (A.gate)
                g = lin_load4(A.gate, (long long)((unsigned)row / A.tokens) * A.gate_stride + col, A.gate_bf16, A.wide, n);
            lin_store4(A.resid_out, row * A.resid_out_stride + col, A.resid_bf16, A.wide, n,
                       make_float4(fmaf(g.x, v[i].x, r[i].x), fmaf(g.y, v[i].y, r[i].y), fmaf(g.z, v[i].z, r[i].z),
                                   fmaf(g.w, v[i].w, r[i].w)));
        }
}

}  // namespace
#endif

}  // namespace cbk
