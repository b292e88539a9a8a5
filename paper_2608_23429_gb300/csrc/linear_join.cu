// The sums of parts of K of cb_linear_run, added in order and taken through the epilogue: bound by their bytes, which lie in L2.
//
// A thread has four columns of a row. The parts' sums are vectors; the other operands and the results go by elements, as any of
// them may lie off the grid (neighbouring threads share their sectors in L1).
#include "linear.cuh"

namespace cbk {
namespace {

constexpr int kJoinThreads = 256;

template <int ACT>
__device__ __forceinline__ void activate(float* v) {
    const float2 f = both(lin_act<ACT>(two(v[0], v[1]))), g = both(lin_act<ACT>(two(v[2], v[3])));
    v[0] = f.x, v[1] = f.y, v[2] = g.x, v[3] = g.y;
}

__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ LinearJoinArgs A) {
    after_previous();
    const LinearEpilogue E = from_here(A.e);
    const unsigned quads = (unsigned)(E.N + 3) / 4;
    const unsigned long long at = (unsigned long long)blockIdx.x * kJoinThreads + threadIdx.x;
    if (at >= (unsigned long long)quads * E.M) return;
    const int row = (int)(at / quads), col = (int)(at % quads) * 4, n = min(E.N - col, 4);
    float scale[4], bias[4], gate[4], resid[4], v[4] = {};
    const float xs = E.x_scale ? __uint_as_float(lin_ld1(E.x_scale, row, 0)) : 1.0f;
    const long long g = E.gate ? (unsigned)row / E.tokens * E.gate_stride + col : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bool on = i < n;
        scale[i] = on && E.w_scale ? __uint_as_float(lin_ld1(E.w_scale, col + i, 0)) : 1.0f;
        bias[i] = on && E.bias ? __uint_as_float(lin_ld1(E.bias, col + i, E.bias_bf16)) : 0.0f;
        gate[i] = on && E.gate ? __uint_as_float(lin_ld1(E.gate, g + i, E.gate_bf16)) : 1.0f;
        resid[i] = on && E.resid_out ? __uint_as_float(lin_ld1(E.resid, row * E.resid_stride + col + i, E.resid_bf16)) : 0.0f;
    }
    const float* p = A.sums + row * A.stride + col;
#pragma unroll 4
    for (int i = 0; i < A.parts; ++i, p += A.part_size) {
        const float4 s = *reinterpret_cast<const float4*>(p);
        v[0] += s.x, v[1] += s.y, v[2] += s.z, v[3] += s.w;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = i < n ? fmaf(v[i] * xs, scale[i], bias[i]) : 0.0f;
    if (E.act == CB_ACT_GELU) activate<CB_ACT_GELU>(v);
    else if (E.act == CB_ACT_SILU) activate<CB_ACT_SILU>(v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= n) break;
        if (E.out) lin_put1(E.out, row * E.out_stride + col + i, E.out_bf16, v[i]);
        if (E.resid_out) lin_put1(E.resid_out, row * E.resid_out_stride + col + i, E.resid_bf16, fmaf(gate[i], v[i], resid[i]));
    }
}

}  // namespace

cudaError_t launch_linear_join(const LinearJoinArgs& a, cudaStream_t s) {
    const long long n = (long long)((a.e.N + 3) / 4) * a.e.M;
    return launch_overlapped(join_kernel, (int)((n + kJoinThreads - 1) / kJoinThreads), kJoinThreads, 0, s, a);
}

}  // namespace cbk
