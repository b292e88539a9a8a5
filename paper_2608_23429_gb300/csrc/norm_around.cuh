// Internal: arguments of cb_norm_around (norm_around.cu) and its kernel for rows reached by vectors (norm_around_rows.cuh).
#pragma once

#include "mx.cuh"
#include "norm.cuh"

namespace cbk {

struct AroundArgs {
    int overlap;
    unsigned rows, tokens;
    int hidden;
    long long x_stride, branch_stride, x_out_stride, out_stride, line_stride;  // out_stride in 4 bits: bytes
    const void *x, *branch, *gate, *after_weight, *after_bias, *weight, *bias, *scale, *shift;
    void *x_out, *out, *out_scale;
    int after, before;  // CB_NORM_*
    float after_eps, before_eps, x_factor, branch_factor, inv_hidden;
    int x_bf16, branch_bf16, param_bf16, out_dtype;
    unsigned out_tiles;  // of scales, of a row in 4 bits
    unsigned team_rows;  // consecutive rows of a CTA, or of a warp
};

// Rows reached by vectors of 8, with lines in bf16 or in fp32.
cudaError_t launch_around_bf16_lines(AroundArgs& a, int sms, cudaStream_t s);
cudaError_t launch_around_fp32_lines(AroundArgs& a, int sms, cudaStream_t s);

}  // namespace cbk
