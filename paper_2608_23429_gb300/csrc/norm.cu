// cb_norm_residual: h = x + gate * branch, x_out = round(h), then the RMS norm of
// h with weight, scale and shift, in bf16, fp32 or e4m3 with one scale a row.
//
// Bound by HBM: a row is read once and written once. It stays in registers between its two reductions (sum of squares,
// largest magnitude), CH chunks in each thread of its W warps: one warp while that holds it, since what a warp does once a
// row (reductions, roots, addresses) counts as much as its elements. A row's own work is a chain of latencies, so the
// CTAs of the vector kernels (norm_rows.cuh) stay and go through consecutive rows: the next row's x and branch are on
// their way to shared memory meanwhile, each thread copying what it will read itself. Rows off the 16-byte grid take
// elements, one CTA a row. GB300, all operands: 16384 x 4096 bf16 90 us (87 % of the copy rate), 32768 x 1152 bf16 to e4m3 49 us, 8192
// x 1152 fp32 to e4m3 25 us; by elements 8192 x 4097 152 us.
#include <cmath>

#include "norm.cuh"

namespace cbk {
namespace {

// Weight, scale and shift are loaded while the sum is, not before: half the registers, twice the CTAs (GB300: 8192 x 4097
// bf16 to e4m3 211 -> 156 us, 16384 x 1153 78 -> 68). Short rows have room all the same.
__host__ __device__ constexpr bool lines_late(int CH, int W) { return CH * W > 32 && CH <= 10; }

// CH elements of a thread, a row of up to 32 W CH elements in registers. HELD = false: three passes over longer rows.
template <int CH, int W, bool HELD>
__global__ void __launch_bounds__(32 * W, lines_late(CH, W) ? 1024 / (32 * W) : 0) norm_elements_kernel(const __grid_constant__ NormArgs args) {
    __shared__ uint32_t slots[2][W];
    constexpr int T = 32 * W;
    const NormArgs A = args;  // in registers, as stores would have them read again
    after_previous();
    const unsigned row = blockIdx.x;
    const int t = threadIdx.x;
    const long long line = (long long)(row / A.tokens) * A.line_stride;
    const long long xo = row * A.x_stride, bo = row * A.branch_stride;
    auto hidden = [&](unsigned e) {
        float v = value_at(A.x, xo + e, A.x_bf16);
        if (A.branch) {
            const float b = value_at(A.branch, bo + e, A.branch_bf16);
            v = A.gate ? fmaf(value_at(A.gate, line + e, A.param_bf16), b, v) : v + b;
        }
        return v;
    };
    auto normed = [&](float v, unsigned e) {
        if (A.weight) v *= value_at(A.weight, e, A.param_bf16);
        if (A.scale) v = fmaf(v, value_at(A.scale, line + e, A.param_bf16), v);
        return A.shift ? v + value_at(A.shift, line + e, A.param_bf16) : v;
    };
    float h[CH], sum = 0.0f;
    float w[CH], sc[CH], sh[CH];
    auto load_lines = [&] {
        if (A.weight) load_all<CH, T>(A.weight, 0, A.param_bf16, t, A.hidden, w);
        if (A.scale) load_all<CH, T>(A.scale, line, A.param_bf16, t, A.hidden, sc);
        if (A.shift) load_all<CH, T>(A.shift, line, A.param_bf16, t, A.hidden, sh);
    };
    if constexpr (HELD) {
        float b[CH], g[CH];
        load_all<CH, T>(A.x, xo, A.x_bf16, t, A.hidden, h);
        if (A.branch) load_all<CH, T>(A.branch, bo, A.branch_bf16, t, A.hidden, b);
        if (A.gate) load_all<CH, T>(A.gate, line, A.param_bf16, t, A.hidden, g);
        if constexpr (!lines_late(CH, W)) load_lines();
        if (A.gate) {
#pragma unroll
            for (int c = 0; c < CH; ++c) h[c] = fmaf(g[c], b[c], h[c]);
        } else if (A.branch) {
#pragma unroll
            for (int c = 0; c < CH; ++c) h[c] += b[c];
        }
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (c * T + t < A.hidden) sum = fmaf(h[c], h[c], sum);
        if constexpr (lines_late(CH, W)) load_lines();
        if (A.x_out) store_all<CH, T>(A.x_out, row * A.x_out_stride, A.x_bf16 ? CB_BF16 : CB_FP32, t, A.hidden, h);
    } else {
        for (unsigned e = t; e < (unsigned)A.hidden; e += T) {  // (an int would pass its end on the way out of the longest rows)
            const float v = hidden(e);
            sum = fmaf(v, v, sum);
        }
    }
    sum = __uint_as_float(row_reduce<W, false>(__float_as_uint(sum), slots[0]));
    const float rstd = 1.0f / sqrtf(fmaf(sum, A.inv_hidden, A.eps));
    float amax = 0.0f, inv = 1.0f;
    if constexpr (HELD) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            float n = h[c] * rstd;
            if (A.weight) n *= w[c];
            if (A.scale) n = fmaf(n, sc[c], n);
            if (A.shift) n += sh[c];
            h[c] = n;
            if (c * T + t < A.hidden) amax = max_abs(amax, n);
        }
    } else if (A.out_dtype == CB_E4M3) {
        for (unsigned e = t; e < (unsigned)A.hidden; e += T) amax = max_abs(amax, normed(hidden(e) * rstd, e));
    }
    if (A.out_dtype == CB_E4M3) {
        const float s = norm_scale_of(row_reduce<W, true>(__float_as_uint(amax) & 0x7FFFFFFFu, slots[1]));
        if (t == 0) A.out_scale[row] = s;
        inv = __frcp_rn(s);
    }
    if constexpr (HELD) {
#pragma unroll
        for (int c = 0; c < CH; ++c) h[c] *= inv;
        store_all<CH, T>(A.out, row * A.out_stride, A.out_dtype, t, A.hidden, h);
    } else {
        for (unsigned e = t; e < (unsigned)A.hidden; e += T) {
            const float v = hidden(e);
            if (A.x_out) put(A.x_out, row * A.x_out_stride + e, A.x_bf16 ? CB_BF16 : CB_FP32, v);
            put(A.out, row * A.out_stride + e, A.out_dtype, normed(v * rstd, e) * inv);
        }
    }
}

template <int CH, int W, bool HELD>
cudaError_t launch_elements(const NormArgs& a, cudaStream_t s) {
    return launch_overlapped(norm_elements_kernel<CH, W, HELD>, (int)a.rows, 32 * W, 0, s, a);
}

cudaError_t launch_row(NormArgs& a, bool vec, int sms, cudaStream_t s) {
    const int n = a.hidden;
    if (vec && n <= 16384) return a.param_bf16 ? launch_norm_bf16_lines(a, sms, s) : launch_norm_fp32_lines(a, sms, s);
    if (n <= 256) return launch_elements<4, 2, true>(a, s);
    if (n <= 384) return launch_elements<6, 2, true>(a, s);
    if (n <= 640) return launch_elements<5, 4, true>(a, s);
    if (n <= 1024) return launch_elements<8, 4, true>(a, s);
    if (n <= 1280) return launch_elements<10, 4, true>(a, s);
    if (n <= 2048) return launch_elements<8, 8, true>(a, s);
    if (n <= 2560) return launch_elements<10, 8, true>(a, s);
    if (n <= 4096) return launch_elements<8, 16, true>(a, s);
    if (n <= 5120) return launch_elements<10, 16, true>(a, s);
    if (n <= 8192) return launch_elements<16, 16, true>(a, s);
    return launch_elements<1, 16, false>(a, s);
}

size_t bytes_of(int dtype) { return dtype == CB_BF16 ? 2 : dtype == CB_FP32 ? 4 : 1; }
bool on_grid(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

}  // namespace
}  // namespace cbk

extern "C" int cb_norm_residual(const cb_norm_desc* d, const void* x, const void* branch, const void* gate,
                                const void* weight, const void* scale, const void* shift, void* x_out, void* out,
                                float* out_scale, void* stream) {
    using namespace cbk;
    auto wide = [](cb_dtype t) { return t == CB_BF16 || t == CB_FP32; };
    if (!d || d->reserved != 0 || d->rows < 0 || d->hidden < 1 || d->tokens < 0) return CB_ERR_ARG;
    if (!wide(d->x_dtype) || !wide(d->branch_dtype) || !wide(d->param_dtype)) return CB_ERR_ARG;
    if (!wide(d->out_dtype) && d->out_dtype != CB_E4M3) return CB_ERR_ARG;
    if (!(d->eps >= 0.0f && std::isfinite(d->eps))) return CB_ERR_ARG;
    if (d->rows > 0x7FFFFFFFLL || d->hidden > 0x7FFFFFFFLL) return CB_ERR_LIMIT;
    const int64_t strides[] = {d->x_stride, d->branch_stride, d->x_out_stride, d->out_stride, d->line_stride};
    for (int64_t s : strides)
        if (s != 0 && (s < d->hidden || s > CB_MAX_NUMEL)) return s < d->hidden ? CB_ERR_ARG : CB_ERR_LIMIT;
    if (d->rows == 0) return CB_OK;
    if (!x || !out || (gate && !branch) || (d->out_dtype == CB_E4M3) != (out_scale != nullptr)) return CB_ERR_ARG;
    NormArgs a{};
    a.overlap = 1;
    a.rows = (unsigned)d->rows;
    a.hidden = (int)d->hidden;
    a.tokens = d->tokens == 0 || d->tokens > d->rows ? a.rows : (unsigned)d->tokens;
    a.x_stride = d->x_stride ? d->x_stride : d->hidden;
    a.branch_stride = d->branch_stride ? d->branch_stride : d->hidden;
    a.x_out_stride = d->x_out_stride ? d->x_out_stride : d->hidden;
    a.out_stride = d->out_stride ? d->out_stride : d->hidden;
    a.line_stride = d->line_stride ? d->line_stride : d->hidden;
    a.x = x, a.branch = branch, a.gate = gate, a.weight = weight, a.scale = scale, a.shift = shift;
    a.x_out = x_out, a.out = out, a.out_scale = out_scale;
    a.eps = d->eps;
    a.inv_hidden = (float)(1.0 / (double)d->hidden);
    a.x_bf16 = d->x_dtype == CB_BF16;
    a.branch_bf16 = d->branch_dtype == CB_BF16;
    a.param_bf16 = d->param_dtype == CB_BF16;
    a.out_dtype = d->out_dtype;
    // a pointer, its element size and the stride behind it (rows start on the grid too)
    const struct {
        const void* p;
        int dtype;
        long long stride;
    } used[] = {{x, d->x_dtype, a.x_stride},           {branch, d->branch_dtype, a.branch_stride},
                {gate, d->param_dtype, a.line_stride}, {weight, d->param_dtype, 0},
                {scale, d->param_dtype, a.line_stride}, {shift, d->param_dtype, a.line_stride},
                {x_out, d->x_dtype, a.x_out_stride},   {out, d->out_dtype, a.out_stride},
                {out_scale, CB_FP32, 0}};
    bool vec = d->hidden % 8 == 0;
    for (const auto& u : used) {
        const size_t es = bytes_of(u.dtype), grid = es == 1 ? 8 : 16;
        if (!u.p) continue;
        if (!on_grid(u.p, es)) return CB_ERR_ALIGN;
        if (u.p != (const void*)out_scale) vec = vec && on_grid(u.p, grid) && (size_t)u.stride * es % grid == 0;
    }
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = launch_row(a, vec, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? CB_OK : cuda_error(e, "norm launch");
}
