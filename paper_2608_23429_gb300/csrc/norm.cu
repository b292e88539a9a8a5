// cb_norm_residual: h = x + gate * branch, x_out = round(h), then the RMS norm of
// h with weight, scale and shift, in bf16, fp32 or e4m3 with one scale a row.
//
// Bound by HBM: a row is read once and written once. It stays in registers
// between its two reductions (sum of squares, largest magnitude): TPR threads hold
// CH chunks of VEC elements each. A warp per row needs no barrier and is used while
// a lane can hold its share; longer rows take 128 to 512 threads.
#include <cuda_bf16.h>

#include <atomic>
#include <cmath>

#include "../../include/chebboost_block.h"
#include "cb_device.h"

namespace cbk {
namespace {

constexpr float kTiny = 1.17549435e-38f;  // 2^-126, the smallest scale: its reciprocal is finite

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
};

// VEC consecutive values as they lie in memory. The loads are predicated, not
// branched around, so that those of all chunks and operands are in flight together.
template <int VEC>
struct Raw {
    uint32_t w[VEC];
};

template <int VEC>
__device__ __forceinline__ Raw<VEC> load(const void* p, long long e, int bf16, bool on) {
    Raw<VEC> r;
    if constexpr (VEC == 8) {
        const char* a = reinterpret_cast<const char*>(p) + (bf16 ? 2 : 4) * e;
        asm("{\n\t.reg .pred p, q;\n\t"
            "setp.ne.s32 p, %9, 0;\n\tsetp.ne.s32 q, %10, 0;\n\t"
            "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
            "mov.b32 %4, 0;\n\tmov.b32 %5, 0;\n\tmov.b32 %6, 0;\n\tmov.b32 %7, 0;\n\t"
            "@p ld.global.v4.u32 {%0,%1,%2,%3}, [%8];\n\t"
            "@q ld.global.v4.u32 {%4,%5,%6,%7}, [%8+16];\n\t}"
            : "=&r"(r.w[0]), "=&r"(r.w[1]), "=&r"(r.w[2]), "=&r"(r.w[3]), "=&r"(r.w[4]), "=&r"(r.w[5]), "=&r"(r.w[6]),
              "=&r"(r.w[7])
            : "l"(a), "r"((int)on), "r"((int)(on && !bf16)));
    } else {
        r.w[0] = 0;
        if (on)
            r.w[0] = bf16 ? (uint32_t) reinterpret_cast<const uint16_t*>(p)[e] : reinterpret_cast<const uint32_t*>(p)[e];
    }
    return r;
}

template <int VEC>
__device__ __forceinline__ void values(const Raw<VEC>& r, int bf16, float* v) {
    if constexpr (VEC == 8) {
        if (bf16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(r.w[i] << 16);
                v[2 * i + 1] = __uint_as_float(r.w[i] & 0xFFFF0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r.w[i]);
        }
    } else {
        v[0] = __uint_as_float(bf16 ? r.w[0] << 16 : r.w[0]);
    }
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack_e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

template <int VEC>
__device__ __forceinline__ void store(void* p, long long e, int dtype, const float* v) {
    if constexpr (VEC == 8) {
        if (dtype == CB_BF16) {
            *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + e) =
                make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        } else if (dtype == CB_FP32) {
            float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + e);
            q[0] = make_float4(v[0], v[1], v[2], v[3]);
            q[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
            *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(p) + e) =
                make_uint2(pack_e4m3x2(v[0], v[1]) | pack_e4m3x2(v[2], v[3]) << 16,
                           pack_e4m3x2(v[4], v[5]) | pack_e4m3x2(v[6], v[7]) << 16);
        }
    } else {
        if (dtype == CB_BF16)
            reinterpret_cast<__nv_bfloat16*>(p)[e] = __float2bfloat16_rn(v[0]);
        else if (dtype == CB_FP32)
            reinterpret_cast<float*>(p)[e] = v[0];
        else
            reinterpret_cast<uint8_t*>(p)[e] = (uint8_t)pack_e4m3x2(v[0], 0.0f);
    }
}

// Sum or largest value over the TPR threads of a row; `slots` has one word per warp.
template <int TPR, bool MAX>
__device__ __forceinline__ uint32_t reduce(uint32_t v, uint32_t* slots) {
    auto join = [](uint32_t a, uint32_t b) {
        return MAX ? max(a, b) : __float_as_uint(__uint_as_float(a) + __uint_as_float(b));
    };
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v = join(v, __shfl_xor_sync(0xFFFFFFFFu, v, d));
    if constexpr (TPR > 32) {
        if (threadIdx.x % 32 == 0) slots[threadIdx.x / 32] = v;
        __syncthreads();
        v = slots[0];
#pragma unroll
        for (int i = 1; i < TPR / 32; ++i) v = join(v, slots[i]);
    }
    return v;
}

// The row's scale from its largest magnitude as bits (NaN above infinity above all others).
__device__ __forceinline__ float scale_of(uint32_t amax) {
    const float s = __uint_as_float(amax) * (1.0f / 448.0f);
    return amax >= 0x7F800000u ? s : fmaxf(s, kTiny);
}

__host__ __device__ constexpr int row_ctas(int tpr) { return tpr == 32 ? 4 : 1; }  // rows of one CTA

template <int TPR, int CH, int VEC>
__global__ void __launch_bounds__(TPR* row_ctas(TPR)) norm_kernel(const __grid_constant__ NormArgs A) {
    __shared__ uint32_t slots[2][TPR / 32];
    after_previous();
    const unsigned row = blockIdx.x * row_ctas(TPR) + (TPR == 32 ? threadIdx.x / 32 : 0);
    if (row >= A.rows) return;
    const int t = threadIdx.x % TPR;
    const long long line = (long long)(row / A.tokens) * A.line_stride;
    const long long xo = row * A.x_stride, ro = row * A.branch_stride;
    float h[CH][VEC];
    {
        Raw<VEC> xr[CH], br[CH], gr[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * VEC;
            const bool on = e < A.hidden;
            xr[c] = load<VEC>(A.x, xo + e, A.x_bf16, on);
            br[c] = load<VEC>(A.branch, ro + e, A.branch_bf16, on && A.branch);
            gr[c] = load<VEC>(A.gate, line + e, A.param_bf16, on && A.gate);
        }
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            values(xr[c], A.x_bf16, h[c]);
            if (A.branch) {
                float b[VEC], g[VEC];
                values(br[c], A.branch_bf16, b);
                values(gr[c], A.param_bf16, g);
#pragma unroll
                for (int i = 0; i < VEC; ++i) h[c][i] = A.gate ? fmaf(g[i], b[i], h[c][i]) : h[c][i] + b[i];
            }
        }
    }
    if (A.x_out) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int e = (c * TPR + t) * VEC;
            if (e < A.hidden) store<VEC>(A.x_out, row * A.x_out_stride + e, A.x_bf16 ? CB_BF16 : CB_FP32, h[c]);
        }
    }
    float sum = 0.0f;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < VEC; ++i) sum = fmaf(h[c][i], h[c][i], sum);
    sum = __uint_as_float(reduce<TPR, false>(__float_as_uint(sum), slots[0]));
    const float rstd = 1.0f / sqrtf(fmaf(sum, A.inv_hidden, A.eps));
    uint32_t amax = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + t) * VEC;
        const bool on = e < A.hidden;
        const Raw<VEC> wr = load<VEC>(A.weight, e, A.param_bf16, on && A.weight);
        const Raw<VEC> sr = load<VEC>(A.scale, line + e, A.param_bf16, on && A.scale);
        const Raw<VEC> tr = load<VEC>(A.shift, line + e, A.param_bf16, on && A.shift);
        float w[VEC], s[VEC], d[VEC];
        values(wr, A.param_bf16, w);
        values(sr, A.param_bf16, s);
        values(tr, A.param_bf16, d);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            float n = h[c][i] * rstd;
            if (A.weight) n *= w[i];
            n = fmaf(n, s[i], n) + d[i];  // scale and shift are zeros where they are not given
            h[c][i] = n;
            amax = max(amax, on ? __float_as_uint(n) & 0x7FFFFFFFu : 0u);
        }
    }
    float inv = 1.0f;
    if (A.out_dtype == CB_E4M3) {
        amax = reduce<TPR, true>(amax, slots[1]);
        const float s = scale_of(amax);
        if (t == 0) A.out_scale[row] = s;
        inv = __frcp_rn(s);
    }
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        const int e = (c * TPR + t) * VEC;
        if (e >= A.hidden) continue;
        if (A.out_dtype == CB_E4M3)
#pragma unroll
            for (int i = 0; i < VEC; ++i) h[c][i] *= inv;
        store<VEC>(A.out, row * A.out_stride + e, A.out_dtype, h[c]);
    }
}

// Rows too long for registers: three passes over the row, one CTA each.
__global__ void __launch_bounds__(512) norm_long_kernel(const __grid_constant__ NormArgs A) {
    __shared__ uint32_t slots[2][16];
    after_previous();
    const unsigned row = blockIdx.x;
    const long long line = (long long)(row / A.tokens) * A.line_stride;
    auto hidden = [&](int e) {
        float v[1], b[1], g[1];
        values(load<1>(A.x, row * A.x_stride + e, A.x_bf16, true), A.x_bf16, v);
        if (!A.branch) return v[0];
        values(load<1>(A.branch, row * A.branch_stride + e, A.branch_bf16, true), A.branch_bf16, b);
        if (!A.gate) return v[0] + b[0];
        values(load<1>(A.gate, line + e, A.param_bf16, true), A.param_bf16, g);
        return fmaf(g[0], b[0], v[0]);
    };
    float sum = 0.0f;
    for (int e = threadIdx.x; e < A.hidden; e += 512) {
        const float h = hidden(e);
        sum = fmaf(h, h, sum);
    }
    sum = __uint_as_float(reduce<512, false>(__float_as_uint(sum), slots[0]));
    const float rstd = 1.0f / sqrtf(fmaf(sum, A.inv_hidden, A.eps));
    auto normed = [&](float h, int e) {
        float w[1], s[1], d[1];
        values(load<1>(A.weight, e, A.param_bf16, A.weight), A.param_bf16, w);
        values(load<1>(A.scale, line + e, A.param_bf16, A.scale), A.param_bf16, s);
        values(load<1>(A.shift, line + e, A.param_bf16, A.shift), A.param_bf16, d);
        float n = h * rstd;
        if (A.weight) n *= w[0];
        return fmaf(n, s[0], n) + d[0];
    };
    float inv = 1.0f;
    if (A.out_dtype == CB_E4M3) {
        uint32_t amax = 0;
        for (int e = threadIdx.x; e < A.hidden; e += 512)
            amax = max(amax, __float_as_uint(normed(hidden(e), e)) & 0x7FFFFFFFu);
        amax = reduce<512, true>(amax, slots[1]);
        const float s = scale_of(amax);
        if (threadIdx.x == 0) A.out_scale[row] = s;
        inv = __frcp_rn(s);
    }
    for (int e = threadIdx.x; e < A.hidden; e += 512) {
        const float h = hidden(e);
        float y = normed(h, e);
        if (A.out_dtype == CB_E4M3) y *= inv;
        if (A.x_out) store<1>(A.x_out, row * A.x_out_stride + e, A.x_bf16 ? CB_BF16 : CB_FP32, &h);
        store<1>(A.out, row * A.out_stride + e, A.out_dtype, &y);
    }
}

template <int TPR, int CH, int VEC>
cudaError_t launch(const NormArgs& a, cudaStream_t s) {
    constexpr unsigned per = row_ctas(TPR);
    return launch_overlapped(norm_kernel<TPR, CH, VEC>, (int)((a.rows + per - 1) / per), TPR * (int)per, 0, s, a);
}

cudaError_t launch_vectors(const NormArgs& a, cudaStream_t s) {
    const int n = a.hidden / 8;
    if (n <= 32) return launch<32, 1, 8>(a, s);
    if (n <= 64) return launch<32, 2, 8>(a, s);
    if (n <= 96) return launch<32, 3, 8>(a, s);
    if (n <= 128) return launch<32, 4, 8>(a, s);
    if (n <= 160) return launch<32, 5, 8>(a, s);
    if (n <= 256) return launch<128, 2, 8>(a, s);
    if (n <= 384) return launch<128, 3, 8>(a, s);
    if (n <= 512) return launch<128, 4, 8>(a, s);
    if (n <= 1024) return launch<256, 4, 8>(a, s);
    if (n <= 2048) return launch<512, 4, 8>(a, s);
    return launch_overlapped(norm_long_kernel, (int)a.rows, 512, 0, s, a);
}

cudaError_t launch_elements(const NormArgs& a, cudaStream_t s) {
    const int n = a.hidden;
    if (n <= 256) return launch<32, 8, 1>(a, s);
    if (n <= 1024) return launch<128, 8, 1>(a, s);
    if (n <= 4096) return launch<256, 16, 1>(a, s);
    if (n <= 16384) return launch<512, 32, 1>(a, s);
    return launch_overlapped(norm_long_kernel, (int)a.rows, 512, 0, s, a);
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
    const cudaError_t e = vec ? launch_vectors(a, (cudaStream_t)stream) : launch_elements(a, (cudaStream_t)stream);
    return e == cudaSuccess ? CB_OK : cuda_error(e, "norm launch");
}
