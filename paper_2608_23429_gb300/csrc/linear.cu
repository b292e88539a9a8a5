// cb_linear_*: the layer's handle, the checks of a call and the choice of its kernel.
#include <atomic>
#include <new>

#include "linear.cuh"

namespace cbk {
namespace {

__device__ int g_linear_status;  // CB_DEV_* codes of this device's launches

template <bool FP8>
__device__ __forceinline__ float operand(const void* p, long long row_bytes, int row, int k) {
    const char* a = reinterpret_cast<const char*>(p) + row * row_bytes;
    if constexpr (!FP8) return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(a)[k] << 16);
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((uint16_t) reinterpret_cast<const uint8_t*>(a)[k]));
    return __half2float(__ushort_as_half((unsigned short)h));
}

// 64 x 64 outputs of a CTA, 4 x 4 of a thread, operands staged as fp32.
template <bool FP8>
__global__ void __launch_bounds__(256) linear_simple_kernel(const __grid_constant__ LinearArgs A) {
    __shared__ float xs[16][65], ws[16][65];
    after_previous();
    const int K = FP8 ? A.k_bytes : A.k_bytes / 2, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64;
    const int tr = threadIdx.x / 16, tc = threadIdx.x % 16;
    float4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int k0 = 0; k0 < K; k0 += 16) {
        for (int i = threadIdx.x; i < 1024; i += 256) {
            const int r = i / 16, k = i % 16;
            xs[k][r] = m0 + r < A.M && k0 + k < K ? operand<FP8>(A.x, A.x_row, m0 + r, k0 + k) : 0.0f;
            ws[k][r] = n0 + r < A.N && k0 + k < K ? operand<FP8>(A.w, A.w_row, n0 + r, k0 + k) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = xs[k][tr * 4 + i];
                v[i].x = fmaf(a, ws[k][tc * 4], v[i].x);
                v[i].y = fmaf(a, ws[k][tc * 4 + 1], v[i].y);
                v[i].z = fmaf(a, ws[k][tc * 4 + 2], v[i].z);
                v[i].w = fmaf(a, ws[k][tc * 4 + 3], v[i].w);
            }
        __syncthreads();
    }
    if (A.x_scale)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = m0 + tr * 4 + i;
            const float s = row < A.M ? A.x_scale[row] : 0.0f;
            v[i] = make_float4(v[i].x * s, v[i].y * s, v[i].z * s, v[i].w * s);
        }
    lin_finish<4>(A, m0 + tr * 4, 1, n0 + tc * 4, v);
}

bool wide_type(cb_dtype t) { return t == CB_BF16 || t == CB_FP32; }
size_t bytes_of(int t) { return t == CB_BF16 ? 2 : t == CB_FP32 ? 4 : 1; }
bool on_grid(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

}  // namespace
}  // namespace cbk

struct cb_linear {
    cb_linear_desc d;
};

extern "C" {

int cb_linear_create(const cb_linear_desc* d, cb_linear** out) {
    using namespace cbk;
    if (!out) return CB_ERR_ARG;
    *out = nullptr;
    if (!d || d->reserved != 0 || d->in_features < 1 || d->out_features < 1 || !d->w) return CB_ERR_ARG;
    if (d->type != CB_BF16 && d->type != CB_E4M3) return CB_ERR_ARG;
    if (d->bias && !wide_type(d->bias_dtype)) return CB_ERR_ARG;
    if (d->activation < CB_ACT_NONE || d->activation > CB_ACT_SILU) return CB_ERR_ARG;
    if (d->w_scale && d->type != CB_E4M3) return CB_ERR_ARG;
    if (d->w_stride != 0 && d->w_stride < d->in_features) return CB_ERR_ARG;
    const long long row = 0x7FFFFF00LL / (long long)bytes_of(d->type);
    if (d->out_features > 0x7FFFFC00LL || d->in_features > row || d->w_stride > row) return CB_ERR_LIMIT;
    if (!on_grid(d->w, bytes_of(d->type)) || !on_grid(d->w_scale, 4)) return CB_ERR_ALIGN;
    if (d->bias && !on_grid(d->bias, bytes_of(d->bias_dtype))) return CB_ERR_ALIGN;
    cb_linear* l = new (std::nothrow) cb_linear;
    if (!l) return CB_ERR_LIMIT;
    l->d = *d;
    if (l->d.w_stride == 0) l->d.w_stride = d->in_features;
    *out = l;
    return CB_OK;
}

void cb_linear_destroy(cb_linear* l) { delete l; }

int cb_linear_run(const cb_linear* l, const cb_linear_io* io, const void* x, const float* x_scale, const void* resid,
                  const void* gate, void* out, void* resid_out, void* stream) {
    using namespace cbk;
    if (!l || !io || io->reserved != 0 || io->rows < 0 || io->tokens < 0) return CB_ERR_ARG;
    const cb_linear_desc& d = l->d;
    if (!wide_type(io->out_dtype) || !wide_type(io->resid_dtype) || !wide_type(io->gate_dtype)) return CB_ERR_ARG;
    const long long es = (long long)bytes_of(d.type), K = d.in_features, N = d.out_features;
    if (io->rows > 0x7FFFFC00LL) return CB_ERR_LIMIT;
    if (io->x_stride != 0 && io->x_stride < K) return CB_ERR_ARG;
    if (io->x_stride > 0x7FFFFF00LL / es) return CB_ERR_LIMIT;
    const int64_t strides[] = {io->out_stride, io->resid_stride, io->resid_out_stride, io->gate_stride};
    for (int64_t s : strides)
        if (s != 0 && (s < N || s > CB_MAX_NUMEL)) return s < N ? CB_ERR_ARG : CB_ERR_LIMIT;
    if (x_scale && d.type != CB_E4M3) return CB_ERR_ARG;
    if ((resid != nullptr) != (resid_out != nullptr) || (gate && !resid)) return CB_ERR_ARG;
    if (io->rows == 0) return CB_OK;
    if (!x || (!out && !resid_out)) return CB_ERR_ARG;

    LinearArgs a{};
    a.overlap = 1;
    a.M = (int)io->rows, a.N = (int)N;
    a.k_bytes = (int)(K * es);
    a.act = d.activation;
    a.tokens = io->tokens == 0 || io->tokens > io->rows ? (unsigned)io->rows : (unsigned)io->tokens;
    a.out_dtype = io->out_dtype, a.resid_bf16 = io->resid_dtype == CB_BF16;
    a.bias_bf16 = d.bias_dtype == CB_BF16, a.gate_bf16 = io->gate_dtype == CB_BF16;
    a.out_stride = io->out_stride ? io->out_stride : N;
    a.resid_stride = io->resid_stride ? io->resid_stride : N;
    a.resid_out_stride = io->resid_out_stride ? io->resid_out_stride : N;
    a.gate_stride = io->gate_stride ? io->gate_stride : N;
    a.x_row = (io->x_stride ? io->x_stride : K) * es, a.w_row = d.w_stride * es;
    a.x = x, a.w = d.w, a.x_scale = x_scale, a.w_scale = d.w_scale, a.bias = d.bias;
    a.resid = resid, a.gate = gate, a.out = out, a.resid_out = resid_out;
    if (!on_grid(x, es) || !on_grid(x_scale, 4)) return CB_ERR_ALIGN;
    const struct {
        const void* p;
        int dtype;
        long long stride;
    } used[] = {{out, io->out_dtype, a.out_stride},     {resid, io->resid_dtype, a.resid_stride},
                {gate, io->gate_dtype, a.gate_stride},  {resid_out, io->resid_dtype, a.resid_out_stride},
                {d.bias, d.bias_dtype, 0},              {d.w_scale, CB_FP32, 0}};
    a.wide = N % 4 == 0;
    for (const auto& u : used) {
        if (!u.p) continue;
        const size_t s = bytes_of(u.dtype);
        if (!on_grid(u.p, s)) return CB_ERR_ALIGN;
        a.wide = a.wide && on_grid(u.p, 4 * s) && u.stride % 4 == 0;
    }
    const dim3 grid((unsigned)((N + 63) / 64), (unsigned)((a.M + 63) / 64));
    if (d.type == CB_E4M3)
        linear_simple_kernel<true><<<grid, 256, 0, (cudaStream_t)stream>>>(a);
    else
        linear_simple_kernel<false><<<grid, 256, 0, (cudaStream_t)stream>>>(a);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? CB_OK : cuda_error(e, "linear launch");
}

int cb_linear_device_status(int* status, void* stream) {
    if (!status) return CB_ERR_ARG;
    const cudaStream_t s = (cudaStream_t)stream;
    int* word = nullptr;
    int v = 0;
    cudaError_t e = cudaGetSymbolAddress(reinterpret_cast<void**>(&word), cbk::g_linear_status);
    if (e == cudaSuccess) e = cudaMemcpyAsync(&v, word, sizeof v, cudaMemcpyDeviceToHost, s);
    if (e == cudaSuccess) e = cudaMemsetAsync(word, 0, sizeof v, s);
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) return cbk::cuda_error(e, "linear status");
    *status = v;
    return CB_OK;
}

}  // extern "C"
