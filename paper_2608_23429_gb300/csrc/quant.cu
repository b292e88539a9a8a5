// The int8 history (cache type CB_INT8): a tensor's features are held as 8-bit
// codes with one bf16 scale per block of kQuantBlock consecutive elements,
//   s = max |x| / 127 over the block, up to the next bf16, at least 2^-126
//   q = x / s rounded to nearest, ties to even (|q| <= 127 by the choice of s)
// and a skipped step predicts from them directly,
//   P = sum_j w_j s_j q_j                     (Sec. 3.3, Eq. for f_t)
// in fp32. Codes are integers rather than e4m3 because the weights of an
// extrapolation amplify what the codes lose (K = 4 one spacing ahead: (-1, 4, -6,
// 4), norm 8.3): an integer step is 1/254 of the block's largest value at most,
// e4m3's is up to 1/16 of the value itself. A tensor in a slot: its codes, padded
// to whole blocks with zeros, on a 256-byte boundary, then its scales on the next.
// Non-finite features take their whole block with them: its scale is not finite,
// and the block's predictions are NaN.
//
// Both kernels are bound by HBM: 1 1/32 bytes per element and entry against 2 of
// bf16. Persistent grids over tiles of 4096 elements, as in push.cu.
#include <cuda_bf16.h>

#include "cb_device.h"

namespace cbk {
namespace {

constexpr float kTiny = 1.17549435e-38f;  // 2^-126, the smallest scale: its reciprocal is finite

__device__ __forceinline__ uint4 ld_v4(const void* p) {
    uint4 v;
    asm("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

__device__ __forceinline__ float bf16_at(const void* p, long long i) {
    return __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[i] << 16);
}
__device__ __forceinline__ float value_at(const void* p, long long i, int bf16) {
    return bf16 ? bf16_at(p, i) : reinterpret_cast<const float*>(p)[i];
}
__device__ __forceinline__ void put(void* p, long long i, float v, int bf16) {
    if (bf16)
        reinterpret_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
    else
        reinterpret_cast<float*>(p)[i] = v;
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

// Eight consecutive values from or to a 16-byte boundary.
__device__ __forceinline__ void load8(const void* p, long long e, int bf16, float* v) {
    if (bf16) {
        const uint4 r = ld_v4(reinterpret_cast<const uint16_t*>(p) + e);
        const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint4 r = ld_v4(reinterpret_cast<const float*>(p) + e + 4 * h);
            v[4 * h] = __uint_as_float(r.x);
            v[4 * h + 1] = __uint_as_float(r.y);
            v[4 * h + 2] = __uint_as_float(r.z);
            v[4 * h + 3] = __uint_as_float(r.w);
        }
    }
}
__device__ __forceinline__ void store8(void* p, long long e, int bf16, const float* v) {
    if (bf16) {
        *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + e) =
            make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    } else {
        float4* q = reinterpret_cast<float4*>(reinterpret_cast<float*>(p) + e);
        q[0] = make_float4(v[0], v[1], v[2], v[3]);
        q[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
}

// Division by a shape's size through its multiplier ceil(2^64 / d) (0: d = 1).
__device__ __forceinline__ unsigned long long div_by(unsigned long long e, unsigned long long magic) {
    return magic ? __umul64hi(e, magic) : e;
}
// Index into a gate [batch, hidden] of element e of [batch, tokens, hidden].
__device__ __forceinline__ long long gate_index(const ExtrapArgs& A, int it, long long e) {
    const unsigned long long b = div_by((unsigned long long)e, A.i_row_magic[it]);
    const unsigned long long r = div_by((unsigned long long)e, A.i_hidden_magic[it]);
    return (long long)(b * A.i_hidden[it] + ((unsigned long long)e - r * A.i_hidden[it]));
}

// Four codes as fp32: a byte under the exponent of 2^23 is 2^23 + byte, exactly.
__device__ __forceinline__ void codes4(uint32_t w, float* v) {
    w ^= 0x80808080u;  // q + 128
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440 + i)) - 8388736.0f;
}

constexpr int kReadElems = 16;  // elements per thread and tile of the read kernel

// Bytes from a tensor's codes to its scales.
__device__ __forceinline__ long long scales_at(long long numel) { return (numel + 255) / 256 * 256; }

// sum_j w_j s_j q_j of the 16 elements from e (a multiple of 16, within the padded codes).
template <int K>
__device__ __forceinline__ void predict16(const ExtrapArgs& A, const unsigned char* base, long long scales, long long e,
                                          float* p) {
    uint4 q[K];
    float c[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        q[j] = ld_v4(base + A.slot_off[j] + e);
        c[j] = bf16_at(base + A.slot_off[j] + scales, e / kQuantBlock);
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const float w = c[j] * A.w_hi[j];
        const uint32_t r[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float v[4];
            codes4(r[i], v);
#pragma unroll
            for (int k = 0; k < 4; ++k) p[4 * i + k] = j == 0 ? w * v[k] : fmaf(w, v[k], p[4 * i + k]);
        }
    }
}

template <int K, bool GROUPED>
__global__ void __launch_bounds__(kThreads) quant_read_kernel(const __grid_constant__ ExtrapArgs A) {
    constexpr long long TE = (long long)kThreads * kReadElems;
    after_previous();
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        while (tile >= A.tile_begin[it + 1]) ++it;
        const long long numel = A.numel[it];
        const long long e = (long long)(tile - A.tile_begin[it]) * TE + (long long)threadIdx.x * kReadElems;
        if (e >= numel) continue;
        const long long scales = scales_at(numel);
        const int left = numel - e < kReadElems ? (int)(numel - e) : kReadElems;
        const bool whole = A.vec_ok[it] && left == kReadElems;
        void* const x = GROUPED ? A.resid[it] : nullptr;
        float acc[kReadElems];
        if (GROUPED && x) {
            if (whole) {
                load8(x, e, A.resid_bf16, acc);
                load8(x, e + 8, A.resid_bf16, acc + 8);
            } else {
#pragma unroll
                for (int k = 0; k < kReadElems; ++k) acc[k] = k < left ? value_at(x, e + k, A.resid_bf16) : 0.0f;
            }
        }
        const int m0 = A.first[it], m1 = m0 + (GROUPED ? A.nb[it] : 1);
        for (int m = m0; m < m1; ++m) {
            float p[kReadElems];
            predict16<K>(A, reinterpret_cast<const unsigned char*>(A.hist_base) + A.m_off[m], scales, e, p);
            if (void* out = A.m_out[m]) {
                if (whole) {
                    store8(out, e, A.out_bf16, p);
                    store8(out, e + 8, A.out_bf16, p + 8);
                } else {
#pragma unroll
                    for (int k = 0; k < kReadElems; ++k)
                        if (k < left) put(out, e + k, p[k], A.out_bf16);
                }
            }
            if (GROUPED && x) {
                const void* g = A.m_gate[m];
                if (!g) {
#pragma unroll
                    for (int k = 0; k < kReadElems; ++k) acc[k] += p[k];
                } else if (whole) {  // vectors of 8 stay inside one gate row
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float gv[8];
                        load8(g, gate_index(A, it, e + 8 * h), A.gate_bf16, gv);
#pragma unroll
                        for (int k = 0; k < 8; ++k) acc[8 * h + k] = fmaf(gv[k], p[8 * h + k], acc[8 * h + k]);
                    }
                } else {
#pragma unroll
                    for (int k = 0; k < kReadElems; ++k)
                        if (k < left) acc[k] = fmaf(value_at(g, gate_index(A, it, e + k), A.gate_bf16), p[k], acc[k]);
                }
            }
        }
        if (GROUPED && x) {
            if (whole) {
                store8(x, e, A.resid_bf16, acc);
                store8(x, e + 8, A.resid_bf16, acc + 8);
            } else {
#pragma unroll
                for (int k = 0; k < kReadElems; ++k)
                    if (k < left) put(x, e + k, acc[k], A.resid_bf16);
            }
        }
    }
}

// ---- the cache write

constexpr int kWriteElems = 8;  // per thread: eight threads share a block

// The block's scale from its largest magnitude (as bits: NaN above infinity above all others).
__device__ __forceinline__ float scale_of(uint32_t amax) {
    if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float s = __uint_as_float(amax) * (1.0f / 127.0f);
    return fmaxf(__uint_as_float((__float_as_uint(s) + 0xFFFFu) & 0xFFFF0000u), kTiny);
}

template <bool GROUPED>
__global__ void __launch_bounds__(kThreads) quant_write_kernel(const __grid_constant__ ExtrapArgs A) {
    constexpr long long TE = (long long)kThreads * kWriteElems;
    after_previous();
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        while (tile >= A.tile_begin[it + 1]) ++it;
        const long long numel = A.numel[it];
        const long long e = (long long)(tile - A.tile_begin[it]) * TE + (long long)threadIdx.x * kWriteElems;
        const long long scales = scales_at(numel);
        // threads behind the end run along: a block's eight threads exchange their maxima
        const int left = e >= numel ? 0 : numel - e < kWriteElems ? (int)(numel - e) : kWriteElems;
        const bool whole = A.vec_ok[it] && left == kWriteElems;
        void* const x = GROUPED ? A.resid[it] : nullptr;
        float acc[kWriteElems];
        if (GROUPED && x) {
            if (whole) {
                load8(x, e, A.resid_bf16, acc);
            } else {
#pragma unroll
                for (int k = 0; k < kWriteElems; ++k) acc[k] = k < left ? value_at(x, e + k, A.resid_bf16) : 0.0f;
            }
        }
        const int m0 = A.first[it], m1 = m0 + (GROUPED ? A.nb[it] : 1);
        for (int m = m0; m < m1; ++m) {
            const void* src = reinterpret_cast<const void*>(A.m_off[m]);
            float f[kWriteElems];
            if (whole) {
                load8(src, e, A.src_bf16, f);
            } else {
#pragma unroll
                for (int k = 0; k < kWriteElems; ++k) f[k] = k < left ? value_at(src, e + k, A.src_bf16) : 0.0f;
            }
            uint32_t amax = 0;
#pragma unroll
            for (int k = 0; k < kWriteElems; ++k) amax = max(amax, __float_as_uint(f[k]) & 0x7FFFFFFFu);
#pragma unroll
            for (int d = 1; d < kQuantBlock / kWriteElems; d <<= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
            const float s = scale_of(amax), inv = __frcp_rn(s);
            uint32_t q[kWriteElems];  // the code is the low byte: adding 1.5 * 2^23 rounds to an integer, ties to even
#pragma unroll
            for (int k = 0; k < kWriteElems; ++k)
                q[k] = __float_as_uint(__fadd_rn(__fmul_rn(f[k], inv), 12582912.0f));
            unsigned char* dst = reinterpret_cast<unsigned char*>(A.m_out[m]);
            if (e < (numel + kQuantBlock - 1) / kQuantBlock * kQuantBlock) {
                const uint32_t lo = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
                const uint32_t hi = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
                *reinterpret_cast<uint2*>(dst + e) = make_uint2(lo, hi);
                if (e % kQuantBlock == 0)
                    reinterpret_cast<uint16_t*>(dst + scales)[e / kQuantBlock] = (uint16_t)(__float_as_uint(s) >> 16);
            }
            if (GROUPED && x) {
                const void* g = A.m_gate[m];
                if (!g) {
#pragma unroll
                    for (int k = 0; k < kWriteElems; ++k) acc[k] += f[k];
                } else if (whole) {
                    float gv[8];
                    load8(g, gate_index(A, it, e), A.gate_bf16, gv);
#pragma unroll
                    for (int k = 0; k < kWriteElems; ++k) acc[k] = fmaf(gv[k], f[k], acc[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < kWriteElems; ++k)
                        if (k < left) acc[k] = fmaf(value_at(g, gate_index(A, it, e + k), A.gate_bf16), f[k], acc[k]);
                }
            }
        }
        if (GROUPED && x) {
            if (whole) {
                store8(x, e, A.resid_bf16, acc);
            } else {
#pragma unroll
                for (int k = 0; k < kWriteElems; ++k)
                    if (k < left) put(x, e + k, acc[k], A.resid_bf16);
            }
        }
    }
}

using ReadKernel = void (*)(ExtrapArgs);
template <int... Ks>
ReadKernel read_kernel(int K, bool grouped) {
    static const ReadKernel plain[] = {quant_read_kernel<Ks, false>...}, group[] = {quant_read_kernel<Ks, true>...};
    return (grouped ? group : plain)[K - 1];
}
ReadKernel read_kernel_of(int K, bool grouped) { return read_kernel<1, 2, 3, 4, 5, 6, 7, 8>(K, grouped); }

}  // namespace

cudaError_t quant_blocks_per_sm(int K, bool grouped, bool write, int* blocks) {
    if (write)
        return cudaOccupancyMaxActiveBlocksPerMultiprocessor(
            blocks, grouped ? quant_write_kernel<true> : quant_write_kernel<false>, kThreads, 0);
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, read_kernel_of(K, grouped), kThreads, 0);
}

long long quant_tile_elems(bool write) { return (long long)kThreads * (write ? kWriteElems : kReadElems); }

cudaError_t launch_quant_read(const ExtrapArgs& a, int K, bool grouped, int grid, cudaStream_t s) {
    return launch_overlapped(read_kernel_of(K, grouped), grid, kThreads, 0, s, a);
}

cudaError_t launch_quant_write(const ExtrapArgs& a, bool grouped, int grid, cudaStream_t s) {
    return launch_overlapped(grouped ? quant_write_kernel<true> : quant_write_kernel<false>, grid, kThreads, 0, s, a);
}

}  // namespace cbk
