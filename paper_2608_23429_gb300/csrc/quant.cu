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
// Buffers off the 16-byte grid (and gate rows of other than whole vectors) are reached by elements: a warp's vectors go
// through shared memory, so that its lanes then stand for consecutive elements (8 x 3 x [3, 333, 577], K = 5, gated hidden
// states: 73.6 us with a lane's elements consecutive instead).
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

// Two fp32 values in one register pair, for the units that take them together.
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
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

// Four codes as fp32: a byte under the exponent of 2^23 is 2^23 + byte, exactly.
__device__ __forceinline__ void codes4(uint32_t w, Two* v) {
    w ^= 0x80808080u;  // q + 128
    const Two less = two(-8388736.0f, -8388736.0f);
#pragma unroll
    for (int i = 0; i < 2; ++i)
        v[i] = add2(two(__uint_as_float(__byte_perm(w, 0x4B000000u, 0x7440 + 2 * i)),
                        __uint_as_float(__byte_perm(w, 0x4B000000u, 0x7441 + 2 * i))), less);
}

constexpr int kReadElems = 16;  // elements per thread and tile of the read kernel

// Bytes from a tensor's codes to its scales.
__device__ __forceinline__ long long scales_at(long long numel) { return (numel + 255) / 256 * 256; }

// sum_j w_j s_j q_j of the 16 elements from e (a multiple of 16, within the padded codes). The loads are volatile so that
// they stay ahead of the arithmetic, all in flight together.
template <int K>
__device__ __forceinline__ void predict16(const ExtrapArgs& A, const unsigned char* base, long long scales, long long e,
                                          float* p) {
    uint4 q[K];
    uint16_t c[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const unsigned char* at = base + A.slot_off[j];
        asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];"
                     : "=r"(q[j].x), "=r"(q[j].y), "=r"(q[j].z), "=r"(q[j].w)
                     : "l"(at + e));
        asm volatile("ld.global.u16 %0, [%1];" : "=h"(c[j]) : "l"(at + scales + e / kQuantBlock * 2));
    }
    Two acc[8];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const float f = __uint_as_float((uint32_t)c[j] << 16) * A.w_hi[j];
        const Two w = two(f, f);
        const uint32_t r[4] = {q[j].x, q[j].y, q[j].z, q[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            Two v[2];
            codes4(r[i], v);
#pragma unroll
            for (int k = 0; k < 2; ++k) acc[2 * i + k] = j == 0 ? mul2(w, v[k]) : fma2(w, v[k], acc[2 * i + k]);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = both(acc[i]);
        p[2 * i] = f.x, p[2 * i + 1] = f.y;
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
        const bool whole = left == kReadElems;
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

// ---- items that are not reached by vectors: lane l of a warp stands for the elements l, l + 32, l + 64, ... of its part

// N of them from or to p, of which `n` exist.
template <int N>
__device__ __forceinline__ void load_strided(const void* p, long long e, int bf16, int n, float* v) {
    if (bf16) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < n ? __uint_as_float((uint32_t)q[32 * i] << 16) : 0.0f;
    } else {
        const float* q = reinterpret_cast<const float*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < n ? q[32 * i] : 0.0f;
    }
}
template <int N>
__device__ __forceinline__ void store_strided(void* p, long long e, int bf16, int n, const float* v) {
    if (bf16) {
        __nv_bfloat16* q = reinterpret_cast<__nv_bfloat16*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) q[32 * i] = __float2bfloat16_rn(v[i]);
    } else {
        float* q = reinterpret_cast<float*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < n) q[32 * i] = v[i];
    }
}

// Indices into the item's gates of the elements e, e + 32, ... (the same for all of a group's members).
template <int N>
__device__ __forceinline__ void gate_indices(const ExtrapArgs& A, int it, long long e, int n, unsigned* at) {
    const unsigned hidden = A.i_hidden[it], row = A.i_row[it];
    unsigned long long sample = div_by((unsigned long long)e, A.i_row_magic[it]);
    unsigned h = (unsigned)((unsigned long long)e - div_by((unsigned long long)e, A.i_hidden_magic[it]) * hidden);
    unsigned long long left = (sample + 1) * row - (unsigned long long)e;  // elements to the sample's end
    unsigned base = (unsigned)sample * hidden;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        at[i] = base + h;
        if (hidden >= 32) {
            h += 32;
            if (h >= hidden) h -= hidden;
            if (left <= 32) base += hidden, left += row;
            left -= 32;
        } else if (i + 1 < n) {
            at[i + 1 < N ? i + 1 : i] = 0;
            const unsigned long long f = (unsigned long long)e + 32 * (i + 1);
            base = (unsigned)div_by(f, A.i_row_magic[it]) * hidden;
            h = (unsigned)(f - div_by(f, A.i_hidden_magic[it]) * hidden);
        }
    }
}

template <int N>
__device__ __forceinline__ void add_gated(const void* g, int bf16, int n, const unsigned* at, const float* p, float* acc) {
    float v[N];
    if (bf16) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = i < n ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(g)[at[i]] << 16) : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = i < n ? reinterpret_cast<const float*>(g)[at[i]] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) acc[i] = fmaf(v[i], p[i], acc[i]);
}

// Where a lane's 16 consecutive values lie in a warp's 512 words, in pieces of four that eight lanes reach without bank
// conflicts, and where element x of the 512 lies.
__device__ __forceinline__ int piece16(int lane, int j) { return lane * 16 + (j ^ (lane / 2 % 4)) * 4; }
__device__ __forceinline__ int word16(int x) { return piece16(x / 16, x / 4 % 4) + x % 4; }

template <int K>
__global__ void __launch_bounds__(kThreads) quant_read_elements_kernel(const __grid_constant__ ExtrapArgs A) {
    __shared__ float turns[kThreads / 32][32 * kReadElems];
    constexpr int N = kReadElems;
    constexpr long long TE = (long long)kThreads * N;
    after_previous();
    const int lane = threadIdx.x % 32;
    float* const turn = turns[threadIdx.x / 32];
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        while (tile >= A.tile_begin[it + 1]) ++it;
        const long long numel = A.numel[it], scales = scales_at(numel);
        const long long e0 = (long long)(tile - A.tile_begin[it]) * TE + (long long)(threadIdx.x / 32) * 32 * N;
        if (e0 >= numel) continue;
        const long long e = e0 + lane;
        const int n = (int)max(0ll, min((long long)N, (numel - e + 31) / 32));  // this lane's elements that exist
        void* const x = A.resid[it];
        const int m0 = A.first[it], m1 = m0 + A.nb[it];
        float acc[N];
        unsigned at[N];
        bool gated = false;
        if (x) {
            load_strided<N>(x, e, A.resid_bf16, n, acc);
            for (int m = m0; m < m1; ++m) gated = gated || A.m_gate[m];
            if (gated) gate_indices<N>(A, it, e, n, at);
        }
        for (int m = m0; m < m1; ++m) {
            float p[N];
            if (e0 + lane * N < numel)
                predict16<K>(A, reinterpret_cast<const unsigned char*>(A.hist_base) + A.m_off[m], scales, e0 + lane * N, p);
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 4; ++j)
                *reinterpret_cast<float4*>(turn + piece16(lane, j)) = make_float4(p[4 * j], p[4 * j + 1], p[4 * j + 2], p[4 * j + 3]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < N; ++i) p[i] = turn[word16(lane + 32 * i)];
            if (void* out = A.m_out[m]) store_strided<N>(out, e, A.out_bf16, n, p);
            if (!x) continue;
            if (const void* g = A.m_gate[m]) {
                add_gated<N>(g, A.gate_bf16, n, at, p, acc);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) acc[i] += p[i];
            }
        }
        if (x) store_strided<N>(x, e, A.resid_bf16, n, acc);
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

// Eight values of a block's thread to codes and, by the block's first thread, its scale. A block's eight threads exchange
// their maxima: threads behind the end run along, with zeros.
__device__ __forceinline__ void quantise8(const float* f, long long e, long long numel, long long scales, unsigned char* dst) {
    uint32_t amax = 0;
#pragma unroll
    for (int k = 0; k < kWriteElems; ++k) amax = max(amax, __float_as_uint(f[k]) & 0x7FFFFFFFu);
#pragma unroll
    for (int d = 1; d < kQuantBlock / kWriteElems; d <<= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
    const float s = scale_of(amax), inv = __frcp_rn(s);
    uint32_t q[kWriteElems];  // the code is the low byte: adding 1.5 * 2^23 rounds to an integer, ties to even
#pragma unroll
    for (int k = 0; k < kWriteElems; ++k) q[k] = __float_as_uint(__fadd_rn(__fmul_rn(f[k], inv), 12582912.0f));
    if (e >= (numel + kQuantBlock - 1) / kQuantBlock * kQuantBlock) return;
    const uint32_t lo = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
    const uint32_t hi = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
    *reinterpret_cast<uint2*>(dst + e) = make_uint2(lo, hi);
    if (e % kQuantBlock == 0)
        reinterpret_cast<uint16_t*>(dst + scales)[e / kQuantBlock] = (uint16_t)(__float_as_uint(s) >> 16);
}

// Where a lane's 8 consecutive values lie in a warp's 256 words, in pieces of four, and where element x of the 256 lies.
__device__ __forceinline__ int piece8(int lane, int j) { return lane * 8 + (j ^ (lane / 4 % 2)) * 4; }
__device__ __forceinline__ int word8(int x) { return piece8(x / 8, x / 4 % 2) + x % 4; }

template <bool GROUPED>
__global__ void __launch_bounds__(kThreads) quant_write_kernel(const __grid_constant__ ExtrapArgs A) {
    constexpr long long TE = (long long)kThreads * kWriteElems;
    after_previous();
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        while (tile >= A.tile_begin[it + 1]) ++it;
        const long long numel = A.numel[it];
        const long long e = (long long)(tile - A.tile_begin[it]) * TE + (long long)threadIdx.x * kWriteElems;
        const int left = e >= numel ? 0 : numel - e < kWriteElems ? (int)(numel - e) : kWriteElems;
        const bool whole = left == kWriteElems;
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
            quantise8(f, e, numel, scales_at(numel), reinterpret_cast<unsigned char*>(A.m_out[m]));
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

__global__ void __launch_bounds__(kThreads) quant_write_elements_kernel(const __grid_constant__ ExtrapArgs A) {
    __shared__ float turns[kThreads / 32][32 * kWriteElems];
    constexpr int N = kWriteElems;
    constexpr long long TE = (long long)kThreads * N;
    after_previous();
    const int lane = threadIdx.x % 32;
    float* const turn = turns[threadIdx.x / 32];
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        while (tile >= A.tile_begin[it + 1]) ++it;
        const long long numel = A.numel[it];
        const long long e0 = (long long)(tile - A.tile_begin[it]) * TE + (long long)(threadIdx.x / 32) * 32 * N;
        if (e0 >= numel) continue;
        const long long e = e0 + lane;
        const int n = (int)max(0ll, min((long long)N, (numel - e + 31) / 32));  // this lane's elements that exist
        void* const x = A.resid[it];
        const int m0 = A.first[it], m1 = m0 + A.nb[it];
        float acc[N];
        unsigned at[N];
        bool gated = false;
        if (x) {
            load_strided<N>(x, e, A.resid_bf16, n, acc);
            for (int m = m0; m < m1; ++m) gated = gated || A.m_gate[m];
            if (gated) gate_indices<N>(A, it, e, n, at);
        }
        for (int m = m0; m < m1; ++m) {
            float f[N];
            load_strided<N>(reinterpret_cast<const void*>(A.m_off[m]), e, A.src_bf16, n, f);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < N; ++i) turn[word8(lane + 32 * i)] = f[i];
            if (x) {
                if (const void* g = A.m_gate[m]) {
                    add_gated<N>(g, A.gate_bf16, n, at, f, acc);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[i] += f[i];
                }
            }
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float4 v = *reinterpret_cast<const float4*>(turn + piece8(lane, j));
                f[4 * j] = v.x, f[4 * j + 1] = v.y, f[4 * j + 2] = v.z, f[4 * j + 3] = v.w;
            }
            quantise8(f, e0 + lane * N, numel, scales_at(numel), reinterpret_cast<unsigned char*>(A.m_out[m]));
        }
        if (x) store_strided<N>(x, e, A.resid_bf16, n, acc);
    }
}

using Kernel = void (*)(ExtrapArgs);
template <int... Ks>
Kernel read_kernel(int K, QuantForm form) {
    static const Kernel plain[] = {quant_read_kernel<Ks, false>...}, group[] = {quant_read_kernel<Ks, true>...},
                        elements[] = {quant_read_elements_kernel<Ks>...};
    return (form == kQuantElements ? elements : form == kQuantGrouped ? group : plain)[K - 1];
}
Kernel kernel_of(int K, QuantForm form, bool write) {
    if (!write) return read_kernel<1, 2, 3, 4, 5, 6, 7, 8>(K, form);
    return form == kQuantElements ? quant_write_elements_kernel
           : form == kQuantGrouped ? quant_write_kernel<true>
                                   : quant_write_kernel<false>;
}

}  // namespace

cudaError_t quant_blocks_per_sm(int K, QuantForm form, bool write, int* blocks) {
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, kernel_of(K, form, write), kThreads, 0);
}

long long quant_tile_elems(bool write) { return (long long)kThreads * (write ? kWriteElems : kReadElems); }

cudaError_t launch_quant(const ExtrapArgs& a, int K, QuantForm form, bool write, int grid, cudaStream_t s) {
    return launch_overlapped(kernel_of(K, form, write), grid, kThreads, 0, s, a);
}

}  // namespace cbk
