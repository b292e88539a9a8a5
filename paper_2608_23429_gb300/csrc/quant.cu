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
// bf16. Persistent grids over tiles of 4096 elements, as in push.cu. GB300: read, 38 x [1, 4608, 3072], K = 5, 546 us (7.05
// TB/s); write, 56 x [8, 256, 1152] bf16, 68 us (5.9 TB/s); off the grid, as above, 34 us (2.7 TB/s).
#include <cuda_bf16.h>

#include <type_traits>

#include "cb_device.h"

namespace cbk {
namespace {

constexpr float kTiny = 1.17549435e-38f;  // 2^-126, the smallest scale: its reciprocal is finite

__device__ __forceinline__ uint4 ld_v4(const void* p) {
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

// Up to the item that `tile` belongs to, first in steps of eight, as a plan may have many small ones (GB300, 148 of 34720
// elements, K = 1: a read of 8.6 us one by one, 5.6 so).
__device__ __forceinline__ void pass_items(const ExtrapArgs& A, int tile, int& it) {
#pragma unroll 1
    while (it + 8 < A.n_items && tile >= A.tile_begin[it + 8]) it += 8;
#pragma unroll 1
    while (tile >= A.tile_begin[it + 1]) ++it;
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

// Sixteen, 32 bytes at a time where they lie on a 32-byte boundary (FLUX.1-dev single-stream blocks, K = 5: 649 -> 555 us
// against two stores of 16 bytes, each of which leaves half a sector for the other).
__device__ __forceinline__ void store32(void* p, uint32_t a, uint32_t b, uint32_t c, uint32_t d, uint32_t e, uint32_t f,
                                        uint32_t g, uint32_t h) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(a), "r"(b), "r"(c), "r"(d), "r"(e), "r"(f),
                 "r"(g), "r"(h)
                 : "memory");
}
__device__ __forceinline__ void store16(void* p, long long e, int bf16, const float* v) {
    char* const q = reinterpret_cast<char*>(p) + e * (bf16 ? 2 : 4);
    if ((uintptr_t)q % 32 != 0) {
        store8(p, e, bf16, v);
        store8(p, e + 8, bf16, v + 8);
    } else if (bf16) {
        store32(q, pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]),
                pack_bf16x2(v[8], v[9]), pack_bf16x2(v[10], v[11]), pack_bf16x2(v[12], v[13]), pack_bf16x2(v[14], v[15]));
    } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(v);
        store32(q, w[0], w[1], w[2], w[3], w[4], w[5], w[6], w[7]);
        store32(q + 32, w[8], w[9], w[10], w[11], w[12], w[13], w[14], w[15]);
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

// acc (+)= w s q for 16 codes.
__device__ __forceinline__ void add_codes(const uint4& q, uint16_t scale, float w, bool first, Two* acc) {
    const float f = __uint_as_float((uint32_t)scale << 16) * w;
    const uint32_t r[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        Two v[2];
        codes4(r[i], v);
#pragma unroll
        for (int k = 0; k < 2; ++k)
            acc[2 * i + k] = first ? mul2(two(f, f), v[k]) : fma2(two(f, f), v[k], acc[2 * i + k]);
    }
}
__device__ __forceinline__ void values_of(const Two* acc, float* p) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = both(acc[i]);
        p[2 * i] = f.x, p[2 * i + 1] = f.y;
    }
}

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
    for (int j = 0; j < K; ++j) add_codes(q[j], c[j], A.w_hi[j], j == 0, acc);
    values_of(acc, p);
}

// Predictions alone.
template <int K>
__global__ void __launch_bounds__(kThreads, 1) quant_read_kernel(const __grid_constant__ ExtrapArgs A) {
    constexpr long long TE = (long long)kThreads * kReadElems;
    after_previous();
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        pass_items(A, tile, it);
        const long long numel = A.numel[it];
        const long long e = (long long)(tile - A.tile_begin[it]) * TE + (long long)threadIdx.x * kReadElems;
        if (e >= numel) continue;
        const int m = A.first[it];
        float p[kReadElems];
        predict16<K>(A, reinterpret_cast<const unsigned char*>(A.hist_base) + A.m_off[m], scales_at(numel), e, p);
        if (numel - e >= kReadElems) {
            store16(A.m_out[m], e, A.out_bf16, p);
        } else {
            const int left = (int)(numel - e);
#pragma unroll
            for (int k = 0; k < kReadElems; ++k)
                if (k < left) put(A.m_out[m], e + k, p[k], A.out_bf16);
        }
    }
}

// ---- items that are not reached by vectors: lane l of a warp stands for the elements l, l + 32, l + 64, ... of its part

// N of them from or to p, of which `n` exist (FULL: all).
template <int N, bool FULL>
__device__ __forceinline__ void load_strided(const void* p, long long e, int bf16, int n, float* v) {
    if (bf16) {
        const uint16_t* q = reinterpret_cast<const uint16_t*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = FULL || i < n ? __uint_as_float((uint32_t)q[32 * i] << 16) : 0.0f;
    } else {
        const float* q = reinterpret_cast<const float*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = FULL || i < n ? q[32 * i] : 0.0f;
    }
}
template <int N, bool FULL>
__device__ __forceinline__ void store_strided(void* p, long long e, int bf16, int n, const float* v) {
    if (bf16) {
        __nv_bfloat16* q = reinterpret_cast<__nv_bfloat16*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (FULL || i < n) q[32 * i] = __float2bfloat16_rn(v[i]);
    } else {
        float* q = reinterpret_cast<float*>(p) + e;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (FULL || i < n) q[32 * i] = v[i];
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
    if (hidden >= 32) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            at[i] = base + h;
            h += 32;
            if (h >= hidden) h -= hidden;
            if (left <= 32) base += hidden, left += row;
            left -= 32;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i)
        at[i] = i < n ? (unsigned)gate_index(A, it, e + 32 * i) : 0u;
}

template <int N, bool FULL>
__device__ __forceinline__ void load_indexed(const void* g, int bf16, int n, const unsigned* at, float* v) {
    if (bf16) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = FULL || i < n ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(g)[at[i]] << 16) : 0.0f;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = FULL || i < n ? reinterpret_cast<const float*>(g)[at[i]] : 0.0f;
    }
}

// Where a lane's 16 consecutive values lie in a warp's 512 words, in pieces of four that eight lanes reach without bank
// conflicts, and where element x of the 512 lies.
__device__ __forceinline__ int piece16(int lane, int j) { return lane * 16 + (j ^ (lane / 2 % 4)) * 4; }
__device__ __forceinline__ int word16(int x) { return piece16(x / 16, x / 4 % 4) + x % 4; }

// Sixteen values as they lie in memory: two vectors of bf16, or four of fp32, the second half from element f on.
struct Raw16 {
    uint4 w[4];
};
__device__ __forceinline__ uint4 ld_v4_now(const void* p) {  // stays where it stands, ahead of a wait
    uint4 v;
    asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ void raw16(const void* p, long long e, long long f, int bf16, Raw16& r) {
    if (bf16) {
        r.w[0] = ld_v4_now(reinterpret_cast<const uint16_t*>(p) + e);
        r.w[1] = ld_v4_now(reinterpret_cast<const uint16_t*>(p) + f);
    } else {
        r.w[0] = ld_v4_now(reinterpret_cast<const float*>(p) + e);
        r.w[1] = ld_v4_now(reinterpret_cast<const float*>(p) + e + 4);
        r.w[2] = ld_v4_now(reinterpret_cast<const float*>(p) + f);
        r.w[3] = ld_v4_now(reinterpret_cast<const float*>(p) + f + 4);
    }
}
__device__ __forceinline__ void values_of(const Raw16& r, int bf16, float* v) {
    if (bf16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4& q = r.w[i / 4];
            const uint32_t w = i % 4 == 0 ? q.x : i % 4 == 1 ? q.y : i % 4 == 2 ? q.z : q.w;
            v[2 * i] = __uint_as_float(w << 16);
            v[2 * i + 1] = __uint_as_float(w & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[4 * i] = __uint_as_float(r.w[i].x), v[4 * i + 1] = __uint_as_float(r.w[i].y);
            v[4 * i + 2] = __uint_as_float(r.w[i].z), v[4 * i + 3] = __uint_as_float(r.w[i].w);
        }
    }
}

// Groups with a hidden state, and items that are not reached by vectors (ELEMENTS). A unit is one member's part of a tile.
// The codes of the next unit are on their way to shared memory while this one is worked on: each thread copies what it
// will read itself, so that nobody waits for anybody.
template <int K, bool ELEMENTS>
__global__ void __launch_bounds__(kThreads, ELEMENTS && K <= 5 ? 0 : 2) quant_read_group_kernel(const __grid_constant__ ExtrapArgs A) {
    extern __shared__ __align__(16) uint8_t shared[];
    constexpr int N = kReadElems;
    constexpr long long TE = (long long)kThreads * N;
    const int lane = threadIdx.x % 32;
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(shared) + threadIdx.x * 16;
    float* const turn = reinterpret_cast<float*>(shared + 2 * K * kThreads * 16) + threadIdx.x / 32 * 32 * N;
    struct Unit {
        int tile, it, m;
    };
    auto seek = [&](Unit& u) {
        if (u.tile >= A.tiles_total) return;
        pass_items(A, u.tile, u.it);
        u.m = A.first[u.it];
    };
    auto element = [&](const Unit& u) { return (long long)(u.tile - A.tile_begin[u.it]) * TE + (long long)threadIdx.x * N; };
    uint16_t c[K], c_next[K];
    auto fetch = [&](const Unit& u, int slot) {
        const long long e = element(u), numel = A.numel[u.it];
        if (e < numel) {
            const unsigned char* base = reinterpret_cast<const unsigned char*>(A.hist_base) + A.m_off[u.m];
            const long long scale = scales_at(numel) + e / kQuantBlock * 2;
#pragma unroll
            for (int j = 0; j < K; ++j) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(mine + (slot * K + j) * kThreads * 16),
                             "l"(base + A.slot_off[j] + e)
                             : "memory");
                asm volatile("ld.global.u16 %0, [%1];" : "=h"(c_next[j]) : "l"(base + A.slot_off[j] + scale));
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    after_previous();
    float acc[N];
    unsigned at[ELEMENTS ? N : 2];  // indices into the item's gates: of every element, or of the two vectors of 8
    Unit u{(int)blockIdx.x, 0, 0};
    seek(u);
    if (u.tile < A.tiles_total) fetch(u, 0);
    for (int slot = 0; u.tile < A.tiles_total; slot ^= 1) {
#pragma unroll
        for (int j = 0; j < K; ++j) c[j] = c_next[j];
        const int it = u.it, m = u.m;
        const bool opens = m == A.first[it], closes = m + 1 == A.first[it] + A.nb[it];
        Unit next = u;
        if (closes) next.tile += gridDim.x, seek(next);
        else ++next.m;
        const bool more = next.tile < A.tiles_total;
        if (more) fetch(next, slot ^ 1);
        const long long numel = A.numel[it], e = element(u);
        void *const x = A.resid[it], *const out = A.m_out[m];
        const void* const g = x ? A.m_gate[m] : nullptr;
        auto landed = [&] {
            if (more) asm volatile("cp.async.wait_group 1;" ::: "memory");
            else asm volatile("cp.async.wait_group 0;" ::: "memory");
        };
        auto predict = [&](float* p) {
            Two sum[8];
#pragma unroll
            for (int j = 0; j < K; ++j) {
                uint4 q;
                asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                             : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                             : "r"(mine + (slot * K + j) * kThreads * 16));
                add_codes(q, c[j], A.w_hi[j], j == 0, sum);
            }
            values_of(sum, p);
        };
        if constexpr (ELEMENTS) {
            const long long e0 = e - lane * N;  // of the warp
            auto unit = [&](auto full, int n) {  // n: this lane's elements that exist
                constexpr bool FULL = decltype(full)::value;
                if (x && opens) {
                    load_strided<N, FULL>(x, e0 + lane, A.resid_bf16, n, acc);
                    if (A.i_hidden[it]) gate_indices<N>(A, it, e0 + lane, n, at);
                }
                float gate[N], p[N];
                if (g) load_indexed<N, FULL>(g, A.gate_bf16, n, at, gate);
                landed();
                if (FULL || e < numel) predict(p);
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<float4*>(turn + piece16(lane, j)) = make_float4(p[4 * j], p[4 * j + 1], p[4 * j + 2], p[4 * j + 3]);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < N; ++i) p[i] = turn[word16(lane + 32 * i)];
                if (out) store_strided<N, FULL>(out, e0 + lane, A.out_bf16, n, p);
                if (!x) return;
                if (g) {
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[i] = fmaf(gate[i], p[i], acc[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[i] += p[i];
                }
                if (closes) store_strided<N, FULL>(x, e0 + lane, A.resid_bf16, n, acc);
            };
            if (e0 + 32 * N <= numel) unit(std::true_type{}, N);
            else if (e0 < numel) unit(std::false_type{}, (int)max(0ll, min((long long)N, (numel - e0 - lane + 31) / 32)));
        } else if (numel - e >= N) {
            Raw16 rx, rg;
            if (x && opens) {
                raw16(x, e, e + 8, A.resid_bf16, rx);
                if (A.i_hidden[it]) at[0] = (unsigned)gate_index(A, it, e), at[1] = (unsigned)gate_index(A, it, e + 8);
            }
            if (g) raw16(g, at[0], at[1], A.gate_bf16, rg);
            landed();
            float p[N];
            predict(p);
            if (out) store16(out, e, A.out_bf16, p);
            if (x) {
                if (opens) values_of(rx, A.resid_bf16, acc);
                if (g) {
                    float gate[N];
                    values_of(rg, A.gate_bf16, gate);
#pragma unroll
                    for (int k = 0; k < N; ++k) acc[k] = fmaf(gate[k], p[k], acc[k]);
                } else {
#pragma unroll
                    for (int k = 0; k < N; ++k) acc[k] += p[k];
                }
                if (closes) store16(x, e, A.resid_bf16, acc);
            }
        } else if (e < numel) {  // the item's last elements
            const int left = (int)(numel - e);
            landed();
            float p[N];
            predict(p);
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (k >= left) continue;
                if (out) put(out, e + k, p[k], A.out_bf16);
                if (!x) continue;
                if (opens) acc[k] = value_at(x, e + k, A.resid_bf16);
                acc[k] = fmaf(g ? value_at(g, gate_index(A, it, e + k), A.gate_bf16) : 1.0f, p[k], acc[k]);
                if (closes) put(x, e + k, acc[k], A.resid_bf16);
            }
        }
        u = next;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
}

// ---- the cache write

constexpr int kWriteElems = 16;  // consecutive, of a thread: four threads share a block
constexpr int kWriteParts = 2;   // such vectors of a thread and tile, loads of both in flight

// The block's scale from its largest magnitude (as bits: NaN above infinity above all others).
__device__ __forceinline__ float scale_of(uint32_t amax) {
    if (amax >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const float s = __uint_as_float(amax) * (1.0f / 127.0f);
    return fmaxf(__uint_as_float((__float_as_uint(s) + 0xFFFFu) & 0xFFFF0000u), kTiny);
}

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.u16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Their values, and the bits of the largest magnitude (which order as the magnitudes do).
__device__ __forceinline__ uint32_t values16(const Raw16& r, int bf16, Two* v) {
    uint32_t amax = 0;
    if (bf16) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4& q = r.w[i / 4];
            const uint32_t w = i % 4 == 0 ? q.x : i % 4 == 1 ? q.y : i % 4 == 2 ? q.z : q.w;
            amax = max_u16x2(amax, w & 0x7FFF7FFFu);
            v[i] = two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
        }
        amax = max(amax << 16, amax & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4& q = r.w[i];
            amax = max(max(amax, q.x & 0x7FFFFFFFu), max(q.y & 0x7FFFFFFFu, max(q.z & 0x7FFFFFFFu, q.w & 0x7FFFFFFFu)));
            v[2 * i] = two(__uint_as_float(q.x), __uint_as_float(q.y));
            v[2 * i + 1] = two(__uint_as_float(q.z), __uint_as_float(q.w));
        }
    }
    return amax;
}

// Sixteen values of a block's thread to codes and, by the block's first thread, its scale. The block's four threads
// exchange their maxima: threads behind the end run along, with zeros.
__device__ __forceinline__ void quantise16(const Two* v, uint32_t amax, long long e, long long numel, long long scales,
                                           unsigned char* dst) {
    amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
    amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
    const float s = scale_of(amax), inv = __frcp_rn(s);
    uint32_t code[4];  // the code is the low byte: adding 1.5 * 2^23 rounds to an integer, ties to even
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        // (products one by one: a packed product and sum become one operation, with one rounding)
        const float2 x = both(v[2 * i]), y = both(v[2 * i + 1]);
        const Two magic = two(12582912.0f, 12582912.0f);
        const float2 a = both(add2(two(__fmul_rn(x.x, inv), __fmul_rn(x.y, inv)), magic));
        const float2 b = both(add2(two(__fmul_rn(y.x, inv), __fmul_rn(y.y, inv)), magic));
        code[i] = __byte_perm(__byte_perm(__float_as_uint(a.x), __float_as_uint(a.y), 0x0040),
                              __byte_perm(__float_as_uint(b.x), __float_as_uint(b.y), 0x0040), 0x5410);
    }
    if (e >= (numel + kQuantBlock - 1) / kQuantBlock * kQuantBlock) return;
    *reinterpret_cast<uint4*>(dst + e) = make_uint4(code[0], code[1], code[2], code[3]);
    if (e % kQuantBlock == 0)
        reinterpret_cast<uint16_t*>(dst + scales)[e / kQuantBlock] = (uint16_t)(__float_as_uint(s) >> 16);
}

template <bool GROUPED>
__global__ void __launch_bounds__(kThreads) quant_write_kernel(const __grid_constant__ ExtrapArgs A) {
    constexpr int N = kWriteElems, P = GROUPED ? 1 : kWriteParts;
    constexpr long long TE = (long long)kThreads * N * kWriteParts;
    after_previous();
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        pass_items(A, tile, it);
        const long long numel = A.numel[it], scales = scales_at(numel);
        const long long tile_e = (long long)(tile - A.tile_begin[it]) * TE;
        for (int part = 0; part < kWriteParts; part += P) {
            const long long e = tile_e + ((long long)part * kThreads + threadIdx.x) * N;  // and, of further parts, kThreads * N on
            const int m0 = A.first[it], m1 = m0 + (GROUPED ? A.nb[it] : 1);
            void* const x = GROUPED ? A.resid[it] : nullptr;
            const long long warp_end = e + (32 - threadIdx.x % 32) * N + (long long)(P - 1) * kThreads * N;
            if (warp_end <= numel) {  // all of the warp's vectors are whole
                float acc[N];
                long long gate[2] = {0, 0};
                if (GROUPED && x) {
                    load8(x, e, A.resid_bf16, acc);
                    load8(x, e + 8, A.resid_bf16, acc + 8);
                    if (A.i_hidden[it]) gate[0] = gate_index(A, it, e), gate[1] = gate_index(A, it, e + 8);
                }
                for (int m = m0; m < m1; ++m) {
                    Raw16 raw[P];
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        const long long ei = e + (long long)i * kThreads * N;
                        raw16(reinterpret_cast<const void*>(A.m_off[m]), ei, ei + 8, A.src_bf16, raw[i]);
                    }
#pragma unroll
                    for (int i = 0; i < P; ++i) {
                        Two v[8];
                        const uint32_t amax = values16(raw[i], A.src_bf16, v);
                        quantise16(v, amax, e + (long long)i * kThreads * N, numel, scales, reinterpret_cast<unsigned char*>(A.m_out[m]));
                        if (!GROUPED || !x) continue;
                        const void* g = A.m_gate[m];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            float gv[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
                            if (g) load8(g, gate[h], A.gate_bf16, gv);
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const float2 f = both(v[4 * h + k]);
                                acc[8 * h + 2 * k] = fmaf(gv[2 * k], f.x, acc[8 * h + 2 * k]);
                                acc[8 * h + 2 * k + 1] = fmaf(gv[2 * k + 1], f.y, acc[8 * h + 2 * k + 1]);
                            }
                        }
                    }
                }
                if (GROUPED && x) store16(x, e, A.resid_bf16, acc);
                continue;
            }
            for (int i = 0; i < P; ++i) {  // at the end of the item: by elements
                const long long ei = e + (long long)i * kThreads * N;
                const int left = (int)max(0ll, min((long long)N, numel - ei));
                for (int m = m0; m < m1; ++m) {
                    const void* src = reinterpret_cast<const void*>(A.m_off[m]);
                    float f[N];
                    uint32_t amax = 0;
#pragma unroll
                    for (int k = 0; k < N; ++k) {
                        f[k] = k < left ? value_at(src, ei + k, A.src_bf16) : 0.0f;
                        amax = max(amax, __float_as_uint(f[k]) & 0x7FFFFFFFu);
                    }
                    Two v[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) v[k] = two(f[2 * k], f[2 * k + 1]);
                    quantise16(v, amax, ei, numel, scales, reinterpret_cast<unsigned char*>(A.m_out[m]));
                }
                if constexpr (GROUPED)
                    for (int k = 0; x && k < left; ++k) {
                        float a = value_at(x, ei + k, A.resid_bf16);
                        for (int m = m0; m < m1; ++m) {
                            const float f = value_at(reinterpret_cast<const void*>(A.m_off[m]), ei + k, A.src_bf16);
                            a = fmaf(A.m_gate[m] ? value_at(A.m_gate[m], gate_index(A, it, ei + k), A.gate_bf16) : 1.0f, f, a);
                        }
                        put(x, ei + k, a, A.resid_bf16);
                    }
            }
        }
    }
}

// Items that are not reached by vectors. Eight elements of a lane: twice the warps for the loads' latency.
__device__ __forceinline__ int piece8(int lane, int j) { return lane * 8 + (j ^ (lane / 4 % 2)) * 4; }
__device__ __forceinline__ int word8(int x) { return piece8(x / 8, x / 4 % 2) + x % 4; }

__global__ void __launch_bounds__(kThreads, 4) quant_write_elements_kernel(const __grid_constant__ ExtrapArgs A) {
    constexpr int N = 8;
    __shared__ float turns[kThreads / 32][32 * N];
    constexpr long long TE = (long long)kThreads * N;
    after_previous();
    const int lane = threadIdx.x % 32;
    float* const turn = turns[threadIdx.x / 32];
    int it = 0;
    for (int tile = blockIdx.x; tile < A.tiles_total; tile += gridDim.x) {
        pass_items(A, tile, it);
        const long long numel = A.numel[it], scales = scales_at(numel);
        const long long e0 = (long long)(tile - A.tile_begin[it]) * TE + (long long)(threadIdx.x / 32) * 32 * N;
        const long long e = e0 + lane;
        void* const x = A.resid[it];
        auto part = [&](auto full, int n) {  // n: this lane's elements that exist
            constexpr bool FULL = decltype(full)::value;
            const int m0 = A.first[it], m1 = m0 + A.nb[it];
            float acc[N];
            unsigned at[N];
            if (x) {
                load_strided<N, FULL>(x, e, A.resid_bf16, n, acc);
                if (A.i_hidden[it]) gate_indices<N>(A, it, e, n, at);
            }
            for (int m = m0; m < m1; ++m) {
                float f[N], gate[N];
                const void* const g = x ? A.m_gate[m] : nullptr;
                load_strided<N, FULL>(reinterpret_cast<const void*>(A.m_off[m]), e, A.src_bf16, n, f);
                if (g) load_indexed<N, FULL>(g, A.gate_bf16, n, at, gate);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < N; ++i) turn[word8(lane + 32 * i)] = f[i];
                if (x)
#pragma unroll
                    for (int i = 0; i < N; ++i) acc[i] = g ? fmaf(gate[i], f[i], acc[i]) : acc[i] + f[i];
                __syncwarp();
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float4 v = *reinterpret_cast<const float4*>(turn + piece8(lane, j));
                    f[4 * j] = v.x, f[4 * j + 1] = v.y, f[4 * j + 2] = v.z, f[4 * j + 3] = v.w;
                }
                uint32_t amax = 0;
#pragma unroll
                for (int k = 0; k < N; ++k) amax = max(amax, __float_as_uint(f[k]) & 0x7FFFFFFFu);
#pragma unroll
                for (int d = 1; d < kQuantBlock / N; d <<= 1) amax = max(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, d));
                const float s = scale_of(amax), inv = __frcp_rn(s);
                uint32_t q[N];
#pragma unroll
                for (int k = 0; k < N; ++k) q[k] = __float_as_uint(__fadd_rn(__fmul_rn(f[k], inv), 12582912.0f));
                const long long ev = e0 + lane * N;
                if (FULL || ev < (numel + kQuantBlock - 1) / kQuantBlock * kQuantBlock) {
                    unsigned char* const dst = reinterpret_cast<unsigned char*>(A.m_out[m]);
                    *reinterpret_cast<uint2*>(dst + ev) =
                        make_uint2(__byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410),
                                   __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410));
                    if (ev % kQuantBlock == 0)
                        reinterpret_cast<uint16_t*>(dst + scales)[ev / kQuantBlock] = (uint16_t)(__float_as_uint(s) >> 16);
                }
            }
            if (x) store_strided<N, FULL>(x, e, A.resid_bf16, n, acc);
        };
        if (e0 + 32 * N <= numel) part(std::true_type{}, N);
        else if (e0 < numel) part(std::false_type{}, (int)max(0ll, min((long long)N, (numel - e + 31) / 32)));
    }
}

using Kernel = void (*)(ExtrapArgs);
template <int... Ks>
Kernel read_kernel(int K, QuantForm form) {
    static const Kernel plain[] = {quant_read_kernel<Ks>...}, group[] = {quant_read_group_kernel<Ks, false>...},
                        elements[] = {quant_read_group_kernel<Ks, true>...};
    return (form == kQuantElements ? elements : form == kQuantGrouped ? group : plain)[K - 1];
}
Kernel kernel_of(int K, QuantForm form, bool write) {
    if (!write) return read_kernel<1, 2, 3, 4, 5, 6, 7, 8>(K, form);
    return form == kQuantElements ? quant_write_elements_kernel
           : form == kQuantGrouped ? quant_write_kernel<true>
                                   : quant_write_kernel<false>;
}
size_t smem_of(int K, QuantForm form, bool write) {
    if (write || form == kQuantPlain) return 0;
    return (size_t)2 * K * kThreads * 16 + (form == kQuantElements ? kThreads * kReadElems * sizeof(float) : 0);
}

}  // namespace

cudaError_t quant_blocks_per_sm(int K, QuantForm form, bool write, int* blocks) {
    const size_t smem = smem_of(K, form, write);
    if (smem) {
        const cudaError_t e = cudaFuncSetAttribute(kernel_of(K, form, write), cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, kernel_of(K, form, write), kThreads, smem);
}

long long quant_tile_elems(QuantForm form, bool write) {
    return (long long)kThreads * (!write ? kReadElems : form == kQuantElements ? 8 : kWriteElems * kWriteParts);
}

cudaError_t launch_quant(const ExtrapArgs& a, int K, QuantForm form, bool write, int grid, cudaStream_t s) {
    return launch_overlapped(kernel_of(K, form, write), grid, kThreads, smem_of(K, form, write), s, a);
}

}  // namespace cbk
