// Internal: the RMS norm of rows reached by vectors (see norm.cu), instantiated per type of the lines
// (norm_lines_*.cu). Types are template arguments, and pairs of values stay in register pairs: with types looked up and
// values unpacked as it went the kernel issued 1450 instructions per row of 1152 elements and was bound by that. Loads
// stand in one piece for all chunks, without branches between them (threads behind the row's end copy zeros and read its
// start): one chunk's after the other's cost a latency each, 5 us a row.
#pragma once

#include "norm.cuh"

namespace cbk {
namespace {

// Eight values as they lie in memory, and as pairs.
template <bool BF16>
struct Raw8 {
    uint4 w[BF16 ? 1 : 2];
};
template <bool BF16>
__device__ __forceinline__ void pairs_of(const Raw8<BF16>& r, Two* v) {
    if constexpr (BF16) {
        const uint32_t w[4] = {r.w[0].x, r.w[0].y, r.w[0].z, r.w[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = two(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xFFFF0000u));
    } else {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint4& q = r.w[BF16 ? 0 : i];
            v[2 * i] = two(__uint_as_float(q.x), __uint_as_float(q.y));
            v[2 * i + 1] = two(__uint_as_float(q.z), __uint_as_float(q.w));
        }
    }
}
template <bool BF16>
__device__ __forceinline__ Raw8<BF16> load8(const void* p, long long e) {
    Raw8<BF16> r;
    const char* a = reinterpret_cast<const char*>(p) + (BF16 ? 2 : 4) * e;
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i)
        asm volatile("ld.global.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w) : "l"(a + 16 * i));
    return r;
}
// fp32 in one store of 32 bytes where it lies on such a boundary: two of 16 leave half a sector for each other.
__device__ __forceinline__ void store8_fp32(float* q, const Two* v) {
    if ((uintptr_t)q % 32 == 0) {
        asm volatile("st.global.v4.b64 [%0], {%1,%2,%3,%4};" ::"l"(q), "l"(v[0]), "l"(v[1]), "l"(v[2]), "l"(v[3]) : "memory");
    } else {
        reinterpret_cast<ulonglong2*>(q)[0] = make_ulonglong2(v[0], v[1]);
        reinterpret_cast<ulonglong2*>(q)[1] = make_ulonglong2(v[2], v[3]);
    }
}
__device__ __forceinline__ void store8_bf16(void* p, long long e, const Two* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = both(v[i]);
        w[i] = norm_bf16x2(f.x, f.y);
    }
    *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + e) = make_uint4(w[0], w[1], w[2], w[3]);
}

constexpr int kWarpRows = 4;  // warps of a CTA whose rows have a warp each
__host__ __device__ constexpr int norm_threads(int W) { return 32 * (W == 1 ? kWarpRows : W); }
__host__ __device__ constexpr int norm_ctas(int CH, int W) { return (CH == 1 ? 1024 : CH == 2 ? 768 : 512) / norm_threads(W); }
// Bytes of shared memory of a thread's chunk: 16-byte pieces of x and of branch.
template <bool XB, bool BB>
__host__ __device__ constexpr int norm_pieces() { return (XB ? 1 : 2) + (BB ? 1 : 2); }

template <int CH, int W, bool XB, bool BB, bool LB>
__global__ void __launch_bounds__(norm_threads(W), norm_ctas(CH, W)) norm_kernel(const __grid_constant__ NormArgs args) {
    __shared__ uint32_t slots[2][2][W];
    extern __shared__ __align__(16) uint8_t ring[];
    constexpr int threads = 32 * W, P = norm_pieces<XB, BB>(), step = norm_threads(W) * 16;
    const NormArgs A = args;  // in registers, as stores would have them read again
    const int t = threadIdx.x % threads;
    const unsigned team = W == 1 ? blockIdx.x * kWarpRows + threadIdx.x / 32 : blockIdx.x;
    const unsigned first = (unsigned)min((unsigned long long)team * A.team_rows, (unsigned long long)A.rows);
    const unsigned end = first + min(A.team_rows, A.rows - first);
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    const int e0 = t * 8;  // its first element; the others follow in steps of 8 * threads
    auto on = [&](int c) { return e0 + c * threads * 8 < A.hidden; };
    auto column = [&](int c) { return on(c) ? c * threads * 8 : -e0; };  // of chunk c behind e0, or the row's start
    auto fetch = [&](unsigned row) {  // the row's chunks of x and branch, in pieces of 16 bytes
        if (row < end) {
            const char* const x = reinterpret_cast<const char*>(A.x) + (row * A.x_stride + e0) * (XB ? 2 : 4);
            auto copy = [&](uint32_t dst, const char* p, int size) {
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(p), "r"(size) : "memory");
            };
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < (XB ? 1 : 2); ++i)
                    copy(mine + (c * P + i) * step, x + column(c) * (XB ? 2 : 4) + 16 * i, on(c) ? 16 : 0);
            if (A.branch) {
                const char* const b = reinterpret_cast<const char*>(A.branch) + (row * A.branch_stride + e0) * (BB ? 2 : 4);
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < (BB ? 1 : 2); ++i)
                        copy(mine + (c * P + (XB ? 1 : 2) + i) * step, b + column(c) * (BB ? 2 : 4) + 16 * i, on(c) ? 16 : 0);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto landed = [&](uint32_t from, auto& r) {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(r) / 16); ++i)
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w)
                         : "r"(from + i * step));
    };
    after_previous();
    unsigned sample = 0, next_sample = 0;  // the next sample's first row
    if (first < end) sample = first / A.tokens, next_sample = sample * A.tokens;
    long long line = 0;
    fetch(first);
    for (unsigned row = first; row < end; ++row) {
        if (row >= next_sample) {
            line = (long long)sample * A.line_stride + e0;
            ++sample, next_sample += min(A.tokens, 0xFFFFFFFFu - next_sample);
        }
        Raw8<LB> lines[2][CH];  // gate; then scale and shift
        if (A.gate)
#pragma unroll
            for (int c = 0; c < CH; ++c) lines[0][c] = load8<LB>(A.gate, line + column(c));
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        uint32_t(*const words)[W] = slots[row % 2];
        Two h[CH][4], sum2 = two(0.0f, 0.0f);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            Raw8<XB> x;
            landed(mine + c * P * step, x);
            pairs_of(x, h[c]);
        }
        if (A.branch)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                Raw8<BB> b;
                Two v[4], g[4];
                landed(mine + (c * P + (XB ? 1 : 2)) * step, b);
                pairs_of(b, v);
                if (A.gate) {
                    pairs_of(lines[0][c], g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[c][i] = fma2(g[i], v[i], h[c][i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[c][i] = add2(h[c][i], v[i]);
                }
            }
        fetch(row + 1);  // into the places just read
        if (A.scale)
#pragma unroll
            for (int c = 0; c < CH; ++c) lines[0][c] = load8<LB>(A.scale, line + column(c));
        if (A.shift)
#pragma unroll
            for (int c = 0; c < CH; ++c) lines[1][c] = load8<LB>(A.shift, line + column(c));
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (on(c)) {  // (zeros behind the row's end, but times its first gates)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum2 = fma2(h[c][i], h[c][i], sum2);
            }
        if (A.x_out) {
            const long long at = row * A.x_out_stride + e0;
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!on(c)) continue;
                if constexpr (XB) store8_bf16(A.x_out, at + c * threads * 8, h[c]);
                else store8_fp32(reinterpret_cast<float*>(A.x_out) + at + c * threads * 8, h[c]);
            }
        }
        const float2 parts = both(sum2);
        const float sum = __uint_as_float(row_reduce<W, false>(__float_as_uint(parts.x + parts.y), words[0]));
        const float rstd = 1.0f / sqrtf(fmaf(sum, A.inv_hidden, A.eps));
        const Two rstd2 = two(rstd, rstd);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) h[c][i] = mul2(h[c][i], rstd2);
        Two v[4];
        if (A.weight) {
            Raw8<LB> w[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) w[c] = load8<LB>(A.weight, e0 + column(c));
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs_of(w[c], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[c][i] = mul2(h[c][i], v[i]);
            }
        }
        if (A.scale)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs_of(lines[0][c], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[c][i] = fma2(h[c][i], v[i], h[c][i]);
            }
        if (A.shift)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                pairs_of(lines[1][c], v);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[c][i] = add2(h[c][i], v[i]);
            }
        float amax = 0.0f;
        if (A.out_dtype == CB_E4M3)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = both(h[c][i]);
                    most = max_abs(max_abs(most, f.x), f.y);
                }
                amax = max_abs(amax, on(c) ? most : 0.0f);
            }
        const long long at = row * A.out_stride + e0;
        if (A.out_dtype == CB_E4M3) {
            const float s = norm_scale_of(row_reduce<W, true>(__float_as_uint(amax) & 0x7FFFFFFFu, words[1]));
            if (t == 0) A.out_scale[row] = s;
            const float inv = __frcp_rn(s);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!on(c)) continue;
                uint32_t w[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = both(mul2(h[c][i], two(inv, inv)));
                    w[i] = norm_e4m3x2(f.x, f.y);
                }
                *reinterpret_cast<uint2*>(reinterpret_cast<uint8_t*>(A.out) + at + c * threads * 8) =
                    make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
            }
        } else {
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                if (!on(c)) continue;
                if (A.out_dtype == CB_BF16) store8_bf16(A.out, at + c * threads * 8, h[c]);
                else store8_fp32(reinterpret_cast<float*>(A.out) + at + c * threads * 8, h[c]);
            }
        }
    }
}

template <int CH, int W, bool XB, bool BB, bool LB>
cudaError_t launch(NormArgs& a, int sms, cudaStream_t s) {
    constexpr int threads = norm_threads(W), teams = W == 1 ? kWarpRows : 1;
    constexpr size_t smem = (size_t)CH * norm_pieces<XB, BB>() * 16 * threads;
    // as many CTAs as are resident together
    const int per_sm = std::max(1, std::min(norm_ctas(CH, W), (int)(224 * 1024 / (smem + 2048))));
    const unsigned long long all = (unsigned long long)sms * per_sm * teams;
    a.team_rows = (unsigned)((a.rows + all - 1) / all);
    const unsigned used = (a.rows + a.team_rows - 1) / a.team_rows;
    const auto k = norm_kernel<CH, W, XB, BB, LB>;
    if (smem > 47 * 1024) {  // with the kernel's own words
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapped(k, (int)((used + teams - 1) / teams), threads, smem, s, a);
}

// The row's warps and chunks: one warp up to 1280 elements, then four, eight or sixteen with up to four chunks a thread.
template <bool XB, bool BB, bool LB>
cudaError_t launch_types(NormArgs& a, int sms, cudaStream_t s) {
    const int n = a.hidden / 8;
    if (n <= 32) return launch<1, 1, XB, BB, LB>(a, sms, s);
    if (n <= 64) return launch<2, 1, XB, BB, LB>(a, sms, s);
    if (n <= 96) return launch<3, 1, XB, BB, LB>(a, sms, s);
    if (n <= 160) return launch<5, 1, XB, BB, LB>(a, sms, s);
    if (n <= 256) return launch<2, 4, XB, BB, LB>(a, sms, s);
    if (n <= 384) return launch<3, 4, XB, BB, LB>(a, sms, s);
    if (n <= 512) return launch<4, 4, XB, BB, LB>(a, sms, s);
    if (n <= 1024) return launch<4, 8, XB, BB, LB>(a, sms, s);
    return launch<4, 16, XB, BB, LB>(a, sms, s);
}

template <bool LB>
cudaError_t launch_lines(NormArgs& a, int sms, cudaStream_t s) {
    if (a.x_bf16) return a.branch_bf16 ? launch_types<true, true, LB>(a, sms, s) : launch_types<true, false, LB>(a, sms, s);
    return a.branch_bf16 ? launch_types<false, true, LB>(a, sms, s) : launch_types<false, false, LB>(a, sms, s);
}

}  // namespace
}  // namespace cbk
