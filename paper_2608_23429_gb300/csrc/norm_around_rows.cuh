// Internal: the norms around a block for rows reached by vectors (see norm_around.cu), instantiated per type of the lines
// (norm_around_*.cu). A row's way is that of cb_norm_residual (norm_rows.cuh): a warp, or 4 to 16, holds it in registers while the next
// one is on its way to shared memory.
#pragma once

#include "norm_around.cuh"
#include "norm_rows.cuh"

namespace cbk {
namespace {

constexpr int kAroundReductions = 5;  // of a row: mean and variance of branch and hidden state, and the largest magnitude

// The row in CH chunks of a thread, off its mean (LAYER) and over its root mean square. on(c): the chunk lies in the row.
template <int CH, int W, typename On>
__device__ __forceinline__ void normalise(Two (&v)[CH][4], int kind, float eps, float inv_hidden, On on, uint32_t (*slots)[W]) {
    if (kind == CB_NORM_LAYER) {
        Two sum2 = two(0.0f, 0.0f);
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if (on(c)) {
#pragma unroll
                for (int i = 0; i < 4; ++i) sum2 = add2(sum2, v[c][i]);
            }
        const float2 parts = both(sum2);
        const float mean = __uint_as_float(row_reduce<W, false>(__float_as_uint(parts.x + parts.y), slots[0])) * inv_hidden;
        const Two off = two(-mean, -mean);
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] = add2(v[c][i], off);
    }
    Two sum2 = two(0.0f, 0.0f);
#pragma unroll
    for (int c = 0; c < CH; ++c)
        if (on(c)) {
#pragma unroll
            for (int i = 0; i < 4; ++i) sum2 = fma2(v[c][i], v[c][i], sum2);
        }
    const float2 parts = both(sum2);
    const float sum = __uint_as_float(row_reduce<W, false>(__float_as_uint(parts.x + parts.y), slots[1]));
    const float rstd = 1.0f / sqrtf(fmaf(sum, inv_hidden, eps));
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) v[c][i] = mul2(v[c][i], two(rstd, rstd));
}

template <bool BF16>
struct RowType {
    static constexpr bool bf16 = BF16;
};

template <int CH, int W, bool XB, bool BB, bool LB>
__global__ void __launch_bounds__(norm_threads(W), norm_ctas(CH, W)) around_kernel(const __grid_constant__ AroundArgs args) {
    __shared__ uint32_t slots[2][kAroundReductions][W];
    extern __shared__ __align__(16) uint8_t ring[];
    constexpr int threads = 32 * W, P = norm_pieces<XB, BB>(), step = norm_threads(W) * 16;
    const AroundArgs A = args;  // in registers, as stores would have them read again
    const int t = threadIdx.x % threads;
    const unsigned team = W == 1 ? blockIdx.x * kWarpRows + threadIdx.x / 32 : blockIdx.x;
    const unsigned first = (unsigned)min((unsigned long long)team * A.team_rows, (unsigned long long)A.rows);
    const unsigned end = first + min(A.team_rows, A.rows - first);
    const int e0 = t * 8;  // its first element; the others follow in steps of 8 * threads
    auto on = [&](int c) { return c + 1 < CH || e0 + c * threads * 8 < A.hidden; };  // (the launch has as few chunks as the row needs)
    auto column = [&](int c) { return on(c) ? c * threads * 8 : -e0; };  // of chunk c behind e0, or the row's start
    // A row comes to shared memory in pieces of 16 bytes. Each lane copies its own of bf16; of fp32, where a lane's eight elements are two,
    // the warp copies 512 bytes at a time (two halves of every sector took the copies twice as long) and reads across lanes.
    const int lane = threadIdx.x % 32;
    const uint32_t own = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * 16;
    const uint32_t across = (uint32_t)__cvta_generic_to_shared(ring) + (threadIdx.x - lane) * 16 + lane / 16 * step + lane % 16 * 32;
    auto copy = [&](uint32_t dst, const char* p, bool in) {
        const int size = in ? 16 : 0;
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(p), "r"(size) : "memory");
    };
    auto fetch_rows = [&](const char* p, auto type, int piece) {  // p: the row's start
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if constexpr (decltype(type)::bf16) {
                copy(own + (c * P + piece) * step, p + (e0 + column(c)) * 2, on(c));
            } else {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int e = c * threads * 8 + (t - lane) * 8 + i * 128 + lane * 4;
                    const bool in = c + 1 < CH || e < A.hidden;
                    copy(own + (c * P + piece + i) * step, p + (in ? e : 0) * 4, in);
                }
            }
        }
    };
    auto fetch = [&](unsigned row) {  // the row's chunks of x and branch
        if (row < end) {
            fetch_rows(reinterpret_cast<const char*>(A.x) + row * A.x_stride * (XB ? 2 : 4), RowType<XB>{}, 0);
            if (A.branch) fetch_rows(reinterpret_cast<const char*>(A.branch) + row * A.branch_stride * (BB ? 2 : 4), RowType<BB>{}, XB ? 1 : 2);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    auto landed = [&](int c, int piece, auto& r) {
        constexpr bool bf16 = sizeof(r) == 16;
#pragma unroll
        for (int i = 0; i < (bf16 ? 1 : 2); ++i)
            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                         : "=r"(r.w[i].x), "=r"(r.w[i].y), "=r"(r.w[i].z), "=r"(r.w[i].w)
                         : "r"((bf16 ? own : across) + (c * P + piece) * step + i * 16));
    };
    // v = f(v, line) with a line's values, which all chunks load together.
    auto with_line = [&](const void* p, long long at, auto& v, auto f) {
        if (!p) return;
        Raw8<LB> raw[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) raw[c] = load8<LB>(p, at + column(c));
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            Two w[4];
            pairs_of(raw[c], w);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] = f(v[c][i], w[i]);
        }
    };
    const auto times = [](Two v, Two w) { return mul2(v, w); };
    const auto plus = [](Two v, Two w) { return add2(v, w); };
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
        asm volatile("cp.async.wait_group 0;" ::: "memory");
        if (!XB || !BB) __syncwarp();
        uint32_t(*const words)[W] = slots[row % 2];
        Two h[CH][4], r[CH][4];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            Raw8<XB> x;
            landed(c, 0, x);
            pairs_of(x, h[c]);
        }
        if (A.branch)
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                Raw8<BB> b;
                landed(c, XB ? 1 : 2, b);
                pairs_of(b, r[c]);
            }
        if (!XB || !BB) __syncwarp();
        fetch(row + 1);  // into the places just read
        auto scaled = [](auto& v, float by) {
            if (by == 1.0f) return;
#pragma unroll
            for (int c = 0; c < CH; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[c][i] = mul2(v[c][i], two(by, by));
        };
        scaled(h, A.x_factor);
        if (A.branch) {
            if (A.after != CB_NORM_NONE) {
                normalise<CH, W>(r, A.after, A.after_eps, A.inv_hidden, on, words);
                with_line(A.after_weight, e0, r, times);
                with_line(A.after_bias, e0, r, plus);
            }
            scaled(r, A.branch_factor);
            if (A.gate) {
                Raw8<LB> raw[CH];
#pragma unroll
                for (int c = 0; c < CH; ++c) raw[c] = load8<LB>(A.gate, line + column(c));
#pragma unroll
                for (int c = 0; c < CH; ++c) {
                    Two g[4];
                    pairs_of(raw[c], g);
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[c][i] = fma2(g[i], r[c][i], h[c][i]);
                }
            } else {
#pragma unroll
                for (int c = 0; c < CH; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[c][i] = add2(h[c][i], r[c][i]);
            }
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
        if (!A.out) continue;
        if (A.before != CB_NORM_NONE) {
            normalise<CH, W>(h, A.before, A.before_eps, A.inv_hidden, on, words + 2);
            with_line(A.weight, e0, h, times);
            with_line(A.bias, e0, h, plus);
        }
        with_line(A.scale, line, h, [](Two v, Two w) { return fma2(v, w, v); });
        with_line(A.shift, line, h, plus);
        const long long at = row * A.out_stride + e0;
        if (A.out_dtype == CB_E4M3) {
            float amax = 0.0f;
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
            const float s = norm_scale_of(row_reduce<W, true>(__float_as_uint(amax) & 0x7FFFFFFFu, words[4]));
            if (t == 0) reinterpret_cast<float*>(A.out_scale)[row] = s;
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
        } else if (A.out_dtype == CB_MXFP4) {
            // a block is four lanes, a word of four scales sixteen
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int e = e0 + c * threads * 8;
                float v[8], top = 0.0f;
                if (!on(c)) h[c][0] = h[c][1] = h[c][2] = h[c][3] = two(0.0f, 0.0f);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = both(h[c][i]);
                    top = mx_max_abs(top, f.x, f.y);
                }
                uint32_t most = __float_as_uint(top);
                most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
                most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
                const uint32_t scale = mx_scale_of(most);
                const float inverse = mx_inverse(scale);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 f = both(mul2(h[c][i], two(inverse, inverse)));
                    v[2 * i] = f.x, v[2 * i + 1] = f.y;
                }
                if (c + 1 < CH || e < (A.hidden + kMxBlock - 1) / kMxBlock * kMxBlock)
                    *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(A.out) + row * A.out_stride + e / 2) = scale == 255 ? 0u : mx_codes8(v);
                uint32_t w = scale << 8 * (t / 4 % 4);
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
                w |= __shfl_xor_sync(0xFFFFFFFFu, w, 8);
                const unsigned k = (unsigned)e / (kMxBlock * kMxTileBlocks);
                if (t % 16 == 0 && k < A.out_tiles)
                    *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(A.out_scale) + mx_word_at(row, k, A.out_tiles)) = w;
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
cudaError_t launch_around(AroundArgs& a, int sms, cudaStream_t s) {
    constexpr int threads = norm_threads(W), teams = W == 1 ? kWarpRows : 1;
    constexpr size_t smem = (size_t)CH * norm_pieces<XB, BB>() * 16 * threads;
    // as many CTAs as are resident together
    const int per_sm = std::max(1, std::min(norm_ctas(CH, W), (int)(224 * 1024 / (smem + 2048))));
    const unsigned long long all = (unsigned long long)sms * per_sm * teams;
    a.team_rows = (unsigned)((a.rows + all - 1) / all);
    const unsigned used = (a.rows + a.team_rows - 1) / a.team_rows;
    const auto k = around_kernel<CH, W, XB, BB, LB>;
    if (smem > 47 * 1024) {  // with the kernel's own words
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapped(k, (int)((used + teams - 1) / teams), threads, smem, s, a);
}

// The row's warps and chunks: one warp up to 1280 elements, then four, eight or sixteen with up to four chunks a thread, of which all but
// the last lie in the row.
template <bool XB, bool BB, bool LB>
cudaError_t launch_around_types(AroundArgs& a, int sms, cudaStream_t s) {
    const int n = a.hidden / 8;
    if (n <= 32) return launch_around<1, 1, XB, BB, LB>(a, sms, s);
    if (n <= 64) return launch_around<2, 1, XB, BB, LB>(a, sms, s);
    if (n <= 96) return launch_around<3, 1, XB, BB, LB>(a, sms, s);
    if (n <= 128) return launch_around<4, 1, XB, BB, LB>(a, sms, s);
    if (n <= 160) return launch_around<5, 1, XB, BB, LB>(a, sms, s);
    if (n <= 256) return launch_around<2, 4, XB, BB, LB>(a, sms, s);
    if (n <= 384) return launch_around<3, 4, XB, BB, LB>(a, sms, s);
    if (n <= 512) return launch_around<4, 4, XB, BB, LB>(a, sms, s);
    if (n <= 768) return launch_around<3, 8, XB, BB, LB>(a, sms, s);
    if (n <= 1024) return launch_around<4, 8, XB, BB, LB>(a, sms, s);
    if (n <= 1536) return launch_around<3, 16, XB, BB, LB>(a, sms, s);
    return launch_around<4, 16, XB, BB, LB>(a, sms, s);
}

template <bool LB>
cudaError_t launch_around_lines(AroundArgs& a, int sms, cudaStream_t s) {
    if (a.x_bf16) return a.branch_bf16 ? launch_around_types<true, true, LB>(a, sms, s) : launch_around_types<true, false, LB>(a, sms, s);
    return a.branch_bf16 ? launch_around_types<false, true, LB>(a, sms, s) : launch_around_types<false, false, LB>(a, sms, s);
}

}  // namespace
}  // namespace cbk
