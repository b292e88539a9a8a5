// cb_norm_around: the norm after a branch, its addition to the hidden state, and the norm before the next branch.
//
// Bound by HBM: a row is read once and written once, and stays on the SM between its reductions: in registers where it is reached by
// vectors (norm_around_rows.cuh) and up to 8192 elements where it is not, else in shared memory (below). A layer norm takes two of them, one after the other:
// the squares of what is left when the mean is off lose nothing where the mean is far larger than the deviation, as sums of squares
// less the mean's square do. GB300, gate and modulation: 16384 x 4096 bf16 97 us (82 % of the copy rate), 8192 x 1152 to 4 bits 16.5, to bf16 16.1; fp32
// stream, branch normed too, to e4m3 25 us; by elements 8192 x 4097 86 us, 16384 x 1153 to bf16 44, to 4 bits 50, x 250 13.
#include <cmath>

#include "norm_around.cuh"

namespace cbk {
namespace {

constexpr int kAroundHeld = 49152;  // elements of a row in shared memory

// Pieces t, t + T, ... of V elements (one, or two on their grid) of a row from p on. The first FULL lie in every row that the kernel is launched
// for, at places that the compiler knows: a select and an address for each of them took a third of the kernel's instructions. Threads behind the
// row's end read its start.
template <int CH, int T, int FULL, int V>
__device__ __forceinline__ void load_row(const void* p, long long e, int bf16, int t, int hidden, float* v) {
    auto at = [&](int c) { return c < FULL || (c * T + t) * V < hidden ? c * T : -t; };
    if (bf16) {
        const uint16_t* const q = reinterpret_cast<const uint16_t*>(p) + e + t * V;
        if constexpr (V == 2) {
            uint32_t w[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) w[c] = reinterpret_cast<const uint32_t*>(q)[at(c)];
#pragma unroll
            for (int c = 0; c < CH; ++c) v[2 * c] = __uint_as_float(w[c] << 16), v[2 * c + 1] = __uint_as_float(w[c] & 0xFFFF0000u);
        } else {
            uint16_t w[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) w[c] = q[at(c)];
#pragma unroll
            for (int c = 0; c < CH; ++c) v[c] = __uint_as_float((uint32_t)w[c] << 16);
        }
    } else {
        const float* const q = reinterpret_cast<const float*>(p) + e + t * V;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            if constexpr (V == 2) {
                const float2 f = reinterpret_cast<const float2*>(q)[at(c)];
                v[2 * c] = f.x, v[2 * c + 1] = f.y;
            } else {
                v[c] = q[at(c)];
            }
        }
    }
}
template <int CH, int T, int V>
__device__ __forceinline__ void store_row(void* p, long long e, int dtype, int t, int hidden, const float* v) {
    if constexpr (V == 1) {
        store_all<CH, T>(p, e, dtype, t, hidden, v);
    } else if (dtype == CB_BF16) {
        uint32_t* const q = reinterpret_cast<uint32_t*>(reinterpret_cast<uint16_t*>(p) + e) + t;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if ((c * T + t) * 2 < hidden) q[c * T] = norm_bf16x2(v[2 * c], v[2 * c + 1]);
    } else if (dtype == CB_FP32) {
        float2* const q = reinterpret_cast<float2*>(reinterpret_cast<float*>(p) + e) + t;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if ((c * T + t) * 2 < hidden) q[c * T] = make_float2(v[2 * c], v[2 * c + 1]);
    } else {
        uint16_t* const q = reinterpret_cast<uint16_t*>(reinterpret_cast<uint8_t*>(p) + e) + t;
#pragma unroll
        for (int c = 0; c < CH; ++c)
            if ((c * T + t) * 2 < hidden) q[c * T] = (uint16_t)norm_e4m3x2(v[2 * c], v[2 * c + 1]);
    }
}

// A row by elements, in registers: CH pieces of V of them in each thread of its W warps. Short rows have a warp each, four to a CTA: there is nothing to wait
// for but the row's own loads, and a CTA is launched for four rows (17300 x 220 one by one, layer norms, to fp32: 11.7 us, with four warps a row 25.9).
// Their lines, and those of many rows above 640 elements, are loaded when they are wanted, which leaves registers for more warps (220 elements 18.3 us
// with the lines loaded early, 16384 x 1153 to 4 bits 93 instead of 51); four warps and up to 640 elements, and 16 and 32 warps of few rows, load them with
// the row, as such rows are bound by their loads' time (999 x 577 4.8 us; a warp each, late, 6.9).
constexpr int kHeldRows = 4;  // warps of a CTA whose rows have a warp each
// (CH: elements of a thread)
__host__ __device__ constexpr int held_rows(int W) { return W == 1 ? kHeldRows : 1; }
__host__ __device__ constexpr bool around_early(int CH, int W) { return W > 1 && (CH * W <= 24 || (CH <= 4 && W >= 16)); }
// CTAs of an SM, by the registers that this leaves a thread: 40 for ten elements, 64 for sixteen, 80 for twenty.
__host__ __device__ constexpr int around_ctas(int CH, int W) {
    if (around_early(CH, W)) return 0;
    if (W == 1) return CH <= 4 ? 12 : CH <= 8 ? 8 : 6;
    if (W == 4) return 8;
    return (CH <= 10 ? 1536 : CH <= 16 ? 1024 : 768) / (32 * W);
}

template <int CH, int W, int FULL, int V>
__global__ void __launch_bounds__(32 * W * held_rows(W), around_ctas(CH * V, W)) around_held_kernel(const __grid_constant__ AroundArgs args) {
    __shared__ uint32_t slots[5][W];
    constexpr int T = 32 * W, N = CH * V;
    constexpr bool EARLY = around_early(CH * V, W);
    const AroundArgs A = args;  // in registers, as stores would have them read again
    after_previous();
    const unsigned row = W == 1 ? blockIdx.x * kHeldRows + threadIdx.x / T : blockIdx.x;
    const int t = threadIdx.x % T;
    if (W == 1 && row >= A.rows) return;
    auto on = [&](int i) { return i / V < FULL || (i / V * T + t) * V < A.hidden; };  // its element i
    const long long line = (long long)(row / A.tokens) * A.line_stride;
    float early[7][CH * V];
    auto look = [&](int i, const void* p, long long at) {
        if (EARLY && p) load_row<CH, T, FULL, V>(p, at, A.param_bf16, t, A.hidden, early[i]);
    };
    // v = f(v, line), of line i at p
    auto with_line = [&](int i, const void* p, long long at, float (&v)[CH * V], auto f) {
        if (!p) return;
        float late[CH * V];
        if (!EARLY) load_row<CH, T, FULL, V>(p, at, A.param_bf16, t, A.hidden, late);
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] = f(v[c], EARLY ? early[i][c] : late[c]);
    };
    auto normalise = [&](float (&v)[CH * V], int kind, float eps, uint32_t (*s)[W]) {
        if (kind == CB_NORM_LAYER) {
            float sum = 0.0f;
#pragma unroll
            for (int c = 0; c < N; ++c)
                if (on(c)) sum += v[c];
            const float mean = __uint_as_float(row_reduce<W, false>(__float_as_uint(sum), s[0])) * A.inv_hidden;
#pragma unroll
            for (int c = 0; c < N; ++c) v[c] -= mean;
        }
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < N; ++c)
            if (on(c)) sum = fmaf(v[c], v[c], sum);
        sum = __uint_as_float(row_reduce<W, false>(__float_as_uint(sum), s[1]));
        const float rstd = 1.0f / sqrtf(fmaf(sum, A.inv_hidden, eps));
#pragma unroll
        for (int c = 0; c < N; ++c) v[c] *= rstd;
    };
    const auto times = [](float v, float w) { return v * w; };
    const auto plus = [](float v, float w) { return v + w; };
    float h[CH * V], r[CH * V];
    load_row<CH, T, FULL, V>(A.x, row * A.x_stride, A.x_bf16, t, A.hidden, h);
    if (A.branch) load_row<CH, T, FULL, V>(A.branch, row * A.branch_stride, A.branch_bf16, t, A.hidden, r);
    look(0, A.after_weight, 0);
    look(1, A.after_bias, 0);
    look(2, A.gate, line);
    look(3, A.weight, 0);
    look(4, A.bias, 0);
    look(5, A.scale, line);
    look(6, A.shift, line);
    if (A.x_factor != 1.0f) {
#pragma unroll
        for (int c = 0; c < N; ++c) h[c] *= A.x_factor;
    }
    if (A.branch) {
        if (A.after != CB_NORM_NONE) {
            normalise(r, A.after, A.after_eps, slots);
            with_line(0, A.after_weight, 0, r, times);
            with_line(1, A.after_bias, 0, r, plus);
        }
        with_line(2, A.gate, line, r, times);
#pragma unroll
        for (int c = 0; c < N; ++c) h[c] = fmaf(r[c], A.branch_factor, h[c]);
    }
    if (A.x_out) store_row<CH, T, V>(A.x_out, row * A.x_out_stride, A.x_bf16 ? CB_BF16 : CB_FP32, t, A.hidden, h);
    if (!A.out) return;
    if (A.before != CB_NORM_NONE) {
        normalise(h, A.before, A.before_eps, slots + 2);
        with_line(3, A.weight, 0, h, times);
        with_line(4, A.bias, 0, h, plus);
    }
    with_line(5, A.scale, line, h, [](float v, float w) { return fmaf(v, w, v); });
    with_line(6, A.shift, line, h, plus);
    if (A.out_dtype == CB_MXFP4) {
        // Through shared memory to eight consecutive elements of a thread, so that a block is four lanes and a word of scales sixteen
        // (a block as a warp, a code by every other lane, took four times the instructions). Zeros fill up the last tile of scales.
        extern __shared__ __align__(16) float turned_rows[];
        const int ends = (int)A.out_tiles * kMxTileBlocks * kMxBlock;
        float* const turned = turned_rows + (W == 1 ? threadIdx.x / T * ends : 0);
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const int e = (c / V * T + t) * V + c % V;
            if (e < ends) turned[e] = on(c) ? h[c] : 0.0f;
        }
        for (int e = N * T + t; e < ends; e += T) turned[e] = 0.0f;
        if (W == 1) __syncwarp();
        else __syncthreads();
        for (int first = t / 32 * 256; first < ends; first += T * 8) {  // (of the warp; it ends with a word of scales, sixteen lanes)
            const int e = first + t % 32 * 8;
            float v[8] = {}, top = 0.0f;
            if (e < ends) {
                *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(turned + e);
                *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(turned + e + 4);
            }
#pragma unroll
            for (int i = 0; i < 8; i += 2) top = mx_max_abs(top, v[i], v[i + 1]);
            uint32_t most = __float_as_uint(top);
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
            most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
            const uint32_t scale = mx_scale_of(most);
            const float inverse = mx_inverse(scale);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= inverse;
            if (e < (A.hidden + kMxBlock - 1) / kMxBlock * kMxBlock)
                *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(A.out) + row * A.out_stride + e / 2) = scale == 255 ? 0u : mx_codes8(v);
            uint32_t w = scale << 8 * (t / 4 % 4);
            w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
            w |= __shfl_xor_sync(0xFFFFFFFFu, w, 8);
            if (t % 16 == 0 && e < ends)
                *reinterpret_cast<uint32_t*>(reinterpret_cast<uint8_t*>(A.out_scale) + mx_word_at(row, e / (kMxBlock * kMxTileBlocks), A.out_tiles)) = w;
        }
        return;
    }
    if (A.out_dtype == CB_E4M3) {
        float amax = 0.0f;
#pragma unroll
        for (int c = 0; c < N; ++c)
            if (on(c)) amax = max_abs(amax, h[c]);
        const float s = norm_scale_of(row_reduce<W, true>(__float_as_uint(amax) & 0x7FFFFFFFu, slots[4]));
        if (t == 0) reinterpret_cast<float*>(A.out_scale)[row] = s;
        const float inv = __frcp_rn(s);
#pragma unroll
        for (int c = 0; c < N; ++c) h[c] *= inv;
    }
    store_row<CH, T, V>(A.out, row * A.out_stride, A.out_dtype, t, A.hidden, h);
}

// Longer rows by elements; HELD: in shared memory, else read again for each reduction.
template <int W, bool HELD>
__global__ void __launch_bounds__(32 * W) around_elements_kernel(const __grid_constant__ AroundArgs args) {
    __shared__ uint32_t slots[5][W];
    extern __shared__ float held[];
    constexpr unsigned T = 32 * W;
    const AroundArgs A = args;  // in registers, as stores would have them read again
    after_previous();
    const unsigned row = blockIdx.x, n = (unsigned)A.hidden, t = threadIdx.x;
    const long long line = (long long)(row / A.tokens) * A.line_stride;
    const long long xo = row * A.x_stride, bo = row * A.branch_stride;
    auto at_line = [&](const void* p, long long e, float none) { return p ? value_at(p, e, A.param_bf16) : none; };
    auto sum_of = [&](uint32_t* s, auto f) {  // over the row; each thread has the same elements in all of them
        float sum = 0.0f;
#pragma unroll 4
        for (unsigned e = t; e < n; e += T) sum += f(e);
        return __uint_as_float(row_reduce<W, false>(__float_as_uint(sum), s));
    };
    // (v - mean) rstd of the values f(e)
    auto moments = [&](int kind, float eps, uint32_t (*s)[W], auto f, float* mean, float* rstd) {
        *mean = kind == CB_NORM_LAYER ? sum_of(s[0], f) * A.inv_hidden : 0.0f;
        const float off = *mean;
        const float squares = sum_of(s[1], [&](unsigned e) {
            const float v = f(e) - off;
            return v * v;
        });
        *rstd = 1.0f / sqrtf(fmaf(squares, A.inv_hidden, eps));
    };
    float after_mean = 0.0f, after_rstd = 1.0f, mean = 0.0f, rstd = 1.0f;
    auto branch_at = [&](unsigned e) { return value_at(A.branch, bo + e, A.branch_bf16); };
    auto hidden_of = [&](float b, unsigned e) {
        const float x = value_at(A.x, xo + e, A.x_bf16) * A.x_factor;
        if (!A.branch) return x;
        if (A.after != CB_NORM_NONE)
            b = (b - after_mean) * after_rstd * at_line(A.after_weight, e, 1.0f) + at_line(A.after_bias, e, 0.0f);
        return fmaf(b * at_line(A.gate, line + e, 1.0f), A.branch_factor, x);
    };
    if (A.after != CB_NORM_NONE) {
        if constexpr (HELD) {
#pragma unroll 4
            for (unsigned e = t; e < n; e += T) held[e] = branch_at(e);
            moments(A.after, A.after_eps, slots, [&](unsigned e) { return held[e]; }, &after_mean, &after_rstd);
        } else {
            moments(A.after, A.after_eps, slots, branch_at, &after_mean, &after_rstd);
        }
    }
    auto made = [&](unsigned e) {
        return hidden_of(HELD && A.after != CB_NORM_NONE ? held[e] : A.branch ? branch_at(e) : 0.0f, e);
    };
    auto put_x = [&](unsigned e, float h) {
        if (A.x_out) put(A.x_out, row * A.x_out_stride + e, A.x_bf16 ? CB_BF16 : CB_FP32, h);
    };
    if constexpr (HELD) {
#pragma unroll 4
        for (unsigned e = t; e < n; e += T) {
            const float h = made(e);
            held[e] = h;
            put_x(e, h);
        }
    }
    auto hidden = [&](unsigned e) { return HELD ? held[e] : made(e); };
    if (A.out && A.before != CB_NORM_NONE) moments(A.before, A.before_eps, slots + 2, hidden, &mean, &rstd);
    auto normed = [&](float h, unsigned e) {
        float y = h;
        if (A.before != CB_NORM_NONE) y = (h - mean) * rstd * at_line(A.weight, e, 1.0f) + at_line(A.bias, e, 0.0f);
        if (A.scale) y = fmaf(y, value_at(A.scale, line + e, A.param_bf16), y);
        return A.shift ? y + value_at(A.shift, line + e, A.param_bf16) : y;
    };
    float inv = 1.0f;
    if (A.out && A.out_dtype == CB_E4M3) {
        float amax = 0.0f;
#pragma unroll 4
        for (unsigned e = t; e < n; e += T) amax = max_abs(amax, normed(hidden(e), e));
        const float s = norm_scale_of(row_reduce<W, true>(__float_as_uint(amax) & 0x7FFFFFFFu, slots[4]));
        if (t == 0) reinterpret_cast<float*>(A.out_scale)[row] = s;
        inv = __frcp_rn(s);
    }
    if (A.out && A.out_dtype == CB_MXFP4) {
        // a block is a warp; those that fill up the last tile of scales are zeros
        uint8_t* const out = reinterpret_cast<uint8_t*>(A.out) + row * A.out_stride;
        const unsigned ends = A.out_tiles * kMxTileBlocks * kMxBlock, codes_end = (n + kMxBlock - 1) / kMxBlock * kMxBlock;
        for (unsigned e = t; e < ends; e += T) {
            float y = 0.0f;
            if (e < n) {
                const float h = hidden(e);
                if (!HELD) put_x(e, h);
                y = normed(h, e);
            }
            const uint32_t scale = mx_scale_of(__reduce_max_sync(0xFFFFFFFFu, __float_as_uint(y) & 0x7FFFFFFFu));
            y *= mx_inverse(scale);
            const float v[8] = {y, __shfl_down_sync(0xFFFFFFFFu, y, 1)};
            if (t % 2 == 0 && e < codes_end) out[e / 2] = scale == 255 ? 0 : (uint8_t)mx_codes8(v);
            const unsigned block = e / kMxBlock;
            if (t % 32 == 0)
                reinterpret_cast<uint8_t*>(A.out_scale)[mx_word_at(row, block / kMxTileBlocks, A.out_tiles) + block % kMxTileBlocks] = (uint8_t)scale;
        }
        return;
    }
    if (HELD && !A.out) return;
    for (unsigned e = t; e < n; e += T) {
        const float h = hidden(e);
        if (!HELD) put_x(e, h);
        if (A.out) put(A.out, row * A.out_stride + e, A.out_dtype, normed(h, e) * inv);
    }
}

template <int CH, int W, int FULL, int V>
cudaError_t launch_held(const AroundArgs& a, cudaStream_t s) {
    constexpr int rows = held_rows(W);
    // (33 KB at most)
    const size_t smem = a.out && a.out_dtype == CB_MXFP4 ? (size_t)a.out_tiles * kMxTileBlocks * kMxBlock * 4 * rows : 0;
    return launch_overlapped(around_held_kernel<CH, W, FULL, V>, (int)((a.rows + rows - 1) / rows), 32 * W * rows, smem, s, a);
}
template <int W, bool HELD>
cudaError_t launch_elements(const AroundArgs& a, cudaStream_t s) {
    const auto k = around_elements_kernel<W, HELD>;
    const size_t smem = HELD ? (size_t)a.hidden * 4 : 0;
    if (smem > 47 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    return launch_overlapped(k, (int)a.rows, 32 * W, smem, s, a);
}

// Rows of up to 8192 elements, by V at a time: pairs where all rows have them, 16384 x 300 17.5 -> 14.9 us, x 1276 55 -> 45, 8192 x 3380 86 -> 72.
template <int V>
cudaError_t launch_held_row(const AroundArgs& a, int sms, cudaStream_t s) {
    const int n = a.hidden;
    // A warp a row up to 256 elements (250: 1000 rows 4.4 us, four warps 5.7; 16384 rows 12.9 and 28.8), and up to 768 where the rows are more
    // than CTAs of four warps fit on the SMs, 12 on each (577: 1000 rows 6.9, four warps 4.8; 1500 rows 7.1 and 7.2; 3000 rows 7.4 and 10.3;
    // 16384 rows 29 and 49; 16384 x 700 34 and 47, x 801 44 and 47, x 1153 59 and 54).
    if (n <= 256 || (n <= 768 && a.rows > 12u * sms)) {
        if (n <= 64) return launch_held<2 / V, 1, 0 / V, V>(a, s);
        if (n <= 128) return launch_held<4 / V, 1, 2 / V, V>(a, s);
        if (n <= 192) return launch_held<6 / V, 1, 4 / V, V>(a, s);
        if (n <= 256) return launch_held<8 / V, 1, 6 / V, V>(a, s);
        if (n <= 384) return launch_held<12 / V, 1, 8 / V, V>(a, s);
        if (n <= 512) return launch_held<16 / V, 1, 12 / V, V>(a, s);
        if (n <= 640) return launch_held<20 / V, 1, 16 / V, V>(a, s);
        return launch_held<24 / V, 1, 20 / V, V>(a, s);
    }
    if (n <= 384) return launch_held<(2 + V) / V, 4, 2 / V, V>(a, s);
    if (n <= 640) return launch_held<(4 + V) / V, 4, 3 / V, V>(a, s);
    // few long rows by as many warps as an SM has room for, lines early: 300 x 2047 7.4 -> 5.1 us (310 rows 7.6, with four warps each), 150 x 3383 8.1 -> 5.6
    // (300 rows 8.1, with eight)
    if (n > 1280 && n <= 2048 && a.rows <= 2u * sms) return launch_held<4 / V, 16, 2 / V, V>(a, s);
    if (n > 2048 && n <= 4096 && a.rows <= 1u * sms) return launch_held<4 / V, 32, 2 / V, V>(a, s);
    // as few warps as hold the row: twice as many with half the elements each took 8192 x 2047 from 45 to 52 us, x 3383 from 88 to 106, x 5001
    // from 114 to 121; half as many with twice the elements 8192 x 2047 to 49, x 4095 from 92 to 94, x 7001 from 193 to 199
    if (n <= 1024) return launch_held<8 / V, 4, 5 / V, V>(a, s);
    if (n <= 1280) return launch_held<10 / V, 4, 8 / V, V>(a, s);
    if (n <= 2048) return launch_held<16 / V, 4, 10 / V, V>(a, s);
    if (n <= 2560) return launch_held<10 / V, 8, 8 / V, V>(a, s);
    if (n <= 4096) return launch_held<16 / V, 8, 10 / V, V>(a, s);
    if (n <= 5120) return launch_held<20 / V, 8, 16 / V, V>(a, s);
    if (n <= 6144) return launch_held<12 / V, 16, 10 / V, V>(a, s);
    return launch_held<16 / V, 16, 10 / V, V>(a, s);
}

cudaError_t launch_row(AroundArgs& a, bool vec, bool pairs, int sms, cudaStream_t s) {
    const int n = a.hidden;
    if (vec && n <= 16384) return a.param_bf16 ? launch_around_bf16_lines(a, sms, s) : launch_around_fp32_lines(a, sms, s);
    if (n <= 8192) return pairs ? launch_held_row<2>(a, sms, s) : launch_held_row<1>(a, sms, s);
    if (n <= kAroundHeld) return launch_elements<16, true>(a, s);
    return launch_elements<16, false>(a, s);
}

size_t bytes_of(int dtype) { return dtype == CB_BF16 ? 2 : dtype == CB_FP32 ? 4 : 1; }
bool on_grid(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

}  // namespace
}  // namespace cbk

extern "C" int cb_norm_around(const cb_norm_around_desc* d, const void* x, const void* branch, const void* gate,
                              const void* after_weight, const void* after_bias, const void* weight, const void* bias,
                              const void* scale, const void* shift, void* x_out, void* out, void* out_scale, void* stream) {
    using namespace cbk;
    auto wide = [](cb_dtype t) { return t == CB_BF16 || t == CB_FP32; };
    auto kind = [](int32_t k) { return k >= CB_NORM_NONE && k <= CB_NORM_LAYER; };
    auto eps = [](float e) { return e >= 0.0f && std::isfinite(e); };
    if (!d || d->reserved != 0 || d->rows < 0 || d->hidden < 1 || d->tokens < 0) return CB_ERR_ARG;
    if (!wide(d->x_dtype) || !wide(d->branch_dtype) || !wide(d->param_dtype)) return CB_ERR_ARG;
    const bool mx = d->out_dtype == CB_MXFP4, scaled = mx || d->out_dtype == CB_E4M3;
    if (!wide(d->out_dtype) && !scaled) return CB_ERR_ARG;
    if (!kind(d->after) || !kind(d->before) || !eps(d->after_eps) || !eps(d->before_eps)) return CB_ERR_ARG;
    if (!std::isfinite(d->x_factor) || !std::isfinite(d->branch_factor)) return CB_ERR_ARG;
    if (d->rows > 0x7FFFFFFFLL || d->hidden > 0x7FFFFF00LL) return CB_ERR_LIMIT;
    const int64_t strides[] = {d->x_stride, d->branch_stride, d->x_out_stride, d->out_stride, d->line_stride};
    for (int64_t s : strides)
        if (s != 0 && (s < d->hidden || s > CB_MAX_NUMEL)) return s < d->hidden ? CB_ERR_ARG : CB_ERR_LIMIT;
    const long long blocks = mx_blocks(d->hidden);
    if (mx && d->out_stride != 0 && (d->out_stride < blocks * kMxBlock || d->out_stride % kMxBlock != 0)) return CB_ERR_ARG;
    if (d->rows == 0) return CB_OK;
    if (!x || (!out && !x_out) || (scaled && out) != (out_scale != nullptr)) return CB_ERR_ARG;
    if (!branch && (gate || d->after != CB_NORM_NONE)) return CB_ERR_ARG;
    if (d->after == CB_NORM_NONE && (after_weight || after_bias)) return CB_ERR_ARG;
    if (d->before == CB_NORM_NONE && (weight || bias)) return CB_ERR_ARG;
    if (!out && (weight || bias || scale || shift)) return CB_ERR_ARG;
    AroundArgs a{};
    a.overlap = 1;
    a.rows = (unsigned)d->rows;
    a.hidden = (int)d->hidden;
    a.tokens = d->tokens == 0 || d->tokens > d->rows ? a.rows : (unsigned)d->tokens;
    a.x_stride = d->x_stride ? d->x_stride : d->hidden;
    a.branch_stride = d->branch_stride ? d->branch_stride : d->hidden;
    a.x_out_stride = d->x_out_stride ? d->x_out_stride : d->hidden;
    a.out_stride = mx ? (d->out_stride ? d->out_stride : blocks * kMxBlock) / 2 : d->out_stride ? d->out_stride : d->hidden;
    a.line_stride = d->line_stride ? d->line_stride : d->hidden;
    a.x = x, a.branch = branch, a.gate = gate, a.after_weight = after_weight, a.after_bias = after_bias;
    a.weight = weight, a.bias = bias, a.scale = scale, a.shift = shift;
    a.x_out = x_out, a.out = out, a.out_scale = out_scale;
    a.after = d->after, a.before = d->before, a.after_eps = d->after_eps, a.before_eps = d->before_eps;
    a.x_factor = d->x_factor, a.branch_factor = d->branch_factor;
    a.inv_hidden = (float)(1.0 / (double)d->hidden);
    a.x_bf16 = d->x_dtype == CB_BF16;
    a.branch_bf16 = d->branch_dtype == CB_BF16;
    a.param_bf16 = d->param_dtype == CB_BF16;
    a.out_dtype = d->out_dtype;
    a.out_tiles = (unsigned)mx_tiles_k(d->hidden);
    // a pointer, its element size and the stride behind it (rows start on the grid too)
    const struct {
        const void* p;
        int dtype;
        long long stride;
    } used[] = {{x, d->x_dtype, a.x_stride},            {branch, d->branch_dtype, a.branch_stride},
                {gate, d->param_dtype, a.line_stride},  {after_weight, d->param_dtype, 0},
                {after_bias, d->param_dtype, 0},        {weight, d->param_dtype, 0},
                {bias, d->param_dtype, 0},              {scale, d->param_dtype, a.line_stride},
                {shift, d->param_dtype, a.line_stride}, {x_out, d->x_dtype, a.x_out_stride},
                {mx ? nullptr : out, d->out_dtype, a.out_stride}};
    bool vec = d->hidden % 8 == 0, pairs = d->hidden % 2 == 0;
    for (const auto& u : used) {
        const size_t es = bytes_of(u.dtype), grid = es == 1 ? 8 : 16;
        if (!u.p) continue;
        if (!on_grid(u.p, es)) return CB_ERR_ALIGN;
        vec = vec && on_grid(u.p, grid) && (size_t)u.stride * es % grid == 0;
        pairs = pairs && on_grid(u.p, 2 * es) && u.stride % 2 == 0;
    }
    if (mx && (!on_grid(out, 16) || !on_grid(out_scale, 16))) return CB_ERR_ALIGN;
    if (!on_grid(out_scale, 4)) return CB_ERR_ALIGN;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e == cudaSuccess) e = launch_row(a, vec, pairs, sms, (cudaStream_t)stream);
    return e == cudaSuccess ? CB_OK : cuda_error(e, "norm launch");
}
