// Internal: arguments and epilogue shared by the kernels of cb_linear_run.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/chebboost_block.h"
#include "cb_device.h"

namespace cbk {

// What the epilogue needs. The kernels copy it out of their arguments first: these stay in registers, while
// arguments would be read again behind every store.
struct LinearEpilogue {
    int M, N;              // rows, output features
    int act;
    unsigned tokens;       // rows of one sample
    int out_bf16, resid_bf16, bias_bf16, gate_bf16;
    long long out_stride, resid_stride, resid_out_stride, gate_stride;  // elements
    const float *x_scale, *w_scale;
    const void *bias, *resid, *gate;
    void *out, *resid_out;
};

// How results leave: an output alone by TMA, a hidden state with or without an output by TMA, either by the threads, or an output in
// 4 bits by the threads; kHiddenLong: kHidden for long sums of operands in 4 bits, whose warps are fewer for the sake of stages.
enum class Results { kOut, kHidden, kDirect, kQuant, kHiddenLong };

// Types of the operands.
enum class Operands { kBf16, kE4m3, kMx };

// Operands in 4 bits: a stage holds scales behind its codes, two tiles of 4 blocks (256 features) of 128 rows of x and of as many of
// w as the tile's columns touch (a multiple of 64 from a multiple of 64 on).
constexpr int kMxScales = 1024;  // bytes for 128 rows
__host__ __device__ constexpr int mx_w_tiles(int tile_n) { return (tile_n + 127) / 128; }
__host__ __device__ constexpr int mx_scale_bytes(int tile_n) { return kMxScales * (1 + mx_w_tiles(tile_n)); }
constexpr int kMxMostN = 192, kMxStepN = 64;  // columns of a tile: TMEM holds two accumulators and scales

// Warps of the epilogue: two for each quarter of the TMEM lanes, or four where the threads load and store the results themselves
// and wait for that (GB300, 8192 x 8191 x 512 bf16 with a gated fp32 hidden state: eight warps, 32 rows at once each, 282 us,
// sixteen, eight rows at once, 195).
// Operands in 4 bits, whose sums are made four times as fast: 12 and 16 (GB300, 8192 x 4608 x 1152 with GELU to bf16 with 8 warps 35.4 us,
// 12 27.3, 16 27.0; to 4 bits 12 33.3, 16 28.7).
__host__ __device__ constexpr int epi_warps(Results r, bool mx = false) {
    if (mx) return r == Results::kDirect ? 16 : r == Results::kHiddenLong ? 8 : r == Results::kQuant ? 16 : 12;
    return r == Results::kDirect ? 16 : 8;
}
// Which chunks of 32 columns of a tile are a warp's of the epilogue: its first one (`share`: the warp's place among those of its quarter of the
// lanes), the one behind chunk c, and the first one of the next tile. Outputs in 4 bits go by pairs of neighbours, three pairs for four warps, of which
// each one in turn has none; in passes over K a chunk has the same warp in every tile, as the sum of its passes is kept in one place of TMEM
// that nothing but the warp's own order guards.
__host__ __device__ constexpr int epi_first_chunk(Results r, int share) { return r == Results::kQuant ? 2 * share : share; }
__host__ __device__ constexpr int epi_chunk_behind(Results r, bool mx, int c) {
    return r != Results::kQuant ? c + epi_warps(r, mx) / 4 : c % 2 == 0 ? c + 1 : c + epi_warps(r, mx) / 2 - 1;
}
__host__ __device__ constexpr int epi_next_first_chunk(Results r, bool passes, int begin) {
    return r == Results::kQuant && !passes ? (begin + 6) % 8 : begin;
}
constexpr int kTurnBytes = 32 * 32 * 4;  // bytes of an epilogue's warp to turn sums in, or two boxes of results

struct LinearArgs {
    Results results;
    Operands operands;
    CUtensorMap x_scale_map, w_scale_map;  // kMx
    uint8_t* out_scales;                   // kQuant
    unsigned out_tiles;                    // kQuant: tiles of scales of a row of the output
    CUtensorMap x_map, w_map;
    CUtensorMap out_map, resid_map, resid_out_map;
    int whole;             // columns of results that leave by TMA; up to seven behind them by the threads
    int out_boxes;         // operands in 4 bits: boxes of an output alone, of a warp
    int ring, more_boxes;  // hidden states of chunks that a warp holds; boxes of shared memory that it needs for them besides two
    LinearEpilogue e;
    int overlap;
    int k_bytes;           // bytes of a row of x and of w
    int x_rows;            // rows of x of a slab that are loaded
    int tiles_m, tiles_n, k_blocks, stages;
    unsigned long long tokens_magic; // the same of tokens; 0 for 1
    unsigned long long group_magic;  // ceil(2^64 / (8 tiles_n)): t group_magic / 2^64 is t / (8 tiles_n) for every 32-bit t
    int tile_n;            // output columns of a tile
    int passes, pass_blocks;  // stretches of K that are summed by themselves, and their slabs
    int parts, part_blocks;   // parts of K that are tiles of their own, and their slabs
    int part_rows;            // rows of the output of a part
    unsigned withheld;        // tests only: bytes of every slab that are announced but never copied
    unsigned long long wait_ns;  // limit of every wait on a barrier
    int* status;
};

// Few rows (linear_few.cu).
struct LinearFewArgs {
    LinearEpilogue e;
    int overlap;
    int k_bytes;             // bytes of a row of x and of w
    long long x_row, w_row;  // bytes from row to row
    const void *x, *w;
};
// `shift`: rows off the 16-byte grid.
cudaError_t launch_linear_few(const LinearFewArgs& a, bool fp8, bool shift, int sms, cudaStream_t s);

// Rows copied onto a grid of 32 bytes, with zeros behind each (linear_pack.cu).
struct PackOperand {
    const char* src;
    char* dst;                  // nullptr: nothing to copy
    long long rows, stride;     // bytes from row to row of src
    int bytes;                  // of a row
    unsigned chunks;            // of 32 bytes, of a row of dst
};
struct LinearPackArgs {
    PackOperand o[2];
    unsigned blocks;            // of the first operand
    int overlap;
};
cudaError_t launch_linear_pack(LinearPackArgs& a, cudaStream_t s);

// Sums of parts of K, `parts` times [part_rows, stride] in fp32, added and taken through the epilogue (linear_join.cu).
struct LinearJoinArgs {
    LinearEpilogue e;
    int overlap, parts;
    long long part_size, stride;  // floats from part to part, and from row to row
    const float* sums;
};
cudaError_t launch_linear_join(const LinearJoinArgs& a, cudaStream_t s);

// The tensor-core kernels (linear_tc.cuh): cg CTAs per tile of 128 cg rows. prepare_linear raises the shared-memory
// limit of those for 16 and 8 bits (launch_linear, at its first use, that of those for 4) and tells how many pairs of CTAs run at once.
size_t linear_stage_bytes(int cg, int tile_n);
size_t linear_fixed_bytes(Results r, int more_boxes);  // shared memory besides the stages
constexpr int kBox = 2048, kMaxRing = 6;
constexpr int kMaxLinStages = 12;
// ...and more of it, of the kernels for operands in 4 bits
constexpr int kMxLines = 128;  // floats of a warp: twice, biases and gates of 32 columns
constexpr size_t mx_more_bytes(Results r, int more_boxes, int out_boxes) {
    return (size_t)epi_warps(r, true) * (out_boxes * kBox + more_boxes * kBox + kMxLines * 4) -
           (size_t)epi_warps(r) * (kTurnBytes + more_boxes * kBox);
}
cudaError_t prepare_linear(size_t smem, int* pairs);
using LinearKernel = void (*)(LinearArgs);
LinearKernel linear_out_kernel(int cg, bool fp8, bool passes);     // linear_tc_out.cu
LinearKernel linear_hidden_kernel(int cg, bool fp8, bool passes);  // linear_tc_hidden.cu
LinearKernel linear_direct_kernel(int cg, bool fp8, bool passes);  // linear_tc_direct.cu
LinearKernel linear_mx_kernel(Results r, int cg, bool passes);     // linear_tc_mx.cu
cudaError_t launch_linear(const LinearArgs& a, int cg, bool fp8, int grid, cudaStream_t s);

#ifdef __CUDACC__
namespace {

// The epilogue with pointers that the compiler knows nothing of before this place, behind the wait for the previous kernel: no load
// through them is moved ahead of it.
__device__ __forceinline__ LinearEpilogue from_here(LinearEpilogue e) {
    asm volatile("" : "+l"(e.x_scale), "+l"(e.w_scale), "+l"(e.bias), "+l"(e.resid), "+l"(e.gate));
    return e;
}

__device__ __forceinline__ uint32_t bf16x2(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

// Loads that no store of the kernel is ordered against: inputs do not overlap outputs, and a hidden state that is
// updated in place is read by the thread that writes it.
// One element as fp32 bits, or its half of them. Not volatile, as the compiler then keeps such loads, and the branches between them, in
// line (GB300, 8192 x 8191 x 512 with a fp32 hidden state 146 -> 156 us, 256 x 1152 x 4608 in parts of K 11.4 -> 12.3): the
// epilogue's pointers come from from_here instead.
__device__ __forceinline__ uint32_t lin_raw1(const void* p, long long e, int bf16) {  // (bf16 in the lower half)
    uint32_t r;
    if (bf16) asm("ld.global.u16 %0, [%1];" : "=r"(r) : "l"(reinterpret_cast<const uint16_t*>(p) + e));
    else asm("ld.global.u32 %0, [%1];" : "=r"(r) : "l"(reinterpret_cast<const uint32_t*>(p) + e));
    return r;
}
__device__ __forceinline__ uint32_t lin_ld1(const void* p, long long e, int bf16) {
    const uint32_t r = lin_raw1(p, e, bf16);
    return bf16 ? r << 16 : r;
}

__device__ __forceinline__ void lin_put1(void* p, long long e, int bf16, float v) {
    if (bf16)
        reinterpret_cast<__nv_bfloat16*>(p)[e] = __float2bfloat16_rn(v);
    else
        reinterpret_cast<float*>(p)[e] = v;
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

// v / (1 + 2^t): SiLU with t = -v log2(e), the tanh form of GELU with t = -2 log2(e) sqrt(2/pi) (v + 0.044715 v^3),
// since (1 + tanh(z)) / 2 = 1 / (1 + exp(-2 z)). At -infinity it is NaN, as the quotients are.
template <int ACT>
__device__ __forceinline__ Two lin_denominators(Two v) {
    constexpr float kSilu = -1.44269504f, kGelu1 = -2.30220820f, kGelu3 = -0.102943239f;
    float2 t = both(ACT == CB_ACT_SILU ? mul2(v, two(kSilu, kSilu))
                                       : mul2(v, fma2(two(kGelu3, kGelu3), mul2(v, v), two(kGelu1, kGelu1))));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t.x));
    asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t.y));
    return add2(two(t.x, t.y), two(1.0f, 1.0f));
}
__device__ __forceinline__ float lin_reciprocal(float d) {
    asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(d));
    return d;
}
template <int ACT>
__device__ __forceinline__ Two lin_act(Two v) {
    if constexpr (ACT == CB_ACT_NONE) return v;
    const float2 d = both(lin_denominators<ACT>(v));
    return mul2(v, two(lin_reciprocal(d.x), lin_reciprocal(d.y)));
}

// The same for N pairs, with one reciprocal of four denominators' product, for epilogues that wait for the unit for special
// functions. Where a product passes 2^120 (four values of t = 30: SiLU at -20.8, GELU at -5.7; or one of 120), or one of its values is a NaN,
// all pairs are made anew with a reciprocal each. Asked for once for all of them: a branch for every four values keeps them from
// being worked on together (GB300, 4096 x 4608 x 1152 e4m3 with GELU, 10 % longer), and where results leave by the threads,
// which wait for loads, a branch costs more than the reciprocals (999 x 1155 x 577 SiLU, fp32 hidden state: 11.9 us as above, 12.7 so).
template <int ACT, int N>
__device__ __forceinline__ void lin_act_all(Two* x) {
    if constexpr (ACT != CB_ACT_NONE) {
        static_assert(N % 2 == 0, "two pairs at a time");
        constexpr float kMost = 1.32922800e36f;  // 2^120
        Two y[N];
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            const Two a = lin_denominators<ACT>(x[i]), b = lin_denominators<ACT>(x[i + 1]);
            const float2 p = both(mul2(a, b));
            float r = p.x * p.y;
            asm("max.NaN.f32 %0, %0, %1;" : "+f"(most) : "f"(r));
            r = lin_reciprocal(r);
            const Two q = mul2(two(r, r), two(p.y, p.x));  // 1 / (a b), pair by pair
            y[i] = mul2(x[i], mul2(q, b));
            y[i + 1] = mul2(x[i + 1], mul2(q, a));
        }
        if (!(most <= kMost)) {
#pragma unroll
            for (int i = 0; i < N; ++i) y[i] = lin_act<ACT>(x[i]);
        }
#pragma unroll
        for (int i = 0; i < N; ++i) x[i] = y[i];
    }
}

}  // namespace
#endif

}  // namespace cbk
