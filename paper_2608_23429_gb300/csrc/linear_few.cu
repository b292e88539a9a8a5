// The matrix product of cb_linear_run for few rows of x: bound by the bytes of w, each read once.
//
// A CTA makes 16 columns for all 8 NT rows (32 at most). Its eight warps, and the CTAs of its cluster, take turns of 64 bytes of K. The
// rows of w are the 16-row operand of mma.sync, so that no row of the tensor cores is wasted on rows that x does not
// have, and fragments come from global memory without a stop in shared memory: a lane's 16 consecutive bytes of a
// row stand for other places of K than the instruction's, but for the same ones in both operands, and a sum does not
// mind. e4m3 is widened to fp16 (exact), whose products the tensor cores sum in fp32. They cut off what a sum loses (65536 features of
// one sign in one such sum a warp: 3e-5 of it), so each of a warp's batches of loads, 128 features of bf16 at most, is summed by itself
// and added rounded to nearest. The partial sums of warps and CTAs are added in a fixed order.
#include <cuda_fp16.h>

#include "linear.cuh"
#include "linear_shift.cuh"

namespace cbk {
namespace {

constexpr int kWarps = 8;
constexpr int kTurn = 64;   // bytes of K of a warp's turn
constexpr int kDeep = 4;    // turns whose loads are in flight together

__device__ __forceinline__ void mma_bf16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_fp16(float* d, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Four e4m3 values as two pairs of fp16.
__device__ __forceinline__ uint2 widen(uint32_t v) {
    uint2 r;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r.x) : "h"((uint16_t)v));
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r.y) : "h"((uint16_t)(v >> 16)));
    return r;
}

template <bool FP8>
__device__ __forceinline__ void product(float* d, const uint4& lo, const uint4& hi, const uint4& x) {
    if constexpr (!FP8) {
        mma_bf16(d, lo.x, hi.x, lo.y, hi.y, x.x, x.y);
        mma_bf16(d, lo.z, hi.z, lo.w, hi.w, x.z, x.w);
    } else {
        const uint32_t l[4] = {lo.x, lo.y, lo.z, lo.w}, h[4] = {hi.x, hi.y, hi.z, hi.w}, y[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint2 a = widen(l[i]), b = widen(h[i]), c = widen(y[i]);
            mma_fp16(d, a.x, b.x, a.y, b.y, c.x, c.y);
        }
    }
}

// A row of an operand, seen by one lane: its 16 bytes of every turn.
struct Line {
    const char *at, *from, *to;  // the lane's place in the row, and the operand's first and last bytes
    bool on;
};

// How rows lie: on 16-byte boundaries and made of whole pieces, on them with a last piece that is not whole, or off them. The kernel for
// the second is one of its own, as the last pieces' bytes take registers from the loads in flight.
enum FewRows { kWhole, kTail, kShift };

// Its 16 bytes `k` bytes on, of which `left` belong to the row; zeros behind them. kTail: zeros for a piece that is not whole, which
// last_bytes reads, so that nothing behind the operand is.
template <FewRows ROWS>
__device__ __forceinline__ uint4 bytes16(const Line& l, int k, int left) {
    const char* const p = l.at + k;
    if constexpr (ROWS != kShift) {
        uint4 v = ld16_if(p, l.on && left >= (ROWS == kWhole ? 1 : 16));
        // (zeros already, but without it fewer loads are in flight: GB300, 1 x 12288 x 4096 18.3 -> 23.6 us)
        if (left < 16) v = first_bytes(v, left);
        return v;
    } else {
        const int m = (int)((uintptr_t)p & 15);
        const bool lo = l.on && left > 0, hi = lo && m && left > 16 - m;
        if (lo && (p - m < l.from || p - m + (hi ? 32 : 16) > l.to)) return bytes_at(p, left);  // at the operand's ends
        return first_bytes(shifted(ld16_if(p - m, lo), ld16_if(p - m + 16, hi), m), left);
    }
}
// A row's last bytes, fewer than 16, in the lane that has them.
__device__ __forceinline__ uint4 last_bytes(const Line& l, int k, int left) { return bytes_at(l.at + k, l.on && left < 16 ? left : 0); }

template <int NT, bool FP8, FewRows ROWS>
__global__ void __launch_bounds__(32 * kWarps) linear_few_kernel(const __grid_constant__ LinearFewArgs A) {
    __shared__ float part[kWarps][8 * NT][16];
    after_previous();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, t = lane % 4;
    uint32_t rank, ranks;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(ranks));
    const int col0 = (int)(blockIdx.x / ranks) * 16;
    const int M = A.e.M, N = A.e.N, k_bytes = A.k_bytes;
    const char *const x = reinterpret_cast<const char*>(A.x), *const w = reinterpret_cast<const char*>(A.w);
    auto line = [&](const char* from, int row, int rows, long long stride) {
        return Line{from + row * stride + 16 * t, from, from + (rows - 1) * stride + k_bytes, row < rows};
    };
    const Line w_lo = line(w, col0 + g, N, A.w_row), w_hi = line(w, col0 + g + 8, N, A.w_row);
    Line xl[NT];
#pragma unroll
    for (int i = 0; i < NT; ++i) xl[i] = line(x, 8 * i + g, M, A.x_row);

    float sum[NT][4];
#pragma unroll
    for (int i = 0; i < NT; ++i) sum[i][0] = sum[i][1] = sum[i][2] = sum[i][3] = 0.0f;
    const int step = kTurn * kWarps * (int)ranks;
    constexpr int DEEP = NT >= 4 ? 2 : kDeep;
    for (int k0 = kTurn * (kWarps * (int)rank + warp); k0 < k_bytes; k0 += DEEP * step) {
        uint4 lo[DEEP], hi[DEEP], xv[DEEP][NT];
#pragma unroll
        for (int j = 0; j < DEEP; ++j) {
            const int k = k0 + j * step, left = k_bytes - k - 16 * t;
            lo[j] = bytes16<ROWS>(w_lo, k, left);
            hi[j] = bytes16<ROWS>(w_hi, k, left);
#pragma unroll
            for (int i = 0; i < NT; ++i) xv[j][i] = bytes16<ROWS>(xl[i], k, left);
        }
        float d[NT][4] = {};
#pragma unroll
        for (int j = 0; j < DEEP; ++j)
#pragma unroll
            for (int i = 0; i < NT; ++i) product<FP8>(d[i], lo[j], hi[j], xv[j][i]);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[i][q] += d[i][q];
    }
    const int last = k_bytes / kTurn * kTurn;  // the last turn, which has the rows' last bytes
    if (ROWS == kTail && last / kTurn % (kWarps * (int)ranks) == kWarps * (int)rank + warp) {
        const int left = k_bytes - last - 16 * t;
        const uint4 lo = last_bytes(w_lo, last, left), hi = last_bytes(w_hi, last, left);
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            float d[4] = {};
            product<FP8>(d, lo, hi, last_bytes(xl[i], last, left));
#pragma unroll
            for (int q = 0; q < 4; ++q) sum[i][q] += d[q];
        }
    }
#pragma unroll
    for (int i = 0; i < NT; ++i) {
        float(*p)[16] = part[warp] + 8 * i;
        p[2 * t][g] = sum[i][0], p[2 * t + 1][g] = sum[i][1];
        p[2 * t][g + 8] = sum[i][2], p[2 * t + 1][g + 8] = sum[i][3];
    }
    __syncthreads();
    // this CTA's sums into part[0]
    for (int i = threadIdx.x; i < 8 * NT * 16; i += 32 * kWarps) {
        float v = 0.0f;
#pragma unroll
        for (int q = 0; q < kWarps; ++q) v += part[q][i / 16][i % 16];
        part[0][i / 16][i % 16] = v;
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
    const LinearEpilogue E = from_here(A.e);
    // the cluster's CTAs share the rest; the loops above and below deal the same elements to a thread
    for (int i = threadIdx.x; i < 8 * NT * 16; i += 32 * kWarps) {
        if (ranks > 1 && (i / (32 * kWarps)) % ranks != rank) continue;
        float v = 0.0f;
        if (ranks == 1) {
            v = part[0][i / 16][i % 16];
        } else {
            const uint32_t mine = (uint32_t)__cvta_generic_to_shared(&part[0][i / 16][i % 16]);
            for (uint32_t q = 0; q < ranks; ++q) {
                uint32_t at;
                float f;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"(mine), "r"(q));
                asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(f) : "r"(at) : "memory");
                v += f;
            }
        }
        const int row = i / 16, col = col0 + i % 16;
        if (row >= M || col >= N) continue;
        if (E.x_scale) v *= E.x_scale[row];
        const float s = E.w_scale ? E.w_scale[col] : 1.0f;
        v = fmaf(v, s, E.bias ? __uint_as_float(lin_ld1(E.bias, col, E.bias_bf16)) : 0.0f);
        if (E.act == CB_ACT_GELU) v = both(lin_act<CB_ACT_GELU>(two(v, v))).x;
        if (E.act == CB_ACT_SILU) v = both(lin_act<CB_ACT_SILU>(two(v, v))).x;
        if (E.out) lin_put1(E.out, row * E.out_stride + col, E.out_bf16, v);
        if (E.resid_out) {
            const float r = __uint_as_float(lin_ld1(E.resid, row * E.resid_stride + col, E.resid_bf16));
            float gate = 1.0f;
            if (E.gate)
                gate = __uint_as_float(lin_ld1(E.gate, (long long)((unsigned)row / E.tokens) * E.gate_stride + col, E.gate_bf16));
            lin_put1(E.resid_out, row * E.resid_out_stride + col, E.resid_bf16, fmaf(gate, v, r));
        }
    }
    // no CTA leaves while another may still read its sums
    if (ranks > 1) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

using Kernel = void (*)(LinearFewArgs);
template <int NT, bool FP8>
Kernel pick(FewRows rows) {
    return rows == kShift ? linear_few_kernel<NT, FP8, kShift> : rows == kTail ? linear_few_kernel<NT, FP8, kTail> : linear_few_kernel<NT, FP8, kWhole>;
}
template <int NT>
Kernel pick(bool fp8, FewRows rows) { return fp8 ? pick<NT, true>(rows) : pick<NT, false>(rows); }

}  // namespace

cudaError_t launch_linear_few(const LinearFewArgs& a, bool fp8, bool shift, int sms, cudaStream_t s) {
    const int nt = a.e.M <= 8 ? 1 : a.e.M <= 16 ? 2 : 4;
    const FewRows rows = shift ? kShift : a.k_bytes % 16 != 0 ? kTail : kWhole;
    const Kernel k = nt == 1 ? pick<1>(fp8, rows) : nt == 2 ? pick<2>(fp8, rows) : pick<4>(fp8, rows);
    const unsigned cols = (unsigned)((a.e.N + 15) / 16);
    // CTAs along K while there are fewer than three per SM and every warp keeps two turns
    unsigned cluster = 1;
    while (cluster < 8 && cols * cluster * 2 <= 3u * (unsigned)sms && (int)(cluster * 2 * kWarps * kTurn * 2) <= a.k_bytes) cluster *= 2;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = a.overlap;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(cluster * cols);
    c.blockDim = dim3(32 * kWarps);
    c.stream = s;
    c.attrs = at;
    c.numAttrs = cluster > 1 ? 2 : 1;
    void* args[] = {const_cast<void*>(static_cast<const void*>(&a))};
    const cudaError_t e = cudaLaunchKernelExC(&c, reinterpret_cast<const void*>(k), args);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e;
}

}  // namespace cbk
