// Operands of cb_linear_run off the 16-byte grid, copied onto a grid of their own so that TMA can load them: bound by their
// bytes, read once and written once (to L2, where they fit). GB300, copy and product: 4096 x 4096 x 4097 bf16 101 us, 999 x 577 x
// 1155 14.3, 90 x 5800 x 5494 53; with warps that loaded the operands through registers and shifted them into the product's stages,
// without a copy, 867, 28.5 and 153.
//
// A thread makes 32 bytes of a row out of the three aligned 16-byte pieces that they touch; neighbours share pieces in L1. Four such
// chunks of a thread are in flight together. Pieces that begin or end outside the operand are read by bytes.
#include "linear.cuh"
#include "linear_shift.cuh"

namespace cbk {
namespace {

constexpr int kPackThreads = 256, kPackDeep = 4;

__global__ void __launch_bounds__(kPackThreads) pack_rows_kernel(const __grid_constant__ LinearPackArgs A) {
    after_previous();
    const bool second = blockIdx.x >= A.blocks;
    const PackOperand o = second ? A.o[1] : A.o[0];
    const unsigned long long first = (unsigned long long)(blockIdx.x - (second ? A.blocks : 0)) * (kPackThreads * kPackDeep) + threadIdx.x;
    const unsigned down = kPackThreads / o.chunks, right = kPackThreads % o.chunks;
    const char *const lo = o.src, *const hi = o.src + (o.rows - 1) * o.stride + o.bytes;
    long long row = (long long)(first / o.chunks);
    unsigned at = (unsigned)(first % o.chunks);
    uint4 p[kPackDeep][3];
    int left[kPackDeep], off[kPackDeep];  // bytes of the row from this chunk on; the chunk's place in its first piece
    const char* from[kPackDeep];
#pragma unroll
    for (int i = 0; i < kPackDeep; ++i) {
        const char* const q = o.src + row * o.stride + 32ll * at;
        left[i] = row < o.rows ? o.bytes - (int)(32 * at) : 0;
        off[i] = (int)((uintptr_t)q & 15);
        from[i] = q - off[i];
        const int end = off[i] + min(left[i], 32);
#pragma unroll
        for (int j = 0; j < 3; ++j)
            p[i][j] = ld16_if(from[i] + 16 * j, left[i] > 0 && 16 * j < end && from[i] + 16 * j >= lo && from[i] + 16 * j + 16 <= hi);
        at += right;
        row += down + (at >= o.chunks);
        if (at >= o.chunks) at -= o.chunks;
    }
#pragma unroll
    for (int i = 0; i < kPackDeep; ++i) {
        if (left[i] <= 0) continue;
        if (from[i] < lo || from[i] + 48 > hi) {
            const int end = off[i] + min(left[i], 32);
#pragma unroll
            for (int j = 0; j < 3; ++j) {
                const char* const q = from[i] + 16 * j;
                if (16 * j < end && (q < lo || q + 16 > hi)) {
                    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
                    for (int b = 0; b < 16; ++b)
                        if (q + b >= lo && q + b < hi) w[b / 4] |= (uint32_t)(uint8_t)q[b] << 8 * (b % 4);
                    p[i][j] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
        const uint4 a = first_bytes(shifted(p[i][0], p[i][1], off[i]), left[i]);
        const uint4 b = first_bytes(shifted(p[i][1], p[i][2], off[i]), left[i] - 16);
        asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(o.dst + 32 * (first + (unsigned)(i * kPackThreads))),
                     "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                     : "memory");
    }
}

}  // namespace

cudaError_t launch_linear_pack(LinearPackArgs& a, cudaStream_t s) {
    long long blocks[2];
    for (int i = 0; i < 2; ++i) {
        const long long n = a.o[i].dst ? a.o[i].rows * a.o[i].chunks : 0;
        blocks[i] = (n + kPackThreads * kPackDeep - 1) / (kPackThreads * kPackDeep);
    }
    if (blocks[0] + blocks[1] > 0x7FFFFFFFLL) return cudaErrorInvalidConfiguration;
    a.blocks = (unsigned)blocks[0];
    return launch_overlapped(pack_rows_kernel, (int)(blocks[0] + blocks[1]), kPackThreads, 0, s, a);
}

}  // namespace cbk
