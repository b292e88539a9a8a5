// Internal: 16 bytes from an address off the 16-byte grid, out of two aligned pieces.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace cbk {
namespace {

// The aligned 16 bytes at p where `on`, else zeros; predicated, so that loads are in flight together.
__device__ __forceinline__ uint4 ld16_if(const char* p, bool on) {
    uint4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %5, 0;\n\t"
        "mov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
        "@p ld.global.v4.u32 {%0,%1,%2,%3}, [%4];\n\t}"
        : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w)
        : "l"(p), "r"((int)on));
    return v;
}

// Bytes [m, m + 16) of the two pieces (m in [0, 16)).
__device__ __forceinline__ uint4 shifted(const uint4& lo, const uint4& hi, int m) {
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = m & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = m & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 8 * (m & 3));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The first n bytes of v, zeros behind them.
__device__ __forceinline__ uint4 first_bytes(uint4 v, int n) {
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if (n < 16) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n < 4 * i + 4) w[i] = n <= 4 * i ? 0 : w[i] & ((1u << 8 * (n - 4 * i)) - 1);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The n bytes at p (16 at most), one by one, zeros behind them.
__device__ __forceinline__ uint4 bytes_at(const char* p, int n) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 16; ++i)
        if (i < n) w[i / 4] |= (uint32_t)(uint8_t)p[i] << 8 * (i % 4);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

}  // namespace
}  // namespace cbk
