// Internal: rows in 4 bits (CB_MXFP4): e2m1 codes, 32 of which share a power of two.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

namespace cbk {

constexpr int kMxBlock = 32;       // elements that share a scale
constexpr int kMxTileRows = 128;   // rows and blocks of a tile of scales
constexpr int kMxTileBlocks = 4;
constexpr int kMxTileBytes = kMxTileRows * kMxTileBlocks;

constexpr long long mx_blocks(long long features) { return (features + kMxBlock - 1) / kMxBlock; }
constexpr long long mx_row_bytes(long long features) { return mx_blocks(features) * (kMxBlock / 2); }
constexpr long long mx_tiles_k(long long features) { return (mx_blocks(features) + kMxTileBlocks - 1) / kMxTileBlocks; }

#ifdef __CUDACC__
namespace {

// Where the four scales of a row in tile `k` of its blocks lie; those of rows 32 apart follow each other.
__device__ __forceinline__ long long mx_word_at(unsigned row, unsigned k, unsigned tiles_k) {
    return ((long long)(row / kMxTileRows) * tiles_k + k) * kMxTileBytes + row % 32 * 16 + row / 32 % 4 * 4;
}

// A block's scale byte from its largest magnitude as bits (a NaN's lie above infinity's): the exponent of the magnitude rounded to two
// significant bits, less that of 4, so that scaled magnitudes lie below 7 and what is cut off by codes up to 6 is no more
// than what is rounded (a bound of 6 wastes the code 6 for maxima of 6 to 7, one of 8 cuts off a quarter; root mean square error of
// normal values 0.1119 of theirs, 0.1154 and 0.1150).
__device__ __forceinline__ uint32_t mx_scale_of(uint32_t amax) {
    const int e = (int)((amax + 0x200000u) >> 23) - 2;
    return amax >= 0x7F800000u ? 255u : (uint32_t)max(e, 0);
}
// 2^(127 - e), by which a block is multiplied (e <= 253); 0 for e = 255.
__device__ __forceinline__ float mx_inverse(uint32_t e) { return __uint_as_float(e == 255 ? 0u : (254u - e) << 23); }
// 2^(e - 127): a subnormal for e = 0, NaN for e = 255.
__device__ __forceinline__ float mx_power(uint32_t e) { return __uint_as_float(e == 0 ? 0x00400000u : e == 255 ? 0x7FC00000u : e << 23); }

// The largest magnitude of three; a NaN wins.
__device__ __forceinline__ float mx_max_abs(float a, float b, float c) {
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}

// Codes of eight scaled values, the first in the lowest bits, to nearest even and 6 at most.
__device__ __forceinline__ uint32_t mx_codes8(const float* v) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return r;
}
// Eight codes as four pairs of fp16.
__device__ __forceinline__ void mx_widen8(uint32_t codes, uint32_t* h) {
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "mov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(codes));
}

}  // namespace
#endif

}  // namespace cbk
