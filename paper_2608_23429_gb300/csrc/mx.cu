// cb_mx_quantize and cb_mx_dequantize: rows to and from 4 bits.
//
// Bound by HBM: an element is read and written once. A lane has eight consecutive elements, so a block is four lanes and two shuffles
// find its largest magnitude; a warp has 256 elements of four rows, 32 apart, whose scales are 16 consecutive bytes of a
// tile of them, and the CTA's eight warps have neighbouring rows, whose are 128. GB300: 129024 x 1152 fp32 written in 93 us (106 % of the copy
// rate) and read back in 100 (99 %); 65536 x 4608 bf16 122 and 111 (93 and 102 %; with each row's loads behind a branch of its own 192);
// rows off the 16-byte grid 16384 x 1153 bf16 16 and 16 (a copy of their bytes: 7).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "../../include/chebboost_block.h"
#include "cb_device.h"
#include "mx.cuh"

namespace cbk {
namespace {

constexpr int kMxWarps = 8, kMxRows = 4, kMxPiece = 256;  // warps of a CTA; rows, and features of a row, of a warp

struct MxArgs {
    int overlap;
    unsigned rows, features, chunks, tiles_k;  // chunks of kMxPiece features
    long long stride, codes_row;               // elements; bytes
    void* x;
    uint8_t *codes, *scales;
};

// Eight elements of a row by vectors, or n by elements and zeros behind them.
template <bool BF16, bool VEC>
__device__ __forceinline__ void load8(const void* p, long long e, int n, float* v) {
    if constexpr (VEC) {
        if constexpr (BF16) {
            const uint4 q = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p) + e);
            const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) v[2 * i] = __uint_as_float(w[i] << 16), v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        } else {
            const float4* q = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p) + e);
            const float4 a = q[0], b = q[1];
            v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = 0.0f;
        if (i < n) v[i] = BF16 ? __uint_as_float((uint32_t) reinterpret_cast<const uint16_t*>(p)[e + i] << 16) : reinterpret_cast<const float*>(p)[e + i];
    }
}
template <bool BF16, bool VEC>
__device__ __forceinline__ void store8(void* p, long long e, int n, const float* v) {
    if (VEC && n >= 8) {
        if constexpr (BF16) {
            __nv_bfloat162 h[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
            *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p) + e) = *reinterpret_cast<const uint4*>(h);
        } else {
            float* const q = reinterpret_cast<float*>(p) + e;
            if ((uintptr_t)q % 32 == 0) {  // a sector in one store
                asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(q), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]),
                             "f"(v[5]), "f"(v[6]), "f"(v[7])
                             : "memory");
            } else {
                reinterpret_cast<float4*>(q)[0] = make_float4(v[0], v[1], v[2], v[3]);
                reinterpret_cast<float4*>(q)[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= n) break;
        if constexpr (BF16) reinterpret_cast<__nv_bfloat16*>(p)[e + i] = __float2bfloat16_rn(v[i]);
        else reinterpret_cast<float*>(p)[e + i] = v[i];
    }
}

// What a warp works on: its first row (the others follow 32 apart) and its lane's first feature.
struct MxPlace {
    unsigned row, col;
};
__device__ __forceinline__ MxPlace mx_place(const MxArgs& A) {
    const unsigned group = blockIdx.x / A.chunks, chunk = blockIdx.x - group * A.chunks;
    return MxPlace{group / 4 * kMxTileRows + group % 4 * kMxWarps + threadIdx.x / 32, chunk * kMxPiece + threadIdx.x % 32 * 8};
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(32 * kMxWarps) mx_quantize_kernel(const __grid_constant__ MxArgs A) {
    after_previous();
    const auto [row0, col] = mx_place(A);
    const int n = (int)min(A.features - min(col, A.features), 8u), lane = threadIdx.x % 32;
    float v[kMxRows][8];
    if (VEC && n == 8) {  // all rows' loads together (rows behind the last: that one's)
#pragma unroll
        for (int j = 0; j < kMxRows; ++j) load8<BF16, true>(A.x, (long long)min(row0 + 32 * j, A.rows - 1) * A.stride + col, 8, v[j]);
    } else {
#pragma unroll
        for (int j = 0; j < kMxRows; ++j)
            load8<BF16, false>(A.x, (long long)(row0 + 32 * j) * A.stride + col, row0 + 32 * j < A.rows ? n : 0, v[j]);
    }
    uint32_t words[kMxRows];
#pragma unroll
    for (int j = 0; j < kMxRows; ++j) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; i += 2) top = mx_max_abs(top, v[j][i], v[j][i + 1]);
        uint32_t most = __float_as_uint(top);
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 1));
        most = max(most, __shfl_xor_sync(0xFFFFFFFFu, most, 2));
        const uint32_t e = mx_scale_of(most);
        const float inverse = mx_inverse(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[j][i] *= inverse;
        const uint32_t codes = e == 255 ? 0u : mx_codes8(v[j]);
        const unsigned row = row0 + 32 * j;
        if (row < A.rows && col < (A.features + kMxBlock - 1) / kMxBlock * kMxBlock)
            *reinterpret_cast<uint32_t*>(A.codes + row * A.codes_row + col / 2) = codes;
        uint32_t w = e << 8 * (lane / 4 % 4);
        w |= __shfl_xor_sync(0xFFFFFFFFu, w, 4);
        words[j] = w | __shfl_xor_sync(0xFFFFFFFFu, w, 8);
    }
    const unsigned k = col / (kMxBlock * kMxTileBlocks);
    if (lane % 16 != 0 || k >= A.tiles_k || row0 >= A.rows) return;
    uint32_t* const to = reinterpret_cast<uint32_t*>(A.scales + mx_word_at(row0, k, A.tiles_k));
    if (row0 + 32 * (kMxRows - 1) < A.rows) {
        *reinterpret_cast<uint4*>(to) = make_uint4(words[0], words[1], words[2], words[3]);
    } else {
#pragma unroll
        for (int j = 0; j < kMxRows; ++j)
            if (row0 + 32 * j < A.rows) to[j] = words[j];
    }
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(32 * kMxWarps) mx_dequantize_kernel(const __grid_constant__ MxArgs A) {
    after_previous();
    const auto [row0, col] = mx_place(A);
    const int n = (int)min(A.features - min(col, A.features), 8u), lane = threadIdx.x % 32;
    if ((VEC && n <= 0) || row0 >= A.rows) return;
    uint32_t words[kMxRows] = {}, codes[kMxRows];
    const unsigned k = col / (kMxBlock * kMxTileBlocks);
    if (k < A.tiles_k) {
        const uint4 q = *reinterpret_cast<const uint4*>(A.scales + mx_word_at(row0, k, A.tiles_k));
        words[0] = q.x, words[1] = q.y, words[2] = q.z, words[3] = q.w;
    }
#pragma unroll
    for (int j = 0; j < kMxRows; ++j) {
        const unsigned row = row0 + 32 * j;
        codes[j] = row < A.rows && n > 0 ? *reinterpret_cast<const uint32_t*>(A.codes + row * A.codes_row + col / 2) : 0u;
    }
#pragma unroll
    for (int j = 0; j < kMxRows; ++j) {
        const unsigned row = row0 + 32 * j;
        if (row >= A.rows) break;
        if constexpr (VEC) {
            const float power = mx_power(words[j] >> 8 * (lane / 4 % 4) & 255u);
            uint32_t h[4];
            float v[8];
            mx_widen8(codes[j], h);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[i]));
                v[2 * i] = f.x * power, v[2 * i + 1] = f.y * power;
            }
            store8<BF16, VEC>(A.x, row * A.stride + col, n, v);
        } else {
            // a block of the warp's eight at a time, an element a lane: neighbours' stores share sectors
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t power = __shfl_sync(0xFFFFFFFFu, words[j], 16 * (i / 4)) >> 8 * (i % 4) & 255u;
                const uint32_t eight = __shfl_sync(0xFFFFFFFFu, codes[j], 4 * i + lane / 8);
                uint32_t h[4];
                mx_widen8(eight >> 4 * (lane % 8) & 15u, h);
                const float v = __half22float2(*reinterpret_cast<const __half2*>(&h[0])).x * mx_power(power);
                const unsigned e = col - lane * 8 + 32 * i + lane;
                if (e < A.features) {
                    if constexpr (BF16) reinterpret_cast<__nv_bfloat16*>(A.x)[row * A.stride + e] = __float2bfloat16_rn(v);
                    else reinterpret_cast<float*>(A.x)[row * A.stride + e] = v;
                }
            }
        }
    }
}

bool on_grid(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

// The checks of either call; *a is for the launch of *grid CTAs (0: nothing to do), *vec: rows on the 16-byte grid.
int checked(const cb_mx_desc* d, const void* x, const void* codes, const void* scales, MxArgs* a, int* grid, bool* vec) {
    *grid = 0;
    if (!d || d->reserved != 0 || d->rows < 0 || d->features < 1) return CB_ERR_ARG;
    if (d->dtype != CB_BF16 && d->dtype != CB_FP32) return CB_ERR_ARG;
    if (d->rows > 0x7FFFFFFFLL || d->features > 0x7FFFFF00LL) return CB_ERR_LIMIT;
    const long long blocks = mx_blocks(d->features), es = d->dtype == CB_BF16 ? 2 : 4;
    if (d->stride != 0 && d->stride < d->features) return CB_ERR_ARG;
    if (d->codes_stride != 0 && (d->codes_stride < blocks * kMxBlock || d->codes_stride % kMxBlock != 0)) return CB_ERR_ARG;
    if (d->stride > CB_MAX_NUMEL || d->codes_stride > CB_MAX_NUMEL) return CB_ERR_LIMIT;
    if (d->rows == 0) return CB_OK;
    if (!x || !codes || !scales) return CB_ERR_ARG;
    if (!on_grid(x, es) || !on_grid(codes, 16) || !on_grid(scales, 16)) return CB_ERR_ALIGN;
    a->overlap = 1;
    a->rows = (unsigned)d->rows, a->features = (unsigned)d->features;
    a->chunks = (unsigned)((d->features + kMxPiece - 1) / kMxPiece);
    a->tiles_k = (unsigned)mx_tiles_k(d->features);
    a->stride = d->stride ? d->stride : d->features;
    a->codes_row = (d->codes_stride ? d->codes_stride : blocks * kMxBlock) / 2;
    a->x = const_cast<void*>(x);
    a->codes = static_cast<uint8_t*>(const_cast<void*>(codes)), a->scales = static_cast<uint8_t*>(const_cast<void*>(scales));
    // groups of kMxWarps rows, 32 of which share a tile with those 32, 64 and 96 further on
    const long long last = (d->rows - 1) / kMxTileRows;
    const long long rest = d->rows - last * kMxTileRows;
    const long long groups = last * 4 + (rest >= 32 ? 4 : (rest + kMxWarps - 1) / kMxWarps);
    if (groups * a->chunks > 0x7FFFFFFFLL) return CB_ERR_LIMIT;
    *grid = (int)(groups * a->chunks);
    *vec = on_grid(x, 16) && a->stride * es % 16 == 0;
    return CB_OK;
}

}  // namespace
}  // namespace cbk

extern "C" {

int cb_mx_scale_bytes(int64_t rows, int64_t features, size_t* bytes) {
    using namespace cbk;
    if (!bytes || rows < 0 || features < 1) return CB_ERR_ARG;
    if (rows > 0x7FFFFFFFLL || features > 0x7FFFFF00LL) return CB_ERR_LIMIT;
    *bytes = (size_t)((rows + kMxTileRows - 1) / kMxTileRows * mx_tiles_k(features) * kMxTileBytes);
    return CB_OK;
}

int cb_mx_quantize(const cb_mx_desc* d, const void* x, void* codes, void* scales, void* stream) {
    using namespace cbk;
    MxArgs a{};
    int grid = 0;
    bool vec = false;
    const int rc = checked(d, x, codes, scales, &a, &grid, &vec);
    if (rc != CB_OK || grid == 0) return rc;
    const auto k = d->dtype == CB_BF16 ? (vec ? mx_quantize_kernel<true, true> : mx_quantize_kernel<true, false>)
                                       : (vec ? mx_quantize_kernel<false, true> : mx_quantize_kernel<false, false>);
    const cudaError_t e = launch_overlapped(k, grid, 32 * kMxWarps, 0, (cudaStream_t)stream, a);
    return e == cudaSuccess ? CB_OK : cuda_error(e, "quantize launch");
}

int cb_mx_dequantize(const cb_mx_desc* d, const void* codes, const void* scales, void* x, void* stream) {
    using namespace cbk;
    MxArgs a{};
    int grid = 0;
    bool vec = false;
    const int rc = checked(d, x, codes, scales, &a, &grid, &vec);
    if (rc != CB_OK || grid == 0) return rc;
    const auto k = d->dtype == CB_BF16 ? (vec ? mx_dequantize_kernel<true, true> : mx_dequantize_kernel<true, false>)
                                       : (vec ? mx_dequantize_kernel<false, true> : mx_dequantize_kernel<false, false>);
    const cudaError_t e = launch_overlapped(k, grid, 32 * kMxWarps, 0, (cudaStream_t)stream, a);
    return e == cudaSuccess ? CB_OK : cuda_error(e, "dequantize launch");
}

}  // extern "C"
