// The matrix product of cb_linear_run on the fifth-generation tensor cores.
//
// A persistent grid of CTAs (CG = 1) or of pairs of CTAs on two SMs (CG = 2) works through output tiles of 128 CG
// rows by tile_n columns. In a CTA
//   one warp (TMA) or eight (words) fill a ring of stages with slabs of 128 bytes of K: 128 rows of x and
//     tile_n / CG rows of w, in the 128-byte swizzle that the tensor cores read,
//   one thread issues tcgen05.mma on them, sums in TMEM (two accumulators of up to 256 columns each),
//   four warps take a finished accumulator out of TMEM while the next tile is summed, turn it in shared memory so
//     that their accesses to global memory are rows, and apply the epilogue (lin_finish).
// A pair of CTAs shares one tile: each loads its 128 rows of x and half of the tile's rows of w, the first one's
// thread issues for both, and each holds the sums of its own rows.
//
// WORDS: operands whose rows do not start on 16-byte boundaries cannot come by TMA. Eight warps load them as
// aligned 32-bit words, a row of a slab per warp and step, shift neighbouring words together and store them where
// TMA would have put them.
//
// Every wait has a limit (kLimitNs); one that runs out sets the CTA's abort flag, so that all its roles leave, after
// the copies under way have landed, and frees the TMEM.
#include "cb_async.cuh"
#include "linear.cuh"

namespace cbk {
namespace {

constexpr int kRows = 128;        // rows of x per CTA
constexpr int kSlab = 128;        // bytes of K per stage
constexpr int kMaxLinStages = 12;
constexpr int kAccStride = 256;   // TMEM columns from one accumulator to the other
constexpr int kLoadWarps = 8;     // WORDS
constexpr unsigned long long kLimitNs = 1000000000ull;

struct Tail {  // behind the stages
    float turn[4][32 * 32];
    uint64_t full[kMaxLinStages], empty[kMaxLinStages], acc_full[2], acc_empty[2];
    uint32_t tmem;
    int abort;
};

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}
// Address of `bar` in the pair's first CTA.
__device__ __forceinline__ uint32_t in_first(uint32_t bar) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(r) : "r"(bar));
    return r;
}
__device__ __forceinline__ void arrive_at(uint32_t cluster_bar) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
}
__device__ __forceinline__ bool try_wait_cluster(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}

// Wait for a phase of a barrier, until the limit or the CTA's abort flag.
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, volatile int* abort, int* status, int code) {
    auto done = [&] { return CLUSTER ? try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity); };
    if (done()) return true;
    const unsigned long long t0 = now_ns();
    while (true) {
        for (int i = 0; i < 8; ++i)
            if (done()) return true;
        if (*abort) return false;
        if (now_ns() - t0 > kLimitNs) {
            *abort = 1;
            record(status, code);
            return false;
        }
    }
}

template <int CG>
__device__ __forceinline__ void tma_2d(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
                dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
    else  // the barrier may be the other CTA's
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, "
            "%3}], [%4];" ::"r"(dst),
            "l"(map), "r"(x), "r"(y), "r"(bar)
            : "memory");
}

// Operand in shared memory: rows of 128 bytes, K innermost, 128-byte swizzle in groups of eight rows (1024 bytes).
__device__ __forceinline__ uint64_t operand_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3FFFF) >> 4) | 1ull << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

template <int CG, bool FP8>
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    const uint32_t on = add;
#define CB_MMA(GROUP, KIND)                                                                         \
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\t"                                   \
                 "tcgen05.mma.cta_group::" GROUP ".kind::" KIND " [%0], %1, %2, %3, p;\n\t}" ::"r"(d), \
                 "l"(a), "l"(b), "r"(idesc), "r"(on)                                                \
                 : "memory")
    if constexpr (CG == 1) {
        if constexpr (FP8) CB_MMA("1", "f8f6f4");
        else CB_MMA("1", "f16");
    } else {
        if constexpr (FP8) CB_MMA("2", "f8f6f4");
        else CB_MMA("2", "f16");
    }
#undef CB_MMA
}

// Arrives on `bar` (of both CTAs of a pair) when all products issued so far are done.
template <int CG>
__device__ __forceinline__ void commit(uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
            "h"((uint16_t)3)
            : "memory");
}

__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }

// 32 columns of the warp's 32 rows, a row per lane.
__device__ __forceinline__ void tmem_load(uint32_t addr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(addr));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

struct Tile {
    int m, n;
};
// Groups of eight rows of tiles, so that tiles worked on together share operands in L2.
__device__ __forceinline__ Tile tile_at(const LinearArgs& A, int t) {
    const int group = 8 * A.tiles_n, g = t / group, r = t - g * group;
    const int rows = min(8, A.tiles_m - 8 * g);
    return Tile{8 * g + r % rows, r / rows};
}

// The aligned word i of the bytes [p, p + n): whole where it lies inside, else byte by byte.
__device__ __forceinline__ uint32_t word_of(const char* p, int n, int i) {
    const int shift = (int)((uintptr_t)p & 3), at = 4 * i - shift;  // byte of the row that the word starts with
    if (at >= 0 && at + 4 <= n) return *reinterpret_cast<const uint32_t*>(p + at);
    uint32_t v = 0;
#pragma unroll
    for (int b = 0; b < 4; ++b)
        if (at + b >= 0 && at + b < n) v |= (uint32_t)(uint8_t)p[at + b] << 8 * b;
    return v;
}

template <int CG, bool FP8, bool WORDS>
__global__ void __launch_bounds__(32 * (5 + (WORDS ? kLoadWarps : 1)), 1)
    linear_kernel(const __grid_constant__ LinearArgs A) {
    static_assert(CG == 1 || !WORDS, "pairs of CTAs load by TMA");
    extern __shared__ uint8_t raw[];
    uint8_t* const base = raw + (1024 - (smem_addr(raw) & 1023)) % 1024;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int w_rows = A.tile_n / CG, stage_bytes = (kRows + w_rows) * kSlab, stages = A.stages;
    Tail& T = *reinterpret_cast<Tail*>(base + stages * stage_bytes);
    const uint32_t ring = smem_addr(base);
    const uint32_t full = smem_addr(T.full), empty = smem_addr(T.empty);
    const uint32_t acc_full = smem_addr(T.acc_full), acc_empty = smem_addr(T.acc_empty);
    volatile int* const abort = &T.abort;

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(full + 8 * s, WORDS ? kLoadWarps : 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, 4 * CG);
        }
        *abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_generic_to_async();
    }
    if (warp == 4) {
        const uint32_t at = smem_addr(&T.tmem);
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(at) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(at) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    fence_before();
    __syncwarp();
    if constexpr (CG == 2) cluster_sync();
    __syncthreads();
    fence_after();
    const uint32_t tmem = T.tmem;
    after_previous();

    const int first = blockIdx.x / CG, step = gridDim.x / CG, total = A.tiles_m * A.tiles_n;
    if (warp < 4) {  // ---- epilogue
        float* const turn = T.turn[warp];
        int n_done = 0;
        for (int t = first; t < total; t += step, ++n_done) {
            const Tile tile = tile_at(A, t);
            const int acc = n_done & 1;
            if (!__all_sync(0xFFFFFFFFu, wait(acc_full + 8 * acc, (n_done >> 1) & 1, abort, A.status, CB_DEV_CONSUMER_TIMEOUT)))
                break;
            fence_after();
            const int row0 = (tile.m * CG + (int)rank) * kRows + warp * 32, col0 = tile.n * A.tile_n;
            const float xs = A.x_scale && row0 + lane < A.M ? A.x_scale[row0 + lane] : 1.0f;
            const int chunks = (min(A.tile_n, A.N - col0) + 31) / 32;
            for (int c = 0; c < chunks; ++c) {
                float v[32];
                tmem_load(tmem + ((uint32_t)(warp * 32) << 16) + acc * kAccStride + c * 32, v);
                if (c + 1 == chunks) {  // all of it has been read
                    fence_before();
                    __syncwarp();
                    if (lane == 0) {
                        if constexpr (CG == 1) mbar_arrive(acc_empty + 8 * acc);
                        else arrive_at(in_first(acc_empty + 8 * acc));
                    }
                }
                // a row per lane to rows of 32 columns across eight lanes: 16-byte pieces, swizzled against bank conflicts
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<float4*>(&turn[lane * 32 + (j ^ (lane & 7)) * 4]) =
                        make_float4(v[4 * j] * xs, v[4 * j + 1] * xs, v[4 * j + 2] * xs, v[4 * j + 3] * xs);
                __syncwarp();
                float4 u[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int r = 4 * i + lane / 8;
                    u[i] = *reinterpret_cast<const float4*>(&turn[r * 32 + ((lane & 7) ^ (r & 7)) * 4]);
                }
                __syncwarp();
                lin_finish<8>(A, row0 + lane / 8, 4, col0 + c * 32 + (lane & 7) * 4, u);
            }
        }
    } else if (warp == 4) {  // ---- products
        if (lane == 0 && rank == 0) {
            // fp32 sums; A and B bf16 (kind f16) or e4m3 (kind f8f6f4), both with K innermost; N / 8, M / 16
            const uint32_t idesc =
                1u << 4 | (FP8 ? 0u : 1u << 7 | 1u << 10) | (uint32_t)(A.tile_n / 8) << 17 | (uint32_t)(kRows * CG / 16) << 24;
            int it = 0, n_done = 0;
            bool ok = true;
            for (int t = first; t < total && ok; t += step, ++n_done) {
                const int acc = n_done & 1;
                ok = wait<CG == 2>(acc_empty + 8 * acc, ((n_done >> 1) & 1) ^ 1, abort, A.status, CB_DEV_PRODUCER_TIMEOUT);
                fence_after();
                for (int kb = 0; kb < A.k_blocks && ok; ++kb, ++it) {
                    const int s = it % stages;
                    ok = wait(full + 8 * s, (it / stages) & 1, abort, A.status, CB_DEV_CONSUMER_TIMEOUT);
                    if (!ok) break;
                    fence_after();
                    const uint64_t a = operand_desc(ring + s * stage_bytes), b = operand_desc(ring + s * stage_bytes + kRows * kSlab);
                    const int steps = min(4, (A.k_bytes - kb * kSlab + 31) / 32);  // of 32 bytes of K
                    for (int j = 0; j < steps; ++j)
                        mma<CG, FP8>(tmem + acc * kAccStride, a + 2 * j, b + 2 * j, idesc, kb + j > 0);
                    commit<CG>(empty + 8 * s);
                }
                if (ok) commit<CG>(acc_full + 8 * acc);
            }
        }
    } else if constexpr (!WORDS) {  // ---- copies
        if (lane == 0) {
            int it = 0;
            bool ok = true;
            for (int t = first; t < total && ok; t += step) {
                const Tile tile = tile_at(A, t);
                const int row = (tile.m * CG + (int)rank) * kRows, col = tile.n * A.tile_n + (int)rank * w_rows;
                for (int kb = 0; kb < A.k_blocks; ++kb, ++it) {
                    const int s = it % stages;
                    ok = wait(empty + 8 * s, ((it / stages) & 1) ^ 1, abort, A.status, CB_DEV_PRODUCER_TIMEOUT);
                    if (!ok) break;
                    if (rank == 0) mbar_expect_tx(full + 8 * s, CG * stage_bytes);
                    const uint32_t bar = CG == 2 ? in_first(full + 8 * s) : full + 8 * s;
                    const uint32_t dst = ring + s * stage_bytes;
                    tma_2d<CG>(dst, &A.x_map, kb * kSlab, row, bar);
                    tma_2d<CG>(dst + kRows * kSlab, &A.w_map, kb * kSlab, col, bar);
                }
            }
            // the stages' last fills have been read, so no copy and no arrival is still under way
            for (int i = max(0, it - stages); i < it; ++i)
                if (!wait(empty + 8 * (i % stages), (i / stages) & 1, abort, A.status, CB_DEV_DRAIN_TIMEOUT)) {
                    const unsigned long long t0 = now_ns();  // given up: copies under way land in microseconds
                    while (now_ns() - t0 < kMinDrainNs) {}
                    break;
                }
        }
    } else {
        const int lw = warp - 5;
        int it = 0;
        bool ok = true;
        for (int t = first; t < total && ok; t += step) {
            const Tile tile = tile_at(A, t);
            const int row0 = tile.m * kRows, col0 = tile.n * A.tile_n;
            for (int kb = 0; kb < A.k_blocks; ++kb, ++it) {
                const int s = it % stages;
                ok = __all_sync(0xFFFFFFFFu, wait(empty + 8 * s, ((it / stages) & 1) ^ 1, abort, A.status,
                                                  CB_DEV_PRODUCER_TIMEOUT));
                if (!ok) break;
                uint8_t* const stage = base + s * stage_bytes;
                const int n = min(kSlab, A.k_bytes - kb * kSlab);
                constexpr int B = 4;  // rows whose loads are in flight together
                for (int r0 = lw * B; r0 < kRows + w_rows; r0 += kLoadWarps * B) {
                    uint32_t lo[B], hi[B];
                    int shift[B];
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        const int r = r0 + i;
                        const bool is_x = r < kRows;
                        const int at = is_x ? row0 + r : col0 + r - kRows;
                        const bool on = at < (is_x ? A.M : A.N);
                        const char* p = reinterpret_cast<const char*>(is_x ? A.x : A.w) +
                                        at * (is_x ? A.x_row : A.w_row) + (long long)kb * kSlab;
                        shift[i] = (int)((uintptr_t)p & 3);
                        lo[i] = on ? word_of(p, n, lane) : 0;
                        hi[i] = on && lane == 31 && shift[i] ? word_of(p, n, 32) : 0;
                    }
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        const int r = r0 + i;
                        const uint32_t next = __shfl_down_sync(0xFFFFFFFFu, lo[i], 1);
                        const uint32_t v = __funnelshift_r(lo[i], lane == 31 ? hi[i] : next, 8 * shift[i]);
                        *reinterpret_cast<uint32_t*>(stage + r * kSlab + ((lane / 4) ^ (r & 7)) * 16 + (lane % 4) * 4) = v;
                    }
                }
                fence_generic_to_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(full + 8 * s);
            }
        }
        for (int i = max(0, it - stages); i < it; ++i)
            wait(empty + 8 * (i % stages), (i / stages) & 1, abort, A.status, CB_DEV_DRAIN_TIMEOUT);
    }
    fence_before();
    __syncwarp();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();  // no CTA leaves while the other may still reach its barriers or TMEM
    fence_after();
    if (warp == 4) {
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

using Kernel = void (*)(LinearArgs);
Kernel kernel_of(int cg, bool fp8, bool words) {
    if (words) return fp8 ? linear_kernel<1, true, true> : linear_kernel<1, false, true>;
    if (cg == 2) return fp8 ? linear_kernel<2, true, false> : linear_kernel<2, false, false>;
    return fp8 ? linear_kernel<1, true, false> : linear_kernel<1, false, false>;
}

}  // namespace

size_t linear_stage_bytes(int cg, int tile_n) { return (size_t)(kRows + tile_n / cg) * kSlab; }

int linear_max_stages(size_t smem, size_t stage_bytes) {
    const size_t room = smem - sizeof(Tail) - 1024;
    const int n = (int)(room / stage_bytes);
    return n < kMaxLinStages ? n : kMaxLinStages;
}

cudaError_t prepare_linear(size_t smem, int* pairs) {
    for (int k = 0; k < 6; ++k) {
        const cudaError_t e = cudaFuncSetAttribute(kernel_of(k / 2 == 1 ? 2 : 1, k % 2 == 1, k / 2 == 2),
                                                   cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    // pairs of CTAs that run at once
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim.x = 2, at.val.clusterDim.y = at.val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3(2);
    c.blockDim = dim3(192);
    c.dynamicSmemBytes = smem;
    c.attrs = &at;
    c.numAttrs = 1;
    return cudaOccupancyMaxActiveClusters(pairs, reinterpret_cast<const void*>(kernel_of(2, false, false)), &c);
}

cudaError_t launch_linear(const LinearArgs& a, int cg, bool fp8, bool words, int grid, cudaStream_t s) {
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = a.overlap;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = (unsigned)cg, at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t c{};
    c.gridDim = dim3((unsigned)grid);
    c.blockDim = dim3(words ? 32 * (5 + kLoadWarps) : 192);
    c.dynamicSmemBytes = (size_t)a.stages * linear_stage_bytes(cg, a.tile_n) + sizeof(Tail) + 1024;
    c.stream = s;
    c.attrs = at;
    c.numAttrs = cg == 2 ? 2 : 1;
    void* args[] = {const_cast<void*>(static_cast<const void*>(&a))};
    const cudaError_t e = cudaLaunchKernelExC(&c, reinterpret_cast<const void*>(kernel_of(cg, fp8, words)), args);
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e;
}

}  // namespace cbk
