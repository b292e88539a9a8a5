// Internal: the matrix product of cb_linear_run on the fifth-generation tensor cores (linear_tc_*.cu).
//
// A persistent grid of CTAs (CG = 1) or of pairs of CTAs on two SMs (CG = 2) works through output tiles of 128 CG
// rows by tile_n columns. In a CTA
//   one warp fills a ring of stages by TMA with slabs of 128 bytes of K: 128 rows of x and tile_n / CG rows of w, in
//     the 128-byte swizzle that the tensor cores read,
//   one thread issues tcgen05.mma on them, sums in TMEM (two accumulators of up to 256 columns each),
//   eight or sixteen warps take a finished accumulator out of TMEM while the next tile is summed, and apply the epilogue.
// A pair of CTAs shares one tile: each loads its 128 rows of x and half of the tile's rows of w, the first one's
// thread issues for both, and each holds the sums of its own rows.
//
// Operands whose rows do not start on 16-byte boundaries cannot come by TMA; linear_pack.cu copies them onto the grid first.
//
// The tensor cores cut off what a sum loses where it is added to, which adds up over K: 1.1e-9 K of a result (bf16, signs mixed; 1.9e-5
// at K = 16384, 2.1e-6 at 2048), up to 6e-9 K where all terms have one sign. Results in fp32, and all of very long sums, are
// therefore summed in passes over parts of K, whose sums the epilogue's warps add, rounded to nearest, into a third part of TMEM
// while the next pass is under way (A.passes > 1, tiles of up to 128 columns).
//
// Few tiles of long sums are split over K (A.parts): each part's sums leave in fp32, and linear_join.cu adds them.
//
// Bound by the tensor cores where tiles fill the SMs' rounds: GB300, 4608 x 3072 x 15360 bf16 with a gated hidden state 264 us (1.65
// PFLOP/s, 85 % of the largest library rate), 8192 x 1152 x 4608 65 us (1.34), 4096 x 4608 x 1152 e4m3 with GELU 22.5 us (1.93).
//
// Every wait has a limit (A.wait_ns); one that runs out sets the CTA's abort flag, so that all its roles leave, after
// the copies under way have landed, and frees the TMEM.
#pragma once

#include <type_traits>

#include "cb_async.cuh"
#include "linear.cuh"
#include "linear_shift.cuh"

namespace cbk {
namespace {

constexpr int kRows = 128;        // rows of x per CTA
constexpr int kSlab = 128;        // bytes of K per stage
constexpr int kAccStride = 256;   // TMEM columns from one accumulator to the other (half of it where there are passes)
// Warps of the epilogue: two for each quarter of the TMEM lanes, or four where the threads load and store the results themselves
// and wait for that (GB300, 8192 x 8191 x 512 bf16 with a gated fp32 hidden state: eight warps, 32 rows at once each, 282 us,
// sixteen, eight rows at once, 195).
__host__ __device__ constexpr int epi_warps(Results r) { return r == Results::kDirect ? 16 : 8; }
__host__ __device__ constexpr int linear_threads(Results r) { return 32 * (epi_warps(r) + 2); }
constexpr int kTurn = 32 * 32 * 4;  // bytes of an epilogue's warp to turn sums in, or two boxes of results

struct alignas(16) Tail {  // behind the stages and the epilogue's warps' kTurn each
    float cols[2][2 * kAccStride];  // scales and biases of a tile's columns (where the output leaves by TMA)
    uint64_t full[kMaxLinStages], empty[kMaxLinStages], acc_full[2], acc_empty[2], cols_full[2];
    uint64_t resid_full[epi_warps(Results::kHidden)][kMaxRing];
    uint32_t tmem;
    int abort;
};
constexpr int kTailBytes = (sizeof(Tail) + 1023) / 1024 * 1024;  // boxes of epilogue's hidden states follow

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
    // relaxed: what it orders are reads of TMEM (tcgen05.wait and fence); a release would wait for the warp's stores
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_bar) : "memory");
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

// What ends a wait: the CTA's abort flag, or the limit, which sets it and notes a code.
struct Limit {
    volatile int* abort;
    int* status;
    unsigned long long ns;
};

// Wait for a phase of a barrier, until the limit or the CTA's abort flag.
template <bool CLUSTER = false>
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, const Limit& limit, int code) {
    unsigned long long t0 = 0;
    while (true) {
        for (int i = 0; i < 64; ++i)
            if (CLUSTER ? try_wait_cluster(bar, parity) : mbar_try_wait(bar, parity)) return true;
        if (*limit.abort) return false;
        const unsigned long long t = now_ns();
        if (t0 == 0) t0 = t;
        if (t - t0 > limit.ns) {
            *limit.abort = 1;
            record(limit.status, code);
            return false;
        }
    }
}

__device__ __forceinline__ bool all(bool ok) { return __all_sync(0xFFFFFFFFu, ok) != 0; }

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

// Stores 32 columns of the warp's 32 rows.
__device__ __forceinline__ void tmem_store(uint32_t addr, const float* v) {
    const uint32_t* r = reinterpret_cast<const uint32_t*>(v);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
        "r"(addr)
        : "memory");
    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}

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

// True in one lane of the warp. The roles' loops are run by whole warps, so that what they compute stays in
// uniform registers (which the tensor cores' and copies' instructions take), and one lane issues.
__device__ __forceinline__ bool elected() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}

// v += what stands at addr, by halves.
__device__ __forceinline__ void tmem_add(uint32_t addr, float* v) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        uint32_t r[16];
        asm volatile(
            "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
            : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
              "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
            : "r"(addr + 16 * h));
        asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
        for (int i = 0; i < 16; ++i) v[16 * h + i] += __uint_as_float(r[i]);
    }
}

struct Tile {
    int m, n, part;
};
// Groups of eight rows of tiles, so that tiles worked on together share operands in L2; SPLIT: parts of K, one after the other.
template <bool SPLIT>
__device__ __forceinline__ Tile tile_at(const LinearArgs& A, int t) {
    const int part = SPLIT ? t % A.parts : 0;
    if (SPLIT) t /= A.parts;
    const int group = 8 * A.tiles_n, g = t / group, r = t - g * group;
    const int rows = min(8, A.tiles_m - 8 * g);
    return Tile{8 * g + r % rows, r / rows, part};
}

// A place in the ring of stages, and the parity of its present use.
struct Place {
    int s = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next(int stages) {
        if (++s == stages) s = 0, phase ^= 1;
    }
};

// Waits until the stages' last fills have been read: no copy and no arrival is under way then. `p`: the place behind
// them, `fills`: how many there were.
__device__ __forceinline__ bool drain(Place p, int fills, int stages, uint32_t empty, const Limit& limit) {
    for (int i = 0; i < min(fills, stages); ++i) {
        p.s = p.s == 0 ? (p.phase ^= 1, stages - 1) : p.s - 1;
        if (!wait(empty + 8 * p.s, p.phase, limit, CB_DEV_DRAIN_TIMEOUT)) return false;
    }
    return true;
}

// ---- epilogue of 32 rows by 32 columns of a warp (a chunk)

// Results by TMA: a row per lane, as the sums come from TMEM. Columns' scale and bias are read from shared memory by all lanes
// alike; hidden states come in and results leave in boxes of 32 rows of 64 bytes (a chunk of 32 columns is one of bf16 or two of
// fp32), swizzled by 64 bytes.

__device__ __forceinline__ uint32_t piece_at(uint32_t box, int lane, int j) { return box + lane * 64 + (j ^ (lane / 2 % 4)) * 16; }
__device__ __forceinline__ void store_box(const CUtensorMap* map, int x, int y, uint32_t box) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y), "r"(box)
                 : "memory");
}
__device__ __forceinline__ uint4 packed8(const Two* x) {
    const float2 a = both(x[0]), b = both(x[1]), c = both(x[2]), d = both(x[3]);
    return make_uint4(bf16x2(a.x, a.y), bf16x2(b.x, b.y), bf16x2(c.x, c.y), bf16x2(d.x, d.y));
}
__device__ __forceinline__ uint4 as_uint4(Two a, Two b) {
    const float2 f = both(a), g = both(b);
    return make_uint4(__float_as_uint(f.x), __float_as_uint(f.y), __float_as_uint(g.x), __float_as_uint(g.y));
}
__device__ __forceinline__ void st_shared16(uint32_t at, uint4 v) {
    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// Two bf16 values of a word.
__device__ __forceinline__ Two widened(uint32_t w) { return two(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }

// The 32 sums of a lane's row to values.
template <int ACT>
__device__ __forceinline__ void values(const LinearEpilogue& E, const float* cols, Two xs2, const float* v, Two* x) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const ulonglong2 s = *reinterpret_cast<const ulonglong2*>(cols + 4 * j);
        const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(cols + kAccStride + 4 * j);
        Two p = two(v[4 * j], v[4 * j + 1]), q = two(v[4 * j + 2], v[4 * j + 3]);
        if (E.x_scale) p = mul2(p, xs2), q = mul2(q, xs2);
        x[2 * j] = fma2(p, s.x, b.x);
        x[2 * j + 1] = fma2(q, s.y, b.y);
        if (j % 4 == 3) lin_act_all<ACT, 8>(x + 2 * j - 6);
    }
}

// A box's worth of values (16 of fp32, 32 of bf16) into shared memory.
template <bool BF16>
__device__ __forceinline__ void put_box(uint32_t box, int lane, const Two* x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) st_shared16(piece_at(box, lane, j), BF16 ? packed8(x + 4 * j) : as_uint4(x[2 * j], x[2 * j + 1]));
}

// The gate of 32 columns as it lies in memory, `row` being this lane's sample's, and its values (1 where there is none). N gates
// are whole pieces of 16 bytes.
__device__ __forceinline__ void look_gate(const LinearEpilogue& E, const char* row, int col, uint4* raw) {
    if (!E.gate) return;
    const int step = E.gate_bf16 ? 8 : 4;
#pragma unroll
    for (int j = 0; j < 8; ++j) raw[j] = ld16_if(row + col * (16 / step) + 16 * j, step * j < 32 && col + step * j < E.N);
}
__device__ __forceinline__ void gate_pairs(const LinearEpilogue& E, const uint4* raw, Two* g) {
    if (!E.gate) {
#pragma unroll
        for (int j = 0; j < 16; ++j) g[j] = two(1.0f, 1.0f);
    } else if (E.gate_bf16) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            g[4 * j] = widened(raw[j].x), g[4 * j + 1] = widened(raw[j].y), g[4 * j + 2] = widened(raw[j].z), g[4 * j + 3] = widened(raw[j].w);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            g[2 * j] = two(__uint_as_float(raw[j].x), __uint_as_float(raw[j].y)),
            g[2 * j + 1] = two(__uint_as_float(raw[j].z), __uint_as_float(raw[j].w));
    }
}

// The hidden state in a box plus gate times x, in place.
template <bool BF16>
__device__ __forceinline__ void add_box(uint32_t box, int lane, const Two* gate, const Two* x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t at = piece_at(box, lane, j);
        const uint4 r = ld_shared16(at);
        if constexpr (BF16) {
            const Two h[4] = {fma2(gate[4 * j], x[4 * j], widened(r.x)), fma2(gate[4 * j + 1], x[4 * j + 1], widened(r.y)),
                              fma2(gate[4 * j + 2], x[4 * j + 2], widened(r.z)), fma2(gate[4 * j + 3], x[4 * j + 3], widened(r.w))};
            st_shared16(at, packed8(h));
        } else {
            st_shared16(at, as_uint4(fma2(gate[2 * j], x[2 * j], two(__uint_as_float(r.x), __uint_as_float(r.y))),
                                     fma2(gate[2 * j + 1], x[2 * j + 1], two(__uint_as_float(r.z), __uint_as_float(r.w)))));
        }
    }
}

// Results by the threads, for rows off the 16-byte grid: a column per lane, eight rows at a time, whose hidden states are loaded
// while the eight before are worked on.

struct Column {  // of a lane
    float scale, bias, gate;  // gate: of the warp's first row's sample
};

__device__ __forceinline__ Column look_column(const LinearEpilogue& E, int row0, int col) {
    Column k{1.0f, 0.0f, 1.0f};
    if (col >= E.N) return k;
    if (E.w_scale) k.scale = __uint_as_float(lin_ld1(E.w_scale, col, 0));
    if (E.bias) k.bias = __uint_as_float(lin_ld1(E.bias, col, E.bias_bf16));
    if (E.gate) k.gate = __uint_as_float(lin_ld1(E.gate, ((unsigned)row0 / E.tokens) * E.gate_stride + col, E.gate_bf16));
    return k;
}

__device__ __forceinline__ void look_rows(const LinearEpilogue& E, int row, int col, uint32_t* r) {
    if (!E.resid_out || col >= E.N) return;
    const int es = E.resid_bf16 ? 2 : 4;
    const char* q = reinterpret_cast<const char*>(E.resid) + (row * E.resid_stride + col) * es;
    const long long step = E.resid_stride * es;
#pragma unroll
    for (int i = 0; i < 8; ++i, q += step)
        if (row + i < E.M) r[i] = lin_ld1(q, 0, E.resid_bf16);
}

__device__ __forceinline__ void put_rows(const LinearEpilogue& E, void* p, long long stride, int bf16, int row, int col, const float* v) {
    const int es = bf16 ? 2 : 4;
    char* q = reinterpret_cast<char*>(p) + (row * stride + col) * es;
    const long long step = stride * es;
#pragma unroll
    for (int i = 0; i < 8; ++i, q += step)
        if (row + i < E.M) lin_put1(q, 0, bf16, v[i]);
}

template <int ACT>
__device__ __forceinline__ void activate(const Column& k, float* v) {
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const float2 f = both(lin_act<ACT>(fma2(two(v[i], v[i + 1]), two(k.scale, k.scale), two(k.bias, k.bias))));
        v[i] = f.x, v[i + 1] = f.y;
    }
}

// Eight rows from `row` on (row0: the warp's first).
__device__ __forceinline__ void finish_rows(const LinearEpilogue& E, int row0, int row, int col, const Column& k, const uint32_t* r, float* v) {
    if (col >= E.N) return;
    if (E.act == CB_ACT_NONE) activate<CB_ACT_NONE>(k, v);
    else if (E.act == CB_ACT_GELU) activate<CB_ACT_GELU>(k, v);
    else activate<CB_ACT_SILU>(k, v);
    if (E.out) put_rows(E, E.out, E.out_stride, E.out_bf16, row, col, v);
    if (!E.resid_out) return;
    const unsigned next = ((unsigned)row0 / E.tokens + 1) * E.tokens;  // rows from here on belong to other samples
    if (!E.gate || (unsigned)row + 7 < next) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(k.gate, v[i], __uint_as_float(r[i]));
    } else {
        for (int i = 0; i < 8; ++i) {
            const unsigned at = (unsigned)min(row + i, E.M - 1) / E.tokens;
            const float g = __uint_as_float(lin_ld1(E.gate, at * E.gate_stride + col, E.gate_bf16));
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (i == j) v[j] = fmaf(g, v[j], __uint_as_float(r[j]));
        }
    }
    put_rows(E, E.resid_out, E.resid_out_stride, E.resid_bf16, row, col, v);
}

template <int CG, bool FP8, bool PASSES, Results RESULTS>
__global__ void __launch_bounds__(linear_threads(RESULTS), 1) linear_kernel(const __grid_constant__ LinearArgs A) {
    constexpr int EPI = epi_warps(RESULTS);
    constexpr bool DIRECT = RESULTS == Results::kDirect, HIDDEN = RESULTS == Results::kHidden, SPLIT = RESULTS == Results::kOut;
    extern __shared__ __align__(1024) uint8_t base[];
    if (smem_addr(base) & 1023) {  // the swizzle goes by addresses
        after_previous();
        if (threadIdx.x == 0) record(A.status, CB_DEV_PLACEMENT);
        return;
    }
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int w_rows = A.tile_n / CG, stage_bytes = (kRows + w_rows) * kSlab, stages = A.stages;
    uint8_t* const turns = base + stages * stage_bytes;
    Tail& T = *reinterpret_cast<Tail*>(turns + EPI * kTurn);
    const uint32_t ring = smem_addr(base);
    const uint32_t full = smem_addr(T.full), empty = smem_addr(T.empty);
    const uint32_t acc_full = smem_addr(T.acc_full), acc_empty = smem_addr(T.acc_empty);
    const Limit limit{&T.abort, A.status, A.wait_ns};

    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) {
            mbar_init(full + 8 * s, 1);
            mbar_init(empty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(acc_full + 8 * i, 1);
            mbar_init(acc_empty + 8 * i, EPI * CG);
            mbar_init(smem_addr(T.cols_full) + 8 * i, EPI);
        }
        for (int i = 0; HIDDEN && i < EPI * kMaxRing; ++i) mbar_init(smem_addr(T.resid_full) + 8 * i, 1);
        *limit.abort = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_generic_to_async();
    }
    if (warp == EPI) {
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

    const int first = blockIdx.x / CG, step = gridDim.x / CG, total = A.tiles_m * A.tiles_n * (SPLIT ? A.parts : 1);
    // slabs of a part of K
    auto slabs_from = [&](int part) { return SPLIT ? part * A.part_blocks : 0; };
    auto slabs_to = [&](int part) { return SPLIT ? min((part + 1) * A.part_blocks, A.k_blocks) : A.k_blocks; };
    if (warp < EPI) {  // ---- epilogue
        const LinearEpilogue E = from_here(A.e);
        float* const turn = reinterpret_cast<float*>(turns + warp * kTurn);
        const int quarter = warp % 4, half = warp / 4;  // this warp's rows, and its share of their chunks of 32 columns
        int n_done = 0, pass = 0, n_boxes = 0;  // tiles, and accumulators, taken
        auto first_row = [&](const Tile& tile) { return (tile.m * CG + (int)rank) * kRows + quarter * 32; };
        // The operands of a tile that do not depend on its sums are loaded a tile ahead: the scale of this lane's row, and
        // where the output leaves by TMA a column's scale and bias by each thread, which the warps then share.
        float xs = 1.0f, scale = 1.0f, bias = 0.0f;
        auto look_tile = [&](int t) {
            if (t >= total) return;
            const Tile tile = tile_at<SPLIT>(A, t);
            const int row = first_row(tile) + lane, col = tile.n * A.tile_n + (int)threadIdx.x;
            if (E.x_scale && row < E.M) xs = __uint_as_float(lin_ld1(E.x_scale, row, 0));
            if (DIRECT || (int)threadIdx.x >= A.tile_n || col >= E.N) return;
            if (E.w_scale) scale = __uint_as_float(lin_ld1(E.w_scale, col, 0));
            if (E.bias) bias = __uint_as_float(lin_ld1(E.bias, col, E.bias_bf16));
        };
        // The hidden state's rows of a tile are on their way to L2 a tile ahead.
        auto to_l2 = [&](int t) {
            if (RESULTS == Results::kOut || !E.resid_out || t >= total) return;
            const Tile tile = tile_at<SPLIT>(A, t);
            const int row = first_row(tile) + lane, col0 = tile.n * A.tile_n, es = E.resid_bf16 ? 2 : 4;
            if (row >= E.M) return;
            const char* const q = reinterpret_cast<const char*>(E.resid) + (row * E.resid_stride + col0) * es;
            const int bytes = min(A.tile_n, E.N - col0) * es;
            for (int b = 128 * half; b < bytes; b += 128 * (EPI / 4)) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + b));
        };
        // Boxes of 2 KB of this warp: the output's, then the ring's, the first two in `turn`.
        const uint32_t turn_at = smem_addr(turn), more_at = smem_addr(&T) + kTailBytes + warp * A.more_boxes * kBox;
        auto box_at = [&](int i) { return i < 2 ? turn_at + i * kBox : more_at + (i - 2) * kBox; };
        const int out_boxes = E.out ? (E.out_bf16 ? 1 : 2) : 0, resid_boxes = E.resid_bf16 ? 1 : 2;
        auto ring_box = [&](int slot, int i = 0) { return box_at(out_boxes + slot * resid_boxes + i); };
        // Hidden states are fetched A.ring - 1 of this warp's chunks ahead; `n_chunks` of them are done.
        int n_chunks = 0, n_fetched = 0;
        Place held, fetched;
        int f_tile = first - step, f_chunk = 0, f_chunks = 0, f_row = 0, f_col = 0;
        auto fetch = [&](int upto) {
            for (; n_fetched <= upto; ++n_fetched) {
                f_chunk += EPI / 4;
                while (f_chunk >= f_chunks) {
                    if ((f_tile += step) >= total) return;
                    const Tile tile = tile_at<SPLIT>(A, f_tile);
                    f_row = first_row(tile), f_col = tile.n * A.tile_n;
                    f_chunks = f_row < E.M ? (min(A.tile_n, E.N - f_col) + 31) / 32 : 0;
                    f_chunk = half;
                }
                const int slot = fetched.s;
                const uint32_t bar = smem_addr(T.resid_full[warp]) + 8 * slot;
                fetched.next(A.ring);
                if (elected()) {
                    const int x = (f_col + f_chunk * 32) * (E.resid_bf16 ? 2 : 4);
                    mbar_expect_tx(bar, resid_boxes * kBox);
                    tma_2d<1>(ring_box(slot), &A.resid_map, x, f_row, bar);
                    if (!E.resid_bf16) tma_2d<1>(ring_box(slot, 1), &A.resid_map, x + 64, f_row, bar);
                }
                __syncwarp();
            }
        };
        look_tile(first);
        to_l2(first);
        if (HIDDEN) fetch(A.ring - 2);
        for (int t = first; t < total; t += step, ++n_done) {
            const Tile tile = tile_at<SPLIT>(A, t);
            const int row0 = first_row(tile), col0 = tile.n * A.tile_n;
            const Two xs2 = two(xs, xs);
            const int chunks = row0 < E.M ? (min(A.tile_n, E.N - col0) + 31) / 32 : 0;
            const float* const cols = T.cols[n_done & 1];
            if (!DIRECT) {
                T.cols[n_done & 1][threadIdx.x] = scale, T.cols[n_done & 1][kAccStride + threadIdx.x] = bias;
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(T.cols_full) + 8 * (n_done & 1));
            }
            look_tile(t + step);
            to_l2(t + step);
            if (!DIRECT && !all(wait(smem_addr(T.cols_full) + 8 * (n_done & 1), (n_done >> 1) & 1, limit, CB_DEV_CONSUMER_TIMEOUT)))
                break;
            Column column;
            uint32_t rows_raw[8];
            if (DIRECT && half < chunks) {
                column = look_column(E, row0, col0 + half * 32 + lane);
                look_rows(E, row0, col0 + half * 32 + lane, rows_raw);
            }
            const char* gate_row = nullptr;  // of this lane's row's sample
            uint4 gate_raw[8];
            if (HIDDEN && half < chunks) {
                gate_row = reinterpret_cast<const char*>(E.gate) +
                           (unsigned)min(row0 + lane, E.M - 1) / E.tokens * E.gate_stride * (E.gate_bf16 ? 2 : 4);
                look_gate(E, gate_row, col0 + half * 32, gate_raw);
            }
            const uint32_t lanes = tmem + ((uint32_t)(quarter * 32) << 16), total_at = lanes + 256;
            constexpr int stride = PASSES ? kAccStride / 2 : kAccStride;
            auto release = [&] {  // the warp has read its part of the accumulator
                fence_before();
                __syncwarp();
                if (lane == 0) {
                    if constexpr (CG == 1) mbar_arrive(acc_empty + 8 * (pass & 1));
                    else arrive_at(in_first(acc_empty + 8 * (pass & 1)));
                }
                ++pass;
            };
            bool ok = true;
            const int passes = PASSES ? (slabs_to(tile.part) - slabs_from(tile.part) + A.pass_blocks - 1) / A.pass_blocks : 1;
            for (int i = 0; PASSES && i + 1 < passes; ++i) {  // all but the last one's sums are added up
                ok = all(wait(acc_full + 8 * (pass & 1), (pass >> 1) & 1, limit, CB_DEV_CONSUMER_TIMEOUT));
                if (!ok) break;
                fence_after();
                for (int c = half; c < chunks; c += EPI / 4) {
                    float v[32];
                    tmem_load(lanes + (pass & 1) * stride + c * 32, v);
                    if (i > 0) tmem_add(total_at + c * 32, v);
                    tmem_store(total_at + c * 32, v);
                }
                release();
            }
            if (!ok || !all(wait(acc_full + 8 * (pass & 1), (pass >> 1) & 1, limit, CB_DEV_CONSUMER_TIMEOUT))) break;
            fence_after();
            const uint32_t acc_at = lanes + (pass & 1) * stride;
            if (half >= chunks) release();
            for (int c = half; c < chunks; c += EPI / 4) {
                Two gate[16];
                if (HIDDEN) {
                    gate_pairs(E, gate_raw, gate);
                    if (c + EPI / 4 < chunks) look_gate(E, gate_row, col0 + (c + EPI / 4) * 32, gate_raw);
                }
                float v[32];
                tmem_load(acc_at + c * 32, v);
                if (PASSES && passes > 1) tmem_add(total_at + c * 32, v);
                if (c + EPI / 4 >= chunks) release();
                if constexpr (!DIRECT) {
                    Two x[16];
                    if (E.act == CB_ACT_NONE) values<CB_ACT_NONE>(E, cols + c * 32, xs2, v, x);
                    else if (E.act == CB_ACT_GELU) values<CB_ACT_GELU>(E, cols + c * 32, xs2, v, x);
                    else values<CB_ACT_SILU>(E, cols + c * 32, xs2, v, x);
                    const int col = col0 + c * 32;
                    if constexpr (!HIDDEN) {
                        for (int h = 0; h < out_boxes; ++h) {
                            // the box before the last has left
                            asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                            __syncwarp();
                            const uint32_t box = box_at(n_boxes++ & 1);
                            if (E.out_bf16) put_box<true>(box, lane, x);
                            else if (h == 0) put_box<false>(box, lane, x);
                            else put_box<false>(box, lane, x + 8);
                            fence_generic_to_async();
                            __syncwarp();
                            if (lane == 0 && col + 16 * h < E.N) store_box(&A.out_map, (col + 16 * h) * (E.out_bf16 ? 2 : 4), row0 + tile.part * A.part_rows, box);
                            asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                        }
                    } else {
                        ok = all(wait(smem_addr(T.resid_full[warp]) + 8 * held.s, held.phase, limit, CB_DEV_CONSUMER_TIMEOUT));
                        if (!ok) break;
                        const uint32_t box = ring_box(held.s), box2 = ring_box(held.s, 1);
                        if (E.resid_bf16) add_box<true>(box, lane, gate, x);
                        else add_box<false>(box, lane, gate, x), add_box<false>(box2, lane, gate + 8, x + 8);
                        // the chunk before has left its boxes
                        asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                        __syncwarp();
                        fetch(n_chunks + A.ring - 1);
                        if (E.out) {
                            if (E.out_bf16) put_box<true>(box_at(0), lane, x);
                            else put_box<false>(box_at(0), lane, x), put_box<false>(box_at(1), lane, x + 8);
                        }
                        ++n_chunks, held.next(A.ring);
                        fence_generic_to_async();
                        __syncwarp();
                        if (lane == 0) {
                            const bool more = col + 16 < E.N;
                            if (E.out) {
                                store_box(&A.out_map, col * (E.out_bf16 ? 2 : 4), row0, box_at(0));
                                if (!E.out_bf16 && more) store_box(&A.out_map, col * 4 + 64, row0, box_at(1));
                            }
                            store_box(&A.resid_out_map, col * (E.resid_bf16 ? 2 : 4), row0, box);
                            if (!E.resid_bf16 && more) store_box(&A.resid_out_map, col * 4 + 64, row0, box2);
                        }
                        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    }
                    continue;
                }
                // a row per lane to rows of 32 columns: 16-byte pieces, swizzled against bank conflicts
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    *reinterpret_cast<ulonglong2*>(&turn[lane * 32 + (j ^ (lane & 7)) * 4]) =
                        make_ulonglong2(mul2(two(v[4 * j], v[4 * j + 1]), xs2), mul2(two(v[4 * j + 2], v[4 * j + 3]), xs2));
                __syncwarp();
                const int col = col0 + c * 32 + lane, next_col = c + EPI / 4 < chunks ? col + EPI * 8 : E.N;
                const Column now = column;
                column = look_column(E, row0, next_col);
#pragma unroll 1
                for (int row = 0; row < 32; row += 8) {
                    uint32_t r[8];
                    float f[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        r[i] = rows_raw[i];
                        f[i] = turn[(row + i) * 32 + ((lane / 4) ^ i) * 4 + lane % 4];
                    }
                    look_rows(E, row0 + (row + 8) % 32, row + 8 < 32 ? col : next_col, rows_raw);
                    finish_rows(E, row0, row0 + row, col, now, r, f);
                }
                __syncwarp();
            }
            if (!ok) break;
        }
        for (; n_chunks < n_fetched; ++n_chunks, held.next(A.ring))  // given up: hidden states under way land first
            if (!all(wait(smem_addr(T.resid_full[warp]) + 8 * held.s, held.phase, limit, CB_DEV_DRAIN_TIMEOUT))) {
                const unsigned long long t0 = now_ns();
                while (now_ns() - t0 < kMinDrainNs) {}
                break;
            }
        asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
    } else if (warp == EPI) {  // ---- products
        if (rank == 0) {
            // fp32 sums; A and B bf16 (kind f16) or e4m3 (kind f8f6f4), both with K innermost; N / 8, M / 16
            const uint32_t idesc =
                1u << 4 | (FP8 ? 0u : 1u << 7 | 1u << 10) | (uint32_t)(A.tile_n / 8) << 17 | (uint32_t)(kRows * CG / 16) << 24;
            const uint64_t desc0 = operand_desc(ring);
            const int last_steps = (A.k_bytes - (A.k_blocks - 1) * kSlab + 31) / 32;  // of 32 bytes of K
            Place at;
            constexpr int stride = PASSES ? kAccStride / 2 : kAccStride;
            int pass = 0;
            bool ok = true;
            // (the slabs' loop is kept short: with passes opened and closed inside it, a slab took 260 clocks longer)
            for (int t = first; t < total && ok; t += step) {
                const int part = SPLIT ? t % A.parts : 0, to = slabs_to(part);
                for (int kb0 = slabs_from(part); kb0 < to && ok; ++pass) {
                    const int end = PASSES ? min(kb0 + A.pass_blocks, to) : to;
                    const uint32_t sums = tmem + (pass & 1) * stride;
                    ok = all(wait<CG == 2>(acc_empty + 8 * (pass & 1), ((pass >> 1) & 1) ^ 1, limit,
                                           CB_DEV_PRODUCER_TIMEOUT));
                    fence_after();
                    for (int kb = kb0; kb < end && ok; ++kb) {
                        const uint64_t a = desc0 + (uint32_t)(at.s * stage_bytes) / 16, b = a + kRows * kSlab / 16;
                        ok = all(wait(full + 8 * at.s, at.phase, limit, CB_DEV_CONSUMER_TIMEOUT));
                        if (!ok) break;
                        fence_after();
                        const int steps = kb + 1 < A.k_blocks ? 4 : last_steps;
                        if (elected()) {
                            mma<CG, FP8>(sums, a, b, idesc, kb > kb0);
                            if (steps > 1) mma<CG, FP8>(sums, a + 2, b + 2, idesc, true);
                            if (steps > 2) mma<CG, FP8>(sums, a + 4, b + 4, idesc, true);
                            if (steps > 3) mma<CG, FP8>(sums, a + 6, b + 6, idesc, true);
                            commit<CG>(empty + 8 * at.s);
                            if (kb + 1 == end) commit<CG>(acc_full + 8 * (pass & 1));
                        }
                        at.next(stages);
                    }
                    kb0 = end;
                }
            }
        }
    } else {  // ---- operands
        Place at;
        int fills = 0;
        bool ok = true;
        const uint32_t bar0 = CG == 2 ? in_first(full) : full;
        const uint32_t announced = CG * stage_bytes + A.withheld;
        for (int t = first; t < total && ok; t += step) {
            const Tile tile = tile_at<SPLIT>(A, t);
            const int row = (tile.m * CG + (int)rank) * kRows, col = tile.n * A.tile_n + (int)rank * w_rows;
            for (int kb = slabs_from(tile.part), to = slabs_to(tile.part); kb < to; ++kb, ++fills) {
                ok = all(wait(empty + 8 * at.s, at.phase ^ 1, limit, CB_DEV_PRODUCER_TIMEOUT));
                if (!ok) break;
                const uint32_t dst = ring + at.s * stage_bytes;
                if (elected()) {
                    if (rank == 0) mbar_expect_tx(full + 8 * at.s, announced);
                    tma_2d<CG>(dst, &A.x_map, kb * kSlab, row, bar0 + 8 * at.s);
                    tma_2d<CG>(dst + kRows * kSlab, &A.w_map, kb * kSlab, col, bar0 + 8 * at.s);
                }
                at.next(stages);
            }
        }
        if (!drain(at, fills, stages, empty, limit)) {
            const unsigned long long t0 = now_ns();  // given up: copies under way land in microseconds
            while (now_ns() - t0 < kMinDrainNs) {}
        }
    }
    fence_before();
    __syncwarp();
    __syncthreads();
    if constexpr (CG == 2) cluster_sync();  // no CTA leaves while the other may still reach its barriers or TMEM
    fence_after();
    if (warp == EPI) {
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <Results RESULTS, bool PASSES>
LinearKernel kernel_of(int cg, bool fp8) {
    if (cg == 2) return fp8 ? linear_kernel<2, true, PASSES, RESULTS> : linear_kernel<2, false, PASSES, RESULTS>;
    return fp8 ? linear_kernel<1, true, PASSES, RESULTS> : linear_kernel<1, false, PASSES, RESULTS>;
}

}  // namespace
}  // namespace cbk
