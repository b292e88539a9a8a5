// cb_linear_*: the layer's handle, the checks of a call and the choice of its kernel.
#include <algorithm>
#include <atomic>
#include <new>

#include "linear.cuh"

namespace cbk {
namespace {

__device__ int g_linear_status[1];  // CB_DEV_* codes of this device's launches

bool wide_type(cb_dtype t) { return t == CB_BF16 || t == CB_FP32; }
size_t bytes_of(int t) { return t == CB_BF16 ? 2 : t == CB_FP32 ? 4 : 1; }
bool on_grid(const void* p, size_t a) { return (uintptr_t)p % a == 0; }

// What the calls need to know of a device, found out by the first one there.
struct Device {
    int sms, smem, pairs;
    int* status;
    cudaMemPool_t pool;  // for operands copied onto the 16-byte grid
};
// What the pool keeps from call to call: an allocation that maps memory anew takes longer than the product it is for.
constexpr unsigned long long kPoolKeeps = 1ull << 30;
std::atomic<const Device*> g_devices[kMaxStatusDevices];
using Encode = decltype(&cuTensorMapEncodeTiled);
std::atomic<Encode> g_encode;

cudaError_t make_pool(int device, cudaMemPool_t* pool) {
    cudaMemPoolProps props{};
    props.allocType = cudaMemAllocationTypePinned;
    props.location.type = cudaMemLocationTypeDevice;
    props.location.id = device;
    cudaError_t e = cudaMemPoolCreate(pool, &props);
    unsigned long long keeps = kPoolKeeps;
    if (e == cudaSuccess) e = cudaMemPoolSetAttribute(*pool, cudaMemPoolAttrReleaseThreshold, &keeps);
    return e;
}

// Layers that exist; the last one gives back what the pools keep.
std::atomic<long long> g_layers;

void give_back() {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // another stream may be captured
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    for (auto& d : g_devices)
        if (const Device* v = d.load(std::memory_order_acquire))
            if (cudaMemPoolTrimTo(v->pool, 0) != cudaSuccess) (void)cudaGetLastError();  // (the process may be ending)
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
}

int device_info(const Device** out) {
    int d = 0;
    cudaError_t e = cudaGetDevice(&d);
    if (e != cudaSuccess) return cuda_error(e, "cudaGetDevice");
    if (d >= kMaxStatusDevices) return CB_ERR_LIMIT;
    if ((*out = g_devices[d].load(std::memory_order_acquire))) return CB_OK;
    Device v{};
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;  // the first call may be one that is captured
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    e = cudaDeviceGetAttribute(&v.sms, cudaDevAttrMultiProcessorCount, d);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&v.smem, cudaDevAttrMaxSharedMemoryPerBlockOptin, d);
    if (e == cudaSuccess) e = cudaGetSymbolAddress(reinterpret_cast<void**>(&v.status), g_linear_status);
    if (e == cudaSuccess) e = prepare_linear((size_t)v.smem, &v.pairs);
    if (e == cudaSuccess) e = make_pool(d, &v.pool);
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult found{};
    if (e == cudaSuccess) e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &fn, 12000, cudaEnableDefault, &found);
    if (e == cudaSuccess && (!fn || found != cudaDriverEntryPointSuccess)) e = cudaErrorNotSupported;
    (void)cudaThreadExchangeStreamCaptureMode(&mode);
    if (e != cudaSuccess) return cuda_error(e, "linear set-up");
    g_encode.store(reinterpret_cast<Encode>(fn), std::memory_order_relaxed);
    const Device* mine = new (std::nothrow) Device(v);  // kept until the process ends
    if (!mine) return CB_ERR_LIMIT;
    const Device* none = nullptr;
    if (!g_devices[d].compare_exchange_strong(none, mine, std::memory_order_acq_rel)) {
        (void)cudaMemPoolDestroy(mine->pool);
        delete mine;
        mine = none;
    }
    *out = mine;
    return CB_OK;
}

// Copies of the operands that are not on the 16-byte grid (x, w: nullptr where they are) into `at`, in stream order; `pack` then
// tells where they lie.
size_t copies_bytes(const void* x, int M, const void* w, int N, int bytes) {
    const size_t row = (size_t)(bytes + 31) / 32 * 32;
    return ((x ? M * row : 0) + 255) / 256 * 256 + ((w ? N * row : 0) + 255) / 256 * 256;
}
cudaError_t make_copies(const void* x, long long x_row, int M, const void* w, long long w_row, int N, int bytes, char* at,
                        LinearPackArgs* pack, cudaStream_t s) {
    const unsigned chunks = (unsigned)(bytes + 31) / 32;
    if (x) pack->o[0] = {static_cast<const char*>(x), at, M, x_row, bytes, chunks};
    if (w) pack->o[1] = {static_cast<const char*>(w), at + copies_bytes(x, M, nullptr, 0, bytes), N, w_row, bytes, chunks};
    pack->overlap = 1;
    return launch_linear_pack(*pack, s);
}

// Rows of bytes, in boxes of `box` rows by `wide` bytes (128, or 64), swizzled by as much; behind the ends zeros come in
// and nothing goes out.
int operand_map(CUtensorMap* map, const void* p, long long rows, long long bytes, long long stride, int box, int wide = 128) {
    const cuuint64_t dims[2] = {(cuuint64_t)bytes, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
    const cuuint32_t boxes[2] = {(cuuint32_t)wide, (cuuint32_t)box}, steps[2] = {1, 1};
    const CUresult r = g_encode.load(std::memory_order_relaxed)(
        map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(p), dims, strides, boxes, steps,
        CU_TENSOR_MAP_INTERLEAVE_NONE, wide == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B,
        CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? CB_OK : cuda_error(cudaErrorInvalidValue, "tensor map");
}

// Boxes of shared memory of a warp, besides two, for hidden states in bf16 and fp32: [1] where sums are short, as the results are
// what takes the time then, [0] where they are long and stages are worth more. GB300, {1, 4} -> {4, 7}: 16384 x 8192 x 512 e4m3
// with a bf16 output and hidden state 178 -> 150 us, fp32 hidden state alone 212 -> 192; 8192 x 1152 x 4608 64.1 -> 66.2 ({2, 5}).
constexpr int kShortBlocks = 16, kMoreBoxes[2][2] = {{1, 4}, {4, 7}};

// Bytes of a row up to which a box's place in it (and a gate's piece's), and that of the box behind, is a positive int.
constexpr long long kMaxRowBytes = (1LL << 31) - 1024;

// Results and hidden states whose rows lie on the 16-byte grid go by TMA, in boxes of 32 rows by 64 bytes.
int results_by_tma(const cb_linear_io* io, LinearArgs* a) {
    const LinearEpilogue& e = a->e;
    a->results = Results::kDirect;
    const struct {
        const void* p;
        long long row, es;
        CUtensorMap* map;
    } used[] = {{e.out, e.out_stride, (long long)bytes_of(io->out_dtype), &a->out_map},
                {e.resid, e.resid_stride, (long long)bytes_of(io->resid_dtype), &a->resid_map},
                {e.resid_out, e.resid_out_stride, (long long)bytes_of(io->resid_dtype), &a->resid_out_map}};
    for (const auto& u : used)
        if (u.p && (!on_grid(u.p, 16) || u.row * u.es % 16 != 0 || u.row * u.es >= 1LL << 40 || e.N * u.es > kMaxRowBytes)) return CB_OK;
    // a gate's pieces of 16 bytes are read whole
    const long long gs = (long long)bytes_of(io->gate_dtype);
    if (e.gate && (!on_grid(e.gate, 16) || e.gate_stride * gs % 16 != 0 || e.N * gs % 16 != 0 || e.N * gs > kMaxRowBytes)) return CB_OK;
    for (const auto& u : used) {
        if (!u.p) continue;
        const int rc = operand_map(u.map, u.p, e.M, e.N * u.es, u.row * u.es, 32, 64);
        if (rc != CB_OK) return rc;
    }
    a->results = e.resid_out ? Results::kHidden : Results::kOut;
    if (e.resid_out) {
        const int out = !e.out ? 0 : e.out_bf16 ? 1 : 2, resid = e.resid_bf16 ? 1 : 2;
        a->more_boxes = std::max(kMoreBoxes[a->k_blocks <= kShortBlocks][resid - 1], out + 2 * resid - 2);
        a->ring = (2 + a->more_boxes - out) / resid;
    }
    return CB_OK;
}

// Rows that linear_few.cu takes. GB300, w in L2, events around one call (about 8 us of them its own), linear_tc.cu ->
// linear_few.cu: 8 x 6912 x 1152 14.2 -> 10.7 us, 32 x 1152 x 4608 18.5 -> 13.2, 8 x 64 x 16384 45 -> 9.6; with 64 rows
// 6912 x 1152 13.2 -> 20.8, 1152 x 4608 18.6 -> 18.4, 12288 x 3072 20.3 -> 55.
constexpr int kFewRows = 32;

// Slabs of 128 bytes of a pass over K, with fp32 results: an error of 5e-7 of a sum, 7e-7 where all terms have one sign (measured:
// linear_tc.cuh; e4m3's products lose less, 1.4e-7 in 2048 features of one sign and 1.8e-6 in 8192; 4096 x 4608 x 8192 takes 104 us in two passes of
// narrower tiles and 89 in one).
constexpr int kPassBf16 = 8, kPassE4m3 = 32;
// Results in bf16 alone: one pass up to kOnePass slabs, as tiles of 256 columns are worth more (4608 x 3072 x 15360 227 -> 274 us, 8192 x
// 8192 x 8192 554 -> 648, 8192 x 1152 x 4608 60.2 -> 62.0 with passes of 16) and what the sums lose is small against the rounding that
// follows, 2e-3 to 4e-3: 7.2e-5 of their size at most (16384 features of bf16, all terms of one sign; 1.9e-5 with signs mixed). Longer sums
// in passes, as it grows with the length: 3.5e-4 at 65536, 6.5e-3 at 2^20.
constexpr int kOnePass = 256, kPassLong = 32;

// CTAs per tile, the tile's columns and the parts of K: the fewest rounds of tiles, each as long as its loads (16 KB of x and
// 16 KB * tile_n / 128 / cg of w per CTA and slab) or its products take, in clocks. Parts cost a launch that adds them, and
// their sums' way through L2. GB300, calls back to back, in one part and in the chosen ones: 256 x 1152 x 4608 bf16 with a gated
// hidden state 15.3 and 12.5 us, 77 x 1152 x 4096 13.3 and 9.4, 640 x 72 x 16384 41.8 and 12.7, 1500 x 300 x 12000 32.8 and 16.6;
// up to 16 parts of four slabs gave the same.
constexpr double kJoinClocks = 5000, kJoinBytesPerClock = 1300;
constexpr int kMaxParts = 8, kPartSlabs = 8;  // no part is shorter
void choose_tile(const Device& dev, int M, int N, int k_blocks, int most, int* cg, int* tile_n, int* parts) {
    double best = 1e300;
    for (int p = 1; p <= kMaxParts && (p == 1 || k_blocks / p >= kPartSlabs); ++p)
        for (int g = 2; g >= 1; --g)
            for (int n = most; n >= 32; n -= 32) {
                if (n > 32 && n - 32 >= N) continue;
                const long long tiles = (long long)((M + 128 * g - 1) / (128 * g)) * ((N + n - 1) / n) * p;
                const long long units = g == 2 ? dev.pairs : dev.sms;
                if (units < 1) break;  // no room for pairs
                if (p > 1 && tiles > units) break;  // smaller tiles are more
                const double join = p > 1 ? kJoinClocks + 4.0 * p * M * N / kJoinBytesPerClock : 0.0;
                const double cost = (double)((tiles + units - 1) / units) * ((k_blocks + p - 1) / p) * (256.0 + 2.0 * n / g) + join;
                if (cost < best * 0.999) best = cost, *cg = g, *tile_n = n, *parts = p;
            }
}

}  // namespace
}  // namespace cbk

struct cb_linear {
    cb_linear_desc d;
    unsigned long long wait_ns = 1000000000ull;
    unsigned withheld = 0;
};

extern "C" {

int cb_linear_create(const cb_linear_desc* d, cb_linear** out) {
    using namespace cbk;
    if (!out) return CB_ERR_ARG;
    *out = nullptr;
    if (!d || d->reserved != 0 || d->in_features < 1 || d->out_features < 1 || !d->w) return CB_ERR_ARG;
    if (d->type != CB_BF16 && d->type != CB_E4M3) return CB_ERR_ARG;
    if (d->bias && !wide_type(d->bias_dtype)) return CB_ERR_ARG;
    if (d->activation < CB_ACT_NONE || d->activation > CB_ACT_SILU) return CB_ERR_ARG;
    if (d->w_scale && d->type != CB_E4M3) return CB_ERR_ARG;
    if (d->w_stride != 0 && d->w_stride < d->in_features) return CB_ERR_ARG;
    const long long row = 0x7FFFFF00LL / (long long)bytes_of(d->type);
    if (d->out_features > 0x7FFFFC00LL || d->in_features > CB_MAX_IN_FEATURES || d->w_stride > row) return CB_ERR_LIMIT;
    if (!on_grid(d->w, bytes_of(d->type)) || !on_grid(d->w_scale, 4)) return CB_ERR_ALIGN;
    if (d->bias && !on_grid(d->bias, bytes_of(d->bias_dtype))) return CB_ERR_ALIGN;
    cb_linear* l = new (std::nothrow) cb_linear;
    if (!l) return CB_ERR_LIMIT;
    l->d = *d;
    if (l->d.w_stride == 0) l->d.w_stride = d->in_features;
    cbk::g_layers.fetch_add(1, std::memory_order_relaxed);
    *out = l;
    return CB_OK;
}

void cb_linear_destroy(cb_linear* l) {
    if (!l) return;
    delete l;
    if (cbk::g_layers.fetch_sub(1, std::memory_order_acq_rel) == 1) cbk::give_back();
}

int cb_linear_set_option(cb_linear* l, int option, int64_t value) {
    if (!l) return CB_ERR_ARG;
    switch (option) {
    case CB_OPT_WAIT_NS:
        if (value < 0 || value > 60000000000LL) return CB_ERR_ARG;
        l->wait_ns = (unsigned long long)value;
        return CB_OK;
    case CB_OPT_TEST_WITHHOLD:
        if (value != 0 && value != 1) return CB_ERR_ARG;
        l->withheld = 16 * (unsigned)value;
        return CB_OK;
    default: return CB_ERR_ARG;
    }
}

int cb_linear_run(const cb_linear* l, const cb_linear_io* io, const void* x, const float* x_scale, const void* resid,
                  const void* gate, void* out, void* resid_out, void* stream) {
    using namespace cbk;
    if (!l || !io || io->reserved != 0 || io->rows < 0 || io->tokens < 0) return CB_ERR_ARG;
    const cb_linear_desc& d = l->d;
    if (!wide_type(io->out_dtype) || !wide_type(io->resid_dtype) || !wide_type(io->gate_dtype)) return CB_ERR_ARG;
    const long long es = (long long)bytes_of(d.type), K = d.in_features, N = d.out_features;
    if (io->rows > 0x7FFFFC00LL) return CB_ERR_LIMIT;
    if (io->x_stride != 0 && io->x_stride < K) return CB_ERR_ARG;
    if (io->x_stride > 0x7FFFFF00LL / es) return CB_ERR_LIMIT;
    const int64_t strides[] = {io->out_stride, io->resid_stride, io->resid_out_stride, io->gate_stride};
    for (int64_t s : strides)
        if (s != 0 && (s < N || s > CB_MAX_NUMEL)) return s < N ? CB_ERR_ARG : CB_ERR_LIMIT;
    if (x_scale && d.type != CB_E4M3) return CB_ERR_ARG;
    if ((resid != nullptr) != (resid_out != nullptr) || (gate && !resid)) return CB_ERR_ARG;
    if (io->rows == 0) return CB_OK;
    if (!x || (!out && !resid_out)) return CB_ERR_ARG;

    LinearArgs a{};
    a.overlap = 1;
    a.k_bytes = (int)(K * es);
    const long long x_row = (io->x_stride ? io->x_stride : K) * es, w_row = d.w_stride * es;
    LinearEpilogue& ep = a.e;
    ep.M = (int)io->rows, ep.N = (int)N;
    ep.act = d.activation;
    ep.tokens = io->tokens == 0 || io->tokens > io->rows ? (unsigned)io->rows : (unsigned)io->tokens;
    ep.out_bf16 = io->out_dtype == CB_BF16, ep.resid_bf16 = io->resid_dtype == CB_BF16;
    ep.bias_bf16 = d.bias_dtype == CB_BF16, ep.gate_bf16 = io->gate_dtype == CB_BF16;
    ep.out_stride = io->out_stride ? io->out_stride : N;
    ep.resid_stride = io->resid_stride ? io->resid_stride : N;
    ep.resid_out_stride = io->resid_out_stride ? io->resid_out_stride : N;
    ep.gate_stride = io->gate_stride ? io->gate_stride : N;
    ep.x_scale = x_scale, ep.w_scale = d.w_scale, ep.bias = d.bias;
    ep.resid = resid, ep.gate = gate, ep.out = out, ep.resid_out = resid_out;
    if (!on_grid(x, es) || !on_grid(x_scale, 4)) return CB_ERR_ALIGN;
    const struct {
        const void* p;
        int dtype;
    } used[] = {{out, io->out_dtype}, {resid, io->resid_dtype}, {gate, io->gate_dtype}, {resid_out, io->resid_dtype}};
    for (const auto& u : used)
        if (u.p && !on_grid(u.p, bytes_of(u.dtype))) return CB_ERR_ALIGN;
    const Device* dev = nullptr;
    int rc = device_info(&dev);
    if (rc != CB_OK) return rc;
    a.status = dev->status, a.wait_ns = l->wait_ns, a.withheld = l->withheld;
    const bool x_on = on_grid(x, 16) && x_row % 16 == 0, w_on = on_grid(d.w, 16) && w_row % 16 == 0;
    if (ep.M <= kFewRows) {
        const LinearFewArgs f{ep, 1, a.k_bytes, x_row, w_row, x, d.w};
        const cudaError_t e = launch_linear_few(f, d.type == CB_E4M3, !x_on || !w_on, dev->sms, (cudaStream_t)stream);
        return e == cudaSuccess ? CB_OK : cuda_error(e, "linear launch");
    }
    int cg = 1;
    a.k_blocks = (a.k_bytes + 127) / 128;
    // fp32 results: passes over K (see linear_tc.cuh)
    const bool fp32 = (out && !ep.out_bf16) || (resid_out && !ep.resid_bf16);
    a.pass_blocks = fp32 ? (d.type == CB_BF16 ? kPassBf16 : kPassE4m3) : a.k_blocks > kOnePass ? kPassLong : a.k_blocks;
    choose_tile(*dev, ep.M, ep.N, a.k_blocks, a.k_blocks > a.pass_blocks ? 128 : 256, &cg, &a.tile_n, &a.parts);
    a.part_blocks = (a.k_blocks + a.parts - 1) / a.parts;
    a.parts = (a.k_blocks + a.part_blocks - 1) / a.part_blocks;
    a.passes = (a.part_blocks + a.pass_blocks - 1) / a.pass_blocks;
    a.tiles_m = (ep.M + 128 * cg - 1) / (128 * cg), a.tiles_n = (ep.N + a.tile_n - 1) / a.tile_n;
    if ((long long)a.tiles_m * a.tiles_n > 0x7FFFFFFFLL / 8) return CB_ERR_LIMIT;

    // memory for copies of operands and for the sums of parts, in stream order
    const cudaStream_t s = (cudaStream_t)stream;
    const void *const x_off = x_on ? nullptr : x, *const w_off = w_on ? nullptr : d.w;
    const size_t copies = copies_bytes(x_off, ep.M, w_off, ep.N, a.k_bytes);
    const long long row = (ep.N + 31) / 32 * 32;  // floats of a row of sums
    a.part_rows = a.tiles_m * 128 * cg;
    const size_t sums = a.parts > 1 ? (size_t)a.parts * a.part_rows * row * 4 : 0;
    void* space = nullptr;
    if (copies + sums) {
        const cudaError_t e = cudaMallocFromPoolAsync(&space, copies + sums, dev->pool, s);
        if (e != cudaSuccess) {
            (void)cudaGetLastError();  // returned here, so not left for a check of the caller's own launches
            return cuda_error(e, "linear workspace");
        }
    }
    LinearPackArgs pack{};
    LinearJoinArgs join{ep, 1, a.parts, (long long)a.part_rows * row, row, nullptr};
    cudaError_t e = cudaSuccess;
    if (copies) e = make_copies(x_off, x_row, ep.M, w_off, w_row, ep.N, a.k_bytes, static_cast<char*>(space), &pack, s);
    if (a.parts > 1) {
        join.sums = reinterpret_cast<const float*>(static_cast<char*>(space) + copies);
        ep = LinearEpilogue{ep.M, ep.N, CB_ACT_NONE, (unsigned)ep.M, 0, 0, 0, 0, row, 0, 0, 0, nullptr, nullptr, nullptr, nullptr, nullptr,
                            const_cast<float*>(join.sums), nullptr};
        a.results = Results::kOut;
        rc = operand_map(&a.out_map, join.sums, (long long)a.parts * a.part_rows, 4ll * ep.N, 4 * row, 32, 64);
    } else {
        rc = results_by_tma(io, &a);
    }
    const PackOperand &px = pack.o[0], &pw = pack.o[1];
    if (rc == CB_OK)
        rc = px.dst ? operand_map(&a.x_map, px.dst, ep.M, 32ll * px.chunks, 32ll * px.chunks, 128)
                    : operand_map(&a.x_map, x, ep.M, a.k_bytes, x_row, 128);
    if (rc == CB_OK)
        rc = pw.dst ? operand_map(&a.w_map, pw.dst, ep.N, 32ll * pw.chunks, 32ll * pw.chunks, a.tile_n / cg)
                    : operand_map(&a.w_map, d.w, ep.N, a.k_bytes, w_row, a.tile_n / cg);
    a.stages = (int)std::min<size_t>(kMaxLinStages, (dev->smem - linear_fixed_bytes(a.results, a.more_boxes)) / linear_stage_bytes(cg, a.tile_n));
    const long long tiles = (long long)a.tiles_m * a.tiles_n * a.parts, units = cg == 2 ? dev->pairs : dev->sms;
    if (rc == CB_OK && e == cudaSuccess) e = launch_linear(a, cg, d.type == CB_E4M3, cg * (int)std::min(tiles, units), s);
    if (rc == CB_OK && e == cudaSuccess && a.parts > 1) e = launch_linear_join(join, s);
    if (space) {
        const cudaError_t f = cudaFreeAsync(space, s);
        if (e == cudaSuccess) e = f;
    }
    return rc != CB_OK ? rc : e == cudaSuccess ? CB_OK : cuda_error(e, "linear launch");
}

int cb_linear_device_status(int* status, void* stream) {
    using namespace cbk;
    if (!status) return CB_ERR_ARG;
    const Device* dev = nullptr;
    const int rc = device_info(&dev);
    if (rc != CB_OK) return rc;
    // one kernel takes the word and clears it: between a copy and a memset another stream's product might note a code
    const cudaStream_t s = (cudaStream_t)stream;
    void* taken = nullptr;
    int v = 0;
    cudaError_t e = cudaMallocFromPoolAsync(&taken, sizeof v, dev->pool, s);
    if (e == cudaSuccess) {
        e = take_status(dev->status, static_cast<int*>(taken), s);
        if (e == cudaSuccess) e = cudaMemcpyAsync(&v, taken, sizeof v, cudaMemcpyDeviceToHost, s);
        const cudaError_t f = cudaFreeAsync(taken, s);
        if (e == cudaSuccess) e = f;
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(s);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();  // returned here
        return cuda_error(e, "linear status");
    }
    *status = v;
    return CB_OK;
}

}  // extern "C"
