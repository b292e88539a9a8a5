/*
 * chebboost_block.h — the full step's operators around the history, in the same
 * library: the norm that takes a block's hidden state with the last branch added,
 * and the matrix product whose epilogue makes a branch output and the new hidden
 * state (paper Sec. 3.1: B(x) = x + S(x) + C(x) + M(x), each branch a norm and
 * matrix products). Their results are what cb_cache_push stores.
 *
 * Conventions are those of chebboost.h: the caller owns every device buffer and
 * stream, work is enqueued on `stream` asynchronously, all arguments are
 * checked before anything is enqueued, and a negative status is an error
 * (cb_status_string, cb_last_error_message). No call but cb_linear_run, where it says so,
 * and cb_linear_device_status (4 bytes) allocates device memory.
 * Buffers given for output must not overlap inputs, but for the one pair that
 * each call names.
 *
 * Rows and samples: a call works on `rows` rows of [batch, tokens, features]
 * flattened; row r belongs to sample r / tokens, whose line of a gate, scale or
 * shift it uses.
 */
#ifndef CHEBBOOST_BLOCK_H
#define CHEBBOOST_BLOCK_H

#include "chebboost.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Sizes and types of cb_norm_residual. Strides are in elements from one row (or
 * sample) to the next; 0 means contiguous. */
typedef struct {
    int64_t rows;          /* >= 0; 0 does nothing */
    int64_t hidden;        /* >= 1 */
    int64_t tokens;        /* rows of one sample; 0: all rows are one sample */
    int64_t x_stride;
    int64_t branch_stride;
    int64_t x_out_stride;
    int64_t out_stride;
    int64_t line_stride;   /* from one sample's gate, scale and shift to the next's */
    cb_dtype x_dtype;      /* of x and x_out: CB_BF16 or CB_FP32 */
    cb_dtype branch_dtype; /* CB_BF16 or CB_FP32 */
    cb_dtype param_dtype;  /* of gate, weight, scale, shift: CB_BF16 or CB_FP32 */
    cb_dtype out_dtype;    /* CB_BF16, CB_FP32 or CB_E4M3 */
    float eps;             /* >= 0, finite */
    int32_t reserved;      /* must be 0 */
} cb_norm_desc;

/* Root-mean-square norm with the residual's addition: the norm of blocks that subtract no
 * mean (DiT-XL/2, PixArt-Sigma and FLUX.1-dev do: theirs is another). For every row
 *     h = x + gate * branch
 *     x_out = round(h)
 *     n = h / sqrt(mean(h^2) + eps) * weight
 *     y = n * (1 + scale) + shift
 * in fp32 (h enters the norm un-rounded), and out = y in bf16 or fp32, or
 *     out_scale = max(max |y| * fp32(1/448), 2^-126) of the row,
 *     out = y * fp32(1/out_scale) in e4m3, to nearest even,
 * so that out * out_scale stands for y. x, branch, x_out, out: rows of `hidden`
 * elements; gate, scale, shift: a line per sample; weight: one line; out_scale:
 * one float a row (CB_E4M3 only). branch, gate (with a branch only), weight,
 * scale, shift and x_out may be NULL: no addition, factors 1, terms 0, h not
 * stored. x_out may be x itself (same stride). With eps > 0 a row of zeros gives
 * zeros (with shift: its values). A row that holds a NaN gives NaN; one that holds an
 * infinity gives NaN in e4m3, otherwise NaN there and what zeros give elsewhere. No
 * other row is touched by either. Squares are summed in fp32: of a row with elements beyond
 * 2^63 the sum is infinite and n is zero.
 * Rows and hidden sizes on the 16-byte grid take vector loads, others elements.
 * Errors: CB_ERR_ARG, CB_ERR_ALIGN (a pointer off its element size), CB_ERR_LIMIT
 * (rows or hidden beyond 2^31 - 1), CB_ERR_CUDA. */
int cb_norm_residual(const cb_norm_desc* desc, const void* x, const void* branch, const void* gate,
                     const void* weight, const void* scale, const void* shift, void* x_out, void* out,
                     float* out_scale, void* stream);

/* Largest in_features: a sum that long takes a fraction of a wait's limit (cb_linear_run). */
#define CB_MAX_IN_FEATURES (1LL << 22)

/* Activations of a matrix product's epilogue, off by a few units in the last place of their own value however small (zero
 * below 2^-126 |v|); NaN at -infinity, as their quotients are. */
enum {
    CB_ACT_NONE = 0,
    CB_ACT_GELU = 1, /* v/2 (1 + tanh(sqrt(2/pi) (v + 0.044715 v^3))), the form of the blocks' MLPs */
    CB_ACT_SILU = 2  /* v / (1 + exp(-v)) */
};

/* A layer: what a program lays out once. w: [out_features, in_features] row-major
 * (w_stride elements from row to row, 0: contiguous), of `type`. */
typedef struct {
    int64_t in_features;   /* >= 1 */
    int64_t out_features;  /* >= 1 */
    int64_t w_stride;
    cb_dtype type;         /* of w and of the rows x: CB_BF16 or CB_E4M3 */
    cb_dtype bias_dtype;   /* CB_BF16 or CB_FP32 */
    int32_t activation;    /* CB_ACT_* */
    int32_t reserved;      /* must be 0 */
    const void* w;
    const float* w_scale;  /* CB_E4M3 only: [out_features] (NULL: 1) */
    const void* bias;      /* [out_features] (NULL: 0) */
} cb_linear_desc;

/* Sizes and types of one cb_linear_run. Strides are in elements; 0 means contiguous. */
typedef struct {
    int64_t rows;             /* >= 0; 0 does nothing */
    int64_t tokens;           /* rows of one sample; 0: all rows are one sample */
    int64_t x_stride;
    int64_t out_stride;
    int64_t resid_stride;
    int64_t resid_out_stride;
    int64_t gate_stride;      /* from one sample's gate to the next's */
    cb_dtype out_dtype;       /* CB_BF16 or CB_FP32 */
    cb_dtype resid_dtype;     /* of resid and resid_out: CB_BF16 or CB_FP32 */
    cb_dtype gate_dtype;      /* CB_BF16 or CB_FP32 */
    int32_t reserved;         /* must be 0 */
} cb_linear_io;

typedef struct cb_linear cb_linear; /* opaque, host-owned; holds no device memory */

/* Errors: CB_ERR_ARG, CB_ERR_ALIGN (a pointer off its element size), CB_ERR_LIMIT (out_features
 * beyond 2^31 - 1024, in_features beyond CB_MAX_IN_FEATURES, or a row stride of w or x
 * beyond 2^31 - 256 bytes). The layer keeps the pointers: its buffers must outlive it. */
int cb_linear_create(const cb_linear_desc* desc, cb_linear** out);
/* The process's last layer gives back the device memory that cb_linear_run keeps (what work under way still
 * uses stays until the next last one). NULL does nothing. */
void cb_linear_destroy(cb_linear* layer);

/* CB_OPT_WAIT_NS: limit of every wait of the layer's kernels on one of their barriers, ns (default 1e9, at most
 * 6e10). CB_OPT_TEST_WITHHOLD: 1: (tests of the failure path only) over 32 rows the kernels announce more
 * bytes of operands than they copy, so that the waits for them run out; results are then
 * invalid. Errors: CB_ERR_ARG. */
int cb_linear_set_option(cb_linear* layer, int option, int64_t value);

/* Matrix product with its epilogue. For every row m and output feature n
 *     v = act(x_scale[m] * w_scale[n] * sum_k x[m, k] w[n, k] + bias[n])
 *     out = round(v)                        the branch output, as cb_cache_push takes it
 *     resid_out = round(resid + gate * v)   the hidden state (gate: a line per sample)
 * with sums, epilogue and hidden state in fp32 and one rounding to each result. The
 * tensor cores cut sums off rather than round them: where a result is fp32 they sum
 * parts of 512 features (e4m3: 4096; up to 32 rows: 128 and 256 at most), which are added
 * rounded to nearest. Measured, in the root mean square relative to the sums': 5e-7 with signs
 * mixed, 8e-7 with all terms of one sign, and up to 2^-24 for every part added (of which most
 * cancel: 2^-24 times the root of their number). bf16 results: parts of 2048 (e4m3: 4096) where rows are longer
 * than 32 KB, else one part, which is off by up to 7.2e-5 (16384 features of one sign) before
 * the rounding to bf16.
 * x_scale: one float a row (CB_E4M3 only, NULL: 1). out may be NULL, resid and resid_out
 * may be NULL together, gate (with resid only) may be NULL: 1; one result at least
 * is wanted. resid_out may be resid itself (same stride). The order of a sum depends
 * on the sizes alone: equal calls give equal bits.
 * Over 32 rows, operands whose rows do not start on 16-byte boundaries are copied onto
 * them first, and few tiles of long sums are split over in_features, whose parts' sums a
 * second kernel adds in order. Memory for either is allocated and freed in stream order,
 * from a pool of the library's own that keeps 1 GiB at most between calls, until the last layer
 * is destroyed; in a graph it belongs to the graph. Where there is none left: CB_ERR_CUDA, and nothing has run.
 * Every wait of the kernels on one of their barriers has a limit (cb_linear_set_option); one that
 * runs out is noted in the status word of cb_linear_device_status and makes the
 * kernel return early, with incomplete results.
 * Errors: CB_ERR_ARG, CB_ERR_ALIGN, CB_ERR_LIMIT (rows beyond 2^31 - 1024, or over 2^28
 * tiles of 128 rows and 32 to 256 columns), CB_ERR_CUDA. */
int cb_linear_run(const cb_linear* layer, const cb_linear_io* io, const void* x, const float* x_scale,
                  const void* resid, const void* gate, void* out, void* resid_out, void* stream);

/* The status word of this device's matrix products (CB_DEV_* codes, 0: nothing noted since the last
 * read) into *status, and clear it, in one step: a code noted meanwhile by another stream's product is
 * left for the next read. Synchronises `stream`. Errors: CB_ERR_ARG, CB_ERR_LIMIT (a device beyond the
 * 64th), CB_ERR_CUDA. */
int cb_linear_device_status(int* status, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* CHEBBOOST_BLOCK_H */
