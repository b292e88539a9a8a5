/*
 * chebboost_block.h — the full step's operators around the history, in the same
 * library: the norms that take a block's hidden state with the last branch added,
 * the matrix product whose epilogue makes a branch output and the new hidden
 * state, and rows in 4 bits that go between them (paper Sec. 3.1: B(x) = x + S(x) + C(x) + M(x), each branch a norm and
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

/* Kinds of norm of cb_norm_around: none, root mean square, layer norm (less the mean first). */
enum {
    CB_NORM_NONE = 0,
    CB_NORM_RMS = 1,
    CB_NORM_LAYER = 2
};

/* Sizes and types of cb_norm_around. Strides are in elements from one row (or sample) to the next; 0 means
 * contiguous. */
typedef struct {
    int64_t rows;          /* >= 0; 0 does nothing */
    int64_t hidden;        /* >= 1 */
    int64_t tokens;        /* rows of one sample; 0: all rows are one sample */
    int64_t x_stride;
    int64_t branch_stride;
    int64_t x_out_stride;
    int64_t out_stride;    /* of an output in CB_MXFP4: a multiple of CB_MX_BLOCK */
    int64_t line_stride;   /* from one sample's gate, scale and shift to the next's */
    cb_dtype x_dtype;      /* of x and x_out: CB_BF16 or CB_FP32 */
    cb_dtype branch_dtype; /* CB_BF16 or CB_FP32 */
    cb_dtype param_dtype;  /* of all lines: CB_BF16 or CB_FP32 */
    cb_dtype out_dtype;    /* CB_BF16, CB_FP32, CB_E4M3 or CB_MXFP4 */
    int32_t after;         /* CB_NORM_* of the branch, after its block */
    int32_t before;        /* CB_NORM_* of the hidden state, before the next block */
    float after_eps;       /* >= 0, finite */
    float before_eps;      /* >= 0, finite */
    float x_factor;        /* finite; 1 where the residual is not scaled */
    float branch_factor;   /* finite; 1 where the branch is not scaled */
    int32_t reserved;      /* must be 0 */
} cb_norm_around_desc;

/* The norms around a block: the branch is normalised and added to the hidden state, and that is normalised
 * for the next branch, row by row:
 *     N(v) = v                                                  CB_NORM_NONE
 *            v / sqrt(mean(v^2) + eps)                          CB_NORM_RMS
 *            (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps)  CB_NORM_LAYER
 *     r = N_after(branch) * after_weight + after_bias
 *     h = x_factor * x + branch_factor * gate * r
 *     x_out = round(h)
 *     y = (N_before(h) * weight + bias) * (1 + scale) + shift
 * in fp32 (h enters its norm un-rounded; mean and squares in two passes), and out = y in bf16 or fp32, in e4m3
 * with a scale a row as cb_norm_residual makes it (out_scale: fp32 [rows]), or in 4 bits as cb_mx_quantize
 * makes it of fp32 rows (out_scale: its scales). It takes layer norms with a modulation (the adaptive ones
 * of diffusion transformers: before = CB_NORM_LAYER, scale, shift, gate) and blocks that are normed on
 * both sides. With CB_NORM_NONE after, no branch or eps = 0 the formulas hold as they stand.
 * x, branch, x_out, out: rows of `hidden` elements; gate, scale, shift: a line per sample; after_weight,
 * after_bias, weight, bias: one line. May be NULL: branch (then without gate, after_weight and after_bias, with
 * after = CB_NORM_NONE), each line (factors 1, terms 0), and x_out or out (with its scale). after_weight
 * and after_bias go with a norm after, weight and bias with one before, and scale and shift with an out. x_out may be
 * x itself (same stride). Rows that are not finite touch no others; in 4 bits a block with a NaN or an
 * infinity is NaN.
 * Hidden sizes up to 16384 that are multiples of 8, with all pointers and strides on the 16-byte grid (8 bytes for rows in e4m3), take vector
 * loads; even sizes up to 8192 whose pointers and strides are whole pairs of elements go by pairs; all others, longer ones on the grid too, by elements.
 * Errors: CB_ERR_ARG, CB_ERR_ALIGN (a pointer off its element size; an output in 4 bits or its scales off 16
 * bytes), CB_ERR_LIMIT (rows beyond 2^31 - 1 or hidden beyond 2^31 - 256), CB_ERR_CUDA. */
int cb_norm_around(const cb_norm_around_desc* desc, const void* x, const void* branch, const void* gate,
                   const void* after_weight, const void* after_bias, const void* weight, const void* bias,
                   const void* scale, const void* shift, void* x_out, void* out, void* out_scale, void* stream);

/* ---- rows in 4 bits (CB_MXFP4)
 *
 * A matrix [rows, features] is held as codes and scales. An element is an e2m1 code c (sign, two
 * bits of exponent, one of mantissa: 0, 1/2, 1, 3/2, 2, 3, 4, 6) times 2^(e - 127), where the byte e is
 * shared by CB_MX_BLOCK consecutive elements of a row (e = 255: all of them are NaN).
 *   codes: two a byte, the even element's in the low half. A row is CB_MX_BLOCK / 2 bytes for every
 *     block begun; codes behind its last feature are 0. Rows start on 16-byte boundaries.
 *   scales: cb_mx_scale_bytes(rows, features) bytes on a 16-byte boundary, in tiles of 128 rows by 4
 *     blocks. Block b of row r is at byte
 *       ((r / 128) * ceil(blocks / 4) + b / 4) * 512 + (r % 32) * 16 + (r / 32 % 4) * 4 + b % 4,
 *     blocks = ceil(features / CB_MX_BLOCK). Bytes of a row's blocks behind the last one are 0; those
 *     of rows behind the last are neither read for a result nor written.
 * The calls below write matrices so; one that comes from elsewhere has to have these zeros too. */
#define CB_MX_BLOCK 32

/* Bytes of the scales of a matrix into *bytes. Errors: CB_ERR_ARG, CB_ERR_LIMIT (as below). */
int cb_mx_scale_bytes(int64_t rows, int64_t features, size_t* bytes);

/* Sizes and types of cb_mx_quantize and cb_mx_dequantize. Strides are in elements from one row to
 * the next; 0 means contiguous. */
typedef struct {
    int64_t rows;         /* >= 0; 0 does nothing */
    int64_t features;     /* >= 1 */
    int64_t stride;       /* of the rows in dtype */
    int64_t codes_stride; /* a multiple of CB_MX_BLOCK */
    cb_dtype dtype;       /* CB_BF16 or CB_FP32 */
    int32_t reserved;     /* must be 0 */
} cb_mx_desc;

/* Rows into CB_MXFP4. Every block's e is that of its largest magnitude, which is taken to two
 * significant bits first: 2^(e - 127) is the power of two that brings it to 3.5 at least and below 7,
 * where 6 to 7 become 6 (root mean square error of normal values 0.112 of theirs; below 6, and nothing cut off,
 * 0.115; below 8 0.115); at least 2^-127. Codes are rounded to nearest, ties to even. A block with a NaN or
 * an infinity has e = 255 and codes of 0.
 * Errors: CB_ERR_ARG, CB_ERR_ALIGN (a pointer off its element size, codes or scales off 16
 * bytes), CB_ERR_LIMIT (rows beyond 2^31 - 1, features beyond 2^31 - 256, or 2^31 pieces of 32 rows by
 * 256 features), CB_ERR_CUDA. */
int cb_mx_quantize(const cb_mx_desc* desc, const void* x, void* codes, void* scales, void* stream);

/* Rows from CB_MXFP4, exact (beyond fp32's range: infinite). Errors: as above. */
int cb_mx_dequantize(const cb_mx_desc* desc, const void* codes, const void* scales, void* x, void* stream);

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
    cb_dtype type;         /* of w and of the rows x: CB_BF16, CB_E4M3 or CB_MXFP4 (w_stride: a multiple of CB_MX_BLOCK) */
    cb_dtype bias_dtype;   /* CB_BF16 or CB_FP32 */
    int32_t activation;    /* CB_ACT_* */
    int32_t reserved;      /* must be 0 */
    const void* w;
    const void* w_scale;   /* CB_E4M3: fp32 [out_features] (NULL: 1); CB_MXFP4: w's scales */
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
    cb_dtype out_dtype;       /* CB_BF16, CB_FP32, or of a CB_MXFP4 layer CB_MXFP4 (out_stride: a multiple of CB_MX_BLOCK) */
    cb_dtype resid_dtype;     /* of resid and resid_out: CB_BF16 or CB_FP32 */
    cb_dtype gate_dtype;      /* CB_BF16 or CB_FP32 */
    int32_t reserved;         /* must be 0 */
    void* out_scale;          /* read for an output in CB_MXFP4 only: its scales */
} cb_linear_io;

typedef struct cb_linear cb_linear; /* opaque, host-owned; holds no device memory */

/* Errors: CB_ERR_ARG, CB_ERR_ALIGN (a pointer off its element size; codes or scales in 4 bits off 16 bytes), CB_ERR_LIMIT (out_features
 * beyond 2^31 - 1024, in_features beyond CB_MAX_IN_FEATURES, or a row stride of w or x
 * beyond 2^31 - 256 bytes). The layer keeps the pointers: its buffers must outlive it. */
int cb_linear_create(const cb_linear_desc* desc, cb_linear** out);
/* The process's last layer gives back the device memory that cb_linear_run keeps (what work under way still
 * uses stays until the next last one). NULL does nothing. */
void cb_linear_destroy(cb_linear* layer);

/* CB_OPT_WAIT_NS: limit of every wait of the layer's kernels on one of their barriers, ns (default 1e9, at most
 * 6e10). CB_OPT_TEST_WITHHOLD: 1: (tests of the failure path only) over 32 rows (CB_MXFP4: always) the kernels announce more
 * bytes of operands than they copy, so that the waits for them run out; results are then
 * invalid. Errors: CB_ERR_ARG. */
int cb_linear_set_option(cb_linear* layer, int option, int64_t value);

/* Matrix product with its epilogue. For every row m and output feature n
 *     v = act(x_scale[m] * w_scale[n] * sum_k x[m, k] w[n, k] + bias[n])
 *     out = round(v)                        the branch output, as cb_cache_push takes it
 *     resid_out = round(resid + gate * v)   the hidden state (gate: a line per sample)
 * with sums, epilogue and hidden state in fp32 and one rounding to each result. The
 * tensor cores cut sums off rather than round them (CB_BF16 and CB_E4M3 layers): where a result is fp32 they sum
 * parts of 512 features (e4m3: 4096; up to 32 rows: 128 and 256 at most), which are added
 * rounded to nearest. Measured, in the root mean square relative to the sums': 5e-7 with signs
 * mixed, 8e-7 with all terms of one sign, and up to 2^-24 for every part added (of which most
 * cancel: 2^-24 times the root of their number). bf16 results: parts of 2048 (e4m3: 4096) where rows are longer
 * than 32 KB, else one part, which is off by up to 7.2e-5 (16384 features of one sign) before
 * the rounding to bf16.
 * CB_MXFP4 layers: x_scale are x's scales, and their factors 2^(e - 127) stand in place of x_scale[m] w_scale[n] within the
 * sum, whose products are exact. fp32 results are sums of parts of 16384 features, other results of one part up to 65536 features and of parts of
 * 8192 beyond, whatever the rows are; under scales that differ much (lognormal) a part is off, in the root mean square relative to the sums' with signs
 * mixed and with all terms of one sign, by 5e-8 and 1.2e-7 at 2048 features, 1.9e-7 and 6.2e-7 at 16384, 3.2e-6 and 6.4e-6 at 65536. out in CB_MXFP4 (no hidden state then): v as cb_mx_quantize makes
 * it of fp32 rows, with io->out_scale.
 * x_scale: one float a row (CB_E4M3, NULL: 1; not for CB_BF16). out may be NULL, resid and resid_out
 * may be NULL together, gate (with resid only) may be NULL: 1; one result at least
 * is wanted. resid_out may be resid itself (same stride). The order of a sum depends
 * on the sizes, the types and what of it lies on the 16-byte grid alone: equal calls give equal bits.
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
int cb_linear_run(const cb_linear* layer, const cb_linear_io* io, const void* x, const void* x_scale,
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
