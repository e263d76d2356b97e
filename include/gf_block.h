/*
 * gf_block.h -- operators of a residual block whose layers are frozen in 8 bits, next to the filtered
 * convolutions (gf.h) and the operators of a fine-tuning step (gf_train.h): dropout from a counter, whose mask is
 * never stored; root-mean-square norm of a residual sum, with results in 8 bits where a frozen
 * layer follows; and the products of 8-bit rows with 8-bit weights, forward and for the gradient
 * of the input.
 *
 * The conventions of gf.h hold: device pointers 16-byte aligned and dense, inputs read-only,
 * outputs overwritten, work enqueued on `stream` without synchronising, errors that the host can
 * detect returned before anything is launched.  Make the first call of a kind on a device outside any
 * stream capture (kernels are set up then).  A device-side wait that runs out (products only) is
 * reported to the library-wide word that gf_last_async_status reads with any zeroed workspace.  Results repeat bit for
 * bit.
 */
#ifndef GF_BLOCK_H_
#define GF_BLOCK_H_

#include "gf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- dropout ---------------------------------------------------------------------------------
 *     y[i] = residual[i] + (keep[i] ? x[i] / (1 - t / 65536) : 0),   t = p * 65536, rounded
 * keep[i] = (b >= t), where b are 16 bits of element i alone: Philox4x32 with ten rounds (Salmon,
 * Moraes, Dror, Shaw 2011) on the counter (i / 8, seed[1]) under the key seed[0] gives
 * 128 bits for eight elements, lowest 16 first.  The mask is a function of (seed, i): it is computed again
 * in the backward pass and never stored.  p is thereby rounded to a multiple of 2^-16, and the scale is
 * that of the rounded one, so that the mean is kept.  The scaled value is rounded to fp32 before the
 * residual is added.  A dropped value counts as 0 whatever it is, NaN included; t = 65536 drops all.
 * seed: DEVICE pointer to two 64-bit words, 8-byte aligned (NULL when t = 0); read when the kernel
 * runs, so that a captured graph takes a new mask from new words.
 * Backward: g_x[i] = keep[i] ? g_y[i] / (1 - t / 65536) : 0; the residual's gradient is g_y. */
typedef struct gf_dropout_desc {
    int64_t count;          /* elements, >= 0 */
    int32_t dtype;          /* gf_dtype of x and g_x */
    int32_t out_dtype;      /* gf_dtype of residual, y and g_y */
    float p;                /* 0 .. 1 */
} gf_dropout_desc;

/* residual NULL: none.  y may be residual (in place), or x where the dtypes are the same; else, as everywhere here
 * where an output would lie over an input of another type, GF_ERR_UNSUPPORTED. */
gf_status gf_dropout_forward(const gf_dropout_desc* desc, const void* x, const void* residual,
                             const uint64_t* seed, void* y, void* stream);
/* g_x may be g_y where the dtypes are the same. */
gf_status gf_dropout_backward(const gf_dropout_desc* desc, const void* g_y, const uint64_t* seed,
                              void* g_x, void* stream);

/* ---- root-mean-square norm of a residual sum ------------------------------------------------------
 * For each of `rows` rows of `cols` values:
 *     h = residual + dropout(x)            (as above, i = row * cols + column), rounded to residual_dtype,
 *     rstd = 1 / sqrt(sum h^2 / cols + eps),      y = h rstd gamma
 * and backwards, for a gradient g_y of y and one, g_h, that comes back to h on its other way:
 *     xh = h rstd,   q = g_y gamma,   g = rstd (q - xh sum(q xh) / cols) + g_h,
 *     g_residual = g,   g_x = dropout's gradient of g,   g_gamma[c] = sum over rows of g_y xh.
 * Without a residual and with p = 0, h is x itself: it is not written, and residual_dtype = dtype.
 * x, y, g_y, g_x have the descriptor's dtype; residual, h, g_h, g_residual its residual_dtype (bf16
 * x with an fp32 residual is possible, the opposite GF_ERR_UNSUPPORTED); rstd (rows values) and
 * g_gamma are fp32.  Arithmetic is fp32: where a row's sum of squares passes its range rstd is 0, as for an
 * infinite value.  A non-finite value spoils its own row, and the sums of the columns it reaches. */
typedef struct gf_rms_desc {
    int64_t rows;           /* >= 0 */
    int32_t cols;           /* >= 1 */
    int32_t dtype, residual_dtype;
    int32_t param_dtype;    /* gf_dtype of gamma */
    float eps;              /* >= 0 */
    float p;                /* 0 .. 1 */
} gf_rms_desc;

/* gamma NULL: ones.  residual NULL: h = dropout(x).  h: required but where it is x, then NULL; it
 * may be residual, or x where the dtypes are the same, and y may be x (in place).  rstd NULL: not wanted. */
gf_status gf_rms_norm_forward(const gf_rms_desc* desc, const void* x, const void* residual,
                              const uint64_t* seed, const void* gamma, void* h, void* y, float* rstd,
                              void* stream);

/* The same with y as an 8-bit matrix (see below) of y's fp32 values: codes and scales. */
gf_status gf_rms_norm_forward_fp8(const gf_rms_desc* desc, const void* x, const void* residual,
                                  const uint64_t* seed, const void* gamma, void* h, void* codes,
                                  float* scales, float* rstd, void* stream);

/* h (or x, where h is x) and rstd from the forward pass; gamma NULL: ones; g_h NULL: zeros.
 * g_residual, g_x and g_gamma may each be NULL and are then skipped; with p = 0 and one dtype g_x and
 * g_residual are the same values.  g_residual may be g_h, or g_y where the dtypes are the same, and g_x may be g_y
 * (in place).  The workspace may be NULL where its size is 0. */
gf_status gf_rms_norm_backward_workspace_bytes(const gf_rms_desc* desc, size_t* bytes);
gf_status gf_rms_norm_backward(const gf_rms_desc* desc, const void* g_y, const void* g_h, const void* h,
                               const float* rstd, const void* gamma, const uint64_t* seed, void* g_residual,
                               void* g_x, float* g_gamma, void* workspace, size_t workspace_bytes,
                               void* stream);

/* ---- matrices in 8 bits -----------------------------------------------------------------------------
 * A matrix of `rows` rows of `cols` values is held as e4m3 codes (4 exponent and 3 mantissa bits, largest value
 * 448), a row every GF_FP8_PITCH(cols) bytes with zeros behind its last code, and fp32 scales; a
 * code stands for its value times its scale.
 *   rows:    a scale for each 128 columns of a row, scales[g * GF_FP8_SCALE_PITCH(rows) + row] for
 *            columns 128 g and on; places behind the last row are not written.
 *   blocks:  a scale for each 128 x 128 block, scales[(row / 128) * ceil(cols / 128) + col / 128].
 * scale = max(largest magnitude * (1 / 448), 2^-126), with 1 / 448 and the product rounded to fp32;
 * code = value / scale, the quotient rounded to fp32 and then to the nearest code, ties to even.
 * A group that holds a non-finite value has a scale that is not finite and stands for NaN throughout. */
#define GF_FP8_PITCH(cols) (((cols) + 15) / 16 * 16)
#define GF_FP8_SCALE_PITCH(rows) (((rows) + 3) / 4 * 4)
typedef struct gf_fp8_desc {
    int32_t rows;           /* >= 0 */
    int32_t cols;           /* >= 1 */
    int32_t dtype;          /* gf_dtype of the matrix that is quantised, [rows, cols] */
} gf_fp8_desc;

gf_status gf_fp8_quantize_rows(const gf_fp8_desc* desc, const void* x, void* codes, float* scales,
                               void* stream);
gf_status gf_fp8_quantize_blocks(const gf_fp8_desc* desc, const void* w, void* codes, float* scales,
                                 void* stream);

/* ---- product of 8-bit rows with an 8-bit weight ---------------------------------------------------------
 * W [N, K] with scales of blocks, as a frozen layer keeps it; A with scales of rows.
 *   transposed 0 (the layer):                 out[M, N] = A[M, K] W^T + bias[N]
 *   transposed 1 (the gradient of its input): out[M, K] = A[M, N] W   + bias[K]
 * Each 128 terms of a sum are added by the tensor cores, the scaled sums of 128 in fp32; the result is
 * rounded once to out_dtype.  The product of a row's scale and a block's need not be a normal number of fp32. */
typedef struct gf_fp8_matmul_desc {
    int32_t M;              /* >= 0 */
    int32_t N, K;           /* >= 1 */
    int32_t transposed;     /* 0 or 1 */
    int32_t out_dtype;      /* gf_dtype */
    int32_t bias_dtype;     /* gf_dtype */
} gf_fp8_matmul_desc;

/* bias NULL: none. */
gf_status gf_fp8_matmul(const gf_fp8_matmul_desc* desc, const void* a, const float* a_scales, const void* w,
                        const float* w_scales, const void* bias, void* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GF_BLOCK_H_ */
