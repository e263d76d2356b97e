/*
 * gf_train.h -- operators of a fine-tuning step around the filtered convolution (gf.h): layer
 * normalisation over channels, forward and backward.
 *
 * The conventions of gf.h hold: device pointers 16-byte aligned and dense, inputs read-only,
 * outputs overwritten, work enqueued on `stream` without synchronising, errors that the host can
 * detect returned before anything is launched, device scratch supplied by the caller.
 */
#ifndef GF_TRAIN_H_
#define GF_TRAIN_H_

#include "gf.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- layer normalisation over the channels ------------------------------------------------
 * A tensor [N, C, H, W] in the order `layout` says: GF_NCHW, or GF_NHWC, which with H = W = 1 is
 * a matrix of N rows of C values.  For each of the R = N H W pixels (rows), over its C channels:
 *     mean = sum x / C,   rstd = 1 / sqrt(sum (x - mean)^2 / C + eps),
 *     y = (x - mean) rstd gamma + beta
 * and, with xh = (x - mean) rstd and h = g_y gamma,
 *     g_x = rstd (h - sum h / C - xh sum (h xh) / C),
 *     g_gamma[c] = sum over pixels of g_y xh,   g_beta[c] = sum over pixels of g_y.
 * x, y, g_y, g_x have the descriptor's dtype; gamma and beta its param_dtype; mean and rstd
 * (R values each, pixels in order n, h, w), g_gamma and g_beta are ALWAYS fp32.  All arithmetic
 * is fp32; the variance is taken about the mean (no difference of large sums); sums over pixels
 * are added in a fixed order, so that results repeat bit for bit.  A non-finite value spoils
 * the outputs of its own pixel, and the two sums of the channels it reaches.
 * N = 0 is allowed: g_gamma and g_beta are then zeros.  */
typedef struct gf_norm_desc {
    int32_t N, C, H, W;
    int32_t dtype;          /* gf_dtype of x, y, g_y, g_x */
    int32_t param_dtype;    /* gf_dtype of gamma and beta */
    int32_t layout;         /* gf_layout */
    float eps;              /* >= 0 */
} gf_norm_desc;

/* gamma NULL: ones; beta NULL: zeros.  mean and rstd may both be NULL (no backward pass to
 * follow).  y may be x (in place). */
gf_status gf_layer_norm_forward(const gf_norm_desc* desc, const void* x, const void* gamma,
                                const void* beta, void* y, float* mean, float* rstd, void* stream);

/* mean and rstd as gf_layer_norm_forward wrote them; gamma NULL: ones.  g_x, g_gamma and g_beta
 * may each be NULL and are then skipped.  g_x may be g_y (in place). */
gf_status gf_layer_norm_backward_workspace_bytes(const gf_norm_desc* desc, size_t* bytes);
gf_status gf_layer_norm_backward(const gf_norm_desc* desc, const void* g_y, const void* x,
                                 const void* gamma, const float* mean, const float* rstd, void* g_x,
                                 float* g_gamma, float* g_beta, void* workspace,
                                 size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GF_TRAIN_H_ */
