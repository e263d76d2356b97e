/*
 * gf_train.h -- operators of a fine-tuning step around the filtered convolution (gf.h): layer
 * normalisation over channels, forward and backward, and the Muon update of the weights with its
 * Newton-Schulz orthogonalisation.
 *
 * The conventions of gf.h hold: device pointers 16-byte aligned and dense, inputs read-only,
 * outputs overwritten, work enqueued on `stream` without synchronising, errors that the host can
 * detect returned before anything is launched, device scratch supplied by the caller.  A
 * device-side wait that runs out is reported by gf_last_async_status on the call's workspace.
 * The layer norms report to the library-wide word that the same call reads: any workspace serves
 * there, a layer norm's own from a backward with g_gamma or g_beta and N > 0, which clears the
 * workspace's word.
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

/* ---- Newton-Schulz orthogonalisation ---------------------------------------------------------
 * For every matrix G [rows, cols] of a batch: X = G / (||G||_F + eps); then for each step k, with
 * its coefficients (a, b, c),
 *     X <- a X + (b A + c A A) X,   A = X X^T
 * (A = X^T X from the other side when rows > cols: the same result from the smaller products);
 * O = X.  A step maps every singular value s to a s + b s^3 + c s^5 and keeps the singular
 * vectors; with the default coefficients five steps bring the singular values near 1.
 * Results repeat bit for bit on one device.
 *   precision GF_NS_F16: the products' operands are rounded to fp16 under a fixed scale (11
 *     significant bits), sums are fp32 -- for updates that are applied in 16 bits or that are
 *     small beside the weights.
 *   precision GF_NS_F32: operands are carried as pairs of fp16, an entry v to within
 *     max(2^-22 |v|, 2^-35), three products each -- results of matrices in the range of real
 *     updates as from fp32 arithmetic (off by 2e-6 to 8e-6 of their norm).  The second bound holds for
 *     entries below 2^-13 of X, whose norm is 1 or, where eps is not small beside ||G||, less: a G
 *     far below eps is orthogonalised to fewer bits.
 * The coefficients have to keep the entries of X, A and b A + c A A below 32 in magnitude (the
 * defaults keep the singular values below 1.3); beyond that the fp16 range ends and the result
 * is not finite.  A matrix of zeros gives zeros; one with a non-finite entry or whose squares
 * overflow fp32 gives non-finite values or zeros, other matrices of the batch are not affected. */
typedef enum gf_ns_precision { GF_NS_F16 = 0, GF_NS_F32 = 1 } gf_ns_precision;
#define GF_NS_MAX_STEPS 16

typedef struct gf_ns_desc {
    int32_t batch;          /* >= 0; matrices lie one behind the other */
    int32_t rows, cols;     /* 1 .. 16384 */
    int32_t in_dtype;       /* gf_dtype of G */
    int32_t out_dtype;      /* gf_dtype of O */
    int32_t precision;      /* gf_ns_precision */
    int32_t steps;          /* 1 .. GF_NS_MAX_STEPS */
    float eps;              /* >= 0 */
} gf_ns_desc;

/* h_coeffs: HOST array of 3 * steps floats (a, b, c of each step; read before the call returns),
 * or NULL for (3.4445, -4.7750, 2.0315) at every step.  O must not be G.  The size of the
 * workspace is that for the device which is current. */
gf_status gf_newton_schulz_workspace_bytes(const gf_ns_desc* desc, size_t* bytes);
gf_status gf_newton_schulz(const gf_ns_desc* desc, const void* G, void* O, void* workspace,
                           size_t workspace_bytes, const float* h_coeffs, void* stream);

/* ---- Muon step -----------------------------------------------------------------------------------
 * For `count` layers of one shape, each with a weight W and a gradient g of [rows, cols, taps]
 * and a momentum M of [rows, cols] (fp32):
 *     M' = momentum M + (1 - momentum) g,
 *     u  = nesterov ? (1 - momentum) g + momentum M' : M',
 *     W' = (1 - lr weight_decay) W - lr scale NS(u)
 * with NS the Newton-Schulz map above of the flattened [rows, cols taps] matrix.
 * taps > 1 is for gradients that have ONE value for all taps of a [rows, cols] pair, as g_W of
 * gf_backward has with r >= 2: g is then read at its first tap, M holds one value per pair, and
 * since the flattened matrix is u (x) (1 .. 1), NS of it is NS(u) / sqrt(taps) at every tap --
 * the products are those of [rows, cols] alone.  Any other convolution weight is given with its
 * taps flattened into cols and taps = 1.
 * h_grad, h_momentum, ... are HOST arrays of `count` DEVICE pointers (read before the call
 * returns); these pointers need only the alignment of their elements (parameters and gradients are
 * often slices of one flat buffer).  The outputs may be the inputs (in place) or other buffers;
 * buffers of different layers must not overlap. */
typedef struct gf_muon_desc {
    int32_t count;          /* >= 0 */
    int32_t rows, cols;     /* 1 .. 16384 */
    int32_t taps;           /* 1 .. 4096 */
    int32_t grad_dtype, weight_dtype;   /* gf_dtype */
    int32_t precision, steps;           /* as gf_ns_desc */
    int32_t nesterov;       /* 0 or 1 */
    float eps, momentum, lr, weight_decay, scale;
} gf_muon_desc;

gf_status gf_muon_workspace_bytes(const gf_muon_desc* desc, size_t* bytes);
gf_status gf_muon_step(const gf_muon_desc* desc, const void* const* h_grad,
                       const float* const* h_momentum, const void* const* h_weight,
                       float* const* h_momentum_out, void* const* h_weight_out, void* workspace,
                       size_t workspace_bytes, const float* h_coeffs, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GF_TRAIN_H_ */
