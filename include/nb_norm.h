/*
 * nb_norm.h -- layer norm over the channels of each row (a pixel of an NHWC tensor, a token), forward and backward, beside
 * the batch norm of nb_cbs.h: the norm of pre-norm MLP blocks, whose products are those of nb_linear.h.
 *
 *   mean_r = (1/c) sum_j x[r][j];  rstd_r = 1 / sqrt((1/c) sum_j (x[r][j] - mean_r)^2 + eps);  xhat = (x - mean_r) * rstd_r
 *   y[r][j] = gamma[j] * xhat[r][j] + beta[j]
 * and, given g = dL/dy:
 *   d = g * gamma;  dx[r][j] = rstd_r * (d - (1/c) sum d - xhat * (1/c) sum d*xhat)  [ + add[r][j] ]
 *   dgamma[j] = sum_r g*xhat;  dbeta[j] = sum_r g
 *
 * x, y, g, add, dx are of `dtype` (nb_dtype), rows x c, the channels contiguous, rows ld_* elements apart (0 = dense, else >= c:
 * a channel slice of a wider tensor); gamma, beta, mean, rstd, dgamma, dbeta are fp32 and dense.  All statistics and sums are
 * formed in fp32 or more from the values as they are stored and each result is rounded once (fp16 saturates at +-65504, uncounted; a NaN stays one).
 * Any c from 1 to 2^24 and any element-aligned pointer is taken; rows of whole 16-byte vectors (pointers, c and pitches) are the fast
 * ones.  y may be x, and dx may be g or add, where pointer and pitch are the same; otherwise outputs overlap nothing.
 * Sums are taken in a fixed order: results are bitwise reproducible on a given device.
 *
 * Device pointers on the CURRENT device; calls enqueue on `stream` and return without synchronising; safe to capture into a
 * CUDA graph.  Status codes and nb_last_error() as in nb_cbs.h.
 * Errors: NB_ERR_INVALID_ARG (a required pointer is NULL, rows or c not positive, eps not positive, a pitch below c, unknown
 * dtype, one of dgamma / dbeta without the other), NB_ERR_ALIGNMENT, NB_ERR_WORKSPACE, NB_ERR_CUDA.
 */
#ifndef NB_NORM_H
#define NB_NORM_H

#include "nb_cbs.h"

#ifdef __cplusplus
extern "C" {
#endif

/* gamma and beta may be NULL (1 and 0); mean and rstd (what the backward call needs) may be NULL together. */
nb_status nb_layer_norm_fwd(int32_t dtype, int64_t rows, int32_t c, const void* x, int64_t ld_x, const float* gamma, const float* beta,
                            float eps, void* y, int64_t ld_y, float* mean, float* rstd, void* stream);

/* Bytes of device workspace (256-byte aligned, no initialisation) of the backward call on the current device; 0 is never
 * returned.  Two calls that may overlap on the device need two workspaces. */
nb_status nb_layer_norm_workspace_bytes(int64_t rows, int32_t c, size_t* bytes);

/* gamma may be NULL (1), add may be NULL (0: else the gradient that reaches x along another branch, e.g. the residual's),
 * dgamma and dbeta may be NULL together (nothing is summed, no workspace is needed). */
nb_status nb_layer_norm_bwd(int32_t dtype, int64_t rows, int32_t c, const void* g, int64_t ld_g, const void* x, int64_t ld_x,
                            const float* gamma, const float* mean, const float* rstd, const void* add, int64_t ld_add, void* dx,
                            int64_t ld_dx, float* dgamma, float* dbeta, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NB_NORM_H */
