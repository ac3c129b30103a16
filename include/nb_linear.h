/*
 * nb_linear.h -- matrix product with bias, activation and residual in its epilogue, its data gradient and its weight gradient:
 * the products of MLP blocks over the rows (pixels, tokens) of a matrix, beside the pointwise convolution with bias of nb_cbs.h.
 *
 * Row-major matrices, the last index contiguous:  x [rows][c_in], w [c_out][c_in], out, res, z, dy [rows][c_out], dx [rows][c_in]
 *   forward:          z = x w^T + bias;   out = act(z) + res
 *   data gradient:    dx = (dy w + add) * act_in'(z_in)      z_in [rows][c_in]: what the activation in front of this layer was given
 *   weight gradient:  dw = dy^T x;  dbias[j] = sum over the rows of dy[r][j]
 * with act one of nb_act: none, SiLU z/(1+e^-z), GELU z*Phi(z) (Phi the normal distribution function, not its tanh approximation)
 * (an infinite z has the value and the derivative of the limit).  A layer whose own activation is not followed by another layer of this kind takes nb_act_bwd for the gradient of its z.
 *
 * x, w, res, z, out, dy, add, z_in, dx are of the plan's dtype; bias, dw, dbias are fp32.  Products are accumulated in fp32 (on the
 * tensor cores, which cut off low bits, no further than a fifth of half a step of the type: longer sums leave them in between), the
 * epilogue works on the fp32 sums and rounds once (z and out each once, from the same sum); fp16 stores saturate at +-65504 (a NaN stays one).
 *   NB_DTYPE_BF16 / NB_DTYPE_F16: tcgen05 tensor cores where c_in and c_out are multiples of 8 and pitches and pointers whole
 *     16-byte vectors, and on padded copies (in the workspace) of layers with other channel counts from 2^27 products on
 *     (nb_linear_paths); CUDA cores elsewhere.  There the activations are those of fp32; on the tensor cores they are approximated, with
 *     errors relative to the value in the tails too: Phi(z) and GELU within 2^-15 for |z| <= 8, the logistic function and SiLU within 2^-18.
 *   NB_DTYPE_F32: plain FMA arithmetic (no TF32).
 * Sums have a fixed order: results are bitwise reproducible on a given device for the same shapes and alignment.
 *
 * Pitches ld_* are elements between rows, 0 = dense, else >= the row's length; z, z_in, w, dw are dense.  All pointers are DEVICE pointers
 * on the plan's device, aligned to their element size (w, bias, dw, dbias: 16 bytes).  Outputs overlap nothing else that the call
 * reads or writes, with two exceptions: out may be res and dx may be add (same pointer and pitch).
 * Calls make the plan's device current while they run, enqueue on `stream` and return without synchronising; safe to capture into a
 * CUDA graph.  Calls of one plan may overlap, on the host and on the device, where their workspaces differ.
 * Status codes and nb_last_error() as in nb_cbs.h.  Errors: NB_ERR_INVALID_ARG (NULL, rows not positive, a pitch too small, unknown act),
 * NB_ERR_UNSUPPORTED (rows or a matrix of 2^31 - 2^16 rows or more), NB_ERR_ALIGNMENT, NB_ERR_WORKSPACE, NB_ERR_CUDA.
 */
#ifndef NB_LINEAR_H
#define NB_LINEAR_H

#include "nb_cbs.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { NB_ACT_NONE = 0, NB_ACT_SILU = 1, NB_ACT_GELU = 2 } nb_act;

#define NB_LINEAR_FLAG_FORCE_SIMT 1u /* 16-bit types: run on the CUDA cores (same contract; for testing and as a cross-check) */

typedef struct nb_linear_desc {
    uint32_t struct_size; /* = sizeof(nb_linear_desc) */
    int32_t c_in, c_out;  /* 1 .. 2^24 */
    int32_t dtype;        /* nb_dtype */
    uint32_t flags;
} nb_linear_desc;

typedef struct nb_linear_plan_s* nb_linear_plan;

/* Create a plan for one layer on CUDA device `device`: allocates a small device status block, nothing else.
 * Errors: NB_ERR_INVALID_ARG, NB_ERR_CUDA, NB_ERR_ARCH. */
nb_status nb_linear_plan_create(const nb_linear_desc* desc, int device, nb_linear_plan* out_plan);

/* Free the plan.  NULL is accepted.  Not while calls of it are in flight. */
nb_status nb_linear_plan_destroy(nb_linear_plan plan);

/* Bytes of device workspace (256-byte aligned, no initialisation) that are enough for every call of the plan on `rows` rows. */
nb_status nb_linear_workspace_bytes(nb_linear_plan plan, int64_t rows, size_t* bytes);

/* Which kernels the forward, data-gradient and weight-gradient call run on for dense, 16-byte aligned operands of `rows` rows:
 * 0 = CUDA cores, 1 = tcgen05 tensor cores, 2 = a few rows streaming the weights (forward only). */
nb_status nb_linear_paths(nb_linear_plan plan, int64_t rows, int32_t* paths3);

/* Synchronise `stream`, then report whether a kernel of this plan gave up a bounded wait (NB_ERR_TIMEOUT) or saturated an fp16 result
 * (still NB_OK; nb_last_error() says so: a loss scaler cannot see it; NaN counts too, and on the tensor cores parts of a row rather than
 * elements).  Clears the status.  nb_act_bwd has no plan and counts nothing. */
nb_status nb_linear_poll_status(nb_linear_plan plan, void* stream);

/* bias, res, z may be NULL (no bias, no residual, z is not kept). */
nb_status nb_linear_fwd(nb_linear_plan plan, int64_t rows, const void* x, int64_t ld_x, const void* w, const float* bias, int32_t act,
                        const void* res, int64_t ld_res, void* z, void* out, int64_t ld_out, void* workspace, size_t workspace_bytes,
                        void* stream);

/* z_in is NULL exactly when act_in is NB_ACT_NONE; add may be NULL. */
nb_status nb_linear_bwd_data(nb_linear_plan plan, int64_t rows, const void* dy, int64_t ld_dy, const void* w, const void* z_in,
                             int32_t act_in, const void* add, int64_t ld_add, void* dx, int64_t ld_dx, void* workspace,
                             size_t workspace_bytes, void* stream);

/* dbias may be NULL. */
nb_status nb_linear_bwd_weight(nb_linear_plan plan, int64_t rows, const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, float* dw,
                               float* dbias, void* workspace, size_t workspace_bytes, void* stream);

/* dz = dy * act'(z) over n elements (dense, element-aligned; dz may be dy), on the CURRENT device.  dtype as above; act SiLU or GELU. */
nb_status nb_act_bwd(int32_t dtype, int64_t n, int32_t act, const void* dy, const void* z, void* dz, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NB_LINEAR_H */
