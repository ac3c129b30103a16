/*
 * nb_adamw.h -- C ABI of the fused AdamW step over a list of tensors, beside the SGD step of nb_sgd.h: global-norm
 * gradient clipping over ALL gradient tensors, optional dynamic loss scaling, decoupled weight decay with per-group
 * learning rate and decay, moments in 32 bits or in 8 bits -- two kernel launches for any number of tensors (three when a
 * list has tensors of both kinds).
 * (The paper's training subsystem names Adam(W) beside SGD, Sec. 3.2 "Optimization", and prints no formula.)
 *
 *   total = sqrt(sum over every tensor and element of g^2);  c = min(max_norm / (total + 1e-6), 1);  g <- c*g
 *   t     = *step + 1
 *   m     = beta1*m + (1-beta1)*g                      (step 1 takes m = v = 0 whatever the buffers hold)
 *   v     = beta2*v + (1-beta2)*g*g
 *   p     = p*(1 - lr[group]*weight_decay[group]) - lr[group] * (m / (1-beta1^t)) / (sqrt(v / (1-beta2^t)) + eps)
 *   copy  = p rounded to bf16 or fp16                  (when the tensor has a 16-bit working copy)
 *   *step = t
 *
 * Moments are fp32 numbers: without clipping a gradient above about 6e20 has v = inf, whose update is m / inf = 0 (the parameter only
 * decays), and v of gradients below about 4e-18 is a subnormal number with fewer bits, whose root is taken all the same.
 *
 * The count of steps lives in DEVICE memory: a step that the loss scaler skips does not count, and a step captured into
 * a CUDA graph goes on counting as it is replayed.
 *
 * Moments in 8 bits (state_bits = 8).  Elements j*128 .. j*128+127 of a tensor share one fp32 scale per moment:
 *   exp_avg    holds e4m3 codes q of m:        m = q*s,      s = (largest |m| of the block) / 448,  q = rn(m * (448/largest))
 *   exp_avg_sq holds e4m3 codes q of sqrt(v):  v = (q*s)^2,  likewise with the largest sqrt(v) of the block; a root that is
 *              not zero is held as at least the smallest code (2^-9), so that it never divides as a zero.
 *              (448/largest and largest/448 are products with a reciprocal that is rounded once.)
 * A block whose largest value is below 2^-100 is held as zeros with scale 0.  A block that meets an inf or a NaN is NaN from then
 * on.  The step's own update uses m and v before they are rounded.  Every operation of m and v is rounded to fp32 by itself (no fused
 * multiply-adds), so that 32-bit moments do not depend on how a compiler contracts expressions.  The root that is coded and divided by is
 * within 2^-22 of the square root of that v (a code may be its neighbour's where the root lies that close to their middle), the quotient of
 * the update within 2^-20, and the parameter takes it in one fused multiply-add.
 *
 * All tensor pointers are DEVICE pointers on the plan's device, 16-byte aligned (scales: 4-byte); the caller owns
 * everything including the workspace.  Calls make the plan's device current while they run, enqueue on `stream` and return
 * without synchronising.  A workspace belongs to one plan; steps of one plan must not overlap on the device.
 * Sums are taken in a fixed order: results are bitwise reproducible for a given list and device.
 */
#ifndef NB_ADAMW_H
#define NB_ADAMW_H

#include "nb_cbs.h"
#include "nb_sgd.h" /* nb_loss_scaler, nb_scaler_hyper, NB_SGD_GROUPS */

#ifdef __cplusplus
extern "C" {
#endif

#define NB_ADAMW_BLOCK 128 /* elements of a tensor that share a scale when its moments are held in 8 bits */

typedef struct nb_adamw_tensor {
    const void* grad;         /* [numel] of grad_dtype; read only */
    float* param;             /* [numel] fp32 master parameter, updated in place */
    void* exp_avg;            /* [numel] first moment: fp32, or e4m3 codes */
    void* exp_avg_sq;         /* [numel] second moment: fp32, or e4m3 codes of its root */
    float* exp_avg_scale;     /* 8 bits: [ceil(numel/128)]; NULL with 32 bits */
    float* exp_avg_sq_scale;  /* 8 bits: [ceil(numel/128)]; NULL with 32 bits */
    void* param_copy;         /* NULL, or [numel] 16-bit working copy, rewritten */
    int64_t numel;            /* > 0 */
    int32_t group;            /* 0 .. NB_SGD_GROUPS-1 */
    int32_t copy_dtype;       /* 0 or NB_DTYPE_BF16 = bf16, NB_DTYPE_F16 = IEEE fp16 (saturating; a NaN stays one) */
    int32_t grad_dtype;       /* nb_dtype */
    int32_t state_bits;       /* 32 or 8; may differ from tensor to tensor of a list */
} nb_adamw_tensor;

typedef struct nb_adamw_hyper {
    uint32_t struct_size; /* = sizeof(nb_adamw_hyper) */
    float eps;            /* >= 0 */
    float max_norm;       /* <= 0 or +inf disables clipping */
    float lr[NB_SGD_GROUPS];
    float weight_decay[NB_SGD_GROUPS];
    double beta1, beta2;  /* in [0, 1); doubles, because 1-beta2 of a beta2 in fp32 is 1e-5 off */
} nb_adamw_hyper;

typedef struct nb_adamw_plan_s* nb_adamw_plan; /* opaque, caller-owned, host memory only */

/* Validate a tensor list (a HOST array of `count` entries) and build the table that spreads the elements over the blocks.
 * Errors: NB_ERR_INVALID_ARG (NULL, count <= 0, numel <= 0, bad group / dtype / state_bits, missing or superfluous scales,
 * two written ranges that overlap, or a gradient that overlaps one), NB_ERR_ALIGNMENT, NB_ERR_UNSUPPORTED (2^43 elements or more),
 * NB_ERR_CUDA (device query failed). */
nb_status nb_adamw_plan_create(const nb_adamw_tensor* host_tensors, int32_t count, int device, nb_adamw_plan* out_plan);

/* Free the plan.  NULL is accepted.  Not before the copy of nb_adamw_upload has completed. */
nb_status nb_adamw_plan_destroy(nb_adamw_plan plan);

/* Bytes of device workspace (256-byte aligned): a device copy of the list and of its table, the norm's partial sums. */
nb_status nb_adamw_workspace_bytes(nb_adamw_plan plan, size_t* bytes);

/* Copy the list and the table into the workspace (one asynchronous copy on `stream`).  Once per workspace. */
nb_status nb_adamw_upload(nb_adamw_plan plan, void* workspace, size_t workspace_bytes, void* stream);

/* One step, ordered on `stream` after the upload.  `step` is a device int64 (8-byte aligned), the number of steps
 * taken so far (initialise to 0).  total_norm (device, may be NULL) receives the gradient norm before clipping; with
 * clipping disabled and total_norm NULL the gradients are read once.  Safe to capture into a CUDA graph.
 * Without a scaler gradients that are inf or NaN reach the parameters; with clipping a NaN makes c and so every parameter NaN.
 * Errors: NB_ERR_INVALID_ARG, NB_ERR_WORKSPACE, NB_ERR_ALIGNMENT, NB_ERR_CUDA. */
nb_status nb_adamw_step(nb_adamw_plan plan, void* workspace, size_t workspace_bytes, const nb_adamw_hyper* hyper, int64_t* step,
                        float* total_norm, void* stream);

/* The same for gradients that arrive multiplied by state->scale, as nb_sgd_clip_nesterov_step_scaled: they are unscaled on
 * the fly, a gradient element that is inf or NaN makes the step a no-op (moments, parameters, copies and *step stay), and
 * the state is advanced. */
nb_status nb_adamw_step_scaled(nb_adamw_plan plan, void* workspace, size_t workspace_bytes, const nb_adamw_hyper* hyper,
                               const nb_scaler_hyper* scaler, nb_loss_scaler* state, int64_t* step, float* total_norm, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* NB_ADAMW_H */
