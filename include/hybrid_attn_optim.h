/*
 * hybrid_attn_optim.h -- gradient norm, clipping and the update of many parameters.
 * Part of the C ABI of libhybridattn.so: the conventions of hybrid_attn.h (device pointers on the current device, the caller's stream and
 * buffers, host checks ahead of the first HIP call, ha_status) hold here too.
 */
#ifndef HYBRID_ATTN_OPTIM_H
#define HYBRID_ATTN_OPTIM_H

#include "hybrid_attn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* The global norm of many gradients, their clipping, and the update of many parameters at once (the optimiser's part of a training step:
 * one norm over all of a model's gradients, one factor, one pass over all parameters).  Tensors are given as host arrays of descriptors that
 * are read before the call returns.  A descriptor's tensor is contiguous, n elements (n = 0 is allowed), aligned to its element size. */
typedef struct ha_tensor {
  void *data;             /* device */
  uint64_t n;             /* elements */
  int32_t dtype;          /* ha_dtype */
  int32_t reserved;       /* 0 */
} ha_tensor;

/* Enqueues result[0] = sqrt(sum of the squares of all elements of all tensors) and result[1] = min(1, max_norm / result[0]), 1 where the
 * norm is 0.  result: device float[2].  Squares are summed in double, in a fixed order (bitwise reproducible).  A NaN among the gradients makes
 * both NaN; an infinity makes the norm infinite and the factor NaN: the calls that take the result then leave what they would write as it was.  (Finite gradients
 * whose norm is beyond fp32 have result[0] infinite, and the factor that brings them down to max_norm.)
 * max_norm: positive, or infinity (the norm alone is wanted: the factor is 1 while the norm is finite).  workspace: device, 8-byte aligned,
 * hybrid_attn_grad_norm_workspace_bytes() bytes, contents undefined before and after.  Errors (nothing is enqueued): HA_ERR_NULL,
 * HA_ERR_SHAPE, HA_ERR_UNSUPPORTED (unknown dtype), HA_ERR_ALIGN, HA_ERR_WORKSPACE, HA_ERR_DEVICE. */
size_t hybrid_attn_grad_norm_workspace_bytes(int32_t n_tensors, const ha_tensor *grads);
ha_status hybrid_attn_grad_norm(int32_t n_tensors, const ha_tensor *grads, float max_norm, float *result, void *workspace,
                                size_t workspace_bytes, void *hip_stream);

/* Enqueues out[i] = result[1] * grads[i], rounded to out's dtype, for all tensors (each pair of one n); out[i] may be grads[i] itself, and
 * otherwise overlaps no gradient, and no tensor is written twice.  result: device float[2] as hybrid_attn_grad_norm leaves it.  In place, a factor of 1 touches nothing.
 * Where the factor is not finite, out is left as it was. */
ha_status hybrid_attn_grad_clip(int32_t n_tensors, const ha_tensor *grads, const ha_tensor *out, const float *result, void *hip_stream);

/* One parameter of hybrid_attn_param_update_many; the pointers as for hybrid_attn_param_update, but the gradient may be bf16. */
typedef struct ha_param {
  float *master;
  const void *grad;
  float *m, *v;
  void *param_io;
  uint64_t n;
  int32_t grad_dtype, io_dtype;
} ha_param;

/* hybrid_attn_param_update of all the parameters in as few launches as they fit.  result: device float[2] as hybrid_attn_grad_norm leaves it
 * or NULL: gradients are scaled by opt->grad_scale * result[1] (where the gradients' scale matters to the norm, it is taken of the gradients as
 * they stand, without grad_scale).  Where result[1] is not finite, nothing is written: a step whose gradients overflowed is skipped on
 * the device.  The rates are opt's floats, 1 - beta too.  No two of the tensors that are written (masters, moments, copies) overlap.  Errors as for hybrid_attn_param_update. */
ha_status hybrid_attn_param_update_many(const ha_optimizer *opt, int32_t n_params, const ha_param *params, const float *result, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* HYBRID_ATTN_OPTIM_H */
