/*
 * libasgd -- the global norm of many gradients, and clipping by it, on one NVIDIA B200 (sm_100a), C ABI.
 *
 * A step of gradient descent on a layer of experts (asgd_experts.h) has gradients in many tensors; one number, the
 * 2-norm of all of them together, says whether the step is too long.
 *
 * The general rules are those of asgd_experts.h; the list of tensors is HOST memory, read before the call returns.
 */
#ifndef ASGD_GRADIENTS_H_
#define ASGD_GRADIENTS_H_

#include <stddef.h>
#include <stdint.h>

#include "asgd_experts.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct asgd_gradient {
  const void *x; /* n numbers of `type`, one after another, aligned to their type (NULL where n = 0)       */
  void *out;     /* the clipped ones, of the same type: x itself or memory that no x and no other out is in
                    (ASGD_EINVAL where they meet); not used by asgd_grad_norm                              */
  int64_t n;     /* 0 .. ASGD_GRADIENT_MAX                                                                 */
  int32_t type;  /* ASGD_F32 / BF16 / F16                                                                  */
  int32_t reserved; /* 0 */
} asgd_gradient;

#define ASGD_GRADIENT_MAX (1ll << 40)

/* Bytes of workspace that either call needs for `count` tensors (at least 1). */
int asgd_gradients_workspace_bytes(int64_t count, size_t *bytes /* HOST out */);

/* norm[0] = sqrt(sum of x^2 over all numbers of all tensors): sums in fp64, in an order that depends on the tensors'
 * sizes, types and addresses modulo 32 alone (other addresses may change the last bit); rounded once to fp32.  0 without numbers; infinite or NaN where a number is, or where the norm passes fp32's
 * range.  `workspace`: 16-byte aligned. */
int asgd_grad_norm(const asgd_gradient *list, int64_t count, float *norm, void *workspace, size_t workspace_bytes,
                   void *stream);

/* The norm, and out = x * f, rounded once, with f = min(1, max_norm / (norm + 1e-6)) in fp32.  With f = 1 tensors that
 * are clipped in place are not written.  A norm of infinity makes f 0 (finite numbers become zeros, infinite ones NaN);
 * a norm of NaN makes every number NaN.  max_norm > 0 (infinity: the norm alone matters; NaN is ASGD_EINVAL). */
int asgd_clip_grads(const asgd_gradient *list, int64_t count, float max_norm, float *norm, void *workspace,
                    size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* ASGD_GRADIENTS_H_ */
