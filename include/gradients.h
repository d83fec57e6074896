/* Lists of tensors trained together: the global norm of their gradients,
 * clipping by it, and Adam with the clipped gradients.
 *
 *   norm = sqrt(sum over every element of every gradient of g^2),
 *   c    = min(1, max_norm / norm)        (1 where norm is 0 or not finite),
 *
 * clip_apply writes c g; adam_step runs the surrogate's Adam (surrogate.h, the
 * same operation order) on c g.  Squares are summed in 64 bits in a fixed
 * order, so a norm neither overflows nor depends on the run; it is rounded to
 * fp32 once.
 *
 * A norm that is not finite (a gradient holds an infinity or a NaN, or the norm
 * passes fp32's range) clips nothing and takes no step: clip_apply writes the
 * gradients as they are, adam_step leaves parameters, moments, copies and step
 * counter untouched.  The norm that both return says so.
 *
 * A list is fixed when its object is created: the object holds the tensors'
 * addresses, not the tensors, which stay the caller's and must live as long as
 * the object is used.  Tensors are contiguous and aligned to their element
 * size; 16-byte alignment (the same for the arrays of one tensor) lets them be
 * read in whole vectors.  Tensors of one list must not overlap.
 *
 * Calls are asynchronous on the given stream, which may be under capture, and
 * allocate nothing.  Calls on one object must not overlap.  The device current
 * at creation must be current in every call (OT_E_STATE otherwise).
 */
#ifndef OT_GRADIENTS_H
#define OT_GRADIENTS_H

#include <stdint.h>

#include "ot_status.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ot_clip ot_clip;
typedef struct ot_adam ot_adam;

/* A list of n gradient tensors (1 <= n <= 65536): grads[i] holds counts[i] >= 0
 * elements of type types[i] (OT_FP32 or OT_BF16, surrogate.h; types NULL: all
 * fp32); at most 2^40 elements in all.  outs[i] receives the clipped tensor, in
 * the same type; outs NULL: in place.  Host arrays, read during the call.
 * Synchronous.  Errors: OT_E_INVAL, OT_E_NOMEM, OT_E_HIP. */
int clip_create(ot_clip** out, int32_t n, const void* const* grads, void* const* outs, const int64_t* counts,
                const int32_t* types);

/* The global norm into the device scalar norm_dev.
 * Errors: OT_E_INVAL, OT_E_STATE, OT_E_HIP. */
int clip_norm(ot_clip* c, float* norm_dev, void* stream);

/* The global norm (into norm_dev, nullable), then every tensor scaled.
 * max_norm: finite, > 0.  In place and with nothing to clip, nothing is
 * written.  Errors: OT_E_INVAL, OT_E_STATE, OT_E_HIP. */
int clip_apply(ot_clip* c, float max_norm, float* norm_dev, void* stream);

/* Free the list (waits for its device). */
int clip_destroy(ot_clip* c);

/* A list of n parameter tensors (1 <= n <= 65536) with their fp32 gradients and
 * both Adam moments, counts[i] >= 0 elements each.  copies: bf16 copies of the
 * parameters (rounded to nearest even) that each step refreshes; NULL, or NULL
 * entries: none.  steps: Adam steps taken so far (>= 0); the counter lives in
 * device memory, so a captured step may be replayed.
 * Errors: OT_E_INVAL, OT_E_NOMEM, OT_E_HIP. */
int adam_create(ot_adam** out, int32_t n, float* const* params, const float* const* grads, float* const* m,
                float* const* v, uint16_t* const* copies, const int64_t* counts, float lr, float beta1, float beta2,
                float eps, int64_t steps);

/* One Adam step with the gradients clipped to max_norm (finite, > 0; 0: not
 * clipped).  norm_dev receives the norm before clipping (nullable).  With
 * max_norm = 0 and no norm_dev the norm is not formed and the step is always
 * taken.  Errors: OT_E_INVAL, OT_E_STATE, OT_E_HIP. */
int adam_step(ot_adam* a, float max_norm, float* norm_dev, void* stream);

/* Learning rate of the steps enqueued (or captured) later. */
int adam_set_lr(ot_adam* a, float lr);

/* Steps taken, without those skipped; set them (a restart).  Synchronous:
 * wait for the device.  Errors: OT_E_INVAL, OT_E_STATE, OT_E_HIP. */
int adam_get_steps(ot_adam* a, int64_t* steps);
int adam_set_steps(ot_adam* a, int64_t steps);

/* Free the list (waits for its device). */
int adam_destroy(ot_adam* a);

#ifdef __cplusplus
}
#endif

#endif /* OT_GRADIENTS_H */
