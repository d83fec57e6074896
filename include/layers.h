/* Building blocks of residual and per-grid-point surrogates beside surrogate.h's
 * plain ones: a dense layer with bias, activation and residual in its epilogue,
 * group norm with an activation over channels-last data, and dropout whose mask
 * is generated again where it is needed and never stored.  Each has a
 * forward and a backward; a trained block is
 *   y = h + dropout(dense(group_norm(h))).
 *
 * Activations, with their derivatives (relu'(0) = 0):
 *   OT_ACT_NONE z;  OT_ACT_RELU max(z, 0);  OT_ACT_SILU z / (1 + exp(-z));
 *   OT_ACT_GELU z Phi(z), Phi the normal distribution's integral.
 *
 * Layout: matrices are rows of contiguous values, leading dimensions in
 * elements between rows.  Precision OT_FP32 or OT_BF16 (surrogate.h) is the type
 * of x, W, dy, dx and the like; biases, the norm's parameters, statistics and
 * the gradients of parameters are fp32.  Sums are fp32; a result is rounded to
 * its type once.
 *
 * Alignment: device pointers to matrices are 16-byte aligned and their leading
 * dimensions multiples of 8 (bf16) or 4 (fp32) elements, at least the row length
 * (ld may be anything where there is one row).  Values between a row's end and
 * its leading dimension may be anything and are not written.  Vectors need
 * their elements' alignment only.
 *
 * Outputs must not overlap each other, nor an input but where a call says that they may be the same.
 *
 * Ownership: tensors are the caller's.  Objects hold sizes and, where said,
 * workspaces (device memory on the device current at creation, which must be
 * current in every call).  Calls are asynchronous on the given stream; calls on
 * one object must not overlap, so a caller that changes streams orders them.  A
 * call that asks for more than the workspaces hold replaces them, which waits for
 * the device and is refused (OT_E_STATE) under stream capture; any other call
 * allocates nothing and may be captured.  Workspaces named by a captured call are
 * kept until the object is destroyed.
 */
#ifndef OT_LAYERS_H
#define OT_LAYERS_H

#include <stdint.h>

#include "ot_status.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ot_dense ot_dense;
typedef struct ot_norm ot_norm;
typedef struct ot_dropout ot_dropout;

enum ot_activation { OT_ACT_NONE = 0, OT_ACT_RELU = 1, OT_ACT_SILU = 2, OT_ACT_GELU = 3 };

/* ---- dense layer -------------------------------------------------------------
 * forward:   z = x W^T + bias;  y = act(z) + residual
 * backward:  dz = dy act'(z);  dx = dz W;  dW = dz^T x;  dbias = column sums of dz
 * (the residual's gradient is dy).  W is out x in.  Products of a bf16 layer take dz
 * whole: relu only drops values of dy; silu's and gelu's dz enters as the sum of three
 * bf16 terms, so where x or W hold an infinity, the gradients it enters may be NaN
 * instead of infinite. */

/* in, out_dim in [1, 2^26]; max_rows: rows of the largest backward that the
 * workspaces are first sized for, in [0, 2^26] (0: a layer that only serves; a
 * forward needs none).  A backward's workspace holds dz where there is an activation
 * (in the layer's precision, its rows padded to 8 values; silu and gelu in bf16: three times that)
 * and at most 0.3 GB of partial sums.  Errors: OT_E_INVAL, OT_E_NOMEM, OT_E_HIP. */
int dense_create(ot_dense** out, int64_t in, int64_t out_dim, int32_t precision, int32_t activation,
                 int64_t max_rows);

/* The layer on n rows (0 <= n <= 2^26; 0 does nothing; no matrix may have more than 2^36
 * values).  bias, residual, pre: nullable.  y and residual are of y_type
 * (OT_FP32 or OT_BF16); y may be the residual (the same address and leading
 * dimension).  pre receives z in the layer's precision, for a later
 * dense_backward.  Errors: OT_E_INVAL, OT_E_STATE, OT_E_HIP. */
int dense_forward(ot_dense* d, const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias,
                  const void* residual, int64_t ldr, int64_t n, void* y, int64_t ldy, int32_t y_type, void* pre,
                  int64_t ldp, void* stream);

/* Gradients on n rows (0 writes zeros to dw and dbias).  pre: what dense_forward
 * stored for these rows (not read and may be NULL with OT_ACT_NONE).  dx, dw, dbias:
 * nullable; w is read for dx only and x for dw only, and may be NULL otherwise.  Gradients are
 * written whole, not accumulated.  Errors: OT_E_INVAL, OT_E_STATE, OT_E_NOMEM,
 * OT_E_HIP. */
int dense_backward(ot_dense* d, const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t n, const void* dy,
                   int64_t lddy, const void* pre, int64_t ldp, void* dx, int64_t lddx, float* dw, int64_t lddw,
                   float* dbias, void* stream);

/* Free the workspaces (waits for the device). */
int dense_destroy(ot_dense* d);

/* ---- group norm --------------------------------------------------------------
 * x holds n samples of `positions` rows of `channels` values (row s positions + p:
 * position p of sample s); group g of a sample is channels g c .. g c + c - 1 with
 * c = channels / groups, at every position.  With a group's mean and its variance
 * (the mean square of the differences from the mean)
 *   xh = (x - mean) rstd, rstd = 1 / sqrt(var + eps);  p = weight xh + bias;  y = act(p)
 * backward:  dp = dy act'(p);  dweight = sum of dp xh;  dbias = sum of dp, both over all samples and
 *   positions;  dx = rstd (weight dp - mean(weight dp) - xh mean(weight dp xh)), means over the group.
 * weight and bias hold one value per channel; NULL: ones, zeros.  positions = 1 and
 * groups = 1 normalise whole rows.  A group's results depend on its own values only.  Squares of
 * differences from the mean are summed in fp32 and have to stay below 2^128. */

/* channels in [1, 65536], groups dividing it, positions in [1, 2^26], eps finite and
 * above 0; max_samples: samples of the largest call that the workspaces are first
 * sized for, in [0, 2^26], of at most 2^36 values.  Errors: OT_E_INVAL, OT_E_NOMEM,
 * OT_E_HIP. */
int norm_create(ot_norm** out, int64_t channels, int32_t groups, int64_t positions, int32_t precision,
                int32_t activation, float eps, int64_t max_samples);

/* n samples (0 does nothing; at most 2^36 values in all).  stats (nullable) receives
 * mean and rstd of every sample and group, n x groups x 2 contiguous values, for a
 * later norm_backward.  y may be x (the same address and leading dimension).
 * Errors: OT_E_INVAL, OT_E_STATE, OT_E_NOMEM, OT_E_HIP. */
int norm_forward(ot_norm* d, const void* x, int64_t ldx, const float* weight, const float* bias, int64_t n, void* y,
                 int64_t ldy, float* stats, void* stream);

/* Gradients on n samples (0 writes zeros to dweight and dbias).  stats: what
 * norm_forward stored for them.  dx, dweight, dbias: nullable, written whole.  dx may
 * be dy (the same address and leading dimension).  Errors: OT_E_INVAL, OT_E_STATE,
 * OT_E_NOMEM, OT_E_HIP. */
int norm_backward(ot_norm* d, const void* x, int64_t ldx, const float* weight, const float* bias, int64_t n,
                  const float* stats, const void* dy, int64_t lddy, void* dx, int64_t lddx, float* dweight,
                  float* dbias, void* stream);

/* Free the workspaces (waits for the device). */
int norm_destroy(ot_norm* d);

/* ---- dropout -----------------------------------------------------------------
 * y = residual + keep x / (1 - p).  The value of row r and column c is dropped where its
 * 16 random bits are below t = round(65536 p), and p is taken as t / 65536.  The
 * bits: Philox4x32-10 (Salmon, Moraes, Dror, Shaw, SC'11) with key (seed mod 2^32,
 * seed / 2^32) and counter (c / 8, r mod 2^32, site, step mod 2^32); columns 8 j .. 8 j + 7 take the
 * low and high halves of words 0 to 3 in order.  A mask depends on nothing else: not on
 * strides, types or the number of rows and columns.  `site` tells the dropouts of one
 * model apart, `step` its training steps.  A dropped value is 0 whatever x holds (infinities, NaN). */

/* p in [0, 1] (1 drops everything).  No workspace.  Errors: OT_E_INVAL, OT_E_NOMEM, OT_E_HIP. */
int dropout_create(ot_dropout** out, double p, uint64_t seed, uint32_t site, int32_t precision);

/* n rows of `cols` values (n, cols in [0, 2^31), 0 does nothing).  residual: nullable, of x's type.
 * step_dev (nullable): a device value that is added to step when the kernel
 * runs, so that replays of a captured call take masks of their own.  y may be x or
 * the residual (the same address and leading dimension).  Errors: OT_E_INVAL, OT_E_STATE, OT_E_HIP. */
int dropout_forward(ot_dropout* d, const void* x, int64_t ldx, const void* residual, int64_t ldr, int64_t n,
                    int64_t cols, void* y, int64_t ldy, int64_t step, const int64_t* step_dev, void* stream);

/* dx = keep dy / (1 - p) with the forward's mask (the residual's gradient is dy). */
int dropout_backward(ot_dropout* d, const void* dy, int64_t lddy, int64_t n, int64_t cols, void* dx, int64_t lddx,
                     int64_t step, const int64_t* step_dev, void* stream);

int dropout_destroy(ot_dropout* d);

#ifdef __cplusplus
}
#endif

#endif /* OT_LAYERS_H */
