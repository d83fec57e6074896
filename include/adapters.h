/* Low-rank adapters beside a frozen projection: one trained layer of a
 * surrogate (surrogate.h) shared by many ensembles, each with a low-rank
 * correction of its own.
 *
 * A bank holds G adapters of rank r for a layer of `out` x `in` weights.  Row m
 * of a batch names its adapter, ids[m]; a negative id, or one of G and more,
 * names none (the row passes the frozen layer alone).  With s_g the scale of
 * adapter g (1 without a scale array)
 *   t_m  = down_g x_m                                  (r values)
 *   y_m  = W x_m + bias + s_g up_g^T t_m,              ReLU if asked
 *   dt_m = s_g up_g dy_m
 *   dx_m = W^T dy_m + down_g^T dt_m,                   masked if asked
 *   ddown_g = sum over the adapter's rows of dt_m x_m^T
 *   dup_g   = sum over the adapter's rows of s_g t_m dy_m^T.
 * Rows may come in any order and any number per adapter; an adapter without
 * rows gets zero gradients.  A row's results depend on its own adapter only,
 * whatever another adapter holds (infinities, NaN), and the order of every sum
 * is fixed by the sizes and the ids.
 *
 * Layout: down is G x r rows of `in` values, up G x r rows of `out` values (so
 * both keep the layer's long axis contiguous; a checkpoint that stores up as
 * out x r is transposed once).  x, dy, dx, y, t: one row per batch row.
 * Leading dimensions are in elements, between rows; rows of a bank follow each
 * other (adapter g's rank j is row g r + j).
 *
 * Precision OT_FP32: x, W, down, up, dy and dx are fp32.  OT_BF16: they are
 * bf16.  y is fp32 or bf16 (y_type).  bias, scale, t and the gradients ddown and
 * dup are fp32.  Sums are fp32; t and dt enter further products unrounded (as fp32
 * operands, or as a sum of three bf16 terms), so a result is rounded to its type once.
 *
 * Alignment: device pointers to x, W, down, up, dy, dx, y, ddown and dup are
 * 16-byte aligned and their leading dimensions multiples of 8 (bf16) or 4
 * (fp32) elements, at least the row length (ld may be anything where there is
 * one row).  Values between a row's end and its leading dimension may be
 * anything and are not written.  bias, scale and t need their elements'
 * alignment only.
 *
 * Ownership: tensors are the caller's.  The object holds sizes and workspaces
 * (device memory on the device current at creation, which must be current in
 * every call).  Calls are asynchronous on the given stream; calls on one object
 * must not overlap, so a caller that changes streams orders them.  The workspaces
 * serve forwards and backwards alike: up to 272 bytes a row, and at most 0.5 GB of
 * partial sums.  A call with
 * more than max_rows rows replaces the workspaces, which waits for the device
 * and is refused (OT_E_STATE) under stream capture; any other call allocates
 * nothing and may be captured.  Workspaces named by a captured call are kept
 * until the object is destroyed.
 */
#ifndef OT_ADAPTERS_H
#define OT_ADAPTERS_H

#include <stdint.h>

#include "ot_status.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ot_adapters ot_adapters;

/* adapters_forward: y = max(y, 0).
 * adapters_backward: the layer's input x is itself a ReLU's output: dx is 0
 *   where x is not above 0. */
enum ot_adapters_flags { OT_ADAPTERS_RELU = 1, OT_ADAPTERS_RELU_INPUT = 2 };

/* Sizes of a bank: in, out in [1, 2^26], rank in [1, 64], n_adapters in
 * [1, 4096]; precision OT_FP32 or OT_BF16 (surrogate.h); max_rows: rows of the
 * largest call that the workspaces are first sized for, in [1, 2^20].
 * Errors: OT_E_INVAL, OT_E_NOMEM, OT_E_HIP. */
int adapters_create(ot_adapters** out, int64_t in, int64_t out_dim, int32_t rank, int32_t n_adapters,
                    int32_t precision, int64_t max_rows);

/* The adapted layer on n rows (0 <= n <= 2^20; 0 does nothing).
 * bias, scale: nullable.  ids: device int32[n].  y_type: OT_FP32 or OT_BF16.
 * t: n rows of rank fp32 at stride ldt, receives down_g x (zeros for rows
 * without an adapter) for a later adapters_backward; nullable.
 * flags: 0 or OT_ADAPTERS_RELU.
 * Errors: OT_E_INVAL, OT_E_STATE, OT_E_NOMEM, OT_E_HIP. */
int adapters_forward(ot_adapters* a, const void* x, int64_t ldx, const void* w, int64_t ldw, const float* bias,
                     const void* down, int64_t ldd, const void* up, int64_t ldu, const float* scale,
                     const int32_t* ids, int64_t n, void* y, int64_t ldy, int32_t y_type, float* t, int64_t ldt,
                     uint32_t flags, void* stream);

/* Gradients on n rows (0 <= n <= 2^20; 0 writes zero gradients of the bank).
 * t: what adapters_forward stored for these rows.  ddown, dup: receive the
 * bank's gradients (whole, not accumulated), at leading dimensions lddd, lddu.
 * dx: nullable (then W and down are not read and may be NULL).
 * flags: 0 or OT_ADAPTERS_RELU_INPUT.
 * Errors: OT_E_INVAL, OT_E_STATE, OT_E_NOMEM, OT_E_HIP. */
int adapters_backward(ot_adapters* a, const void* x, int64_t ldx, const void* w, int64_t ldw, const void* down,
                      int64_t ldd, const void* up, int64_t ldu, const float* scale, const int32_t* ids, int64_t n,
                      const void* dy, int64_t lddy, const float* t, int64_t ldt, float* ddown, int64_t lddd,
                      float* dup, int64_t lddu, void* dx, int64_t lddx, uint32_t flags, void* stream);

/* Free the workspaces (waits for the device). */
int adapters_destroy(ot_adapters* a);

#ifdef __cplusplus
}
#endif

#endif /* OT_ADAPTERS_H */
