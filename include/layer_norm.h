/*
 * layer_norm.h -- C ABI of layer normalisation, forward and backward, part of the same library as vp_ce.h (sm_100a).
 * It is what runs directly before the output head: its output is the head's H and its upstream gradient the head's dH.
 *
 * For every row x of d elements:
 *     mu = mean(x),  var = mean((x - mu)^2),  rstd = 1 / sqrt(var + eps),  xh = (x - mu) rstd,  y = xh g + b
 * and with the upstream gradient dy, a = dy g:
 *     dx = rstd (a - mean(a) - xh mean(a xh)),     dg = sum over rows of dy xh,     db = sum over rows of dy
 * All statistics, sums and products are fp32; each result is rounded once to its own type.  The variance is taken from
 * the centred values (never mean(x^2) - mu^2), so a large common offset costs no digits.  The sums over rows have a
 * fixed order: the same call gives the same bits every time.  A NaN or infinity in a row stays in that row's y and dx
 * (and in dg, db, which sum over all rows).
 *
 * Element types (x_dtype, w_dtype): VPCE_BF16, VPCE_F16, VPCE_F32 of vp_ce_types.h.  x, y, dy, dx share x_dtype;
 * weight, bias and their gradients share w_dtype, which is x_dtype or VPCE_F32.
 * Row strides are in elements and at least d; elements inside a row are contiguous.  Any alignment of the element type
 * is accepted; rows that all start on 16-byte boundaries take the faster kernels.
 *
 * Status codes are those of vp_ce.h (0 ok, 1 invalid argument, 2 unsupported, 3 workspace too small, 4 CUDA error).
 * Every call only enqueues work on `stream` (cudaStream_t as void*) of the current device.
 */
#ifndef LAYER_NORM_H_
#define LAYER_NORM_H_

#include <stddef.h>
#include <stdint.h>

#include "vp_ce_types.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * y [rows, d]; mean and rstd (fp32 [rows]) are what the backward pass needs and may both be NULL.  weight NULL: ones;
 * bias NULL: zeros (w_dtype is then ignored if both are NULL).  rows == 0 is a no-op; d >= 1; eps >= 0.
 * y may be x itself (same pointer and stride).
 */
int vp_ln_forward(const void* x, int x_dtype, int64_t rows, int64_t d, int64_t x_stride, const void* weight,
                  const void* bias, int w_dtype, double eps, void* y, int64_t y_stride, float* mean, float* rstd,
                  void* stream);

/* Device bytes of workspace for vp_ln_backward: the partial sums over rows.  0 for invalid sizes. */
size_t vp_ln_workspace_bytes(int64_t rows, int64_t d);

/*
 * dx [rows, d], dweight [d], dbias [d] (w_dtype) from dy, x and the forward call's mean and rstd.  Each of the three
 * outputs may be NULL and is then not computed.  rows == 0 writes zeros to dweight and dbias.  dx may be dy itself
 * (same pointer and stride).  workspace: 16-byte aligned; unused (may be NULL) when dweight and dbias are NULL.
 */
int vp_ln_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int x_dtype, int64_t rows,
                   int64_t d, const void* weight, int w_dtype, const float* mean, const float* rstd, void* dx,
                   int64_t dx_stride, void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* LAYER_NORM_H_ */
