/*
 * rms_norm.h -- C ABI of the root-mean-square norm with the residual's addition, forward and backward, part of the same library as
 * vp_ce.h (sm_100a).  It stands where layer_norm.h stands, for models whose last block ends in an RMS norm of the residual stream.
 *
 * For every row x of d elements, with the residual's row r (or none):
 *     z = x + r (rounded to the element type),  rstd = 1 / sqrt(mean(z^2) + eps),  y = z rstd g
 * The norm is of z as it is stored, so the backward pass, which reads z, differentiates what was computed.  With the upstream
 * gradients dy of y and dz of z (the residual stream's), a = dy g and zh = z rstd:
 *     dx = dr = rstd (a - zh mean(a zh)) + dz,     dg = sum over rows of dy zh
 * All statistics, sums and products are fp32; each result is rounded once to its own type.  So z^2 has to stay in fp32's range:
 * elements beyond about 1e19 make rstd 0, and with eps = 0 a row of zeros or of elements below about 1e-23 makes it infinite.  The sums
 * over rows have a fixed order: the same call gives the same bits every time.  A NaN or infinity in a row stays in that row's outputs
 * (and in dg, which sums over all rows).
 *
 * 8-bit output: y in groups of 128 neighbouring columns (the last one may be shorter), each with its own scale
 *     s = max|y| / 448  (at least 2^-126; 1 where the group is all zeros),     q = e4m3(y / s)
 * so that y = q s; s is max|y| times the fp32 number next to 1 / 448, q is rounded to nearest even from the fp32 y times the fp32
 * reciprocal of s: each within an fp32 unit of the quotient.  A NaN takes no part in the maximum
 * and stays a NaN; where a group holds an infinity its scale is infinite, the infinities become NaN and the rest 0.
 *
 * Element types (x_dtype, w_dtype): VPCE_BF16, VPCE_F16, VPCE_F32 of vp_ce_types.h.  x, residual, y, z, dy, dz, dx share x_dtype;
 * weight and its gradient share w_dtype, which is x_dtype or VPCE_F32.
 * Row strides are in elements and at least d; elements inside a row are contiguous.  Any alignment of the element type is accepted;
 * rows that all start on 16-byte boundaries take the faster kernels.
 *
 * Status codes are those of vp_ce.h (0 ok, 1 invalid argument, 2 unsupported, 3 workspace too small, 4 CUDA error).
 * Every call only enqueues work on `stream` (cudaStream_t as void*) of the current device.
 */
#ifndef RMS_NORM_H_
#define RMS_NORM_H_

#include <stddef.h>
#include <stdint.h>

#include "vp_ce_types.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * y [rows, d]; rstd (fp32 [rows]) is what the backward pass needs and may be NULL.  residual NULL: z is x, and z must be NULL.
 * z may be NULL where the sum is not wanted, and may be x or residual itself (same pointer and stride), as may y where z is not
 * wanted there.  weight NULL: ones (w_dtype is then ignored).  rows == 0 is a no-op; d >= 1; eps >= 0.
 */
int vp_rms_forward(const void* x, int x_dtype, int64_t rows, int64_t d, int64_t x_stride, const void* residual,
                   int64_t residual_stride, const void* weight, int w_dtype, double eps, void* y, int64_t y_stride, void* z,
                   int64_t z_stride, float* rstd, void* stream);

/*
 * The same with y as q [rows, d] (e4m3 bytes, row stride in bytes) and scales [rows][ceil(d / 128)] fp32, contiguous.
 */
int vp_rms_forward_fp8(const void* x, int x_dtype, int64_t rows, int64_t d, int64_t x_stride, const void* residual,
                       int64_t residual_stride, const void* weight, int w_dtype, double eps, void* q, int64_t q_stride, float* scales,
                       void* z, int64_t z_stride, float* rstd, void* stream);

/* Device bytes of workspace for vp_rms_backward: the partial sums over rows.  0 for invalid sizes. */
size_t vp_rms_workspace_bytes(int64_t rows, int64_t d);

/*
 * dx [rows, d] and dweight [d] (w_dtype) from dy, z (x itself where there was no residual), the forward call's rstd and dz
 * [rows, d] (NULL: zeros).  Either output may be NULL and is then not computed.  rows == 0 writes zeros to dweight.  dx may be dy or
 * dz itself (same pointer and stride).  workspace: 16-byte aligned; unused (may be NULL) when dweight is NULL.
 */
int vp_rms_backward(const void* dy, int64_t dy_stride, const void* dz, int64_t dz_stride, const void* z, int64_t z_stride, int x_dtype,
                    int64_t rows, int64_t d, const void* weight, int w_dtype, const float* rstd, void* dx, int64_t dx_stride,
                    void* dweight, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RMS_NORM_H_ */
