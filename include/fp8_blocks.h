/*
 * fp8_blocks.h -- C ABI of the quantisation of a weight to 8 bits in blocks of 128 x 128, part of the same library as vp_ce.h
 * (sm_100a).  It makes what vp_token_logp_fp8_forward (token_logp.h) takes as its weight.
 *
 * For every block of 128 rows by 128 columns (the last ones may be smaller):
 *     s = max|w| / 448  (at least 2^-126; 1 where the block is all zeros),     q = e4m3(w / s)
 * so that w = q s; s is max|w| times the fp32 number next to 1 / 448, q is rounded to nearest even from w times the fp32 reciprocal
 * of s: each within an fp32 unit of the quotient.  A NaN takes no part in the maximum and stays
 * a NaN; where a block holds an infinity its scale is infinite, the infinities become NaN and the rest 0.
 *
 * w: VPCE_BF16, VPCE_F16 or VPCE_F32 (vp_ce_types.h), any alignment of its type; row strides in elements (bytes for q), at least d.
 * scales [ceil(rows / 128)][ceil(d / 128)] fp32, contiguous.  Status codes are those of vp_ce.h; rows == 0 is a no-op.
 */
#ifndef FP8_BLOCKS_H_
#define FP8_BLOCKS_H_

#include <stdint.h>

#include "vp_ce_types.h"

#ifdef __cplusplus
extern "C" {
#endif

int vp_fp8_quantize_blocks(const void* w, int w_dtype, int64_t rows, int64_t d, int64_t w_stride, void* q, int64_t q_stride,
                           float* scales, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FP8_BLOCKS_H_ */
