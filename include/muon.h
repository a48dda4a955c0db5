/*
 * muon.h -- C ABI of the Muon update: momentum, orthogonalisation of the update by Newton-Schulz products, and the fused
 * write-back to the fp32 master and the bf16 working weight; part of the same library as vp_ce.h (sm_100a).  It stands
 * beside osadamw_update_device (stream_adamw.h) for weights that are matrices.
 *
 * For each of `batch` matrices of one shape (C order, contiguous), with gradient G:
 *     M <- mu M + G,        U = G + mu M (nesterov) or M
 *     X_0 = U / max(|U|_F, eps)                       (worked on as its transpose where rows > cols)
 *     A = X X^T,   B = b A + c A A,   X <- a X + B X  for each of the `steps` triples (a, b, c)
 *     p <- p (1 - lr weight_decay) - lr scale X,      w = bf16(p)
 *
 * The three products run on the tensor cores.  X, A and B are held in fp16 between products, each multiplied by a power
 * of two that follows from the iteration's own bound (the spectral norm of X stays below the largest |a s + b s^3 + c s^5|
 * over 0 <= s <= its bound before the step), so nothing overflows and eleven bits of every entry survive; products
 * accumulate in fp32, the last X never leaves fp32.  M, p, the norm and all elementwise arithmetic are fp32 (squares are
 * formed and summed in fp32 over up to eight neighbours, in double beyond: entries above 1e19 overflow, as they would in
 * a plain fp32 norm).  The rounding to fp16 shows in the result as about 1.5e-3 of its Frobenius norm for gradients of full
 * rank; in directions that a gradient lacks (a rank below the smaller side) it is amplified like the iteration amplifies
 * everything small, by the product of the a's (485 for the default steps), and reaches some 4e-2 for a rank of a fifteenth.  A NaN or infinity in one matrix's gradient stays in that matrix.
 *
 * Status codes are those of vp_ce.h.  VPCE_UNSUPPORTED: coefficients whose bound leaves the fp16 range (a bound on X
 * above 8), sizes whose tiles do not fit 31 bits.  Every call only enqueues work on `stream` of the current device.
 */
#ifndef MUON_H_
#define MUON_H_

#include <stddef.h>
#include <stdint.h>

#include "vp_ce_types.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Device bytes of workspace for `batch` matrices rows x cols.  0 for invalid or unsupported sizes. */
size_t muon_workspace_bytes(int64_t batch, int64_t rows, int64_t cols);

/*
 * O = the orthogonalised G (X after the last step), without momentum.  g_dtype and o_dtype: VPCE_BF16, VPCE_F16 or
 * VPCE_F32.  coeffs: HOST double [steps][3], or NULL for (3.4445, -4.7750, 2.0315) in every step; 1 <= steps <= 32.
 * O may be G itself when the types agree.  workspace: 256-byte aligned.  batch, rows or cols == 0 is a no-op.
 */
int muon_orthogonalize(const void* G, int g_dtype, void* O, int o_dtype, int64_t batch, int64_t rows, int64_t cols,
                       const double* coeffs, int steps, double eps, void* workspace, size_t workspace_bytes,
                       void* stream);

/*
 * One update.  p (fp32 master) and m (fp32 momentum) are updated in place; w_bf16 (may be NULL) is written; grad is
 * VPCE_BF16, VPCE_F16 or VPCE_F32.  0 <= mu < 1.
 */
int muon_step(float* p, float* m, const void* grad, int g_dtype, void* w_bf16, int64_t batch, int64_t rows, int64_t cols,
              double lr, double mu, int nesterov, double weight_decay, double scale, const double* coeffs, int steps,
              double eps, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Reads back the status word that the last call wrote to its workspace (synchronises `stream`): 0, or
 * VPCE_DEV_WAIT_EXPIRED (vp_ce.h) when a wait inside the kernels ran out (vp_ce_set_wait_limit_ns).  The call has then
 * given up: m is updated, but each element of p, w_bf16 and O holds either its old or its new value.  What was in flight
 * has ended, the context stays usable and the next call on the workspace starts clean.
 */
int muon_device_status(const void* workspace, int32_t* status_out, void* stream);

/*
 * TEST HOOK: makes a signal of the next launch "get lost", so that the give-up path can be exercised without any invalid
 * access.  kernel_kind 0, the kernel of large matrices: the operand copies of k-block `index` of the first tile of its
 * work list are not issued in the CTAs named by `cta_ranks` (bit 0: the leader of a CTA pair, bit 1: the other one).
 * kernel_kind 1, the one-launch kernel of small matrices: the end of product `index` (three a step) of the first matrix
 * is not signalled.  One-shot: the launch that consumes it disarms it; kernel_kind < 0 disarms.  VPCE_INVALID_ARG for
 * values out of range.
 */
int muon_debug_drop(int kernel_kind, int index, int cta_ranks);

#ifdef __cplusplus
}
#endif
#endif /* MUON_H_ */
