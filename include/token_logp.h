/*
 * token_logp.h -- C ABI of the log probabilities of given tokens with entropy and top alternatives, part of the same library as
 * vp_ce.h (sm_100a).  Like the head's loss it starts from hidden states and the projection weight and never forms the tokens x
 * vocabulary logits in memory; beside the loss's  -log p(token)  it gives what policy training and generation also ask for.
 *
 * For every token n with logits x = H[n, :] W^T / temperature and p = softmax(x):
 *     lse = log sum_v exp(x_v),   logp = x_{tokens[n]} - lse,   entropy = lse - sum_v p_v x_v,
 *     alternatives: the `top` largest x_v, larger first and among equals the lower v, as (x_v - lse, v)
 * The alternatives' order is that of the fp32 logits before the division by the temperature.  With upstream gradients dlogp, dent:
 *     dx_v = dlogp ([v = tokens[n]] - p_v) - dent p_v (x_v - lse + entropy),     dH = dx W / temperature,  dW = dx^T H / temperature
 * Alternatives have no gradient.
 *
 * Tokens: int32; ignore_index, or any number outside [0, V), gives logp 0 and no gradient of logp (the latter also sets
 * VPCE_DEV_LABEL_OUT_OF_RANGE in the status word); lse, entropy (with its gradient) and alternatives do not depend on the token.
 * Products are exact products of the inputs accumulated in fp32; statistics are fp32 (exponentials the hardware's approximate ones, 2^-22
 * relative) and joined in a fixed order: the same call gives the same bits every time.  A NaN among a token's logits makes its lse, logp
 * and entropy NaN and is not an alternative; alternatives that do not exist for that reason have id -1 and value -inf.  Where a logit is infinite (an overflow, or an infinity among the inputs) or
 * lies 2e38 x temperature or more below the token's largest one, that token's lse, logp and entropy are undefined; other tokens'
 * are not touched.
 *
 * 8-bit operands: e4m3 numbers with fp32 scales, one for each 128 columns of a row of H and for each 128 x 128 block of W
 *     x_v = sum over blocks b of 128 columns:  Hs[n, b] Ws[v / 128, b] (sum over k in b of Hq[n, k] Wq[v, k])
 * (what vp_rms_forward_fp8 and vp_fp8_quantize_blocks write).  The scales are applied in fp32 to each block's sum.
 *
 * Where a wait in a forward call runs out (VPCE_DEV_WAIT_EXPIRED, vp_ce_set_wait_limit_ns), every token that it may concern gets NaN as
 * lse, entropy and logp (0 without a token) and no alternatives (-1, -inf), so that it shows where the status word is not read, too.
 *
 * Conventions (alignment, streams, status codes) are vp_ce.h's: tensors are contiguous device memory and 16-byte aligned; bf16: d a
 * multiple of 8; 8 bits: d a multiple of 16, at most 16384.  The workspace's first word is the status word of vp_ce_device_status.
 */
#ifndef TOKEN_LOGP_H_
#define TOKEN_LOGP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define VP_TOKEN_LOGP_MAX_TOP 20

/* Bytes of workspace of the two forward calls: bounded, whatever T and V (under 100 MB).  0 for sizes that they would reject. */
size_t vp_token_logp_workspace_bytes(int64_t T, int64_t d, int64_t V, int top);
size_t vp_token_logp_fp8_workspace_bytes(int64_t T, int64_t d, int64_t V, int top);

/*
 * H [T, d] and W [V, d] bf16.  tokens and logp may both be NULL; lse, entropy may be NULL; top_logp [T, top] fp32 and top_ids [T, top]
 * int32 are needed where top > 0 (0 <= top <= min(V, VP_TOKEN_LOGP_MAX_TOP)).  temperature: 1e-6 to 1e6.  T == 0 launches nothing.
 */
int vp_token_logp_forward(const void* H, const void* W, const int32_t* tokens, int64_t T, int64_t d, int64_t V, double temperature,
                          int32_t ignore_index, float* logp, float* lse, float* entropy, float* top_logp, int32_t* top_ids, int top,
                          void* workspace, size_t workspace_bytes, void* stream);

/* The same from 8-bit operands: Hq [T, d], Wq [V, d] e4m3, Hs [T, ceil(d / 128)], Ws [ceil(V / 128), ceil(d / 128)] fp32. */
int vp_token_logp_fp8_forward(const void* Hq, const float* Hs, const void* Wq, const float* Ws, const int32_t* tokens, int64_t T,
                              int64_t d, int64_t V, double temperature, int32_t ignore_index, float* logp, float* lse, float* entropy,
                              float* top_logp, int32_t* top_ids, int top, void* workspace, size_t workspace_bytes, void* stream);

/*
 * dH [T, d] bf16 (overwritten) and dW [V, d] fp32 (overwritten, or added to when accumulate_dW) from the forward call's lse and
 * entropy (needed with dent only).  dlogp or dent [T] may be NULL (zeros), as may dH or dW (not computed), one of each at least given.
 * block_v, T_chunk, chunk_index_base and the workspace (vp_ce_workspace_bytes) are those of vp_ce_backward, which this call extends.
 *
 * temperature: 0.01 to 100, narrower than the forward call's.  p is formed anew as exp(x - lse) from lse in one fp32 number, so that it is off
 * by up to 2^-22 (|lse| + |log p| + 1) relative (7e-4 at temperature 0.01 and logits of 30), and log p + entropy by up to
 * 2^-21 (|lse| + |log p| + entropy) absolute.
 * dx is rounded to bf16 before both products (half a step, 2^-8 of each entry; the token's own entry is put back exactly), as in
 * vp_ce_backward: errors that average out where p varies, and add up where all of p lies within a step (nearly uniform p) and rows
 * of W have a common mean.  Sums and dW are fp32, dH is rounded once.
 */
int vp_token_logp_backward(const void* H, const void* W, const int32_t* tokens, const float* lse, const float* entropy,
                           const float* dlogp, const float* dent, void* dH, float* dW, int64_t T, int64_t d, int64_t V, double temperature,
                           int64_t block_v, int32_t ignore_index, int64_t T_chunk, int64_t chunk_index_base, int accumulate_dW,
                           void* workspace, size_t workspace_bytes, void* stream);

/*
 * TEST HOOK: the next forward launch loses the copies of k-block `k_block` of its first tile (nothing is accessed out of bounds), so
 * that its waits run out and it gives up as vp_ce_set_wait_limit_ns describes.  One-shot; k_block < 0 disarms.
 */
int vp_token_logp_debug_drop(int k_block);

#ifdef __cplusplus
}
#endif
#endif /* TOKEN_LOGP_H_ */
