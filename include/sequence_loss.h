/*
 * sequence_loss.h -- C ABI of the two post-training losses over packed sequences of token log probabilities, part of the
 * same library as vp_ce.h (sm_100a).  They run directly behind the output head: logp is minus its per-token loss, and
 * minus dlogp is the upstream gradient (`dloss`) of its backward pass.
 *
 * Layout.  T tokens in one flat array; sequence s is the token range [seq_offsets[s], seq_offsets[s + 1]) (DEVICE int64,
 * rising; entries are clamped to [0, T], so a wrong one gives a wrong result but no access out of range).  Tokens outside
 * every sequence, and tokens whose mask byte is 0, take part in nothing: their values may be anything (NaN, infinity) and
 * their gradient is 0.  mask NULL: every token of every sequence counts.  All values are fp32, sums over tokens are fp32
 * inside a tile of tokens and double across tiles (and in what is formed from them: a pair's difference, a sequence's
 * weight), in a fixed order: the same call gives the same bits every time.
 *
 * Status codes are those of vp_ce.h.  Every call only enqueues work on `stream` of the current device.  Workspaces are
 * DEVICE buffers, 16-byte aligned, owned by the caller; they need no initialisation.  A workspace keeps, until its next
 * use, what vp_*_loss_backward needs of the call that filled it.
 */
#ifndef SEQUENCE_LOSS_H_
#define SEQUENCE_LOSS_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Clipped policy loss with a KL term.  Per token, with r = exp(logp - old_logp) and A its advantage:
 *     l = - min(r A, clip(r, 1 - clip_low, 1 + clip_high) A) + kl_coef (e^q - q - 1),      q = ref_logp - logp
 * aggregate VPCE_TOKEN_MEAN: mean of l over all valid tokens; VPCE_SEQ_MEAN: the mean over the sequences that have a
 * valid token of each one's mean over its valid tokens.  0 when there is no valid token.
 *     dl / dlogp = - A r  where the minimum takes the unclipped term, else 0,     + kl_coef (1 - e^q)
 * The minimum takes the clipped term where A > 0 and r > 1 + clip_high, or A < 0 and r < 1 - clip_low.
 *
 *   ref_logp            NULL: no KL term (kl_coef is then ignored)
 *   advantages          fp32 [T] (adv_per_token != 0) or [n_seqs]
 *   stats               fp32 [4], written: loss; means over valid tokens of the KL estimate, of "clipped", of r
 *   dlogp               fp32 [T], written with upstream * dloss/dlogp (every element), or NULL: forward only
 *   upstream            DEVICE fp32 scalar or NULL (= 1)
 * T == 0 or n_seqs == 0: stats (and dlogp) are 0.
 *
 * A batch in parts (over ranks, or accumulated): the mean is over the tokens (or sequences) of one call.  With n valid
 * tokens here and N in all parts, upstream = n / N gives this part's gradient of the mean over all of them, and the sum of
 * the parts' loss n / N is that mean; with VPCE_SEQ_MEAN, n and N count sequences that have a valid token.
 */
enum { VPCE_TOKEN_MEAN = 0, VPCE_SEQ_MEAN = 1 };
size_t vp_policy_loss_workspace_bytes(int64_t T, int64_t n_seqs);
int vp_policy_loss(const float* logp, const float* old_logp, const float* ref_logp, const float* advantages,
                   int adv_per_token, const uint8_t* mask, const int64_t* seq_offsets, int64_t T, int64_t n_seqs,
                   double clip_low, double clip_high, double kl_coef, int aggregate, float* stats, float* dlogp,
                   const float* upstream, void* workspace, size_t workspace_bytes, void* stream);
/* The gradient alone, after vp_policy_loss with the same inputs, settings and workspace. */
int vp_policy_loss_backward(const float* logp, const float* old_logp, const float* ref_logp, const float* advantages,
                            int adv_per_token, const uint8_t* mask, const int64_t* seq_offsets, int64_t T,
                            int64_t n_seqs, double clip_low, double clip_high, double kl_coef, int aggregate,
                            float* dlogp, const float* upstream, const void* workspace, size_t workspace_bytes,
                            void* stream);

/*
 * Preference loss over n_pairs pairs: sequence i is the preferred answer of pair i and sequence n_pairs + i the other
 * one (2 n_pairs sequences).  With s = sum over a sequence's valid tokens of (logp - ref_logp), divided by their number
 * if `average` (0 for a sequence without valid tokens), and D = s_i - s_{n_pairs + i}:
 *     VPCE_PREF_SIGMOID  z = beta D - margin,  l = - (1 - e) log sigmoid(z) - e log sigmoid(-z),  e = label_smoothing
 *     VPCE_PREF_IPO      l = (D - 1 / (2 beta))^2
 * and the loss is the mean of l over the pairs.
 *
 *   ref_logp            NULL: zeros
 *   stats               fp32 [3], written: loss, share of pairs with D > 0, mean of beta D
 *   rewards             fp32 [2 n_pairs], written: beta s; or NULL
 *   dlogp, upstream     as above
 * n_pairs == 0 or T == 0 is allowed (n_pairs == 0: stats are 0).
 */
enum { VPCE_PREF_SIGMOID = 0, VPCE_PREF_IPO = 1 };
size_t vp_preference_loss_workspace_bytes(int64_t T, int64_t n_pairs);
int vp_preference_loss(const float* logp, const float* ref_logp, const uint8_t* mask, const int64_t* seq_offsets,
                       int64_t T, int64_t n_pairs, double beta, double margin, double label_smoothing, int kind,
                       int average, float* stats, float* rewards, float* dlogp, const float* upstream, void* workspace,
                       size_t workspace_bytes, void* stream);
/* The gradient alone, after vp_preference_loss with the same inputs, settings and workspace. */
int vp_preference_loss_backward(const uint8_t* mask, const int64_t* seq_offsets, int64_t T, int64_t n_pairs,
                                float* dlogp, const float* upstream, const void* workspace, size_t workspace_bytes,
                                void* stream);

#ifdef __cplusplus
}
#endif
#endif /* SEQUENCE_LOSS_H_ */
