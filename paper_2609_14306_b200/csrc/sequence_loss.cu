// Clipped policy loss and preference loss over packed sequences (sequence_loss.h).
//
// Sums over ragged sequences are split over tokens, not over sequences, so one sequence of a million tokens and a thousand
// of a thousand cost the same: a warp owns a tile of consecutive tokens and sums, for every sequence that meets its tile,
// the tokens inside it.  A sequence that lies inside one tile is finished there; of one that spans tiles each tile leaves
// its piece (`first`: the piece of the sequence that reaches into the tile from before, `last`: of the one that leaves it at
// the end).  One block then joins the pieces in the order of the tiles, forms the loss and a weight per sequence; a third
// pass over the tokens writes the gradient.

#include <cuda_runtime.h>

#include <cstdint>

#include "sequence_loss.h"
#include "vp_ce.h"

namespace {

constexpr int THREADS = 128;                    // four warps, each with a tile of its own
constexpr int WARPS = THREADS / 32;
constexpr int PER_LANE = 8;                     // tokens of one lane in a step: a step covers 256 tokens
constexpr int STEP = 32 * PER_LANE;
constexpr int64_t MAX_TILES = 2048;             // the tile grows with T beyond 512 Ki tokens: bounds what one block joins
constexpr int FIN_THREADS = 1024;
constexpr unsigned ALL = 0xffffffffu;

// What the kernels of one call share.  Everything below `seq_sum` lies in the workspace.
struct SeqArgs {
    const float *logp, *old_logp, *ref_logp, *adv;
    const uint8_t* mask;
    const int64_t* offsets;
    long T, n_seqs;
    int steps;                                  // steps of 256 tokens per tile
    long n_tiles;
    int adv_per_token, by_seq;                  // by_seq: the loss needs sums per sequence
    float lo, hi, kl_coef;
    float2 *first, *last;                       // [n_tiles] pieces: (sum, count)
    float2* seq_sum;                            // [n_seqs] (sum, count)
    float* tile_stats;                          // [5][n_tiles] count, sum of l, KL, clipped, r
    float* weight;                              // [n_seqs + 1] weight of a sequence's tokens; the last: of every token
    // preference
    double beta, margin, smoothing;
    int kind, average;
    float *stats, *rewards, *dlogp;
    const float* upstream;
};

__device__ __forceinline__ float wsum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(ALL, v, o);
    return v;
}

__device__ __forceinline__ long seq_begin(const SeqArgs& a, long s) {
    const long v = a.offsets[s];
    return v < 0 ? 0 : v > a.T ? a.T : v;
}

// The first sequence that ends behind token t (n_seqs if none does): 32 probes a round.
__device__ __forceinline__ long first_seq(const SeqArgs& a, long t, int lane) {
    long lo = 0, hi = a.n_seqs;                 // the answer is in [lo, hi]
    while (hi > lo) {
        const long step = (hi - lo + 31) / 32;
        const long probe = lo + step * (lane + 1) - 1;
        const bool beyond = probe >= hi || seq_begin(a, probe + 1) > t;   // the answer is <= probe
        const unsigned ball = __ballot_sync(ALL, beyond);
        const int k = ball ? __ffs(ball) - 1 : 32;
        const long nlo = lo + step * k;
        const long nhi = k == 32 ? hi : lo + step * (k + 1) - 1;
        lo = nlo < hi ? nlo : hi;
        hi = nhi < hi ? nhi : hi;
    }
    return lo;
}

// Terms of one token of the policy loss.  `clipped` compares in fp32, so a ratio exactly on a bound counts as unclipped.
struct Policy { float l, grad, kl, clipped, r; };
__device__ __forceinline__ Policy policy_token(const SeqArgs& a, float logp, float old_logp, float ref, float adv) {
    Policy p;
    p.r = expf(logp - old_logp);
    const bool clip = (adv > 0.f && p.r > a.hi) || (adv < 0.f && p.r < a.lo);
    p.clipped = clip ? 1.f : 0.f;
    p.l = -((clip ? (adv > 0.f ? a.hi : a.lo) : p.r) * adv);
    p.grad = clip ? 0.f : -adv * p.r;
    p.kl = 0.f;
    if (a.ref_logp) {
        const float q = ref - logp, e = expf(q);
        p.kl = e - q - 1.f;
        p.l += a.kl_coef * p.kl;
        p.grad += a.kl_coef * (1.f - e);
    }
    return p;
}

// Calls f(s, begin, end) for every sequence s that meets the tokens [t0, t1), with its range cut to them.
template <typename F>
__device__ __forceinline__ void for_sequences(const SeqArgs& a, long t0, long t1, int lane, F f) {
    for (long s = first_seq(a, t0, lane); s < a.n_seqs; ++s) {
        const long b = seq_begin(a, s), e = seq_begin(a, s + 1);
        if (b >= t1) break;
        if (e > b && e > t0) f(s, b, e);
    }
}

// Pass 1: sums of each tile.  POLICY: value = l and the four statistics; else value = logp - ref_logp.
template <bool POLICY>
__global__ void __launch_bounds__(THREADS) seq_sums_kernel(const SeqArgs a) {
    const int lane = threadIdx.x & 31;
    const long tile = static_cast<long>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
    if (tile >= a.n_tiles) return;                                          // the whole warp
    const long span = static_cast<long>(a.steps) * STEP;
    const long t0 = tile * span, t1 = t0 + span < a.T ? t0 + span : a.T;
    float2 first = make_float2(0.f, 0.f), last = first;
    float cnt = 0.f, sl = 0.f, skl = 0.f, sclip = 0.f, sr = 0.f;
    for_sequences(a, t0, t1, lane, [&](long s, long sb, long se) {
        const long b = sb > t0 ? sb : t0, e = se < t1 ? se : t1;
        const float adv_s = POLICY && !a.adv_per_token ? a.adv[s] : 0.f;
        float sum = 0.f, n = 0.f;
        for (long c = b; c < e; c += STEP) {
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                const long t = c + j * 32 + lane;
                if (t < e && (!a.mask || a.mask[t])) {
                    n += 1.f;
                    if (POLICY) {
                        const Policy p = policy_token(a, a.logp[t], a.old_logp[t], a.ref_logp ? a.ref_logp[t] : 0.f,
                                                      a.adv_per_token ? a.adv[t] : adv_s);
                        sum += p.l;
                        skl += p.kl; sclip += p.clipped; sr += p.r;
                    } else {
                        sum += a.logp[t] - (a.ref_logp ? a.ref_logp[t] : 0.f);
                    }
                }
            }
        }
        if (a.by_seq) {
            const float2 v = make_float2(wsum(sum), wsum(n));
            if (sb >= t0 && se <= t1) { if (lane == 0) a.seq_sum[s] = v; }
            else if (sb < t0) first = v;
            else last = v;
        }
        cnt += n; sl += sum;
    });
    if (a.by_seq && lane == 0) { a.first[tile] = first; a.last[tile] = last; }
    if (POLICY) {
        cnt = wsum(cnt); sl = wsum(sl); skl = wsum(skl); sclip = wsum(sclip); sr = wsum(sr);
        if (lane == 0) {
            float* o = a.tile_stats + tile;
            o[0] = cnt; o[a.n_tiles] = sl; o[2 * a.n_tiles] = skl; o[3 * a.n_tiles] = sclip; o[4 * a.n_tiles] = sr;
        }
    }
}

// Sums of K doubles over the block (fixed order); every thread receives them.
template <int K>
__device__ __forceinline__ void block_sum(double (&v)[K], double (*part)[K]) {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(ALL, v[k], o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        for (int k = 0; k < K; ++k) part[threadIdx.x >> 5][k] = v[k];
    __syncthreads();
    for (int k = 0; k < K; ++k) {
        v[k] = part[threadIdx.x & 31][k];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v[k] += __shfl_xor_sync(ALL, v[k], o);
    }
}

// (sum, count) of sequence s by the lanes of a group of `width` lanes (a power of two up to 32), pieces in a fixed order.
__device__ __forceinline__ double2 join_pieces(const SeqArgs& a, long s, int sub, int width) {
    double2 v = make_double2(0.0, 0.0);
    if (s < a.n_seqs) {
        const long b = seq_begin(a, s), e = seq_begin(a, s + 1);
        if (e > b) {
            const long span = static_cast<long>(a.steps) * STEP;
            const long ta = b / span, tb = (e - 1) / span;
            if (ta == tb) {
                // inside one tile: finished there
                if (sub == 0) { const float2 f = a.seq_sum[s]; v.x = f.x; v.y = f.y; }
            } else {
                if (sub == 0) { const float2 f = a.last[ta]; v.x = f.x; v.y = f.y; }
                for (long t = ta + 1 + sub; t <= tb; t += width) { const float2 f = a.first[t]; v.x += f.x; v.y += f.y; }
            }
        }
    }
    for (int o = width / 2; o > 0; o >>= 1) {
        v.x += __shfl_xor_sync(ALL, v.x, o);
        v.y += __shfl_xor_sync(ALL, v.y, o);
    }
    return v;
}

// Lanes that join one sequence's pieces: enough that all sequences are in flight at once, 32 at most.
__device__ __forceinline__ int join_width(long n_seqs) {
    int w = 32;
    while (w > 1 && static_cast<long>(FIN_THREADS / w) < n_seqs) w >>= 1;
    return w;
}

__global__ void __launch_bounds__(FIN_THREADS) policy_finish_kernel(const SeqArgs a) {
    __shared__ double part[32][5];
    __shared__ double part2[32][2];
    double v[5] = {0, 0, 0, 0, 0};
    for (long t = threadIdx.x; t < a.n_tiles; t += FIN_THREADS)
#pragma unroll
        for (int k = 0; k < 5; ++k) v[k] += a.tile_stats[k * a.n_tiles + t];
    block_sum<5>(v, part);
    const double inv = v[0] > 0 ? 1.0 / v[0] : 0.0;
    double loss = v[1] * inv;
    if (a.by_seq) {
        const int width = join_width(a.n_seqs), per_round = FIN_THREADS / width;
        double u[2] = {0, 0};                                               // sum of the sequences' means, sequences that have one
        for (long s0 = 0; s0 < a.n_seqs; s0 += per_round) {
            const long s = s0 + threadIdx.x / width;
            const double2 w = join_pieces(a, s, threadIdx.x % width, width);
            if (threadIdx.x % width == 0 && s < a.n_seqs) {
                a.weight[s] = w.y > 0 ? static_cast<float>(w.y) : 0.f;      // the count, until the number of sequences is known
                if (w.y > 0) { u[0] += w.x / w.y; u[1] += 1.0; }
            }
        }
        block_sum<2>(u, part2);
        loss = u[1] > 0 ? u[0] / u[1] : 0.0;
        for (long s0 = 0; s0 < a.n_seqs; s0 += per_round) {                 // each thread meets the entries that it wrote
            const long s = s0 + threadIdx.x / width;
            if (threadIdx.x % width == 0 && s < a.n_seqs) {
                const double n = a.weight[s];
                a.weight[s] = n > 0 ? static_cast<float>(1.0 / (n * u[1])) : 0.f;
            }
        }
    }
    if (threadIdx.x == 0) {
        a.weight[a.n_seqs] = static_cast<float>(inv);
        a.stats[0] = static_cast<float>(loss);
        a.stats[1] = static_cast<float>(v[2] * inv);
        a.stats[2] = static_cast<float>(v[3] * inv);
        a.stats[3] = static_cast<float>(v[4] * inv);
    }
}

__global__ void __launch_bounds__(FIN_THREADS) preference_finish_kernel(const SeqArgs a) {
    __shared__ double part[32][3];
    const long pairs = a.n_seqs / 2;
    const int width = join_width(a.n_seqs), per_round = FIN_THREADS / width;
    for (long s0 = 0; s0 < a.n_seqs; s0 += per_round) {
        const long s = s0 + threadIdx.x / width;
        const double2 w = join_pieces(a, s, threadIdx.x % width, width);
        if (threadIdx.x % width == 0 && s < a.n_seqs) {
            const double n = a.average ? (w.y > 0 ? w.y : 1.0) : 1.0;
            a.seq_sum[s] = make_float2(static_cast<float>(w.x / n), static_cast<float>(n));
            if (a.rewards) a.rewards[s] = static_cast<float>(a.beta * (w.x / n));
        }
    }
    __syncthreads();
    double v[3] = {0, 0, 0};
    for (long i = threadIdx.x; i < pairs; i += FIN_THREADS) {
        const float2 c = a.seq_sum[i], r = a.seq_sum[pairs + i];
        const double diff = static_cast<double>(c.x) - static_cast<double>(r.x);
        double l, slope;
        if (a.kind == VPCE_PREF_SIGMOID) {
            const double z = a.beta * diff - a.margin;
            const double tail = log1p(exp(-fabs(z)));                       // log(1 + e^-|z|)
            const double neg = (z < 0 ? -z : 0.0) + tail;                   // -log sigmoid(z)
            const double pos = (z > 0 ? z : 0.0) + tail;                    // -log sigmoid(-z)
            l = (1.0 - a.smoothing) * neg + a.smoothing * pos;
            slope = a.beta * (a.smoothing - 1.0 / (1.0 + exp(z)));
        } else {
            const double g = diff - 1.0 / (2.0 * a.beta);
            l = g * g;
            slope = 2.0 * g;
        }
        v[0] += l;
        v[1] += diff > 0 ? 1.0 : 0.0;
        v[2] += a.beta * diff;
        slope /= static_cast<double>(pairs);
        a.weight[i] = static_cast<float>(slope / c.y);
        a.weight[pairs + i] = static_cast<float>(-slope / r.y);
    }
    block_sum<3>(v, part);
    if (threadIdx.x == 0)
        for (int k = 0; k < 3; ++k) a.stats[k] = pairs > 0 ? static_cast<float>(v[k] / static_cast<double>(pairs)) : 0.f;
}

// Pass 3: the gradient of every token.
template <bool POLICY>
__global__ void __launch_bounds__(THREADS) seq_grad_kernel(const SeqArgs a) {
    const int lane = threadIdx.x & 31;
    const long tile = static_cast<long>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
    if (tile >= a.n_tiles) return;
    const long span = static_cast<long>(a.steps) * STEP;
    const long t0 = tile * span, t1 = t0 + span < a.T ? t0 + span : a.T;
    const float up = a.upstream ? *a.upstream : 1.f;
    const float w_all = POLICY && !a.by_seq ? a.weight[a.n_seqs] * up : 0.f;
    long done = t0;                                                         // everything before is written
    auto zeros = [&](long to) { for (long t = done + lane; t < to; t += 32) a.dlogp[t] = 0.f; };
    for_sequences(a, t0, t1, lane, [&](long s, long sb, long se) {
        const long b = sb > t0 ? sb : t0, e = se < t1 ? se : t1;
        if (b < done) return;                                               // offsets that do not rise: every token is written once
        zeros(b);
        const float w = POLICY && !a.by_seq ? w_all : a.weight[s] * up;
        const float adv_s = POLICY && !a.adv_per_token ? a.adv[s] : 0.f;
        for (long c = b; c < e; c += STEP) {
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                const long t = c + j * 32 + lane;
                if (t < e) {
                    float g = 0.f;
                    if (!a.mask || a.mask[t]) {
                        if (POLICY)
                            g = w * policy_token(a, a.logp[t], a.old_logp[t], a.ref_logp ? a.ref_logp[t] : 0.f,
                                                 a.adv_per_token ? a.adv[t] : adv_s).grad;
                        else
                            g = w;
                    }
                    a.dlogp[t] = g;
                }
            }
        }
        done = e;
    });
    zeros(t1);
}

// ------------------------------------------------------------------------------------ host side
constexpr int64_t MAX_T = int64_t{1} << 40, MAX_SEQS = int64_t{1} << 30;

int64_t steps_for(int64_t T) {
    const int64_t tiles = (T + STEP - 1) / STEP;
    return tiles <= MAX_TILES ? 1 : (tiles + MAX_TILES - 1) / MAX_TILES;
}
int64_t tiles_for(int64_t T) {
    const int64_t span = steps_for(T) * STEP;
    return (T + span - 1) / span;
}

size_t up16(size_t x) { return (x + 15) / 16 * 16; }

size_t workspace_for(int64_t T, int64_t n_seqs, SeqArgs* a, void* base) {
    const size_t tiles = static_cast<size_t>(tiles_for(T)), n = static_cast<size_t>(n_seqs);
    char* p = static_cast<char*>(base);
    size_t off = 0;
    auto take = [&](size_t bytes) { char* q = p ? p + off : nullptr; off += up16(bytes); return q; };
    float* weight = reinterpret_cast<float*>(take(4 * (n + 1)));
    float2* seq_sum = reinterpret_cast<float2*>(take(8 * n));
    float2* first = reinterpret_cast<float2*>(take(8 * tiles));
    float2* last = reinterpret_cast<float2*>(take(8 * tiles));
    float* tile_stats = reinterpret_cast<float*>(take(20 * tiles));
    if (a) { a->weight = weight; a->seq_sum = seq_sum; a->first = first; a->last = last; a->tile_stats = tile_stats; }
    return off + 16;
}

bool bad_align(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// Checks what both losses and both directions share and fills the launch arguments.
int common(SeqArgs* a, const float* logp, const float* ref_logp, const uint8_t* mask, const int64_t* offsets, int64_t T,
           int64_t n_seqs, float* dlogp, const float* upstream, void* ws, size_t ws_bytes) {
    if (T < 0 || T > MAX_T || n_seqs < 0 || n_seqs > MAX_SEQS) return VPCE_INVALID_ARG;
    if (!ws || (n_seqs > 0 && !offsets)) return VPCE_INVALID_ARG;
    if (bad_align(ws, 16) || bad_align(logp, 4) || bad_align(ref_logp, 4) || bad_align(offsets, 8) || bad_align(dlogp, 4) ||
        bad_align(upstream, 4))
        return VPCE_UNSUPPORTED;
    if (ws_bytes < workspace_for(T, n_seqs, a, ws)) return VPCE_WORKSPACE_TOO_SMALL;
    a->logp = logp; a->ref_logp = ref_logp; a->mask = mask; a->offsets = offsets;
    a->T = static_cast<long>(T); a->n_seqs = static_cast<long>(n_seqs);
    a->steps = static_cast<int>(steps_for(T)); a->n_tiles = static_cast<long>(tiles_for(T));
    a->dlogp = dlogp; a->upstream = upstream;
    return VPCE_OK;
}

unsigned blocks_for(const SeqArgs& a) { return static_cast<unsigned>((a.n_tiles + WARPS - 1) / WARPS); }

template <bool POLICY> void launch_sums(const SeqArgs& a, cudaStream_t st) {
    if (a.n_tiles > 0) seq_sums_kernel<POLICY><<<blocks_for(a), THREADS, 0, st>>>(a);
}
template <bool POLICY> void launch_grad(const SeqArgs& a, cudaStream_t st) {
    if (a.n_tiles > 0 && a.dlogp) seq_grad_kernel<POLICY><<<blocks_for(a), THREADS, 0, st>>>(a);
}
int done() { return cudaGetLastError() == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR; }

int policy_args(SeqArgs* a, const float* logp, const float* old_logp, const float* ref_logp, const float* adv, int adv_per_token,
                const uint8_t* mask, const int64_t* offsets, int64_t T, int64_t n_seqs, double clip_low, double clip_high,
                double kl_coef, int aggregate, float* dlogp, const float* upstream, void* ws, size_t ws_bytes) {
    if (!(clip_low >= 0.0) || !(clip_high >= 0.0) || !(kl_coef == kl_coef)) return VPCE_INVALID_ARG;
    if (aggregate != VPCE_TOKEN_MEAN && aggregate != VPCE_SEQ_MEAN) return VPCE_INVALID_ARG;
    if (T > 0 && (!logp || !old_logp)) return VPCE_INVALID_ARG;
    if ((adv_per_token ? T : n_seqs) > 0 && !adv) return VPCE_INVALID_ARG;
    if (bad_align(old_logp, 4) || bad_align(adv, 4)) return VPCE_UNSUPPORTED;
    if (const int rc = common(a, logp, ref_logp, mask, offsets, T, n_seqs, dlogp, upstream, ws, ws_bytes)) return rc;
    a->old_logp = old_logp; a->adv = adv; a->adv_per_token = adv_per_token != 0;
    a->by_seq = aggregate == VPCE_SEQ_MEAN;
    a->lo = static_cast<float>(1.0 - clip_low); a->hi = static_cast<float>(1.0 + clip_high);
    a->kl_coef = static_cast<float>(kl_coef);
    return VPCE_OK;
}

}  // namespace

extern "C" {

size_t vp_policy_loss_workspace_bytes(int64_t T, int64_t n_seqs) {
    if (T < 0 || T > MAX_T || n_seqs < 0 || n_seqs > MAX_SEQS) return 0;
    return workspace_for(T, n_seqs, nullptr, nullptr);
}

int vp_policy_loss(const float* logp, const float* old_logp, const float* ref_logp, const float* advantages, int adv_per_token,
                   const uint8_t* mask, const int64_t* seq_offsets, int64_t T, int64_t n_seqs, double clip_low, double clip_high,
                   double kl_coef, int aggregate, float* stats, float* dlogp, const float* upstream, void* workspace,
                   size_t workspace_bytes, void* stream) {
    if (!stats) return VPCE_INVALID_ARG;
    if (bad_align(stats, 4)) return VPCE_UNSUPPORTED;
    SeqArgs a{};
    if (const int rc = policy_args(&a, logp, old_logp, ref_logp, advantages, adv_per_token, mask, seq_offsets, T, n_seqs, clip_low,
                                   clip_high, kl_coef, aggregate, dlogp, upstream, workspace, workspace_bytes))
        return rc;
    a.stats = stats;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    launch_sums<true>(a, st);
    policy_finish_kernel<<<1, FIN_THREADS, 0, st>>>(a);
    launch_grad<true>(a, st);
    return done();
}

int vp_policy_loss_backward(const float* logp, const float* old_logp, const float* ref_logp, const float* advantages,
                            int adv_per_token, const uint8_t* mask, const int64_t* seq_offsets, int64_t T, int64_t n_seqs,
                            double clip_low, double clip_high, double kl_coef, int aggregate, float* dlogp, const float* upstream,
                            const void* workspace, size_t workspace_bytes, void* stream) {
    if (T > 0 && !dlogp) return VPCE_INVALID_ARG;
    SeqArgs a{};
    if (const int rc = policy_args(&a, logp, old_logp, ref_logp, advantages, adv_per_token, mask, seq_offsets, T, n_seqs, clip_low,
                                   clip_high, kl_coef, aggregate, dlogp, upstream, const_cast<void*>(workspace), workspace_bytes))
        return rc;
    launch_grad<true>(a, static_cast<cudaStream_t>(stream));
    return done();
}

size_t vp_preference_loss_workspace_bytes(int64_t T, int64_t n_pairs) {
    if (n_pairs < 0 || n_pairs > MAX_SEQS / 2) return 0;
    return vp_policy_loss_workspace_bytes(T, 2 * n_pairs);
}

int vp_preference_loss(const float* logp, const float* ref_logp, const uint8_t* mask, const int64_t* seq_offsets, int64_t T,
                       int64_t n_pairs, double beta, double margin, double label_smoothing, int kind, int average, float* stats,
                       float* rewards, float* dlogp, const float* upstream, void* workspace, size_t workspace_bytes, void* stream) {
    if (!stats || (T > 0 && !logp) || n_pairs < 0 || n_pairs > MAX_SEQS / 2) return VPCE_INVALID_ARG;
    if (!(beta > 0.0) || !(margin == margin) || !(label_smoothing >= 0.0 && label_smoothing <= 1.0)) return VPCE_INVALID_ARG;
    if (kind != VPCE_PREF_SIGMOID && kind != VPCE_PREF_IPO) return VPCE_INVALID_ARG;
    if (bad_align(stats, 4) || bad_align(rewards, 4)) return VPCE_UNSUPPORTED;
    SeqArgs a{};
    if (const int rc = common(&a, logp, ref_logp, mask, seq_offsets, T, 2 * n_pairs, dlogp, upstream, workspace, workspace_bytes))
        return rc;
    a.by_seq = 1;
    a.beta = beta; a.margin = margin; a.smoothing = label_smoothing; a.kind = kind; a.average = average != 0;
    a.stats = stats; a.rewards = rewards;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    launch_sums<false>(a, st);
    preference_finish_kernel<<<1, FIN_THREADS, 0, st>>>(a);
    launch_grad<false>(a, st);
    return done();
}

int vp_preference_loss_backward(const uint8_t* mask, const int64_t* seq_offsets, int64_t T, int64_t n_pairs, float* dlogp,
                                const float* upstream, const void* workspace, size_t workspace_bytes, void* stream) {
    if ((T > 0 && !dlogp) || n_pairs < 0 || n_pairs > MAX_SEQS / 2) return VPCE_INVALID_ARG;
    SeqArgs a{};
    if (const int rc = common(&a, nullptr, nullptr, mask, seq_offsets, T, 2 * n_pairs, dlogp, upstream, const_cast<void*>(workspace),
                              workspace_bytes))
        return rc;
    a.by_seq = 1;
    launch_grad<false>(a, static_cast<cudaStream_t>(stream));
    return done();
}

}  // extern "C"
