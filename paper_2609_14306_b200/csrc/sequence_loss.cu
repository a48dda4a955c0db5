// Clipped policy loss and preference loss over packed sequences (sequence_loss.h).
//
// Sums over ragged sequences are split over tokens, not over sequences, so one sequence of a million tokens and a thousand
// of a thousand cost the same: a warp owns a tile of consecutive tokens and sums, for every sequence that meets its tile,
// the tokens inside it.  A sequence that lies inside one tile is finished there; of one that spans tiles each tile leaves
// its piece (`first`: the piece of the sequence that reaches into the tile from before, `last`: of the one that leaves it at
// the end).  One block then joins the pieces in the order of the tiles, forms the loss and a weight per sequence; a third
// pass over the tokens writes the gradient.
//
// These are latencies, not bandwidth (22 MB at 2^20 tokens: 3.4 us).  Up to SMALL_T tokens in SMALL_SEQS sequences one block
// does it all in one launch: its warps keep their tokens in registers and everything between the passes in shared memory.  A call
// of the policy loss against one of three launches: 9.4 and 18.6 us at 1021 tokens, 9.7 and 17.2 at 4096, 12.4 and 13.1 at 8192,
// 14.4 and 32.8 there in 1024 sequences.  (Replayed from a graph, without the launches' cost: 7.3 and 7.3, 8.1 and 6.3, 11.1 and
// 6.3, 13.4 and 30.0.)
// Beyond, each pass is a launch that starts while the one before drains (programmatic launch) and first reads what does not
// depend on it.

#include <cuda_runtime.h>

#include <algorithm>
#include <cstdint>

#include "sequence_loss.h"
#include "vp_ce.h"

namespace {

constexpr int THREADS = 128;                    // four warps, each with a tile of its own
constexpr int WARPS = THREADS / 32;
constexpr int64_t SMALL_T = 8192, SMALL_SEQS = 1024;   // of the one-block kernel: 32 warps with 256 tokens each
constexpr int PER_LANE = 4;                     // tokens of one lane in a step: a step covers 128 tokens
constexpr int STEP = 32 * PER_LANE;
constexpr int SMALL_PER_LANE = 8, SMALL_TILE = 32 * SMALL_PER_LANE;   // of the one-block kernel
constexpr int64_t MAX_TILES = 4096;             // the tile grows with T beyond 2^19 tokens: bounds what one block joins
constexpr int FIN_THREADS = 1024;
constexpr unsigned ALL = 0xffffffffu;

// What the kernels of one call share.  Everything below `seq_sum` lies in the workspace.
struct SeqArgs {
    const float *logp, *old_logp, *ref_logp, *adv;
    const uint8_t* mask;
    const int64_t* offsets;
    long T, n_seqs;
    long span;                                  // tokens per tile
    long n_tiles;
    int adv_per_token, by_seq;                  // by_seq: the loss needs sums per sequence
    float lo, hi, kl_coef;
    float2 *first, *last;                       // [n_tiles] pieces: (sum, count)
    float2* seq_sum;                            // [n_seqs] (sum, count); from preference_finish on a double
    float* tile_stats;                          // [5][n_stats] count, sum of l, KL, clipped, r of a block's (or warp's) tiles
    long n_stats;
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

// The first sequence that ends behind token t (n_seqs if none does): 256 probes a round, so one round of loads for up to 256
// sequences and two for 65536.
__device__ __forceinline__ long first_seq(const SeqArgs& a, long t, int lane) {
    constexpr int PROBES = 8;
    long lo = 0, hi = a.n_seqs;                 // the answer is in [lo, hi]
    while (hi > lo) {
        const long step = (hi - lo + 32 * PROBES - 1) / (32 * PROBES);
        // this lane's probes: the ends of its PROBES pieces of `step` sequences; how many of them does t lie behind?
        long begin[PROBES];
#pragma unroll
        for (int k = 0; k < PROBES; ++k) {
            const long probe = lo + step * (lane * PROBES + k + 1) - 1;
            begin[k] = probe < hi ? seq_begin(a, probe + 1) : a.T + 1;
        }
        int behind = 0;
#pragma unroll
        for (int k = 0; k < PROBES; ++k) behind += begin[k] <= t ? 1 : 0;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) behind += __shfl_xor_sync(ALL, behind, o);
        const long nlo = lo + step * behind, nhi = nlo + step - 1;
        lo = nlo < hi ? nlo : hi;
        hi = nhi < hi ? nhi : hi;
        if (step == 1) hi = lo;                 // every sequence was probed
    }
    return lo;
}

// e^q - q - 1 and e^q - 1.  As differences from e^q they lose the digits that e^q shares with 1 + q: all of them at the |q| of a
// policy that has just left its reference.  Below 1/2 the series of the first (to q^9 / 9!, which leaves out less than u / 25 of it)
// stands instead, of the right sign by its form, and the second follows from it; from there on the differences are good to 20 u and 4 u.
// Here and in policy_token the products that are fused with a sum are named, so that every kernel rounds alike: the gradient call
// repeats the joint call's bits.
__device__ __forceinline__ void kl_terms(float q, float& kl, float& x) {
    if (fabsf(q) < 0.5f) {
        float h = 1.f / 362880;
        h = fmaf(q, h, 1.f / 40320);
        h = fmaf(q, h, 1.f / 5040);
        h = fmaf(q, h, 1.f / 720);
        h = fmaf(q, h, 1.f / 120);
        h = fmaf(q, h, 1.f / 24);
        h = fmaf(q, h, 1.f / 6);
        h = fmaf(q, h, 0.5f);
        kl = __fmul_rn(__fmul_rn(q, q), h);
        x = __fadd_rn(q, kl);
    } else {
        x = __fsub_rn(expf(q), 1.f);
        kl = x - q;
    }
}

// Terms of one token of the policy loss.  `clipped` compares in fp32, so a ratio exactly on a bound counts as unclipped.
struct Policy { float l, grad, kl, clipped, r; };
__device__ __forceinline__ Policy policy_token(const SeqArgs& a, float logp, float old_logp, float ref, float adv) {
    Policy p;
    p.r = expf(logp - old_logp);
    const bool clip = (adv > 0.f && p.r > a.hi) || (adv < 0.f && p.r < a.lo);
    p.clipped = clip ? 1.f : 0.f;
    p.l = -((clip ? (adv > 0.f ? a.hi : a.lo) : p.r) * adv);
    p.grad = clip ? 0.f : __fmul_rn(-adv, p.r);
    p.kl = 0.f;
    if (a.ref_logp) {
        float x;
        kl_terms(ref - logp, p.kl, x);
        p.l += a.kl_coef * p.kl;
        p.grad = fmaf(-a.kl_coef, x, p.grad);
    }
    return p;
}

// Waits for the kernel before this one in the stream (a no-op where the launch did not ask for an early start).
__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
// Lets the kernel behind this one start.
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// N tokens of a lane, read whether their mask says so or not (one memory latency instead of two; what lies under the mask
// is not used): those at base + i + 32 j + lane that lie before base + e.  i, e: offsets inside a tile, in 32 bits.
template <bool POLICY, bool VALUES, int N> struct Tokens {
    bool on[N];
    float logp[N], old_logp[N], ref[N], adv[N];
    __device__ __forceinline__ void load(const SeqArgs& a, long base, int i, int e, int lane, float adv_s) {
        const int at = i + lane;
        const uint8_t* mask = a.mask ? a.mask + base + at : nullptr;
        const float *lp = a.logp + base + at, *op = a.old_logp + base + at, *rp = a.ref_logp + base + at, *ap = a.adv + base + at;
        const bool has_ref = VALUES && a.ref_logp, has_adv = VALUES && POLICY && a.adv_per_token;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool in = at + j * 32 < e;
            on[j] = in;
            if (mask && in) on[j] = mask[j * 32] != 0;
            logp[j] = VALUES && in ? lp[j * 32] : 0.f;
            old_logp[j] = VALUES && POLICY && in ? op[j * 32] : 0.f;
            ref[j] = has_ref && in ? rp[j * 32] : 0.f;
            adv[j] = has_adv && in ? ap[j * 32] : adv_s;
        }
    }
};

// Calls f(s, begin, end) for every sequence s that meets the tokens [t0, t1), with its range cut to them.
template <typename F>
__device__ __forceinline__ void for_sequences(const SeqArgs& a, long t0, long t1, int lane, F f) {
    for (long s = first_seq(a, t0, lane); s < a.n_seqs; ++s) {
        const long b = seq_begin(a, s), e = seq_begin(a, s + 1);
        if (b >= t1) break;
        if (e > b && e > t0) f(s, b, e);
    }
}

// Pass 1: sums of one tile, by one warp.  POLICY: value = l and the four statistics; else value = logp - ref_logp.
template <bool POLICY>
__device__ __forceinline__ void sum_tile(const SeqArgs& a, long tile, int lane, float (&stats)[5]) {
    const long t0 = tile * a.span, t1 = t0 + a.span < a.T ? t0 + a.span : a.T;
    float2 first = make_float2(0.f, 0.f), last = first;
    float cnt = 0.f, sl = 0.f, skl = 0.f, sclip = 0.f, sr = 0.f;
    for_sequences(a, t0, t1, lane, [&](long s, long sb, long se) {
        const long b = sb > t0 ? sb : t0, e = se < t1 ? se : t1;
        const float adv_s = POLICY && !a.adv_per_token ? a.adv[s] : 0.f;
        float sum = 0.f, n = 0.f;
        const int end = static_cast<int>(e - t0);
        for (int c = static_cast<int>(b - t0); c < end; c += STEP) {
            Tokens<POLICY, true, PER_LANE> k;
            k.load(a, t0, c, end, lane, adv_s);
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                if (!k.on[j]) continue;
                n += 1.f;
                if (POLICY) {
                    const Policy p = policy_token(a, k.logp[j], k.old_logp[j], k.ref[j], k.adv[j]);
                    sum += p.l;
                    skl += p.kl; sclip += p.clipped; sr += p.r;
                } else {
                    sum += k.logp[j] - k.ref[j];
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
    if (POLICY) { stats[0] = wsum(cnt); stats[1] = wsum(sl); stats[2] = wsum(skl); stats[3] = wsum(sclip); stats[4] = wsum(sr); }
}

__device__ __forceinline__ double wsum(double v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(ALL, v, o);
    return v;
}
// Sums of K doubles over the block (fixed order); every thread receives them.
template <int K>
__device__ __forceinline__ void block_sum(double (&v)[K], double (*part)[K]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, warps = blockDim.x >> 5;
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wsum(v[k]);
    if (lane == 0)
        for (int k = 0; k < K; ++k) part[warp][k] = v[k];
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = wsum(lane < warps ? part[lane][k] : 0.0);
}

// (sum, count) of sequence s by the lanes of a group of `width` lanes (a power of two up to 32), pieces in a fixed order.
__device__ __forceinline__ double2 join_pieces(const SeqArgs& a, long s, int sub, int width) {
    double2 v = make_double2(0.0, 0.0);
    if (s < a.n_seqs) {
        const long b = seq_begin(a, s), e = seq_begin(a, s + 1);
        if (e > b) {
            const long ta = b / a.span, tb = (e - 1) / a.span;
            if (ta == tb) {
                // inside one tile: finished there
                if (sub == 0) { const float2 f = a.seq_sum[s]; v.x = f.x; v.y = f.y; }
            } else {
                if (sub == 0) { const float2 f = a.last[ta]; v.x = f.x; v.y = f.y; }
#pragma unroll 4
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
    while (w > 1 && static_cast<long>(blockDim.x / w) < n_seqs) w >>= 1;
    return w;
}

// Pass 2, by one block of FIN_THREADS.
__device__ __forceinline__ void policy_finish(const SeqArgs& a) {
    __shared__ double total[5];
    __shared__ double part[32][2];
    // one warp (or, in a block of fewer than five, a few turns) for each of the five sums
    for (int k = threadIdx.x >> 5; k < 5; k += blockDim.x >> 5) {
        double t = 0.0;
#pragma unroll 8
        for (long i = threadIdx.x & 31; i < a.n_stats; i += 32) t += a.tile_stats[k * a.n_stats + i];
        t = wsum(t);
        if ((threadIdx.x & 31) == 0) total[k] = t;
    }
    double loss = 0.0;
    if (a.by_seq) {
        const int width = join_width(a.n_seqs), per_round = blockDim.x / width;
        double u[2] = {0, 0};                                               // sum of the sequences' means, sequences that have one
        for (long s0 = 0; s0 < a.n_seqs; s0 += per_round) {
            const long s = s0 + threadIdx.x / width;
            const double2 w = join_pieces(a, s, threadIdx.x % width, width);
            if (threadIdx.x % width == 0 && s < a.n_seqs) {
                a.weight[s] = w.y > 0 ? static_cast<float>(w.y) : 0.f;      // the count, until the number of sequences is known
                if (w.y > 0) { u[0] += w.x / w.y; u[1] += 1.0; }
            }
        }
        block_sum<2>(u, part);
        loss = u[1] > 0 ? u[0] / u[1] : 0.0;
        for (long s0 = 0; s0 < a.n_seqs; s0 += per_round) {                 // each thread meets the entries that it wrote
            const long s = s0 + threadIdx.x / width;
            if (threadIdx.x % width == 0 && s < a.n_seqs) {
                const double n = a.weight[s];
                a.weight[s] = n > 0 ? static_cast<float>(1.0 / (n * u[1])) : 0.f;
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        const double inv = total[0] > 0 ? 1.0 / total[0] : 0.0;
        if (!a.by_seq) loss = total[1] * inv;
        a.weight[a.n_seqs] = static_cast<float>(inv);
        a.stats[0] = static_cast<float>(loss);
        a.stats[1] = static_cast<float>(total[2] * inv);
        a.stats[2] = static_cast<float>(total[3] * inv);
        a.stats[3] = static_cast<float>(total[4] * inv);
    }
}

// A sequence's joined sum in the place of its (sum, count): D is a small difference of sums that may be large, so it is formed from
// what the join has, in double.
__device__ __forceinline__ float2 as_float2(double v) { return make_float2(__int_as_float(__double2loint(v)), __int_as_float(__double2hiint(v))); }
__device__ __forceinline__ double as_double(float2 v) { return __hiloint2double(__float_as_int(v.y), __float_as_int(v.x)); }

__device__ __forceinline__ void preference_finish(const SeqArgs& a) {
    __shared__ double part[32][3];
    const long pairs = a.n_seqs / 2;
    const int width = join_width(a.n_seqs), per_round = blockDim.x / width;
    for (long s0 = 0; s0 < a.n_seqs; s0 += per_round) {
        const long s = s0 + threadIdx.x / width;
        const double2 w = join_pieces(a, s, threadIdx.x % width, width);
        if (threadIdx.x % width == 0 && s < a.n_seqs) {
            const double n = a.average ? (w.y > 0 ? w.y : 1.0) : 1.0;
            a.seq_sum[s] = as_float2(w.x / n);
            a.weight[s] = static_cast<float>(n);                            // the divisor, until the slope is known
            if (a.rewards) a.rewards[s] = static_cast<float>(a.beta * (w.x / n));
        }
    }
    __syncthreads();
    double v[3] = {0, 0, 0};
    for (long i = threadIdx.x; i < pairs; i += blockDim.x) {
        const double diff = as_double(a.seq_sum[i]) - as_double(a.seq_sum[pairs + i]);
        double l, slope;
        if (a.kind == VPCE_PREF_SIGMOID) {
            // z carries D's digits; the curve itself is smooth enough for fp32 (a few u of the loss and of beta)
            const float z = static_cast<float>(a.beta * diff - a.margin), eps = static_cast<float>(a.smoothing);
            const float tail = log1pf(expf(-fabsf(z)));                     // log(1 + e^-|z|)
            const float neg = (z < 0.f ? -z : 0.f) + tail;                  // -log sigmoid(z)
            const float pos = (z > 0.f ? z : 0.f) + tail;                   // -log sigmoid(-z)
            l = (1.f - eps) * neg + eps * pos;
            slope = a.beta * (eps - 1.f / (1.f + expf(z)));
        } else {
            const double g = diff - 1.0 / (2.0 * a.beta);
            l = g * g;
            slope = 2.0 * g;
        }
        v[0] += l;
        v[1] += diff > 0.0 ? 1.0 : 0.0;
        v[2] += a.beta * diff;
        slope /= static_cast<double>(pairs);
        a.weight[i] = static_cast<float>(slope / a.weight[i]);
        a.weight[pairs + i] = static_cast<float>(-slope / a.weight[pairs + i]);
    }
    block_sum<3>(v, part);
    if (threadIdx.x == 0)
        for (int k = 0; k < 3; ++k) a.stats[k] = pairs > 0 ? static_cast<float>(v[k] / static_cast<double>(pairs)) : 0.f;
}

// Pass 3: the gradient of one tile's tokens, by one warp.
template <bool POLICY>
__device__ __forceinline__ void grad_tile(const SeqArgs& a, long tile, int lane) {
    const long t0 = tile * a.span, t1 = t0 + a.span < a.T ? t0 + a.span : a.T;
    long done = t0;                                                         // everything before is written
    auto zeros = [&](long to) { for (long t = done + lane; t < to; t += 32) a.dlogp[t] = 0.f; };
    for_sequences(a, t0, t1, lane, [&](long s, long sb, long se) {
        const long b = sb > t0 ? sb : t0, e = se < t1 ? se : t1;
        if (b < done) return;                                               // offsets that do not rise: every token is written once
        zeros(b);
        const float adv_s = POLICY && !a.adv_per_token ? a.adv[s] : 0.f;
        const int end = static_cast<int>(e - t0);
        float* out = a.dlogp + t0 + lane;
        for (int c = static_cast<int>(b - t0); c < end; c += STEP) {
            Tokens<POLICY, POLICY, PER_LANE> k;
            k.load(a, t0, c, end, lane, adv_s);
            wait_for_previous();                                            // the weights come from pass 2
            const float w = a.weight[POLICY && !a.by_seq ? a.n_seqs : s] * (a.upstream ? *a.upstream : 1.f);
#pragma unroll
            for (int j = 0; j < PER_LANE; ++j) {
                if (c + j * 32 + lane < end)
                    out[c + j * 32] = !k.on[j] ? 0.f : POLICY ? w * policy_token(a, k.logp[j], k.old_logp[j], k.ref[j], k.adv[j]).grad : w;
            }
        }
        done = e;
    });
    zeros(t1);
}

// Eight blocks an SM: all tiles run at once.
template <bool POLICY> __global__ void __launch_bounds__(THREADS, 8) seq_sums_kernel(const SeqArgs a) {
    __shared__ float part[WARPS][5];
    let_next_start();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long tile = static_cast<long>(blockIdx.x) * WARPS + warp;
    float stats[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
    if (tile < a.n_tiles) sum_tile<POLICY>(a, tile, lane, stats);
    if (!POLICY) return;
    if (lane == 0)
        for (int k = 0; k < 5; ++k) part[warp][k] = stats[k];
    __syncthreads();
    if (threadIdx.x < 5) {
        float v = 0.f;
        for (int w = 0; w < WARPS; ++w) v += part[w][threadIdx.x];
        a.tile_stats[threadIdx.x * a.n_stats + blockIdx.x] = v;
    }
}
template <bool POLICY> __global__ void __launch_bounds__(FIN_THREADS) seq_finish_kernel(const SeqArgs a) {
    let_next_start();
    wait_for_previous();
    if (POLICY) policy_finish(a); else preference_finish(a);
}
template <bool POLICY> __global__ void __launch_bounds__(THREADS, 8) seq_grad_kernel(const SeqArgs a) {
    const long tile = static_cast<long>(blockIdx.x) * WARPS + (threadIdx.x >> 5);
    if (tile < a.n_tiles) grad_tile<POLICY>(a, tile, threadIdx.x & 31);
    wait_for_previous();                                                    // what follows this kernel follows pass 2 as well
}
// All passes of a small call: a warp's 256 tokens stay in registers, the sequences and what joins the passes in shared memory.
template <bool POLICY> __global__ void __launch_bounds__(FIN_THREADS) seq_small_kernel(const SeqArgs a) {
    __shared__ int64_t offsets[SMALL_SEQS + 1];
    __shared__ float2 seq_sum[SMALL_SEQS], first[32], last[32];
    __shared__ float weight[SMALL_SEQS + 1], adv[SMALL_SEQS], tile_stats[5 * 32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = static_cast<int>(a.n_seqs);
    const int t0 = warp * SMALL_TILE, t1 = min(t0 + SMALL_TILE, static_cast<int>(a.T));
    Tokens<POLICY, true, SMALL_PER_LANE> k;
    k.load(a, 0, t0, t1, lane, 0.f);                                        // nothing where t0 >= T
    const float up = a.upstream ? *a.upstream : 1.f;
    if (n > 0)                                                              // without sequences a.offsets may be null
        for (int i = threadIdx.x; i <= n; i += blockDim.x) offsets[i] = seq_begin(a, i);
    for (int i = threadIdx.x; i < n; i += blockDim.x) seq_sum[i] = make_float2(0.f, 0.f);   // of offsets that do not rise nobody may write it
    if (POLICY && !a.adv_per_token)
        for (int i = threadIdx.x; i < n; i += blockDim.x) adv[i] = a.adv[i];
    __syncthreads();
    // the sequence of each token: the last that begins at or before it, if it also ends behind it
    int seq[SMALL_PER_LANE];
#pragma unroll
    for (int j = 0; j < SMALL_PER_LANE; ++j) {
        const int t = t0 + j * 32 + lane;
        int lo = 0, hi = n;                                                 // first sequence that ends behind t
        while (lo < hi) { const int mid = (lo + hi) >> 1; if (offsets[mid + 1] > t) hi = mid; else lo = mid + 1; }
        seq[j] = lo < n && offsets[lo] <= t && t < t1 ? lo : -1;
        k.on[j] = k.on[j] && seq[j] >= 0;
    }
    float value[SMALL_PER_LANE], grad[SMALL_PER_LANE], st[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < SMALL_PER_LANE; ++j) {
        value[j] = grad[j] = 0.f;
        if (!k.on[j]) continue;
        if (POLICY) {
            const Policy p = policy_token(a, k.logp[j], k.old_logp[j], k.ref[j], a.adv_per_token ? k.adv[j] : adv[seq[j]]);
            value[j] = p.l; grad[j] = p.grad;
            st[0] += 1.f; st[1] += p.l; st[2] += p.kl; st[3] += p.clipped; st[4] += p.r;
        } else {
            value[j] = k.logp[j] - k.ref[j];
        }
    }
    SeqArgs b = a;                                                          // the same, with what lies in shared memory here
    b.offsets = offsets; b.seq_sum = seq_sum; b.first = first; b.last = last; b.weight = weight; b.tile_stats = tile_stats;
    b.span = SMALL_TILE; b.n_stats = blockDim.x >> 5;
    if (POLICY) {
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            st[i] = wsum(st[i]);
            if (lane == 0) tile_stats[i * b.n_stats + warp] = st[i];
        }
    }
    if (a.by_seq && t0 < t1) {
        float2 head = make_float2(0.f, 0.f), tail = head;
        int s = 1 << 30, s_end = -1;                                        // sequences of this tile
#pragma unroll
        for (int j = 0; j < SMALL_PER_LANE; ++j) { if (seq[j] >= 0) { s = min(s, seq[j]); s_end = max(s_end, seq[j]); } }
        s = __reduce_min_sync(ALL, s);
        s_end = __reduce_max_sync(ALL, s_end);
        for (; s <= s_end; ++s) {
            float sum = 0.f, cnt = 0.f;
#pragma unroll
            for (int j = 0; j < SMALL_PER_LANE; ++j) if (seq[j] == s && k.on[j]) { sum += value[j]; cnt += 1.f; }
            const float2 v = make_float2(wsum(sum), wsum(cnt));
            const bool begins = offsets[s] >= t0, ends = offsets[s + 1] <= t1;
            if (!begins) head = v;
            else if (!ends) tail = v;
            else if (lane == 0) seq_sum[s] = v;
        }
        if (lane == 0) { first[warp] = head; last[warp] = tail; }
    }
    __syncthreads();
    if (POLICY) policy_finish(b); else preference_finish(b);
    __syncthreads();
    for (int i = threadIdx.x; i <= n; i += blockDim.x) a.weight[i] = weight[i];    // for a later gradient call
    if (!a.dlogp) return;
#pragma unroll
    for (int j = 0; j < SMALL_PER_LANE; ++j) {
        const int t = t0 + j * 32 + lane;
        if (t < t1) a.dlogp[t] = !k.on[j] ? 0.f : (POLICY ? grad[j] : 1.f) * (weight[POLICY && !a.by_seq ? n : seq[j]] * up);
    }
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
    a->span = static_cast<long>(steps_for(T) * STEP); a->n_tiles = static_cast<long>(tiles_for(T));
    a->n_stats = (a->n_tiles + WARPS - 1) / WARPS;
    a->dlogp = dlogp; a->upstream = upstream;
    return VPCE_OK;
}

unsigned blocks_for(const SeqArgs& a) { return static_cast<unsigned>((a.n_tiles + WARPS - 1) / WARPS); }

// `early`: may start before the kernel in front of it has ended (it waits for it where it needs its results).
template <typename K> cudaError_t launch(K kern, unsigned blocks, int threads, const SeqArgs& a, bool early, cudaStream_t st) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(threads); cfg.stream = st;
    cfg.attrs = &attr; cfg.numAttrs = early ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

// `backward`: the gradient alone (the call that filled the workspace is an ordinary predecessor in the stream).
template <bool POLICY> int launch_all(const SeqArgs& a, bool backward, cudaStream_t st) {
    cudaError_t e = cudaSuccess;
    const bool grad = a.dlogp && a.n_tiles > 0;
    if (!backward) {
        if (a.T <= SMALL_T && a.n_seqs <= SMALL_SEQS)
            // as many warps as there are tiles; the join of many sequences takes a few more
            return launch(seq_small_kernel<POLICY>, 1, static_cast<int>(32 * std::max<int64_t>((a.T + SMALL_TILE - 1) / SMALL_TILE, a.n_seqs > 64 ? 16 : 4)), a, false, st) == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
        if (a.n_tiles > 0) e = launch(seq_sums_kernel<POLICY>, blocks_for(a), THREADS, a, false, st);   // many sequences may share no token at all
        if (e == cudaSuccess) e = launch(seq_finish_kernel<POLICY>, 1, FIN_THREADS, a, a.n_tiles > 0, st);
    }
    if (e == cudaSuccess && grad) e = launch(seq_grad_kernel<POLICY>, blocks_for(a), THREADS, a, !backward, st);
    return e == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

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
    return launch_all<true>(a, false, static_cast<cudaStream_t>(stream));
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
    return launch_all<true>(a, true, static_cast<cudaStream_t>(stream));
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
    return launch_all<false>(a, false, static_cast<cudaStream_t>(stream));
}

int vp_preference_loss_backward(const uint8_t* mask, const int64_t* seq_offsets, int64_t T, int64_t n_pairs, float* dlogp,
                                const float* upstream, const void* workspace, size_t workspace_bytes, void* stream) {
    if ((T > 0 && !dlogp) || n_pairs < 0 || n_pairs > MAX_SEQS / 2) return VPCE_INVALID_ARG;
    SeqArgs a{};
    if (const int rc = common(&a, nullptr, nullptr, mask, seq_offsets, T, 2 * n_pairs, dlogp, upstream, const_cast<void*>(workspace),
                              workspace_bytes))
        return rc;
    a.by_seq = 1;
    return launch_all<false>(a, true, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
