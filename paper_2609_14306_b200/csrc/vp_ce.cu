// Fused vocabulary projection + cross-entropy for sm_100a (B200).
//
// A warp-specialised, persistent tcgen05 GEMM kernel is instantiated with four epilogues:
//   FOLD   strip Y = H_c W_q^T  -> per-tile partial (max, sum-exp) + target logit   (Eq. 2)
//   RESID  the same strip       -> G = dloss (exp(Y - lse) - onehot) as bf16       (App. C)
//   DH     dH_c += G W_q        (contract over the shard's vocabulary)  fp32 tiles leave by TMA store / TMA fp32
//   DW     dW_q += G^T H_c      (contract over the chunk's tokens)      reduction (the running sums stay in memory)
// Operands reach shared memory by TMA (128-byte swizzle), accumulators live in tensor
// memory (two buffers, so the epilogue of tile i overlaps the MMAs of tile i+1), and the
// logit strip never reaches global memory.
//
// Two variants of the kernel exist:
//   vpce_gemm_pair_kernel  two CTAs of a cluster share one 256 x 256 tile (tcgen05 cta_group::2);
//                          the default whenever a launch has at least two 128-row tiles;
//   vpce_gemm_kernel       one CTA per 128 x BN tile, tiles handed out by an atomic counter;
//                          used for narrow problems and by vp_ce_forward_static.
//
// Warp roles (192 threads): warp 0 = TMA producer, warp 1 = MMA issuer + TMEM owner,
// warps 2..5 = epilogue (one thread per accumulator row).
//
// After a chunk's last meeting the exact one-hot terms are added (vp_ce_fixup.cuh): what bf16 rounding took from each
// token's target entry of G goes back into dH and dW in fp32, in a fixed order.
//
// Every wait on an mbarrier is bounded: when it runs out the CTA records
// VPCE_DEV_WAIT_EXPIRED in the workspace status word, all roles leave their loops, pending
// copies and MMAs are drained (bounded again), TMEM is freed and the kernel returns.

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <functional>
#include <map>
#include <mutex>
#include <tuple>
#include <vector>

#include "token_logp.h"
#include "vp_ce.h"
#include "vp_ce_kernels.cuh"
#include "vp_ce_fixup.cuh"

namespace {

using namespace vpce;

// ------------------------------------------------------------------------------------ host side
std::atomic<long long> g_launches{0};

// Optional per-kernel timing: when enabled, every GEMM launch is bracketed by two events on the
// launching stream; vp_ce_profile_collect sums the elapsed times per kernel kind.
struct ProfEntry { int kind; cudaEvent_t a, b; };
std::mutex g_prof_mu;
bool g_prof_on = false;
std::vector<ProfEntry> g_prof;

// Limit of every wait inside the kernels (vp_ce_set_wait_limit_ns) and the one-shot test hook that makes the next
// launch of one kernel kind lose a copy (vp_ce_debug_drop_copy): kind in bits 0-7, k-block in bits 8-23, CTA ranks
// in bits 24-27; -1 = nothing armed.
std::atomic<unsigned long long> g_wait_limit_ns{kDefaultWaitLimitNs};
std::atomic<int> g_drop{-1};
// vp_ce_set_tail_parts: -1 the host decides, 0 never split, k > 1 the remainder tiles in k parts.
std::atomic<int> g_tail_parts{-1};

// Fills the launch-time fields every GEMM launch shares.
GemmParams finish_params(const GemmParams& p, int epi) {
    GemmParams q = p;
    q.wait_limit_ns = g_wait_limit_ns.load(std::memory_order_relaxed);
    q.drop_kb = -1;
    q.drop_ranks = 0;
    int armed = g_drop.load(std::memory_order_relaxed);
    if (armed >= 0 && (armed & 0xff) == epi && g_drop.compare_exchange_strong(armed, -1)) {
        q.drop_kb = (armed >> 8) & 0xffff;
        q.drop_ranks = (armed >> 24) & 0xf;
    }
    return q;
}

// Tile counters of the dynamic scheduler: one per launch, zeroed in bulk; a call that needs more
// launches than counters zeroes them again when it wraps (stream order makes that safe).
constexpr int NUM_TILE_COUNTERS = 1024;
struct CounterPool {
    int* base; int next; cudaStream_t st; bool failed;
    CounterPool(int* b, cudaStream_t s) : base(b), next(0), st(s), failed(false) {
        failed = cudaMemsetAsync(base, 0, 4 * NUM_TILE_COUNTERS, st) != cudaSuccess;
    }
    int* take() {
        if (next == NUM_TILE_COUNTERS) {
            failed = failed || cudaMemsetAsync(base, 0, 4 * NUM_TILE_COUNTERS, st) != cudaSuccess;
            next = 0;
        }
        return base + next++;
    }
    // k consecutive zeroed counters.  All that one launch needs is taken at once: a second call may zero the pool again and hand
    // the launch's first ones out to a later launch, which would find what this one has left in them.
    int* take_n(int k) {
        if (next + k > NUM_TILE_COUNTERS) {
            failed = failed || cudaMemsetAsync(base, 0, 4 * NUM_TILE_COUNTERS, st) != cudaSuccess;
            next = 0;
        }
        int* p = base + next;
        next += k;
        return p;
    }
};

struct WsLayout {
    size_t status, scalars, counters, sm, sz, ylab, pm, pz, G, acc, delta, keys, partials, total;
};
inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

bool ws_layout(int64_t T_chunk, int64_t d, int64_t block_v, WsLayout* L, int g_elem_bytes = 2) {
    if (T_chunk <= 0 || d <= 0 || block_v <= 0) return false;
    if (T_chunk % BM || block_v % BN_VOCAB || d % 8) return false;
    if (T_chunk > (1 << 24) || block_v > (1 << 24) || d > (1 << 20)) return false;
    const size_t nt = static_cast<size_t>(block_v / BN_VOCAB);
    size_t off = 0;
    L->status = off;  off += 256;
    L->scalars = off; off += 256;
    L->counters = off; off += 4 * NUM_TILE_COUNTERS;
    L->sm = off;      off = align_up(off + 4 * T_chunk, 1024);
    L->sz = off;      off = align_up(off + 4 * T_chunk, 1024);
    L->ylab = off;    off = align_up(off + 4 * T_chunk, 1024);
    L->pm = off;      off = align_up(off + 4 * T_chunk * nt, 1024);
    L->pz = off;      off = align_up(off + 4 * T_chunk * nt, 1024);
    L->G = off;       off = align_up(off + g_elem_bytes * static_cast<size_t>(T_chunk) * block_v, 1024);
    L->acc = off;     off = align_up(off + 4 * static_cast<size_t>(T_chunk) * d, 1024);
    // exact one-hot terms (bf16 path): per-token rounding residue, sorted (target, token) keys, split-run partial sums
    L->delta = off;   off = align_up(off + 4 * T_chunk, 1024);
    L->keys = off;    off = align_up(off + 8 * T_chunk, 1024);
    const size_t segs = (static_cast<size_t>(T_chunk < SORT_MAX ? T_chunk : SORT_MAX) + FIX_SEG - 1) / FIX_SEG;
    L->partials = off; off = align_up(off + 4 * segs * 2 * static_cast<size_t>(d), 1024);
    L->total = off;
    return true;
}

PFN_cuTensorMapEncodeTiled_v12000 get_encode() {
    static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* ptr = nullptr;
        cudaDriverEntryPointQueryResult qres;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &ptr, cudaEnableDefault, &qres) == cudaSuccess &&
            qres == cudaDriverEntryPointSuccess)
            fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(ptr);
    });
    return fn;
}

// 2-D tensor map over a row-major [rows, cols] matrix of bf16 (elem_bytes 2) or fp32 (4): dim0 = cols
// (contiguous), 128-byte swizzle.
bool make_map(CUtensorMap* map, const void* ptr, uint64_t rows, uint64_t cols, uint64_t ld_elems, uint32_t box_cols,
              uint32_t box_rows, int elem_bytes = 2) {
    auto enc = get_encode();
    if (!enc) return false;
    cuuint64_t dims[2] = {cols, rows};
    cuuint64_t strides[1] = {ld_elems * elem_bytes};
    cuuint32_t box[2] = {box_cols, box_rows};
    cuuint32_t estr[2] = {1, 1};
    const CUtensorMapDataType dt = elem_bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    CUresult r = enc(map, dt, 2, const_cast<void*>(ptr), dims, strides, box, estr,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

// MN-major operand of a row-major [k_rows, mn_cols] matrix (mn_cols % 64 == 0) as a 3-D tensor
// {64 contiguous elements, k_rows, mn_cols / 64}: one box {64, 64, chunks} per k-block lands in
// shared memory as `chunks` consecutive 64 x 128-byte blocks, the layout the MMA descriptor expects.
// (fp32: chunks of 32 elements and 32 k-rows per box.)
bool make_map_mn3d(CUtensorMap* map, const void* ptr, uint64_t k_rows, uint64_t mn_cols, uint64_t ld_elems, uint32_t chunks,
                   int elem_bytes = 2) {
    auto enc = get_encode();
    const uint64_t ce = 128 / elem_bytes;                 // elements per 128-byte chunk row = k-rows per stage
    if (!enc || mn_cols % ce) return false;
    cuuint64_t dims[3] = {ce, k_rows, mn_cols / ce};
    cuuint64_t strides[2] = {ld_elems * elem_bytes, 128};
    cuuint32_t box[3] = {static_cast<cuuint32_t>(ce), static_cast<cuuint32_t>(ce), chunks};
    cuuint32_t estr[3] = {1, 1, 1};
    const CUtensorMapDataType dt = elem_bytes == 4 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    // MN-major 32-bit operands are swizzled in 32-byte units (what the tensor core expects for them)
    const CUtensorMapSwizzle sw = elem_bytes == 4 ? CU_TENSOR_MAP_SWIZZLE_128B_ATOM_32B : CU_TENSOR_MAP_SWIZZLE_128B;
    CUresult r = enc(map, dt, 3, const_cast<void*>(ptr), dims, strides, box, estr,
                     CU_TENSOR_MAP_INTERLEAVE_NONE, sw, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                     CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS;
}

// Per-device host-side caches are atomics: concurrent callers may both do the (idempotent) set-up, none reads
// a half-written value.
int num_sms() {
    static std::atomic<int> cached[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 148;
    int n = cached[dev].load(std::memory_order_acquire);
    if (!n) {
        if (cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) n = 148;
        cached[dev].store(n, std::memory_order_release);
    }
    return n;
}

// Raises the dynamic shared-memory limit of `kern` once per device (the attribute is per device and function).
template <typename K>
cudaError_t ensure_smem_attr(K kern, int smem_bytes, std::atomic<bool>* done) {
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64)
        return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes);
    if (!done[dev].load(std::memory_order_acquire)) {
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes);
        if (e != cudaSuccess) return e;
        done[dev].store(true, std::memory_order_release);
    }
    return cudaSuccess;
}

template <int BN, bool A_MN, bool B_MN, int EPI>
cudaError_t launch_gemm(const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, const GemmParams& p,
                        cudaStream_t st) {
    constexpr int SMEM = smem_total<BN, EPI>();
    auto kern = vpce_gemm_kernel<BN, A_MN, B_MN, EPI>;
    static std::atomic<bool> attr_set[64];
    if (cudaError_t e = ensure_smem_attr(kern, SMEM, attr_set); e != cudaSuccess) return e;
    const int tiles = p.m_tiles * p.n_tiles;
    if (tiles <= 0 || p.num_kb <= 0) return cudaSuccess;
    const int grid = tiles < num_sms() ? tiles : num_sms();
    ProfEntry pe{kind_of(EPI), nullptr, nullptr};
    bool prof = false;
    {
        std::lock_guard<std::mutex> lk(g_prof_mu);
        prof = g_prof_on;
    }
    if (prof && cudaEventCreate(&pe.a) == cudaSuccess && cudaEventCreate(&pe.b) == cudaSuccess) cudaEventRecord(pe.a, st);
    else prof = false;
    kern<<<grid, NUM_THREADS, SMEM, st>>>(tmA, tmB, tmC, finish_params(p, kind_of(EPI)));
    if (prof) {
        cudaEventRecord(pe.b, st);
        std::lock_guard<std::mutex> lk(g_prof_mu);
        g_prof.push_back(pe);
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError();
}

template <int BN, bool A_MN, bool B_MN, int EPI, bool TF32 = false>
cudaError_t launch_pair(const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, const GemmParams& p,
                        cudaStream_t st) {
    constexpr int SMEM = pair_smem_total<BN, EPI>();
    auto kern = vpce_gemm_pair_kernel<BN, A_MN, B_MN, EPI, TF32>;
    static std::atomic<bool> attr_set[64];
    if (cudaError_t e = ensure_smem_attr(kern, SMEM, attr_set); e != cudaSuccess) return e;
    const int tiles = ((p.m_tiles + 1) / 2) * p.n_tiles;
    if (tiles <= 0 || p.num_kb <= 0) return cudaSuccess;
    const int max_pairs = num_sms() / 2;
    const int n_cut = (EPI == EPI_DH || EPI == EPI_DW) ? std::min(p.n_cut, tiles) : 0;
    const int entries = tiles + n_cut * (std::max(p.k_split, 1) - 1);          // split tiles count once per part
    const int grid = 2 * (entries < max_pairs ? entries : max_pairs);
    ProfEntry pe{kind_of(EPI), nullptr, nullptr};
    bool prof = false;
    {
        std::lock_guard<std::mutex> lk(g_prof_mu);
        prof = g_prof_on;
    }
    if (prof && cudaEventCreate(&pe.a) == cudaSuccess && cudaEventCreate(&pe.b) == cudaSuccess) cudaEventRecord(pe.a, st);
    else prof = false;
    kern<<<grid, NUM_THREADS, SMEM, st>>>(tmA, tmB, tmC, finish_params(p, kind_of(EPI)));
    if (prof) {
        cudaEventRecord(pe.b, st);
        std::lock_guard<std::mutex> lk(g_prof_mu);
        g_prof.push_back(pe);
    }
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError();
}

// The tail of a gradient GEMM's work list.  The pair kernel hands out 256 x 256 tiles greedily; when their number is
// not a multiple of the number of CTA pairs the last round runs with most pairs idle.  The last n_cut tiles of the list
// are therefore run as ks parts along K (the parts add into the output in a fixed order, see the kernel).  n_cut and ks
// come from simulating the greedy hand-out, in units of one k-block of a whole tile: a narrower last n-tile of a row is
// bound by its operand loads and costs about 7/8 of a whole tile down to an MMA width of half a tile; every part pays
// for filling the pipeline (TAIL_FILL) and its epilogue, which starts only after the epilogue of the part before it
// (TAIL_EPI; both constants fitted to measured launch times of the two benchmark geometries).  Part j + 1 is made
// TAIL_EPI k-blocks longer than part j so that parts that start together finish an epilogue apart.  Decisions are
// cached per geometry.
struct SplitChoice { int n_cut, ks, stagger; };
constexpr int MAX_SPLIT_TILES = 64;            // 8 flags each: half of the counter pool at most
constexpr double TAIL_FILL = 6.0, TAIL_EPI = 15.0;
constexpr int TAIL_MIN_PART = 8;               // k-blocks of the shortest part

double simulate_tail(int pm_tiles, int n_tiles, int group_n, double c_last, int n_cut, int ks, int stagger, int num_kb,
                     int pairs) {
    const int total = pm_tiles * n_tiles;
    std::vector<double> heap(pairs, 0.0);       // min-heap of the times at which the pairs become free
    auto take = [&]() {
        std::pop_heap(heap.begin(), heap.end(), std::greater<double>());
        return heap.back();
    };
    auto put = [&](double t) {
        heap.back() = t;
        std::push_heap(heap.begin(), heap.end(), std::greater<double>());
    };
    auto cost = [&](int t) {
        const int per_group = group_n * pm_tiles;
        const int g = t / per_group, r = t - g * per_group, n0 = g * group_n;
        const int gw = std::min(group_n, n_tiles - n0);
        const int nt = n0 + (r - (r / gw) * gw);
        return nt == n_tiles - 1 ? c_last : 1.0;
    };
    for (int t = 0; t < total - n_cut; ++t) put(take() + num_kb * cost(t));
    const int base_len = ks > 0 ? (num_kb - stagger * (ks * (ks - 1) / 2)) / ks : num_kb;
    for (int t = total - n_cut; t < total; ++t) {
        double prev_done = 0.0;
        int k0 = 0;
        for (int j = 0; j < ks; ++j) {
            const int k1 = j + 1 == ks ? num_kb : k0 + base_len + stagger * j;
            const double computed = take() + TAIL_FILL + (k1 - k0) * cost(t);
            prev_done = std::max(computed, prev_done) + TAIL_EPI;
            put(prev_done);
            k0 = k1;
        }
    }
    return *std::max_element(heap.begin(), heap.end());
}

SplitChoice pick_split(int pm_tiles, int n_tiles, int group_n, int last_width, int num_kb, int pairs) {
    if (pairs <= 0 || pm_tiles <= 0 || n_tiles <= 0) return {0, 1, 0};
    const int total = pm_tiles * n_tiles;
    const int stagger = static_cast<int>(TAIL_EPI);
    auto fits = [&](int ks) { return (num_kb - stagger * (ks * (ks - 1) / 2)) / ks >= TAIL_MIN_PART; };
    const int forced = g_tail_parts.load(std::memory_order_relaxed);          // vp_ce_set_tail_parts overrides the choice
    if (forced == 0) return {0, 1, 0};
    if (forced > 1) {                      // as asked, staggered when K is long enough for it, else in equal parts
        const int cut = std::min(std::min(total % pairs, total), MAX_SPLIT_TILES);
        if (cut <= 0 || num_kb < forced) return {0, 1, 0};
        return fits(forced) ? SplitChoice{cut, forced, stagger} : SplitChoice{cut, forced, 0};
    }
    struct Key {
        int a, b, c, d, e, f;
        bool operator<(const Key& o) const { return std::tie(a, b, c, d, e, f) < std::tie(o.a, o.b, o.c, o.d, o.e, o.f); }
    };
    static std::mutex mu;
    static std::map<Key, SplitChoice> cache;
    const Key key{pm_tiles, n_tiles, group_n, last_width, num_kb, pairs};
    {
        std::lock_guard<std::mutex> lk(mu);
        auto it = cache.find(key);
        if (it != cache.end()) return it->second;
    }
    const double c_last = last_width >= 256 ? 1.0 : std::max(0.875, last_width / 256.0);
    SplitChoice best{0, 1, 0};
    double best_t = simulate_tail(pm_tiles, n_tiles, group_n, c_last, 0, 1, 0, num_kb, pairs) * 0.98;   // a split must pay 2 %
    const int R = total % pairs;
    for (int cut : {R, R + pairs}) {
        cut = std::min(std::min(cut, total), MAX_SPLIT_TILES);
        if (cut <= 0) continue;
        // two or three parts only: measured inside the power-capped benchmark step, more parts made the launch
        // itself shorter but the step no faster (every part costs an epilogue and a pipeline fill of energy); a third
        // part has to pay for itself
        for (int ks : {2, 3}) {
            if (!fits(ks)) break;
            const double t = simulate_tail(pm_tiles, n_tiles, group_n, c_last, cut, ks, stagger, num_kb, pairs);
            if (t < best_t) { best_t = t * (ks == 2 ? 0.985 : 1.0); best = {cut, ks, stagger}; }
        }
    }
    std::lock_guard<std::mutex> lk(mu);
    cache[key] = best;
    return best;
}

// Which GEMMs run as CTA pairs (bit 0 strip kernels, bit 1 input-gradient, bit 2 weight-gradient).
// All of them by default; VPCE_PAIR in the environment overrides it for A/B measurements.
int pair_mask() {
    static const int mask = [] {
        const char* e = getenv("VPCE_PAIR");
        return e ? atoi(e) : 7;
    }();
    return mask;
}

// Output-column tile for the two gradient GEMMs: 256 unless d is narrower; the last tile of a
// row runs with its own (narrower) MMA width, so d need not be a multiple of the tile.
int pick_bn(int64_t d) {
    if (d <= 64) return 64;
    if (d <= 128) return 128;
    if (d <= 192) return 192;
    return 256;
}

template <bool A_MN, bool B_MN, int EPI>
cudaError_t launch_grad(int bn, const CUtensorMap& tmA, const CUtensorMap& tmB, const CUtensorMap& tmC, const GemmParams& p,
                        cudaStream_t st) {
    switch (bn) {
        case 256: return launch_gemm<256, A_MN, B_MN, EPI>(tmA, tmB, tmC, p, st);
        case 192: return launch_gemm<192, A_MN, B_MN, EPI>(tmA, tmB, tmC, p, st);
        case 128: return launch_gemm<128, A_MN, B_MN, EPI>(tmA, tmB, tmC, p, st);
        default:  return launch_gemm<64, A_MN, B_MN, EPI>(tmA, tmB, tmC, p, st);
    }
}

// n-tiles per raster group: the B operand slice a group touches should stay L2-resident
// (<= ~48 MB), and groups are balanced.
int pick_group_n(int n_tiles, double b_total_bytes) {
    const double budget = 48.0 * 1024 * 1024;
    int groups = static_cast<int>((b_total_bytes + budget - 1) / budget);
    if (groups < 1) groups = 1;
    if (groups > n_tiles) groups = n_tiles;
    return (n_tiles + groups - 1) / groups;
}

// L2 eviction hints: the shard-side operand B is reused by every m-tile (keep it), the residual
// strip G is streamed out by RESID and streamed in by the two gradient GEMMs (let it go first).
void apply_tuning(GemmParams& p, int epi) {
    p.hint_a = 0;
    p.hint_b = 2;
    p.hint_c = (epi == EPI_RESID) ? 1 : 0;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

vpce_status check_common(const void* H, const void* W, const int32_t* labels, int64_t T, int64_t d, int64_t V,
                         int64_t block_v, int64_t T_chunk, int64_t chunk_index_base, const void* ws, size_t ws_bytes,
                         WsLayout* L) {
    if (!H || !W || !labels || !ws) return VPCE_INVALID_ARG;
    if (T <= 0 || d <= 0 || V <= 0 || block_v <= 0 || T_chunk <= 0 || chunk_index_base < 0) return VPCE_INVALID_ARG;
    if (!aligned16(H) || !aligned16(W) || !aligned16(ws)) return VPCE_UNSUPPORTED;
    if (T >= (1ll << 31) || V >= (1ll << 31)) return VPCE_UNSUPPORTED;
    if (!ws_layout(T_chunk, d, block_v, L)) return VPCE_UNSUPPORTED;
    if (ws_bytes < L->total) return VPCE_WORKSPACE_TOO_SMALL;
    return VPCE_OK;
}

// ------------------------------------------------------------------------------------ one meeting
// A "meeting" is what Algorithm 3 does when one token batch X (rows) is co-located with one vocabulary shard
// W_q (cols rows of the weight): forward = form the strip X W_q^T and fold it into the batch's running state;
// backward = recompute the strip, form the residual and contract it into the two gradients.  vp_ce_forward /
// vp_ce_backward loop over (chunk, shard) meetings on one device; vp_ce_meeting_* expose a single meeting to a
// ring driver that moves the shard or the batch between devices.

// Tensor maps and workspace pointers of the forward meetings of one call.
struct FoldCtx {
    CUtensorMap tmX, tmW, tmW_half;
    int* status; float *sm, *sz, *ylab, *pm, *pz;
    int part_ld, num_kb, ignore_index, V;
    int64_t d;
    bool pair_strip;
};

bool make_fold_ctx(FoldCtx* c, const void* X, int64_t x_rows, const void* W, int64_t w_rows, int64_t d) {
    c->d = d;
    c->num_kb = static_cast<int>((d + BK - 1) / BK);
    c->pair_strip = (pair_mask() & 1) != 0;
    return make_map(&c->tmX, X, x_rows, d, d, BK, BM) && make_map(&c->tmW, W, w_rows, d, d, BK, BN_VOCAB) &&
           make_map(&c->tmW_half, W, w_rows, d, d, BK, BN_VOCAB / 2);
}

// Forward meeting: rows [x_row0, x_row0 + rows) of the X map meet rows [w_row0, w_row0 + cols) of the W map, which
// are vocabulary ids [v_lo, v_lo + cols).  labels / lse / loss point at the batch's first token.  first: the state
// starts from (-inf, 0, 0); last: lse and loss are emitted (Algorithm 3, output line).
cudaError_t fold_meeting(const FoldCtx& c, int x_row0, int rows, int w_row0, int cols, int v_lo, const int32_t* labels,
                         bool first, bool last, float* lse, float* loss, CounterPool& counters, cudaStream_t st) {
    GemmParams p{};
    p.m_tiles = (rows + BM - 1) / BM;
    p.n_tiles = (cols + BN_VOCAB - 1) / BN_VOCAB;
    p.num_kb = c.num_kb;
    p.group_n = pick_group_n(p.n_tiles, 2.0 * cols * c.d);
    p.a_mn0 = x_row0; p.a_k0 = 0;
    p.b_mn0 = w_row0; p.b_k0 = 0;
    p.rows_valid = rows; p.cols_valid = cols;
    p.v_lo = v_lo;
    p.labels = labels;
    p.ignore_index = c.ignore_index; p.V = c.V;
    p.pm = c.pm; p.pz = c.pz; p.ylab = c.ylab; p.part_ld = c.part_ld;
    p.status = c.status;
    apply_tuning(p, EPI_FOLD);
    p.tile_counter = counters.take();
    cudaError_t e;
    if (c.pair_strip && p.m_tiles >= 2) e = launch_pair<BN_VOCAB, false, false, EPI_FOLD>(c.tmX, c.tmW_half, c.tmX, p, st);
    else e = launch_gemm<BN_VOCAB, false, false, EPI_FOLD>(c.tmX, c.tmW, c.tmX, p, st);
    if (e != cudaSuccess) return e;
    vpce_merge_kernel<<<(rows + 255) / 256, 256, 0, st>>>(c.pm, c.pz, c.part_ld, p.n_tiles, c.sm, c.sz, c.ylab, rows, first,
                                                          last, labels, c.ignore_index, c.V, lse, loss, c.status);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError();
}

// Tail split of a gradient GEMM launched as CTA pairs (p.m_tiles, p.n_tiles, p.group_n, p.num_kb set; out_cols = N), and the
// launch's tile counter.
void set_split(GemmParams& p, int64_t out_cols, CounterPool& counters, int width_unit = 128) {
    const int left = static_cast<int>(out_cols - static_cast<int64_t>(p.n_tiles - 1) * 256);
    const int last_width = left >= 256 ? 256 : (left + width_unit - 1) / width_unit * width_unit;
    const SplitChoice c = pick_split((p.m_tiles + 1) / 2, p.n_tiles, p.group_n, last_width, p.num_kb, num_sms() / 2);
    p.n_cut = c.n_cut;
    p.k_split = c.ks;
    p.k_stagger = c.stagger;
    int* taken = counters.take_n(8 * c.n_cut + 1);
    p.tile_counter = taken + 8 * c.n_cut;
    p.split_flags = c.n_cut > 0 ? taken : nullptr;
}

// Tensor maps and workspace pointers of the backward meetings of one call.
struct GradCtx {
    CUtensorMap tmX_k, tmW_k, tmW_khalf, tmG_st, tmG_k, tmW_mn, tmG_mn, tmX_mn, tmW_mn2, tmX_mn2;
    int* status; float* inv_n; __nv_bfloat16* G;
    const __nv_bfloat16* X;                 // first row of the X map
    float* delta; unsigned long long* keys; float* partials;   // exact one-hot terms (see vp_ce_fixup.cuh)
    int g_rows, g_ld;                       // rows and row pitch (elements) of the residual strip in the workspace
    int bn, pmask, ignore_index, V;
    int64_t d;
    bool pair_ok, mn3d;
    // gradients of log probabilities and entropies instead of the loss's (vp_token_logp_backward)
    bool score = false;
    float inv_temp = 1.f;
    const float *entropy = nullptr, *dent = nullptr;          // of the batch's first token
};

bool make_grad_ctx(GradCtx* c, const void* X, int64_t x_rows, const void* W, int64_t w_rows, int64_t d,
                   __nv_bfloat16* G, int64_t g_rows, int64_t g_ld) {
    c->d = d; c->G = G; c->g_rows = static_cast<int>(g_rows); c->g_ld = static_cast<int>(g_ld);
    c->X = static_cast<const __nv_bfloat16*>(X);
    c->bn = pick_bn(d);
    c->pmask = pair_mask();
    c->pair_ok = (c->bn == 256) && (d % 64 == 0);
    c->mn3d = (d % 64 == 0);             // one-instruction fetch of MN-major operands when the contiguous extent allows
    if (!make_map(&c->tmG_st, G, g_rows, g_ld, g_ld, 64, 32) ||
        !make_map(&c->tmX_k, X, x_rows, d, d, BK, BM) || !make_map(&c->tmW_k, W, w_rows, d, d, BK, BN_VOCAB) ||
        !make_map(&c->tmW_khalf, W, w_rows, d, d, BK, BN_VOCAB / 2) ||
        !make_map(&c->tmG_k, G, g_rows, g_ld, g_ld, BK, BM) || !make_map(&c->tmW_mn, W, w_rows, d, d, 64, BK) ||
        !make_map(&c->tmG_mn, G, g_rows, g_ld, g_ld, 64, BK) || !make_map(&c->tmX_mn, X, x_rows, d, d, 64, BK))
        return false;
    // CTA-pair variants: half-width B boxes
    if (c->pair_ok && (!make_map_mn3d(&c->tmW_mn2, W, w_rows, d, d, 2) || !make_map_mn3d(&c->tmX_mn2, X, x_rows, d, d, 2)))
        return false;
    if (c->mn3d && (!make_map_mn3d(&c->tmW_mn, W, w_rows, d, d, c->bn / 64) ||
                    !make_map_mn3d(&c->tmX_mn, X, x_rows, d, d, c->bn / 64) ||
                    !make_map_mn3d(&c->tmG_mn, G, g_rows, g_ld, g_ld, BM / 64)))
        return false;
    return true;
}

enum { PHASE_RESIDUAL = VPCE_PHASE_RESIDUAL, PHASE_INPUT_GRAD = VPCE_PHASE_INPUT_GRAD,
       PHASE_WEIGHT_GRAD = VPCE_PHASE_WEIGHT_GRAD };

// Backward meeting, in up to three phases (a ring driver may wait for a travelling accumulator between them):
//   residual     recompute the strip, G = dloss (exp(Y - lse) - onehot) as bf16 into the workspace
//   input grad   acc (+)= G W_q   (fp32 [rows, d], pitch d; first: overwrite; last: write bf16 dX instead)
//   weight grad  dW_q (+)= G^T X  (fp32 [cols, d])
// labels / lse / dloss / acc / dX point at the batch's first token, dW_q at the shard's first row.
// The range of vocabulary ids whose exact one-hot terms a meeting adds after its GEMMs (nv == 0: none), with the rows
// of the weight and of the weight gradient that belong to id v0.
struct FixRange { int v0, nv; const __nv_bfloat16* W_v0; float* dW_v0; bool sort_now; };

cudaError_t sort_targets(const GradCtx& c, const int32_t* labels, int rows, cudaStream_t st) {
    const int subs = (rows + SORT_MAX - 1) / SORT_MAX;
    vpce_sort_targets_kernel<<<subs * (SORT_MAX / RANK_TOKENS), RANK_TOKENS * RANK_PARTS, 0, st>>>(labels, rows, c.ignore_index,
                                                                                                c.V, c.keys);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError();
}

cudaError_t grad_meeting(const GradCtx& c, int phases, int x_row0, int rows, int w_row0, int cols, int v_lo,
                         const int32_t* labels, const float* lse, const float* dloss, bool first, bool last, float* acc,
                         __nv_bfloat16* dX, float* dW_q, bool accumulate_dW, const FixRange& fix, CounterPool& counters,
                         cudaStream_t st) {
    const int strip_tiles_n = (cols + BN_VOCAB - 1) / BN_VOCAB;
    const int m_tiles = (rows + BM - 1) / BM;
    const int d = static_cast<int>(c.d);
    cudaError_t e = cudaSuccess;
    if ((phases & PHASE_RESIDUAL) && fix.sort_now && (e = sort_targets(c, labels, rows, st)) != cudaSuccess) return e;
    if (phases & PHASE_RESIDUAL) {
        GemmParams p{};
        p.m_tiles = m_tiles;
        p.n_tiles = strip_tiles_n;
        p.num_kb = (d + BK - 1) / BK;
        p.group_n = pick_group_n(p.n_tiles, 2.0 * cols * d);
        p.a_mn0 = x_row0; p.b_mn0 = w_row0;
        p.rows_valid = rows; p.cols_valid = cols;
        p.v_lo = v_lo;
        p.labels = labels; p.lse = lse; p.dloss = dloss;
        p.inv_n_valid = c.inv_n; p.ignore_index = c.ignore_index; p.V = c.V;
        p.G = c.G; p.g_ld = c.g_ld; p.g_rows = c.g_rows;
        p.delta = c.delta;
        p.status = c.status;
        apply_tuning(p, EPI_RESID);
        p.tile_counter = counters.take();
        const bool pairs = (c.pmask & 1) && p.m_tiles >= 2;
        if (c.score) {
            p.entropy = c.entropy; p.dent = c.dent; p.inv_temp = c.inv_temp;
            e = pairs ? launch_pair<BN_VOCAB, false, false, EPI_RESID_SCORE>(c.tmX_k, c.tmW_khalf, c.tmG_st, p, st)
                      : launch_gemm<BN_VOCAB, false, false, EPI_RESID_SCORE>(c.tmX_k, c.tmW_k, c.tmG_st, p, st);
        } else if (pairs) e = launch_pair<BN_VOCAB, false, false, EPI_RESID>(c.tmX_k, c.tmW_khalf, c.tmG_st, p, st);
        else e = launch_gemm<BN_VOCAB, false, false, EPI_RESID>(c.tmX_k, c.tmW_k, c.tmG_st, p, st);
        if (e != cudaSuccess) return e;
    }
    const int k_cols = strip_tiles_n * BN_VOCAB;               // columns of G written by the residual phase
    const int m_rows = m_tiles * BM;                           // rows of G written by the residual phase
    const int grad_n_tiles = (d + c.bn - 1) / c.bn;
    if (phases & PHASE_INPUT_GRAD) {
        // dX += G W_q : M = tokens, N = d, K = shard vocabulary.  The fp32 running sum lives in `acc`; the tile is
        // stored on the batch's first meeting and added (TMA reduction) afterwards; rows past the batch are dropped
        // by the output map's extent.  After the last meeting the sum is rounded to the bf16 output.
        CUtensorMap tmAcc;
        if (!make_map(&tmAcc, acc, rows, d, d, 32, 32, 4)) return cudaErrorInvalidValue;
        GemmParams ph{};
        ph.m_tiles = m_tiles;
        ph.n_tiles = grad_n_tiles;
        ph.num_kb = k_cols / BK;
        ph.group_n = pick_group_n(ph.n_tiles, 2.0 * k_cols * d);
        ph.a_mn0 = 0; ph.a_k0 = 0;
        ph.b_mn0 = 0; ph.b_k0 = w_row0;
        ph.rows_valid = rows; ph.cols_valid = d;
        ph.c_row0 = 0; ph.accumulate = first ? 0 : 1;
        ph.status = c.status;
        ph.b_3d = c.mn3d;
        set_split(ph, d, counters);
        apply_tuning(ph, EPI_DH);
        if ((c.pmask & 2) && c.pair_ok && ph.m_tiles >= 2) e = launch_pair<256, false, true, EPI_DH>(c.tmG_k, c.tmW_mn2, tmAcc, ph, st);
        else e = launch_grad<false, true, EPI_DH>(c.bn, c.tmG_k, c.tmW_mn, tmAcc, ph, st);
        if (e != cudaSuccess) return e;
        // one pass over the accumulator: dX[n, :] += delta_n W[t_n, :] for the targets in the fix range and, after
        // the batch's last meeting, the rounding to the bf16 output
        if (fix.nv > 0 || (last && dX)) {
            vpce_finish_dx_kernel<<<rows, 128, 0, st>>>(acc, last ? dX : nullptr, fix.nv > 0 ? fix.W_v0 : nullptr, labels,
                                                       c.delta, d, fix.v0, fix.nv, c.ignore_index);
            g_launches.fetch_add(1, std::memory_order_relaxed);
            if ((e = cudaGetLastError()) != cudaSuccess) return e;
        }
    }
    if (phases & PHASE_WEIGHT_GRAD) {
        // dW_q += G^T X : M = shard vocabulary, N = d, K = batch tokens; stored or added like the input gradient
        CUtensorMap tmDW;
        if (!make_map(&tmDW, dW_q, cols, d, d, 32, 32, 4)) return cudaErrorInvalidValue;
        GemmParams pw{};
        pw.m_tiles = (cols + BM - 1) / BM;
        pw.n_tiles = grad_n_tiles;
        pw.num_kb = m_rows / BK;
        pw.group_n = pick_group_n(pw.n_tiles, 2.0 * m_rows * d);
        pw.a_mn0 = 0; pw.a_k0 = 0;
        pw.b_mn0 = 0; pw.b_k0 = x_row0;
        pw.rows_valid = cols; pw.cols_valid = d;
        pw.c_row0 = 0; pw.accumulate = accumulate_dW ? 1 : 0;
        pw.status = c.status;
        pw.a_3d = c.mn3d; pw.b_3d = c.mn3d;
        set_split(pw, d, counters);
        apply_tuning(pw, EPI_DW);
        if ((c.pmask & 4) && c.pair_ok && pw.m_tiles >= 2) e = launch_pair<256, true, true, EPI_DW>(c.tmG_mn, c.tmX_mn2, tmDW, pw, st);
        else e = launch_grad<true, true, EPI_DW>(c.bn, c.tmG_mn, c.tmX_mn, tmDW, pw, st);
        if (e != cudaSuccess) return e;
        if (fix.nv > 0) {                                     // dW[t_n, :] += delta_n X[n, :] for targets in the range
            const int col_blocks = (d + 255) / 256;
            for (int r0 = 0; r0 < rows; r0 += SORT_MAX) {     // sub-chunks one after the other: a target may recur
                const int n_sub = rows - r0 < SORT_MAX ? rows - r0 : SORT_MAX;
                dim3 grid((n_sub + FIX_SEG - 1) / FIX_SEG, col_blocks);
                vpce_onehot_dw_kernel<<<grid, 256, 0, st>>>(c.keys + r0, n_sub, c.X + static_cast<size_t>(x_row0) * d,
                                                            c.delta, d, fix.v0, fix.nv, fix.dW_v0, c.partials);
                vpce_onehot_dw_combine_kernel<<<grid, 256, 0, st>>>(c.keys + r0, n_sub, d, fix.v0, fix.nv, fix.dW_v0, c.partials);
                g_launches.fetch_add(2, std::memory_order_relaxed);
                if ((e = cudaGetLastError()) != cudaSuccess) return e;
            }
        }
    }
    return cudaSuccess;
}

// clear_status: whether the call starts by zeroing the device status word (the public entry points do; the
// backward half of vp_ce_fwd_bwd_host does not, so that what its forward half flagged is still there at the end).
vpce_status forward_impl(const void* H, const void* W, const int32_t* labels, int64_t T, int64_t d, int64_t V,
                         int64_t block_v, int32_t ignore_index, float* loss, float* lse, int64_t T_chunk,
                         int64_t chunk_index_base, void* workspace, size_t workspace_bytes, void* stream,
                         bool clear_status) {
    WsLayout L;
    if (T == 0) return VPCE_OK;                                        // empty batch: nothing to compute
    if (!loss || !lse) return VPCE_INVALID_ARG;
    vpce_status s = check_common(H, W, labels, T, d, V, block_v, T_chunk, chunk_index_base, workspace, workspace_bytes, &L);
    if (s != VPCE_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    FoldCtx c;
    if (!make_fold_ctx(&c, H, T, W, V, d)) return VPCE_CUDA_ERROR;
    c.status = reinterpret_cast<int*>(ws + L.status);
    c.sm = reinterpret_cast<float*>(ws + L.sm);
    c.sz = reinterpret_cast<float*>(ws + L.sz);
    c.ylab = reinterpret_cast<float*>(ws + L.ylab);
    c.pm = reinterpret_cast<float*>(ws + L.pm);
    c.pz = reinterpret_cast<float*>(ws + L.pz);
    c.part_ld = static_cast<int>(T_chunk);
    c.ignore_index = ignore_index; c.V = static_cast<int>(V);

    if (clear_status) {
        vpce_clear_status_kernel<<<1, 32, 0, st>>>(c.status);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    CounterPool counters(reinterpret_cast<int*>(ws + L.counters), st);

    const int64_t P = (V + block_v - 1) / block_v;
    const int64_t n_chunks = (T + T_chunk - 1) / T_chunk;
    for (int64_t ch = 0; ch < n_chunks; ++ch) {
        const int64_t tok0 = ch * T_chunk;
        const int rows = static_cast<int>((T - tok0) < T_chunk ? (T - tok0) : T_chunk);
        const int64_t cg = chunk_index_base + ch;
        for (int64_t i = 0; i < P; ++i) {
            const int64_t q = ((cg - i) % P + P) % P;                  // Algorithm 3: q = (r - i) mod P
            const int64_t v_lo = q * block_v;
            const int cols = static_cast<int>((V - v_lo) < block_v ? (V - v_lo) : block_v);
            if (fold_meeting(c, static_cast<int>(tok0), rows, static_cast<int>(v_lo), cols, static_cast<int>(v_lo),
                             labels + tok0, i == 0, i == P - 1, lse + tok0, loss + tok0, counters, st) != cudaSuccess)
                return VPCE_CUDA_ERROR;
        }
    }
    return counters.failed ? VPCE_CUDA_ERROR : VPCE_OK;
}

// What the backward pass of token_logp.h adds to the head's: dloss is then the gradient of the log probability (or null).
struct ScoreGrad { const float *entropy, *dent; float inv_temp; };

vpce_status backward_impl(const void* H, const void* W, const int32_t* labels, const float* lse,
                          const float* dloss, void* dH, float* dW, int64_t T, int64_t d, int64_t V,
                          int64_t block_v, int32_t ignore_index, int64_t T_chunk, int64_t chunk_index_base,
                          int accumulate_dW, void* workspace, size_t workspace_bytes, void* stream,
                          bool clear_status, const ScoreGrad* score = nullptr) {
    WsLayout L;
    if (T == 0) {                                                      // empty batch: dW gets no contribution
        if (!accumulate_dW && dW && V > 0 && d > 0 &&
            cudaMemsetAsync(dW, 0, static_cast<size_t>(V) * d * 4, static_cast<cudaStream_t>(stream)) != cudaSuccess)
            return VPCE_CUDA_ERROR;
        return VPCE_OK;
    }
    if (!lse || (!dH && !dW)) return VPCE_INVALID_ARG;                 // either gradient may be left out, not both
    vpce_status s = check_common(H, W, labels, T, d, V, block_v, T_chunk, chunk_index_base, workspace, workspace_bytes, &L);
    if (s != VPCE_OK) return s;
    if (!aligned16(dH) || !aligned16(dW)) return VPCE_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    GradCtx c;
    if (!make_grad_ctx(&c, H, T, W, V, d, reinterpret_cast<__nv_bfloat16*>(ws + L.G), T_chunk, block_v)) return VPCE_CUDA_ERROR;
    c.status = reinterpret_cast<int*>(ws + L.status);
    c.inv_n = reinterpret_cast<float*>(ws + L.scalars);
    c.delta = reinterpret_cast<float*>(ws + L.delta);
    c.keys = reinterpret_cast<unsigned long long*>(ws + L.keys);
    c.partials = reinterpret_cast<float*>(ws + L.partials);
    c.ignore_index = ignore_index; c.V = static_cast<int>(V);
    float* acc = reinterpret_cast<float*>(ws + L.acc);

    if (clear_status) {
        vpce_clear_status_kernel<<<1, 32, 0, st>>>(c.status);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    CounterPool counters(reinterpret_cast<int*>(ws + L.counters), st);
    if (!dloss && !score) {
        vpce_count_valid_kernel<<<1, 1024, 0, st>>>(labels, T, static_cast<int>(V), ignore_index, c.inv_n, nullptr, c.status);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    const int phases = PHASE_RESIDUAL | (dH ? PHASE_INPUT_GRAD : 0) | (dW ? PHASE_WEIGHT_GRAD : 0);
    const int64_t P = (V + block_v - 1) / block_v;
    const int64_t n_chunks = (T + T_chunk - 1) / T_chunk;
    for (int64_t ch = 0; ch < n_chunks; ++ch) {
        const int64_t tok0 = ch * T_chunk;
        const int rows = static_cast<int>((T - tok0) < T_chunk ? (T - tok0) : T_chunk);
        const int64_t cg = chunk_index_base + ch;
        for (int64_t i = 0; i < P; ++i) {
            const int64_t q = ((cg - i) % P + P) % P;
            const int64_t v_lo = q * block_v;
            const int cols = static_cast<int>((V - v_lo) < block_v ? (V - v_lo) : block_v);
            // the chunk's tokens are sorted by target before its first meeting; after its last one the exact one-hot
            // terms of ALL shards are added in one go (every token's residue is on record by then)
            FixRange fix{0, i == P - 1 ? static_cast<int>(V) : 0, static_cast<const __nv_bfloat16*>(W), dW, i == 0};
            if (score) {
                c.score = true;
                c.inv_temp = score->inv_temp;
                c.entropy = score->entropy ? score->entropy + tok0 : nullptr;
                c.dent = score->dent ? score->dent + tok0 : nullptr;
            }
            if (grad_meeting(c, phases, static_cast<int>(tok0), rows, static_cast<int>(v_lo), cols, static_cast<int>(v_lo),
                             labels + tok0, lse + tok0, dloss ? dloss + tok0 : nullptr, i == 0, i == P - 1, acc,
                             dH ? static_cast<__nv_bfloat16*>(dH) + tok0 * d : nullptr, dW ? dW + v_lo * d : nullptr,
                             (accumulate_dW != 0) || (ch > 0), fix, counters, st) != cudaSuccess)
                return VPCE_CUDA_ERROR;
        }
    }
    return counters.failed ? VPCE_CUDA_ERROR : VPCE_OK;
}

}  // namespace

// ------------------------------------------------------------------------------------ C ABI
extern "C" {

size_t vp_ce_workspace_bytes(int64_t T_chunk, int64_t d, int64_t block_v) {
    WsLayout L;
    return ws_layout(T_chunk, d, block_v, &L) ? L.total : 0;
}

const char* vp_ce_status_string(vpce_status s) {
    switch (s) {
        case VPCE_OK: return "ok";
        case VPCE_INVALID_ARG: return "invalid argument (null pointer or non-positive size)";
        case VPCE_UNSUPPORTED: return "unsupported (alignment, d % 8, block_v % 256 or T_chunk % 128)";
        case VPCE_WORKSPACE_TOO_SMALL: return "workspace too small";
        case VPCE_CUDA_ERROR: return "CUDA error";
        case VPCE_STATIC_SCRATCH_EXCEEDED:
            return "T_chunk * block_v too large for the built-in scratch of vp_ce_forward_static";
        default: return "unknown status";
    }
}

int64_t vp_ce_launch_count(void) { return g_launches.load(std::memory_order_relaxed); }

vpce_status vp_ce_forward(const void* H, const void* W, const int32_t* labels, int64_t T, int64_t d, int64_t V,
                          int64_t block_v, int32_t ignore_index, float* loss, float* lse, int64_t T_chunk,
                          int64_t chunk_index_base, void* workspace, size_t workspace_bytes, void* stream) {
    return forward_impl(H, W, labels, T, d, V, block_v, ignore_index, loss, lse, T_chunk, chunk_index_base, workspace,
                        workspace_bytes, stream, true);
}

vpce_status vp_ce_backward(const void* H, const void* W, const int32_t* labels, const float* lse, const float* dloss,
                           void* dH, float* dW, int64_t T, int64_t d, int64_t V, int64_t block_v, int32_t ignore_index,
                           int64_t T_chunk, int64_t chunk_index_base, int accumulate_dW, void* workspace,
                           size_t workspace_bytes, void* stream) {
    return backward_impl(H, W, labels, lse, dloss, dH, dW, T, d, V, block_v, ignore_index, T_chunk, chunk_index_base,
                         accumulate_dW, workspace, workspace_bytes, stream, true);
}

// ---- single meetings for a ring driver (Algorithm 3 across devices)
size_t vp_ce_meeting_workspace_bytes(int64_t N, int64_t d, int64_t shard_rows) {
    if (N <= 0 || shard_rows <= 0) return 0;
    WsLayout L;
    return ws_layout(align_up(N, BM), d, align_up(shard_rows, BN_VOCAB), &L) ? L.total : 0;
}

vpce_status vp_ce_meeting_forward(const void* X, const void* W_shard, const int32_t* targets, int64_t N, int64_t d,
                                  int64_t shard_rows, int64_t v_lo, int64_t V, int32_t ignore_index, float* state,
                                  int first, int last, float* loss, float* lse, void* workspace, size_t workspace_bytes,
                                  void* stream) {
    if (!X || !W_shard || !targets || !state || !workspace) return VPCE_INVALID_ARG;
    if (N <= 0 || d <= 0 || shard_rows <= 0 || v_lo < 0 || V <= 0 || v_lo + shard_rows > V) return VPCE_INVALID_ARG;
    if (last && (!loss || !lse)) return VPCE_INVALID_ARG;
    if (!aligned16(X) || !aligned16(W_shard) || !aligned16(workspace)) return VPCE_UNSUPPORTED;
    if (N >= (1ll << 31) || V >= (1ll << 31)) return VPCE_UNSUPPORTED;
    WsLayout L;
    const int64_t n_pad = align_up(N, BM);
    if (!ws_layout(n_pad, d, align_up(shard_rows, BN_VOCAB), &L)) return VPCE_UNSUPPORTED;
    if (workspace_bytes < L.total) return VPCE_WORKSPACE_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    FoldCtx c;
    if (!make_fold_ctx(&c, X, N, W_shard, shard_rows, d)) return VPCE_CUDA_ERROR;
    c.status = reinterpret_cast<int*>(ws + L.status);
    c.sm = state; c.sz = state + N; c.ylab = state + 2 * N;              // the state is the caller's: it may travel
    c.pm = reinterpret_cast<float*>(ws + L.pm);
    c.pz = reinterpret_cast<float*>(ws + L.pz);
    c.part_ld = static_cast<int>(n_pad);
    c.ignore_index = ignore_index; c.V = static_cast<int>(V);
    if (first) {                                                       // a batch's first meeting starts a clean status word
        vpce_clear_status_kernel<<<1, 32, 0, st>>>(c.status);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    CounterPool counters(reinterpret_cast<int*>(ws + L.counters), st);
    if (fold_meeting(c, 0, static_cast<int>(N), 0, static_cast<int>(shard_rows), static_cast<int>(v_lo), targets, first != 0,
                     last != 0, lse, loss, counters, st) != cudaSuccess)
        return VPCE_CUDA_ERROR;
    return counters.failed ? VPCE_CUDA_ERROR : VPCE_OK;
}

vpce_status vp_ce_meeting_backward(const void* X, const void* W_shard, const int32_t* targets, const float* lse,
                                   const float* dloss, int64_t N, int64_t d, int64_t shard_rows, int64_t v_lo, int64_t V,
                                   int32_t ignore_index, int phases, float* dX_acc, int first, int last, void* dX,
                                   float* dW_shard, int accumulate_dW, void* workspace, size_t workspace_bytes,
                                   void* stream) {
    if (!X || !W_shard || !targets || !lse || !dloss || !workspace) return VPCE_INVALID_ARG;
    if (N <= 0 || d <= 0 || shard_rows <= 0 || v_lo < 0 || V <= 0 || v_lo + shard_rows > V) return VPCE_INVALID_ARG;
    if (phases <= 0 || phases > 7) return VPCE_INVALID_ARG;
    if ((phases & PHASE_INPUT_GRAD) && ((!(first && last) && !dX_acc) || (last && !dX))) return VPCE_INVALID_ARG;
    if ((phases & PHASE_WEIGHT_GRAD) && !dW_shard) return VPCE_INVALID_ARG;
    if (!aligned16(X) || !aligned16(W_shard) || !aligned16(workspace) || !aligned16(dX_acc) || !aligned16(dX) ||
        !aligned16(dW_shard))
        return VPCE_UNSUPPORTED;
    if (N >= (1ll << 31) || V >= (1ll << 31)) return VPCE_UNSUPPORTED;
    WsLayout L;
    const int64_t n_pad = align_up(N, BM), s_pad = align_up(shard_rows, BN_VOCAB);
    if (!ws_layout(n_pad, d, s_pad, &L)) return VPCE_UNSUPPORTED;
    if (workspace_bytes < L.total) return VPCE_WORKSPACE_TOO_SMALL;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    GradCtx c;
    if (!make_grad_ctx(&c, X, N, W_shard, shard_rows, d, reinterpret_cast<__nv_bfloat16*>(ws + L.G), n_pad, s_pad))
        return VPCE_CUDA_ERROR;
    c.status = reinterpret_cast<int*>(ws + L.status);
    c.inv_n = reinterpret_cast<float*>(ws + L.scalars);
    c.delta = reinterpret_cast<float*>(ws + L.delta);
    c.keys = reinterpret_cast<unsigned long long*>(ws + L.keys);
    c.partials = reinterpret_cast<float*>(ws + L.partials);
    c.ignore_index = ignore_index; c.V = static_cast<int>(V);
    if (first && (phases & PHASE_RESIDUAL)) {
        vpce_clear_status_kernel<<<1, 32, 0, st>>>(c.status);
        g_launches.fetch_add(1, std::memory_order_relaxed);
    }
    CounterPool counters(reinterpret_cast<int*>(ws + L.counters), st);
    // a batch whose only meeting this is (first and last) needs no travelling accumulator: the workspace's own serves
    float* acc = dX_acc ? dX_acc : reinterpret_cast<float*>(ws + L.acc);
    // every meeting sorts the batch it is handed (it may be another batch each round) and adds the exact one-hot
    // terms of the targets that lie in its own shard
    FixRange fix{static_cast<int>(v_lo), static_cast<int>(shard_rows), static_cast<const __nv_bfloat16*>(W_shard), dW_shard,
                 true};
    if (grad_meeting(c, phases, 0, static_cast<int>(N), 0, static_cast<int>(shard_rows), static_cast<int>(v_lo), targets, lse,
                     dloss, first != 0, last != 0, acc, static_cast<__nv_bfloat16*>(dX), dW_shard, accumulate_dW != 0,
                     fix, counters, st) != cudaSuccess)
        return VPCE_CUDA_ERROR;
    return counters.failed ? VPCE_CUDA_ERROR : VPCE_OK;
}

vpce_status vp_ce_mean_loss(const float* loss, const int32_t* labels, int64_t T, int64_t V, int32_t ignore_index,
                            float* mean_out, int32_t* n_valid_out, void* stream) {
    if (!mean_out || !n_valid_out || T < 0 || V <= 0 || (T > 0 && (!loss || !labels))) return VPCE_INVALID_ARG;
    // T == 0 (an empty batch) gives mean 0 and n_valid 0, like the empty-batch rule of the other calls
    vpce_mean_loss_kernel<<<1, 1024, 0, static_cast<cudaStream_t>(stream)>>>(loss, labels, T, static_cast<int>(V),
                                                                           ignore_index, mean_out, n_valid_out);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

vpce_status vp_ce_mean_loss_grad(const int32_t* labels, int64_t T, int64_t V, int32_t ignore_index,
                                 const int32_t* n_valid, const float* upstream, float* dloss_out, void* stream) {
    if (!n_valid || T < 0 || V <= 0 || (T > 0 && (!labels || !dloss_out))) return VPCE_INVALID_ARG;
    if (T == 0) return VPCE_OK;
    vpce_mean_grad_kernel<<<static_cast<unsigned>((T + 255) / 256), 256, 0, static_cast<cudaStream_t>(stream)>>>(
        labels, T, static_cast<int>(V), ignore_index, n_valid, upstream, dloss_out);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    return cudaGetLastError() == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

vpce_status vp_ce_device_status(const void* workspace, int32_t* host_out, void* stream) {
    if (!workspace || !host_out) return VPCE_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(host_out, workspace, sizeof(int32_t), cudaMemcpyDeviceToHost, st) != cudaSuccess)
        return VPCE_CUDA_ERROR;
    return cudaStreamSynchronize(st) == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

int64_t vp_ce_set_wait_limit_ns(int64_t ns) {
    const unsigned long long prev = g_wait_limit_ns.load(std::memory_order_relaxed);
    if (ns > 0) {
        unsigned long long v = static_cast<unsigned long long>(ns);
        if (v < 1000000ull) v = 1000000ull;                     // at least 1 ms: far longer than any copy is in flight
        if (v > 60000000000ull) v = 60000000000ull;
        g_wait_limit_ns.store(v, std::memory_order_relaxed);
    }
    return static_cast<int64_t>(prev);
}

int vp_ce_set_tail_parts(int parts) {
    const int prev = g_tail_parts.load(std::memory_order_relaxed);
    if (parts >= -1 && parts != 1 && parts <= 8) g_tail_parts.store(parts, std::memory_order_relaxed);
    return prev;
}

vpce_status vp_ce_tail_choice(int row_tiles, int col_tiles, int group_cols, int last_width, int k_blocks, int pairs,
                              int* n_tiles_split, int* parts, int* stagger) {
    if (row_tiles <= 0 || col_tiles <= 0 || group_cols <= 0 || last_width <= 0 || last_width > 256 || k_blocks <= 0 ||
        pairs <= 0 || !n_tiles_split || !parts || !stagger)
        return VPCE_INVALID_ARG;
    const SplitChoice c = pick_split(row_tiles, col_tiles, group_cols, last_width, k_blocks, pairs);
    *n_tiles_split = c.n_cut;
    *parts = c.ks;
    *stagger = c.stagger;
    return VPCE_OK;
}

vpce_status vp_ce_debug_drop_copy(int kernel_kind, int k_block, int cta_ranks) {
    if (kernel_kind < 0) { g_drop.store(-1, std::memory_order_relaxed); return VPCE_OK; }
    if (kernel_kind > 3 || k_block < 0 || k_block > 0xffff || cta_ranks <= 0 || cta_ranks > 3) return VPCE_INVALID_ARG;
    g_drop.store(kernel_kind | (k_block << 8) | (cta_ranks << 24), std::memory_order_relaxed);
    return VPCE_OK;
}

void vp_ce_profile_enable(int on) {
    std::lock_guard<std::mutex> lk(g_prof_mu);
    g_prof_on = on != 0;
}

vpce_status vp_ce_profile_collect(double* ms_out, int64_t* launches_out) {
    if (!ms_out || !launches_out) return VPCE_INVALID_ARG;
    std::vector<ProfEntry> entries;
    {
        std::lock_guard<std::mutex> lk(g_prof_mu);
        entries.swap(g_prof);
    }
    for (int k = 0; k < 4; ++k) { ms_out[k] = 0.0; launches_out[k] = 0; }
    vpce_status rc = VPCE_OK;
    for (auto& e : entries) {
        float ms = 0.f;
        if (cudaEventSynchronize(e.b) == cudaSuccess && cudaEventElapsedTime(&ms, e.a, e.b) == cudaSuccess) {
            ms_out[e.kind] += ms;
            launches_out[e.kind] += 1;
        } else {
            rc = VPCE_CUDA_ERROR;
        }
        cudaEventDestroy(e.a);
        cudaEventDestroy(e.b);
    }
    return rc;
}

vpce_status vp_ce_fwd_bwd_host(const void* H_host, const int32_t* labels_host, const void* W, float* loss_host,
                               void* dH_host, float* dW, int64_t T, int64_t d, int64_t V, int64_t block_v,
                               int32_t ignore_index, int64_t T_chunk, int64_t chunk_index_base, int accumulate_dW,
                               void* H_dev, int32_t* labels_dev, float* loss_dev, float* lse_dev, void* dH_dev,
                               void* workspace, size_t workspace_bytes, void* stream) {
    if (!H_host || !labels_host || !loss_host || !dH_host || !H_dev || !labels_dev || !loss_dev || !lse_dev || !dH_dev)
        return VPCE_INVALID_ARG;
    if (T <= 0 || d <= 0) return VPCE_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t hbytes = static_cast<size_t>(T) * d * 2;
    if (cudaMemcpyAsync(H_dev, H_host, hbytes, cudaMemcpyHostToDevice, st) != cudaSuccess) return VPCE_CUDA_ERROR;
    if (cudaMemcpyAsync(labels_dev, labels_host, static_cast<size_t>(T) * 4, cudaMemcpyHostToDevice, st) != cudaSuccess)
        return VPCE_CUDA_ERROR;
    vpce_status s = vp_ce_forward(H_dev, W, labels_dev, T, d, V, block_v, ignore_index, loss_dev, lse_dev, T_chunk,
                                  chunk_index_base, workspace, workspace_bytes, stream);
    if (s != VPCE_OK) return s;
    // the status word keeps what the forward half flagged: it is cleared once, at the start of the whole pass
    s = backward_impl(H_dev, W, labels_dev, lse_dev, nullptr, dH_dev, dW, T, d, V, block_v, ignore_index, T_chunk,
                      chunk_index_base, accumulate_dW, workspace, workspace_bytes, stream, false);
    if (s != VPCE_OK) return s;
    if (cudaMemcpyAsync(loss_host, loss_dev, static_cast<size_t>(T) * 4, cudaMemcpyDeviceToHost, st) != cudaSuccess)
        return VPCE_CUDA_ERROR;
    if (cudaMemcpyAsync(dH_host, dH_dev, hbytes, cudaMemcpyDeviceToHost, st) != cudaSuccess) return VPCE_CUDA_ERROR;
    return cudaStreamSynchronize(st) == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

// ------------------------------------------------------------------------------------ forward without a caller workspace
}  // extern "C"

namespace {

// Scratch of vp_ce_forward_static.  It is part of the loaded module: every GPU that loads this
// library holds these bytes until the process exits.  In host code the NAME of a __device__
// array is only a handle for the runtime, never an address a kernel may use; the device address
// is looked up once per device with cudaGetSymbolAddress and that pointer is what kernels get.
constexpr size_t STATIC_SCRATCH_BYTES = VPCE_STATIC_SCRATCH_BYTES;
static __device__ __align__(256) unsigned char g_static_scratch[STATIC_SCRATCH_BYTES];

std::mutex g_static_mu;
unsigned char* g_static_ptr[64] = {nullptr};

// Device address of g_static_scratch on the current device (looked up on first use).
vpce_status static_scratch_address(unsigned char** out) {
    int dev = -1;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return VPCE_CUDA_ERROR;
    std::lock_guard<std::mutex> lk(g_static_mu);
    if (!g_static_ptr[dev]) {
        void* ptr = nullptr;
        if (cudaGetSymbolAddress(&ptr, g_static_scratch) != cudaSuccess || !ptr) return VPCE_CUDA_ERROR;
        g_static_ptr[dev] = static_cast<unsigned char*>(ptr);
    }
    *out = g_static_ptr[dev];
    return VPCE_OK;
}

__global__ void vpce_copy_status_kernel(const int* status, int* out) { if (threadIdx.x == 0) *out = *status; }

}  // namespace

extern "C" {

vpce_status vp_ce_forward_static(const void* H, const void* W, const int32_t* labels, int64_t T, int64_t d, int64_t V,
                                 int64_t block_v, int32_t ignore_index, float* loss, float* lse, int64_t T_chunk,
                                 int64_t chunk_index_base, int32_t* device_status_out, void* stream) {
    if (!H || !W || !labels || !loss || !lse) return VPCE_INVALID_ARG;
    if (T <= 0 || d <= 0 || V <= 0 || block_v <= 0 || T_chunk <= 0 || chunk_index_base < 0) return VPCE_INVALID_ARG;
    if (!aligned16(H) || !aligned16(W)) return VPCE_UNSUPPORTED;
    if (T >= (1ll << 31) || V >= (1ll << 31)) return VPCE_UNSUPPORTED;
    WsLayout L;
    if (!ws_layout(T_chunk, d, block_v, &L)) return VPCE_UNSUPPORTED;
    // The forward touches the layout up to (not including) the residual strip G.
    if (L.G > STATIC_SCRATCH_BYTES) return VPCE_STATIC_SCRATCH_EXCEEDED;
    unsigned char* ws = nullptr;
    vpce_status s = static_scratch_address(&ws);
    if (s != VPCE_OK) return s;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    int* status = reinterpret_cast<int*>(ws + L.status);
    float* sm = reinterpret_cast<float*>(ws + L.sm);
    float* sz = reinterpret_cast<float*>(ws + L.sz);
    float* ylab = reinterpret_cast<float*>(ws + L.ylab);
    float* pm = reinterpret_cast<float*>(ws + L.pm);
    float* pz = reinterpret_cast<float*>(ws + L.pz);

    CUtensorMap tmH, tmW;
    if (!make_map(&tmH, H, T, d, d, BK, BM) || !make_map(&tmW, W, V, d, d, BK, BN_VOCAB)) return VPCE_CUDA_ERROR;
    using Cfg = StageCfg<BN_VOCAB>;
    auto kern = vpce_gemm_kernel<BN_VOCAB, false, false, EPI_FOLD>;
    static std::atomic<bool> attr_set[64];
    if (ensure_smem_attr(kern, Cfg::SMEM_TOTAL, attr_set) != cudaSuccess) return VPCE_CUDA_ERROR;

    // The array keeps whatever the previous call left: the status word must start at zero; the
    // running state is initialised by the first merge of every chunk and the partial slots are
    // fully rewritten before they are read.
    vpce_clear_status_kernel<<<1, 32, 0, st>>>(status);
    g_launches.fetch_add(1, std::memory_order_relaxed);
    CounterPool counters(reinterpret_cast<int*>(ws + L.counters), st);   // a memset, not an allocation

    const int64_t P = (V + block_v - 1) / block_v;
    const int64_t n_chunks = (T + T_chunk - 1) / T_chunk;
    const int num_kb = static_cast<int>((d + BK - 1) / BK);
    for (int64_t c = 0; c < n_chunks; ++c) {
        const int64_t tok0 = c * T_chunk;
        const int rows = static_cast<int>((T - tok0) < T_chunk ? (T - tok0) : T_chunk);
        const int64_t cg = chunk_index_base + c;
        for (int64_t i = 0; i < P; ++i) {
            const int64_t q = ((cg - i) % P + P) % P;
            const int64_t v_lo = q * block_v;
            const int cols = static_cast<int>((V - v_lo) < block_v ? (V - v_lo) : block_v);
            GemmParams p{};
            p.m_tiles = (rows + BM - 1) / BM;
            p.n_tiles = (cols + BN_VOCAB - 1) / BN_VOCAB;
            p.num_kb = num_kb;
            p.group_n = pick_group_n(p.n_tiles, 2.0 * cols * d);
            p.a_mn0 = static_cast<int>(tok0); p.b_mn0 = static_cast<int>(v_lo);
            p.rows_valid = rows; p.cols_valid = cols;
            p.v_lo = static_cast<int>(v_lo);
            p.labels = labels + tok0;
            p.ignore_index = ignore_index; p.V = static_cast<int>(V);
            p.pm = pm; p.pz = pz; p.ylab = ylab; p.part_ld = static_cast<int>(T_chunk);
            p.status = status;
            apply_tuning(p, EPI_FOLD);
            p.tile_counter = counters.take();
            const int tiles = p.m_tiles * p.n_tiles;
            const int grid = tiles < num_sms() ? tiles : num_sms();
            kern<<<grid, NUM_THREADS, Cfg::SMEM_TOTAL, st>>>(tmH, tmW, tmH, finish_params(p, EPI_FOLD));
            vpce_merge_kernel<<<(rows + 255) / 256, 256, 0, st>>>(pm, pz, static_cast<int>(T_chunk), p.n_tiles, sm, sz, ylab,
                                                                  rows, i == 0, i == P - 1, labels + tok0, ignore_index,
                                                                  static_cast<int>(V), lse + tok0, loss + tok0, status);
            g_launches.fetch_add(2, std::memory_order_relaxed);
            if (cudaGetLastError() != cudaSuccess) return VPCE_CUDA_ERROR;
        }
    }
    if (device_status_out) {
        vpce_copy_status_kernel<<<1, 32, 0, st>>>(status, device_status_out);
        g_launches.fetch_add(1, std::memory_order_relaxed);
        if (cudaGetLastError() != cudaSuccess) return VPCE_CUDA_ERROR;
    }
    return VPCE_OK;
}

}  // extern "C"

#include "vp_ce_f32.inc"

// ------------------------------------------------------------------------------------ token_logp.h, backward
extern "C" int vp_token_logp_backward(const void* H, const void* W, const int32_t* tokens, const float* lse, const float* entropy,
                                      const float* dlogp, const float* dent, void* dH, float* dW, int64_t T, int64_t d, int64_t V,
                                      double temperature, int64_t block_v, int32_t ignore_index, int64_t T_chunk,
                                      int64_t chunk_index_base, int accumulate_dW, void* workspace, size_t workspace_bytes, void* stream) {
    // p is formed anew from lse as one number, which leaves nothing of it where lse / temperature is large, nor of an entropy's gradient
    // where the logits lie close together over the temperature: narrower than the forward call's range
    if (!(temperature >= 0.01) || !(temperature <= 100.0)) return VPCE_INVALID_ARG;
    if (T > 0 && ((!dlogp && !dent) || (dent && !entropy))) return VPCE_INVALID_ARG;
    const ScoreGrad score{entropy, dent, static_cast<float>(1.0 / temperature)};
    return backward_impl(H, W, tokens, lse, dlogp, dH, dW, T, d, V, block_v, ignore_index, T_chunk, chunk_index_base, accumulate_dW, workspace,
                         workspace_bytes, stream, true, &score);
}
