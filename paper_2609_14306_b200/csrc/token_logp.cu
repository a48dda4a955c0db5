// Log probabilities of given tokens with entropy and top alternatives, forward (token_logp.h); the backward pass extends the head's own
// and lives with it (vp_ce.cu).
//
// Up to 64 tokens: one pass over the weight, then one over the 148 slices that it leaves per token.  More: chunks of up to 4096 tokens,
// whose hidden states stay in L2 while the vocabulary goes by in strips; each strip leaves (m, z, u) per token and 128 columns, and
// the candidates for the alternatives, and the join folds them into the token's running state.  Candidates cost little: what slices
// have found so far bounds the token's list from below (`floor`, `marks`), and slices that come later compare their maxima with it.
// The strips' width follows from the workspace that partial states and candidates may take (64 MB).

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <mutex>

#include "token_logp.h"
#include "token_logp_kernels.cuh"
#include "vp_ce.h"

namespace {

using namespace vptl;

constexpr int64_t CHUNK = 4096;                     // tokens whose hidden states stay in L2 beside a strip of the weight
constexpr size_t SLICE_BYTES = size_t{64} << 20;    // partial states and candidates of a launch
constexpr int FEW_CTAS = 148;                       // slices of the kernel for few tokens: a CTA per SM
static_assert(FEW_CTAS <= JOIN_FEW_SLICES, "the join takes them all at once");

std::atomic<int> g_drop{-1};

size_t up(size_t x) { return (x + 255) / 256 * 256; }

struct Plan {
    int64_t chunk;                                  // tokens per launch
    int strip_tiles, slices;                        // 256-column tiles per launch; slices per token and launch
    bool few;
    size_t floor, marks, chosen, run, run_list, part, cand, total;
};

bool plan(int64_t T, int64_t d, int64_t V, int top, int d_unit, int64_t d_most, Plan* p) {
    if (T < 0 || d <= 0 || V <= 0 || top < 0 || top > MAX_TOP || top > V) return false;
    if (d % d_unit || d > d_most || T >= (int64_t{1} << 31) || V >= (int64_t{1} << 31) - TILE_N) return false;
    p->few = T <= FEW_TOKENS;
    const int tiles = static_cast<int>((V + TILE_N - 1) / TILE_N);
    if (p->few) {
        p->chunk = std::max<int64_t>(T, 1);
        p->strip_tiles = tiles;
        p->slices = static_cast<int>(std::min<int64_t>(FEW_CTAS, (V + FEW_ROWS - 1) / FEW_ROWS));
    } else {
        p->chunk = std::min(T, CHUNK);
        const size_t per_tile = static_cast<size_t>(p->chunk) * 2 * (sizeof(float4) + sizeof(uint2) * top);
        const int most = static_cast<int>(std::max<size_t>(32, SLICE_BYTES / per_tile));
        const int strips = (tiles + most - 1) / most;
        p->strip_tiles = (tiles + strips - 1) / strips;                     // strips of one size
        p->slices = 2 * p->strip_tiles;
    }
    size_t off = 256;                                                       // the status word
    p->floor = off;    off = up(off + sizeof(unsigned) * p->chunk);
    p->marks = off;    off = up(off + (p->few || top == 0 ? 0 : 32 * sizeof(unsigned) * p->chunk));
    p->chosen = off;   off = up(off + sizeof(float) * p->chunk);
    p->run = off;      off = up(off + sizeof(float4) * p->chunk);
    p->run_list = off; off = up(off + sizeof(Key) * p->chunk * top);
    p->part = off;     off = up(off + sizeof(float4) * p->chunk * p->slices);
    p->cand = off;     off = up(off + sizeof(uint2) * p->chunk * p->slices * top);
    p->total = off;
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

// Map over a contiguous [rows, cols] matrix of bf16 or bytes: boxes of 128 bytes x box_rows, 128-byte swizzle.
bool make_map(CUtensorMap* map, const void* ptr, int64_t rows, int64_t cols, int elem, int box_rows) {
    auto enc = get_encode();
    if (!enc) return false;
    cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)};
    cuuint64_t strides[1] = {static_cast<cuuint64_t>(cols) * elem};
    cuuint32_t box[2] = {static_cast<cuuint32_t>(KB_BYTES / elem), static_cast<cuuint32_t>(box_rows)};
    cuuint32_t estr[2] = {1, 1};
    return enc(map, elem == 1 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(ptr), dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

int sm_count() {
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

// Raises the dynamic shared-memory limit of `kern` once per device.
template <typename K> cudaError_t raise_smem(K kern, std::atomic<bool>* done) {
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (known && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MAX);
    if (e == cudaSuccess && known) done[dev].store(true, std::memory_order_release);
    return e;
}

template <bool F8, bool TOP> cudaError_t launch_strip(const CUtensorMap& h, const CUtensorMap& w, const Params& p, cudaStream_t st) {
    auto kern = tl_strip_kernel<F8, TOP>;
    static std::atomic<bool> done[64];
    if (cudaError_t e = raise_smem(kern, done); e != cudaSuccess) return e;
    const int grid = 2 * std::min(p.m_tiles * p.n_tiles, std::max(1, sm_count() / 2));
    kern<<<grid, THREADS, Strip<F8, TOP>::SMEM, st>>>(h, w, p);
    return cudaGetLastError();
}

template <int NT, bool F8, bool TOP> cudaError_t launch_few(const CUtensorMap& h, const CUtensorMap& w, const Params& p, cudaStream_t st) {
    auto kern = tl_few_kernel<NT, F8, TOP>;
    static std::atomic<bool> done[64];
    if (cudaError_t e = raise_smem(kern, done); e != cudaSuccess) return e;
    kern<<<p.slices, Few<NT, F8>::THREADS, Few<NT, F8>::SMEM_FIXED + (F8 ? NT * p.kbs * 4 : 0), st>>>(h, w, p);
    return cudaGetLastError();
}
template <bool F8, bool TOP> cudaError_t launch_few(int nt, const CUtensorMap& h, const CUtensorMap& w, const Params& p, cudaStream_t st) {
    if (nt == 16) return launch_few<16, F8, TOP>(h, w, p, st);
    if (nt == 32) return launch_few<32, F8, TOP>(h, w, p, st);
    return launch_few<64, F8, TOP>(h, w, p, st);
}

// Brought up while the kernel before it still runs (it waits for that one's end before it reads anything).
template <bool TOP> cudaError_t launch_join(bool few, const JoinParams& j, cudaStream_t st) {
    cudaLaunchConfig_t cfg{};
    const bool many = j.rows >= JOIN_MANY;
    cfg.gridDim = dim3(few || !many ? j.rows : (j.rows + JOIN_WARPS - 1) / JOIN_WARPS);
    cfg.blockDim = dim3(few ? JOIN_FEW_THREADS : JOIN_THREADS);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, few ? tl_join_few_kernel<TOP> : many ? tl_join_kernel<TOP, 1> : tl_join_kernel<TOP, JOIN_WARPS>, j);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

constexpr int64_t D_MOST_BF16 = 1 << 20, D_MOST_F8 = FEW_MAX_KBS * 128;

template <bool F8>
int forward(const void* H, const float* Hs, const void* W, const float* Ws, const int32_t* tokens, int64_t T, int64_t d, int64_t V,
            double temperature, int32_t ignore_index, float* logp, float* lse, float* entropy, float* top_logp, int32_t* top_ids, int top,
            void* workspace, size_t workspace_bytes, cudaStream_t st) {
    if (T < 0 || d <= 0 || V <= 0 || top < 0 || top > MAX_TOP || top > V || !(temperature >= 1e-6) || !(temperature <= 1e6)) return VPCE_INVALID_ARG;
    if ((logp != nullptr) != (tokens != nullptr) && T > 0) return VPCE_INVALID_ARG;
    if (T == 0) return VPCE_OK;
    if (!H || !W || (F8 && (!Hs || !Ws)) || !workspace || (top > 0 && (!top_logp || !top_ids))) return VPCE_INVALID_ARG;
    Plan pl;
    if (!aligned16(H) || !aligned16(W) || !aligned16(workspace) || !plan(T, d, V, top, F8 ? 16 : 8, F8 ? D_MOST_F8 : D_MOST_BF16, &pl))
        return VPCE_UNSUPPORTED;
    for (const void* q : {static_cast<const void*>(Hs), static_cast<const void*>(Ws), static_cast<const void*>(tokens), static_cast<const void*>(logp),
                          static_cast<const void*>(lse), static_cast<const void*>(entropy), static_cast<const void*>(top_logp), static_cast<const void*>(top_ids)})
        if (reinterpret_cast<uintptr_t>(q) & 3u) return VPCE_UNSUPPORTED;
    if (workspace_bytes < pl.total) return VPCE_WORKSPACE_TOO_SMALL;

    const int elem = F8 ? 1 : 2;
    const int nt = T <= 16 ? 16 : T <= 32 ? 32 : 64;
    CUtensorMap tmH, tmW;
    if (!make_map(&tmH, H, T, d, elem, pl.few ? nt : TILE_M) || !make_map(&tmW, W, V, d, elem, pl.few ? FEW_ROWS : HALF_N)) return VPCE_CUDA_ERROR;
    uint8_t* ws = static_cast<uint8_t*>(workspace);
    Params p{};
    p.kbs = static_cast<int>((d * elem + KB_BYTES - 1) / KB_BYTES);
    p.V = static_cast<int>(V);
    p.scale = static_cast<float>(1.4426950408889634074 / temperature);
    p.top = top;
    p.slices = pl.slices;
    p.part = reinterpret_cast<float4*>(ws + pl.part);
    p.cand = reinterpret_cast<uint2*>(ws + pl.cand);
    p.floor = reinterpret_cast<unsigned*>(ws + pl.floor);
    p.chosen = reinterpret_cast<float*>(ws + pl.chosen);
    p.hs = Hs; p.ws = Ws;
    p.status = reinterpret_cast<int*>(ws);
    p.wait_limit_ns = static_cast<unsigned long long>(vp_ce_set_wait_limit_ns(0));
    p.drop_kb = g_drop.exchange(-1, std::memory_order_relaxed);
    JoinParams j{};
    j.slices = pl.slices; j.top = top; j.scale = p.scale; j.inv_temp = static_cast<float>(1.0 / temperature);
    j.part = p.part; j.cand = p.cand; j.floor = p.floor; j.chosen = p.chosen;
    j.run = reinterpret_cast<float4*>(ws + pl.run);
    j.run_list = reinterpret_cast<Key*>(ws + pl.run_list);
    j.ignore_index = ignore_index; j.V = p.V; j.status = p.status;

    for (int64_t t0 = 0; t0 < T; t0 += pl.chunk) {
        // strips: the status word before the first chunk, the tokens' bounds before every one
        const size_t from = t0 == 0 ? 0 : pl.floor, to = top > 0 ? pl.chosen : pl.floor;
        if (!pl.few && from < to && cudaMemsetAsync(ws + from, 0, to - from, st) != cudaSuccess) return VPCE_CUDA_ERROR;
        p.rows = j.rows = static_cast<int>(std::min(pl.chunk, T - t0));
        p.row0 = static_cast<int>(t0);
        p.tokens = j.tokens = tokens ? tokens + t0 : nullptr;
        j.logp = logp ? logp + t0 : nullptr;
        j.lse = lse ? lse + t0 : nullptr;
        j.entropy = entropy ? entropy + t0 : nullptr;
        j.top_logp = top ? top_logp + t0 * top : nullptr;
        j.top_ids = top ? top_ids + t0 * top : nullptr;
        p.m_tiles = (p.rows + 2 * TILE_M - 1) / (2 * TILE_M);
        const int64_t strip = static_cast<int64_t>(pl.strip_tiles) * TILE_N;
        for (int64_t c0 = 0; c0 < V; c0 += strip) {
            p.col0 = static_cast<int>(c0);
            p.cols = static_cast<int>(std::min(strip, V - c0));
            p.n_tiles = (p.cols + TILE_N - 1) / TILE_N;
            p.marks = top > 0 && c0 == 0 ? reinterpret_cast<unsigned*>(ws + pl.marks) : nullptr;
            if (!pl.few) p.slices = j.slices = 2 * p.n_tiles;
            cudaError_t e;
            if (pl.few) e = top ? launch_few<F8, true>(nt, tmH, tmW, p, st) : launch_few<F8, false>(nt, tmH, tmW, p, st);
            else e = top ? launch_strip<F8, true>(tmH, tmW, p, st) : launch_strip<F8, false>(tmH, tmW, p, st);
            if (e != cudaSuccess) return VPCE_CUDA_ERROR;
            j.first = c0 == 0;
            j.last = c0 + strip >= V;
            e = top ? launch_join<true>(pl.few, j, st) : launch_join<false>(pl.few, j, st);
            if (e != cudaSuccess) return VPCE_CUDA_ERROR;
            p.drop_kb = -1;
        }
    }
    return VPCE_OK;
}

}  // namespace

extern "C" {

size_t vp_token_logp_workspace_bytes(int64_t T, int64_t d, int64_t V, int top) {
    Plan p;
    return plan(T, d, V, top, 8, D_MOST_BF16, &p) ? p.total : 0;
}

size_t vp_token_logp_fp8_workspace_bytes(int64_t T, int64_t d, int64_t V, int top) {
    Plan p;
    return plan(T, d, V, top, 16, D_MOST_F8, &p) ? p.total : 0;
}

int vp_token_logp_forward(const void* H, const void* W, const int32_t* tokens, int64_t T, int64_t d, int64_t V, double temperature,
                          int32_t ignore_index, float* logp, float* lse, float* entropy, float* top_logp, int32_t* top_ids, int top,
                          void* workspace, size_t workspace_bytes, void* stream) {
    return forward<false>(H, nullptr, W, nullptr, tokens, T, d, V, temperature, ignore_index, logp, lse, entropy, top_logp, top_ids, top,
                          workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int vp_token_logp_fp8_forward(const void* Hq, const float* Hs, const void* Wq, const float* Ws, const int32_t* tokens, int64_t T,
                              int64_t d, int64_t V, double temperature, int32_t ignore_index, float* logp, float* lse, float* entropy,
                              float* top_logp, int32_t* top_ids, int top, void* workspace, size_t workspace_bytes, void* stream) {
    return forward<true>(Hq, Hs, Wq, Ws, tokens, T, d, V, temperature, ignore_index, logp, lse, entropy, top_logp, top_ids, top, workspace,
                         workspace_bytes, static_cast<cudaStream_t>(stream));
}

int vp_token_logp_debug_drop(int k_block) {
    g_drop.store(k_block < 0 ? -1 : k_block, std::memory_order_relaxed);
    return VPCE_OK;
}

}  // extern "C"
