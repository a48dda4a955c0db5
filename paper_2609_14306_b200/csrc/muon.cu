// The Muon update (muon.h): momentum and norm in one pass, the scaled fp16 start of the iteration, then three products per
// step on the tensor cores, the last of which updates the weights in its epilogue.
//
// Every matrix is worked on in its wide orientation R x C, R <= C (the transposition happens while the start is written and
// while the weights are updated), so the Gram matrix A = X X^T has the smaller side.  A and B = b A + c A A are symmetric:
// only the tiles on and right of the diagonal are computed, the others are written as mirror images.  Per step that leaves
// R^2 C + R^3 + 2 R^2 C operations instead of 4 R^2 C + 2 R^3.

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <cudaTypedefs.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdint>
#include <mutex>

#include "muon.h"
#include "muon_kernels.cuh"
#include "vp_ce.h"

namespace {

using namespace vpmuon;

constexpr double DEFAULT_COEFFS[3] = {3.4445, -4.7750, 2.0315};
// muon_debug_drop: kernel kind in bits 0-7, index in bits 8-23, CTA ranks in bits 24-27; -1: nothing armed.
std::atomic<int> g_drop{-1};
// Takes what is armed for a launch of this kind.
void take_drop(GemmParams* q, int kind) {
    q->drop = -1;
    int armed = g_drop.load(std::memory_order_relaxed);
    if (armed >= 0 && (armed & 0xff) == kind && g_drop.compare_exchange_strong(armed, -1)) {
        q->drop = (armed >> 8) & 0xffff;
        q->drop_ranks = armed >> 24 & 0xf;
    }
}

constexpr double MAX_BOUND = 8.0;               // of |X|_2 along the iteration: its square and the polynomial still fit fp16

int64_t up64(int64_t x) { return (x + 63) / 64 * 64; }

struct Layout {
    int64_t R, C, lda, ldx, parts;
    size_t done, sumsq, X0, X1, A, B, total;
};

bool layout(int64_t batch, int64_t rows, int64_t cols, Layout* L) {
    if (batch < 0 || rows < 0 || cols < 0) return false;
    L->R = std::min(rows, cols); L->C = std::max(rows, cols);
    if (batch > 65535 || L->C > (1 << 22) || L->R > (1 << 17)) return false;
    L->lda = up64(L->R); L->ldx = up64(L->C);
    const int64_t row_tiles = (L->R + TM - 1) / TM, col_tiles = (L->C + 63) / 64;
    if (batch * row_tiles * col_tiles > (int64_t{1} << 20)) return false;   // work-list positions and counts fit 31 bits
    L->parts = std::max<int64_t>(1, std::min<int64_t>(MAX_PARTS, (rows * cols + 16 * PREP_THREADS - 1) / (16 * PREP_THREADS)));
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    size_t off = 256;                                                      // the status word, the work list's counter
    L->done = off;  off = up(off + sizeof(int) * DONE_PITCH * batch);
    L->sumsq = off; off = up(off + sizeof(double) * batch * L->parts);
    L->X0 = off;    off = up(off + 2 * static_cast<size_t>(batch) * L->R * L->ldx);
    L->X1 = off;    off = up(off + 2 * static_cast<size_t>(batch) * L->R * L->ldx);
    L->A = off;     off = up(off + 2 * static_cast<size_t>(batch) * L->R * L->lda);
    L->B = off;     off = up(off + 2 * static_cast<size_t>(batch) * L->R * L->lda);
    L->total = off;
    return true;
}

// Power of two s such that a matrix of spectral norm `bound` (hence entries of at most that size), stored times s, stays
// below 2^15: fp16 ends at 65504.
double fp16_scale(double bound) { return std::exp2(std::floor(15.0 - std::log2(std::max(bound, 1e-6)))); }

// max of |a s + b s^3 + c s^5| over [0, r]: at an end or where the derivative a + 3 b s^2 + 5 c s^4 vanishes.
double odd_poly_bound(const double* k, double r) {
    auto f = [&](double s) { return std::fabs(s * (k[0] + s * s * (k[1] + s * s * k[2]))); };
    double m = f(r);
    double roots[2] = {-1.0, -1.0};
    if (k[2] != 0.0) {
        const double disc = 9 * k[1] * k[1] - 20 * k[0] * k[2];
        if (disc >= 0) { roots[0] = (-3 * k[1] + std::sqrt(disc)) / (10 * k[2]); roots[1] = (-3 * k[1] - std::sqrt(disc)) / (10 * k[2]); }
    } else if (k[1] != 0.0) {
        roots[0] = -k[0] / (3 * k[1]);
    }
    for (double q : roots) if (q > 0 && q < r * r) m = std::max(m, f(std::sqrt(q)));
    return m;
}
// max of |b l + c l^2| over [0, r^2]
double poly_bound(const double* k, double r) {
    auto f = [&](double l) { return std::fabs(l * (k[1] + l * k[2])); };
    double m = f(r * r);
    if (k[2] != 0.0) { const double q = -k[1] / (2 * k[2]); if (q > 0 && q < r * r) m = std::max(m, f(q)); }
    return m;
}

// Scales and epilogue factors of every product.  X, A and B are stored times sx, sa, sb:
//   GRAM   acc = sx^2 A                     A stored: acc sa / sx^2
//   POLY   acc = sa^2 A A                   B stored: acc c sb / sa^2 + A_stored b sb / sa
//   APPLY  acc = sb sx B X                  X' stored: acc sx' / (sb sx) + X_stored a sx' / sx      (sx' = 1 after the last step)
struct Plan { double scale0; float alpha[3 * MAX_STEPS], beta[3 * MAX_STEPS]; };
bool make_plan(const double* coeffs, int steps, Plan* P) {
    double r = 1.001;                                                       // |X_0|_2 <= |X_0|_F <= 1 up to rounding
    double sx = fp16_scale(r);
    P->scale0 = sx;
    for (int k = 0; k < steps; ++k) {
        const double* c = coeffs ? coeffs + 3 * k : DEFAULT_COEFFS;
        if (!std::isfinite(c[0]) || !std::isfinite(c[1]) || !std::isfinite(c[2])) return false;
        const double sa = fp16_scale(r * r), sb = fp16_scale(poly_bound(c, r * 1.01));
        r = odd_poly_bound(c, r) * 1.02;                                    // 2 %: the roundings of a step
        if (!(r <= MAX_BOUND)) return false;
        const double sn = k + 1 == steps ? 1.0 : fp16_scale(r);
        float *al = P->alpha + 3 * k, *be = P->beta + 3 * k;
        al[GRAM] = static_cast<float>(sa / (sx * sx)); be[GRAM] = 0.f;
        al[POLY] = static_cast<float>(c[2] * sb / (sa * sa)); be[POLY] = static_cast<float>(c[1] * sb / sa);
        al[APPLY] = static_cast<float>(sn / (sb * sx)); be[APPLY] = static_cast<float>(c[0] * sn / sx);
        sx = sn;
    }
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

bool encode(CUtensorMap* map, void* ptr, int rank, const cuuint64_t* dims, const cuuint64_t* strides, const cuuint32_t* box) {
    auto enc = get_encode();
    const cuuint32_t ones[4] = {1, 1, 1, 1};
    return enc && enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank, ptr, dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                      box[0] == 64 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// [batch][rows][ld] fp16, ld a multiple of 64; see Maps.
bool map_operand(CUtensorMap* map, __half* ptr, int64_t batch, int64_t rows, int64_t ld, int box_rows, int box_chunks, int box_elems) {
    const cuuint64_t dims[4] = {64, static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(ld / 64), static_cast<cuuint64_t>(batch)};
    const cuuint64_t strides[3] = {static_cast<cuuint64_t>(2 * ld), 128, static_cast<cuuint64_t>(2 * ld * rows)};
    const cuuint32_t box[4] = {static_cast<cuuint32_t>(box_elems), static_cast<cuuint32_t>(box_rows), static_cast<cuuint32_t>(box_chunks), 1};
    return encode(map, ptr, 4, dims, strides, box);
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

cudaError_t ensure_smem() {
    static std::atomic<bool> done[64];
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
    if (dev >= 0 && dev < 64 && done[dev].load(std::memory_order_acquire)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(muon_products_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, GEMM_SMEM);
    if (e == cudaSuccess && dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
    return e;
}

// Tiles of one matrix in a product.
int64_t tiles_of(int mode, int64_t R, int64_t C, int bn) {
    const int64_t mt = (R + TM - 1) / TM, nj = ((mode == APPLY ? C : R) + bn - 1) / bn;
    return mode == APPLY ? mt * nj : mt * nj - (TM / bn) * (mt * (mt - 1) / 2);
}

// Tile width of a product.  A 256 x 128 step was measured at 494 cycles per 64 of K, a 256 x 256 step at 530.  (What holds the narrow
// one back was not isolated: its products alone are 256 cycles.)  So narrow tiles only pay when they find idle SMs: they then
// cut the tile's epilogue.  Hence the narrowest width whose tiles all run at once, else 256.  A step against one with 256
// throughout: 512 x 512 126 and 172 us, 1024 x 1024 164 and 211, 501 x 1999 162 and 209, 1024 x 4096 255 and 289.
// APPLY's right operand comes in chunks of 64 columns per CTA, so 128 is its least.
int pick_bn(int mode, int64_t batch, int64_t R, int64_t C, int pairs) {
    for (int bn = mode == APPLY ? 128 : 64; bn < TN; bn *= 2)
        if (batch * tiles_of(mode, R, C, bn) <= pairs) return bn;
    return TN;
}

bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

template <typename G, int V> void launch_prep_v(const PrepParams& p, cudaStream_t st) {
    const unsigned nb = static_cast<unsigned>(p.batch);
    muon_momentum_kernel<G, V><<<dim3(p.parts, nb), PREP_THREADS, 0, st>>>(p);
    if (p.rows > p.cols) {
        muon_start_tall_kernel<G, V><<<dim3(p.ldx / 64, (p.R + 63) / 64, nb), PREP_THREADS, 0, st>>>(p);
    } else {
        const int64_t blocks = (static_cast<int64_t>(p.R) * (p.ldx / 8) + PREP_THREADS - 1) / PREP_THREADS;
        const int64_t most = std::max<int64_t>(1, 8 * sm_count() / p.batch);    // eight blocks fit an SM
        muon_start_kernel<G, V><<<dim3(static_cast<unsigned>(std::min(blocks, most)), nb), PREP_THREADS, 0, st>>>(p);
    }
}
template <typename G> void launch_prep(const PrepParams& p, cudaStream_t st) {
    if (p.four) launch_prep_v<G, 4>(p, st);
    else launch_prep_v<G, 1>(p, st);
}

// CTAs that hold a matrix in the one-launch kernel, 0: it does not fit.  Where it fits it is the faster one, at any batch (a step
// in fp32 against the general kernels): 64 x 64 31 and 84 us, 128 x 512 80 and 104, 256 x 256 74 and 102; 64 matrices of 128 x 512
// 83 and 193, 256 of 256 x 256 323 and 496.
int small_cg(int64_t R, int64_t C) {
    if (R <= 128 && C <= SmallShape<1>::MAX_C) return 1;
    return R <= SmallShape<2>::ROWS && C <= SmallShape<2>::MAX_C ? 2 : 0;
}

template <int CG, typename G> cudaError_t launch_small_cg(const GemmParams& q, const PrepParams& pp, cudaStream_t st) {
    static std::atomic<bool> raised[64];
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
    auto kern = muon_small_kernel<CG, G>;
    if (dev < 0 || dev >= 64 || !raised[dev].load(std::memory_order_acquire)) {
        if (cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, SmallShape<CG>::SMEM); e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev].store(true, std::memory_order_release);
    }
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = CG; attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>(CG * q.batch)); cfg.blockDim = dim3(SMALL_THREADS);
    cfg.dynamicSmemBytes = SmallShape<CG>::SMEM; cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, q, pp);
}
template <typename G> cudaError_t launch_small(const GemmParams& q, const PrepParams& pp, int cg, cudaStream_t st) {
    return cg == 1 ? launch_small_cg<1, G>(q, pp, st) : launch_small_cg<2, G>(q, pp, st);
}

struct Target {                                 // what the last product writes
    void* out; int out_dtype;
    float *p; __nv_bfloat16* w; float decay, step;
};

int run(const void* g, int g_dtype, float* m, float mu, int nesterov, int64_t batch, int64_t rows, int64_t cols, const Target& tgt,
        const double* coeffs, int steps, double eps, void* ws, size_t ws_bytes, cudaStream_t st) {
    Layout L;
    if (!layout(batch, rows, cols, &L)) return VPCE_UNSUPPORTED;
    if (!ws) return VPCE_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(ws) & 255u) return VPCE_UNSUPPORTED;
    if (ws_bytes < L.total) return VPCE_WORKSPACE_TOO_SMALL;
    Plan plan;
    if (!make_plan(coeffs, steps, &plan)) return VPCE_UNSUPPORTED;

    char* base = static_cast<char*>(ws);
    GemmParams q{};
    q.batch = static_cast<int>(batch); q.R = static_cast<int>(L.R); q.C = static_cast<int>(L.C);
    q.lda = static_cast<int>(L.lda); q.ldx = static_cast<int>(L.ldx);
    q.X[0] = reinterpret_cast<__half*>(base + L.X0); q.X[1] = reinterpret_cast<__half*>(base + L.X1);
    q.A = reinterpret_cast<__half*>(base + L.A); q.B = reinterpret_cast<__half*>(base + L.B);
    q.transposed = rows > cols;
    q.out = tgt.out; q.out_dtype = tgt.out_dtype; q.p = tgt.p; q.w = tgt.w; q.decay = tgt.decay; q.step = tgt.step;
    q.status = reinterpret_cast<int*>(base); q.next = q.status + 16; q.done = reinterpret_cast<int*>(base + L.done);
    q.wait_limit_ns = static_cast<unsigned long long>(vp_ce_set_wait_limit_ns(0));
    Maps maps;
    PrepParams pp{};
    pp.g = g; pp.m = m; pp.mu = mu; pp.nesterov = nesterov;
    pp.batch = q.batch; pp.rows = rows; pp.cols = cols; pp.parts = static_cast<int>(L.parts);
    pp.sumsq = reinterpret_cast<double*>(base + L.sumsq);
    pp.eps = static_cast<float>(eps); pp.scale = static_cast<float>(plan.scale0);
    pp.X = q.X[0]; pp.R = q.R; pp.C = q.C; pp.ldx = q.ldx; pp.status = q.status; pp.next = q.next; pp.done = q.done;
    // four elements per access where every matrix (and every row, for the start) begins on a boundary of four elements
    pp.four = cols % 4 == 0 && aligned(g, g_dtype == VPCE_F32 ? 16 : 8) && aligned(m, 16);
    q.steps = steps;
    std::copy(plan.alpha, plan.alpha + 3 * steps, q.alpha);
    std::copy(plan.beta, plan.beta + 3 * steps, q.beta);
    const int cg = small_cg(L.R, L.C);
    take_drop(&q, cg ? 1 : 0);
    if (cg) {
        if (batch > 1 && cudaMemsetAsync(q.status, 0, sizeof(int), st) != cudaSuccess) return VPCE_CUDA_ERROR;
        if (cg == 2) q.ldx = static_cast<int>((L.C + 127) / 128 * 128);     // two halves of whole chunks
        const cudaError_t e = g_dtype == VPCE_F32 ? launch_small<float>(q, pp, cg, st)
                              : g_dtype == VPCE_F16 ? launch_small<__half>(q, pp, cg, st) : launch_small<__nv_bfloat16>(q, pp, cg, st);
        return e == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
    }
    const int pairs = sm_count() / 2;
    int64_t most = 0;
    for (int mode = 0; mode < 3; ++mode) {
        q.bn[mode] = pick_bn(mode, batch, L.R, L.C, pairs);
        q.tiles[mode] = static_cast<int>(tiles_of(mode, L.R, L.C, q.bn[mode]));
        most = std::max(most, std::min<int64_t>(pairs, batch * q.tiles[mode]));
    }
    auto map = [&](CUtensorMap* m, __half* ptr, int64_t ld, int box_rows, int box_chunks, int box_elems = 64) {
        return map_operand(m, ptr, batch, L.R, ld, box_rows, box_chunks, box_elems);
    };
    bool ok = map(&maps.a_l, q.A, L.lda, 128, 1) && map(&maps.a_r, q.A, L.lda, q.bn[POLY] / 2, 1) && map(&maps.b_l, q.B, L.lda, 128, 1) &&
              map(&maps.a_blk, q.A, L.lda, 32, 1, 32) && map(&maps.b_blk, q.B, L.lda, 32, 1, 32);
    for (int i = 0; i < 2; ++i)
        ok = ok && map(&maps.x_l[i], q.X[i], L.ldx, 128, 1) && map(&maps.x_r[i], q.X[i], L.ldx, q.bn[GRAM] / 2, 1) &&
             map(&maps.x_mn[i], q.X[i], L.ldx, 64, q.bn[APPLY] / 128) && map(&maps.x_blk[i], q.X[i], L.ldx, 32, 1, 32);
    if (!ok || ensure_smem() != cudaSuccess) return VPCE_CUDA_ERROR;

    if (g_dtype == VPCE_F32) launch_prep<float>(pp, st);
    else if (g_dtype == VPCE_F16) launch_prep<__half>(pp, st);
    else launch_prep<__nv_bfloat16>(pp, st);

    muon_products_kernel<<<2 * static_cast<unsigned>(most), GEMM_THREADS, GEMM_SMEM, st>>>(maps, q);
    return cudaGetLastError() == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

bool known_type(int t) { return t == VPCE_BF16 || t == VPCE_F16 || t == VPCE_F32; }
bool misaligned(const void* p, int dtype) { return reinterpret_cast<uintptr_t>(p) % (dtype == VPCE_F32 ? 4 : 2) != 0; }

}  // namespace

extern "C" {

size_t muon_workspace_bytes(int64_t batch, int64_t rows, int64_t cols) {
    Layout L;
    return layout(batch, rows, cols, &L) ? L.total : 0;
}

int muon_orthogonalize(const void* G, int g_dtype, void* O, int o_dtype, int64_t batch, int64_t rows, int64_t cols,
                       const double* coeffs, int steps, double eps, void* workspace, size_t workspace_bytes, void* stream) {
    if (batch < 0 || rows < 0 || cols < 0 || steps < 1 || steps > MAX_STEPS || !(eps >= 0.0)) return VPCE_INVALID_ARG;
    if (!known_type(g_dtype) || !known_type(o_dtype)) return VPCE_INVALID_ARG;
    if (batch == 0 || rows == 0 || cols == 0) return VPCE_OK;
    if (!G || !O) return VPCE_INVALID_ARG;
    if (misaligned(G, g_dtype) || misaligned(O, o_dtype)) return VPCE_UNSUPPORTED;
    const Target t{O, o_dtype, nullptr, nullptr, 0.f, 0.f};
    return run(G, g_dtype, nullptr, 0.f, 0, batch, rows, cols, t, coeffs, steps, eps, workspace, workspace_bytes,
               static_cast<cudaStream_t>(stream));
}

int muon_step(float* p, float* m, const void* grad, int g_dtype, void* w_bf16, int64_t batch, int64_t rows, int64_t cols, double lr,
              double mu, int nesterov, double weight_decay, double scale, const double* coeffs, int steps, double eps,
              void* workspace, size_t workspace_bytes, void* stream) {
    if (batch < 0 || rows < 0 || cols < 0 || steps < 1 || steps > MAX_STEPS || !(eps >= 0.0) || !(mu >= 0.0 && mu < 1.0) ||
        !std::isfinite(lr) || !std::isfinite(weight_decay) || !std::isfinite(scale))
        return VPCE_INVALID_ARG;
    if (!known_type(g_dtype)) return VPCE_INVALID_ARG;
    if (batch == 0 || rows == 0 || cols == 0) return VPCE_OK;
    if (!p || !m || !grad) return VPCE_INVALID_ARG;
    if (misaligned(p, VPCE_F32) || misaligned(m, VPCE_F32) || misaligned(grad, g_dtype) || misaligned(w_bf16, VPCE_BF16))
        return VPCE_UNSUPPORTED;
    const Target t{nullptr, 0, p, static_cast<__nv_bfloat16*>(w_bf16), static_cast<float>(1.0 - lr * weight_decay),
                   static_cast<float>(lr * scale)};
    return run(grad, g_dtype, m, static_cast<float>(mu), nesterov != 0, batch, rows, cols, t, coeffs, steps, eps, workspace,
               workspace_bytes, static_cast<cudaStream_t>(stream));
}

int muon_debug_drop(int kernel_kind, int index, int cta_ranks) {
    if (kernel_kind < 0) { g_drop.store(-1, std::memory_order_relaxed); return VPCE_OK; }
    if (kernel_kind > 1 || index < 0 || index > 0xffff || cta_ranks <= 0 || cta_ranks > 3) return VPCE_INVALID_ARG;
    g_drop.store(kernel_kind | (index << 8) | (cta_ranks << 24), std::memory_order_relaxed);
    return VPCE_OK;
}

int muon_device_status(const void* workspace, int32_t* status_out, void* stream) {
    if (!workspace || !status_out) return VPCE_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (cudaMemcpyAsync(status_out, workspace, sizeof(int32_t), cudaMemcpyDeviceToHost, st) != cudaSuccess) return VPCE_CUDA_ERROR;
    return cudaStreamSynchronize(st) == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

}  // extern "C"
