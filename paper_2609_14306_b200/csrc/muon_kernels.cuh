// Device code of the Muon update (muon.h): momentum and norm, the scaled fp16 start of the iteration, and one
// tensor-core kernel for its three products.  See muon.cu for the overall description.
#pragma once

#include <cuda_fp16.h>

#include "muon.h"
#include "sm100_ptx.cuh"
#include "vp_ce.h"

namespace vpmuon {

using namespace vpce;

constexpr int TM = 256;                     // rows of a tile: one CTA pair, 128 rows per CTA
constexpr int TN = 256;                     // most columns of a tile; a launch runs 256 or 128
constexpr int KB = 64;                      // K per pipeline stage: one 128-byte swizzle row of fp16
constexpr int BOX_BYTES = 64 * 128;         // one TMA box: 64 rows of 128 bytes
constexpr int A_BYTES = 2 * BOX_BYTES;      // per CTA: its 128 rows of the left operand
constexpr int STAGE_BYTES = 2 * A_BYTES;    // and its half (128 at most) of the right operand's columns
constexpr int STAGES = 6;
constexpr int GEMM_THREADS = 192;           // warp 0 TMA, warp 1 MMA, warps 2..5 epilogue
constexpr int EPI_PITCH = 33;               // floats: a 32 x 32 block per epilogue warp, read back by columns
constexpr int EPI_BYTES = 4 * 32 * EPI_PITCH * 4;
constexpr int GEMM_SMEM = STAGES * STAGE_BYTES + EPI_BYTES + 2048;
constexpr int MAX_STEPS = 32;
constexpr int PREP_THREADS = 256;
constexpr int MAX_PARTS = 512;              // partial sums of squares per matrix

// The three products of a step.
enum Mode { GRAM = 0, POLY = 1, APPLY = 2 };

struct Maps {
    CUtensorMap x_k[2];                     // X (both buffers) read along its rows: K = columns
    CUtensorMap x_mn[2];                    // X as right operand of B X: K = rows
    CUtensorMap a_k, b_k;
};

struct GemmParams {
    int batch, R, C;                        // matrices R x C with R <= C
    int lda, ldx;                           // row pitches (elements, multiples of 64; columns beyond R / C hold zeros)
    int phase;                              // 3 step + mode
    int bn;                                 // 256 or 128
    int tiles;                              // per matrix
    float alpha, beta;                      // stored result = alpha acc + beta addend (stored units)
    __half *X[2], *A, *B;
    // last product: what becomes of X
    int last, transposed;                   // transposed: the user's matrices are C x R
    void* out; int out_dtype;               // muon_orthogonalize
    float* p; __nv_bfloat16* w; float decay, step; // muon_step: p <- p decay - step X
    int* status;
    unsigned long long wait_limit_ns;
};

__device__ __forceinline__ void tma2_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma2_load_3d_plain(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}

// ------------------------------------------------------------------------------------ element types
__device__ __forceinline__ float load_as_float(const void* p, int dtype, size_t i) {
    if (dtype == VPCE_F32) return static_cast<const float*>(p)[i];
    if (dtype == VPCE_F16) return __half2float(static_cast<const __half*>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
__device__ __forceinline__ void store_as(void* p, int dtype, size_t i, float v) {
    if (dtype == VPCE_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == VPCE_F16) static_cast<__half*>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

// ------------------------------------------------------------------------------------ momentum, norm, start
struct PrepParams {
    const void* g; int g_dtype;
    float* m;                               // null: no momentum (U = G)
    float mu; int nesterov;
    int batch; long rows, cols;
    int parts; double* sumsq;               // [batch][parts]
    float eps, scale;                       // X_0 is stored times `scale`
    __half* X; int R, C, ldx;
    int* status;
};

// M <- mu M + G and the sum of squares of U over one part of one matrix: grid (parts, batch).
__global__ void __launch_bounds__(PREP_THREADS) muon_momentum_kernel(const PrepParams p) {
    __shared__ double part[PREP_THREADS / 32];
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *p.status = 0;
    const size_t n = static_cast<size_t>(p.rows) * p.cols;
    const size_t per = (n + p.parts - 1) / p.parts, i0 = blockIdx.x * per, i1 = i0 + per < n ? i0 + per : n;
    const size_t base = blockIdx.y * n;
    double s = 0.0;
    for (size_t i = i0 + threadIdx.x; i < i1; i += PREP_THREADS) {
        const float g = load_as_float(p.g, p.g_dtype, base + i);
        float u = g;
        if (p.m) {
            const float m = p.mu * p.m[base + i] + g;
            p.m[base + i] = m;
            u = p.nesterov ? g + p.mu * m : m;
        }
        s += static_cast<double>(u) * u;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < PREP_THREADS / 32; ++i) s += part[i];
        p.sumsq[static_cast<size_t>(blockIdx.y) * p.parts + blockIdx.x] = s;
    }
}

// X_0 = U / max(|U|_F, eps), stored as fp16 times `scale` in the wide orientation with zeros in the padding columns.
// 64 x 64 blocks through shared memory (the user's matrix may be the transpose): grid (column blocks, row blocks, batch).
__global__ void __launch_bounds__(PREP_THREADS) muon_start_kernel(const PrepParams p) {
    __shared__ float blk[64][65];
    __shared__ float inv_s;
    const bool tall = p.rows > p.cols;
    if (threadIdx.x < 32) {
        double s = 0.0;
        for (int i = threadIdx.x; i < p.parts; i += 32) s += p.sumsq[static_cast<size_t>(blockIdx.z) * p.parts + i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (threadIdx.x == 0) {
            const float norm = static_cast<float>(sqrt(s));
            inv_s = p.scale / (norm < p.eps ? p.eps : norm);                // NaN stays NaN
        }
    }
    // the user's block: rows r0.., columns c0.. of [rows, cols]
    const long x0 = static_cast<long>(blockIdx.x) * 64, y0 = static_cast<long>(blockIdx.y) * 64;   // of X: columns, rows
    const long r0 = tall ? x0 : y0, c0 = tall ? y0 : x0;
    const size_t base = static_cast<size_t>(blockIdx.z) * p.rows * p.cols;
    for (int k = threadIdx.x; k < 64 * 64; k += PREP_THREADS) {
        const int r = k >> 6, c = k & 63;
        float u = 0.f;
        if (r0 + r < p.rows && c0 + c < p.cols) {
            const size_t i = base + static_cast<size_t>(r0 + r) * p.cols + (c0 + c);
            u = load_as_float(p.g, p.g_dtype, i);
            if (p.m) u = p.nesterov ? u + p.mu * p.m[i] : p.m[i];
        }
        blk[r][c] = u;
    }
    __syncthreads();
    const float inv = inv_s;
    for (int k = threadIdx.x; k < 64 * 32; k += PREP_THREADS) {
        const int y = k >> 5, x = (k & 31) * 2;
        if (y0 + y >= p.R) continue;
        const float a = (tall ? blk[x][y] : blk[y][x]) * inv, b = (tall ? blk[x + 1][y] : blk[y][x + 1]) * inv;
        // ldx is a multiple of 64: the whole block lies inside the row; U is 0 beyond the matrix
        const __half2 h = __floats2half2_rn(x0 + x < p.C ? a : 0.f, x0 + x + 1 < p.C ? b : 0.f);
        *reinterpret_cast<__half2*>(p.X + (static_cast<size_t>(blockIdx.z) * p.R + y0 + y) * p.ldx + x0 + x) = h;
    }
}

// ------------------------------------------------------------------------------------ the products
struct Tile { int b, i, j; };               // matrix, row tile (256), column tile (bn)

// GRAM and POLY are symmetric: only the tiles that reach the diagonal or lie right of it are listed (the others are
// written as mirror images).  A row of tiles i starts at column tile i * 256 / bn.
__device__ __forceinline__ Tile decode(const GemmParams& p, int t) {
    Tile w;
    w.b = t / p.tiles;
    int r = t - w.b * p.tiles;
    if (p.phase % 3 == APPLY) {
        const int nj = (p.C + p.bn - 1) / p.bn;
        w.i = r / nj;
        w.j = r - w.i * nj;
    } else {
        const int nj = (p.R + p.bn - 1) / p.bn, f = TM / p.bn;
        w.i = 0;
        while (r >= nj - w.i * f) { r -= nj - w.i * f; ++w.i; }
        w.j = w.i * f + r;
    }
    return w;
}

// Whether the tile that holds element (row, col) is listed in a symmetric product.
__device__ __forceinline__ bool listed(const GemmParams& p, int row, int col) { return (col / p.bn + 1) * p.bn > (row / TM) * TM; }

__device__ __forceinline__ void unpack8(uint4 q, float* f) {
    const __half2* h = reinterpret_cast<const __half2*>(&q);
#pragma unroll
    for (int i = 0; i < 4; ++i) { const float2 t = __half22float2(h[i]); f[2 * i] = t.x; f[2 * i + 1] = t.y; }
}
__device__ __forceinline__ uint4 pack8(const float* f) {
    uint4 q;
    __half2* h = reinterpret_cast<__half2*>(&q);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    return q;
}

// One warp's 32 x 32 block of the accumulator: result rows row0 + lane, columns col0 .. col0 + 31.
__device__ __forceinline__ void epilogue_block(const GemmParams& p, int b, int row0, int col0, int lane, float* v, float* stage) {
    const int mode = p.phase % 3, row = row0 + lane;
    const int ld = mode == APPLY ? p.ldx : p.lda;
    const size_t at = (static_cast<size_t>(b) * p.R + row) * ld + col0;
    if (mode == GRAM) {
#pragma unroll
        for (int j = 0; j < 32; ++j) v[j] *= p.alpha;
    } else {
        const __half* add = (mode == POLY ? p.A : p.X[(p.phase / 3) & 1]) + at;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (row < p.R) unpack8(__ldcg(reinterpret_cast<const uint4*>(add) + q), f);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[8 * q + j] = p.alpha * v[8 * q + j] + p.beta * f[j];
        }
    }
    if (mode == APPLY && p.last) {
        // to the caller's arrays: coalesced along their rows, through a transpose in shared memory where X's rows are theirs
        const size_t base = static_cast<size_t>(b) * p.R * p.C;
        if (!p.transposed) {
#pragma unroll
            for (int j = 0; j < 32; ++j) stage[lane * EPI_PITCH + j] = v[j];
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 32; ++j) v[j] = stage[j * EPI_PITCH + lane];   // now row row0 + j, column col0 + lane
            __syncwarp();
        }
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const int r = p.transposed ? row : row0 + j, c = p.transposed ? col0 + j : col0 + lane;
            if (r < p.R && c < p.C) {
                const size_t i = base + (p.transposed ? static_cast<size_t>(c) * p.R + r : static_cast<size_t>(r) * p.C + c);
                if (p.p) {
                    const float n = p.p[i] * p.decay - p.step * v[j];
                    p.p[i] = n;
                    if (p.w) p.w[i] = __float2bfloat16_rn(n);
                } else {
                    store_as(p.out, p.out_dtype, i, v[j]);
                }
            }
        }
        return;
    }
    __half* out = mode == GRAM ? p.A : mode == POLY ? p.B : p.X[((p.phase / 3) & 1) ^ 1];
    if (row < p.R) {
#pragma unroll
        for (int q = 0; q < 4; ++q) reinterpret_cast<uint4*>(out + at)[q] = pack8(v + 8 * q);
    }
    if (mode != APPLY && !listed(p, col0, row0)) {                          // the mirror image: row col0 + j, column `row`
#pragma unroll
        for (int j = 0; j < 32; ++j)
            if (col0 + j < p.R && row < p.lda) out[(static_cast<size_t>(b) * p.R + col0 + j) * ld + row] = __float2half_rn(v[j]);
    }
}

// One product for the whole batch on CTA pairs (tcgen05 cta_group::2, 256 x bn tiles, fp32 accumulators in tensor memory,
// two of them so that a tile's epilogue overlaps the next tile's products).
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GEMM_THREADS, 1)
muon_gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ GemmParams p) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw);
    const uint32_t base = (raw + 1023u) & ~1023u;                          // swizzle atoms need 1024-byte alignment
    uint8_t* smem = smem_raw + (base - raw);
    const uint32_t bars = base + STAGES * STAGE_BYTES;
    auto full_bar = [&](int s) { return bars + 8u * s; };                    // the leader's is used
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto tfull_bar = [&](int a) { return bars + 8u * (2 * STAGES + a); };
    auto tempty_bar = [&](int a) { return bars + 8u * (2 * STAGES + 2 + a); };   // the leader's is used
    const uint32_t drain_bar = bars + 8u * (2 * STAGES + 4);
    constexpr int NUM_BARS = 2 * STAGES + 5;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + STAGES * STAGE_BYTES + 8 * NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    float* epi = reinterpret_cast<float*>(smem + STAGES * STAGE_BYTES + 256);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const int pair = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    const int total = p.tiles * p.batch;
    const int mode = p.phase % 3, xb = (p.phase / 3) & 1;
    const int num_kb = (mode == GRAM ? p.ldx : p.lda) / KB;
    const int b_boxes = p.bn / 128;                                          // boxes of 64 columns in this CTA's half of a tile

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 8); }
        mbar_init(drain_bar, 1);
        fence_barrier_init();
        fence_proxy_async();
    }
    if (warp == 1) {
        tmem2_alloc(smem_u32(tmem_slot), 512);
        tmem2_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                                                      // the peer's barriers exist before any remote signal
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        if (lane == 0) {
            const CUtensorMap* ma = mode == GRAM ? &maps.x_k[xb] : mode == POLY ? &maps.a_k : &maps.b_k;
            const CUtensorMap* mb = mode == GRAM ? &maps.x_k[xb] : mode == POLY ? &maps.a_k : &maps.x_mn[xb];
            int stage = 0; uint32_t phase = 0; bool ok = true;
            long issued = 0;
            for (int t = pair; t < total && ok; t += pairs) {
                const Tile w = decode(p, t);
                const int arow = w.i * TM + static_cast<int>(rank) * 128;
                const int bcol = w.j * p.bn + static_cast<int>(rank) * (p.bn / 2);
                for (int kb = 0; kb < num_kb; ++kb) {
                    if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    if (leader) mbar_arrive_expect_tx(full_bar(stage), 2 * (A_BYTES + b_boxes * BOX_BYTES));
                    const uint32_t bar = mapa_shared(full_bar(stage), 0);
                    const uint32_t sa = base + stage * STAGE_BYTES, sb = sa + A_BYTES;
                    // rows beyond the matrix arrive as zeros
                    tma2_load_3d_plain(sa, ma, bar, kb * KB, arow, w.b);
                    tma2_load_3d_plain(sa + BOX_BYTES, ma, bar, kb * KB, arow + 64, w.b);
                    for (int q = 0; q < b_boxes; ++q) {
                        if (mode == APPLY) tma2_load_4d(sb + q * BOX_BYTES, mb, bar, 0, kb * KB, bcol / 64 + q, w.b);
                        else tma2_load_3d_plain(sb + q * BOX_BYTES, mb, bar, kb * KB, bcol + 64 * q, w.b);
                    }
                    ++issued;
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if ((!ok || *abort_flag) && leader) {
                // give-up path (the leader's barriers count both CTAs' bytes): let copies in flight land
                const long back = issued < STAGES ? issued : STAGES;
                int s = stage; uint32_t ph = phase;
                for (long i = 0; i < back; ++i) {
                    if (--s < 0) { s = STAGES - 1; ph ^= 1u; }
                    const unsigned long long t0 = globaltimer_ns();
                    while (!mbar_try_wait(full_bar(s), ph) && globaltimer_ns() - t0 < p.wait_limit_ns) {}
                }
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && leader) {
            const uint32_t idesc = make_idesc(p.bn, false, mode == APPLY, TM, 0u);    // fp16 operands
            int stage = 0; uint32_t phase = 0; bool ok = true;
            int it = 0;
            for (int t = pair; t < total && ok; t += pairs, ++it) {
                const int ab = it & 1;
                if (!mbar_wait_cluster(tempty_bar(ab), ((it >> 1) & 1u) ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                tc_fence_after();
                const uint32_t tmem_d = tmem_base + ab * TN;
                for (int kb = 0; kb < num_kb; ++kb) {
                    if (!mbar_wait(full_bar(stage), phase, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = base + stage * STAGE_BYTES, sb = sa + A_BYTES;
                    const uint64_t adesc = make_smem_desc(sa, 16, 1024);
                    const uint64_t bdesc = mode == APPLY ? make_smem_desc(sb, BOX_BYTES, 1024) : make_smem_desc(sb, 16, 1024);
#pragma unroll
                    for (int k = 0; k < KB / 16; ++k) {
                        // K-major: 16 elements = 32 bytes along the swizzled row; MN-major: 16 rows of 128 bytes
                        const uint64_t boff = static_cast<uint64_t>((mode == APPLY ? k * 16 * 128 : k * 32) >> 4);
                        umma2_f16(tmem_d, adesc + static_cast<uint64_t>((k * 32) >> 4), bdesc + boff, idesc, (kb | k) != 0 ? 1u : 0u);
                    }
                    umma2_commit_both(empty_bar(stage));
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
                if (ok) umma2_commit_both(tfull_bar(ab));
            }
            if (!ok || *abort_flag) {
                umma2_commit_local(drain_bar);
                const unsigned long long t0 = globaltimer_ns();
                while (!mbar_try_wait(drain_bar, 0) && globaltimer_ns() - t0 < p.wait_limit_ns) {}
            }
        }
    } else {
        const int quad = warp & 3;
        float* stage = epi + (warp - 2) * 32 * EPI_PITCH;
        int it = 0;
        for (int t = pair; t < total; t += pairs, ++it) {
            const Tile w = decode(p, t);
            const int ab = it & 1;
            const bool ok = mbar_wait(tfull_bar(ab), (it >> 1) & 1u, abort_flag, p.wait_limit_ns);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const uint32_t tmem_row = tmem_base + ab * TN + (static_cast<uint32_t>(quad * 32) << 16);
            const int row0 = w.i * TM + static_cast<int>(rank) * 128 + quad * 32;
            const int ncols = mode == APPLY ? p.ldx : p.lda;
            for (int c = 0; c < p.bn / 32; ++c) {
                const int col0 = w.j * p.bn + c * 32;
                if (row0 >= p.R || col0 >= ncols) break;                     // uniform in the warp
                float v[32];
                __syncwarp();
                tmem_ld32(tmem_row + c * 32, v);
                tmem_ld_wait();
                epilogue_block(p, w.b, row0, col0, lane, v, stage);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_shared(tempty_bar(ab), 0));
        }
    }

    tc_fence_before();
    __syncthreads();
    cluster_sync_all();                          // no CTA leaves while its pair may still signal it or read its memory
    if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, VPCE_DEV_WAIT_EXPIRED);
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem2_dealloc(tmem_base, 512);
    }
}

}  // namespace vpmuon
