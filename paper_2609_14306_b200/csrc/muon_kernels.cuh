// Device code of the Muon update (muon.h): momentum and norm, the scaled fp16 start of the iteration, and one
// tensor-core kernel for its three products.  See muon.cu for the overall description.
#pragma once

#include <cuda_fp16.h>

#include "muon.h"
#include "sm100_ptx.cuh"
#include "vp_ce.h"

namespace vpmuon {

using namespace vpce;

constexpr int TM = 256, TN = 256;           // a tile: one CTA pair, 128 rows and bn / 2 columns' worth of operands per CTA; bn <= TN
constexpr int KB = 64;                      // K per pipeline stage: one 128-byte swizzle row of fp16
constexpr int A_BYTES = 128 * 128;          // 128 rows of the left operand
constexpr int STAGE_BYTES = 2 * A_BYTES;
constexpr int STAGES = 5;
constexpr int EPI_WARPS = 8;                // two per quarter of the tensor memory's lanes, each every other 32 columns
constexpr int GEMM_THREADS = 64 + 32 * EPI_WARPS;   // warp 0 TMA, warp 1 MMA, the others epilogue
constexpr int BLOCK_BYTES = 32 * 64;        // a 32 x 32 block of fp16: 64-byte rows, 64-byte swizzle
constexpr int WARP_BLOCKS = TN / 32 / 2;    // blocks of one warp in a tile
constexpr int EPI_WARP_BYTES = WARP_BLOCKS * BLOCK_BYTES;   // see the epilogue
constexpr int EPI_BYTES = EPI_WARPS * EPI_WARP_BYTES;
constexpr int GEMM_SMEM = STAGES * STAGE_BYTES + EPI_BYTES + 2048;   // barriers (1024) and alignment slack
static_assert(GEMM_SMEM <= 227 * 1024, "shared memory per CTA");
constexpr int MAX_STEPS = 32;
constexpr int DONE_PITCH = 32;              // a counter has a line of its own: its matrix's CTAs poll it
constexpr int PREP_THREADS = 256;
constexpr int MAX_PARTS = 512;              // partial sums of squares per matrix

// The three products of a step.
enum Mode { GRAM = 0, POLY = 1, APPLY = 2 };

// Operands as 4-D arrays {64 elements, rows, 64-element chunks of a row, batch}.  Along the rows (K = columns) a stage takes one
// box of 128 rows x 1 chunk (left operand) or bn / 2 rows x 1 chunk (right, *_r), down the columns (X as right operand of B X,
// K = rows) one of 64 rows x bn / 128 chunks.  The chunk as a
// dimension of its own matters: boxes at column offsets of a 3-D array {columns, rows, batch} arrived at 48 bytes a cycle and
// SM, these at 70 (loads alone, 128-row boxes; the products need 64).
// The epilogue moves boxes of 32 rows x 32 elements of the same arrays (*_blk).
struct Maps { CUtensorMap x_l[2], x_r[2], x_mn[2], a_l, a_r, b_l, x_blk[2], a_blk, b_blk; };

struct GemmParams {
    int batch, R, C;                        // matrices R x C with R <= C
    int lda, ldx;                           // row pitches (elements, multiples of 64; columns beyond R / C hold zeros)
    int steps;
    int bn[3], tiles[3];                    // per mode: tile width (256, 128, 64), tiles of one matrix
    float alpha[3 * MAX_STEPS], beta[3 * MAX_STEPS];   // stored result = alpha acc + beta addend (stored units)
    __half *X[2], *A, *B;
    // last product: what becomes of X
    int transposed;                         // the user's matrices are C x R
    void* out; int out_dtype;               // muon_orthogonalize
    float* p; __nv_bfloat16* w; float decay, step; // muon_step: p <- p decay - step X
    int *status, *next;                     // next: work-list position to be taken, zero before the launch
    int* done;                              // [batch][DONE_PITCH] epilogue warps that have finished a tile of this matrix, zero before the launch
    unsigned long long wait_limit_ns;
    int drop, drop_ranks;                   // test hook (muon_debug_drop): the k-block or product that is lost, -1: none
};

__device__ __forceinline__ void tma2_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_store_4d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(src), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
// 32 lanes x 16 consecutive fp32 columns of tensor memory.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}
__device__ __forceinline__ void bulk_wait_read_all() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ uint4 ld_shared_v4(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float ld_shared_f32(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void st_shared_f32(uint32_t addr, float v) {
    asm volatile("st.shared.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}
__device__ __forceinline__ void st_shared_b16(uint32_t addr, uint16_t v) {
    asm volatile("st.shared.b16 [%0], %1;" ::"r"(addr), "h"(v) : "memory");
}

// ------------------------------------------------------------------------------------ element types
__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
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

// ------------------------------------------------------------------------------------ momentum, norm, start
struct PrepParams {
    const void* g;
    float* m;                               // null: no momentum (U = G)
    float mu; int nesterov;
    int batch; long rows, cols;
    int parts; double* sumsq;               // [batch][parts]
    float eps, scale;                       // X_0 is stored times `scale`
    int four;                               // four elements per access: see the host
    __half* X; int R, C, ldx;
    int *status, *next, *done;
};

// Four consecutive elements (one load of 16 or 8 bytes) or one.
template <typename G, int V>
__device__ __forceinline__ void load_v(const G* p, float* f) {
    if constexpr (V == 1) {
        f[0] = to_float(*p);
    } else if constexpr (sizeof(G) == 4) {
        const float4 q = *reinterpret_cast<const float4*>(p);
        f[0] = q.x; f[1] = q.y; f[2] = q.z; f[3] = q.w;
    } else {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        const G* h = reinterpret_cast<const G*>(&q);
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = to_float(h[i]);
    }
}
template <int V> __device__ __forceinline__ void store_v(float* p, const float* f) {
    if constexpr (V == 1) *p = f[0];
    else *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
}

// M <- mu M + G and the sum of squares of U over one part of one matrix: grid (parts, batch).  V: elements per access, 4
// where every matrix starts on a 16-byte boundary.  Each thread has UNROLL accesses in flight.  Bound: memory; four 2880 x 2880
// matrices with bf16 gradients take 49 us (332 MB: 6.7 TB/s).
template <typename G, int V>
__global__ void __launch_bounds__(PREP_THREADS) muon_momentum_kernel(const PrepParams p) {
    constexpr int UNROLL = V == 4 ? 4 : 8;
    __shared__ double part[PREP_THREADS / 32];
    if (blockIdx.x == 0 && threadIdx.x == 0) {                              // the products' bookkeeping starts at zero
        p.done[blockIdx.y * DONE_PITCH] = 0;
        if (blockIdx.y == 0) { *p.status = 0; *p.next = 0; }
    }
    const long n = p.rows * p.cols / V;                                     // accesses of a matrix
    const long per = (n + p.parts - 1) / p.parts, i0 = blockIdx.x * per, i1 = i0 + per < n ? i0 + per : n;
    const G* g = static_cast<const G*>(p.g) + static_cast<size_t>(blockIdx.y) * p.rows * p.cols;
    float* m = p.m ? p.m + static_cast<size_t>(blockIdx.y) * p.rows * p.cols : nullptr;
    double s = 0.0;
    for (long i = i0 + threadIdx.x; i < i1; i += UNROLL * PREP_THREADS) {
        float gv[UNROLL][V], mv[UNROLL][V];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const long at = i + k * PREP_THREADS;
            if (at < i1) {
                load_v<G, V>(g + at * V, gv[k]);
                if (m) load_v<float, V>(m + at * V, mv[k]);
            }
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const long at = i + k * PREP_THREADS;
            if (at < i1) {
                float q = 0.f;
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    float u = gv[k][j];
                    if (m) {
                        mv[k][j] = p.mu * mv[k][j] + u;
                        u = p.nesterov ? u + p.mu * mv[k][j] : mv[k][j];
                    }
                    q += u * u;
                }
                s += q;
                if (m) store_v<V>(m + at * V, mv[k]);
            }
        }
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

// scale / max(|U|_F, eps) of matrix b, by every block that needs it (the parts in a fixed order).
__device__ __forceinline__ float start_factor(const PrepParams& p, int b) {
    __shared__ float inv_s;
    if (threadIdx.x < 32) {
        double s = 0.0;
        for (int i = threadIdx.x; i < p.parts; i += 32) s += p.sumsq[static_cast<size_t>(b) * p.parts + i];
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (threadIdx.x == 0) {
            const float norm = static_cast<float>(sqrt(s));
            inv_s = p.scale / (norm < p.eps ? p.eps : norm);                // NaN stays NaN
        }
    }
    __syncthreads();
    return inv_s;
}

template <typename G, int V>
__device__ __forceinline__ void load_u(const PrepParams& p, size_t at, float* u) {
    load_v<G, V>(static_cast<const G*>(p.g) + at, u);
    if (p.m) {
        float m[V];
        load_v<float, V>(p.m + at, m);
#pragma unroll
        for (int j = 0; j < V; ++j) u[j] = p.nesterov ? u[j] + p.mu * m[j] : m[j];
    }
}

// X_0 = U / max(|U|_F, eps), stored as fp16 times `scale` with zeros in the padding columns, where the user's matrices are
// wide already: grid (blocks, batch), eight columns a thread.  Four 2880 x 2880 with momentum: 41 us (265 MB: 6.5 TB/s).
template <typename G, int V>
__global__ void __launch_bounds__(PREP_THREADS) muon_start_kernel(const PrepParams p) {
    const float inv = start_factor(p, blockIdx.y);
    const size_t base = static_cast<size_t>(blockIdx.y) * p.rows * p.cols;
    const int chunks = p.ldx / 8;
    const long n = static_cast<long>(p.R) * chunks;
    for (long k = static_cast<long>(blockIdx.x) * PREP_THREADS + threadIdx.x; k < n; k += static_cast<long>(gridDim.x) * PREP_THREADS) {
        const long r = k / chunks;
        const int c = static_cast<int>(k - r * chunks) * 8;
        float u[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; j += V)
            if (c + j < p.C) load_u<G, V>(p, base + r * p.C + c + j, u + j);
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] *= inv;
        *reinterpret_cast<uint4*>(p.X + (static_cast<size_t>(blockIdx.y) * p.R + r) * p.ldx + c) = pack8(u);
    }
}

// The same where they are tall: 64 x 64 blocks pass through shared memory.  Grid (column blocks of X, row blocks, batch).
template <typename G, int V>
__global__ void __launch_bounds__(PREP_THREADS) muon_start_tall_kernel(const PrepParams p) {
    __shared__ float blk[64][65];                                           // [column of X][row of X]
    const float inv = start_factor(p, blockIdx.z);
    const long x0 = static_cast<long>(blockIdx.x) * 64, y0 = static_cast<long>(blockIdx.y) * 64;
    const size_t base = static_cast<size_t>(blockIdx.z) * p.rows * p.cols;
#pragma unroll
    for (int q = 0; q < 64 * 64 / V / PREP_THREADS; ++q) {
        const int k = q * PREP_THREADS + threadIdx.x, x = k / (64 / V), y = k % (64 / V) * V;
        float u[V] = {};
        if (x0 + x < p.rows && y0 + y < p.cols) load_u<G, V>(p, base + (x0 + x) * p.cols + y0 + y, u);
#pragma unroll
        for (int j = 0; j < V; ++j) blk[x][y + j] = u[j];
    }
    __syncthreads();
    for (int k = threadIdx.x; k < 64 * 8; k += PREP_THREADS) {
        const int y = k >> 3, x = (k & 7) * 8;
        if (y0 + y >= p.R) continue;
        float u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = blk[x + j][y] * inv;             // columns beyond the matrix hold zeros
        *reinterpret_cast<uint4*>(p.X + (static_cast<size_t>(blockIdx.z) * p.R + y0 + y) * p.ldx + x0 + x) = pack8(u);
    }
}

// ------------------------------------------------------------------------------------ the products
// Entry of the work list: the tiles of every product of every matrix, product by product, inside a product matrix by matrix.
struct Tile {
    int k, mode, b, i, j;                   // product number 3 step + mode, matrix, row tile, column tile (bn wide)
    int bn, need;                         // need: value of done[b] from which on this product's inputs are complete
    bool last;
};

// GRAM and POLY are symmetric: only the tiles that reach the diagonal or lie right of it are listed (the others are written as
// mirror images).  A row of tiles i starts at column tile i * 256 / bn.
__device__ __forceinline__ Tile decode(const GemmParams& p, int e) {
    Tile w;
    const int per_step = p.tiles[0] + p.tiles[1] + p.tiles[2];
    const int step = e / (per_step * p.batch);
    int r = e - step * per_step * p.batch;
    w.mode = 0;
    int before = step * per_step;                                           // tiles of the matrix in earlier products
    while (r >= p.tiles[w.mode] * p.batch) { r -= p.tiles[w.mode] * p.batch; before += p.tiles[w.mode]; ++w.mode; }
    w.k = 3 * step + w.mode;
    w.last = w.k + 1 == 3 * p.steps;
    w.need = before * 2 * EPI_WARPS;
    w.b = r / p.tiles[w.mode];
    r -= w.b * p.tiles[w.mode];
    w.bn = p.bn[w.mode];
    const int nj = ((w.mode == APPLY ? p.C : p.R) + w.bn - 1) / w.bn, f = TM / w.bn;
    if (w.mode == APPLY) {
        w.i = r / nj;
        w.j = r - w.i * nj;
    } else {
        w.i = 0;
        while (r >= nj - w.i * f) { r -= nj - w.i * f; ++w.i; }
        w.j = w.i * f + r;
    }
    return w;
}

// Whether the tile that holds element (row, col) is listed in a symmetric product with tiles bn wide.
__device__ __forceinline__ bool listed(int bn, int row, int col) { return (col / bn + 1) * bn > (row / TM) * TM; }

// Adds to a counter once this lane's TMA stores have been performed, for whoever loads the written data after seeing the new
// value (the fences order the copies of the async proxy and the counter on both sides).
__device__ __forceinline__ void signal_stored(int* counter) {
    bulk_wait_all();
    asm volatile("fence.proxy.async;" ::: "memory");
    asm volatile("red.release.gpu.global.add.s32 [%0], 1;" ::"l"(counter) : "memory");
}

// A CTA's producer polls `done` in global memory for all of its CTA; the epilogue warps learn of it here (list positions rise).
__device__ __forceinline__ void store_ready(uint32_t addr, int t) { asm volatile("st.release.cta.shared::cta.s32 [%0], %1;" ::"r"(addr), "r"(t) : "memory"); }
__device__ __forceinline__ bool wait_ready(uint32_t addr, int t, volatile int* abort_flag, unsigned long long limit_ns) {
    unsigned long long t0 = 0;
    for (uint32_t it = 0;; ++it) {
        int v;
        asm volatile("ld.acquire.cta.shared::cta.s32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
        if (v >= t) {
            asm volatile("fence.proxy.async;" ::: "memory");
            return true;
        }
        if ((it & 63u) == 63u) {
            if (*abort_flag) return false;
            const unsigned long long now = globaltimer_ns();
            if (t0 == 0) t0 = now;
            else if (now - t0 > limit_ns) { *abort_flag = 1; return false; }
        }
        __nanosleep(32);
    }
}

__device__ __forceinline__ int steps_of_k(const GemmParams& p, const Tile& w) { return ((w.mode == GRAM ? p.ldx : p.lda) + KB - 1) / KB; }

// Byte offset of 16-byte chunk c (8 halves) of row r in a 64-byte-swizzled block.
__device__ __forceinline__ uint32_t block_at(int r, int c) { return static_cast<uint32_t>(r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); }

// One warp's 32 x 32 block of the accumulator (result rows row0 + lane, columns col0 ..): the addend lies in `blk`, the result
// takes its place and leaves by TMA store, as does its mirror image through `mir`.
__device__ __forceinline__ void epilogue_block(const GemmParams& p, const Maps& maps, const Tile& w, int row0, int col0, int lane,
                                               float* v, uint32_t blk, uint32_t mir) {
    const float alpha = p.alpha[w.k], beta = p.beta[w.k];
    uint4 h[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (w.mode != GRAM) unpack8(ld_shared_v4(blk + block_at(lane, q)), f);
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = alpha * v[8 * q + j] + beta * f[j];
        h[q] = pack8(f);
        st_shared_v4(blk + block_at(lane, q), h[q]);
    }
    const bool mirror = w.mode != APPLY && col0 < p.R && !listed(w.bn, col0, row0);
    if (mirror) {
        const uint16_t* hv = reinterpret_cast<const uint16_t*>(h);
#pragma unroll
        for (int j = 0; j < 32; ++j) st_shared_b16(mir + block_at(j, lane >> 3) + (lane & 7) * 2, hv[j]);
    }
    fence_proxy_async();
    __syncwarp();
    if (lane == 0) {
        const CUtensorMap* out = w.mode == GRAM ? &maps.a_blk : w.mode == POLY ? &maps.b_blk : &maps.x_blk[((w.k / 3) & 1) ^ 1];
        tma_store_4d(out, blk, col0 & 63, row0, col0 >> 6, w.b);
        if (mirror) tma_store_4d(out, mir, row0 & 63, col0, row0 >> 6, w.b);
        bulk_commit();
    }
}

// N columns (16 or 32) of one warp's rows of the last product, to the caller's arrays: coalesced along their rows.  Where those
// are X's columns (TRANSPOSED) a lane keeps its row of X and element i is column col0 + i; else 16 columns at a time pass through
// 2 KB of shared memory (`scratch`) and element i is row row0 + 2 (i % 16) + lane / 16, column col0 + 16 (i / 16) + lane % 16.
// addend(q, f): eight elements of this lane's row of X, from column col0 + 8 q (read before `scratch`, which may be their place,
// is written).  All loads are issued before the stores (p could alias itself for all the compiler knows): one memory latency for
// N elements.  Nothing here is used again soon: evict-first, so that the operands stay in the L2.
template <int N, bool TRANSPOSED, typename Addend>
__device__ __forceinline__ void epilogue_last(const GemmParams& p, int k, int b, int row0, int col0, int lane, uint32_t tmem, uint32_t scratch,
                                              Addend addend) {
    const int r = row0 + (TRANSPOSED ? lane : lane >> 4), c = col0 + (TRANSPOSED ? 0 : lane & 15);
    const long at = static_cast<long>(b) * p.R * p.C + (TRANSPOSED ? static_cast<long>(c) * p.R + r : static_cast<long>(r) * p.C + c);
    const int pitch = TRANSPOSED ? p.R : 2 * p.C;
    auto offset = [&](int i) { return TRANSPOSED ? i * pitch : (i & 15) * pitch + (i & 16); };
    auto inside = [&](int i) { return TRANSPOSED ? r < p.R && c + i < p.C : r + 2 * (i & 15) < p.R && c + (i & 16) < p.C; };
    float old[N];
    if (p.p) {
#pragma unroll
        for (int i = 0; i < N; ++i) old[i] = inside(i) ? __ldcs(p.p + at + offset(i)) : 0.f;
    }
    float v[N];
    __syncwarp();
    if constexpr (N == 32) tmem_ld32(tmem, v);
    else tmem_ld16(tmem, v);
    tmem_ld_wait();
    const float alpha = p.alpha[k], beta = p.beta[k];
#pragma unroll
    for (int q = 0; q < N / 8; ++q) {
        float f[8];
        addend(q, f);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[8 * q + j] = alpha * v[8 * q + j] + beta * f[j];
    }
    if (!TRANSPOSED) {
        // element (row, j) of 16 columns at word 16 row + (j ^ row % 16): no bank is hit more than twice
#pragma unroll
        for (int h = 0; h < N / 16; ++h) {
            __syncwarp();
#pragma unroll
            for (int j = 0; j < 16; ++j) st_shared_f32(scratch + 4 * (16 * lane + (j ^ (lane & 15))), v[16 * h + j]);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int row = 2 * i + (lane >> 4);
                v[16 * h + i] = ld_shared_f32(scratch + 4 * (16 * row + ((lane & 15) ^ (row & 15))));
            }
        }
    }
    if (p.p) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = old[i] * p.decay - p.step * v[i];
            if (inside(i)) __stcs(p.p + at + offset(i), v[i]);
        }
        if (p.w) {
            unsigned short* wp = reinterpret_cast<unsigned short*>(p.w) + at;
#pragma unroll
            for (int i = 0; i < N; ++i) if (inside(i)) __stcs(wp + offset(i), __bfloat16_as_ushort(__float2bfloat16_rn(v[i])));
        }
    } else if (p.out_dtype == VPCE_F32) {
#pragma unroll
        for (int i = 0; i < N; ++i) if (inside(i)) __stcs(static_cast<float*>(p.out) + at + offset(i), v[i]);
    } else {
        unsigned short* o = static_cast<unsigned short*>(p.out) + at;
        const bool f16 = p.out_dtype == VPCE_F16;
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (inside(i)) __stcs(o + offset(i), f16 ? __half_as_ushort(__float2half_rn(v[i])) : __bfloat16_as_ushort(__float2bfloat16_rn(v[i])));
    }
}

// All products of all matrices in one launch, on CTA pairs (tcgen05 cta_group::2, 256 x bn tiles, fp32 accumulators in tensor
// memory, two of them so that a tile's epilogue overlaps the next tile's products).
//
// Pairs take the entries of the work list in order from a counter.  An entry whose inputs other pairs are still writing waits
// for its matrix's `done` count; an entry only ever waits for entries before it in the list, which running pairs hold, so
// there is always one that can finish, however many pairs the GPU runs at a time.
// Bound: tensor cores where matrices are large (four 2880 x 2880, 15 products: 1.67 ms, 2.27e12 operations with the padding to
// tiles, 1.36 PFLOP/s, tensor pipe 78 % busy); the chain of dependent products where they are not (8 to 15 us each).
constexpr int SCHED_DEPTH = 4;

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GEMM_THREADS, 1)
muon_products_kernel(const __grid_constant__ Maps maps, const __grid_constant__ GemmParams p) {
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
    auto sfull_bar = [&](int s) { return bars + 8u * (2 * STAGES + 5 + s); };
    auto sempty_bar = [&](int s) { return bars + 8u * (2 * STAGES + 5 + SCHED_DEPTH + s); };   // the leader's is used
    auto add_bar = [&](int q) { return bars + 8u * (2 * STAGES + 5 + 2 * SCHED_DEPTH + q); };   // one per epilogue warp
    constexpr int NUM_BARS = 2 * STAGES + 5 + 2 * SCHED_DEPTH + EPI_WARPS;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(smem + STAGES * STAGE_BYTES + 8 * NUM_BARS);
    volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
    volatile int* sched_slot = reinterpret_cast<volatile int*>(tmem_slot + 2);   // [SCHED_DEPTH] list positions
    const uint32_t sched_slot_addr = bars + 8u * NUM_BARS + 8u;
    const uint32_t ready_addr = sched_slot_addr + 4u * SCHED_DEPTH;          // the last list position whose inputs the producer found complete
    const uint32_t epi = bars + 1024u;                                       // 1024-byte aligned
    static_assert(8 * NUM_BARS + 12 + 4 * SCHED_DEPTH <= 1024, "barriers before the epilogue's staging");

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const int total = p.steps * (p.tiles[0] + p.tiles[1] + p.tiles[2]) * p.batch;

    if (threadIdx.x == 0) {
        *abort_flag = 0;
        store_ready(ready_addr, -1);
        for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 2 * EPI_WARPS); }
        mbar_init(drain_bar, 1);
        // a slot is free again when the leader's MMA lane and epilogue warps and the peer's producer and epilogue warps have read it
        for (int s = 0; s < SCHED_DEPTH; ++s) { mbar_init(sfull_bar(s), 1); mbar_init(sempty_bar(s), 2 + 2 * EPI_WARPS); }
        for (int q = 0; q < EPI_WARPS; ++q) mbar_init(add_bar(q), 1);
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
    auto sched_ack = [&](int ss) { mbar_arrive_cluster(mapa_shared(sempty_bar(ss), 0)); };

    if (warp == 0) {
        // ---------------------------------------------------------------- scheduler (leader) + TMA producer (both CTAs)
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0; bool ok = true;
            int ss = 0; uint32_t sphase = 0;
            long issued = 0;
            bool exhausted = false;
            auto publish = [&]() -> int {                                    // takes the next list position for both CTAs
                if (exhausted) return -1;
                if (!mbar_wait_cluster(sempty_bar(ss), sphase ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; return -1; }
                int t = atomicAdd(p.next, 1);
                if (t >= total) { t = -1; exhausted = true; }
                sched_slot[ss] = t;
                asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa_shared(sched_slot_addr + 4u * ss, 1)), "r"(t) : "memory");
                mbar_arrive(sfull_bar(ss));
                mbar_arrive_cluster(mapa_shared(sfull_bar(ss), 1));          // release.cluster: the peer sees its slot
                if (++ss == SCHED_DEPTH) { ss = 0; sphase ^= 1u; }
                return t;
            };
            while (ok) {
                int t;
                if (leader) {
                    t = publish();
                    if (!ok) break;
                } else {
                    if (!mbar_wait_cluster(sfull_bar(ss), sphase, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    t = sched_slot[ss];
                    sched_ack(ss);
                    if (++ss == SCHED_DEPTH) { ss = 0; sphase ^= 1u; }
                }
                if (t < 0) break;
                const Tile w = decode(p, t);
                if (w.k > 0 && !flag_wait_ge(p.done + w.b * DONE_PITCH, w.need, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                store_ready(ready_addr, t);
                const int xb = (w.k / 3) & 1;
                const CUtensorMap* ma = w.mode == GRAM ? &maps.x_l[xb] : w.mode == POLY ? &maps.a_l : &maps.b_l;
                const CUtensorMap* mb = w.mode == GRAM ? &maps.x_r[xb] : w.mode == POLY ? &maps.a_r : &maps.x_mn[xb];
                const int num_kb = steps_of_k(p, w);
                const int arow = w.i * TM + static_cast<int>(rank) * 128, bcol = w.j * w.bn + static_cast<int>(rank) * (w.bn / 2);
                const int lost = t == 0 && (p.drop_ranks >> rank & 1) ? p.drop : -1;   // test hook
                for (int kb = 0; kb < num_kb; ++kb) {
                    if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    if (leader) mbar_arrive_expect_tx(full_bar(stage), 2 * (A_BYTES + w.bn / 2 * 128));
                    const uint32_t bar = mapa_shared(full_bar(stage), 0);
                    const uint32_t sa = base + stage * STAGE_BYTES;
                    // rows and chunks beyond the matrix arrive as zeros
                    if (kb != lost) {
                        tma2_load_4d(sa, ma, bar, 0, arow, kb, w.b);
                        if (w.mode == APPLY) tma2_load_4d(sa + A_BYTES, mb, bar, 0, kb * KB, bcol / 64, w.b);
                        else tma2_load_4d(sa + A_BYTES, mb, bar, 0, bcol, kb, w.b);
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
        // ---------------------------------------------------------------- MMA issuer (leader CTA only)
        if (lane == 0 && leader) {
            int stage = 0; uint32_t phase = 0; bool ok = true;
            int ss = 0; uint32_t sphase = 0;
            for (int it = 0; ok; ++it) {
                if (!mbar_wait(sfull_bar(ss), sphase, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                const int t = sched_slot[ss];
                sched_ack(ss);
                if (++ss == SCHED_DEPTH) { ss = 0; sphase ^= 1u; }
                if (t < 0) break;
                const Tile w = decode(p, t);
                const bool apply = w.mode == APPLY;
                const uint32_t idesc = make_idesc(w.bn, false, apply, TM, 0u);     // fp16 operands
                const int num_kb = steps_of_k(p, w);
                const int ab = it & 1;
                if (!mbar_wait_cluster(tempty_bar(ab), ((it >> 1) & 1u) ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                tc_fence_after();
                const uint32_t tmem_d = tmem_base + ab * TN;
                for (int kb = 0; kb < num_kb; ++kb) {
                    if (!mbar_wait(full_bar(stage), phase, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = base + stage * STAGE_BYTES, sb = sa + A_BYTES;
                    const uint64_t adesc = make_smem_desc(sa, 16, 1024);
                    const uint64_t bdesc = make_smem_desc(sb, apply ? 64 * 128 : 16, 1024);
#pragma unroll
                    for (int k = 0; k < KB / 16; ++k) {
                        // K-major: 16 elements = 32 bytes along the swizzled row; MN-major: 16 rows of 128 bytes
                        const uint32_t along = k * 32, down = k * 16 * 128;
                        umma2_f16(tmem_d, adesc + (along >> 4), bdesc + ((apply ? down : along) >> 4), idesc, (kb | k) != 0 ? 1u : 0u);
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
        // ---------------------------------------------------------------- epilogue warps (both CTAs)
        const int quad = warp & 3, half = (warp - 2) >> 2;
        // A warp has four blocks of shared memory.  A block of the result takes the place of its addend, which was loaded there.
        // APPLY has one for each of a tile's four blocks, all loaded while the products run.  The symmetric products need half
        // of them for the mirror images: their blocks take turns in two, and the addends of POLY's last two blocks arrive
        // while the blocks before them are worked on.
        const uint32_t blocks = epi + (warp - 2) * EPI_WARP_BYTES, abar = add_bar(warp - 2);
        uint32_t aphase = 0;
        int ss = 0; uint32_t sphase = 0;
        for (int it = 0;; ++it) {
            int t = -2;
            if (lane == 0 && mbar_wait_cluster(sfull_bar(ss), sphase, abort_flag, p.wait_limit_ns)) {
                t = sched_slot[ss];
                sched_ack(ss);
            }
            t = __shfl_sync(0xffffffffu, t, 0);
            if (++ss == SCHED_DEPTH) { ss = 0; sphase ^= 1u; }
            if (t < 0) break;                                                // -1: list exhausted, -2: gave up
            const Tile w = decode(p, t);
            const int ab = it & 1;
            const int row0 = w.i * TM + static_cast<int>(rank) * 128 + quad * 32;
            const int ncols = w.mode == APPLY ? p.ldx : p.lda;
            // blocks of this warp: columns w.j * bn + 64 n + 32 half
            const int col_first = w.j * w.bn + half * 32;
            int blocks_here = row0 < p.R && col_first < ncols ? (ncols - col_first + 63) / 64 : 0;
            if (blocks_here > w.bn / 64) blocks_here = w.bn / 64;
            // the addends of all its blocks arrive while the products run
            const bool addend = w.mode != GRAM && blocks_here > 0;
            const CUtensorMap* from = w.mode == POLY ? &maps.a_blk : &maps.x_blk[(w.k / 3) & 1];
            auto place = [&](int n) { return blocks + (w.mode == APPLY ? n : n & 1) * BLOCK_BYTES; };
            auto load_block = [&](int n) { tma_load_4d(place(n), from, abar, half * 32, row0, w.j * (w.bn / 64) + n, w.b); };
            auto await_addend = [&]() {
                const bool got = mbar_wait(abar, aphase, abort_flag, p.wait_limit_ns);
                aphase ^= 1u;
                if (__all_sync(0xffffffffu, got)) return true;
                const unsigned long long t0 = globaltimer_ns();              // give-up path: the copies in flight land first
                while (!mbar_try_wait(abar, aphase ^ 1u) && globaltimer_ns() - t0 < p.wait_limit_ns) {}
                return false;
            };
            int ok = 1;
            if (lane == 0) {
                if (addend) ok = wait_ready(ready_addr, t, abort_flag, p.wait_limit_ns);
                bulk_wait_read_all();                                        // the stores of the tile before have left the blocks
                if (addend && ok) {
                    const int now = w.mode == POLY ? min(blocks_here, 2) : blocks_here;
                    mbar_arrive_expect_tx(abar, now * BLOCK_BYTES);
                    for (int n = 0; n < now; ++n) load_block(n);
                }
            }
            ok = __shfl_sync(0xffffffffu, ok, 0);
            if (!ok) break;
            if (addend && !await_addend()) break;
            ok = mbar_wait(tfull_bar(ab), (it >> 1) & 1u, abort_flag, p.wait_limit_ns);
            if (!__all_sync(0xffffffffu, ok)) break;
            tc_fence_after();
            const uint32_t tmem_row = tmem_base + ab * TN + (static_cast<uint32_t>(quad * 32) << 16) + half * 32;
            for (int n = 0; n < blocks_here; ++n) {
                const int col0 = col_first + 64 * n;
                if (w.last) {
                    const uint32_t blk = place(n);
                    auto from_block = [&](int q, float* f) { unpack8(ld_shared_v4(blk + block_at(lane, q)), f); };
                    if (p.transposed) epilogue_last<32, true>(p, w.k, w.b, row0, col0, lane, tmem_row + 64 * n, blk, from_block);
                    else epilogue_last<32, false>(p, w.k, w.b, row0, col0, lane, tmem_row + 64 * n, blk, from_block);
                } else {
                    float v[32];
                    __syncwarp();
                    tmem_ld32(tmem_row + 64 * n, v);
                    if (w.mode == POLY) {
                        if (n >= 2 && !await_addend()) { ok = 0; break; }
                        if (n >= 1 && lane == 0) {
                            bulk_wait_read_all();                            // block n - 1 has left its places:
                            if (n + 1 < blocks_here) {                       // the addend of block n + 1 may come
                                mbar_arrive_expect_tx(abar, BLOCK_BYTES);
                                load_block(n + 1);
                            }
                        }
                    } else if (w.mode == GRAM && n >= 2 && lane == 0) {
                        bulk_wait_read_1();                                  // block n - 2 has left its places
                    }
                    __syncwarp();
                    tmem_ld_wait();
                    epilogue_block(p, maps, w, row0, col0, lane, v, place(n), blocks + (2 + (n & 1)) * BLOCK_BYTES);
                }
            }
            if (!ok) break;
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_cluster(mapa_shared(tempty_bar(ab), 0));
            if (!w.last && lane == 0) signal_stored(p.done + w.b * DONE_PITCH);
        }
        if (lane == 0) bulk_wait_all();                                      // nothing reads this CTA's shared memory any more
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

// ------------------------------------------------------------------------------------ small matrices
// The whole update of a matrix that fits the shared memory of one CTA (CG = 1: R <= 128, C <= 512) or a CTA pair (CG = 2: R and
// C <= 256, 128 rows in each), one launch for a batch: momentum, norm, all products, write-back.  X and A (later B) stay in
// shared memory as fp16 in the operands' layout: 64-column chunks of rows of 128 bytes, 128-byte swizzle.  A row of X is K-major
// for X X^T, and the same bytes are the MN-major right operand of B X, whose K are the rows.  In a pair the right operand's
// columns are split, not its rows, so B X reads a second copy, XN: all 256 rows of this CTA's half of the columns, to which the
// other CTA's epilogue writes its rows.
// Each product is issued by one thread, waited for by all 16 warps (four per quarter of the tensor memory's lanes), and turned
// into the next operand in place.  Bound: latency.  256 x 256 in fp32: 74 us, of which 15 products of 3.4 us (barrier 0.6 to 0.9,
// tensor cores 1.35, epilogue 1.1 to 2.4), 9.7 us to bring the matrix in and 8.3 us to write it back.
constexpr int SMALL_WARPS = 16, SMALL_THREADS = 32 * SMALL_WARPS;
constexpr int SMALL_KEPT = 8;                           // pieces of 8 elements of U that a thread keeps while the norm is formed
template <int CG> struct SmallShape {
    static constexpr int ROWS = 128 * CG;               // of the padded X
    static constexpr int MAX_C = CG == 1 ? 512 : 256;
    static constexpr int A_CHUNKS = 2 * CG;             // 64-column chunks of A
    static constexpr int X_CHUNK = 128 * 128;           // bytes: this CTA's 128 rows
    static constexpr int XN_CHUNK = 256 * 128;
    static constexpr int X_BYTES = MAX_C / 64 * X_CHUNK, A_OFFSET = X_BYTES, XN_OFFSET = A_OFFSET + A_CHUNKS * X_CHUNK;
    static constexpr int SCRATCH = XN_OFFSET + (CG == 2 ? MAX_C / 128 * XN_CHUNK : 0);
    static constexpr int SMEM = SCRATCH + 1024;   // the scratch (2 KB a warp, in A) and alignment slack
};
static_assert(SmallShape<1>::SMEM <= 227 * 1024 && SmallShape<2>::SMEM <= 227 * 1024, "shared memory per CTA");

template <int CG> __device__ __forceinline__ void small_sync() {
    if (CG == 2) cluster_sync_all();
    else __syncthreads();
}
__device__ __forceinline__ void st_cluster_v4(uint32_t addr, uint4 v) {
    asm volatile("st.shared::cluster.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
// Byte offset of 16-byte piece q (8 halves) of row r inside a chunk.
__device__ __forceinline__ uint32_t chunk_at(int r, int q) { return static_cast<uint32_t>(r * 128 + ((q ^ (r & 7)) << 4)); }

template <int CG, typename G>
__global__ void __launch_bounds__(SMALL_THREADS, 1) muon_small_kernel(const __grid_constant__ GemmParams p, const __grid_constant__ PrepParams pp) {
    using S = SmallShape<CG>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ double part[SMALL_WARPS];
    __shared__ uint64_t bar_slot, drain_slot;
    __shared__ uint32_t tmem_slot;
    __shared__ int abort_word, gave_up_word;
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    const uint32_t bar = smem_u32(&bar_slot);
    volatile int* abort_flag = &abort_word;
    volatile int* gave_up = &gave_up_word;                                  // 1 + the product that a warp of either CTA gave up, 0: none
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = CG == 2 ? static_cast<int>(cluster_ctarank()) : 0;
    const int b = blockIdx.x / CG;
    const int chunks = p.ldx / 64;                                          // CG = 2: an even number (ldx a multiple of 128)

    if (threadIdx.x == 0) {
        abort_word = gave_up_word = 0;
        mbar_init(bar, 1);
        mbar_init(smem_u32(&drain_slot), 1);
        fence_barrier_init();
        if (gridDim.x == CG && rank == 0) *p.status = 0;                    // of several matrices the host clears it
    }
    if (warp == 0) {
        if (CG == 2) { tmem2_alloc(smem_u32(&tmem_slot), 512); tmem2_relinquish(); }
        else { tmem_alloc(smem_u32(&tmem_slot), 512); tmem_relinquish(); }
    }

    // ---- momentum and sum of squares over this CTA's rows of X, in pieces of 8 neighbouring columns of a row of X.  Neighbouring
    // threads take neighbouring elements of the caller's array: along X's rows, or down them where it holds X^T.
    const size_t mat = static_cast<size_t>(b) * p.R * p.C;
    const G* g = static_cast<const G*>(pp.g) + mat;
    float* m = pp.m ? pp.m + mat : nullptr;
    const int rows_here = min(128, p.R - rank * 128);                       // 0 or less: this CTA holds zeros only
    const int pieces = 128 * chunks * 8;
    auto row_of = [&](int k) { return p.transposed ? k & 127 : k / (chunks * 8); };
    auto col_of = [&](int k) { return (p.transposed ? k >> 7 : k % (chunks * 8)) * 8; };
    const size_t along = p.transposed ? p.R : 1, down = p.transposed ? 1 : p.C, origin = static_cast<size_t>(rank) * 128 * down;
    // U of a piece (0 beyond the matrix); UPDATE: with the momentum brought up to date
    auto load_piece = [&](int k, float* u, bool update) {
        const int r = row_of(k), c = col_of(k);
        const int n = r < rows_here ? min(8, p.C - c) : 0;
        const size_t at = origin + r * down + c * along;
        const bool four = pp.four && !p.transposed;                         // n is then 0, 4 or 8
        float mv[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = 0.f;
        if (four) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) {
                if (j < n) load_v<G, 4>(g + at + j, u + j);
                if (m && j < n) load_v<float, 4>(m + at + j, mv + j);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j < n) u[j] = to_float(g[at + j * along]);
                if (m && j < n) mv[j] = m[at + j * along];
            }
        }
        if (m) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (update) mv[j] = pp.mu * mv[j] + u[j];
                u[j] = pp.nesterov ? u[j] + pp.mu * mv[j] : mv[j];
            }
            if (update) {
                if (four) {
#pragma unroll
                    for (int j = 0; j < 8; j += 4) if (j < n) store_v<4>(m + at + j, mv + j);
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) if (j < n) m[at + j * along] = mv[j];
                }
            }
        }
    };
    // What bounds this part is one SM's share of the L2's bandwidth (256 x 256 in fp32: 384 KB in and out per CTA), so U is kept
    // rather than read again, as far as registers go.
    double sq = 0.0;
    float kept[SMALL_KEPT][8];
    auto squares = [&](const float* u) {
        float q = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) q += u[j] * u[j];
        sq += q;
    };
#pragma unroll
    for (int i = 0; i < SMALL_KEPT; ++i) {
        const int k = i * SMALL_THREADS + threadIdx.x;
        if (k < pieces) { load_piece(k, kept[i], true); squares(kept[i]); }
    }
#pragma unroll 1
    for (int k = SMALL_KEPT * SMALL_THREADS + threadIdx.x; k < pieces; k += SMALL_THREADS) {
        float u[8];
        load_piece(k, u, true);
        squares(u);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sq += __shfl_xor_sync(0xffffffffu, sq, o);
    if (lane == 0) part[warp] = sq;
    tc_fence_before();
    small_sync<CG>();
    tc_fence_after();
    double total = 0.0;
    for (int r = 0; r < CG; ++r)
        for (int i = 0; i < SMALL_WARPS; ++i) {
            double v;
            if (CG == 2) asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(mapa_shared(smem_u32(part + i), r)) : "memory");
            else v = part[i];
            total += v;
        }
    const float norm = static_cast<float>(sqrt(total));
    const float inv = pp.scale / (norm < pp.eps ? pp.eps : norm);           // NaN stays NaN
    const uint32_t tmem = tmem_slot;

    // Eight neighbouring elements of this CTA's row r of X from column c on: into X, and into XN where that lies.
    auto put_x = [&](int r, int c, uint4 v) {
        const uint32_t at = base + (c >> 6) * S::X_CHUNK + chunk_at(r, (c >> 3) & 7);
        st_shared_v4(at, v);
        if (CG == 2) {
            const int half = p.ldx / 2, to = c >= half ? 1 : 0, cc = c - to * half;
            st_cluster_v4(mapa_shared(base + S::XN_OFFSET + (cc >> 6) * S::XN_CHUNK + chunk_at(rank * 128 + r, (cc >> 3) & 7), to), v);
        }
    };
    // ---- X_0; rows and columns beyond the matrix hold zeros.  A piece that was not kept is formed again.
    auto start_piece = [&](int k, float* u) {
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] *= inv;
        put_x(row_of(k), col_of(k), pack8(u));
    };
#pragma unroll
    for (int i = 0; i < SMALL_KEPT; ++i) {
        const int k = i * SMALL_THREADS + threadIdx.x;
        if (k < pieces) start_piece(k, kept[i]);
    }
#pragma unroll 1
    for (int k = SMALL_KEPT * SMALL_THREADS + threadIdx.x; k < pieces; k += SMALL_THREADS) {
        float u[8];
        load_piece(k, u, false);
        start_piece(k, u);
    }

    const int quad = warp & 3, first = warp >> 2, row = quad * 32 + lane;
    const uint32_t tmem_row = tmem + (static_cast<uint32_t>(quad * 32) << 16);
    uint32_t parity = 0;
    bool got = true;                                                        // the product before has come to its end (alike in a warp)
    for (int k = 0; k < 3 * p.steps; ++k) {
        const int mode = k % 3;
        // what was written to either CTA's shared memory is read by the tensor cores next
        asm volatile("fence.proxy.async;" ::: "memory");
        tc_fence_before();
        small_sync<CG>();
        tc_fence_after();
        if (threadIdx.x == 0 && rank == 0) {
            asm volatile("fence.proxy.async;" ::: "memory");
            const int k_steps = mode == GRAM ? p.ldx / 16 : S::ROWS / 16;
            const int groups = mode == APPLY ? (p.ldx + 255) / 256 : 1;     // of up to 256 result columns
            for (int n = 0; n < groups; ++n) {
                const int width = mode == APPLY ? min(256, p.ldx - 256 * n) : S::ROWS;
                const uint32_t idesc = make_idesc(width, false, mode == APPLY, 128 * CG, 0u);
                for (int q = 0; q < k_steps; ++q) {
                    const uint32_t along = (q >> 2) * S::X_CHUNK + (q & 3) * 32;            // K-major: 32 bytes of a chunk's rows
                    const uint64_t ad = make_smem_desc(base + (mode == GRAM ? 0 : S::A_OFFSET) + along, 16, 1024);
                    uint64_t bd;
                    if (mode != APPLY) bd = ad;                                             // the same rows
                    else if (CG == 1) bd = make_smem_desc(base + 4 * n * S::X_CHUNK + q * 2048, S::X_CHUNK, 1024);
                    else bd = make_smem_desc(base + S::XN_OFFSET + q * 2048, S::XN_CHUNK, 1024);
                    if (CG == 2) umma2_f16(tmem + 256 * n, ad, bd, idesc, q != 0 ? 1u : 0u);
                    else umma_f16(tmem + 256 * n, ad, bd, idesc, q != 0 ? 1u : 0u);
                }
            }
            if (k == p.drop && b == 0) {}                                   // test hook: the signal is lost
            else if (CG == 2) umma2_commit_both(bar);
            else umma_commit(bar);
        }
        // All threads of the CTA or pair leave here or none: only waits for product k write k + 1, and all waits for the products
        // before it lie before the barrier.  (Behind the product's start, where it costs nothing; of a product that should not have
        // been started nothing is used.)
        if (const int lost = *gave_up; lost != 0 && lost <= k) { got = false; break; }
        got = __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, p.wait_limit_ns));
        parity ^= 1u;
        tc_fence_after();
        if (!got) {                                                         // nothing that the product may still read is written
            if (lane < CG) {
                if (CG == 2) asm volatile("st.shared::cluster.s32 [%0], %1;" ::"r"(mapa_shared(smem_u32(&gave_up_word), lane)), "r"(k + 1) : "memory");
                else *gave_up = k + 1;
            }
            __syncwarp();
            continue;
        }
        if (k + 1 == 3 * p.steps) break;
        const float alpha = p.alpha[k], beta = p.beta[k];
        const int blocks = (mode == APPLY ? p.ldx : S::ROWS) / 32;
        for (int n = first; n < blocks; n += SMALL_WARPS / 4) {
            float v[32];
            __syncwarp();
            tmem_ld32(tmem_row + 32 * n, v);
            tmem_ld_wait();
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = 32 * n + 8 * q;
                const uint32_t at = base + (mode == APPLY ? 0 : S::A_OFFSET) + (c >> 6) * S::X_CHUNK + chunk_at(row, (c >> 3) & 7);
                float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
                if (mode != GRAM) unpack8(ld_shared_v4(at), f);
#pragma unroll
                for (int j = 0; j < 8; ++j) f[j] = alpha * v[8 * q + j] + beta * f[j];
                if (mode == APPLY) put_x(row, c, pack8(f));
                else st_shared_v4(at, pack8(f));
            }
        }
    }
    // ---- the last X, to the caller's arrays, 16 columns at a time
    if (!got && threadIdx.x == 0 && rank == 0) {                            // give-up path: the products in flight end first
        if (CG == 2) umma2_commit_local(smem_u32(&drain_slot));
        else umma_commit(smem_u32(&drain_slot));
        const unsigned long long t0 = globaltimer_ns();
        while (!mbar_try_wait(smem_u32(&drain_slot), 0) && globaltimer_ns() - t0 < p.wait_limit_ns) {}
    }
    __syncwarp();
#pragma unroll 1
    for (int n = first; got && n < p.ldx / 16; n += SMALL_WARPS / 4) {
        if (16 * n >= p.C || quad * 32 >= rows_here) break;                 // uniform in the warp
        auto from_x = [&](int q, float* f) {
            const int c = 16 * n + 8 * q;
            unpack8(ld_shared_v4(base + (c >> 6) * S::X_CHUNK + chunk_at(row, (c >> 3) & 7)), f);
        };
        const uint32_t scratch = base + S::A_OFFSET + warp * 2048;          // B is spent
        const int last = 3 * p.steps - 1, row0 = rank * 128 + quad * 32;
        if (p.transposed) epilogue_last<16, true>(p, last, b, row0, 16 * n, lane, tmem_row + 16 * n, scratch, from_x);
        else epilogue_last<16, false>(p, last, b, row0, 16 * n, lane, tmem_row + 16 * n, scratch, from_x);
    }
    tc_fence_before();
    small_sync<CG>();                                                       // no CTA leaves while its pair may still write to it
    if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, VPCE_DEV_WAIT_EXPIRED);
    if (warp == 0) {
        __syncwarp();
        tc_fence_after();
        if (CG == 2) tmem2_dealloc(tmem, 512);
        else tmem_dealloc(tmem, 512);
    }
}

}  // namespace vpmuon
