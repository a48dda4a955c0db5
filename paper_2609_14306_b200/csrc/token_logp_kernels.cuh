// Device code of the token log probabilities (token_logp.h): the strip kernel (a CTA pair per 256 x 256 tile of logits), the kernel
// for few tokens (one pass over the weight) and the kernel that joins what either leaves per token.
//
// Per token and slice of the vocabulary the first two leave (m, z, u, n): with t = (x - m) / temperature * log2(e) for logit x,
//     m = max x,   z = sum 2^t,   u = sum t 2^t,   n = how many candidates for the alternatives lie beside it
// two of which join like two online softmax states: m = max(m1, m2), and with t' = (m1 - m) / temperature * log2(e)
//     z1 -> z1 2^t',   u1 -> 2^t' (u1 + t' z1)
// Then lse = m / temperature + ln z and the entropy is ln z - ln 2 u / z: no difference of large numbers anywhere.
#pragma once

#include "sm100_ptx.cuh"
#include "vp_ce.h"

namespace vptl {

using namespace vpce;

constexpr int MAX_TOP = 20;                                 // alternatives per token
constexpr float LOG2E_F = 1.4426950408889634f, LN2_F = 0.6931471805599453f;
constexpr float MINUS_INF = -__builtin_huge_valf();

constexpr int KB_BYTES = 128;                               // a k-block: 128 bytes of every row (64 bf16 or 128 e4m3)
constexpr int TILE_M = 128, TILE_N = 256, HALF_N = 128;     // rows per CTA, columns per pair tile, columns per epilogue thread
// Warps: 0 copies, 1 issues the products, 2 and 3 have nothing to do (the first four are one warp group, which gives up registers), 4 to 11
// are the epilogue.
constexpr int EPI_WARPS = 8, EPI_THREADS = 32 * EPI_WARPS, EPI_FIRST = 128, THREADS = EPI_FIRST + EPI_THREADS;

struct Params {
    int rows, cols;                         // tokens of this launch, vocabulary columns of this launch
    int row0, col0;                         // first token (coordinates of H's map), first column (coordinates of W's map)
    int kbs;                                // k-blocks
    int m_tiles, n_tiles;                   // strip kernel: 256-token and 256-column tiles
    int slices;                             // slices per token in `part` and `cand`
    int V;
    float scale;                            // log2(e) / temperature
    const int32_t* tokens;                  // of this launch's first token; null: none
    float4* part;                           // [rows][slices]: m, z, u, number of candidates
    uint2* cand;                            // [rows][slices][top]: logit, column
    int top;
    // Bounds from below on a token's top-th largest logit, as ordered bits (0: none): from the strips before, and of the first strip the
    // largest logits of its slices so far, by the slice's number modulo 32 (null in later strips).  The top-th largest of those is
    // one: each stands in another column.
    unsigned *floor, *marks;                // [rows], [rows][32]
    float* chosen;                          // [rows]: logit of the given token
    const float *hs, *ws;                   // 8 bits: scales of H's rows [.][kbs], of W's blocks [.][kbs]
    int* status;
    unsigned long long wait_limit_ns;
    int drop_kb;                            // test hook: the copies of this k-block of the first tile get lost; < 0: off
};

// Floats as unsigned numbers of the same order; 0 stands below all of them.
__device__ __forceinline__ unsigned ordered(float v) {
    const unsigned b = __float_as_uint(v);
    return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float from_ordered(unsigned o) {
    return o == 0u ? MINUS_INF : __uint_as_float(o ^ ((o >> 31) ? 0x80000000u : 0xffffffffu));
}
// The number just below v: "> below(v)" accepts v itself (of either sign where it is a zero).
__device__ __forceinline__ float below(float v) {
    if (v == 0.f) return -1.40129846e-45f;
    return v == MINUS_INF ? MINUS_INF : from_ordered(ordered(v) - 1u);
}

using f2 = unsigned long long;
__device__ __forceinline__ f2 pair(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 split(f2 v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

// kind::f8f6f4 (K = 32): e4m3 x e4m3 -> fp32.
__device__ __forceinline__ void umma_f8(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void umma2_f8(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(tmem_d), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate) : "memory");
}
// 32 lanes x 8 or 16 consecutive fp32 columns.
__device__ __forceinline__ void tmem_ld8(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr) : "memory");
}

// 64 consecutive columns.
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, float* v) {
    uint32_t* r = reinterpret_cast<uint32_t*>(v);
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(taddr) : "memory");
}
// "This warp has read the accumulator", to the leader's barrier.  It hands over tensor memory only, which the tcgen05 wait and fence before it
// order, so it needs no release of this thread's own memory accesses at cluster scope: that would wait for all of them, the loads of
// scales ahead included, and took 1.2 us a k-block where 0.58 remain (8 bits, 4096 x 7168 x 32768: 1027 and 2150 TFLOP/s).
__device__ __forceinline__ void arrive_leader(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// Registers of the 8-bit strip kernel: launched with 168 a thread (384 threads: 64512), 40 are left to the first warp group's and the
// epilogue's have 232: 128 x 40 + 256 x 232 = 64512.
__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 40;"); }
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 232;"); }
// Programmatic launch: the grid that follows may be brought up; what it does after its wait comes after this one's end.
__device__ __forceinline__ void launch_next() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_for_last() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

// ------------------------------------------------------------------------------------ one token's slice, held by one thread
struct State { float m, z, u; };

// The state with its sums about another maximum m >= s.m.  A state without a maximum has seen nothing (z = u = 0), or NaN only.
__device__ __forceinline__ void move(State& s, float m, float scale) {
    if (s.m != MINUS_INF) {
        const float t = (s.m - m) * scale, f = ex2f(t);
        s.u = f * fmaf(t, s.z, s.u);
        s.z *= f;
    }
    s.m = m;
}

// Folds 32 logits (columns of which the first `valid` exist) into the state; leaves the maxima of each four in quads[8].
__device__ __forceinline__ void fold32(State& s, float* v, int valid, float scale, float* quads) {
    if (valid < 32) {
#pragma unroll
        for (int j = 0; j < 32; ++j) if (j >= valid) v[j] = MINUS_INF;
    }
    float m = s.m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        quads[j] = fmaxf(fmaxf(v[4 * j], v[4 * j + 1]), fmaxf(v[4 * j + 2], v[4 * j + 3]));
        m = fmaxf(m, quads[j]);
    }
    const f2 scale2 = pair(scale, scale), minus = pair(-m, -m);
    f2 z0 = 0ull, u0 = 0ull, z1 = 0ull, u1 = 0ull;
    if (valid < 32) {
        float z = 0.f, u = 0.f;
#pragma unroll
        for (int j = 0; j < 32; ++j) {
            const float t = (v[j] - m) * scale, e = ex2f(t);
            if (j < valid) { z += e; u = fmaf(t, e, u); }
        }
        z0 = pair(z, 0.f); u0 = pair(u, 0.f);
    } else {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const f2 ta = mul2(add2(pair(v[j], v[j + 1]), minus), scale2), tb = mul2(add2(pair(v[j + 2], v[j + 3]), minus), scale2);
            const float2 a = split(ta), b = split(tb);
            const f2 ea = pair(ex2f(a.x), ex2f(a.y)), eb = pair(ex2f(b.x), ex2f(b.y));
            z0 = add2(z0, ea); z1 = add2(z1, eb);
            u0 = fma2(ta, ea, u0); u1 = fma2(tb, eb, u1);
        }
    }
    const float2 z = split(add2(z0, z1)), u = split(add2(u0, u1));
    move(s, m, scale);
    s.z += z.x + z.y;
    s.u += u.x + u.y;
}

// A thread's best `top` logits of its slice, unordered, in shared memory: entry j of a thread at j * EPI_THREADS (both arrays).
// What comes is taken if it is above `lim`; columns come in ascending order, so among equals the lower column stays.
struct Best {
    float* val;
    uint8_t* col;
    int n, top, at;                                         // entries, their most, where the least is (once full)
    float lim;
    __device__ __forceinline__ void offer(float x, int c) {
        if (!(x > lim)) return;
        if (n < top) { val[n * EPI_THREADS] = x; col[n * EPI_THREADS] = static_cast<uint8_t>(c); if (++n < top) return; }
        else { val[at * EPI_THREADS] = x; col[at * EPI_THREADS] = static_cast<uint8_t>(c); }
        // the least entry, of equals the one with the highest column, goes next
        float least = val[0];
        int cl = col[0];
        at = 0;
#pragma unroll 4
        for (int j = 1; j < top; ++j) {
            const float y = val[j * EPI_THREADS];
            const int cy = col[j * EPI_THREADS];
            if (y < least || (y == least && cy > cl)) { least = y; cl = cy; at = j; }
        }
        lim = least;
    }
};

// The top-th largest of 32 numbers (in whose place they are sorted, larger first, by a bitonic network in registers).
template <typename T> __device__ __forceinline__ T top_th(T* t, int top) {
#pragma unroll
    for (int w = 2; w <= 32; w <<= 1)
#pragma unroll
        for (int k = w >> 1; k > 0; k >>= 1)
#pragma unroll
            for (int j = 0; j < 32; ++j)
                if ((j & k) == 0) {
                    const T a = t[j], b = t[j | k], more = a > b ? a : b, less = a > b ? b : a;
                    const bool down = (j & w) == 0;
                    t[j] = down ? more : less;
                    t[j | k] = down ? less : more;
                }
    T r = t[MAX_TOP - 1];
#pragma unroll
    for (int j = MAX_TOP - 2; j >= 0; --j) if (top <= j + 1) r = t[j];
    return r;
}
// A token's bound, as a number to be above.
__device__ __forceinline__ float above_floor(const Params& p, int row) {
    unsigned o = __ldcg(p.floor + row);
    if (p.marks) {
        unsigned t[32];
        const uint4* from = reinterpret_cast<const uint4*>(p.marks) + 8 * static_cast<size_t>(row);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint4 q = __ldcg(from + i);
            t[4 * i] = q.x; t[4 * i + 1] = q.y; t[4 * i + 2] = q.z; t[4 * i + 3] = q.w;
        }
        o = max(o, top_th(t, p.top));
    }
    return below(from_ordered(o));
}

// Which of a slice's 128 columns may matter, by groups of eight: the bits of those with an entry above best.lim.  Where many are (a
// token's first slices, before its bound has settled), that is first raised to what the slice itself says: the top-th largest
// of its 32 quads' maxima is a bound for its top-th logit.  (65 tokens of 2880 x 201088 with 20 alternatives: 413 us without this and
// the marks, 275 with both.)
__device__ __forceinline__ unsigned groups_above(Best& best, const float* quads) {
    int n = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) n += quads[j] > best.lim ? 1 : 0;
    if (!__any_sync(0xffffffffu, n > 0)) return 0u;
    if (__any_sync(0xffffffffu, n > best.top)) {
        float t[32];
#pragma unroll
        for (int j = 0; j < 32; ++j) t[j] = fmaxf(quads[j], MINUS_INF);    // four NaN have a NaN as their maximum: it has no place in an order
        const float bound = top_th(t, best.top);
        best.lim = fmaxf(best.lim, below(bound));
    }
    unsigned mine = 0u;
#pragma unroll
    for (int j = 0; j < 16; ++j) mine |= fmaxf(quads[2 * j], quads[2 * j + 1]) > best.lim ? 1u << j : 0u;
    return __reduce_or_sync(0xffffffffu, mine);
}

// ------------------------------------------------------------------------------------ the strip kernel
// Two CTAs of a cluster per 256 x 256 tile (cta_group::2), persistent, tiles dealt round robin with the token tiles fastest (the tokens
// of a launch stay in L2, the weight streams).  An epilogue thread has one token's 128 columns.
//   bf16   the accumulator of a tile is complete in tensor memory; two of them, so the epilogue of one runs beside the products of
//          the next.  Bound: the tensor cores under the power cap; 4096 x 2880 x 201088 with 8 alternatives in 3.3 to 3.5 ms (boards
//          differ), 1360 to 1440 TFLOP/s: cuBLAS's sustained rate.  Alternatives are 5 % of it, most of that in the first strip, where
//          everything is new; of 65 tokens 240 us with 8 alternatives and 275 with 20, 220 without.
//   8 bits every k-block of 128 has its own scale, so its product is its own accumulator, and the epilogue threads add it to their
//          128 sums in registers with fp32 factors; the two buffers alternate by k-block.  Bound: that hand-over, 0.57 us a k-block
//          where the product alone takes 0.44 (4096 x 7168 x 32768: 0.89 ms, 0.69 with one accumulator per tile, which is not the
//          operator); 8192 x 7168 x 129280 in 7.7 ms, 1960 TFLOP/s.  Not better: four buffers of 128 columns (1.07 ms: narrower
//          products, twice the hand-overs), 16 epilogue warps of 64 columns (0.95), scales through shared memory from a warp of their
//          own (0.91), one signal for accumulator and stage (0.93), spinning waits (0.92).  A few spilled registers in the warps
//          before the epilogue cost 15 %.
constexpr int SMEM_MAX = 227 * 1024;
constexpr int STAGE = TILE_M * KB_BYTES + HALF_N * KB_BYTES;       // 32 KB
constexpr int LIST_BYTES = EPI_THREADS * MAX_TOP * 5, SCRATCH_BYTES = EPI_THREADS * 8 * 4;
template <bool F8, bool TOP> struct Strip {
    static constexpr int STAGES = TOP ? 6 : 7;
    static constexpr int BARS = 2 * STAGES + 5;
    static constexpr int LISTS = STAGES * STAGE + 512;              // offset behind barriers and slots
    static constexpr int SMEM = 1024 + LISTS + (TOP ? LIST_BYTES + (F8 ? SCRATCH_BYTES : 0) : 0);
    static_assert(8 * BARS + 16 <= 512 && SMEM <= SMEM_MAX, "shared memory per CTA");
};

template <bool F8, bool TOP>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS, 1)
tl_strip_kernel(const __grid_constant__ CUtensorMap tmH, const __grid_constant__ CUtensorMap tmW, const Params p) {
    using S = Strip<F8, TOP>;
    constexpr int STAGES = S::STAGES;
    constexpr int KE = F8 ? 128 : 64;                               // elements of a k-block
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    const uint32_t bars = base + STAGES * STAGE;
    auto full_bar = [&](int s) { return bars + 8u * s; };                        // used in the leader only
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto tfull_bar = [&](int a) { return bars + 8u * (2 * STAGES + a); };
    auto tempty_bar = [&](int a) { return bars + 8u * (2 * STAGES + 2 + a); };   // used in the leader only
    const uint32_t drain_bar = bars + 8u * (2 * STAGES + 4);
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + STAGES * STAGE + 8 * S::BARS);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < 2; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), 2 * EPI_WARPS); }
        mbar_init(drain_bar, 1);
        fence_barrier_init();
        fence_proxy_async();
        prefetch_tensormap(&tmH);
        prefetch_tensormap(&tmW);
    }
    if (warp == 1) {
        tmem2_alloc(smem_u32(tmem_slot), 512);
        tmem2_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const int tiles = p.m_tiles * p.n_tiles, first = blockIdx.x >> 1, step = gridDim.x >> 1;
    constexpr uint32_t IDESC = F8 ? make_idesc(TILE_N, false, false, 2 * TILE_M, 0u) : make_idesc(TILE_N, false, false, 2 * TILE_M, 1u);

    if (F8 && warp < EPI_FIRST / 32) give_registers();
    if (warp == 0) {
        // ---------------------------------------------------------------- copies (both CTAs)
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0; bool ok = true;
            long issued = 0;
            const uint64_t keep = make_policy(2), stream = make_policy(0);
            for (int tile = first; ok && tile < tiles; tile += step) {
                const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
                const int r0 = p.row0 + mt * 2 * TILE_M + static_cast<int>(rank) * TILE_M;
                const int c0 = p.col0 + nt * TILE_N + static_cast<int>(rank) * HALF_N;
                for (int kb = 0; kb < p.kbs; ++kb) {
                    if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    if (leader) mbar_arrive_expect_tx(full_bar(stage), 2 * STAGE);
                    const uint32_t bar = mapa_shared(full_bar(stage), 0), sa = base + stage * STAGE;
                    if (!(tile == 0 && kb == p.drop_kb)) {
                        tma2_load_2d(sa, &tmH, bar, kb * KE, r0, keep);
                        tma2_load_2d(sa + TILE_M * KB_BYTES, &tmW, bar, kb * KE, c0, stream);
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
        // ---------------------------------------------------------------- products (leader)
        if (lane == 0 && leader) {
            int stage = 0; uint32_t phase = 0; bool ok = true;
            int unit = 0;                                               // accumulators so far
            for (int tile = first; ok && tile < tiles; tile += step) {
                for (int kb = 0; kb < p.kbs; ++kb) {
                    const int ab = unit & 1;
                    if ((F8 || kb == 0) && !mbar_wait(tempty_bar(ab), ((unit >> 1) & 1) ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    if (!mbar_wait(full_bar(stage), phase, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = base + stage * STAGE, tmem_d = tmem_base + ab * TILE_N;
                    const uint64_t adesc = make_smem_desc(sa, 16, 1024), bdesc = make_smem_desc(sa + TILE_M * KB_BYTES, 16, 1024);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {                       // 32 bytes of every row per instruction
                        const uint32_t more = (F8 ? k != 0 : (kb | k) != 0) ? 1u : 0u;
                        if (F8) umma2_f8(tmem_d, adesc + 2 * k, bdesc + 2 * k, IDESC, more);
                        else umma2_f16(tmem_d, adesc + 2 * k, bdesc + 2 * k, IDESC, more);
                    }
                    umma2_commit_both(empty_bar(stage));
                    if (F8 || kb + 1 == p.kbs) { umma2_commit_both(tfull_bar(ab)); ++unit; }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok || *abort_flag) {
                umma2_commit_local(drain_bar);
                const unsigned long long t0 = globaltimer_ns();
                while (!mbar_try_wait(drain_bar, 0) && globaltimer_ns() - t0 < p.wait_limit_ns) {}
            }
        }
    } else if (warp >= EPI_FIRST / 32) {
        // ---------------------------------------------------------------- epilogue (both CTAs)
        if (F8) take_registers();
        const int quad = warp & 3, half = (warp - EPI_FIRST / 32) >> 2;
        const int et = threadIdx.x - EPI_FIRST;
        const uint32_t tmem_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + half * HALF_N;
        Best best;
        best.top = p.top;
        best.val = reinterpret_cast<float*>(smem + S::LISTS) + et;
        best.col = smem + S::LISTS + EPI_THREADS * MAX_TOP * 4 + et;
        float* const scratch = reinterpret_cast<float*>(smem + S::LISTS + LIST_BYTES) + et;
        auto release = [&](int ab) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) arrive_leader(mapa_shared(tempty_bar(ab), 0));
        };
        bool ok = true;
        int unit = 0;
        for (int tile = first; ok && tile < tiles; tile += step) {
            const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
            const int row = mt * 2 * TILE_M + static_cast<int>(rank) * TILE_M + quad * 32 + lane;
            const bool row_ok = row < p.rows;
            const int c0 = nt * TILE_N + half * HALF_N;                 // first column within the launch
            const int valid = p.cols - c0;                              // columns that exist (may be <= 0)
            const int token = p.tokens && row_ok ? p.tokens[row] : -1;
            const int rel = token - (p.col0 + c0);                      // the token's column within this thread's, if 0 <= rel < 128
            State s{MINUS_INF, 0.f, 0.f};
            if (TOP) { best.n = 0; best.lim = row_ok ? above_floor(p, row) : __builtin_huge_valf(); }
            auto pick = [&](const float* v, int c) {                    // c: first of 32 columns
                if (static_cast<unsigned>(rel - c) < 32u && rel < valid) {
                    float x = 0.f;
#pragma unroll
                    for (int j = 0; j < 32; ++j) if (j == rel - c) x = v[j];
                    p.chosen[row] = x;
                }
            };
            if constexpr (!F8) {
                const int ab = unit & 1;
                ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(ab), (unit >> 1) & 1, abort_flag, p.wait_limit_ns));
                if (!ok) break;
                tc_fence_after();
                const uint32_t acc = tmem_row + ab * TILE_N;
                auto fold = [&](int c, float* quads) {
                    float v[32];
                    __syncwarp();
                    tmem_ld32(acc + c, v);
                    tmem_ld_wait();
                    pick(v, c);
                    fold32(s, v, valid - c, p.scale, quads);
                };
                if constexpr (TOP) {
                    float quads[32];
#pragma unroll
                    for (int c = 0; c < HALF_N; c += 32) {
                        if (c < valid) fold(c, quads + c / 4);
                        else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) quads[c / 4 + j] = MINUS_INF;
                        }
                    }
                    for (unsigned todo = groups_above(best, quads); todo; todo &= todo - 1) {
                        const int h = 8 * (__ffs(todo) - 1);
                        float w[8];
                        __syncwarp();
                        tmem_ld8(acc + h, w);
                        tmem_ld_wait();
#pragma unroll
                        for (int j = 0; j < 8; ++j) if (h + j < valid) best.offer(w[j], h + j);
                    }
                    __syncwarp();
                } else {
#pragma unroll 1
                    for (int c = 0; c < HALF_N && c < valid; c += 32) {
                        float quads[8];
                        fold(c, quads);
                    }
                }
                ++unit;
                release(ab);
            } else {
                f2 acc[HALF_N / 2];
#pragma unroll
                for (int j = 0; j < HALF_N / 2; ++j) acc[j] = 0ull;
                const float* hs = p.hs + static_cast<size_t>(p.row0 + (row_ok ? row : 0)) * p.kbs;
                const float* ws = p.ws + static_cast<size_t>(min(p.col0 + c0, p.V - 1) / 128) * p.kbs;
                // factors of the next k-blocks, AHEAD of them under way
                constexpr int AHEAD = 4;
                float fh[AHEAD], fw[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) { fh[i] = i < p.kbs ? __ldg(hs + i) : 0.f; fw[i] = i < p.kbs ? __ldg(ws + i) : 0.f; }
                for (int kb = 0; kb < p.kbs; ++kb) {
                    const float f = fh[0] * fw[0];
#pragma unroll
                    for (int i = 0; i + 1 < AHEAD; ++i) { fh[i] = fh[i + 1]; fw[i] = fw[i + 1]; }
                    if (kb + AHEAD < p.kbs) { fh[AHEAD - 1] = __ldg(hs + kb + AHEAD); fw[AHEAD - 1] = __ldg(ws + kb + AHEAD); }
                    const int ab = unit & 1;
                    ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(ab), (unit >> 1) & 1, abort_flag, p.wait_limit_ns));
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t from = tmem_row + ab * TILE_N;
                    const f2 factor = pair(f, f);
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < HALF_N; c += 64) {
                        float v[64];
                        tmem_ld64(from + c, v);
                        tmem_ld_wait();
                        if (c + 64 == HALF_N) release(ab);              // all of it is in registers
#pragma unroll
                        for (int j = 0; j < 32; ++j) acc[c / 2 + j] = fma2(pair(v[2 * j], v[2 * j + 1]), factor, acc[c / 2 + j]);
                    }
                    ++unit;
                }
                if (!ok) break;
                float quads[TOP ? 32 : 8];
#pragma unroll
                for (int c = 0; c < HALF_N; c += 32) {
                    float* const to = quads + (TOP ? c / 4 : 0);
                    if (c < valid) {
                        float v[32];
#pragma unroll
                        for (int j = 0; j < 16; ++j) { const float2 t = split(acc[c / 2 + j]); v[2 * j] = t.x; v[2 * j + 1] = t.y; }
                        pick(v, c);
                        fold32(s, v, valid - c, p.scale, to);
                    } else if (TOP) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) to[j] = MINUS_INF;
                    }
                }
                if constexpr (TOP) {
                    const unsigned todo = groups_above(best, quads);
                    if (todo) {
#pragma unroll
                        for (int h = 0; h < HALF_N; h += 8) {
                            if (todo >> (h / 8) & 1u) {
#pragma unroll
                                for (int j = 0; j < 4; ++j) {
                                    const float2 t = split(acc[h / 2 + j]);
                                    scratch[2 * j * EPI_THREADS] = t.x;
                                    scratch[(2 * j + 1) * EPI_THREADS] = t.y;
                                }
#pragma unroll 1
                                for (int j = 0; j < 8; ++j) if (h + j < valid) best.offer(scratch[j * EPI_THREADS], h + j);
                            }
                        }
                        __syncwarp();
                    }
                }
            }
            if (row_ok) {
                const size_t at = static_cast<size_t>(row) * p.slices + 2 * nt + half;
                p.part[at] = make_float4(s.m, s.z, s.u, TOP ? __int_as_float(best.n) : 0.f);
                if (TOP) {
                    uint2* const to = p.cand + at * p.top;
                    for (int j = 0; j < best.n; ++j)
                        to[j] = make_uint2(__float_as_uint(best.val[j * EPI_THREADS]), static_cast<unsigned>(p.col0 + c0 + best.col[j * EPI_THREADS]));
                    if (best.n == p.top) atomicMax(p.floor + row, ordered(best.lim));
                    if (p.marks && best.n > 0) atomicMax(p.marks + 32 * static_cast<size_t>(row) + ((2 * nt + half) & 31), ordered(s.m));
                }
            }
        }
        launch_next();
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

// ------------------------------------------------------------------------------------ a token's list, held by one warp
// A logit with its column as one number, the better the larger: larger logits first, among equals the lower column.  0: nothing.
using Key = unsigned long long;
__device__ __forceinline__ Key key_of(float x, int c) {
    return static_cast<Key>(ordered(x + 0.f)) << 32 | static_cast<unsigned>(~c);            // + 0: a zero is a zero
}
__device__ __forceinline__ float logit_of(Key k) { return from_ordered(static_cast<unsigned>(k >> 32)); }
__device__ __forceinline__ int column_of(Key k) { return static_cast<int>(~static_cast<unsigned>(k)); }

// Lane j has the (j + 1)-th best entry.
struct List {
    Key key;
    int lane, top;
    __device__ __forceinline__ Key last() const { return __shfl_sync(0xffffffffu, key, top - 1); }
    // Takes the candidates of the given lanes, one after the other: a chain of three dependent exchanges each.
    __device__ __forceinline__ void insert(unsigned from_lanes, Key k) {
        while (from_lanes) {
            const int from = __ffs(from_lanes) - 1;
            from_lanes &= from_lanes - 1;
            const Key now = __shfl_sync(0xffffffffu, k, from);
            const int at = __popc(__ballot_sync(0xffffffffu, key > now));
            const Key up = __shfl_up_sync(0xffffffffu, key, 1);
            if (lane >= at) key = lane == at ? now : up;
        }
    }
};
// A step of a bitonic network over the warp, for N independent sequences: lanes `mask` apart are put in order.
template <int N> __device__ __forceinline__ void in_order(Key* k, int mask, bool better_first) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Key o = __shfl_xor_sync(0xffffffffu, k[i], mask);
        if ((k[i] > o) != better_first) k[i] = o;
    }
}
// Merges a warp's 32 candidates into each list: sorts them (15 steps), then the better half of the list and the turned-round newcomers
// is a bitonic sequence (6 steps).
template <int N> __device__ __forceinline__ void sort_in(List* list, Key* k) {
    const int lane = list[0].lane;
#pragma unroll
    for (int w = 2; w <= 32; w <<= 1)
#pragma unroll
        for (int j = w >> 1; j > 0; j >>= 1) in_order<N>(k, j, ((lane & j) == 0) == ((lane & w) == 0));
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const Key o = __shfl_xor_sync(0xffffffffu, k[i], 31);
        k[i] = o > list[i].key ? o : list[i].key;
    }
#pragma unroll
    for (int j = 16; j > 0; j >>= 1) in_order<N>(k, j, (lane & j) == 0);
#pragma unroll
    for (int i = 0; i < N; ++i) list[i].key = k[i];
}
// Every lane offers a key (0: none); a few are inserted, more sorted and merged.  Returns whether there were any.
__device__ __forceinline__ bool offer(List& list, Key k) {
    const unsigned todo = __ballot_sync(0xffffffffu, k > list.last());
    if (todo == 0) return false;
    if (__popc(todo) <= 4) list.insert(todo, k);
    else sort_in<1>(&list, &k);
    return true;
}

// Offers N lists 128 columns c0 ... each, of which the first `valid` exist, lane l holding column c0 + 32 q + l of list i in x[q][i];
// all columns are above those of earlier calls.  What may matter is told by a bound from below: the list's last entry or, while the
// list is young, the top-th largest of the lanes' maxima.  The candidates above it (about as many as the list is long in the first
// tile, few later on) are brought together through `scratch` (64 floats of shared memory for each list, `pitch` apart) and merged at
// once.
template <int N> __device__ __forceinline__ void offer_tile(List* list, unsigned has, float (*x)[N], int c0, int valid, float* scratch, int pitch) {
    const int lane = list[0].lane, top = list[0].top;
    float above[N];
    unsigned left[N][4];                                            // candidates not yet taken, by quarter
    int most = 0;
    auto filter = [&](bool again) {
        most = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int n = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const unsigned now = __ballot_sync(0xffffffffu, ((has >> i) & 1u) && 32 * q + lane < valid && x[q][i] > above[i]);
                left[i][q] = again ? left[i][q] & now : now;
                n += __popc(left[i][q]);
            }
            most = max(most, n);
        }
    };
#pragma unroll
    for (int i = 0; i < N; ++i) above[i] = logit_of(list[i].last());
    filter(false);
    if (most > 32) {
        float m[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            m[i] = MINUS_INF;
#pragma unroll
            for (int q = 0; q < 4; ++q) if (32 * q + lane < valid) m[i] = fmaxf(m[i], x[q][i]);
        }
#pragma unroll
        for (int k = 2; k <= 32; k <<= 1)
#pragma unroll
            for (int j = k >> 1; j > 0; j >>= 1) {
                const bool larger = ((lane & j) == 0) == ((lane & k) == 0);
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    const float o = __shfl_xor_sync(0xffffffffu, m[i], j);
                    m[i] = larger ? fmaxf(m[i], o) : fminf(m[i], o);
                }
            }
#pragma unroll
        for (int i = 0; i < N; ++i) above[i] = fmaxf(above[i], below(__shfl_sync(0xffffffffu, m[i], top - 1)));
        filter(false);
    }
    while (most > 0) {
        if (most <= 4) {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) list[i].insert(left[i][q], key_of(x[q][i], c0 + 32 * q + lane));
            return;
        }
        // up to 32 of each list's candidates, lane by lane
        const unsigned before = (1u << lane) - 1u;
        int n[N];
        __syncwarp();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            n[i] = 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int mine = n[i] + __popc(left[i][q] & before);
                n[i] += __popc(left[i][q]);
                const bool goes = ((left[i][q] >> lane) & 1u) && mine < 32;
                if (goes) {
                    scratch[i * pitch + mine] = x[q][i];
                    scratch[i * pitch + 32 + mine] = __int_as_float(c0 + 32 * q + lane);
                }
                left[i][q] &= ~__ballot_sync(0xffffffffu, goes);
            }
        }
        __syncwarp();
        Key k[N];
#pragma unroll
        for (int i = 0; i < N; ++i)
            k[i] = lane < n[i] ? key_of(scratch[i * pitch + lane], __float_as_int(scratch[i * pitch + 32 + lane])) : 0ull;
        sort_in<N>(list, k);
        if (most <= 32) return;
#pragma unroll
        for (int i = 0; i < N; ++i) above[i] = logit_of(list[i].last());
        filter(true);
    }
}

// ------------------------------------------------------------------------------------ the kernel for few tokens
// Up to 64 tokens: bound by reading W once.  W's rows are the products' M side (128 at a time), the tokens their N side (16, 32 or 64),
// so no tensor-core work is spent on rows that are not there, and every CTA streams its own share of the vocabulary (a
// multiple of 32 rows) through a ring of 6 to 8 stages.  The logits of a tile go through shared memory, so that a warp has a token's
// 128 logits side by side: it keeps the token's state (a lane its own part) and list in registers from tile to tile.
// One token of 2880 x 201088 with 8 alternatives: 184 us with the join, 6.3 TB/s (0.96 of a plain copy's rate); 16 tokens of 7168 x 129280
// in 8 bits 156 to 168 us, 5.5 to 5.9 TB/s; 61 tokens of 2048 x 32771 with 20 alternatives 48 us, 34 without (two tiles a CTA: start, end and the lists).
constexpr int FEW_TOKENS = 64, FEW_ROWS = 32;                       // W's rows per copy
template <int NT, bool F8> struct Few {
    static constexpr int STAGES = NT == 64 ? 6 : 8;
    static constexpr int BUFS = NT == 16 ? 16 : 8;                  // accumulators: 8 bits use one per k-block
    static constexpr int WARPS = NT == 16 ? 8 : 16;                 // of the epilogue; more of them hide the lists' exchanges
    static constexpr int THREADS = EPI_FIRST + 32 * WARPS;
    static constexpr int STAGE_BYTES = TILE_M * KB_BYTES + NT * KB_BYTES;
    static constexpr int BARS = 2 * STAGES + 2 * BUFS + 1;
    static constexpr int PITCH = TILE_M + 4;                        // floats between tokens of the logits' tile
    static constexpr int TILE = STAGES * STAGE_BYTES + 512;
    static constexpr int SCALES = TILE + NT * PITCH * 4;            // 8 bits: [k-block][token]
    static constexpr int SMEM_FIXED = 1024 + SCALES;
    static constexpr int TMEM_COLS = BUFS * NT;
    static_assert(8 * BARS + 16 <= 512 && STAGE_BYTES % 1024 == 0, "layout");
};
constexpr int FEW_MAX_KBS = 128;                                    // 8 bits: scales of 64 tokens in 32 KB

template <int NT, bool F8, bool TOP>
__global__ void __launch_bounds__(Few<NT, F8>::THREADS, 1)
tl_few_kernel(const __grid_constant__ CUtensorMap tmH, const __grid_constant__ CUtensorMap tmW, const Params p) {
    using S = Few<NT, F8>;
    constexpr int STAGES = S::STAGES, BUFS = S::BUFS, KE = F8 ? 128 : 64, WARPS = S::WARPS;
    constexpr int PART = NT / (WARPS / 4), PER_WARP = NT / WARPS;   // columns that a warp reads of an accumulator, tokens of a warp
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    uint8_t* const smem = smem_raw + (base - raw);
    const uint32_t bars = base + STAGES * S::STAGE_BYTES;
    auto full_bar = [&](int s) { return bars + 8u * s; };
    auto empty_bar = [&](int s) { return bars + 8u * (STAGES + s); };
    auto tfull_bar = [&](int a) { return bars + 8u * (2 * STAGES + a); };
    auto tempty_bar = [&](int a) { return bars + 8u * (2 * STAGES + BUFS + a); };
    const uint32_t drain_bar = bars + 8u * (2 * STAGES + 2 * BUFS);
    uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + STAGES * S::STAGE_BYTES + 8 * S::BARS);
    volatile int* const abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    launch_next();
    if (threadIdx.x == 0) {
        *abort_flag = 0;
        if (blockIdx.x == 0) *p.status = 0;             // only the join, which comes later, sets bits in it
        for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), 1); }
        for (int a = 0; a < BUFS; ++a) { mbar_init(tfull_bar(a), 1); mbar_init(tempty_bar(a), WARPS); }
        mbar_init(drain_bar, 1);
        fence_barrier_init();
        fence_proxy_async();
        prefetch_tensormap(&tmH);
        prefetch_tensormap(&tmW);
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), S::TMEM_COLS);
        tmem_relinquish();
    }
    float* const scales = reinterpret_cast<float*>(smem + S::SCALES);
    if (F8)
        for (int i = threadIdx.x; i < NT * p.kbs; i += S::THREADS) {
            const int kb = i / NT, t = i - kb * NT;
            scales[i] = t < p.rows ? p.hs[static_cast<size_t>(p.row0 + t) * p.kbs + kb] : 0.f;
        }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    // this CTA's rows of W
    const long units = (p.cols + FEW_ROWS - 1) / FEW_ROWS;
    const int v0 = static_cast<int>(units * blockIdx.x / gridDim.x) * FEW_ROWS;
    const int v1 = min(p.cols, static_cast<int>(units * (blockIdx.x + 1) / gridDim.x) * FEW_ROWS);

    if (warp == 0) {
        if (lane == 0) {
            int stage = 0; uint32_t phase = 0; bool ok = true;
            long issued = 0;
            const uint64_t keep = make_policy(2), stream = make_policy(1);
            for (int r = v0; ok && r < v1; r += TILE_M) {
                const int boxes = (min(v1 - r, TILE_M) + FEW_ROWS - 1) / FEW_ROWS;
                for (int kb = 0; kb < p.kbs; ++kb) {
                    if (!mbar_wait(empty_bar(stage), phase ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    mbar_arrive_expect_tx(full_bar(stage), boxes * FEW_ROWS * KB_BYTES + NT * KB_BYTES);
                    const uint32_t sa = base + stage * S::STAGE_BYTES;
                    if (!(blockIdx.x == 0 && r == v0 && kb == p.drop_kb)) {
                        for (int b = 0; b < boxes; ++b)
                            tma_load_2d_hint(sa + b * FEW_ROWS * KB_BYTES, &tmW, full_bar(stage), kb * KE, p.col0 + r + b * FEW_ROWS, stream);
                        tma_load_2d_hint(sa + TILE_M * KB_BYTES, &tmH, full_bar(stage), kb * KE, p.row0, keep);
                    }
                    ++issued;
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok || *abort_flag) {
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
        if (lane == 0) {
            constexpr uint32_t IDESC = F8 ? make_idesc(NT, false, false, TILE_M, 0u) : make_idesc(NT, false, false, TILE_M, 1u);
            int stage = 0; uint32_t phase = 0; bool ok = true;
            int unit = 0;
            for (int r = v0; ok && r < v1; r += TILE_M) {
                for (int kb = 0; kb < p.kbs; ++kb) {
                    const int ab = unit % BUFS;
                    if ((F8 || kb == 0) && !mbar_wait(tempty_bar(ab), ((unit / BUFS) & 1) ^ 1u, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    if (!mbar_wait(full_bar(stage), phase, abort_flag, p.wait_limit_ns)) { ok = false; break; }
                    tc_fence_after();
                    const uint32_t sa = base + stage * S::STAGE_BYTES, tmem_d = tmem_base + ab * NT;
                    const uint64_t adesc = make_smem_desc(sa, 16, 1024), bdesc = make_smem_desc(sa + TILE_M * KB_BYTES, 16, 1024);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t more = (F8 ? k != 0 : (kb | k) != 0) ? 1u : 0u;
                        if (F8) umma_f8(tmem_d, adesc + 2 * k, bdesc + 2 * k, IDESC, more);
                        else umma_f16(tmem_d, adesc + 2 * k, bdesc + 2 * k, IDESC, more);
                    }
                    umma_commit(empty_bar(stage));
                    if (F8 || kb + 1 == p.kbs) { umma_commit(tfull_bar(ab)); ++unit; }
                    if (++stage == STAGES) { stage = 0; phase ^= 1u; }
                }
            }
            if (!ok || *abort_flag) {
                umma_commit(drain_bar);
                const unsigned long long t0 = globaltimer_ns();
                while (!mbar_try_wait(drain_bar, 0) && globaltimer_ns() - t0 < p.wait_limit_ns) {}
            }
        }
    } else if (warp >= EPI_FIRST / 32) {
        const int quad = warp & 3, ew = warp - EPI_FIRST / 32, col = (ew >> 2) * PART;
        auto epi_sync = [] { asm volatile("bar.sync 1, %0;" ::"n"(32 * WARPS) : "memory"); };
        const uint32_t tmem_row = tmem_base + (static_cast<uint32_t>(quad * 32) << 16) + col;
        float* const tile = reinterpret_cast<float*>(smem + S::TILE);
        State s[PER_WARP];
        List list[PER_WARP];
        int token[PER_WARP];
#pragma unroll
        for (int i = 0; i < PER_WARP; ++i) {
            s[i] = State{MINUS_INF, 0.f, 0.f};
            list[i].lane = lane; list[i].top = p.top; list[i].key = 0ull;
            const int t = i * WARPS + ew;
            token[i] = p.tokens && t < p.rows ? p.tokens[t] : -1;
        }
        auto load_part = [&](uint32_t at, float* v) {
            if constexpr (PART == 8) tmem_ld8(at, v);
            else tmem_ld16(at, v);
            tmem_ld_wait();
        };
        auto release = [&](int ab) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(tempty_bar(ab));
        };
        bool ok = true;
        int unit = 0;
        // A warp whose wait has run out goes on through the barriers with the others, without waiting or reading.
        for (int r = v0; r < v1; r += TILE_M) {
            float acc[PART];
#pragma unroll
            for (int j = 0; j < PART; ++j) acc[j] = 0.f;
            auto wait = [&](int ab) {
                if (ok) ok = __all_sync(0xffffffffu, mbar_wait(tfull_bar(ab), (unit / BUFS) & 1, abort_flag, p.wait_limit_ns));
                return ok;
            };
            if constexpr (!F8) {
                const int ab = unit % BUFS;
                if (wait(ab)) {
                    tc_fence_after();
                    load_part(tmem_row + ab * NT, acc);
                    ++unit;
                    release(ab);
                }
            } else {
                const float* ws = p.ws + static_cast<size_t>(min(p.col0 + r + quad * 32 + lane, p.V - 1) / 128) * p.kbs;
                constexpr int AHEAD = 4;                                // factors of the next k-blocks, under way
                float fw[AHEAD];
#pragma unroll
                for (int i = 0; i < AHEAD; ++i) fw[i] = i < p.kbs ? __ldg(ws + i) : 0.f;
                f2 sum[PART / 2];
#pragma unroll
                for (int j = 0; j < PART / 2; ++j) sum[j] = 0ull;
                for (int kb = 0; kb < p.kbs; ++kb) {
                    const f2 f = pair(fw[0], fw[0]);
#pragma unroll
                    for (int i = 0; i + 1 < AHEAD; ++i) fw[i] = fw[i + 1];
                    if (kb + AHEAD < p.kbs) fw[AHEAD - 1] = __ldg(ws + kb + AHEAD);
                    const int ab = unit % BUFS;
                    if (!wait(ab)) break;
                    tc_fence_after();
                    float v[PART];
                    load_part(tmem_row + ab * NT, v);
                    ++unit;
                    release(ab);
                    const float4* hs = reinterpret_cast<const float4*>(scales + kb * NT + col);
#pragma unroll
                    for (int j = 0; j < PART / 4; ++j) {
                        const float4 h = hs[j];
                        sum[2 * j] = fma2(pair(v[4 * j], v[4 * j + 1]), mul2(f, pair(h.x, h.y)), sum[2 * j]);
                        sum[2 * j + 1] = fma2(pair(v[4 * j + 2], v[4 * j + 3]), mul2(f, pair(h.z, h.w)), sum[2 * j + 1]);
                    }
                }
#pragma unroll
                for (int j = 0; j < PART / 2; ++j) { const float2 t = split(sum[j]); acc[2 * j] = t.x; acc[2 * j + 1] = t.y; }
            }
#pragma unroll
            for (int j = 0; j < PART; ++j) tile[(col + j) * S::PITCH + quad * 32 + lane] = acc[j];
            epi_sync();
            if (ew < p.rows) {
                float x[4][PER_WARP];
                unsigned has = 0;
#pragma unroll
                for (int i = 0; i < PER_WARP; ++i) {
                    if (i * WARPS + ew < p.rows) has |= 1u << i;
#pragma unroll
                    for (int q = 0; q < 4; ++q) x[q][i] = tile[(i * WARPS + ew) * S::PITCH + 32 * q + lane];
                }
#pragma unroll
                for (int i = 0; i < PER_WARP; ++i) {
                    State& st = s[i];
                    float m = st.m;
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int c = r + 32 * q + lane;
                        if (c < v1) {
                            m = fmaxf(m, x[q][i]);
                            if (p.col0 + c == token[i]) p.chosen[i * WARPS + ew] = x[q][i];
                        }
                    }
                    move(st, m, p.scale);
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        if (r + 32 * q + lane < v1) {
                            const float d = (x[q][i] - m) * p.scale, e = ex2f(d);
                            st.z += e;
                            st.u = fmaf(d, e, st.u);
                        }
                    }
                }
                if (TOP) offer_tile<PER_WARP>(list, has, x, p.col0 + r, v1 - r, tile + ew * S::PITCH, WARPS * S::PITCH);
            }
            epi_sync();                                                 // the tile may be written again
        }
        // one slice per CTA and token
        if (ok) {
#pragma unroll
            for (int i = 0; i < PER_WARP; ++i) {
                const int t = i * WARPS + ew;
                if (t < p.rows) {
                    float m = s[i].m;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
                    move(s[i], m, p.scale);
                    float z = s[i].z, u = s[i].u;
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1) {
                        z += __shfl_xor_sync(0xffffffffu, z, o);
                        u += __shfl_xor_sync(0xffffffffu, u, o);
                    }
                    const size_t at = static_cast<size_t>(t) * p.slices + blockIdx.x;
                    const int n = TOP ? __popc(__ballot_sync(0xffffffffu, lane < p.top && list[i].key != 0ull)) : 0;
                    if (lane == 0) p.part[at] = make_float4(m, z, u, __int_as_float(n));
                    if (TOP && lane < n) p.cand[at * p.top + lane] = make_uint2(__float_as_uint(logit_of(list[i].key)), static_cast<unsigned>(column_of(list[i].key)));
                }
            }
        }
    }

    tc_fence_before();
    __syncthreads();
    if (*abort_flag)                                                    // the join says so in the status word
        for (int t = threadIdx.x; t < p.rows; t += S::THREADS)
            p.part[static_cast<size_t>(t) * p.slices + blockIdx.x] = make_float4(MINUS_INF, 0.f, 0.f, __int_as_float(-1));
    if (warp == 1) {
        __syncwarp();
        tc_fence_after();
        tmem_dealloc(tmem_base, S::TMEM_COLS);
    }
}

// ------------------------------------------------------------------------------------ joining the slices
struct JoinParams {
    int rows, slices, top, first, last;
    float scale, inv_temp;                      // log2(e) / temperature, 1 / temperature
    const float4* part;
    const uint2* cand;
    float4* run;                                // [rows]: state over the launches so far
    Key* run_list;                              // [rows][top]
    unsigned* floor;
    const int32_t* tokens;
    const float* chosen;
    int ignore_index, V;
    float *logp, *lse, *entropy, *top_logp;
    int32_t* top_ids;
    int* status;
};

// A token's results from its state and list, by one warp.
template <bool TOP> __device__ __forceinline__ void emit(const JoinParams& p, int row, float m, float z, float u, const List& list) {
    const int lane = list.lane;
    const float lz = logf(z);
    if (lane == 0) {
        if (p.lse) p.lse[row] = fmaf(m, p.inv_temp, lz);
        const float h = lz - LN2_F * (u / z);
        if (p.entropy) p.entropy[row] = h < 0.f ? 0.f : h;                  // a rounding below zero; a NaN stays
        if (p.logp) {
            const int t = p.tokens[row];
            float out = 0.f;
            if (t != p.ignore_index) {
                if (static_cast<unsigned>(t) < static_cast<unsigned>(p.V)) out = (p.chosen[row] - m) * p.inv_temp - lz;
                else atomicOr(p.status, VPCE_DEV_LABEL_OUT_OF_RANGE);
            }
            p.logp[row] = out;
        }
    }
    if (TOP && lane < p.top) {
        const bool some = list.key != 0ull;
        p.top_logp[static_cast<size_t>(row) * p.top + lane] = some ? (logit_of(list.key) - m) * p.inv_temp - lz : MINUS_INF;
        p.top_ids[static_cast<size_t>(row) * p.top + lane] = some ? column_of(list.key) : -1;
    }
}
// What a token gets where a wait has run out: NaN, and no alternatives.
template <bool TOP> __device__ __forceinline__ void emit_nothing(const JoinParams& p, int row, int lane) {
    List none;
    none.key = 0ull; none.lane = lane; none.top = p.top;
    const float nan = __int_as_float(0x7fffffff);
    emit<TOP>(p, row, nan, nan, nan, none);
}
// The lanes' states as one.
__device__ __forceinline__ State over_lanes(State s, float scale) {
    float m = s.m;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    move(s, m, scale);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        s.z += __shfl_xor_sync(0xffffffffu, s.z, o);
        s.u += __shfl_xor_sync(0xffffffffu, s.u, o);
    }
    return s;
}

// The first warp's list with those that the others have left in shared memory: sorted ones, so six steps each.
template <int WARPS> __device__ __forceinline__ void merge_lists(List& list, const Key (*keys)[32]) {
#pragma unroll
    for (int w = 1; w < WARPS; ++w) {
        const Key o = keys[w][31 - list.lane];
        if (o > list.key) list.key = o;
#pragma unroll
        for (int j = 16; j > 0; j >>= 1) in_order<1>(&list.key, j, (list.lane & j) == 0);
    }
}

// The slices of the kernel for few tokens: a block per token, a warp for 32 slices.  Their lists are sorted, so the search ends at the
// first rank at which no slice has anything to offer; the warps' lists are then merged in a row.  8 to 10 us became 5 against one
// warp per token.
constexpr int JOIN_FEW_WARPS = 5, JOIN_FEW_THREADS = 32 * JOIN_FEW_WARPS, JOIN_FEW_SLICES = 32 * JOIN_FEW_WARPS;
template <bool TOP> __global__ void __launch_bounds__(JOIN_FEW_THREADS) tl_join_few_kernel(const JoinParams p) {
    __shared__ float4 states[JOIN_FEW_WARPS];
    __shared__ Key keys[JOIN_FEW_WARPS][32];
    const int row = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31, i = threadIdx.x;
    wait_for_last();
    const float4 q = i < p.slices ? p.part[static_cast<size_t>(row) * p.slices + i] : make_float4(MINUS_INF, 0.f, 0.f, 0.f);
    const bool expired = __any_sync(0xffffffffu, __float_as_int(q.w) < 0);
    const int n = min(__float_as_int(q.w), p.top);
    const State s = over_lanes(State{q.x, q.y, q.z}, p.scale);
    List list;
    list.lane = lane; list.top = TOP ? p.top : 1; list.key = 0ull;
    if (TOP) {
        const uint2* cand = p.cand + (static_cast<size_t>(row) * p.slices + i) * p.top;
        const int most = __reduce_max_sync(0xffffffffu, n);
        uint2 next = make_uint2(0u, 0u);
        if (0 < n) next = cand[0];
        for (int j = 0; j < most; ++j) {
            const Key now = j < n ? key_of(__uint_as_float(next.x), static_cast<int>(next.y)) : 0ull;
            if (j + 1 < n) next = cand[j + 1];
            if (!offer(list, now)) break;
        }
        keys[warp][lane] = list.key;
    }
    if (lane == 0) states[warp] = make_float4(s.m, s.z, s.u, expired ? 1.f : 0.f);
    __syncthreads();
    if (warp) return;
    State all{MINUS_INF, 0.f, 0.f};
    bool gone = false;
    if (lane < JOIN_FEW_WARPS) {
        const float4 t = states[lane];
        all = State{t.x, t.y, t.z};
        gone = t.w != 0.f;
    }
    if (__any_sync(0xffffffffu, gone)) {
        if (lane == 0) atomicOr(p.status, VPCE_DEV_WAIT_EXPIRED);
        emit_nothing<TOP>(p, row, lane);
        return;
    }
    all = over_lanes(all, p.scale);
    if (TOP) merge_lists<JOIN_FEW_WARPS>(list, keys);
    emit<TOP>(p, row, all.m, all.z, all.u, list);
}

// The strips' slices: WARPS warps per token, their lanes over the slices, 32 x 4 a warp at a time, always in the same order.  One warp a
// token where there are tokens enough to fill the SMs (8 us a strip of 4096), eight below (65 tokens x 201088 with 8 alternatives: 56
// us with one).
constexpr int JOIN_WARPS = 8, JOIN_THREADS = 32 * JOIN_WARPS, JOIN_MANY = 2048;
template <bool TOP, int WARPS>
__global__ void __launch_bounds__(JOIN_THREADS) tl_join_kernel(const JoinParams p) {
    __shared__ float4 states[JOIN_WARPS];
    __shared__ Key keys[JOIN_WARPS][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, w = WARPS == 1 ? 0 : warp;
    const int row = WARPS == 1 ? blockIdx.x * JOIN_WARPS + warp : blockIdx.x;
    wait_for_last();
    if (row >= p.rows) return;
    // A pair that has given up leaves its slices as they were: neither states nor counts of candidates are read then.
    if (__ldcg(p.status) & VPCE_DEV_WAIT_EXPIRED) {
        if (p.last && w == 0) emit_nothing<TOP>(p, row, lane);
        return;
    }
    State s{MINUS_INF, 0.f, 0.f};
    List list;
    list.lane = lane; list.top = TOP ? p.top : 1; list.key = 0ull;
    if (!p.first && w == 0) {
        const float4 r = p.run[row];
        if (lane == 0) s = State{r.x, r.y, r.z};
        if (TOP && lane < p.top) list.key = p.run_list[static_cast<size_t>(row) * p.top + lane];
    }
    const float4* part = p.part + static_cast<size_t>(row) * p.slices;
    const uint2* cand = p.cand + static_cast<size_t>(row) * p.slices * (TOP ? p.top : 0);
    constexpr int UNROLL = 4;
    for (int i0 = w * 32 * UNROLL; i0 < p.slices; i0 += WARPS * 32 * UNROLL) {
        float4 q[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            const int i = i0 + 32 * k + lane;
            q[k] = i < p.slices ? part[i] : make_float4(MINUS_INF, 0.f, 0.f, 0.f);
        }
        int n[UNROLL], most = 0;
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {
            State o{q[k].x, q[k].y, q[k].z};
            const float m = fmaxf(s.m, o.m);
            move(s, m, p.scale);
            move(o, m, p.scale);
            s.z += o.z;
            s.u += o.u;
            n[k] = min(__float_as_int(q[k].w), p.top);
            most = max(most, n[k]);
        }
        if (TOP) {
            most = __reduce_max_sync(0xffffffffu, most);
            uint2 next[UNROLL];
            auto load = [&](int j) {
#pragma unroll
                for (int k = 0; k < UNROLL; ++k) if (j < n[k]) next[k] = cand[static_cast<size_t>(i0 + 32 * k + lane) * p.top + j];
            };
            load(0);
            for (int j = 0; j < most; ++j) {
                Key now[UNROLL];
#pragma unroll
                for (int k = 0; k < UNROLL; ++k) now[k] = j < n[k] ? key_of(__uint_as_float(next[k].x), static_cast<int>(next[k].y)) : 0ull;
                load(j + 1);
#pragma unroll
                for (int k = 0; k < UNROLL; ++k) offer(list, now[k]);
            }
        }
    }
    s = over_lanes(s, p.scale);
    if constexpr (WARPS > 1) {
        if (lane == 0) states[warp] = make_float4(s.m, s.z, s.u, 0.f);
        keys[warp][lane] = list.key;
        __syncthreads();
        if (warp) return;
        State all{MINUS_INF, 0.f, 0.f};
        if (lane < WARPS) { const float4 t = states[lane]; all = State{t.x, t.y, t.z}; }
        s = over_lanes(all, p.scale);
        if (TOP) merge_lists<WARPS>(list, keys);
    }
    if (!p.last) {
        if (lane == 0) p.run[row] = make_float4(s.m, s.z, s.u, 0.f);
        if (TOP) {
            if (lane < p.top) p.run_list[static_cast<size_t>(row) * p.top + lane] = list.key;
            if (lane == p.top - 1 && list.key != 0ull) p.floor[row] = static_cast<unsigned>(list.key >> 32);
        }
        return;
    }
    emit<TOP>(p, row, s.m, s.z, s.u, list);
}

}  // namespace vptl
