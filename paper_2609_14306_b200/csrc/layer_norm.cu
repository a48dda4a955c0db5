// Layer normalisation, forward and backward (layer_norm.h).
//
// Row kernels (16-bit rows of up to 16384 columns, fp32 ones of up to 14336 forward and 11320 backward: two rows in flight and the
// weights as fp32 have to fit shared memory): a group of 1 to 16 warps owns a row at a time, 8 to 32 elements a thread.  Rows arrive by bulk
// copies into a ring in shared memory, several rows ahead: what is in flight does not depend on registers or on how many warps
// wait at a reduction.  A thread owns the same columns in every row: in the backward pass it sums dy xh and dy of its columns
// in registers over all rows of its group, so the weight's gradient costs no second pass over the data, only one partial sum
// per block.  The variance is taken from the centred values in registers.  Bound: memory, two passes over the rows forward,
// three backward; at 16-bit types the arithmetic is nearly as scarce, so it runs on pairs (fp32x2 instructions).  Measured on
// 65536 x 7168 bf16, fp32 weights: 299 us forward, 426 us backward (6.3 and 6.6 TB/s, the rate of a plain copy), 845 us for
// both in sustained repetition (796 on another board), where the lowered clock shows the arithmetic; 16384 x 2880: 102 us for both.
// Spills matter: 24 to 60 bytes in the row loop cost 10 to 25 %.  The aligned row kernels have none; the unaligned backward ones of
// 24 and 32 elements a thread have 4 and 20 bytes.
//   VEC      every row starts on a 16-byte boundary: 16-byte accesses
//   !VEC     any alignment: the copies take the 16-byte granules that a row touches (cut at the tensor's ends, whose few
//            elements are copied one by one), threads read single elements at the row's offset, neighbours side by side:
//            2.8 to 4.3 TB/s forward and 2.7 to 3.6 backward in 16 bits, where VEC has 4.7 to 5.7 and 3.4 to 5.3 (2^26 elements,
//            512 to 16384 columns: 0.58 to 0.79 of its rate); 5.3 and 4.8 in fp32, where VEC has 5.4 and 5.9
//
// Generic kernels (wider rows): one block per row, elements read one at a time in the order of the threads, three passes over
// a row that the caches hold after the first, and a pass of their own for the column sums.  Slow: 2^26 elements take 187 and 567 us
// at 16384 columns of fp32 (floor 82 and 123), 555 backward at 12288 (row kernel forward: 97), 175 and 542 at 20000 of bf16 (floor
// 41 and 62).
//
// Narrow kernels (aligned rows of up to 512 bytes): several rows to a warp, see there.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cstdint>
#include <type_traits>

#include "layer_norm.h"
#include "sm100_ptx.cuh"
#include "vp_ce.h"

namespace {

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

constexpr int GEN_THREADS = 256;
constexpr int COL_TILE = 32;            // columns per block of the column sums
constexpr int COL_ROWS = 8;             // rows that a block of the column sums takes at a time
constexpr int MAX_SLICES = 296;         // partial sums over rows: two blocks per SM of a 148-SM device

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Sum of two values over the block; every thread receives both.
template <int THREADS>
__device__ __forceinline__ float2 block_sum2(float a, float b, float2* part) {
    a = warp_sum(a);
    b = warp_sum(b);
    __syncthreads();                                        // the last use of `part` is over
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = make_float2(a, b);
    __syncthreads();
    float2 s = make_float2(0.f, 0.f);
#pragma unroll
    for (int i = 0; i < THREADS / 32; ++i) { s.x += part[i].x; s.y += part[i].y; }
    return s;
}

// ------------------------------------------------------------------------------------ row kernels
constexpr int MAX_GROUP_WARPS = 16;
// One block per SM.  Forward: 28 warps of 72 registers (a row's 32 elements a thread and what is worked on); backward: 16 warps
// of 128 (64 column sums).
constexpr int FORWARD_REGS = 72, FORWARD_WARPS = 28, BACKWARD_REGS = 128, BACKWARD_WARPS = 16;
constexpr int MAX_GROUPS = FORWARD_WARPS;               // per block; a group of more than one warp has a named barrier
constexpr int MAX_STAGES = 8;
constexpr int MAX_EPT = 32;                             // elements per thread
constexpr int MAX_SMEM = 227 * 1024;
constexpr int64_t MAX_ROWS = (int64_t{1} << 31) - (1 << 20);   // row numbers and the look-ahead stay below 2^31
constexpr int64_t MAX_ROW = 32 * MAX_GROUP_WARPS * MAX_EPT;

// Shared memory of a block: barriers [MAX_GROUPS][MAX_STAGES], weights, reduction scratch (`part`, float2 [group][turn][warp]), ring.
// The scratch is for the groups that the launch has: at 8192 columns of 16 bits that is what lets the backward pass's two groups
// have three stages each (two: 108 us for 8192 rows, three: 82).
constexpr int FULL_BYTES = MAX_GROUPS * MAX_STAGES * 8, PART_BYTES = 2 * MAX_GROUP_WARPS * 8;
static_assert(FULL_BYTES % 128 == 0 && PART_BYTES % 128 == 0, "what follows begins on a 128-byte boundary");

__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// An array's rows, as the launch gives them (used where needed rather than kept in registers).
struct Rows {
    const void* base;
    long pitch;                                         // bytes between rows
    __device__ __forceinline__ const char* at(int r) const { return static_cast<const char*>(base) + r * pitch; }
    // bytes by which row r starts behind a 16-byte boundary
    __device__ __forceinline__ uint32_t shift(int r) const {
        return (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(base)) + static_cast<uint32_t>(r) * static_cast<uint32_t>(pitch)) & 15u;
    }
};

struct RowArgs {
    Rows x, dy;                                         // dy: backward only
    int rows, d, warps;                                 // warps per group
    int groups, stages, cap, slot;                      // groups per block, ring depth, bytes of a row and of a slot in the ring
    int ring;                                           // byte offset of the ring in shared memory
    long out_stride;
    const void *g, *b;
    float eps;
    void* out;                                          // y or dx (may be null in the backward pass)
    float *mean, *rstd;                                 // written (forward, may be null) or read (backward)
    float* partial;                                     // [blocks][2][d] or null
};
// The same, longer.  With more than 112 bytes of arguments the compiler keeps them in registers instead of reading them where they
// are used.  That serves the forward kernels (2^26 bf16 elements: 54 us instead of 58 at 10000 columns, 52 instead of 56 at 64)
// and the backward pass on unaligned rows (120 instead of 170 at 2881); on aligned rows that spills and
// takes 91 instead of 78.  So with nvcc 12.9; a compiler that decides otherwise costs that much speed and nothing else.
struct LongRowArgs : RowArgs { int64_t none; };
template <typename Args> Args args_of(const RowArgs& a) {
    Args r{};
    static_cast<RowArgs&>(r) = a;
    return r;
}
template <bool VEC> using BackwardArgs = std::conditional_t<VEC, RowArgs, LongRowArgs>;

// What row r of an array takes: `*from`, the address from which the bulk copy reads, `*at`, where it lands in the slot, and the
// bytes that it moves.  The row's first element lands shift(r) bytes into the slot.  A granule that reaches over the tensor's
// first or last byte is left to plain element copies, made here.
template <typename T, bool VEC>
__device__ __forceinline__ uint32_t copy_extent(const Rows& a, int r, int rows, int d, const char** from, uint32_t* at, uint8_t* slot) {
    const char* row = a.at(r);
    const size_t bytes = static_cast<size_t>(d) * sizeof(T);
    if (VEC) { *from = row; *at = 0; return static_cast<uint32_t>(bytes); }
    const uintptr_t lo = reinterpret_cast<uintptr_t>(row), hi = lo + bytes;
    uintptr_t b = lo & ~static_cast<uintptr_t>(15), e = (hi + 15) & ~static_cast<uintptr_t>(15);
    const uintptr_t origin = b;
    // by address, not by row number: several rows may lie in the tensor's first granule
    const uintptr_t begin = reinterpret_cast<uintptr_t>(a.base), end = reinterpret_cast<uintptr_t>(a.at(rows - 1)) + bytes;
    if (b < begin || e > end) {
        if (b < begin) b += 16;
        if (e > end) e -= 16;
        if (e < b) e = b;
        const T* src = reinterpret_cast<const T*>(lo);
        T* dst = reinterpret_cast<T*>(slot + (lo - origin));
        for (int c = 0; c < d && lo + c * sizeof(T) < b; ++c) dst[c] = src[c];
        for (int c = d - 1; c >= 0 && lo + c * sizeof(T) >= e; --c) dst[c] = src[c];
    }
    *from = reinterpret_cast<const char*>(b);
    *at = static_cast<uint32_t>(b - origin);
    return static_cast<uint32_t>(e - b);
}

// One thread: row r of the NA arrays into ring slot `slot`, signalled on `bar`.  With dy the row's mean and rstd come along, to
// the slot's end (the barrier counts their arrival, too).
template <typename T, bool VEC, int NA>
__device__ __forceinline__ void fetch_row(const RowArgs& a, int r, uint8_t* slot, uint32_t bar) {
    const char* from[NA];
    uint32_t at[NA], bytes[NA], total = 0;
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        bytes[i] = copy_extent<T, VEC>(i ? a.dy : a.x, r, a.rows, a.d, &from[i], &at[i], slot + i * a.cap);
        total += bytes[i];
    }
    const uint32_t dst = vpce::smem_u32(slot);
    if (!VEC) vpce::fence_proxy_async();                    // plain stores to a slot come before a later row's bulk copy to it
    if (NA == 2) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + 2 * a.cap), "l"(a.mean + r) : "memory");
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + 2 * a.cap + 4), "l"(a.rstd + r) : "memory");
        asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
    }
    vpce::mbar_arrive_expect_tx(bar, total);
#pragma unroll
    for (int i = 0; i < NA; ++i)
        if (bytes[i]) bulk_load(dst + i * a.cap + at[i], from[i], bytes[i], bar);
}

// All waits are for bulk copies of this block's own from arrays that the caller vouches for, so they end.  The limit only keeps a copy
// that never lands from hanging the GPU; what is computed then is undefined and not reported: a flag in the row loop, in any of the
// forms tried, costs the widest backward kernel 24 to 150 bytes of spill.
__device__ __forceinline__ void wait_row(uint32_t bar, uint32_t parity) {
    for (int i = 0; i < (1 << 26); ++i)
        if (vpce::mbar_try_wait(bar, parity)) return;
}

__device__ __forceinline__ void group_sync(int group, int warps) {
    if (warps == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(warps * 32) : "memory");
}

// Sum over 16 neighbouring lanes; after a group's barrier lane l of either half holds what warp l has left.
__device__ __forceinline__ float half_warp_sum(float v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float ld_shared(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// Pairs of fp32 in one 64-bit register.
using f2 = unsigned long long;
__device__ __forceinline__ f2 pair(float a, float b) { f2 r; asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float2 split(f2 v) { float2 r; asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v)); return r; }
__device__ __forceinline__ f2 add2(f2 a, f2 b) { f2 r; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) { f2 r; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b)); return r; }
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) { f2 r; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c)); return r; }

template <typename T> __device__ __forceinline__ f2 widen(uint32_t w);      // two 16-bit elements of a word
template <> __device__ __forceinline__ f2 widen<__nv_bfloat16>(uint32_t w) { return pair(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <> __device__ __forceinline__ f2 widen<__half>(uint32_t w) {
    const float2 t = __half22float2(*reinterpret_cast<const __half2*>(&w));
    return pair(t.x, t.y);
}
template <typename T> __device__ __forceinline__ uint32_t narrow(float a, float b);
template <> __device__ __forceinline__ uint32_t narrow<__nv_bfloat16>(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}
template <> __device__ __forceinline__ uint32_t narrow<__half>(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// A thread's EPT columns: a warp owns 32 EPT neighbouring columns, in pieces of 32 N: lane l has N neighbours of each (N = 16 /
// sizeof(T) where VEC, else 1).  Piece k begins at column first + 32 N k; pairs are neighbours in the thread's order.
// SPLIT: code of its own for warps that have all their columns (it pays in the forward pass, not in the longer backward one).
template <typename T, bool VEC, int EPT, bool SPLIT> struct Columns {
    static constexpr int N = VEC ? 16 / static_cast<int>(sizeof(T)) : 1;
    static constexpr int PAIRS = EPT / 2, STEP = 32 * N, PART = 8 / N;
    int first, d;
    bool all;                                           // no lane of the warp lacks a column
    __device__ __forceinline__ Columns(int warp, int lane, int d_) : first(warp * 32 * EPT + lane * N), d(d_), all((warp + 1) * 32 * EPT <= d_) {}
    __device__ __forceinline__ bool has(int k) const { return first + STEP * k < d; }    // VEC: d is a multiple of N

    // Eight of the thread's elements (part q of EPT / 8) of a row in shared memory (address of its first element); columns beyond
    // d read as 0.
    __device__ __forceinline__ void read(uint32_t row, int q, f2* v) const {
        const uint32_t at = row + (first + STEP * q * PART) * static_cast<int>(sizeof(T));
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < PART; ++k) {
                uint32_t w[4] = {0u, 0u, 0u, 0u};
                if (has(q * PART + k)) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at + k * 512));
                if constexpr (sizeof(T) == 4) {
                    v[2 * k] = pair(__uint_as_float(w[0]), __uint_as_float(w[1]));
                    v[2 * k + 1] = pair(__uint_as_float(w[2]), __uint_as_float(w[3]));
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[4 * k + i] = widen<T>(w[i]);
                }
            }
        } else {
            if (SPLIT && all) read_single<true>(at, q, v);
            else read_single<false>(at, q, v);
        }
    }
    template <bool ALL> __device__ __forceinline__ void read_single(uint32_t at, int q, f2* v) const {
        if constexpr (sizeof(T) == 4) {
            float f[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                f[k] = 0.f;
                if (ALL || has(q * PART + k)) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(f[k]) : "r"(at + k * 128));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = pair(f[2 * i], f[2 * i + 1]);
        } else {
            uint16_t h[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                h[k] = 0;
                if (ALL || has(q * PART + k)) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h[k]) : "r"(at + k * 64));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = widen<T>(static_cast<uint32_t>(h[2 * i]) | static_cast<uint32_t>(h[2 * i + 1]) << 16);
        }
    }

    // Weights as fp32 in shared memory, in the order of the threads' elements: four of a lane's in 16 bytes, lanes side by side.
    // fill: this warp's (W of any alignment; `none` where p is null; 0 beyond d); weights: part q of this thread's.
    template <typename W> __device__ __forceinline__ void fill(float* to, int warp, int lane, const W* p, float none) const {
        float f[EPT];
#pragma unroll
        for (int e = 0; e < EPT; ++e) f[e] = has(e / N) ? (p ? to_f(p[first + STEP * (e / N) + e % N]) : none) : 0.f;
#pragma unroll
        for (int e = 0; e < EPT; e += 4)
            *reinterpret_cast<float4*>(to + ((warp * (EPT / 4) + e / 4) * 32 + lane) * 4) = make_float4(f[e], f[e + 1], f[e + 2], f[e + 3]);
    }
    __device__ __forceinline__ void weights(uint32_t at, int q, f2* v) const {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[2 * i]), "=l"(v[2 * i + 1]) : "r"(at + (2 * q + i) * 512));
    }

    __device__ __forceinline__ void store(T* row, int q, const f2* v) const {
        T* at = row + first + STEP * q * PART;
        if constexpr (VEC) {
#pragma unroll
            for (int k = 0; k < PART; ++k) {
                uint32_t w[4];
                if constexpr (sizeof(T) == 4) {
                    const float2 a = split(v[2 * k]), b = split(v[2 * k + 1]);
                    w[0] = __float_as_uint(a.x); w[1] = __float_as_uint(a.y); w[2] = __float_as_uint(b.x); w[3] = __float_as_uint(b.y);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) { const float2 a = split(v[4 * k + i]); w[i] = narrow<T>(a.x, a.y); }
                }
                if (has(q * PART + k)) *reinterpret_cast<uint4*>(at + STEP * k) = make_uint4(w[0], w[1], w[2], w[3]);
            }
        } else {
            if (SPLIT && all) store_single<true>(at, q, v);
            else store_single<false>(at, q, v);
        }
    }
    template <bool ALL> __device__ __forceinline__ void store_single(T* at, int q, const f2* v) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 a = split(v[i]);
            if (ALL || has(q * PART + 2 * i)) at[STEP * (2 * i)] = from_f<T>(a.x);
            if (ALL || has(q * PART + 2 * i + 1)) at[STEP * (2 * i + 1)] = from_f<T>(a.y);
        }
    }
};

// What every row kernel sets up: the group's place and its ring.
struct Group {
    int id, warp, lane;
    int first, step;                                    // rows of this group: first, first + step, ...
    uint8_t* ring;
    uint32_t bars;
};
template <typename T, bool VEC, int NA>
__device__ __forceinline__ Group group_setup(const RowArgs& a, uint8_t* raw) {
    Group g;
    g.id = (threadIdx.x >> 5) / a.warps;
    g.warp = (threadIdx.x >> 5) - g.id * a.warps;
    g.lane = threadIdx.x & 31;
    g.first = blockIdx.x * a.groups + g.id;
    g.step = gridDim.x * a.groups;
    g.ring = raw + a.ring + g.id * a.stages * a.slot;
    g.bars = vpce::smem_u32(raw) + g.id * MAX_STAGES * 8;
    if (g.warp == 0 && g.lane == 0) {
        for (int s = 0; s < a.stages; ++s) vpce::mbar_init(g.bars + 8 * s, NA);
        vpce::fence_barrier_init();
        vpce::fence_proxy_async();
    }
    group_sync(g.id, a.warps);
    if (g.warp == 0 && g.lane == 0)
        for (int s = 0; s < a.stages; ++s) {
            const int r = g.first + s * g.step;
            if (r < a.rows) fetch_row<T, VEC, NA>(a, r, g.ring + s * a.slot, g.bars + 8 * s);
        }
    return g;
}

template <typename T, typename W, bool VEC, int EPT>
__global__ void __maxnreg__(FORWARD_REGS) ln_forward_rows(const LongRowArgs a) {
    extern __shared__ __align__(128) uint8_t raw[];
    const Group g = group_setup<T, VEC, 1>(a, raw);
    const Columns<T, VEC, EPT, true> cols(g.warp, g.lane, a.d);
    using C = Columns<T, VEC, EPT, true>;
    float* const weights = reinterpret_cast<float*>(raw + FULL_BYTES);
    const int n_weights = 32 * EPT * a.warps;
    if (g.id == 0) cols.fill(weights, g.warp, g.lane, static_cast<const W*>(a.g), 1.f);
    if (g.id == a.groups - 1) cols.fill(weights + n_weights, g.warp, g.lane, static_cast<const W*>(a.b), 0.f);
    __syncthreads();
    const uint32_t gw = vpce::smem_u32(weights) + (g.warp * (EPT / 4) * 32 + g.lane) * 16, bw = gw + 4 * n_weights;
    float2(*part)[MAX_GROUP_WARPS] = reinterpret_cast<float2(*)[MAX_GROUP_WARPS]>(raw + a.ring - (a.groups - g.id) * PART_BYTES);
    const float inv_d = 1.f / static_cast<float>(a.d);
    auto columns_of = [&](int warp) { return static_cast<float>(min(max(a.d - warp * 32 * EPT, 0), 32 * EPT)); };
    const float inv_mine = 1.f / columns_of(g.warp);
    const float n_lane = (g.lane & 15) < a.warps ? columns_of(g.lane & 15) : 0.f;
    const float inv_lane = n_lane > 0.f ? 1.f / n_lane : 0.f;
    int s = 0, pass = 0, turn = 0;                                          // the warps take turns at starting copies
    uint32_t parity = 0;
    for (int r = g.first; r < a.rows; r += g.step) {
        const uint32_t xr = vpce::smem_u32(g.ring + s * a.slot) + (VEC ? 0u : a.x.shift(r));
        wait_row(g.bars + 8 * s, parity);
        f2 v[C::PAIRS];
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) cols.read(xr, q, v + 4 * q);
        // A warp's statistics: its columns' sum, and the sum of the squares around their own mean, which needs no other warp.
        f2 s0 = v[0], s1 = v[1];
#pragma unroll
        for (int i = 2; i < C::PAIRS; i += 2) { s0 = add2(s0, v[i]); s1 = add2(s1, v[i + 1]); }
        const float2 t = split(add2(s0, s1));
        const float sum = warp_sum(t.x + t.y), mine = sum * inv_mine;
        const f2 minus = pair(-mine, -mine);
        f2 q0 = 0ull, q1 = 0ull;
        if (cols.all) {
#pragma unroll
            for (int i = 0; i < C::PAIRS; i += 2) {
                const f2 e = add2(v[i], minus), f = add2(v[i + 1], minus);
                q0 = fma2(e, e, q0);
                q1 = fma2(f, f, q1);
            }
        } else {                                                            // columns beyond d count nothing
#pragma unroll
            for (int i = 0; i < C::PAIRS; ++i) {
                const float2 e = split(add2(v[i], minus));
                const f2 f = pair(cols.has(2 * i / C::N) ? e.x : 0.f, cols.has((2 * i + 1) / C::N) ? e.y : 0.f);
                q0 = fma2(f, f, q0);
            }
        }
        const float2 u = split(add2(q0, q1));
        const float squares = warp_sum(u.x + u.y);
        if (g.lane == 0) part[pass][g.warp] = make_float2(sum, squares);
        group_sync(g.id, a.warps);
        // everyone has read the slot: it takes the next row that is not under way yet
        if (g.warp == turn && g.lane == 0 && r + a.stages * g.step < a.rows) fetch_row<T, VEC, 1>(a, r + a.stages * g.step, g.ring + s * a.slot, g.bars + 8 * s);
        if (++turn == a.warps) turn = 0;
        if (++s == a.stages) { s = 0; parity ^= 1u; }
        // The row's statistics from the warps': squares around the row's mean = sum of theirs + n (their mean - the row's)^2.
        const float2 w = (g.lane & 15) < a.warps ? part[pass][g.lane & 15] : make_float2(0.f, 0.f);
        pass ^= 1;
        const float mu = half_warp_sum(w.x) * inv_d;
        const float off = w.x * inv_lane - mu;
        const float rs = 1.f / sqrtf(half_warp_sum(fmaf(n_lane * off, off, w.y)) * inv_d + a.eps);
        // (x - mu) rs as x rs - mu rs: the rounding of mu rs is that of mu itself
        const f2 minus_mu = pair(-mu * rs, -mu * rs), rs2 = pair(rs, rs);
        T* out = static_cast<T*>(a.out) + r * a.out_stride;
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) {
            f2 gq[4], bq[4];
            cols.weights(gw, q, gq);
            cols.weights(bw, q, bq);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * q + i] = fma2(fma2(v[4 * q + i], rs2, minus_mu), gq[i], bq[i]);
            cols.store(out, q, v + 4 * q);
        }
        if (g.warp == 0 && g.lane == 0) {
            if (a.mean) a.mean[r] = mu;
            if (a.rstd) a.rstd[r] = rs;
        }
    }
}

template <typename T, typename W, bool VEC, int EPT>
__global__ void __maxnreg__(BACKWARD_REGS) ln_backward_rows(const BackwardArgs<VEC> a) {
    extern __shared__ __align__(128) uint8_t raw[];
    const Group g = group_setup<T, VEC, 2>(a, raw);
    const Columns<T, VEC, EPT, false> cols(g.warp, g.lane, a.d);
    using C = Columns<T, VEC, EPT, false>;
    float2(*part)[MAX_GROUP_WARPS] = reinterpret_cast<float2(*)[MAX_GROUP_WARPS]>(raw + a.ring - (a.groups - g.id) * PART_BYTES);
    const float inv_d = 1.f / static_cast<float>(a.d);
    float* const weights = reinterpret_cast<float*>(raw + FULL_BYTES);
    if (g.id == 0) cols.fill(weights, g.warp, g.lane, static_cast<const W*>(a.g), 1.f);
    __syncthreads();
    const uint32_t gw = vpce::smem_u32(weights) + (g.warp * (EPT / 4) * 32 + g.lane) * 16;
    f2 dg[C::PAIRS], db[C::PAIRS];
#pragma unroll
    for (int i = 0; i < C::PAIRS; ++i) dg[i] = db[i] = 0ull;
    // The row is read from the ring twice, before and after the group's sums: the registers that would keep it hold the column
    // sums.  Weights of columns beyond d are 0, so those columns add nothing to the sums.  The first reading of a row comes
    // before the second reading of the row before it, so the group's barrier finds everyone with work in between.
    auto slot_of = [&](int s) { return g.ring + s * a.slot; };
    auto first_reading = [&](int r, int s, uint32_t parity, float2* to) {
        const uint32_t slot = vpce::smem_u32(slot_of(s));
        const uint32_t xr = slot + (VEC ? 0u : a.x.shift(r)), dyr = slot + a.cap + (VEC ? 0u : a.dy.shift(r));
        wait_row(g.bars + 8 * s, parity);
        const float mu = ld_shared(slot + 2 * a.cap), rs = ld_shared(slot + 2 * a.cap + 4);
        const f2 minus_mu = pair(-mu * rs, -mu * rs), rs2 = pair(rs, rs);   // xh = x rs - mu rs
        f2 sa = 0ull, sax = 0ull;
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) {
            f2 x[4], u[4], gq[4];
            cols.read(xr, q, x);
            cols.read(dyr, q, u);
            cols.weights(gw, q, gq);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f2 t = mul2(u[i], gq[i]);
                sa = add2(sa, t);
                sax = fma2(t, fma2(x[i], rs2, minus_mu), sax);
            }
        }
        const float2 pa = split(sa), pax = split(sax);
        const float2 v = make_float2(warp_sum(pa.x + pa.y), warp_sum(pax.x + pax.y));
        if (g.lane == 0) to[g.warp] = v;
    };
    if (g.first < a.rows) {
        int s = 0, pass = 0, turn = 0;                                      // the warps take turns at starting copies
        uint32_t parity = 0;
        first_reading(g.first, 0, 0u, part[0]);
        for (int r = g.first; r < a.rows; r += g.step) {
            group_sync(g.id, a.warps);
            float2 t = make_float2(0.f, 0.f);
            if ((g.lane & 15) < a.warps) t = part[pass][g.lane & 15];
            t.x = half_warp_sum(t.x);
            t.y = half_warp_sum(t.y);
            pass ^= 1;
            const int here = s;
            if (++s == a.stages) { s = 0; parity ^= 1u; }
            // the slot of the row before is spent: it takes the next row that is not under way yet
            if (g.warp == turn && g.lane == 0 && r > g.first && r + (a.stages - 1) * g.step < a.rows) {
                const int before = here == 0 ? a.stages - 1 : here - 1;
                fetch_row<T, VEC, 2>(a, r + (a.stages - 1) * g.step, slot_of(before), g.bars + 8 * before);
            }
            if (++turn == a.warps) turn = 0;
            if (r + g.step < a.rows) first_reading(r + g.step, s, parity, part[pass]);
            const uint32_t slot = vpce::smem_u32(slot_of(here));
            const uint32_t xr = slot + (VEC ? 0u : a.x.shift(r)), dyr = slot + a.cap + (VEC ? 0u : a.dy.shift(r));
            const float mu = ld_shared(slot + 2 * a.cap), rs = ld_shared(slot + 2 * a.cap + 4);
            const float ma = -rs * t.x * inv_d, mx = -rs * t.y * inv_d;
            const f2 minus_mu = pair(-mu * rs, -mu * rs), rs2 = pair(rs, rs), ma2 = pair(ma, ma), mx2 = pair(mx, mx);
            T* dx = static_cast<T*>(a.out) + r * a.out_stride;
#pragma unroll
            for (int q = 0; q < EPT / 8; ++q) {
                f2 x[4], u[4], gq[4];
                cols.read(xr, q, x);
                cols.read(dyr, q, u);
                cols.weights(gw, q, gq);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f2 xh = fma2(x[i], rs2, minus_mu);
                    dg[4 * q + i] = fma2(u[i], xh, dg[4 * q + i]);
                    db[4 * q + i] = add2(u[i], db[4 * q + i]);
                    x[i] = fma2(mul2(u[i], gq[i]), rs2, fma2(xh, mx2, ma2));
                }
                if (a.out) cols.store(dx, q, x);
            }
        }
    }
    if (!a.partial) return;
    // The block's sums: every group leaves its own in the ring (all copies have landed and been read), then all threads add
    // them, the groups in order.
    float* sums = reinterpret_cast<float*>(raw + a.ring);
    __syncthreads();
    float* mine = sums + static_cast<size_t>(g.id) * 2 * a.d;
#pragma unroll
    for (int i = 0; i < C::PAIRS; ++i) {
        const float2 p = split(dg[i]), q = split(db[i]);
        const int c0 = cols.first + C::STEP * (2 * i / C::N) + 2 * i % C::N, c1 = cols.first + C::STEP * ((2 * i + 1) / C::N) + (2 * i + 1) % C::N;
        if (c0 < a.d) { mine[c0] = p.x; mine[a.d + c0] = q.x; }
        if (c1 < a.d) { mine[c1] = p.y; mine[a.d + c1] = q.y; }
    }
    __syncthreads();
    float* out = a.partial + static_cast<size_t>(blockIdx.x) * 2 * a.d;
    for (int c = threadIdx.x; c < 2 * a.d; c += blockDim.x) {
        float v = sums[c];
        for (int q = 1; q < a.groups; ++q) v += sums[static_cast<size_t>(q) * 2 * a.d + c];
        out[c] = v;
    }
}

// ------------------------------------------------------------------------------------ narrow rows
// Rows of up to 512 bytes on 16-byte boundaries (a norm over one head's 64 to 256 elements): L lanes hold a row, 16 bytes each,
// so a warp has 32 / L rows at once, and UNROLL times as many under way.  A ring would be all barriers here: 2^26 bf16
// elements take 52 us forward and 75 backward here at any of these widths; in the ring 285 and 408 at 64 columns, 147 and 211 at
// 128, 78 and 115 at 256.
constexpr int NARROW_BYTES = 512, NARROW_THREADS = 512, NARROW_WARPS = NARROW_THREADS / 32, UNROLL = 4;

template <int L> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
// 16 bytes as pairs, and back.
template <typename T> struct Piece {
    static constexpr int N = 16 / static_cast<int>(sizeof(T)), PAIRS = N / 2;
    __device__ static __forceinline__ void unpack(uint4 q, f2* v) {
        if constexpr (sizeof(T) == 4) {
            v[0] = pair(__uint_as_float(q.x), __uint_as_float(q.y));
            v[1] = pair(__uint_as_float(q.z), __uint_as_float(q.w));
        } else {
            v[0] = widen<T>(q.x); v[1] = widen<T>(q.y); v[2] = widen<T>(q.z); v[3] = widen<T>(q.w);
        }
    }
    __device__ static __forceinline__ uint4 pack(const f2* v) {
        uint32_t w[4];
        if constexpr (sizeof(T) == 4) {
            const float2 a = split(v[0]), b = split(v[1]);
            w[0] = __float_as_uint(a.x); w[1] = __float_as_uint(a.y); w[2] = __float_as_uint(b.x); w[3] = __float_as_uint(b.y);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) { const float2 a = split(v[i]); w[i] = narrow<T>(a.x, a.y); }
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    }
    template <typename W> __device__ static __forceinline__ void weights(const W* p, int c, bool has, float none, f2* v) {
#pragma unroll
        for (int i = 0; i < PAIRS; ++i) {
            const float a = has ? (p ? to_f(p[c + 2 * i]) : none) : 0.f, b = has ? (p ? to_f(p[c + 2 * i + 1]) : none) : 0.f;
            v[i] = pair(a, b);
        }
    }
};

template <typename T, typename W, int L>
__global__ void __launch_bounds__(NARROW_THREADS) ln_forward_narrow(const LongRowArgs a) {
    using P = Piece<T>;
    constexpr int PER = 32 / L;                         // rows of a warp at once
    const int lane = threadIdx.x & 31, c = (lane & (L - 1)) * P::N;
    const bool has = c < a.d;
    const float inv_d = 1.f / static_cast<float>(a.d);
    f2 gw[P::PAIRS], bw[P::PAIRS];
    P::weights(static_cast<const W*>(a.g), c, has, 1.f, gw);
    P::weights(static_cast<const W*>(a.b), c, has, 0.f, bw);
    const int step = gridDim.x * NARROW_WARPS * PER * UNROLL;
    for (int r0 = (blockIdx.x * NARROW_WARPS + (threadIdx.x >> 5)) * PER * UNROLL; r0 < a.rows; r0 += step) {
        uint4 q[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int r = r0 + u * PER + lane / L;
            q[u] = make_uint4(0u, 0u, 0u, 0u);
            if (has && r < a.rows) q[u] = *reinterpret_cast<const uint4*>(a.x.at(r) + c * sizeof(T));
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int r = r0 + u * PER + lane / L;
            f2 v[P::PAIRS];
            P::unpack(q[u], v);
            f2 sum = v[0];
#pragma unroll
            for (int i = 1; i < P::PAIRS; ++i) sum = add2(sum, v[i]);
            const float2 t = split(sum);
            const float mu = lanes_sum<L>(t.x + t.y) * inv_d;
            const f2 minus = has ? pair(-mu, -mu) : 0ull;                   // lanes beyond d hold 0 and stay 0
            f2 sq = 0ull;
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) { v[i] = add2(v[i], minus); sq = fma2(v[i], v[i], sq); }
            const float2 w = split(sq);
            const float rs = 1.f / sqrtf(lanes_sum<L>(w.x + w.y) * inv_d + a.eps);
            const f2 rs2 = pair(rs, rs);
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) v[i] = fma2(mul2(v[i], rs2), gw[i], bw[i]);
            if (r < a.rows) {
                if (has) *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + r * a.out_stride + c) = P::pack(v);
                if (c == 0) {
                    if (a.mean) a.mean[r] = mu;
                    if (a.rstd) a.rstd[r] = rs;
                }
            }
        }
    }
}

template <typename T, typename W, int L>
__global__ void __launch_bounds__(NARROW_THREADS, 2) ln_backward_narrow(const RowArgs a) {
    using P = Piece<T>;
    constexpr int PER = 32 / L, ROWS = UNROLL / 2;
    __shared__ float sums[NARROW_WARPS][2][NARROW_BYTES / 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (lane & (L - 1)) * P::N;
    const bool has = c < a.d;
    const float inv_d = 1.f / static_cast<float>(a.d);
    f2 gw[P::PAIRS], dg[P::PAIRS], db[P::PAIRS];
    P::weights(static_cast<const W*>(a.g), c, has, 1.f, gw);
#pragma unroll
    for (int i = 0; i < P::PAIRS; ++i) dg[i] = db[i] = 0ull;
    const int step = gridDim.x * NARROW_WARPS * PER * ROWS;
    for (int r0 = (blockIdx.x * NARROW_WARPS + warp) * PER * ROWS; r0 < a.rows; r0 += step) {
        uint4 qx[ROWS], qu[ROWS];
        float mu[ROWS], rs[ROWS];
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int r = r0 + u * PER + lane / L;
            qx[u] = qu[u] = make_uint4(0u, 0u, 0u, 0u);
            mu[u] = rs[u] = 0.f;
            if (has && r < a.rows) {
                qx[u] = *reinterpret_cast<const uint4*>(a.x.at(r) + c * sizeof(T));
                qu[u] = *reinterpret_cast<const uint4*>(a.dy.at(r) + c * sizeof(T));
                mu[u] = a.mean[r];
                rs[u] = a.rstd[r];
            }
        }
#pragma unroll
        for (int u = 0; u < ROWS; ++u) {
            const int r = r0 + u * PER + lane / L;
            f2 x[P::PAIRS], w[P::PAIRS], t[P::PAIRS];
            P::unpack(qx[u], x);
            P::unpack(qu[u], w);
            const f2 minus_mu = pair(-mu[u] * rs[u], -mu[u] * rs[u]), rs2 = pair(rs[u], rs[u]);
            f2 sa = 0ull, sax = 0ull;
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) {
                x[i] = fma2(x[i], rs2, minus_mu);                           // xh; 0 in lanes and rows that do not exist
                dg[i] = fma2(w[i], x[i], dg[i]);
                db[i] = add2(w[i], db[i]);
                t[i] = mul2(w[i], gw[i]);
                sa = add2(sa, t[i]);
                sax = fma2(t[i], x[i], sax);
            }
            const float2 pa = split(sa), pax = split(sax);
            const float ma = -rs[u] * lanes_sum<L>(pa.x + pa.y) * inv_d, mx = -rs[u] * lanes_sum<L>(pax.x + pax.y) * inv_d;
            const f2 ma2 = pair(ma, ma), mx2 = pair(mx, mx);
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) x[i] = fma2(t[i], rs2, fma2(x[i], mx2, ma2));
            if (a.out && has && r < a.rows) *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + r * a.out_stride + c) = P::pack(x);
        }
    }
    if (!a.partial) return;
    // the warp's rows at once, then the block's warps in order
#pragma unroll
    for (int i = 0; i < P::PAIRS; ++i) {
        float2 p = split(dg[i]), q = split(db[i]);
#pragma unroll
        for (int o = L; o < 32; o <<= 1) {
            p.x += __shfl_xor_sync(0xffffffffu, p.x, o); p.y += __shfl_xor_sync(0xffffffffu, p.y, o);
            q.x += __shfl_xor_sync(0xffffffffu, q.x, o); q.y += __shfl_xor_sync(0xffffffffu, q.y, o);
        }
        if (lane < L && has) {
            sums[warp][0][c + 2 * i] = p.x; sums[warp][0][c + 2 * i + 1] = p.y;
            sums[warp][1][c + 2 * i] = q.x; sums[warp][1][c + 2 * i + 1] = q.y;
        }
    }
    __syncthreads();
    float* out = a.partial + static_cast<size_t>(blockIdx.x) * 2 * a.d;
    for (int k = threadIdx.x; k < 2 * a.d; k += NARROW_THREADS) {
        const int which = k >= a.d ? 1 : 0, col = k - which * a.d;
        float v = 0.f;
        for (int w = 0; w < NARROW_WARPS; ++w) v += sums[w][which][col];
        out[k] = v;
    }
}

// ------------------------------------------------------------------------------------ generic kernels
template <typename T, typename W>
__global__ void __launch_bounds__(GEN_THREADS)
ln_forward_generic(const T* x, long rows, long d, long x_stride, const W* __restrict__ g, const W* __restrict__ b, float eps,
                   T* y, long y_stride, float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float2 part[GEN_THREADS / 32];
    const float inv_d = 1.f / static_cast<float>(d);
    for (long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T* xr = x + r * x_stride;
        float s = 0.f;
        for (long c = threadIdx.x; c < d; c += GEN_THREADS) s += to_f(xr[c]);
        const float mu = block_sum2<GEN_THREADS>(s, 0.f, part).x * inv_d;
        float q = 0.f;
        for (long c = threadIdx.x; c < d; c += GEN_THREADS) {
            const float t = to_f(xr[c]) - mu;
            q += t * t;
        }
        const float rs = 1.f / sqrtf(block_sum2<GEN_THREADS>(q, 0.f, part).x * inv_d + eps);
        for (long c = threadIdx.x; c < d; c += GEN_THREADS) {
            float v = (to_f(xr[c]) - mu) * rs;
            if (g) v *= to_f(g[c]);
            if (b) v += to_f(b[c]);
            y[r * y_stride + c] = from_f<T>(v);
        }
        if (threadIdx.x == 0) {
            if (mean) mean[r] = mu;
            if (rstd) rstd[r] = rs;
        }
    }
}

template <typename T, typename W>
__global__ void __launch_bounds__(GEN_THREADS)
ln_backward_dx_generic(const T* dy, long dy_stride, const T* __restrict__ x, long x_stride, long rows, long d,
                       const W* __restrict__ g, const float* __restrict__ mean, const float* __restrict__ rstd, T* dx,
                       long dx_stride) {
    __shared__ float2 part[GEN_THREADS / 32];
    const float inv_d = 1.f / static_cast<float>(d);
    for (long r = blockIdx.x; r < rows; r += gridDim.x) {
        const T *xr = x + r * x_stride, *dyr = dy + r * dy_stride;
        const float mu = mean[r], rs = rstd[r];
        float sa = 0.f, sax = 0.f;
        for (long c = threadIdx.x; c < d; c += GEN_THREADS) {
            const float a = to_f(dyr[c]) * (g ? to_f(g[c]) : 1.f);
            sa += a;
            sax += a * ((to_f(xr[c]) - mu) * rs);
        }
        const float2 s = block_sum2<GEN_THREADS>(sa, sax, part);
        const float ma = s.x * inv_d, max_ = s.y * inv_d;
        for (long c = threadIdx.x; c < d; c += GEN_THREADS) {
            const float a = to_f(dyr[c]) * (g ? to_f(g[c]) : 1.f);
            const float xh = (to_f(xr[c]) - mu) * rs;
            dx[r * dx_stride + c] = from_f<T>(rs * (a - ma - xh * max_));
        }
    }
}

// Column sums of dy xh and dy over one slice of rows: block (column tile, slice) -> partial[slice][2][d].
template <typename T>
__global__ void __launch_bounds__(COL_TILE * COL_ROWS)
ln_backward_columns(const T* __restrict__ dy, long dy_stride, const T* __restrict__ x, long x_stride, long rows, long d,
                    const float* __restrict__ mean, const float* __restrict__ rstd, float* __restrict__ partial) {
    __shared__ float2 part[COL_ROWS][COL_TILE];
    const long c = static_cast<long>(blockIdx.x) * COL_TILE + (threadIdx.x % COL_TILE);
    const int rr = threadIdx.x / COL_TILE;
    const long per = (rows + gridDim.y - 1) / gridDim.y;
    const long r0 = blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
    float sg = 0.f, sb = 0.f;
    if (c < d)
        for (long r = r0 + rr; r < r1; r += COL_ROWS) {
            const float u = to_f(dy[r * dy_stride + c]);
            sg += u * ((to_f(x[r * x_stride + c]) - mean[r]) * rstd[r]);
            sb += u;
        }
    part[rr][threadIdx.x % COL_TILE] = make_float2(sg, sb);
    __syncthreads();
    if (rr == 0 && c < d) {
        for (int i = 1; i < COL_ROWS; ++i) { sg += part[i][threadIdx.x].x; sb += part[i][threadIdx.x].y; }
        float* o = partial + static_cast<long>(blockIdx.y) * 2 * d;
        o[c] = sg;
        o[d + c] = sb;
    }
}

// dweight, dbias = sums of the partial column sums, slices in a fixed order: 32 columns per block, 32 threads a column.
constexpr int FIN_ROWS = 32;
template <typename W>
__global__ void __launch_bounds__(COL_TILE * FIN_ROWS)
ln_backward_finish(const float* __restrict__ partial, int slices, long d, W* __restrict__ dg, W* __restrict__ db) {
    __shared__ float2 part[FIN_ROWS][COL_TILE + 1];
    const int cc = threadIdx.x % COL_TILE, rr = threadIdx.x / COL_TILE;
    const long c = static_cast<long>(blockIdx.x) * COL_TILE + cc;
    float sg = 0.f, sb = 0.f;
    if (c < d) {
#pragma unroll 4
        for (int s = rr; s < slices; s += FIN_ROWS) {
            sg += partial[static_cast<long>(s) * 2 * d + c];
            sb += partial[static_cast<long>(s) * 2 * d + d + c];
        }
    }
    part[rr][cc] = make_float2(sg, sb);
    __syncthreads();
    const float2 v = part[cc][rr];                          // warp rr: the 32 sums of column rr
    sg = warp_sum(v.x);
    sb = warp_sum(v.y);
    const long out = static_cast<long>(blockIdx.x) * COL_TILE + rr;
    if (cc == 0 && out < d) {
        if (dg) dg[out] = from_f<W>(sg);
        if (db) db[out] = from_f<W>(sb);
    }
}

// ------------------------------------------------------------------------------------ host side
constexpr int64_t MAX_D = int64_t{1} << 30;

size_t elem_bytes(int t) { return t == VPCE_F32 ? 4 : 2; }
bool known_type(int t) { return t == VPCE_BF16 || t == VPCE_F16 || t == VPCE_F32; }
bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int slices_for(int64_t rows) {
    const int64_t s = rows;
    return static_cast<int>(s < 1 ? 1 : s > MAX_SLICES ? MAX_SLICES : s);
}

int grid_rows(int64_t rows) { return static_cast<int>(rows < 148 * 8 ? rows : 148 * 8); }

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

// Shape of a row kernel's launch: `na` arrays in the ring.  grid 0: the row is too wide for shared memory.
struct RowShape { int ept, threads, grid, smem; };
RowShape row_shape(RowArgs* a, size_t elem, int na) {
    RowShape s;
    // Elements per thread: a warp costs about 8 instructions for each of its threads' elements and 110 for the rest of a row
    // (waits, sums over the warp and the group).  At d = 7168 in 16 bits: 7 warps of 32 rather than 14 of 16.
    s.ept = 8;
    int best = 1 << 30;
    for (int ept = 8; ept <= MAX_EPT; ept += 8) {
        const int warps = (a->d + 32 * ept - 1) / (32 * ept), cost = warps * (8 * ept + 110);
        if (warps <= MAX_GROUP_WARPS && cost < best) { best = cost; s.ept = ept; a->warps = warps; }
    }
    const int most = (na == 1 ? FORWARD_WARPS : BACKWARD_WARPS) / a->warps;
    a->groups = std::max(1, a->warps > 1 ? std::min(most, 15) : most);          // named barriers 1 to 15
    while (a->groups > 1 && static_cast<int64_t>(a->groups - 1) * sm_count() >= a->rows) --a->groups;   // few rows: spread over the SMs
    a->cap = static_cast<int>((a->d * elem + 15) / 16 * 16 + 16);
    a->slot = na * a->cap + (na == 2 ? 16 : 0);
    auto ring = [&] { return FULL_BYTES + a->groups * PART_BYTES + (na == 1 ? 2 : 1) * 4 * 32 * s.ept * a->warps; };
    while (a->groups > 1 && ring() + a->groups * 2 * a->slot > MAX_SMEM) --a->groups;
    a->ring = ring();
    a->stages = std::min(MAX_STAGES, (MAX_SMEM - a->ring) / (a->groups * a->slot));
    s.threads = 32 * a->warps * a->groups;
    s.smem = a->ring + a->groups * a->stages * a->slot;
    if (na == 2) s.smem = std::max<int>(s.smem, a->ring + 8 * a->d * a->groups);    // the groups' sums take its place
    const int64_t blocks = (a->rows + a->groups - 1) / a->groups;
    s.grid = a->stages >= 2 && s.smem <= MAX_SMEM ? static_cast<int>(std::min<int64_t>(blocks, std::min(sm_count(), MAX_SLICES))) : 0;
    return s;
}

template <typename Args, void (*kern)(const Args)> cudaError_t launch_rows(const RowArgs& a, const RowShape& s, cudaStream_t st) {
    static std::atomic<int> raised[64];                                         // of this kernel, per device
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !raised[dev].load(std::memory_order_acquire)) {
        if (cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM); e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev].store(1, std::memory_order_release);
    }
    kern<<<s.grid, s.threads, s.smem, st>>>(args_of<Args>(a));
    return cudaGetLastError();
}

bool rows_aligned(const void* p, int64_t stride, size_t e) { return aligned_to(p, 16) && stride * e % 16 == 0; }

template <typename T, typename W, bool VEC> cudaError_t forward_rows(const RowArgs& a, const RowShape& s, cudaStream_t st) {
    switch (s.ept) {
        case 8: return launch_rows<LongRowArgs, ln_forward_rows<T, W, VEC, 8>>(a, s, st);
        case 16: return launch_rows<LongRowArgs, ln_forward_rows<T, W, VEC, 16>>(a, s, st);
        case 24: return launch_rows<LongRowArgs, ln_forward_rows<T, W, VEC, 24>>(a, s, st);
        default: return launch_rows<LongRowArgs, ln_forward_rows<T, W, VEC, 32>>(a, s, st);
    }
}
template <typename T, typename W, bool VEC> cudaError_t backward_rows(const RowArgs& a, const RowShape& s, cudaStream_t st) {
    switch (s.ept) {
        case 8: return launch_rows<BackwardArgs<VEC>, ln_backward_rows<T, W, VEC, 8>>(a, s, st);
        case 16: return launch_rows<BackwardArgs<VEC>, ln_backward_rows<T, W, VEC, 16>>(a, s, st);
        case 24: return launch_rows<BackwardArgs<VEC>, ln_backward_rows<T, W, VEC, 24>>(a, s, st);
        default: return launch_rows<BackwardArgs<VEC>, ln_backward_rows<T, W, VEC, 32>>(a, s, st);
    }
}

// Blocks of a narrow launch: `per_sm` an SM at most, none without rows.
int narrow_grid(int64_t rows, int lanes, int unroll, int per_sm) {
    const int64_t per = static_cast<int64_t>(NARROW_WARPS) * (32 / lanes) * unroll;
    return static_cast<int>(std::min<int64_t>((rows + per - 1) / per, static_cast<int64_t>(per_sm) * sm_count()));
}
int narrow_lanes(int64_t bytes) { return bytes <= 128 ? 8 : bytes <= 256 ? 16 : 32; }

int code(cudaError_t e) { return e == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR; }

template <typename T, typename W>
int forward_typed(const void* x, int64_t rows, int64_t d, int64_t xs, const void* g, const void* b, float eps, void* y, int64_t ys,
                  float* mean, float* rstd, cudaStream_t st) {
    if (d <= MAX_ROW && rows <= MAX_ROWS) {
        RowArgs a{};
        a.x = Rows{x, static_cast<long>(xs * sizeof(T))}; a.rows = static_cast<int>(rows); a.out_stride = ys; a.d = static_cast<int>(d); a.g = g; a.b = b; a.eps = eps; a.out = y;
        a.mean = mean; a.rstd = rstd;
        const bool vec = d * sizeof(T) % 16 == 0 && rows_aligned(x, xs, sizeof(T)) && rows_aligned(y, ys, sizeof(T));
        if (vec && d * sizeof(T) <= NARROW_BYTES) {
            const int lanes = narrow_lanes(d * sizeof(T)), grid = narrow_grid(rows, lanes, UNROLL, 4);
            if (lanes == 8) ln_forward_narrow<T, W, 8><<<grid, NARROW_THREADS, 0, st>>>(args_of<LongRowArgs>(a));
            else if (lanes == 16) ln_forward_narrow<T, W, 16><<<grid, NARROW_THREADS, 0, st>>>(args_of<LongRowArgs>(a));
            else ln_forward_narrow<T, W, 32><<<grid, NARROW_THREADS, 0, st>>>(args_of<LongRowArgs>(a));
            return code(cudaGetLastError());
        }
        const RowShape s = row_shape(&a, sizeof(T), 1);
        if (s.grid > 0) return code(vec ? forward_rows<T, W, true>(a, s, st) : forward_rows<T, W, false>(a, s, st));
    }
    ln_forward_generic<T, W><<<grid_rows(rows), GEN_THREADS, 0, st>>>(
        static_cast<const T*>(x), rows, d, xs, static_cast<const W*>(g), static_cast<const W*>(b), eps, static_cast<T*>(y), ys, mean, rstd);
    return code(cudaGetLastError());
}

template <typename T, typename W>
int backward_typed(const void* dy, int64_t dys, const void* x, int64_t xs, int64_t rows, int64_t d, const void* g, const float* mean,
                   const float* rstd, void* dx, int64_t dxs, void* dg, void* db, float* partial, cudaStream_t st) {
    const T *dyt = static_cast<const T*>(dy), *xt = static_cast<const T*>(x);
    const unsigned col_tiles = static_cast<unsigned>((d + COL_TILE - 1) / COL_TILE);
    int slices = slices_for(rows);
    if (d <= MAX_ROW && rows > 0 && rows <= MAX_ROWS) {
        RowArgs a{};
        a.x = Rows{x, static_cast<long>(xs * sizeof(T))}; a.dy = Rows{dy, static_cast<long>(dys * sizeof(T))};
        a.rows = static_cast<int>(rows); a.out_stride = dxs; a.d = static_cast<int>(d); a.g = g;
        a.out = dx; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
        a.partial = dg || db ? partial : nullptr;
        const bool vec = d * sizeof(T) % 16 == 0 && rows_aligned(x, xs, sizeof(T)) && rows_aligned(dy, dys, sizeof(T)) &&
                         rows_aligned(dx, dxs, sizeof(T));
        if (vec && d * sizeof(T) <= NARROW_BYTES) {
            const int lanes = narrow_lanes(d * sizeof(T)), grid = std::min(narrow_grid(rows, lanes, UNROLL / 2, 2), slices);
            if (lanes == 8) ln_backward_narrow<T, W, 8><<<grid, NARROW_THREADS, 0, st>>>(a);
            else if (lanes == 16) ln_backward_narrow<T, W, 16><<<grid, NARROW_THREADS, 0, st>>>(a);
            else ln_backward_narrow<T, W, 32><<<grid, NARROW_THREADS, 0, st>>>(a);
            if (a.partial)
                ln_backward_finish<W><<<col_tiles, COL_TILE * FIN_ROWS, 0, st>>>(partial, grid, d, static_cast<W*>(dg), static_cast<W*>(db));
            return code(cudaGetLastError());
        }
        const RowShape s = row_shape(&a, sizeof(T), 2);
        if (s.grid > 0) {
            if (cudaError_t e = vec ? backward_rows<T, W, true>(a, s, st) : backward_rows<T, W, false>(a, s, st); e != cudaSuccess)
                return VPCE_CUDA_ERROR;
            if (a.partial)
                ln_backward_finish<W><<<col_tiles, COL_TILE * FIN_ROWS, 0, st>>>(partial, s.grid, d, static_cast<W*>(dg), static_cast<W*>(db));
            return code(cudaGetLastError());
        }
    }
    if (dg || db) {
        ln_backward_columns<T><<<dim3(col_tiles, slices), COL_TILE * COL_ROWS, 0, st>>>(dyt, dys, xt, xs, rows, d, mean, rstd, partial);
        ln_backward_finish<W><<<col_tiles, COL_TILE * FIN_ROWS, 0, st>>>(partial, slices, d, static_cast<W*>(dg), static_cast<W*>(db));
    }
    if (dx && rows > 0)                                     // after the column sums: dx may be dy itself
        ln_backward_dx_generic<T, W><<<grid_rows(rows), GEN_THREADS, 0, st>>>(dyt, dys, xt, xs, rows, d, static_cast<const W*>(g), mean,
                                                                            rstd, static_cast<T*>(dx), dxs);
    return code(cudaGetLastError());
}

// Calls f with the element types of (x_dtype, w_dtype) as null pointers.
template <typename F> int with_types(int x_dtype, int w_dtype, F f) {
    if (x_dtype == VPCE_BF16 && w_dtype == VPCE_BF16) return f((__nv_bfloat16*)nullptr, (__nv_bfloat16*)nullptr);
    if (x_dtype == VPCE_BF16 && w_dtype == VPCE_F32) return f((__nv_bfloat16*)nullptr, (float*)nullptr);
    if (x_dtype == VPCE_F16 && w_dtype == VPCE_F16) return f((__half*)nullptr, (__half*)nullptr);
    if (x_dtype == VPCE_F16 && w_dtype == VPCE_F32) return f((__half*)nullptr, (float*)nullptr);
    if (x_dtype == VPCE_F32 && w_dtype == VPCE_F32) return f((float*)nullptr, (float*)nullptr);
    return VPCE_INVALID_ARG;
}

bool sizes_ok(int64_t rows, int64_t d) { return rows >= 0 && d >= 1 && d <= MAX_D && rows <= (int64_t{1} << 40); }

}  // namespace

extern "C" {

int vp_ln_forward(const void* x, int x_dtype, int64_t rows, int64_t d, int64_t x_stride, const void* weight, const void* bias,
                  int w_dtype, double eps, void* y, int64_t y_stride, float* mean, float* rstd, void* stream) {
    if (!sizes_ok(rows, d) || !known_type(x_dtype) || !(eps >= 0.0)) return VPCE_INVALID_ARG;
    if (!weight && !bias) w_dtype = x_dtype;
    if (!known_type(w_dtype) || (w_dtype != x_dtype && w_dtype != VPCE_F32)) return VPCE_INVALID_ARG;
    if (rows == 0) return VPCE_OK;
    if (!x || !y || x_stride < d || y_stride < d) return VPCE_INVALID_ARG;
    const size_t e = elem_bytes(x_dtype), we = elem_bytes(w_dtype);
    if (!aligned_to(x, e) || !aligned_to(y, e) || !aligned_to(weight, we) || !aligned_to(bias, we) || !aligned_to(mean, 4) ||
        !aligned_to(rstd, 4))
        return VPCE_UNSUPPORTED;
    return with_types(x_dtype, w_dtype, [&](auto* t, auto* w) {
        return forward_typed<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>(
            x, rows, d, x_stride, weight, bias, static_cast<float>(eps), y, y_stride, mean, rstd, static_cast<cudaStream_t>(stream));
    });
}

size_t vp_ln_workspace_bytes(int64_t rows, int64_t d) {
    if (!sizes_ok(rows, d)) return 0;
    return static_cast<size_t>(slices_for(rows)) * 2 * static_cast<size_t>(d) * sizeof(float);
}

int vp_ln_backward(const void* dy, int64_t dy_stride, const void* x, int64_t x_stride, int x_dtype, int64_t rows, int64_t d,
                   const void* weight, int w_dtype, const float* mean, const float* rstd, void* dx, int64_t dx_stride,
                   void* dweight, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    if (!sizes_ok(rows, d) || !known_type(x_dtype)) return VPCE_INVALID_ARG;
    if (!weight && !dweight && !dbias) w_dtype = x_dtype;
    if (!known_type(w_dtype) || (w_dtype != x_dtype && w_dtype != VPCE_F32)) return VPCE_INVALID_ARG;
    if (!dx && !dweight && !dbias) return VPCE_OK;
    if (rows > 0 && (!dy || !x || !mean || !rstd || dy_stride < d || x_stride < d || (dx && dx_stride < d))) return VPCE_INVALID_ARG;
    const size_t e = elem_bytes(x_dtype), we = elem_bytes(w_dtype);
    if (!aligned_to(dy, e) || !aligned_to(x, e) || !aligned_to(dx, e) || !aligned_to(weight, we) || !aligned_to(dweight, we) ||
        !aligned_to(dbias, we) || !aligned_to(mean, 4) || !aligned_to(rstd, 4))
        return VPCE_UNSUPPORTED;
    if (dweight || dbias) {
        if (!workspace) return VPCE_INVALID_ARG;
        if (!aligned_to(workspace, 16)) return VPCE_UNSUPPORTED;
        if (workspace_bytes < vp_ln_workspace_bytes(rows, d)) return VPCE_WORKSPACE_TOO_SMALL;
    }
    return with_types(x_dtype, w_dtype, [&](auto* t, auto* w) {
        return backward_typed<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>(
            dy, dy_stride, x, x_stride, rows, d, weight, mean, rstd, dx, dx_stride, dweight, dbias, static_cast<float*>(workspace),
            static_cast<cudaStream_t>(stream));
    });
}

}  // extern "C"
