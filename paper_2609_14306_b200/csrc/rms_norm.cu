// RMS norm with the residual's addition, forward (also to 8 bits) and backward (rms_norm.h).
//
// Bound: memory.  Forward reads x and r and writes z and y (four passes; 8-bit output: three and a half), backward reads z, dy and dz
// and writes dx (four).  The kernels are built like the layer norm's (row_kernels.cuh):
//   rows     a group of 1 to 16 warps owns a row at a time, rows arrive by bulk copies in a ring in shared memory, several rows
//            ahead; one barrier per row (the warps' sums of squares, or of a z); weights as fp32 in shared memory.  A thread keeps its 8
//            to 32 elements of a row in registers from the ring to the store: forward as fp32, backward z, dy and dz in their own type
//            beside the column sums of dy zh over all rows of its group (one partial sum per block at the end).
//   narrow   aligned rows of up to 512 bytes (a norm over one head): 8, 16 or 32 lanes a row, several rows to a warp, no ring
//   generic  rows too wide for shared memory: a block per row, 128 columns to a warp at a time, 0.1 to 0.15 of the memory's rate
// The largest magnitude of 128 columns is a maximum over 16 lanes (16-bit rows: 8 neighbours a lane) or a warp, in registers: the
// 8-bit output costs no pass of its own.
// Measured: 16384 x 2880 bf16 with a residual 59 us forward, 62 backward (58 each at a plain copy's rate), 140 for both and the sums
// in repetition; 32768 x 7168 bf16 to 8 bits 268 us (252); rows off every 16-byte boundary 0.5 to 0.65 of the aligned rate in 16 bits (0.4 to
// 8 bits, whose stores are single bytes), 0.8 to 0.95 in fp32.

#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "rms_norm.h"
#include "row_kernels.cuh"

namespace {

constexpr int GROUP = 128;                              // columns that share a scale of the 8-bit output
constexpr int MAX_GROUP_WARPS = 16;
constexpr int FORWARD_REGS = 72, FORWARD_WARPS = 28, BACKWARD_REGS = 128, BACKWARD_WARPS = 16;     // one block per SM
constexpr int MAX_GROUPS = FORWARD_WARPS;               // per block; a group of more than one warp has a named barrier
constexpr int MAX_STAGES = 8;
constexpr int MAX_SMEM = 227 * 1024;
constexpr int64_t MAX_ROWS = (int64_t{1} << 31) - (1 << 20);   // row numbers and the look-ahead stay below 2^31
constexpr int MAX_EPT = 32;                             // elements per thread
constexpr int64_t MAX_ROW = 32 * MAX_GROUP_WARPS * MAX_EPT;
constexpr int MAX_SLICES = 296;                         // partial sums over rows

// Shared memory of a block: barriers [MAX_GROUPS][MAX_STAGES], weights, the warps' sums (float [group][turn][warp]), ring.
constexpr int FULL_BYTES = MAX_GROUPS * MAX_STAGES * 8, PART_BYTES = 2 * MAX_GROUP_WARPS * 4;
static_assert(FULL_BYTES % 128 == 0 && PART_BYTES % 128 == 0, "what follows begins on a 128-byte boundary");

struct RmsArgs {
    Rows in[3];                                         // forward: x, r; backward: z, dy, dz
    int rows, d, warps;                                 // warps per group
    int groups, stages, cap, slot;                      // groups per block, ring depth, bytes of a row and of a slot in the ring
    int ring;                                           // byte offset of the ring in shared memory
    int w_fp32;
    float eps;
    const void* g;
    void* out;                                          // y, q or dx (backward: may be null)
    void* z;                                            // forward: may be null
    long out_stride, z_stride;                          // elements
    float* scales;                                      // 8-bit output: [rows][n_scales]
    int n_scales;
    float* rstd;                                        // written (forward, may be null) or read (backward)
    float* partial;                                     // [blocks][d] or null
};

// ------------------------------------------------------------------------------------ 8-bit output
// Scale of a group from its largest magnitude, and its reciprocal.  Below 2^-126 the reciprocal would overflow.
__device__ __forceinline__ float2 scale_of(float amax) {
    const float s = amax > 0.f ? fmaxf(amax * (1.f / 448.f), 1.1754944e-38f) : 1.f;
    return make_float2(s, 1.f / s);
}
__device__ __forceinline__ uint32_t e4m3x2(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ uint8_t e4m3(float a) { return __nv_cvt_float_to_fp8(a, __NV_SATFINITE, __NV_E4M3); }
__device__ __forceinline__ float max_abs(f2 v, float m) {
    const float2 p = split(v);
    return fmaxf(m, fmaxf(fabsf(p.x), fabsf(p.y)));      // fmaxf passes a NaN over
}
template <int L> __device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// ------------------------------------------------------------------------------------ row kernels
// One thread: row r of the first NA arrays into ring slot `slot`, signalled on `bar`; with STAT the row's rstd, too, to the slot's end
// (the barrier counts its arrival).
template <typename T, bool VEC, int NA, bool STAT>
__device__ __forceinline__ void fetch_row(const RmsArgs& a, int r, uint8_t* slot, uint32_t bar) {
    const char* from[NA];
    uint32_t at[NA], bytes[NA], total = 0;
#pragma unroll
    for (int i = 0; i < NA; ++i) {
        bytes[i] = copy_extent<T, VEC>(a.in[i], r, a.rows, a.d, &from[i], &at[i], slot + i * a.cap);
        total += bytes[i];
    }
    const uint32_t dst = vpce::smem_u32(slot);
    if (!VEC) vpce::fence_proxy_async();                    // plain stores to a slot come before a later row's bulk copy to it
    if (STAT) {
        asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst + NA * a.cap), "l"(a.rstd + r) : "memory");
        asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];" ::"r"(bar) : "memory");
    }
    vpce::mbar_arrive_expect_tx(bar, total);
#pragma unroll
    for (int i = 0; i < NA; ++i)
        if (bytes[i]) bulk_load(dst + i * a.cap + at[i], from[i], bytes[i], bar);
}

struct Group {
    int id, warp, lane;
    int first, step;                                    // rows of this group: first, first + step, ...
    uint8_t* ring;
    uint32_t bars;
};
template <typename T, bool VEC, int NA, bool STAT>
__device__ __forceinline__ Group group_setup(const RmsArgs& a, uint8_t* raw) {
    Group g;
    g.id = (threadIdx.x >> 5) / a.warps;
    g.warp = (threadIdx.x >> 5) - g.id * a.warps;
    g.lane = threadIdx.x & 31;
    g.first = blockIdx.x * a.groups + g.id;
    g.step = gridDim.x * a.groups;
    g.ring = raw + a.ring + g.id * a.stages * a.slot;
    g.bars = vpce::smem_u32(raw) + g.id * MAX_STAGES * 8;
    if (g.warp == 0 && g.lane == 0) {
        for (int s = 0; s < a.stages; ++s) vpce::mbar_init(g.bars + 8 * s, STAT ? 2 : 1);
        vpce::fence_barrier_init();
        vpce::fence_proxy_async();
    }
    group_sync(g.id, a.warps);
    if (g.warp == 0 && g.lane == 0)
        for (int s = 0; s < a.stages; ++s) {
            const int r = g.first + s * g.step;
            if (r < a.rows) fetch_row<T, VEC, NA, STAT>(a, r, g.ring + s * a.slot, g.bars + 8 * s);
        }
    return g;
}

// The group's weights as fp32 in shared memory, in the order of the threads' elements.
template <typename T, typename C>
__device__ __forceinline__ void fill_weights(const RmsArgs& a, const C& cols, float* to, int warp, int lane) {
    if (a.w_fp32) cols.fill(to, warp, lane, static_cast<const float*>(a.g), 1.f);
    else cols.fill(to, warp, lane, static_cast<const T*>(a.g), 1.f);
}

// Part q (8 elements) of a thread's columns as 8 bits, each group of 128 columns with its scale.  The warp's columns begin at a
// multiple of 128, so a group lies in one part of one warp.
template <typename T, bool VEC, typename C>
__device__ __forceinline__ void store_fp8(const RmsArgs& a, const C& cols, int r, int q, int lane, const f2* v) {
    uint8_t* row = static_cast<uint8_t*>(a.out) + r * a.out_stride;
    float* scales = a.scales + static_cast<long>(r) * a.n_scales;
    if constexpr (VEC && sizeof(T) == 2) {                                  // 16 lanes x 8 neighbours
        const int c = cols.first + C::STEP * q;
        const float2 s = scale_of(lanes_max<16>(max_abs(v[0], max_abs(v[1], max_abs(v[2], max_abs(v[3], 0.f))))));
        if (c < a.d) {
            float2 e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = split(mul2(v[i], pair(s.y, s.y)));
            *reinterpret_cast<uint2*>(row + c) = make_uint2(e4m3x2(e[0].x, e[0].y) | e4m3x2(e[1].x, e[1].y) << 16,
                                                            e4m3x2(e[2].x, e[2].y) | e4m3x2(e[3].x, e[3].y) << 16);
            if ((lane & 15) == 0) scales[c / GROUP] = s.x;
        }
    } else {
#pragma unroll
        for (int h = 0; h < 2; ++h) {                                       // VEC: 32 lanes x 4 neighbours; else 4 x 32 lanes
            const int c = cols.first + C::STEP * (q * C::PART + h * (C::PART / 2));
            const float2 s = scale_of(lanes_max<32>(max_abs(v[2 * h], max_abs(v[2 * h + 1], 0.f))));
            const float2 e = split(mul2(v[2 * h], pair(s.y, s.y))), f = split(mul2(v[2 * h + 1], pair(s.y, s.y)));
            if constexpr (VEC) {
                if (c < a.d) *reinterpret_cast<uint32_t*>(row + c) = e4m3x2(e.x, e.y) | e4m3x2(f.x, f.y) << 16;
            } else {
                if (c < a.d) row[c] = e4m3(e.x);
                if (c + 32 < a.d) row[c + 32] = e4m3(e.y);
                if (c + 64 < a.d) row[c + 64] = e4m3(f.x);
                if (c + 96 < a.d) row[c + 96] = e4m3(f.y);
            }
            if (lane == 0 && c < a.d) scales[c / GROUP] = s.x;
        }
    }
}

template <typename T> __device__ __forceinline__ f2 round_pair(f2 v) {
    if constexpr (sizeof(T) == 4) return v;
    else { const float2 p = split(v); return widen<T>(narrow<T>(p.x, p.y)); }
}

template <typename T, bool VEC, int EPT, bool RES, bool F8>
__global__ void __maxnreg__(FORWARD_REGS) rms_forward_rows(const RmsArgs a) {
    extern __shared__ __align__(128) uint8_t raw[];
    constexpr int NA = RES ? 2 : 1;
    const Group g = group_setup<T, VEC, NA, false>(a, raw);
    using C = Columns<T, VEC, EPT, true>;
    const C cols(g.warp, g.lane, a.d);
    float* const weights = reinterpret_cast<float*>(raw + FULL_BYTES);
    if (g.id == 0) fill_weights<T>(a, cols, weights, g.warp, g.lane);
    __syncthreads();
    const uint32_t gw = vpce::smem_u32(weights) + (g.warp * (EPT / 4) * 32 + g.lane) * 16;
    float(*part)[MAX_GROUP_WARPS] = reinterpret_cast<float(*)[MAX_GROUP_WARPS]>(raw + a.ring - (a.groups - g.id) * PART_BYTES);
    const float inv_d = 1.f / static_cast<float>(a.d);
    int s = 0, pass = 0, turn = 0;                                          // the warps take turns at starting copies
    uint32_t parity = 0;
    for (int r = g.first; r < a.rows; r += g.step) {
        const uint32_t slot = vpce::smem_u32(g.ring + s * a.slot);
        const uint32_t xr = slot + (VEC ? 0u : a.in[0].shift(r)), rr = slot + a.cap + (VEC || !RES ? 0u : a.in[1].shift(r));
        wait_row(g.bars + 8 * s, parity);
        f2 v[C::PAIRS], s0 = 0ull, s1 = 0ull;
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) {
            f2* const p = v + 4 * q;
            cols.read(xr, q, p);
            if constexpr (RES) {
                f2 u[4];
                cols.read(rr, q, u);
#pragma unroll
                for (int i = 0; i < 4; ++i) p[i] = round_pair<T>(add2(p[i], u[i]));
            }
            s0 = fma2(p[0], p[0], s0); s1 = fma2(p[1], p[1], s1);           // columns beyond d read as 0
            s0 = fma2(p[2], p[2], s0); s1 = fma2(p[3], p[3], s1);
        }
        const float2 t = split(add2(s0, s1));
        const float squares = warp_sum(t.x + t.y);
        if (g.lane == 0) part[pass][g.warp] = squares;
        group_sync(g.id, a.warps);
        // everyone has read the slot: it takes the next row that is not under way yet
        if (g.warp == turn && g.lane == 0 && r + a.stages * g.step < a.rows)
            fetch_row<T, VEC, NA, false>(a, r + a.stages * g.step, g.ring + s * a.slot, g.bars + 8 * s);
        if (++turn == a.warps) turn = 0;
        if (++s == a.stages) { s = 0; parity ^= 1u; }
        const float w = (g.lane & 15) < a.warps ? part[pass][g.lane & 15] : 0.f;
        pass ^= 1;
        const float rs = 1.f / sqrtf(fmaf(half_warp_sum(w), inv_d, a.eps));
        const f2 rs2 = pair(rs, rs);
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) {
            if (RES && a.z) cols.store(static_cast<T*>(a.z) + r * a.z_stride, q, v + 4 * q);
            f2 gq[4];
            cols.weights(gw, q, gq);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * q + i] = mul2(mul2(v[4 * q + i], rs2), gq[i]);
            if constexpr (F8) store_fp8<T, VEC>(a, cols, r, q, g.lane, v + 4 * q);
            else cols.store(static_cast<T*>(a.out) + r * a.out_stride, q, v + 4 * q);
        }
        if (g.warp == 0 && g.lane == 0 && a.rstd) a.rstd[r] = rs;
    }
}

// Part q (8 elements) of a thread's columns of a row in shared memory as they are, and as pairs.
template <typename T> constexpr int PART_WORDS = 2 * static_cast<int>(sizeof(T));
template <typename T, bool VEC, typename C> __device__ __forceinline__ void read_words(const C& cols, uint32_t row, int q, uint32_t* w) {
    const uint32_t at = row + (cols.first + C::STEP * q * C::PART) * static_cast<int>(sizeof(T));
    if constexpr (VEC) {
#pragma unroll
        for (int k = 0; k < C::PART; ++k) {
            w[4 * k] = w[4 * k + 1] = w[4 * k + 2] = w[4 * k + 3] = 0u;
            if (cols.has(q * C::PART + k))
                asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4 * k]), "=r"(w[4 * k + 1]), "=r"(w[4 * k + 2]), "=r"(w[4 * k + 3]) : "r"(at + k * 512));
        }
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k] = 0u;
            if (cols.has(q * C::PART + k)) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(w[k]) : "r"(at + k * 128));
        }
    } else {
        uint16_t h[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            h[k] = 0;
            if (cols.has(q * C::PART + k)) asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h[k]) : "r"(at + k * 64));
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = static_cast<uint32_t>(h[2 * i]) | static_cast<uint32_t>(h[2 * i + 1]) << 16;
    }
}
template <typename T> __device__ __forceinline__ f2 word_pair(const uint32_t* w, int i) {
    if constexpr (sizeof(T) == 4) return pair(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    else return widen<T>(w[i]);
}

template <typename T, bool VEC, int EPT, bool RES>
__global__ void __maxnreg__(BACKWARD_REGS) rms_backward_rows(const RmsArgs a) {
    extern __shared__ __align__(128) uint8_t raw[];
    constexpr int NA = RES ? 3 : 2, W = PART_WORDS<T>;
    const Group g = group_setup<T, VEC, NA, true>(a, raw);
    using C = Columns<T, VEC, EPT, false>;
    const C cols(g.warp, g.lane, a.d);
    float(*part)[MAX_GROUP_WARPS] = reinterpret_cast<float(*)[MAX_GROUP_WARPS]>(raw + a.ring - (a.groups - g.id) * PART_BYTES);
    const float inv_d = 1.f / static_cast<float>(a.d);
    float* const weights = reinterpret_cast<float*>(raw + FULL_BYTES);
    if (g.id == 0) fill_weights<T>(a, cols, weights, g.warp, g.lane);
    __syncthreads();
    const uint32_t gw = vpce::smem_u32(weights) + (g.warp * (EPT / 4) * 32 + g.lane) * 16;
    f2 dg[C::PAIRS];
#pragma unroll
    for (int i = 0; i < C::PAIRS; ++i) dg[i] = 0ull;
    // A row is read from the ring once and stays in registers in its own type, beside the column sums, so that its slot is free for
    // another row at the group's barrier.
    int s = 0, pass = 0, turn = 0;                                          // the warps take turns at starting copies
    uint32_t parity = 0;
    for (int r = g.first; r < a.rows; r += g.step) {
        const uint32_t slot = vpce::smem_u32(g.ring + s * a.slot);
        const uint32_t zr = slot + (VEC ? 0u : a.in[0].shift(r)), dyr = slot + a.cap + (VEC ? 0u : a.in[1].shift(r));
        const uint32_t dzr = slot + 2 * a.cap + (VEC || !RES ? 0u : a.in[2].shift(r));
        wait_row(g.bars + 8 * s, parity);
        uint32_t zw[EPT / 8 * W], uw[EPT / 8 * W], ww[RES ? EPT / 8 * W : 1];
        f2 s0 = 0ull, s1 = 0ull;
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) {
            f2 gq[4];
            read_words<T, VEC>(cols, zr, q, zw + q * W);
            read_words<T, VEC>(cols, dyr, q, uw + q * W);
            if constexpr (RES) read_words<T, VEC>(cols, dzr, q, ww + q * W);
            cols.weights(gw, q, gq);
            s0 = fma2(mul2(word_pair<T>(uw + q * W, 0), gq[0]), word_pair<T>(zw + q * W, 0), s0);
            s1 = fma2(mul2(word_pair<T>(uw + q * W, 1), gq[1]), word_pair<T>(zw + q * W, 1), s1);
            s0 = fma2(mul2(word_pair<T>(uw + q * W, 2), gq[2]), word_pair<T>(zw + q * W, 2), s0);
            s1 = fma2(mul2(word_pair<T>(uw + q * W, 3), gq[3]), word_pair<T>(zw + q * W, 3), s1);
        }
        const float rs = ld_shared(slot + NA * a.cap);
        const float2 p = split(add2(s0, s1));
        const float mine = warp_sum(p.x + p.y);
        if (g.lane == 0) part[pass][g.warp] = mine;
        group_sync(g.id, a.warps);
        if (g.warp == turn && g.lane == 0 && r + a.stages * g.step < a.rows)
            fetch_row<T, VEC, NA, true>(a, r + a.stages * g.step, g.ring + s * a.slot, g.bars + 8 * s);
        if (++turn == a.warps) turn = 0;
        if (++s == a.stages) { s = 0; parity ^= 1u; }
        const float sum = half_warp_sum((g.lane & 15) < a.warps ? part[pass][g.lane & 15] : 0.f);
        pass ^= 1;
        // zh mean(a zh) rstd = zh (rstd^2 mean(a z)): the three factors apart, since rstd^3 leaves fp32's range early
        const float mx = -rs * (rs * (sum * inv_d));
        const f2 rs2 = pair(rs, rs), mx2 = pair(mx, mx);
        T* dx = static_cast<T*>(a.out) + r * a.out_stride;
#pragma unroll
        for (int q = 0; q < EPT / 8; ++q) {
            f2 gq[4], o[4];
            cols.weights(gw, q, gq);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f2 zh = mul2(word_pair<T>(zw + q * W, i), rs2), u = word_pair<T>(uw + q * W, i);
                dg[4 * q + i] = fma2(u, zh, dg[4 * q + i]);
                if constexpr (RES) o[i] = fma2(mul2(u, gq[i]), rs2, fma2(zh, mx2, word_pair<T>(ww + q * W, i)));
                else o[i] = fma2(mul2(u, gq[i]), rs2, mul2(zh, mx2));
            }
            if (a.out) cols.store(dx, q, o);
        }
    }
    if (!a.partial) return;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");         // the sums' last step may be brought up
    // The block's sums: every group leaves its own in the ring (all copies have landed and been read), then all threads add
    // them, the groups in order.
    float* sums = reinterpret_cast<float*>(raw + a.ring);
    __syncthreads();
    float* mine = sums + static_cast<size_t>(g.id) * a.d;
#pragma unroll
    for (int i = 0; i < C::PAIRS; ++i) {
        const float2 p = split(dg[i]);
        const int c0 = cols.first + C::STEP * (2 * i / C::N) + 2 * i % C::N, c1 = cols.first + C::STEP * ((2 * i + 1) / C::N) + (2 * i + 1) % C::N;
        if (c0 < a.d) mine[c0] = p.x;
        if (c1 < a.d) mine[c1] = p.y;
    }
    __syncthreads();
    float* out = a.partial + static_cast<size_t>(blockIdx.x) * a.d;
    for (int c = threadIdx.x; c < a.d; c += blockDim.x) {
        float v = sums[c];
        for (int q = 1; q < a.groups; ++q) v += sums[static_cast<size_t>(q) * a.d + c];
        out[c] = v;
    }
}

// ------------------------------------------------------------------------------------ narrow rows
constexpr int NARROW_BYTES = 512, NARROW_THREADS = 512, NARROW_WARPS = NARROW_THREADS / 32;
constexpr int FORWARD_UNROLL = 4, BACKWARD_UNROLL = 2;  // rows under way per lane group

template <typename T> __device__ __forceinline__ void narrow_weights(const RmsArgs& a, int c, bool has, f2* gw) {
    if (a.w_fp32) Piece<T>::weights(static_cast<const float*>(a.g), c, has, 1.f, gw);
    else Piece<T>::weights(static_cast<const T*>(a.g), c, has, 1.f, gw);
}

template <typename T, int L, bool RES, bool F8>
__global__ void __launch_bounds__(NARROW_THREADS) rms_forward_narrow(const RmsArgs a) {
    using P = Piece<T>;
    constexpr int PER = 32 / L;                         // rows of a warp at once
    constexpr int GL = sizeof(T) == 2 && L > 16 ? 16 : L;                   // lanes of 128 columns
    const int lane = threadIdx.x & 31, c = (lane & (L - 1)) * P::N;
    const bool has = c < a.d;
    const float inv_d = 1.f / static_cast<float>(a.d);
    f2 gw[P::PAIRS];
    narrow_weights<T>(a, c, has, gw);
    const int step = gridDim.x * NARROW_WARPS * PER * FORWARD_UNROLL;
    for (int r0 = (blockIdx.x * NARROW_WARPS + (threadIdx.x >> 5)) * PER * FORWARD_UNROLL; r0 < a.rows; r0 += step) {
        uint4 qx[FORWARD_UNROLL], qr[FORWARD_UNROLL];
#pragma unroll
        for (int u = 0; u < FORWARD_UNROLL; ++u) {
            const int r = r0 + u * PER + lane / L;
            qx[u] = qr[u] = make_uint4(0u, 0u, 0u, 0u);
            if (has && r < a.rows) {
                qx[u] = *reinterpret_cast<const uint4*>(a.in[0].at(r) + c * sizeof(T));
                if constexpr (RES) qr[u] = *reinterpret_cast<const uint4*>(a.in[1].at(r) + c * sizeof(T));
            }
        }
#pragma unroll
        for (int u = 0; u < FORWARD_UNROLL; ++u) {
            const int r = r0 + u * PER + lane / L;
            const bool mine = has && r < a.rows;
            f2 v[P::PAIRS];
            P::unpack(qx[u], v);
            if constexpr (RES) {
                f2 w[P::PAIRS];
                P::unpack(qr[u], w);
#pragma unroll
                for (int i = 0; i < P::PAIRS; ++i) v[i] = round_pair<T>(add2(v[i], w[i]));
                if (a.z && mine) *reinterpret_cast<uint4*>(static_cast<T*>(a.z) + r * a.z_stride + c) = P::pack(v);
            }
            f2 sq = 0ull;
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) sq = fma2(v[i], v[i], sq);
            const float2 t = split(sq);
            const float rs = 1.f / sqrtf(fmaf(lanes_sum<L>(t.x + t.y), inv_d, a.eps));
            const f2 rs2 = pair(rs, rs);
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) v[i] = mul2(mul2(v[i], rs2), gw[i]);
            if constexpr (F8) {
                float m = 0.f;
#pragma unroll
                for (int i = 0; i < P::PAIRS; ++i) m = max_abs(v[i], m);
                const float2 s = scale_of(lanes_max<GL>(m));
                uint32_t w[P::PAIRS];
#pragma unroll
                for (int i = 0; i < P::PAIRS; ++i) { const float2 e = split(mul2(v[i], pair(s.y, s.y))); w[i] = e4m3x2(e.x, e.y); }
                if (mine) {
                    uint8_t* to = static_cast<uint8_t*>(a.out) + r * a.out_stride + c;
                    if constexpr (P::PAIRS == 4) *reinterpret_cast<uint2*>(to) = make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
                    else *reinterpret_cast<uint32_t*>(to) = w[0] | w[1] << 16;
                    if (c % GROUP == 0) a.scales[static_cast<long>(r) * a.n_scales + c / GROUP] = s.x;
                }
            } else if (mine) *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + r * a.out_stride + c) = P::pack(v);
            if (mine && c == 0 && a.rstd) a.rstd[r] = rs;
        }
    }
}

template <typename T, int L, bool RES>
__global__ void __launch_bounds__(NARROW_THREADS, 2) rms_backward_narrow(const RmsArgs a) {
    using P = Piece<T>;
    constexpr int PER = 32 / L;
    __shared__ float sums[NARROW_WARPS][NARROW_BYTES / 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, c = (lane & (L - 1)) * P::N;
    const bool has = c < a.d;
    const float inv_d = 1.f / static_cast<float>(a.d);
    f2 gw[P::PAIRS], dg[P::PAIRS];
    narrow_weights<T>(a, c, has, gw);
#pragma unroll
    for (int i = 0; i < P::PAIRS; ++i) dg[i] = 0ull;
    const int step = gridDim.x * NARROW_WARPS * PER * BACKWARD_UNROLL;
    for (int r0 = (blockIdx.x * NARROW_WARPS + warp) * PER * BACKWARD_UNROLL; r0 < a.rows; r0 += step) {
        uint4 qz[BACKWARD_UNROLL], qu[BACKWARD_UNROLL], qw[BACKWARD_UNROLL];
        float rs[BACKWARD_UNROLL];
#pragma unroll
        for (int u = 0; u < BACKWARD_UNROLL; ++u) {
            const int r = r0 + u * PER + lane / L;
            qz[u] = qu[u] = qw[u] = make_uint4(0u, 0u, 0u, 0u);
            rs[u] = 0.f;
            if (has && r < a.rows) {
                qz[u] = *reinterpret_cast<const uint4*>(a.in[0].at(r) + c * sizeof(T));
                qu[u] = *reinterpret_cast<const uint4*>(a.in[1].at(r) + c * sizeof(T));
                if constexpr (RES) qw[u] = *reinterpret_cast<const uint4*>(a.in[2].at(r) + c * sizeof(T));
                rs[u] = a.rstd[r];
            }
        }
#pragma unroll
        for (int u = 0; u < BACKWARD_UNROLL; ++u) {
            const int r = r0 + u * PER + lane / L;
            f2 z[P::PAIRS], dy[P::PAIRS];
            P::unpack(qz[u], z);
            P::unpack(qu[u], dy);
            const f2 rs2 = pair(rs[u], rs[u]);
            f2 sum = 0ull;
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) {
                z[i] = mul2(z[i], rs2);                                     // zh; 0 in lanes and rows that do not exist
                dg[i] = fma2(dy[i], z[i], dg[i]);
                dy[i] = mul2(dy[i], gw[i]);
                sum = fma2(dy[i], z[i], sum);
            }
            const float2 p = split(sum);
            const float mx = -rs[u] * (lanes_sum<L>(p.x + p.y) * inv_d);
            const f2 mx2 = pair(mx, mx);
            f2 w[P::PAIRS];
            P::unpack(qw[u], w);
#pragma unroll
            for (int i = 0; i < P::PAIRS; ++i) z[i] = fma2(dy[i], rs2, RES ? fma2(z[i], mx2, w[i]) : mul2(z[i], mx2));
            if (a.out && has && r < a.rows) *reinterpret_cast<uint4*>(static_cast<T*>(a.out) + r * a.out_stride + c) = P::pack(z);
        }
    }
    if (!a.partial) return;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    // the warp's rows at once, then the block's warps in order
#pragma unroll
    for (int i = 0; i < P::PAIRS; ++i) {
        float2 p = split(dg[i]);
#pragma unroll
        for (int o = L; o < 32; o <<= 1) { p.x += __shfl_xor_sync(0xffffffffu, p.x, o); p.y += __shfl_xor_sync(0xffffffffu, p.y, o); }
        if (lane < L && has) { sums[warp][c + 2 * i] = p.x; sums[warp][c + 2 * i + 1] = p.y; }
    }
    __syncthreads();
    float* out = a.partial + static_cast<size_t>(blockIdx.x) * a.d;
    for (int k = threadIdx.x; k < a.d; k += NARROW_THREADS) {
        float v = 0.f;
        for (int w = 0; w < NARROW_WARPS; ++w) v += sums[w][k];
        out[k] = v;
    }
}

// ------------------------------------------------------------------------------------ generic kernels
// A block per row; a warp takes 128 columns at a time, a lane every 32nd of them.
constexpr int GEN_THREADS = 512, GEN_WARPS = GEN_THREADS / 32;
struct GenArgs {
    const void *x, *r, *g;                              // backward: z, dz, weight
    const void* dy;
    long rows, d, x_stride, r_stride, dy_stride, out_stride, z_stride;
    int w_fp32;
    float eps;
    void *out, *z;
    float *scales, *rstd;
    long n_scales;
};
template <typename T> __device__ __forceinline__ float weight_at(const GenArgs& a, long c) {
    if (!a.g) return 1.f;
    return a.w_fp32 ? static_cast<const float*>(a.g)[c] : to_f(static_cast<const T*>(a.g)[c]);
}

template <typename T, bool F8>
__global__ void __launch_bounds__(GEN_THREADS) rms_forward_generic(const GenArgs a) {
    __shared__ float2 part[GEN_WARPS];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* x = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* r = a.r ? static_cast<const T*>(a.r) + row * a.r_stride : nullptr;
        T* z = a.z ? static_cast<T*>(a.z) + row * a.z_stride : nullptr;
        float s = 0.f;
        for (long c = threadIdx.x; c < a.d; c += GEN_THREADS) {
            T v = x[c];
            if (r) v = from_f<T>(to_f(v) + to_f(r[c]));
            if (z) z[c] = v;
            s += to_f(v) * to_f(v);
        }
        const float rs = 1.f / sqrtf(block_sum2<GEN_THREADS>(s, 0.f, part).x / static_cast<float>(a.d) + a.eps);
        // block_sum2's barriers: z is complete, whichever thread wrote it
        for (long c0 = static_cast<long>(warp) * GROUP; c0 < a.d; c0 += GEN_WARPS * GROUP) {
            float v[4], m = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const long c = c0 + 32 * i + lane;
                v[i] = 0.f;
                if (c < a.d) {
                    T e = z ? z[c] : x[c];
                    if (r && !z) e = from_f<T>(to_f(e) + to_f(r[c]));
                    v[i] = to_f(e) * rs * weight_at<T>(a, c);
                }
                m = fmaxf(m, fabsf(v[i]));
            }
            float2 sc = make_float2(1.f, 1.f);
            if constexpr (F8) {
                sc = scale_of(lanes_max<32>(m));
                if (lane == 0) a.scales[row * a.n_scales + c0 / GROUP] = sc.x;
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const long c = c0 + 32 * i + lane;
                if (c < a.d) {
                    if constexpr (F8) static_cast<uint8_t*>(a.out)[row * a.out_stride + c] = e4m3(v[i] * sc.y);
                    else static_cast<T*>(a.out)[row * a.out_stride + c] = from_f<T>(v[i]);
                }
            }
        }
        if (threadIdx.x == 0 && a.rstd) a.rstd[row] = rs;
    }
}

template <typename T>
__global__ void __launch_bounds__(GEN_THREADS) rms_backward_dx_generic(const GenArgs a) {
    __shared__ float2 part[GEN_WARPS];
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* z = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const T* dz = a.r ? static_cast<const T*>(a.r) + row * a.r_stride : nullptr;
        const float rs = a.rstd[row];
        float s = 0.f;
#pragma unroll 4
        for (long c = threadIdx.x; c < a.d; c += GEN_THREADS) s += to_f(dy[c]) * weight_at<T>(a, c) * to_f(z[c]);
        const float mx = rs * (rs * (block_sum2<GEN_THREADS>(s, 0.f, part).x / static_cast<float>(a.d)));
        T* dx = static_cast<T*>(a.out) + row * a.out_stride;
#pragma unroll 4
        for (long c = threadIdx.x; c < a.d; c += GEN_THREADS) {
            float v = rs * (to_f(dy[c]) * weight_at<T>(a, c)) - to_f(z[c]) * rs * mx;
            if (dz) v += to_f(dz[c]);
            dx[c] = from_f<T>(v);
        }
    }
}

// Column sums of dy zh over one slice of rows: block (column tile, slice) -> partial[slice][d].
constexpr int COL_TILE = 32, COL_ROWS = 16, FIN_ROWS = 32;
template <typename T>
__global__ void __launch_bounds__(COL_TILE * COL_ROWS)
rms_backward_columns(const T* __restrict__ dy, long dy_stride, const T* __restrict__ z, long z_stride, long rows, long d,
                     const float* __restrict__ rstd, float* __restrict__ partial) {
    __shared__ float part[COL_ROWS][COL_TILE];
    const int cc = threadIdx.x % COL_TILE, rr = threadIdx.x / COL_TILE;
    const long c = static_cast<long>(blockIdx.x) * COL_TILE + cc;
    const long per = (rows + gridDim.y - 1) / gridDim.y;
    const long r0 = blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
    float s = 0.f;
    if (c < d)
#pragma unroll 4
        for (long r = r0 + rr; r < r1; r += COL_ROWS) s += to_f(dy[r * dy_stride + c]) * (to_f(z[r * z_stride + c]) * rstd[r]);
    part[rr][cc] = s;
    __syncthreads();
    if (rr == 0 && c < d) {
        for (int i = 1; i < COL_ROWS; ++i) s += part[i][cc];
        partial[static_cast<long>(blockIdx.y) * d + c] = s;
    }
}

// dweight = sums of the partial column sums, slices in a fixed order: 32 columns per block, 32 threads a column.
template <typename W>
__global__ void __launch_bounds__(COL_TILE * FIN_ROWS)
rms_backward_finish(const float* __restrict__ partial, int slices, long d, W* __restrict__ dg) {
    __shared__ float part[FIN_ROWS][COL_TILE + 1];
    const int cc = threadIdx.x % COL_TILE, rr = threadIdx.x / COL_TILE;
    const long c = static_cast<long>(blockIdx.x) * COL_TILE + cc;
    float s = 0.f;
    asm volatile("griddepcontrol.wait;" ::: "memory");                      // for the end of the kernel before
    if (c < d) {
#pragma unroll 4
        for (int i = rr; i < slices; i += FIN_ROWS) s += partial[static_cast<long>(i) * d + c];
    }
    part[rr][cc] = s;
    __syncthreads();
    s = warp_sum(part[cc][rr]);                             // warp rr: the 32 sums of column rr
    const long out = static_cast<long>(blockIdx.x) * COL_TILE + rr;
    if (cc == 0 && out < d) dg[out] = from_f<W>(s);
}

// ------------------------------------------------------------------------------------ host side
constexpr int64_t MAX_D = int64_t{1} << 30;

int slices_for(int64_t rows) { return static_cast<int>(rows < 1 ? 1 : rows > MAX_SLICES ? MAX_SLICES : rows); }
int grid_rows(int64_t rows) { return static_cast<int>(std::min<int64_t>(rows, static_cast<int64_t>(sm_count()) * 4)); }

// Shape of a row kernel's launch: `na` arrays in the ring.  grid 0: the row is too wide for shared memory.
struct RowShape { int ept, threads, grid, smem; };
RowShape row_shape(RmsArgs* a, size_t elem, int na, bool backward) {
    RowShape s;
    // Elements per thread: a warp costs about 8 instructions for each of its threads' elements and 110 for the rest of a row
    // (waits, sums over the warp and the group).  Backward, three rows in their own type and the column sums stay in registers: 24
    // elements are the most without spills (2^25 bf16 elements, with dz: 52 to 58 us at 1024 to 12288 columns; 32 elements: 62 to
    // 66), so 32 are taken only for 16-bit rows that 24 cannot hold.
    const int widest = backward && (elem == 4 || na == 3) ? 24 : 32;
    s.ept = 0;
    int best = 1 << 30;
    for (int ept : {8, 16, widest}) {
        const int warps = (a->d + 32 * ept - 1) / (32 * ept), cost = warps * (8 * ept + 110);
        if (warps <= MAX_GROUP_WARPS && cost < best) { best = cost; s.ept = ept; a->warps = warps; }
    }
    if (s.ept == 0 && elem == 2) { s.ept = 32; a->warps = (a->d + 1023) / 1024; }
    if (s.ept == 0) { s.grid = 0; return s; }
    const int most = (backward ? BACKWARD_WARPS : FORWARD_WARPS) / a->warps, sms = sm_count();
    a->groups = std::max(1, a->warps > 1 ? std::min(most, 15) : most);          // named barriers 1 to 15
    while (a->groups > 1 && static_cast<int64_t>(a->groups - 1) * sms >= a->rows) --a->groups;   // few rows: spread over the SMs
    a->cap = static_cast<int>((a->d * elem + 15) / 16 * 16 + 16);
    a->slot = na * a->cap + (backward ? 16 : 0);
    auto ring = [&] { return FULL_BYTES + a->groups * PART_BYTES + 4 * 32 * s.ept * a->warps; };
    while (a->groups > 1 && ring() + a->groups * 2 * a->slot > MAX_SMEM) --a->groups;
    a->ring = ring();
    a->stages = std::min(MAX_STAGES, (MAX_SMEM - a->ring) / (a->groups * a->slot));
    s.threads = 32 * a->warps * a->groups;
    s.smem = a->ring + a->groups * a->stages * a->slot;
    if (backward) s.smem = std::max<int>(s.smem, a->ring + 4 * a->d * a->groups);   // the groups' sums take its place
    const int64_t blocks = (a->rows + a->groups - 1) / a->groups;
    s.grid = a->stages >= 1 && s.smem <= MAX_SMEM ? static_cast<int>(std::min<int64_t>(blocks, std::min(sms, MAX_SLICES))) : 0;
    return s;
}

template <void (*kern)(const RmsArgs)> cudaError_t launch_rows(const RmsArgs& a, const RowShape& s, cudaStream_t st) {
    static std::atomic<int> raised[64];                                         // of this kernel, per device
    int dev = 0;
    if (cudaError_t e = cudaGetDevice(&dev); e != cudaSuccess) return e;
    if (dev < 0 || dev >= 64 || !raised[dev].load(std::memory_order_acquire)) {
        if (cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM); e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64) raised[dev].store(1, std::memory_order_release);
    }
    kern<<<s.grid, s.threads, s.smem, st>>>(a);
    return cudaGetLastError();
}
template <typename T, bool VEC, bool RES, bool F8> cudaError_t forward_rows(const RmsArgs& a, const RowShape& s, cudaStream_t st) {
    switch (s.ept) {
        case 8: return launch_rows<rms_forward_rows<T, VEC, 8, RES, F8>>(a, s, st);
        case 16: return launch_rows<rms_forward_rows<T, VEC, 16, RES, F8>>(a, s, st);
        default: return launch_rows<rms_forward_rows<T, VEC, 32, RES, F8>>(a, s, st);
    }
}
template <typename T, bool VEC, bool RES> cudaError_t backward_rows(const RmsArgs& a, const RowShape& s, cudaStream_t st) {
    switch (s.ept) {
        case 8: return launch_rows<rms_backward_rows<T, VEC, 8, RES>>(a, s, st);
        case 16: return launch_rows<rms_backward_rows<T, VEC, 16, RES>>(a, s, st);
        case 24: return launch_rows<rms_backward_rows<T, VEC, 24, RES>>(a, s, st);
        default: return launch_rows<rms_backward_rows<T, VEC, sizeof(T) == 4 ? 24 : 32, RES>>(a, s, st);     // fp32: at most 24
    }
}

// Blocks of a narrow launch: `per_sm` an SM at most, none without rows.
int narrow_grid(int64_t rows, int lanes, int unroll, int per_sm) {
    const int64_t per = static_cast<int64_t>(NARROW_WARPS) * (32 / lanes) * unroll;
    return static_cast<int>(std::min<int64_t>((rows + per - 1) / per, static_cast<int64_t>(per_sm) * sm_count()));
}
int narrow_lanes(int64_t bytes) { return bytes <= 128 ? 8 : bytes <= 256 ? 16 : 32; }

// Calls f with true or false as a type.
template <typename F> auto with_bool(bool b, F f) { return b ? f(std::true_type{}) : f(std::false_type{}); }
// Calls f with a null pointer of the element type.
template <typename F> int with_type(int dtype, F f) {
    if (dtype == VPCE_BF16) return f(static_cast<__nv_bfloat16*>(nullptr));
    if (dtype == VPCE_F16) return f(static_cast<__half*>(nullptr));
    return f(static_cast<float*>(nullptr));
}

struct Forward {
    const void* x; int x_dtype; int64_t rows, d, xs; const void* r; int64_t rs; const void* g; int w_dtype; double eps;
    void* out; int64_t os; float* scales; void* z; int64_t zs; float* rstd; cudaStream_t st;
};

template <typename T, bool RES, bool F8> int forward_typed(const Forward& f) {
    const size_t e = sizeof(T);
    const int64_t n_scales = (f.d + GROUP - 1) / GROUP;
    if (f.d <= MAX_ROW && f.rows <= MAX_ROWS) {
        RmsArgs a{};
        a.in[0] = Rows{f.x, static_cast<long>(f.xs * e)};
        a.in[1] = Rows{f.r, static_cast<long>(f.rs * e)};
        a.rows = static_cast<int>(f.rows); a.d = static_cast<int>(f.d); a.w_fp32 = f.w_dtype == VPCE_F32; a.eps = static_cast<float>(f.eps);
        a.g = f.g; a.out = f.out; a.z = f.z; a.out_stride = f.os; a.z_stride = f.zs; a.scales = f.scales;
        a.n_scales = static_cast<int>(n_scales); a.rstd = f.rstd;
        // 8-bit rows: a thread stores 16 / e bytes at once
        const bool out_vec = F8 ? aligned_to(f.out, 16 / e) && f.os % (16 / e) == 0 : rows_aligned(f.out, f.os, e);
        const bool vec = f.d * e % 16 == 0 && rows_aligned(f.x, f.xs, e) && (!RES || rows_aligned(f.r, f.rs, e)) && out_vec &&
                         (!f.z || rows_aligned(f.z, f.zs, e));
        if (vec && f.d * e <= NARROW_BYTES) {
            const int lanes = narrow_lanes(f.d * e), grid = narrow_grid(f.rows, lanes, FORWARD_UNROLL, 4);
            if (lanes == 8) rms_forward_narrow<T, 8, RES, F8><<<grid, NARROW_THREADS, 0, f.st>>>(a);
            else if (lanes == 16) rms_forward_narrow<T, 16, RES, F8><<<grid, NARROW_THREADS, 0, f.st>>>(a);
            else rms_forward_narrow<T, 32, RES, F8><<<grid, NARROW_THREADS, 0, f.st>>>(a);
            return code(cudaGetLastError());
        }
        const RowShape s = row_shape(&a, e, RES ? 2 : 1, false);
        if (s.grid > 0) return code(vec ? forward_rows<T, true, RES, F8>(a, s, f.st) : forward_rows<T, false, RES, F8>(a, s, f.st));
    }
    GenArgs a{};
    a.x = f.x; a.r = f.r; a.g = f.g; a.rows = f.rows; a.d = f.d; a.x_stride = f.xs; a.r_stride = f.rs; a.out_stride = f.os; a.z_stride = f.zs;
    a.w_fp32 = f.w_dtype == VPCE_F32; a.eps = static_cast<float>(f.eps); a.out = f.out; a.z = f.z; a.scales = f.scales; a.rstd = f.rstd;
    a.n_scales = n_scales;
    rms_forward_generic<T, F8><<<grid_rows(f.rows), GEN_THREADS, 0, f.st>>>(a);
    return code(cudaGetLastError());
}

struct Backward {
    const void* dy; int64_t dys; const void* dz; int64_t dzs; const void* z; int64_t zs; int x_dtype; int64_t rows, d; const void* g;
    int w_dtype; const float* rstd; void* dx; int64_t dxs; void* dg; float* partial; cudaStream_t st;
};

// The last step of the sums over rows, brought up while the kernel before it still runs (2 us less in a small backward pass).
cudaError_t finish(const Backward& b, int slices) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(static_cast<unsigned>((b.d + COL_TILE - 1) / COL_TILE));
    cfg.blockDim = dim3(COL_TILE * FIN_ROWS);
    cfg.stream = b.st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaError_t e = cudaSuccess;
    with_type(b.w_dtype, [&](auto* w) {
        using W = std::remove_pointer_t<decltype(w)>;
        const float* partial = b.partial;
        e = cudaLaunchKernelEx(&cfg, rms_backward_finish<W>, partial, slices, static_cast<long>(b.d), static_cast<W*>(b.dg));
        return 0;
    });
    return e;
}

template <typename T, bool RES> int backward_typed(const Backward& b) {
    const size_t e = sizeof(T);
    const int slices = slices_for(b.rows);
    if (b.d <= MAX_ROW && b.rows > 0 && b.rows <= MAX_ROWS) {
        RmsArgs a{};
        a.in[0] = Rows{b.z, static_cast<long>(b.zs * e)};
        a.in[1] = Rows{b.dy, static_cast<long>(b.dys * e)};
        a.in[2] = Rows{b.dz, static_cast<long>(b.dzs * e)};
        a.rows = static_cast<int>(b.rows); a.d = static_cast<int>(b.d); a.w_fp32 = b.w_dtype == VPCE_F32; a.g = b.g;
        a.out = b.dx; a.out_stride = b.dxs; a.rstd = const_cast<float*>(b.rstd); a.partial = b.dg ? b.partial : nullptr;
        const bool vec = b.d * e % 16 == 0 && rows_aligned(b.z, b.zs, e) && rows_aligned(b.dy, b.dys, e) &&
                         (!RES || rows_aligned(b.dz, b.dzs, e)) && (!b.dx || rows_aligned(b.dx, b.dxs, e));
        if (vec && b.d * e <= NARROW_BYTES) {
            const int lanes = narrow_lanes(b.d * e), grid = std::min(narrow_grid(b.rows, lanes, BACKWARD_UNROLL, 2), slices);
            if (lanes == 8) rms_backward_narrow<T, 8, RES><<<grid, NARROW_THREADS, 0, b.st>>>(a);
            else if (lanes == 16) rms_backward_narrow<T, 16, RES><<<grid, NARROW_THREADS, 0, b.st>>>(a);
            else rms_backward_narrow<T, 32, RES><<<grid, NARROW_THREADS, 0, b.st>>>(a);
            if (a.partial && finish(b, grid) != cudaSuccess) return VPCE_CUDA_ERROR;
            return code(cudaGetLastError());
        }
        const RowShape s = row_shape(&a, e, RES ? 3 : 2, true);
        if (s.grid > 0) {
            if (cudaError_t err = vec ? backward_rows<T, true, RES>(a, s, b.st) : backward_rows<T, false, RES>(a, s, b.st); err != cudaSuccess)
                return VPCE_CUDA_ERROR;
            if (a.partial && finish(b, s.grid) != cudaSuccess) return VPCE_CUDA_ERROR;
            return code(cudaGetLastError());
        }
    }
    if (b.dg) {
        const unsigned tiles = static_cast<unsigned>((b.d + COL_TILE - 1) / COL_TILE);
        rms_backward_columns<T><<<dim3(tiles, slices), COL_TILE * COL_ROWS, 0, b.st>>>(
            static_cast<const T*>(b.dy), b.dys, static_cast<const T*>(b.z), b.zs, b.rows, b.d, b.rstd, b.partial);
        if (finish(b, slices) != cudaSuccess) return VPCE_CUDA_ERROR;
    }
    if (b.dx && b.rows > 0) {                               // after the column sums: dx may be dy itself
        GenArgs a{};
        a.x = b.z; a.r = b.dz; a.dy = b.dy; a.g = b.g; a.rows = b.rows; a.d = b.d; a.x_stride = b.zs; a.r_stride = b.dzs; a.dy_stride = b.dys;
        a.out_stride = b.dxs; a.w_fp32 = b.w_dtype == VPCE_F32; a.out = b.dx; a.rstd = const_cast<float*>(b.rstd);
        rms_backward_dx_generic<T><<<grid_rows(b.rows), GEN_THREADS, 0, b.st>>>(a);
    }
    return code(cudaGetLastError());
}

bool sizes_ok(int64_t rows, int64_t d) { return rows >= 0 && d >= 1 && d <= MAX_D && rows <= (int64_t{1} << 40); }

int forward_any(Forward f, bool fp8) {
    if (!sizes_ok(f.rows, f.d) || !known_type(f.x_dtype) || !(f.eps >= 0.0)) return VPCE_INVALID_ARG;
    if (!f.g) f.w_dtype = f.x_dtype;
    if (!known_type(f.w_dtype) || (f.w_dtype != f.x_dtype && f.w_dtype != VPCE_F32)) return VPCE_INVALID_ARG;
    if (!f.r && f.z) return VPCE_INVALID_ARG;
    if (f.rows == 0) return VPCE_OK;
    if (!f.x || !f.out || f.xs < f.d || f.os < f.d || (f.r && f.rs < f.d) || (f.z && f.zs < f.d) || (fp8 && !f.scales)) return VPCE_INVALID_ARG;
    const size_t e = elem_bytes(f.x_dtype);
    if (!aligned_to(f.x, e) || !aligned_to(f.r, e) || !aligned_to(f.z, e) || (!fp8 && !aligned_to(f.out, e)) ||
        !aligned_to(f.g, elem_bytes(f.w_dtype)) || !aligned_to(f.rstd, 4) || !aligned_to(f.scales, 4))
        return VPCE_UNSUPPORTED;
    return with_type(f.x_dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return with_bool(f.r != nullptr, [&](auto res) {
            return with_bool(fp8, [&](auto f8) { return forward_typed<T, decltype(res)::value, decltype(f8)::value>(f); });
        });
    });
}

}  // namespace

extern "C" {

int vp_rms_forward(const void* x, int x_dtype, int64_t rows, int64_t d, int64_t x_stride, const void* residual, int64_t residual_stride,
                   const void* weight, int w_dtype, double eps, void* y, int64_t y_stride, void* z, int64_t z_stride, float* rstd,
                   void* stream) {
    return forward_any(Forward{x, x_dtype, rows, d, x_stride, residual, residual_stride, weight, w_dtype, eps, y, y_stride, nullptr, z, z_stride,
                               rstd, static_cast<cudaStream_t>(stream)}, false);
}

int vp_rms_forward_fp8(const void* x, int x_dtype, int64_t rows, int64_t d, int64_t x_stride, const void* residual, int64_t residual_stride,
                       const void* weight, int w_dtype, double eps, void* q, int64_t q_stride, float* scales, void* z, int64_t z_stride,
                       float* rstd, void* stream) {
    return forward_any(Forward{x, x_dtype, rows, d, x_stride, residual, residual_stride, weight, w_dtype, eps, q, q_stride, scales, z, z_stride,
                               rstd, static_cast<cudaStream_t>(stream)}, true);
}

size_t vp_rms_workspace_bytes(int64_t rows, int64_t d) {
    if (!sizes_ok(rows, d)) return 0;
    return static_cast<size_t>(slices_for(rows)) * static_cast<size_t>(d) * sizeof(float);
}

int vp_rms_backward(const void* dy, int64_t dy_stride, const void* dz, int64_t dz_stride, const void* z, int64_t z_stride, int x_dtype,
                    int64_t rows, int64_t d, const void* weight, int w_dtype, const float* rstd, void* dx, int64_t dx_stride, void* dweight,
                    void* workspace, size_t workspace_bytes, void* stream) {
    if (!sizes_ok(rows, d) || !known_type(x_dtype)) return VPCE_INVALID_ARG;
    if (!weight && !dweight) w_dtype = x_dtype;
    if (!known_type(w_dtype) || (w_dtype != x_dtype && w_dtype != VPCE_F32)) return VPCE_INVALID_ARG;
    if (!dx && !dweight) return VPCE_OK;
    if (rows > 0 && (!dy || !z || !rstd || dy_stride < d || z_stride < d || (dz && dz_stride < d) || (dx && dx_stride < d)))
        return VPCE_INVALID_ARG;
    const size_t e = elem_bytes(x_dtype), we = elem_bytes(w_dtype);
    if (!aligned_to(dy, e) || !aligned_to(dz, e) || !aligned_to(z, e) || !aligned_to(dx, e) || !aligned_to(weight, we) ||
        !aligned_to(dweight, we) || !aligned_to(rstd, 4))
        return VPCE_UNSUPPORTED;
    if (dweight) {
        if (!workspace) return VPCE_INVALID_ARG;
        if (!aligned_to(workspace, 16)) return VPCE_UNSUPPORTED;
        if (workspace_bytes < vp_rms_workspace_bytes(rows, d)) return VPCE_WORKSPACE_TOO_SMALL;
    }
    const Backward b{dy, dy_stride, dz, dz_stride, z, z_stride, x_dtype, rows, d, weight, w_dtype, rstd, dx, dx_stride, dweight,
                     static_cast<float*>(workspace), static_cast<cudaStream_t>(stream)};
    return with_type(x_dtype, [&](auto* t) {
        using T = std::remove_pointer_t<decltype(t)>;
        return with_bool(dz != nullptr, [&](auto res) { return backward_typed<T, decltype(res)::value>(b); });
    });
}

}  // extern "C"
