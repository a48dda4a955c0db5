// What the norms' row kernels share: conversions, pairs of fp32, sums over a warp, rows as bulk copies into shared memory, and how a
// row's columns lie over a warp's threads.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "sm100_ptx.cuh"
#include "vp_ce.h"
#include "vp_ce_types.h"

namespace {

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
template <typename T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

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

// ------------------------------------------------------------------------------------ host side
size_t elem_bytes(int t) { return t == VPCE_F32 ? 4 : 2; }
bool known_type(int t) { return t == VPCE_BF16 || t == VPCE_F16 || t == VPCE_F32; }
bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

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

bool rows_aligned(const void* p, int64_t stride, size_t e) { return aligned_to(p, 16) && stride * e % 16 == 0; }

int code(cudaError_t e) { return e == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR; }


}  // namespace
