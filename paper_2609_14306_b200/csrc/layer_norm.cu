// Layer normalisation, forward and backward (layer_norm.h).
//
// Generic kernels: one block per row (grid-stride), elements read one at a time in the order of the threads, three passes
// over a row that the caches hold after the first.  They take any width, stride and alignment.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <type_traits>

#include "layer_norm.h"
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
constexpr int MAX_SLICES = 296;         // row slices of the column sums: two blocks per SM of a 148-SM device

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

// dweight, dbias = sums of the partial column sums, slices in a fixed order: 32 columns per block, 8 threads a column.
template <typename W>
__global__ void __launch_bounds__(COL_TILE * COL_ROWS)
ln_backward_finish(const float* __restrict__ partial, int slices, long d, W* __restrict__ dg, W* __restrict__ db) {
    __shared__ float2 part[COL_ROWS][COL_TILE];
    const int cc = threadIdx.x % COL_TILE, rr = threadIdx.x / COL_TILE;
    const long c = static_cast<long>(blockIdx.x) * COL_TILE + cc;
    float sg = 0.f, sb = 0.f;
    if (c < d)
        for (int s = rr; s < slices; s += COL_ROWS) {
            sg += partial[static_cast<long>(s) * 2 * d + c];
            sb += partial[static_cast<long>(s) * 2 * d + d + c];
        }
    part[rr][cc] = make_float2(sg, sb);
    __syncthreads();
    if (rr == 0 && c < d) {
        for (int i = 1; i < COL_ROWS; ++i) { sg += part[i][cc].x; sb += part[i][cc].y; }
        if (dg) dg[c] = from_f<W>(sg);
        if (db) db[c] = from_f<W>(sb);
    }
}

// ------------------------------------------------------------------------------------ host side
constexpr int64_t MAX_D = int64_t{1} << 30;

size_t elem_bytes(int t) { return t == VPCE_F32 ? 4 : 2; }
bool known_type(int t) { return t == VPCE_BF16 || t == VPCE_F16 || t == VPCE_F32; }
bool aligned_to(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

int slices_for(int64_t rows) {
    const int64_t s = (rows + 15) / 16;
    return static_cast<int>(s < 1 ? 1 : s > MAX_SLICES ? MAX_SLICES : s);
}

int grid_rows(int64_t rows) { return static_cast<int>(rows < 148 * 8 ? rows : 148 * 8); }

template <typename T, typename W>
int forward_typed(const void* x, int64_t rows, int64_t d, int64_t xs, const void* g, const void* b, float eps, void* y, int64_t ys,
                  float* mean, float* rstd, cudaStream_t st) {
    ln_forward_generic<T, W><<<grid_rows(rows), GEN_THREADS, 0, st>>>(
        static_cast<const T*>(x), rows, d, xs, static_cast<const W*>(g), static_cast<const W*>(b), eps, static_cast<T*>(y), ys, mean, rstd);
    return cudaGetLastError() == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
}

template <typename T, typename W>
int backward_typed(const void* dy, int64_t dys, const void* x, int64_t xs, int64_t rows, int64_t d, const void* g, const float* mean,
                   const float* rstd, void* dx, int64_t dxs, void* dg, void* db, float* partial, cudaStream_t st) {
    const T *dyt = static_cast<const T*>(dy), *xt = static_cast<const T*>(x);
    const unsigned col_tiles = static_cast<unsigned>((d + COL_TILE - 1) / COL_TILE);
    if (dg || db) {
        const int slices = slices_for(rows);
        ln_backward_columns<T><<<dim3(col_tiles, slices), COL_TILE * COL_ROWS, 0, st>>>(dyt, dys, xt, xs, rows, d, mean, rstd, partial);
        ln_backward_finish<W><<<col_tiles, COL_TILE * COL_ROWS, 0, st>>>(partial, slices, d, static_cast<W*>(dg), static_cast<W*>(db));
    }
    if (dx && rows > 0)                                     // after the column sums: dx may be dy itself
        ln_backward_dx_generic<T, W><<<grid_rows(rows), GEN_THREADS, 0, st>>>(dyt, dys, xt, xs, rows, d, static_cast<const W*>(g), mean,
                                                                            rstd, static_cast<T*>(dx), dxs);
    return cudaGetLastError() == cudaSuccess ? VPCE_OK : VPCE_CUDA_ERROR;
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
