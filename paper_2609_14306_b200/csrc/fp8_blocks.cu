// A weight to 8 bits in blocks of 128 x 128 with a scale each (fp8_blocks.h).
//
// Bound: memory, 2 + 1 bytes an element from 16-bit types: 201088 x 2880 bf16 in 272 us, 6.4 TB/s (a plain copy: 6.56).  A CTA of 8 warps has a block: a warp 16 of its rows, which it holds in
// registers in the input's type from the load to the store, so the block is read once; its largest magnitude goes over the warps through
// shared memory.  Rows of 16-byte pieces where every row starts on a 16-byte boundary, else single elements.

#include <cuda_fp8.h>

#include <algorithm>
#include <type_traits>

#include "fp8_blocks.h"
#include "row_kernels.cuh"

namespace {

constexpr int BLOCK = 128, QB_THREADS = 256, QB_WARPS = QB_THREADS / 32, WARP_ROWS = BLOCK / QB_WARPS;

__device__ __forceinline__ uint32_t e4m3x2(float a, float b) { return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3); }

// The block's scale from its threads' largest magnitudes; writes it and returns its reciprocal.
__device__ __forceinline__ float block_scale(float m, float* out) {
    __shared__ float part[QB_WARPS];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < QB_WARPS; ++i) m = fmaxf(m, part[i]);
    const float s = m > 0.f ? fmaxf(m * (1.f / 448.f), 1.1754944e-38f) : 1.f;
    if (threadIdx.x == 0) *out = s;
    return 1.f / s;
}

template <typename T>
__global__ void __launch_bounds__(QB_THREADS) quantize_blocks_vec(const T* __restrict__ w, long rows, long d, long w_stride,
                                                               uint8_t* __restrict__ q, long q_stride, float* __restrict__ scales) {
    using P = Piece<T>;
    constexpr int LANES = BLOCK / P::N, PER = 32 / LANES, PIECES = WARP_ROWS / PER;      // lanes a row, rows at once, pieces a thread
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long c = static_cast<long>(blockIdx.x) * BLOCK + (lane % LANES) * P::N;
    const long r0 = static_cast<long>(blockIdx.y) * BLOCK + warp * WARP_ROWS + lane / LANES;
    uint4 v[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        v[i] = make_uint4(0u, 0u, 0u, 0u);
        if (c < d && r0 + i * PER < rows) v[i] = __ldcs(reinterpret_cast<const uint4*>(w + (r0 + i * PER) * w_stride + c));
    }
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        f2 e[P::PAIRS];
        P::unpack(v[i], e);
#pragma unroll
        for (int k = 0; k < P::PAIRS; ++k) { const float2 t = split(e[k]); m = fmaxf(m, fmaxf(fabsf(t.x), fabsf(t.y))); }
    }
    const float inv = block_scale(m, scales + static_cast<long>(blockIdx.y) * gridDim.x + blockIdx.x);
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        f2 e[P::PAIRS];
        P::unpack(v[i], e);
        uint32_t o[P::PAIRS];
#pragma unroll
        for (int k = 0; k < P::PAIRS; ++k) { const float2 t = split(mul2(e[k], pair(inv, inv))); o[k] = e4m3x2(t.x, t.y); }
        if (c < d && r0 + i * PER < rows) {
            uint8_t* to = q + (r0 + i * PER) * q_stride + c;
            if constexpr (P::PAIRS == 4) *reinterpret_cast<uint2*>(to) = make_uint2(o[0] | o[1] << 16, o[2] | o[3] << 16);
            else *reinterpret_cast<uint32_t*>(to) = o[0] | o[1] << 16;
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(QB_THREADS) quantize_blocks_any(const T* __restrict__ w, long rows, long d, long w_stride,
                                                               uint8_t* __restrict__ q, long q_stride, float* __restrict__ scales) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const long c0 = static_cast<long>(blockIdx.x) * BLOCK + lane, r0 = static_cast<long>(blockIdx.y) * BLOCK + warp * WARP_ROWS;
    T v[WARP_ROWS][4];
#pragma unroll
    for (int i = 0; i < WARP_ROWS; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i][k] = c0 + 32 * k < d && r0 + i < rows ? w[(r0 + i) * w_stride + c0 + 32 * k] : from_f<T>(0.f);
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < WARP_ROWS; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) m = fmaxf(m, fabsf(to_f(v[i][k])));
    const float inv = block_scale(m, scales + static_cast<long>(blockIdx.y) * gridDim.x + blockIdx.x);
#pragma unroll
    for (int i = 0; i < WARP_ROWS; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (c0 + 32 * k < d && r0 + i < rows)
                q[(r0 + i) * q_stride + c0 + 32 * k] = __nv_cvt_float_to_fp8(to_f(v[i][k]) * inv, __NV_SATFINITE, __NV_E4M3);
}

template <typename T> int quantize(const void* w, int64_t rows, int64_t d, int64_t ws, void* q, int64_t qs, float* scales, cudaStream_t st) {
    const int64_t row_blocks = (rows + BLOCK - 1) / BLOCK;
    const unsigned col_blocks = static_cast<unsigned>((d + BLOCK - 1) / BLOCK);
    constexpr int PIECE = 16 / static_cast<int>(sizeof(T));
    const bool vec = d % PIECE == 0 && rows_aligned(w, ws, sizeof(T)) && aligned_to(q, PIECE) && qs % PIECE == 0;
    for (int64_t b = 0; b < row_blocks; b += 65535) {                       // the grid's second extent ends there
        const int64_t r = b * BLOCK, n = std::min<int64_t>(rows - r, int64_t{65535} * BLOCK);
        const dim3 grid(col_blocks, static_cast<unsigned>((n + BLOCK - 1) / BLOCK));
        const T* from = static_cast<const T*>(w) + r * ws;
        uint8_t* to = static_cast<uint8_t*>(q) + r * qs;
        if (vec) quantize_blocks_vec<T><<<grid, QB_THREADS, 0, st>>>(from, n, d, ws, to, qs, scales + b * col_blocks);
        else quantize_blocks_any<T><<<grid, QB_THREADS, 0, st>>>(from, n, d, ws, to, qs, scales + b * col_blocks);
    }
    return code(cudaGetLastError());
}

}  // namespace

extern "C" int vp_fp8_quantize_blocks(const void* w, int w_dtype, int64_t rows, int64_t d, int64_t w_stride, void* q, int64_t q_stride,
                                      float* scales, void* stream) {
    if (rows < 0 || rows > (int64_t{1} << 40) || d < 1 || d > (int64_t{1} << 30) || !known_type(w_dtype)) return VPCE_INVALID_ARG;
    if (rows == 0) return VPCE_OK;
    if (!w || !q || !scales || w_stride < d || q_stride < d) return VPCE_INVALID_ARG;
    if (!aligned_to(w, elem_bytes(w_dtype)) || !aligned_to(scales, 4)) return VPCE_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (w_dtype == VPCE_BF16) return quantize<__nv_bfloat16>(w, rows, d, w_stride, q, q_stride, scales, st);
    if (w_dtype == VPCE_F16) return quantize<__half>(w, rows, d, w_stride, q, q_stride, scales, st);
    return quantize<float>(w, rows, d, w_stride, q, q_stride, scales, st);
}
