// C = A B^T on microscaled 4-bit operands (see include/qesgd.h for the layout).
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qesgd_internal.h"

namespace {

constexpr int THREADS = 256;
constexpr int TILE = 64, DEPTH = 32;

__device__ __forceinline__ float grid_value(uint32_t code)
{
    const uint32_t l = code & 7u;
    const float v = l < 4u ? 0.5f * (float)l : l < 6u ? (float)l - 2.0f : 2.0f * (float)l - 8.0f;
    return code & 8u ? -v : v;
}
__device__ __forceinline__ float scale_value(uint32_t byte, bool mx)
{
    if (mx) return byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
    return __uint_as_float((byte & 0x7Fu) << 20) * 0x1p120f;
}
__device__ __forceinline__ int exponent_of(const int32_t *p) { return p ? min(max(*p, -126), 126) : 0; }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// One CTA computes 64 x 64 of C from decoded operands in shared memory.
template <typename T>
__global__ __launch_bounds__(THREADS) void qesgd_fp4_matmul_kernel(const __grid_constant__ Fp4MatmulArgs a, bool mx)
{
    __shared__ float as[DEPTH][TILE + 1], bs[DEPTH][TILE + 1];
    qesgd_wait_for_previous();
    const uint32_t block = mx ? 32u : 16u;
    const uint64_t tiles_n = (a.N + TILE - 1) / TILE, tiles = tiles_n * ((a.M + TILE - 1) / TILE);
    const uint64_t row_bytes = (a.K + 31) / 32 * 16, scale_tiles = (a.K + 4 * block - 1) / (4 * block);
    const float power = ldexpf(1.0f, exponent_of(a.a_exponent)) , power2 = ldexpf(1.0f, exponent_of(a.b_exponent));
    const uint32_t tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    for (uint64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const uint64_t m0 = tile / tiles_n * TILE, n0 = tile % tiles_n * TILE;
        float acc[4][4] = {};
        for (uint64_t k0 = 0; k0 < a.K; k0 += DEPTH) {
            for (uint32_t i = threadIdx.x; i < TILE * DEPTH; i += THREADS) {
                const uint64_t k = k0 + i % DEPTH, block_k = k / block;
                for (int side = 0; side < 2; ++side) {
                    const uint64_t r = (side ? n0 : m0) + i / DEPTH;
                    float v = 0.0f;
                    if (r < (side ? a.N : a.M) && k < a.K) {
                        const uint32_t byte = (side ? a.b_codes : a.a_codes)[r * row_bytes + k / 2];
                        const uint32_t s = (side ? a.b_scales : a.a_scales)[(r / 128 * scale_tiles + block_k / 4) * 512 + r % 32 * 16 + r / 32 % 4 * 4 + block_k % 4];
                        v = grid_value(k % 2 ? byte >> 4 : byte & 15u) * scale_value(s, mx);
                    }
                    (side ? bs : as)[i % DEPTH][i / DEPTH] = v;
                }
            }
            __syncthreads();
            for (int k = 0; k < DEPTH; ++k)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[i][j] += as[k][ty + 16 * i] * bs[k][tx + 16 * j];
            __syncthreads();
        }
        for (int i = 0; i < 4; ++i)
            for (int j = 0; j < 4; ++j) {
                const uint64_t r = m0 + ty + 16 * i, c = n0 + tx + 16 * j;
                if (r >= a.M || c >= a.N) continue;
                T *const out = static_cast<T *>(a.c) + r * a.ldc + c;
                const float v = acc[i][j] * power * power2;
                *out = from_float<T>(a.accumulate ? (float)*out + v : v);
            }
    }
}

template <typename T>
cudaError_t launch(const Fp4MatmulArgs &a, uint32_t format, cudaStream_t stream)
{
    const uint64_t tiles = qesgd_div_up(a.M, TILE) * qesgd_div_up(a.N, TILE);
    return qesgd_launch(qesgd_fp4_matmul_kernel<T>, dim3((unsigned)(tiles < 0x7FFFFFFF ? tiles : 0x7FFFFFFF)), dim3(THREADS), stream, a, format == QESGD_FP4_MX);
}

}  // namespace

int qesgd_launch_fp4_matmul(const Fp4MatmulArgs &a, uint32_t dtype, uint32_t format, int, cudaStream_t stream, int *launched)
{
    *launched = 1;
    switch (dtype) {
        case QESGD_F32: return (int)launch<float>(a, format, stream);
        case QESGD_BF16: return (int)launch<__nv_bfloat16>(a, format, stream);
        default: return (int)launch<__half>(a, format, stream);
    }
}
