// Elements of the matrix operators: their types, and eight of a row at a time.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "qesgd_internal.h"

namespace {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// Eight elements from column c on; zeros past the last column.
template <typename T>
__device__ __forceinline__ void load_octet(const T *row, uint64_t c, uint64_t cols, bool vec, float (&v)[8])
{
    if (vec && c + 8 <= cols) {
        if (sizeof(T) == 4) {
            const float4 a = __ldg(reinterpret_cast<const float4 *>(row + c)), b = __ldg(reinterpret_cast<const float4 *>(row + c) + 1);
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        } else {
            const uint4 a = __ldg(reinterpret_cast<const uint4 *>(row + c));
            const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint16_t h = (uint16_t)(w[j / 2] >> (16 * (j % 2)));
                v[j] = to_float(*reinterpret_cast<const T *>(&h));
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = c + j < cols ? to_float(row[c + j]) : 0.0f;
    }
}

}  // namespace
