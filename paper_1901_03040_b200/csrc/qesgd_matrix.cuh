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

// Bits of a 16-bit magnitude as a 32-bit float's, in order, infinities and NaN at 0x7F800000 or more.
template <typename T>
__device__ __forceinline__ uint32_t top16(uint32_t bits);
template <>
__device__ __forceinline__ uint32_t top16<__nv_bfloat16>(uint32_t bits) { return bits << 16; }
template <>
__device__ __forceinline__ uint32_t top16<__half>(uint32_t bits)
{
    const uint16_t h = (uint16_t)bits;
    return bits >= 0x7C00u ? 0x7F800000u : __float_as_uint(__half2float(*reinterpret_cast<const __half *>(&h)));
}
// ---- octets: eight neighbouring elements as they lie in memory -------------------------------------------------
// A 16-bit octet is four words, a 32-bit one eight.
template <typename T>
struct Octet {
    static constexpr int WORDS = (int)sizeof(T) * 2;
    uint32_t w[WORDS];
};
template <typename T>
__device__ __forceinline__ Octet<T> no_octet()
{
    Octet<T> o;
#pragma unroll
    for (int i = 0; i < Octet<T>::WORDS; ++i) o.w[i] = 0u;
    return o;
}
// Elements c to c + 7 of a row; zeros past the last column.  vec: rows lie on 16 bytes.  Else the 16-byte lines around a
// whole octet are loaded and shifted: every one of them holds some of its bytes, so none is outside its allocation's lines.
template <typename T>
__device__ __forceinline__ Octet<T> load_octet(const T *row, uint64_t c, uint64_t cols, bool vec)
{
    constexpr int LINES = Octet<T>::WORDS / 4;
    Octet<T> o = no_octet<T>();
    if (c + 8 <= cols) {
        if (vec) {
#pragma unroll
            for (int i = 0; i < LINES; ++i) *reinterpret_cast<uint4 *>(&o.w[4 * i]) = __ldg(reinterpret_cast<const uint4 *>(row + c) + i);
        } else {
            const uint32_t off = (uint32_t)(reinterpret_cast<uintptr_t>(row + c) & 15u), words = off / 4u, bits = off % 4u * 8u;
            const uint4 *const line = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(row + c) - off);
            uint32_t u[4 * LINES + 4];
#pragma unroll
            for (int i = 0; i < LINES; ++i) *reinterpret_cast<uint4 *>(&u[4 * i]) = __ldg(line + i);
            *reinterpret_cast<uint4 *>(&u[4 * LINES]) = off ? __ldg(line + LINES) : make_uint4(0u, 0u, 0u, 0u);
            if (words & 1u)
#pragma unroll
                for (int i = 0; i < 4 * LINES + 3; ++i) u[i] = u[i + 1];
            if (words & 2u)
#pragma unroll
                for (int i = 0; i < 4 * LINES + 2; ++i) u[i] = u[i + 2];
#pragma unroll
            for (int i = 0; i < 4 * LINES; ++i) o.w[i] = sizeof(T) == 4 ? u[i] : __funnelshift_r(u[i], u[i + 1], bits);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (c + j < cols) {
                if (sizeof(T) == 4) o.w[j % Octet<T>::WORDS] = reinterpret_cast<const uint32_t *>(row)[c + j];
                else o.w[j / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[c + j] << (16 * (j % 2));
            }
    }
    return o;
}
// Element j of an octet, and two of them (j even) from the word that holds them.
__device__ __forceinline__ float2 pair_of(uint32_t w, __nv_bfloat16) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)); }
__device__ __forceinline__ float2 pair_of(uint32_t w, __half) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
template <typename T>
__device__ __forceinline__ void values(const Octet<T> &o, float (&v)[8])
{
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(o.w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 f = pair_of(o.w[j], T());
            v[2 * j] = f.x;
            v[2 * j + 1] = f.y;
        }
    }
}
// The largest magnitude of three numbers, NaN where one of them is.
__device__ __forceinline__ float max_magnitude(float a, float b, float c)
{
    float r;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
}
// Bits of the largest magnitude, as a 32-bit float: 0x7F800000 or more where an element is not finite.  16-bit magnitudes
// are compared as they lie, by twos.
template <typename T>
__device__ __forceinline__ uint32_t top_of(const Octet<T> &o)
{
    if constexpr (sizeof(T) == 4) {
        float t = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; j += 2) t = max_magnitude(t, __uint_as_float(o.w[j]), __uint_as_float(o.w[j + 1]));
        return __float_as_uint(t);
    } else {
        uint32_t t = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) t = __vmaxu2(t, o.w[j] & 0x7FFF7FFFu);
        return top16<T>(max(t & 0xFFFFu, t >> 16));
    }
}

}  // namespace
