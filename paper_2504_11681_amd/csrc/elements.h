// Elements of the operators along time: float32 or BF16 in memory, float32 in registers.
#pragma once
#include "common.h"

namespace tfno {

struct bf16 { unsigned short bits; };

// Strides of a tensor [B, T, heads, D] in elements; its last axis is contiguous.
struct Strides { long long batch, token, head; };

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(bf16 v) { return __uint_as_float((unsigned)v.bits << 16); }

// The nearest BF16 value, ties to the even one; a NaN stays one.
__device__ __forceinline__ unsigned bf16_bits(float v)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    pair p;
    p.x = (__bf16)v;
    p.y = (__bf16)0.0f;
    return __builtin_bit_cast(unsigned, p) & 0xffffu;
}
__device__ __forceinline__ unsigned bf16_pair(float lo, float hi)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    pair p;
    p.x = (__bf16)lo;
    p.y = (__bf16)hi;
    return __builtin_bit_cast(unsigned, p);
}
__device__ __forceinline__ void store_element(float *p, float v) { *p = v; }
__device__ __forceinline__ void store_element(bf16 *p, float v) { p->bits = (unsigned short)bf16_bits(v); }

// Four neighbouring elements whose address is a multiple of their size.
__device__ __forceinline__ void load4(const float *p, float (&v)[4])
{
    const float4 t = *reinterpret_cast<const float4 *>(p);
    v[0] = t.x, v[1] = t.y, v[2] = t.z, v[3] = t.w;
}
__device__ __forceinline__ void load4(const bf16 *p, float (&v)[4])
{
    const uint2 t = *reinterpret_cast<const uint2 *>(p);
    v[0] = __uint_as_float(t.x << 16), v[1] = __uint_as_float(t.x & 0xffff0000u);
    v[2] = __uint_as_float(t.y << 16), v[3] = __uint_as_float(t.y & 0xffff0000u);
}
// The same as they stand in memory, for values that wait in registers.
template <class E>
struct Quad;
template <>
struct Quad<float> {
    float4 at;
    __device__ __forceinline__ void load(const float *p) { at = *reinterpret_cast<const float4 *>(p); }
    __device__ __forceinline__ void values(float (&v)[4]) const { v[0] = at.x, v[1] = at.y, v[2] = at.z, v[3] = at.w; }
};
template <>
struct Quad<bf16> {
    uint2 at;
    __device__ __forceinline__ void load(const bf16 *p) { at = *reinterpret_cast<const uint2 *>(p); }
    __device__ __forceinline__ void values(float (&v)[4]) const
    {
        v[0] = __uint_as_float(at.x << 16), v[1] = __uint_as_float(at.x & 0xffff0000u);
        v[2] = __uint_as_float(at.y << 16), v[3] = __uint_as_float(at.y & 0xffff0000u);
    }
};
__device__ __forceinline__ void store4(float *p, const float (&v)[4]) { *reinterpret_cast<float4 *>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void store4(bf16 *p, const float (&v)[4])
{
    *reinterpret_cast<uint2 *>(p) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
}

// Sum over the lanes of a group of `width` neighbouring lanes (a power of two up to 64).
__device__ __forceinline__ float group_sum(float v, int width)
{
    for (int s = 1; s < width; s <<= 1) v += __shfl_xor(v, s, 64);
    return v;
}

}  // namespace tfno
