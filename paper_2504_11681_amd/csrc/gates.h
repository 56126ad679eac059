// The sigmoid of gates: exp2 and 1 / x of the hardware, one unit in the last place each; with the product in the exponent 2^-24 (1 + |z|) of the result or of what is left of 1.
#pragma once
#include "common.h"

namespace tfno {

constexpr float LOG2E = 1.44269504088896340736f;

// 1 / (1 + exp(-z)), and what is left of 1.
__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * z)); }
__device__ __forceinline__ void sigmoid(float z, float &s, float &rest)
{
    const float e = __builtin_amdgcn_exp2f(-LOG2E * fabsf(z)), big = __builtin_amdgcn_rcpf(1.0f + e), small = e * big;
    s = z < 0.0f ? small : big;
    rest = z < 0.0f ? big : small;
}

}  // namespace tfno
