// Device-side helpers of the 8-bit integer matrices (tq_i8.h).
#pragma once

#include "tq_i8.h"
#include "tq_reduce.h"

namespace tq {

// What a row's elements are rounded with, from the bits of its largest magnitude A.  The code of x is the whole number nearest to
// 127 x / A.  p = x * (127 / A) in binary32 is off by two roundings, at most 127 * 2^-23 < 2^-16; where p lies nearer than 2^-14 to the
// middle between two numbers, the sides are compared exactly: 254 |x| against (2 k + 1) A, whole numbers of 32 bits and a power of two,
// which binary64 holds.  Of random elements that is one in 2^13.
struct I8Row {
    float scale, up, inverse, largest;         // up: a power of two that keeps 127 / A in range

    __device__ __forceinline__ explicit I8Row(uint32_t bits)
    {
        const float a = __uint_as_float(bits);
        const bool some = bits != 0 && bits < 0x7F800000u;
        scale = bits < 0x7F800000u ? a / 127.0f : __builtin_nanf("");
        up = !some ? 0.0f : a < 0x1p-64f ? 0x1p64f : 1.0f;
        largest = a * up;
        inverse = some ? 127.0f / largest : 0.0f;
    }
    __device__ __forceinline__ int code(float x) const
    {
        x *= up;
        const float p = x * inverse;
        float q = __builtin_rintf(p);
        if (fabsf(p - q) > 0.5f - 0x1p-14f) {
            const float k = floorf(fabsf(p));
            const double twice = 254.0 * (double)fabsf(x), middle = (2.0 * (double)k + 1.0) * (double)largest;
            const bool odd = ((int)k & 1) != 0;
            q = copysignf(twice > middle || (twice == middle && odd) ? k + 1.0f : k, p);
        }
        return (int)q;
    }
    // 8 codes, the first in the lowest byte.  A row without a usable scale has zeros: its elements may be NaN.
    __device__ __forceinline__ u32x2 codes(const float (&v)[8]) const
    {
        u32x2 w = {0, 0};
        if (inverse == 0.0f) return w;
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j / 4] |= (uint32_t)(code(v[j]) & 255) << (j % 4 * 8);
        return w;
    }
};

}  // namespace tq
