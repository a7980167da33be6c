// Device-side helpers of the 4-bit matrix kernels and the distillation kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tq_device.h"
#include "tq_mx.h"

namespace tq {

constexpr uint32_t kMxGroup = 128;         // elements of a row that are kept together: 4 blocks of 32, 64 bytes of codes

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

template <int DTYPE>
struct Element;
template <>
struct Element<TQ_F32> {
    using type = float;
    static __device__ __forceinline__ float load(float x) { return x; }
    static __device__ __forceinline__ float store(float x) { return x; }
};
template <>
struct Element<TQ_BF16> {
    using type = uint16_t;
    static __device__ __forceinline__ float load(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
    static __device__ __forceinline__ uint16_t store(float x)
    {
        const bf16x2 r = {(__bf16)x, (__bf16)0.0f};
        return (uint16_t)__builtin_bit_cast(uint32_t, r);
    }
};
template <>
struct Element<TQ_F16> {
    using type = uint16_t;
    static __device__ __forceinline__ float load(uint16_t x) { return (float)__builtin_bit_cast(_Float16, x); }
    static __device__ __forceinline__ uint16_t store(float x) { return __builtin_bit_cast(uint16_t, (_Float16)x); }
};

// Two fp32 values as two 16-bit ones in a word, each rounded to the nearest.
template <int DTYPE>
__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    if constexpr (DTYPE == TQ_BF16) return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    else return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b});
}

// The same two values back.
template <int DTYPE>
__device__ __forceinline__ void unpack2(uint32_t w, float& a, float& b)
{
    if constexpr (DTYPE == TQ_BF16) {
        a = __uint_as_float(w << 16);
        b = __uint_as_float(w & 0xFFFF0000u);
    } else {
        const f16x2 h = __builtin_bit_cast(f16x2, w);
        a = (float)h.x;
        b = (float)h.y;
    }
}

// 8 consecutive elements, `n` of them there (the rest 0).  VEC: the address is 16-byte aligned.
template <int DTYPE, bool VEC>
__device__ __forceinline__ void load8(const typename Element<DTYPE>::type* p, int n, float (&v)[8])
{
    using E = Element<DTYPE>;
    if (VEC && n >= 8) {
        if constexpr (DTYPE == TQ_F32) {
            const float4_native a = *reinterpret_cast<const float4_native*>(p), b = *reinterpret_cast<const float4_native*>(p + 4);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v[j] = a[j];
                v[4 + j] = b[j];
            }
        } else {
            const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack2<DTYPE>(w[j], v[2 * j], v[2 * j + 1]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? E::load(p[j]) : 0.0f;
    }
}

template <int DTYPE, bool VEC>
__device__ __forceinline__ void store8(typename Element<DTYPE>::type* p, int n, const float (&v)[8])
{
    using E = Element<DTYPE>;
    if (VEC && n >= 8) {
        if constexpr (DTYPE == TQ_F32) {
            reinterpret_cast<float4_native*>(p)[0] = float4_native{v[0], v[1], v[2], v[3]};
            reinterpret_cast<float4_native*>(p)[1] = float4_native{v[4], v[5], v[6], v[7]};
        } else {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack2<DTYPE>(v[2 * j], v[2 * j + 1]);
            *reinterpret_cast<u32x4*>(p) = w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) p[j] = E::store(v[j]);
    }
}

// A block's scale byte from the bits of its largest magnitude (as integers magnitudes order like their values, infinities and
// NaN above every number).
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t mx_scale_byte(uint32_t largest)
{
    const int e = (int)(largest >> 23) - 2 + (STOCHASTIC && (largest & 0x7FFFFFu) > 0x400000u ? 1 : 0);
    return largest >= 0x7F800000u ? 255u : (uint32_t)max(e, 0);
}

// The magnitude code 0..7 of |v| <= 6 * 2^(byte - 127), rounded stochastically by the 16 bits r.  k is the magnitude in units of
// 2^-17 of the scale, so that a step of the grid is 2^16 units below 2, 2^17 below 4 and 2^18 above.
__device__ __forceinline__ uint32_t mx_draw(float v, int byte, uint32_t r)
{
    const uint32_t k = (uint32_t)__builtin_amdgcn_ldexpf(fabsf(v), 144 - byte);
    const uint32_t s = min(k >> 18, 2u);
    return (((k >> s) + r) >> 16) + 2 * s;
}

// 8 codes in a word, the first element's lowest.
template <bool STOCHASTIC>
__device__ __forceinline__ uint32_t mx_codes(const float (&v)[8], uint32_t byte, const uint32_t (&draws)[4])
{
    uint32_t w = 0;
    if constexpr (STOCHASTIC) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t r = j & 1 ? draws[j / 2] >> 16 : draws[j / 2] & 0xFFFFu;
            w |= (mx_draw(v[j], (int)byte, r) | (__float_as_uint(v[j]) >> 28 & 8u)) << (4 * j);
        }
    } else {
        const float scale = __uint_as_float(byte << 23);                // the instruction takes the exponent field alone
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
    }
    return byte == 255 ? 0u : w;
}

template <int CTRL>
__device__ __forceinline__ uint32_t dpp_move(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, CTRL, 0xf, 0xf, false);
}
// The largest of 4 neighbouring lanes (0-3, 4-7, ...), in each of them.
__device__ __forceinline__ uint32_t quad_max(uint32_t v)
{
    v = max(v, dpp_move<0xB1>(v));         // lanes 1 0 3 2
    return max(v, dpp_move<0x4E>(v));      // lanes 2 3 0 1
}
// The largest of the lanes 4 apart among 16 (0 4 8 12, ...), in each of them.
__device__ __forceinline__ uint32_t stride4_max(uint32_t v)
{
    v = max(v, dpp_move<0x128>(v));        // turned by 8 lanes
    return max(v, dpp_move<0x124>(v));     // by 4
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

}  // namespace tq
