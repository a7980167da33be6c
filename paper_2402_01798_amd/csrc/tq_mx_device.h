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
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
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
    if constexpr (DTYPE == TQ_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
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

// 8 consecutive elements, `n` of them there (the rest 0).  Whole ones are fetched 16 bytes at a time from any address: the memory
// unit takes addresses that are no multiple of 16 (rows of an odd length) at little more than the cost of aligned ones.
template <int DTYPE>
__device__ __forceinline__ void load8(const typename Element<DTYPE>::type* p, int n, float (&v)[8])
{
    using E = Element<DTYPE>;
    if (n >= 8) {
        if constexpr (DTYPE == TQ_F32) {
            __builtin_memcpy(v, p, 32);
        } else {
            u32x4 w;
            __builtin_memcpy(&w, p, 16);
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack2<DTYPE>(w[j], v[2 * j], v[2 * j + 1]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = j < n ? E::load(p[j]) : 0.0f;
    }
}

// The same, left as they are in memory.  `unpack` makes fp32 values of them, and new ones each time: kept from one use to the
// next they would take twice the registers.
template <int DTYPE>
struct Eight {
    u32x4 w[DTYPE == TQ_F32 ? 2 : 1];

    __device__ __forceinline__ void load(const typename Element<DTYPE>::type* p) { __builtin_memcpy(w, p, sizeof(w)); }
    __device__ __forceinline__ void load(const typename Element<DTYPE>::type* p, int n)      // n < 8 of them
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const typename Element<DTYPE>::type v = j < n ? p[j] : 0;
            if constexpr (DTYPE == TQ_F32) w[j / 4][j % 4] = __float_as_uint(v);
            else w[0][j / 2] = j & 1 ? w[0][j / 2] | (uint32_t)v << 16 : (uint32_t)v;
        }
    }
    __device__ __forceinline__ void clear()
    {
        w[0] = u32x4{0, 0, 0, 0};
        if constexpr (DTYPE == TQ_F32) w[1] = w[0];
    }
    // Largest magnitudes, of 16-bit types two at a time: as integers they order like their values.  `most` is one of the columns' words.
    static constexpr int kWords = DTYPE == TQ_F32 ? 8 : 4;
    __device__ __forceinline__ void largest_of_columns(uint32_t (&most)[kWords]) const
    {
#pragma unroll
        for (int j = 0; j < kWords; ++j) most[j] = larger(most[j], word(j));
    }
    __device__ __forceinline__ uint32_t largest() const                 // of the eight, as fp32 bits
    {
        uint32_t m = word(0);
#pragma unroll
        for (int j = 1; j < kWords; ++j) m = larger(m, word(j));
        return DTYPE == TQ_F32 ? m : max(bits(m, 0), bits(m, 1));
    }
    static __device__ __forceinline__ uint32_t bits(uint32_t m, int half)      // one half of a word of magnitudes as fp32 bits
    {
        if constexpr (DTYPE == TQ_F32) return m;
        else return __float_as_uint(Element<DTYPE>::load((uint16_t)(half ? m >> 16 : m)));
    }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b)
    {
        if constexpr (DTYPE == TQ_F32) return max(a, b);
        else return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
    }
    __device__ __forceinline__ uint32_t word(int j) const
    {
        return DTYPE == TQ_F32 ? w[j / 4][j % 4] & 0x7FFFFFFFu : w[0][j % 4] & 0x7FFF7FFFu;
    }
    __device__ __forceinline__ void unpack(float (&v)[8])
    {
        asm volatile("" : "+v"(w[0]));
        if constexpr (DTYPE == TQ_F32) {
            asm volatile("" : "+v"(w[1]));
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = __uint_as_float(w[j / 4][j % 4]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) unpack2<DTYPE>(w[0][j], v[2 * j], v[2 * j + 1]);
        }
    }
};

template <int DTYPE>
__device__ __forceinline__ void store8(typename Element<DTYPE>::type* p, int n, const float (&v)[8])
{
    using E = Element<DTYPE>;
    if (n >= 8) {
        if constexpr (DTYPE == TQ_F32) {
            __builtin_memcpy(p, v, 32);
        } else {
            u32x4 w;
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pack2<DTYPE>(v[2 * j], v[2 * j + 1]);
            __builtin_memcpy(p, &w, 16);
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

// Stochastic rounding.  A magnitude t (in units of the scale, at most 6) times 2^-126 has, as an fp32 number, the grid's own
// structure: below 1 it is subnormal and a step of 0.5 is 2^22 units in the last place, above it has one bit of the mantissa above
// those 22.  So its bits, 16 random bits added where the fraction begins, are the code << 22 and what is dropped.  The product
// has to be cut off, not rounded, where it is subnormal: round_toward_zero.  4 instructions an element and form and one for an
// element's draw, 11 as comparisons and shifts of a fixed-point number.
__device__ __forceinline__ uint32_t round_toward_zero()
{
    // bits 0 and 1 of the wavefront's mode: fp32 arithmetic.  Gives 0: what is loaded from an address that it is added to comes after.
    uint32_t zero = 0;
    asm volatile("s_setreg_imm32_b32 hwreg(HW_REG_MODE, 0, 2), 3" : "+s"(zero));
    return zero;
}
// The element's 16 bits of a word of draws, as high as mx_push wants them.
__device__ __forceinline__ uint32_t mx_draw(uint32_t word, bool high) { return high ? (word >> 16) << 12 : (word & 0xFFFFu) << 12; }
// The word's codes, one to the left, and this element's.
__device__ __forceinline__ uint32_t mx_push(uint32_t w, float v, uint32_t byte, uint32_t draw)
{
    const uint32_t bits = __float_as_uint(__builtin_amdgcn_ldexpf(fabsf(v), 1 - (int)byte));
    const uint32_t x = (bits << 6) + draw;                              // the magnitude's code in bits 28..30
    uint32_t code;                                                      // and v's sign above it, in one instruction
    asm("v_bfi_b32 %0, %1, %2, %3" : "=v"(code) : "s"(0x7FFFFFFFu), "v"(x), "v"(v));
    return __builtin_amdgcn_alignbit(w, code, 28);
}

// 8 codes in a word, the first element's lowest.
__device__ __forceinline__ uint32_t mx_nearest(const float (&v)[8], uint32_t byte)
{
    const float scale = __uint_as_float(byte << 23);                    // the instruction takes the exponent field alone
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
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

// The largest of 16 neighbouring lanes, in each of them.
__device__ __forceinline__ uint32_t row16_max(uint32_t v)
{
    v = quad_max(v);
    v = max(v, dpp_move<0x141>(v));        // mirrored within 8
    return max(v, dpp_move<0x140>(v));     // within 16
}
// The largest of the lanes 16 apart (l, l + 16, l + 32, l + 48), in each of them.
__device__ __forceinline__ uint32_t stride16_max(uint32_t v)
{
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(a[0], a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return max(b[0], b[1]);
}

__device__ __forceinline__ uint32_t magnitude_bits(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

}  // namespace tq
