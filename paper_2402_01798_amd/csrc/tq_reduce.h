// Sums and maxima over a wavefront or over the wavefronts that share a row.
#pragma once

#include "tq_mx_device.h"

namespace tq {

template <int CTRL>
__device__ __forceinline__ float dpp_move_float(float v) { return __uint_as_float(dpp_move<CTRL>(__float_as_uint(v))); }

// The sum of a wavefront's values, the same bits in every lane.
__device__ __forceinline__ float wave_total(float v)
{
    v += dpp_move_float<0xB1>(v);           // lanes 1 0 3 2
    v += dpp_move_float<0x4E>(v);           // lanes 2 3 0 1
    v += dpp_move_float<0x141>(v);          // mirrored within 8
    v += dpp_move_float<0x140>(v);          // within 16
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

__device__ __forceinline__ double wave_total(double v)
{
#pragma unroll
    for (int d = 32; d; d /= 2) v += __shfl_xor(v, d);
    return v;
}

__device__ __forceinline__ uint32_t wave_largest(uint32_t v) { return stride16_max(row16_max(v)); }

// Of N values over the WAVES wavefronts of a row, in a fixed order.  `part` [WAVES][N] is this row's and is used once between two
// barriers: successive calls take turns at two of them.
template <int WAVES, int N, typename Sum>
__device__ __forceinline__ void row_totals(Sum (&v)[N], Sum (*part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = wave_total(v[i]);
    if constexpr (WAVES > 1) {
        const uint32_t wave = (threadIdx.x >> 6) % WAVES;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) part[wave][i] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = part[0][i];
#pragma unroll
        for (int w = 1; w < WAVES; ++w)
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] += part[w][i];
    }
}

template <int WAVES, typename Sum>
__device__ __forceinline__ void row_total(Sum& x, Sum& y, Sum (*part)[2])
{
    Sum v[2] = {x, y};
    row_totals<WAVES>(v, part);
    x = v[0];
    y = v[1];
}

template <int WAVES>
__device__ __forceinline__ uint32_t row_largest(uint32_t x, uint32_t* part)
{
    x = wave_largest(x);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) part[(threadIdx.x >> 6) % WAVES] = x;
        __syncthreads();
        x = part[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x = max(x, part[w]);
    }
    return x;
}

}  // namespace tq
