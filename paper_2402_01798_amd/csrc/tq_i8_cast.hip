// Matrices to 8-bit integers with a scale for each row and back (tq_i8.h).
#include <type_traits>

#include "tq_i8_device.h"

namespace tq {
namespace {

struct I8CastArgs {
    const void* x;
    int8_t* codes;
    float* scales;
    uint64_t ld;
    uint32_t rows, cols, octs;                 // octs: eights of a row of codes, padding included
};

// A row by WAVES wavefronts; V > 0: it stays in their registers, 8 V elements a lane, else it is read twice.  Short rows four to a workgroup.
// Memory: 2056 x 4097 fp32 10 us, 4.2 TB/s; 4104 columns, whose rows begin at multiples of 32 bytes, 0.5 us less, 4096, two eights a lane in place of
// three, 1.7 less.
template <int DTYPE, int WAVES, int V>
__global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void i8_cast_kernel(I8CastArgs a)
{
    using T = typename Element<DTYPE>::type;
    constexpr uint32_t kThreads = WAVES * 64, kRows = WAVES < 4 ? 4 / WAVES : 1;
    static_assert(WAVES == 1 || kRows == 1, "barriers are for whole workgroups");
    __shared__ uint32_t part[WAVES];
    const uint32_t tid = threadIdx.x % kThreads;
    const uint64_t row = (uint64_t)linear_block() * kRows + threadIdx.x / kThreads;
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    auto left = [&](uint32_t oct) {
        const int64_t n = (int64_t)a.cols - (int64_t)oct * 8;
        return n >= 8 ? 8 : n > 0 ? (int)n : 0;
    };
    Eight<DTYPE> w[V ? V : 1];
    auto fetch = [&](Eight<DTYPE>& e, uint32_t oct) {
        const int n = left(oct);
        if (n == 8) e.load(x + (uint64_t)oct * 8);
        else if (n) e.load(x + (uint64_t)oct * 8, n);
        else e.clear();
    };
    uint32_t largest = 0;
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) fetch(w[i], tid + i * kThreads);
#pragma unroll
        for (int i = 0; i < V; ++i) largest = max(largest, w[i].largest());
    } else {
        for (uint32_t oct = tid; oct < a.octs; oct += kThreads) {
            fetch(w[0], oct);
            largest = max(largest, w[0].largest());
        }
    }
    const I8Row s(row_largest<WAVES>(largest, part));
    if (tid == 0) a.scales[row] = s.scale;
    int8_t* codes = a.codes + row * ((uint64_t)a.octs * 8);
    auto put = [&](Eight<DTYPE>& e, uint32_t oct) {
        if (oct >= a.octs) return;
        float v[8];
        e.unpack(v);
        *reinterpret_cast<u32x2*>(codes + (uint64_t)oct * 8) = s.codes(v);
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i) put(w[i], tid + i * kThreads);
    } else {
        for (uint32_t oct = tid; oct < a.octs; oct += kThreads) {
            fetch(w[0], oct);
            put(w[0], oct);
        }
    }
}

// 2056 x 4097 to fp32 12 us, 3.4 TB/s, and no less to rows at multiples of 32 bytes.
struct I8ValuesArgs {
    const int8_t* codes;
    const float* scales;
    void* out;
    uint64_t ldo;
    uint32_t rows, cols, octs, used;           // eights of a row of codes, and those with elements
};

template <int DTYPE>
__global__ __launch_bounds__(256) void i8_values_kernel(I8ValuesArgs a)
{
    using T = typename Element<DTYPE>::type;
    const uint64_t at = (uint64_t)linear_block() * 256 + threadIdx.x;          // rows follow each other: no workgroup is left with a row's few last
    const uint64_t row = at >> 32 ? at / a.used : (uint32_t)at / a.used;
    if (row >= a.rows) return;
    const uint32_t oct = (uint32_t)(at - row * a.used);
    const float scale = a.scales[row];
    const u32x2 w = *reinterpret_cast<const u32x2*>(a.codes + (row * a.octs + oct) * 8);
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = (float)(int8_t)(w[j / 4] >> (j % 4 * 8)) * scale;
    store8<DTYPE>(static_cast<T*>(a.out) + row * a.ldo + (uint64_t)oct * 8, (int)min((int64_t)a.cols - (int64_t)oct * 8, (int64_t)8), v);
}

template <int DTYPE, int WAVES, int V>
hipError_t launch_cast(const I8CastArgs& a, hipStream_t st)
{
    constexpr uint32_t kBlock = WAVES < 4 ? 256 : WAVES * 64, kRows = WAVES < 4 ? 4 / WAVES : 1;
    dim3 grid;
    if (!fold_grid(((uint64_t)a.rows + kRows - 1) / kRows, kBlock, 1, grid)) return hipErrorInvalidValue;
    i8_cast_kernel<DTYPE, WAVES, V><<<grid, kBlock, 0, st>>>(a);
    return hipGetLastError();
}

template <int DTYPE>
hipError_t launch_cast(const I8CastArgs& a, hipStream_t st)
{
    if (a.octs <= 64) return launch_cast<DTYPE, 1, 1>(a, st);
    if (a.octs <= 256) return launch_cast<DTYPE, 4, 1>(a, st);
    if (a.octs <= 512) return launch_cast<DTYPE, 4, 2>(a, st);
    if (a.octs <= 768) return launch_cast<DTYPE, 4, 3>(a, st);
    if (a.octs <= 1024) return launch_cast<DTYPE, 4, 4>(a, st);
    if (a.octs <= 4096) return launch_cast<DTYPE, 16, 4>(a, st);
    return launch_cast<DTYPE, 16, 0>(a, st);
}

}  // namespace
}  // namespace tq

hipError_t tq_launch_i8_quantize(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, void* codes, float* scales,
                                 hipStream_t st)
{
    using namespace tq;
    const I8CastArgs a = {x, static_cast<int8_t*>(codes), scales, ld, (uint32_t)rows, (uint32_t)cols, (uint32_t)((cols + 127) / 128 * 16)};
    if (dtype == TQ_F32) return launch_cast<TQ_F32>(a, st);
    return dtype == TQ_BF16 ? launch_cast<TQ_BF16>(a, st) : launch_cast<TQ_F16>(a, st);
}

hipError_t tq_launch_i8_dequantize(const void* codes, const float* scales, uint64_t rows, uint64_t cols, void* out, int dtype,
                                   uint64_t ldo, hipStream_t st)
{
    using namespace tq;
    const I8ValuesArgs a = {static_cast<const int8_t*>(codes), scales, out, ldo, (uint32_t)rows, (uint32_t)cols,
                            (uint32_t)((cols + 127) / 128 * 16), (uint32_t)((cols + 7) / 8)};
    dim3 grid;
    if (!fold_grid((rows * a.used + 255) / 256, 256, 1, grid)) return hipErrorInvalidValue;
    if (dtype == TQ_F32) i8_values_kernel<TQ_F32><<<grid, 256, 0, st>>>(a);
    else if (dtype == TQ_BF16) i8_values_kernel<TQ_BF16><<<grid, 256, 0, st>>>(a);
    else i8_values_kernel<TQ_F16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
