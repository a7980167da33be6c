// Layer norm (tq_norm.h): forward and backward pass, the gradients of weight and bias.
#include <type_traits>

#include "tq_reduce.h"

namespace tq {
namespace {

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    const float* stats_in;
    void* out;                                 // y, or dx; dx may be NULL
    float* stats;
    float* partial;                            // [parts][2][cols]: sums of dy h and of dy
    float* rest;                               // [rows]: the mean of h from rounded statistics, for rows over 16384 columns
    float *dweight, *dbias;
    uint64_t ldx, lddy, ldo;
    uint32_t rows, cols, parts;
    float eps;
    int accumulate;
};

// How many of the 8 elements at 8 `oct` a row has.
__device__ __forceinline__ int left_of(uint32_t cols, uint32_t oct)
{
    const int64_t n = (int64_t)cols - (int64_t)oct * 8;
    return n >= 8 ? 8 : n > 0 ? (int)n : 0;
}

// A row's mean m, its rest c (m + c is nearer to the mean than m) and 1 / deviation, from passes over its elements:
// each(f) calls f(value) for all of this thread's.  Where a square or a sum leaves binary32's range, once more in units of 2^80.
// Sums are of type Sum: binary64 for rows that do not fit the registers, for a thread adds up cols / 1024 elements of those, whose roundings in binary32
// would be seen (2^26 equal elements of 33000 had h = 1.5).
struct RowStats {
    float unit;                                // x in units of 1 / unit
    float m, c, r;                             // of x * unit; (x * unit - m - c) * r = h
    float mean, rstd;                          // of x
};

template <int WAVES, typename Sum, typename Each>
__device__ __forceinline__ RowStats row_stats(uint32_t cols, float eps, Sum (*part)[WAVES][2], Each each)
{
    const Sum n = (Sum)cols;
    RowStats s;
    s.unit = 1.0f;
    Sum sum = 0, none = 0;
    each([&](float x) { sum += x; });
    row_total<WAVES>(sum, none, part[0]);
    s.m = (float)(sum / n);
    Sum d1 = 0, d2 = 0;
    auto deviation = [&](float d) {
        d1 += d;
        if constexpr (std::is_same_v<Sum, float>) d2 = fmaf(d, d, d2);
        else d2 = fma((double)d, (double)d, d2);
    };
    auto variance = [&]() {                    // around m + d1 / n
        const Sum c = d1 / n;
        s.c = (float)c;
        if constexpr (std::is_same_v<Sum, float>) return fmaf(-c, c, d2 / n);
        else return fma(-c, c, d2 / n);
    };
    each([&](float x) { deviation(x - s.m); });
    row_total<WAVES>(d1, d2, part[1]);
    const float var = fmaxf((float)variance(), 0.0f);
    s.r = 1.0f / sqrtf(var + eps);
    s.mean = s.m + s.c;
    s.rstd = s.r;
    if (!((float)d2 < __builtin_inff())) {     // the whole row's: all its threads take this turn
        s.unit = 0x1p-80f;
        sum = none = 0;
        each([&](float x) { sum += x * s.unit; });
        if constexpr (WAVES > 1) __syncthreads();                  // a wavefront with a row of its own goes on alone
        row_total<WAVES>(sum, none, part[0]);
        s.m = (float)(sum / n);
        d1 = d2 = 0;
        each([&](float x) { deviation(x * s.unit - s.m); });
        row_total<WAVES>(d1, d2, part[1]);
        const double v = (double)variance(), r = 1.0 / sqrt((v > 0.0 || v != v ? v : 0.0) * 0x1p160 + (double)eps);
        s.r = (float)(r * 0x1p80);
        s.mean = (s.m + s.c) * 0x1p80f;
        s.rstd = (float)r;
    }
    return s;
}

// A row by WAVES wavefronts that hold it in registers, 8 V elements each lane; short rows several to a workgroup.  Read once, written once:
// memory bounds it (16384 x 4096 bf16 57 to 62 us, 4.5 TB/s; 4096 x 32768 122), a launch where there are few rows (1 x 4096 3.2).
template <int DTYPE, int WTYPE, int WAVES, int V>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_forward_kernel(NormArgs a)
{
    using T = typename Element<DTYPE>::type;
    using W = typename Element<WTYPE>::type;
    constexpr uint32_t kThreads = WAVES * 64, kRows = WAVES == 1 ? 4 : 1;
    __shared__ float part[kRows][2][WAVES][2];
    const uint32_t sub = threadIdx.x / kThreads, tid = threadIdx.x % kThreads;
    const uint64_t row = (uint64_t)linear_block() * kRows + sub;
    static_assert(WAVES == 1 || kRows == 1, "barriers are for whole workgroups");
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    Eight<DTYPE> w[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t oct = tid + i * kThreads;
        const int n = left_of(a.cols, oct);
        if (n == 8) w[i].load(x + (uint64_t)oct * 8);
        else if (n) w[i].load(x + (uint64_t)oct * 8, n);
        else w[i].clear();
    }
    auto each = [&](auto f) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int n = left_of(a.cols, tid + i * kThreads);
            float v[8];
            w[i].unpack(v);
            if (n == 8) {
#pragma unroll
                for (int j = 0; j < 8; ++j) f(v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) f(v[j]);
            }
        }
    };
    const RowStats s = row_stats<WAVES>(a.cols, a.eps, part[sub], each);
    if (a.stats && tid == 0) {
        a.stats[2 * row] = s.mean;
        a.stats[2 * row + 1] = s.rstd;
    }
    T* y = static_cast<T*>(a.out) + row * a.ldo;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const uint32_t oct = tid + i * kThreads;
        const int n = left_of(a.cols, oct);
        if (n == 0) continue;
        float v[8], weight[8], bias[8];
        w[i].unpack(v);
        if (a.weight) load8<WTYPE>(static_cast<const W*>(a.weight) + (uint64_t)oct * 8, n, weight);
        if (a.bias) load8<WTYPE>(static_cast<const W*>(a.bias) + (uint64_t)oct * 8, n, bias);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float h = ((v[j] * s.unit - s.m) - s.c) * s.r;
            v[j] = a.weight ? h * weight[j] : h;
            if (a.bias) v[j] += bias[j];
        }
        store8<DTYPE>(y + (uint64_t)oct * 8, n, v);
    }
}

constexpr int kLongWaves = 16;

// Rows that do not fit the registers, by a workgroup each, read anew for every pass, from the caches if they are there: 1000 x 60000 bf16 73 us.
template <int DTYPE, int WTYPE>
__global__ __launch_bounds__(kLongWaves * 64) void norm_forward_long_kernel(NormArgs a)
{
    using T = typename Element<DTYPE>::type;
    using W = typename Element<WTYPE>::type;
    __shared__ double part[2][kLongWaves][2];
    const uint64_t row = linear_block();
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const uint32_t octs = (uint32_t)(((uint64_t)a.cols + 7) / 8);
    auto each = [&](auto f) {
        for (uint32_t oct = threadIdx.x; oct < octs; oct += kLongWaves * 64) {
            const int n = left_of(a.cols, oct);
            float v[8];
            load8<DTYPE>(x + (uint64_t)oct * 8, n, v);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (j < n) f(v[j]);
        }
    };
    const RowStats s = row_stats<kLongWaves>(a.cols, a.eps, part, each);
    if (a.stats && threadIdx.x == 0) {
        a.stats[2 * row] = s.mean;
        a.stats[2 * row + 1] = s.rstd;
    }
    T* y = static_cast<T*>(a.out) + row * a.ldo;
    for (uint32_t oct = threadIdx.x; oct < octs; oct += kLongWaves * 64) {
        const int n = left_of(a.cols, oct);
        float v[8], weight[8], bias[8];
        load8<DTYPE>(x + (uint64_t)oct * 8, n, v);
        if (a.weight) load8<WTYPE>(static_cast<const W*>(a.weight) + (uint64_t)oct * 8, n, weight);
        if (a.bias) load8<WTYPE>(static_cast<const W*>(a.bias) + (uint64_t)oct * 8, n, bias);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float h = ((v[j] * s.unit - s.m) - s.c) * s.r;
            v[j] = a.weight ? h * weight[j] : h;
            if (a.bias) v[j] += bias[j];
        }
        store8<DTYPE>(y + (uint64_t)oct * 8, n, v);
    }
}

// The backward pass has the mean as one binary32 number m, up to 2^-24 |m| from the row's: where that is no small part of the deviation, h by it
// is off in the whole row.  Its own mean d says how far, for that of h is 0: h - d takes m's place, and mean(g (h - d)) = mean(g h) - d mean(g), so
// that d is one sum more beside the two that dx takes.

// h of an element by m: the difference in quarters, which two numbers of the largest magnitude do not take out of range.
__device__ __forceinline__ float deviation(float x, float quarter_mean, float four_rstd)
{
    return fmaf(x, 0.25f, -quarter_mean) * four_rstd;
}

// Of 8 columns of which a row has n.  Behind its end h is 0: of the 0 that is held there it may be infinite, which no factor of 0 takes back.
__device__ __forceinline__ void deviations(const float (&x)[8], int n, float quarter_mean, float four_rstd, float (&h)[8])
{
#pragma unroll
    for (int j = 0; j < 8; ++j) h[j] = j < n ? deviation(x[j], quarter_mean, four_rstd) : 0.0f;
}

// dx of a row and the sums over rows: a workgroup's wavefronts hold WAVES to a row, 8 V columns to a lane, and take rows one after the
// other, the next row's elements on their way meanwhile; their sums over rows are joined at the end.  16384 x 4096 bf16 77 to 83 us, 5.0 TB/s:
// memory; without the next row's requests, with weights read for every row and twice the parts, 127.
template <int DTYPE, int WTYPE, int WAVES, int V>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * 64) void norm_backward_kernel(NormArgs a)
{
    using T = typename Element<DTYPE>::type;
    using W = typename Element<WTYPE>::type;
    constexpr uint32_t kThreads = WAVES * 64, kRows = WAVES == 1 ? 4 : 1;
    __shared__ float part[2][WAVES][3];
    __shared__ float sums[kRows > 1 ? kThreads * V * 8 : 1];
    static_assert(WAVES == 1 || kRows == 1, "barriers are for whole workgroups");
    const uint32_t sub = threadIdx.x / kThreads, tid = threadIdx.x % kThreads, block = linear_block();
    if (block >= a.parts) return;
    constexpr bool kAhead = WAVES < 16;                            // 16 wavefronts of a workgroup have no registers for that
    const float n_inv = 1.0f / (float)a.cols;
    const uint64_t first = (uint64_t)block * kRows + sub, step = (uint64_t)a.parts * kRows;
    float dw[V][8] = {}, db[V][8] = {}, weights[V][8];
    Eight<DTYPE> next_x[V], next_dy[V];
    float next_mean = 0.0f, next_r = 0.0f;
    auto fetch = [&](uint64_t row) {
        if (row >= a.rows) return;
        const T* x = static_cast<const T*>(a.x) + row * a.ldx;
        const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t oct = tid + i * kThreads;
            const int n = left_of(a.cols, oct);
            if (n == 8) {
                next_x[i].load(x + (uint64_t)oct * 8);
                next_dy[i].load(dy + (uint64_t)oct * 8);
            } else if (n) {                                        // behind the end: dy = 0, weight = 0 and h = 0, which add nothing
                next_x[i].load(x + (uint64_t)oct * 8, n);
                next_dy[i].load(dy + (uint64_t)oct * 8, n);
            } else {
                next_x[i].clear();
                next_dy[i].clear();
            }
        }
        next_mean = a.stats_in[2 * row];
        next_r = a.stats_in[2 * row + 1];
    };
    auto weights_of = [&](int i, float (&w)[8]) {
        const uint32_t oct = tid + i * kThreads;
        const int n = left_of(a.cols, oct);
        if (a.weight) load8<WTYPE>(static_cast<const W*>(a.weight) + (uint64_t)oct * 8, n, w);
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = j < n ? 1.0f : 0.0f;
        }
    };
    if constexpr (kAhead) {
        fetch(first);
#pragma unroll
        for (int i = 0; i < V; ++i) weights_of(i, weights[i]);
    }
    uint32_t turn = 0;
    for (uint64_t row = first; row < a.rows; row += step) {
        if constexpr (!kAhead) fetch(row);
        Eight<DTYPE> wx[V], wdy[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            wx[i] = next_x[i];
            wdy[i] = next_dy[i];
        }
        const float quarter = 0.25f * next_mean, r = next_r, four = 4.0f * r;
        if constexpr (kAhead) fetch(row + step);
        float sum[3] = {};                                         // of g, of g h and of h
#pragma unroll
        for (int i = 0; i < V; ++i) {
            float v[8], g[8], h[8];
            wx[i].unpack(v);
            wdy[i].unpack(g);
            deviations(v, left_of(a.cols, tid + i * kThreads), quarter, four, h);
            if constexpr (!kAhead) weights_of(i, weights[0]);
            const float(&weight)[8] = weights[kAhead ? i : 0];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float gw = g[j] * weight[j];
                sum[0] += gw;
                sum[1] = fmaf(gw, h[j], sum[1]);
                sum[2] += h[j];
            }
        }
        row_totals<WAVES>(sum, part[turn]);
        turn ^= 1;
        const float d = sum[2] * n_inv, s1 = sum[0] * n_inv, s2 = sum[1] * n_inv - d * s1;
        T* dx = static_cast<T*>(a.out) + row * a.ldo;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const uint32_t oct = tid + i * kThreads;
            const int n = left_of(a.cols, oct);
            if (!kAhead && n == 0) continue;                       // without this 16 wavefronts spill: 2048 x 16384 fp32 110 -> 137 us
            float v[8], g[8];
            wx[i].unpack(v);
            wdy[i].unpack(g);
            if constexpr (!kAhead) weights_of(i, weights[0]);
            const float(&weight)[8] = weights[kAhead ? i : 0];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = deviation(v[j], quarter, four) - d;
                dw[i][j] = fmaf(g[j], h, dw[i][j]);
                db[i][j] += g[j];
                v[j] = r * ((g[j] * weight[j] - s1) - h * s2);
            }
            if (a.out && n) store8<DTYPE>(dx + (uint64_t)oct * 8, n, v);
        }
    }
    if (!a.partial) return;
    float* to = a.partial + (uint64_t)block * 2 * a.cols;
    for (int which = 0; which < 2; ++which) {
        if constexpr (kRows > 1) {                                 // the workgroup's rows, in their order
            for (uint32_t k = 1; k < kRows; ++k) {
                __syncthreads();
                if (sub == k) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) sums[(i * 8 + j) * kThreads + tid] = which ? db[i][j] : dw[i][j];
                }
                __syncthreads();
                if (sub == 0) {
#pragma unroll
                    for (int i = 0; i < V; ++i)
#pragma unroll
                        for (int j = 0; j < 8; ++j) (which ? db[i][j] : dw[i][j]) += sums[(i * 8 + j) * kThreads + tid];
                }
            }
        }
        if (sub == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const uint32_t oct = tid + i * kThreads;
                const int n = left_of(a.cols, oct);
                if (n) store8<TQ_F32>(to + (uint64_t)which * a.cols + (uint64_t)oct * 8, n, which ? db[i] : dw[i]);
            }
        }
    }
}

// dx of a row whose sums over rows are left to norm_columns_kernel: held in registers (V > 0, 8 V elements a lane) or read twice.  4096 x 32768
// bf16 225 us (3.6 TB/s), 213 without the sum of h; two workgroups on a unit, whose registers then spill, 266.
template <int DTYPE, int WTYPE, int V>
__global__ __launch_bounds__(kLongWaves * 64) void norm_backward_long_kernel(NormArgs a)
{
    using T = typename Element<DTYPE>::type;
    using W = typename Element<WTYPE>::type;
    using Sum = std::conditional_t<V != 0, float, double>;         // as in row_stats
    constexpr uint32_t kThreads = kLongWaves * 64;
    __shared__ Sum part[kLongWaves][3];
    const uint64_t row = linear_block();
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const T* dy = static_cast<const T*>(a.dy) + row * a.lddy;
    T* dx = static_cast<T*>(a.out) + row * a.ldo;
    const float quarter = 0.25f * a.stats_in[2 * row], r = a.stats_in[2 * row + 1], four = 4.0f * r;
    const uint32_t octs = (uint32_t)(((uint64_t)a.cols + 7) / 8);
    Eight<DTYPE> wx[V ? V : 1], wdy[V ? V : 1];
    auto fetch = [&](int i, uint32_t oct) {
        const int n = left_of(a.cols, oct);
        if (n == 8) {
            wx[i].load(x + (uint64_t)oct * 8);
            wdy[i].load(dy + (uint64_t)oct * 8);
        } else {                                                   // behind the end dy = 0 and h = 0, which add nothing
            wx[i].load(x + (uint64_t)oct * 8, n);
            wdy[i].load(dy + (uint64_t)oct * 8, n);
        }
    };
    auto values = [&](int i, uint32_t oct, float (&h)[8], float (&g)[8]) {
        const int n = left_of(a.cols, oct);
        float v[8], weight[8];
        wx[i].unpack(v);
        wdy[i].unpack(g);
        deviations(v, n, quarter, four, h);
        if (a.weight) load8<WTYPE>(static_cast<const W*>(a.weight) + (uint64_t)oct * 8, n, weight);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (a.weight) g[j] *= weight[j];
    };
    Sum sum[3] = {};                                               // of g, of g h and of h
    float s1 = 0.0f, s2 = 0.0f, d = 0.0f, h[8], g[8];
    auto add = [&](int i, uint32_t oct) {
        values(i, oct, h, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            sum[0] += g[j];
            if constexpr (V != 0) sum[1] = fmaf(g[j], h[j], sum[1]);
            else sum[1] = fma((double)g[j], (double)h[j], sum[1]);
            sum[2] += h[j];
        }
    };
    auto put = [&](int i, uint32_t oct) {
        values(i, oct, h, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) h[j] = r * ((g[j] - s1) - (h[j] - d) * s2);
        store8<DTYPE>(dx + (uint64_t)oct * 8, left_of(a.cols, oct), h);
    };
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (threadIdx.x + i * kThreads < octs) fetch(i, threadIdx.x + i * kThreads);
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (threadIdx.x + i * kThreads < octs) add(i, threadIdx.x + i * kThreads);
    } else {
        for (uint32_t oct = threadIdx.x; oct < octs; oct += kThreads) {
            fetch(0, oct);
            add(0, oct);
        }
    }
    row_totals<kLongWaves>(sum, part);
    d = (float)(sum[2] / (Sum)a.cols);
    s1 = (float)(sum[0] / (Sum)a.cols);
    s2 = (float)(sum[1] / (Sum)a.cols) - d * s1;
    if (a.rest && threadIdx.x == 0) a.rest[row] = d;
    if constexpr (V > 0) {
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (threadIdx.x + i * kThreads < octs) put(i, threadIdx.x + i * kThreads);
    } else {
        for (uint32_t oct = threadIdx.x; oct < octs; oct += kThreads) {
            fetch(0, oct);
            put(0, oct);
        }
    }
}

// The mean of such a row's h alone, summed as above, bit for bit: where dx is not wanted, or takes the place of what norm_columns_kernel reads.
template <int DTYPE, typename Sum>
__global__ __launch_bounds__(kLongWaves * 64) void norm_rest_kernel(NormArgs a)
{
    using T = typename Element<DTYPE>::type;
    __shared__ Sum part[kLongWaves][1];
    const uint64_t row = linear_block();
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.ldx;
    const float quarter = 0.25f * a.stats_in[2 * row], four = 4.0f * a.stats_in[2 * row + 1];
    const uint32_t octs = (uint32_t)(((uint64_t)a.cols + 7) / 8);
    Sum sum[1] = {};
    for (uint32_t oct = threadIdx.x; oct < octs; oct += kLongWaves * 64) {
        const int n = left_of(a.cols, oct);
        float v[8], h[8];
        load8<DTYPE>(x + (uint64_t)oct * 8, n, v);
        deviations(v, n, quarter, four, h);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[0] += h[j];
    }
    row_totals<kLongWaves>(sum, part);
    if (threadIdx.x == 0) a.rest[row] = (float)(sum[0] / (Sum)a.cols);
}

// Sums over the rows of such a matrix: a thread takes 8 columns of every parts-th row.  4096 x 32768 bf16 112 us, 4.8 TB/s.
template <int DTYPE>
__global__ __launch_bounds__(256) void norm_columns_kernel(NormArgs a, uint32_t across)
{
    using T = typename Element<DTYPE>::type;
    const uint32_t block = linear_block(), by = block / across, oct = (block - by * across) * 256 + threadIdx.x;
    if (by >= a.parts) return;
    const int n = left_of(a.cols, oct);
    if (n == 0) return;
    float dw[8] = {}, db[8] = {};
    for (uint64_t row = by; row < a.rows; row += a.parts) {
        float v[8], g[8];
        load8<DTYPE>(static_cast<const T*>(a.x) + row * a.ldx + (uint64_t)oct * 8, n, v);
        load8<DTYPE>(static_cast<const T*>(a.dy) + row * a.lddy + (uint64_t)oct * 8, n, g);
        const float quarter = 0.25f * a.stats_in[2 * row], four = 4.0f * a.stats_in[2 * row + 1], d = a.rest[row];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            dw[j] = fmaf(g[j], deviation(v[j], quarter, four) - d, dw[j]);
            db[j] += g[j];
        }
    }
    float* to = a.partial + (uint64_t)by * 2 * a.cols + (uint64_t)oct * 8;
    store8<TQ_F32>(to, n, dw);
    store8<TQ_F32>(to + a.cols, n, db);
}

// The parts' sums, joined in a fixed order: 32 columns of dweight and dbias by 32 threads each.  512 parts of 4096 columns 5 us.
__global__ __launch_bounds__(1024) void norm_join_kernel(NormArgs a)
{
    __shared__ float sums[32][33];
    const uint32_t lane = threadIdx.x & 31, strip = threadIdx.x >> 5;
    const uint64_t at = (uint64_t)linear_block() * 32 + lane, all = 2 * (uint64_t)a.cols;
    if ((uint64_t)linear_block() * 32 >= all) return;
    float v = 0.0f;
    if (at < all) {
#pragma unroll 8
        for (uint32_t p = strip; p < a.parts; p += 32) v += a.partial[p * all + at];
    }
    sums[strip][lane] = v;
    __syncthreads();
    if (strip || at >= all) return;
    for (int s = 1; s < 32; ++s) v += sums[s][lane];
    float* to = at < a.cols ? a.dweight : a.dbias;
    if (!to) return;
    to += at < a.cols ? at : at - a.cols;
    *to = a.accumulate ? *to + v : v;
}

// The wavefronts of a row and the elements of a lane in eighths, for rows of up to 512 WAVES V elements.  From 513 to 1024 columns forward and
// backward pass take, by one / two / four wavefronts a row, us:
//   300 x 1024 bf16      16.1   10.8   11.0        16384 x 1024 bf16   46.5   51.3   61.0
//   1000 x 600 fp32      20.3   14.1   14.6        65536 x 700 bf16     167    280    334
//   4099 x 1001 fp32     37.1   30.7   31.6        16384 x 1024 fp32   84.2   60.2   65.5
//   4096 x 1024 bf16     24.7   21.7   25.1        65536 x 1024 fp32    293    246    257
// Few rows want many wavefronts; many rows no barriers, if a wavefront has a row's two times 2 KiB on their way and the next row's.
bool wave_a_row(uint64_t rows, uint64_t cols, int dtype) { return cols <= 512 || (cols <= 1024 && dtype != TQ_F32 && rows >= 8192); }

template <typename F>
hipError_t by_shape(uint32_t rows, uint32_t cols, int dtype, F f)
{
    auto as = [&](auto w, auto v) { return f(w, v); };
#define TQ_NORM_SHAPE(WAVES, V) return as(std::integral_constant<int, WAVES>{}, std::integral_constant<int, V>{})
    if (cols <= 512) TQ_NORM_SHAPE(1, 1);
    if (wave_a_row(rows, cols, dtype)) TQ_NORM_SHAPE(1, 2);
    if (cols <= 1024) TQ_NORM_SHAPE(2, 1);
    if (cols <= 2048) TQ_NORM_SHAPE(4, 1);
    if (cols <= 4096) TQ_NORM_SHAPE(4, 2);
    if (cols <= 8192) TQ_NORM_SHAPE(8, 2);
    if (cols <= 16384) TQ_NORM_SHAPE(16, 2);
    TQ_NORM_SHAPE(16, 4);
#undef TQ_NORM_SHAPE
}

// Columns of rows that stay in registers: forward and for dx alone; with sums over rows.
constexpr uint32_t kMostForward = 32768, kMostInRegisters = 16384;

template <typename F>
hipError_t by_type(int dtype, F f)
{
    if (dtype == TQ_F32) return f(std::integral_constant<int, TQ_F32>{});
    return dtype == TQ_BF16 ? f(std::integral_constant<int, TQ_BF16>{}) : f(std::integral_constant<int, TQ_F16>{});
}

// Workgroups that share the rows of a backward pass, and with it the partial sums: each of them writes sums of its columns, which the last
// kernel reads, so not more than it takes to keep memory busy.  16384 x 4096 bf16, us of the backward pass: 512 of them 83, 768 86, 1024
// (without the next row's requests) 138.
uint32_t parts_of(uint64_t rows, uint64_t cols, int dtype)
{
    if (cols > kMostInRegisters) return (uint32_t)(rows < 64 ? rows : 64);
    const bool alone = wave_a_row(rows, cols, dtype);              // four rows in a workgroup then
    const uint64_t most = alone ? (rows < 8192 ? 256 : 512) : cols <= 2048 ? 768 : cols <= 8192 ? 512 : 256;
    const uint64_t wanted = alone ? (rows + 3) / 4 : rows;
    return (uint32_t)(wanted < most ? wanted : most);
}

}  // namespace
}  // namespace tq

hipError_t tq_launch_layernorm_forward(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* weight,
                                       const void* bias, int wtype, float eps, void* y, uint64_t ldy, float* stats, hipStream_t st)
{
    using namespace tq;
    NormArgs a = {};
    a.x = x;
    a.ldx = ldx;
    a.weight = weight;
    a.bias = bias;
    a.out = y;
    a.ldo = ldy;
    a.stats = stats;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.eps = eps;
    return by_type(dtype, [&](auto D) {
        return by_type(wtype, [&](auto W) -> hipError_t {
            constexpr int kD = decltype(D)::value, kW = decltype(W)::value;
            dim3 grid;
            if (cols > kMostForward) {
                if (!fold_grid(rows, kLongWaves * 64, 1, grid)) return hipErrorInvalidValue;
                norm_forward_long_kernel<kD, kW><<<grid, kLongWaves * 64, 0, st>>>(a);
                return hipGetLastError();
            }
            return by_shape(a.rows, a.cols, dtype, [&](auto N, auto V) -> hipError_t {
                constexpr int kN = decltype(N)::value, kThreads = kN == 1 ? 256 : kN * 64;
                const uint32_t each = kThreads / (kN * 64);
                if (!fold_grid((rows + each - 1) / each, kThreads, 1, grid)) return hipErrorInvalidValue;
                norm_forward_kernel<kD, kW, kN, decltype(V)::value><<<grid, kThreads, 0, st>>>(a);
                return hipGetLastError();
            });
        });
    });
}

uint64_t tq_layernorm_workspace_bytes_impl(uint64_t rows, uint64_t cols)
{
    const uint64_t a = tq::parts_of(rows, cols, TQ_F32), b = tq::parts_of(rows, cols, TQ_BF16);
    return (a > b ? a : b) * 2 * cols * sizeof(float) + (cols > tq::kMostInRegisters ? rows * sizeof(float) : 0);
}

hipError_t tq_launch_layernorm_backward(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ldx, const void* dy, uint64_t lddy,
                                        const void* weight, int wtype, const float* stats, void* dx, uint64_t lddx, float* dweight,
                                        float* dbias, int accumulate, void* workspace, hipStream_t st)
{
    using namespace tq;
    NormArgs a = {};
    a.x = x;
    a.ldx = ldx;
    a.dy = dy;
    a.lddy = lddy;
    a.weight = weight;
    a.stats_in = stats;
    a.out = dx;
    a.ldo = lddx;
    a.dweight = dweight;
    a.dbias = dbias;
    a.accumulate = accumulate;
    a.partial = dweight || dbias ? static_cast<float*>(workspace) : nullptr;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.parts = parts_of(rows, cols, dtype);
    dim3 grid;
    const hipError_t e = by_type(dtype, [&](auto D) {
        return by_type(wtype, [&](auto W) -> hipError_t {
            constexpr int kD = decltype(D)::value, kW = decltype(W)::value;
            if (cols > kMostInRegisters) {
                dim3 by_row;
                if (!fold_grid(rows, kLongWaves * 64, 1, by_row)) return hipErrorInvalidValue;
                auto put_dx = [&]() -> hipError_t {
                    if (cols <= kMostForward) norm_backward_long_kernel<kD, kW, 4><<<by_row, kLongWaves * 64, 0, st>>>(a);
                    else norm_backward_long_kernel<kD, kW, 0><<<by_row, kLongWaves * 64, 0, st>>>(a);
                    return hipGetLastError();
                };
                if (!a.partial) return put_dx();
                a.rest = a.partial + (uint64_t)a.parts * 2 * cols;
                const bool apart = a.out && a.out != x && a.out != dy;     // dx leaves what the columns' sums read: it may come first
                hipError_t e;
                if (apart) {
                    e = put_dx();
                } else {
                    if (cols <= kMostForward) norm_rest_kernel<kD, float><<<by_row, kLongWaves * 64, 0, st>>>(a);
                    else norm_rest_kernel<kD, double><<<by_row, kLongWaves * 64, 0, st>>>(a);
                    e = hipGetLastError();
                }
                if (e != hipSuccess) return e;
                const uint32_t across = (uint32_t)(((cols + 7) / 8 + 255) / 256);
                if (!fold_grid((uint64_t)across * a.parts, 256, 1, grid)) return hipErrorInvalidValue;
                norm_columns_kernel<kD><<<grid, 256, 0, st>>>(a, across);
                e = hipGetLastError();
                return e != hipSuccess || apart || !a.out ? e : put_dx();
            }
            return by_shape(a.rows, a.cols, dtype, [&](auto N, auto V) -> hipError_t {
                constexpr int kN = decltype(N)::value, kV = decltype(V)::value, kThreads = kN == 1 ? 256 : kN * 64;
                if constexpr (kN * kV * 512 > (int)kMostInRegisters) {
                    return hipErrorInvalidValue;                   // taken above
                } else {
                    if (!fold_grid(a.parts, kThreads, 1, grid)) return hipErrorInvalidValue;
                    norm_backward_kernel<kD, kW, kN, kV><<<grid, kThreads, 0, st>>>(a);
                    return hipGetLastError();
                }
            });
        });
    });
    if (e != hipSuccess || !a.partial) return e;
    if (!fold_grid((2 * cols + 31) / 32, 1024, 1, grid)) return hipErrorInvalidValue;
    norm_join_kernel<<<grid, 1024, 0, st>>>(a);
    return hipGetLastError();
}
