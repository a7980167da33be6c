// Distillation from a teacher's top logits (tq_distill.h): loss and gradient.
#include "tq_mx_device.h"
#include "tq_distill.h"

namespace tq {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct DistillArgs {
    const void* z;
    const void* ids;
    const float* t;
    const float* grad;
    const float* stats_in;
    float *loss, *stats;
    void* dz;
    uint64_t ldz, lddz;
    uint32_t rows, vocab, top;
    int wide_ids;
    float tau, inv_tau;
};

__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
// Over the workgroup, in a fixed order; `part` holds one value per wavefront.  Begins and ends with a barrier.
template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float* part)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) s += part[w];
    return s;
}
template <int WAVES>
__device__ __forceinline__ float group_max(float v, float* part)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = part[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s = fmaxf(s, part[w]);
    return s;
}

// Running maximum (of z) and sum of exp((z - max) / tau).
struct Softmax {
    float m = -INFINITY, s = 0.0f;
    // -inf - -inf has no value: while nothing but -inf was seen, the sum of nothing is 0
    static __device__ __forceinline__ float scale(float from, float to, float c) { return from == -INFINITY ? 0.0f : exp2f((from - to) * c); }
    __device__ __forceinline__ void take(const float (&v)[8], float c)
    {
        float top = v[0];
#pragma unroll
        for (int j = 1; j < 8; ++j) top = fmaxf(top, v[j]);
        if (top > m) {
            s *= scale(m, top, c);
            m = top;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) s += v[j] == -INFINITY ? 0.0f : exp2f((v[j] - m) * c);
    }
    __device__ __forceinline__ void join(float m2, float s2, float c)
    {
        const float to = fmaxf(m, m2);
        s = s * scale(m, to, c) + s2 * scale(m2, to, c);
        m = to;
    }
};

enum { kForward = 0, kBackward = 1, kBoth = 2 };

// One workgroup a row, 8 elements a thread at a time.
template <int DTYPE, int MODE, int THREADS>
__global__ __launch_bounds__(THREADS) void distill_kernel(DistillArgs a)
{
    using E = Element<DTYPE>;
    using T = typename E::type;
    constexpr int WAVES = THREADS / 64;
    __shared__ float part[WAVES], part_s[WAVES];
    __shared__ int id[TQ_DISTILL_MAX_TOP];
    __shared__ float prob[TQ_DISTILL_MAX_TOP];
    const uint32_t row = linear_block(), tid = threadIdx.x;
    if (row >= a.rows) return;
    const T* z = static_cast<const T*>(a.z) + (uint64_t)row * a.ldz;
    T* dz = MODE == kForward ? nullptr : static_cast<T*>(a.dz) + (uint64_t)row * a.lddz;
    const float grad = MODE == kForward ? 0.0f : a.grad[row];
    const float c = a.inv_tau * kLog2e;

    // the teacher
    float peak = -INFINITY;
    bool bad = false;
    for (uint32_t i = tid; i < a.top; i += THREADS) {
        const uint64_t at = (uint64_t)row * a.top + i;
        const int64_t w = a.wide_ids ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int32_t*>(a.ids)[at];
        const float t = a.t[at];
        const bool there = w >= 0 && w < (int64_t)a.vocab && t != -INFINITY;
        id[i] = there ? (int)w : -1;
        prob[i] = t;
        if (there) {
            peak = fmaxf(peak, t);
            bad |= !(t < INFINITY);
        }
    }
    peak = group_max<WAVES>(peak, part);
    float sum = 0.0f;
    for (uint32_t i = tid; i < a.top; i += THREADS) sum += id[i] < 0 ? 0.0f : exp2f((prob[i] - peak) * c);
    sum = group_sum<WAVES>(bad ? NAN : sum, part);
    const bool empty = sum == 0.0f;
    const float log_sum = empty ? 0.0f : logf(sum);

    // the student
    float top = 0.0f, log_total = 0.0f;                          // the row's largest logit, ln sum exp((z - top) / tau)
    if (MODE == kBackward) {
        top = a.stats_in[2 * (uint64_t)row];
        log_total = a.stats_in[2 * (uint64_t)row + 1];
    } else {
        Softmax q;
        for (uint64_t i = (uint64_t)tid * 8; i < a.vocab; i += THREADS * 8) {
            float v[8];
            const int n = (int)min((uint64_t)a.vocab - i, (uint64_t)8);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < n ? E::load(z[i + j]) : -INFINITY;
            q.take(v, c);
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) q.join(__shfl_xor(q.m, d), __shfl_xor(q.s, d), c);
        __syncthreads();
        if ((tid & 63) == 0) {
            part[tid >> 6] = q.m;
            part_s[tid >> 6] = q.s;
        }
        __syncthreads();
        Softmax all;
        for (int w = 0; w < WAVES; ++w) all.join(part[w], part_s[w], c);
        top = all.m;
        log_total = logf(all.s);
    }
    // where nothing is left of the row every z is -inf and q is 0: any finite numbers do
    const bool none = log_total == -INFINITY;
    const float low = none ? 0.0f : top, log_low = none ? 0.0f : log_total;

    // loss, and the elements that the teacher names; an id's first entry takes the probabilities of all its entries
    float loss = 0.0f;
    float named[TQ_DISTILL_MAX_TOP / THREADS ? TQ_DISTILL_MAX_TOP / THREADS : 1];
    int k = 0;
#pragma unroll
    for (uint32_t i0 = 0; i0 < TQ_DISTILL_MAX_TOP; i0 += THREADS, ++k) {
        const uint32_t i = i0 + tid;
        named[k] = 0.0f;
        if (i < a.top && id[i] >= 0 && !empty) {
            const float x = (prob[i] - peak) * a.inv_tau - log_sum, p = expf(x), zi = E::load(z[id[i]]);
            if (!(p <= 0.0f)) loss += p * (x - ((zi - low) * a.inv_tau - log_low));
            named[k] = zi;
        }
    }
    if (MODE != kBackward) {
        loss = group_sum<WAVES>(loss, part);
        if (tid == 0) {
            a.loss[row] = empty ? 0.0f : loss * a.tau * a.tau;
            if (MODE == kForward) {
                a.stats[2 * (uint64_t)row] = top;
                a.stats[2 * (uint64_t)row + 1] = log_total;
            }
        }
    }
    if (MODE == kForward) return;

    const bool counts = !empty && grad != 0.0f;
    const float g = sum != sum ? NAN : a.tau * grad;             // a teacher without a value leaves none to any element
    __syncthreads();                                            // z is read: dz may be z
    for (uint64_t i = tid; i < a.vocab; i += THREADS) {
        const float q = counts ? expf((E::load(z[i]) - low) * a.inv_tau - log_low) : 0.0f;
        dz[i] = E::store(counts ? g * q : 0.0f);
    }
    if (!counts) return;
    __syncthreads();
    k = 0;
#pragma unroll
    for (uint32_t i0 = 0; i0 < TQ_DISTILL_MAX_TOP; i0 += THREADS, ++k) {
        const uint32_t i = i0 + tid;
        if (i < a.top && id[i] >= 0) {
            bool first = true;
            for (uint32_t j = 0; j < i; ++j) first &= id[j] != id[i];
            if (first) {
                float p = 0.0f;
                for (uint32_t j = i; j < a.top; ++j)
                    if (id[j] == id[i]) p += expf((prob[j] - peak) * a.inv_tau - log_sum);
                dz[id[i]] = E::store(g * (expf((named[k] - low) * a.inv_tau - log_low) - p));
            }
        }
    }
}

template <int MODE>
hipError_t launch(const DistillArgs& a, int dtype, hipStream_t st)
{
    dim3 grid;
    if (!fold_grid(a.rows, 256, 1, grid)) return hipErrorInvalidValue;
    if (dtype == TQ_F32) distill_kernel<TQ_F32, MODE, 256><<<grid, 256, 0, st>>>(a);
    else if (dtype == TQ_BF16) distill_kernel<TQ_BF16, MODE, 256><<<grid, 256, 0, st>>>(a);
    else distill_kernel<TQ_F16, MODE, 256><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}

}  // namespace
}  // namespace tq

hipError_t tq_launch_distill(const void* z, int dtype, uint64_t rows, uint64_t vocab, uint64_t ldz, const void* ids, int ids_bytes,
                             const float* t, uint64_t top, float temperature, const float* stats_in, const float* grad, float* loss,
                             float* stats, void* dz, uint64_t lddz, hipStream_t st)
{
    using namespace tq;
    DistillArgs a = {};
    a.z = z;
    a.ids = ids;
    a.t = t;
    a.grad = grad;
    a.stats_in = stats_in;
    a.loss = loss;
    a.stats = stats;
    a.dz = dz;
    a.ldz = ldz;
    a.lddz = lddz;
    a.rows = (uint32_t)rows;
    a.vocab = (uint32_t)vocab;
    a.top = (uint32_t)top;
    a.wide_ids = ids_bytes == 8;
    a.tau = temperature;
    a.inv_tau = 1.0f / temperature;
    if (!dz) return launch<kForward>(a, dtype, st);
    return stats_in ? launch<kBackward>(a, dtype, st) : launch<kBoth>(a, dtype, st);
}
