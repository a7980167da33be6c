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
    uint32_t rows, vocab, top, pieces;                             // workgroups of a row (kBackward)
    int wide_ids;
    float tau, inv_tau;
};

constexpr uint32_t kSeenBits = 32768;                              // a set of ids, by their low bits

enum { kForward = 0, kBackward = 1, kBoth = 2 };

// A row as whole 16-byte vectors at aligned addresses, up to kIn - 1 loose elements before them and as many behind.
template <int DTYPE>
struct Row {
    using E = Element<DTYPE>;
    using T = typename E::type;
    static constexpr uint32_t kIn = 16 / sizeof(T);                // elements of a vector
    static constexpr uint32_t kNothing = DTYPE == TQ_F32 ? 0xFF800000u : DTYPE == TQ_BF16 ? 0xFF80FF80u : 0xFC00FC00u;      // -inf
    uint32_t head, vectors, tail;

    __device__ __forceinline__ Row(const T* p, uint32_t n)
    {
        head = min((uint32_t)(-(reinterpret_cast<uintptr_t>(p) / sizeof(T))) & (kIn - 1), n);
        vectors = (n - head) / kIn;
        tail = n - head - vectors * kIn;
    }
    // The loose element of this thread (of the first 2 kIn ones), or -1.
    __device__ __forceinline__ int64_t loose(uint32_t tid) const
    {
        if (tid < head) return tid;
        if (tid >= kIn && tid - kIn < tail) return (int64_t)head + (uint64_t)vectors * kIn + (tid - kIn);
        return -1;
    }
    // Whether element `at` is in the vectors k0 .. k1 - 1, or a loose one where k0 is 0.
    __device__ __forceinline__ bool within(uint32_t at, uint32_t k0, uint32_t k1) const
    {
        const uint32_t k = (at - head) / kIn;
        return at < head || k >= vectors ? k0 == 0 : k >= k0 && k < k1;
    }
    // NEAR: the row is short of 4 GiB, so that a vector's place in it is a 32-bit number beside the row's address, which all
    // threads share.
    template <bool NEAR>
    __device__ __forceinline__ u32x4 load(const T* p, uint32_t k) const
    {
        const char* q = reinterpret_cast<const char*>(p + head);
        if constexpr (NEAR) return *reinterpret_cast<const u32x4*>(q + k * 16u);
        else return *reinterpret_cast<const u32x4*>(q + (uint64_t)k * 16);
    }
    static __device__ __forceinline__ void unpack(u32x4 w, float (&v)[kIn])
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (uint32_t e = 0; e < kIn; ++e) v[e] = __uint_as_float(w[e]);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < kIn / 2; ++e) unpack2<DTYPE>(w[e], v[2 * e], v[2 * e + 1]);
        }
    }
    // Vector k of the gradient, which begins at p and lies as the row does (WHOLE) or not.
    template <bool NEAR, bool WHOLE>
    __device__ __forceinline__ void store(T* p, uint32_t k, const float (&v)[kIn]) const
    {
        T* q = NEAR ? p + head + k * kIn : p + head + (uint64_t)k * kIn;
        u32x4 w;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (uint32_t e = 0; e < kIn; ++e) w[e] = __float_as_uint(v[e]);
        } else {
#pragma unroll
            for (uint32_t e = 0; e < kIn / 2; ++e) w[e] = pack2<DTYPE>(v[2 * e], v[2 * e + 1]);
        }
        if constexpr (!WHOLE) __builtin_memcpy(q, &w, 16);         // stored at any address
        else *reinterpret_cast<u32x4*>(q) = w;
    }
};

template <int CTRL>
__device__ __forceinline__ float dpp_float(float v) { return __uint_as_float(dpp_move<CTRL>(__float_as_uint(v))); }

// The sum or the maximum of a wavefront's values, the same bits in every lane, by moves inside the vector unit (through LDS each of
// the six steps takes some hundred clocks, and a short row has six such reductions).
template <bool MAX>
__device__ __forceinline__ float wave_reduce(float v)
{
    auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    v = op(v, dpp_float<0xB1>(v));          // lanes 1 0 3 2
    v = op(v, dpp_float<0x4E>(v));          // lanes 2 3 0 1
    v = op(v, dpp_float<0x141>(v));         // mirrored within 8
    v = op(v, dpp_float<0x140>(v));         // within 16
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Of two values over the workgroup, in a fixed order.  `part` holds two values per wavefront and is used once.
template <int WAVES, bool MAX>
__device__ __forceinline__ void group_reduce(float& x, float& y, float (*part)[2])
{
    auto op = [](float a, float b) { return MAX ? fmaxf(a, b) : a + b; };
    x = wave_reduce<MAX>(x);
    y = wave_reduce<MAX>(y);
    if constexpr (WAVES > 1) {
        if ((threadIdx.x & 63) == 0) {
            part[threadIdx.x >> 6][0] = x;
            part[threadIdx.x >> 6][1] = y;
        }
        __syncthreads();
        x = part[0][0];
        y = part[0][1];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            x = op(x, part[w][0]);
            y = op(y, part[w][1]);
        }
    }
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;                                                       // fmaxf would first rewrite each operand, lest it be a signalling NaN
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
    return d;
}

// Running maximum and sum of exp((z - maximum) / tau) of a thread's elements.
struct Softmax {
    float m = -INFINITY, s = 0.0f;
    template <int N>
    __device__ __forceinline__ void take(const float (&v)[N], float c)
    {
        float top = v[0];
#pragma unroll
        for (int j = 1; j < N; ++j) top = fmaxf(top, v[j]);
        if (top > m) {
            s = m == -INFINITY ? s : s * __builtin_amdgcn_exp2f((m - top) * c);
            m = top;
        }
        const float low = m == -INFINITY ? 0.0f : m;               // -inf - -inf has no value; there the sum stays 0
#pragma unroll
        for (int j = 0; j < N; ++j) s += __builtin_amdgcn_exp2f((v[j] - low) * c);
    }
};

// The compiler would keep the values that it has unpacked for the next pass over them, in twice the registers.
__device__ __forceinline__ void keep_packed(u32x4& w) { asm volatile("" : "+v"(w)); }

__host__ __device__ constexpr uint32_t whole_fours(uint32_t n) { return (n + 3) & ~3u; }

// Whether another entry has entry i's id, whether one before it does, and the sum of t over those behind it, in order.  Four entries
// at a time and no branch between them: one by one, a row of 512 entries with ids that occur twice took 150 us, so 77.
struct Alike {
    bool any = false, before = false;
    float sum = 0.0f;
};
__device__ __forceinline__ Alike alike(const int* id, const float* t, uint32_t top, uint32_t i)
{
    const int mine = id[i];
    Alike r;
#pragma unroll 4
    for (uint32_t j = 0; j < top; j += 4) {
        const u32x4 ids = *reinterpret_cast<const u32x4*>(id + j), ts = *reinterpret_cast<const u32x4*>(t + j);
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const bool same = (int)ids[u] == mine && j + u < top && j + u != i;
            r.any |= same;
            r.before |= same && j + u < i;
            r.sum += same ? __uint_as_float(ts[u]) : 0.0f;
        }
    }
    return r;
}

// One workgroup a row.  VECTORS > 0: the row stays in the registers, VECTORS x 16 bytes a thread, so memory is read once; 0: it is
// read again for the gradient.  WHOLE: dz lies to its 16-byte lines as z does.
template <int DTYPE, int MODE, int THREADS, int VECTORS, bool WHOLE>
__global__ __launch_bounds__(THREADS) void distill_kernel(DistillArgs a)
{
    using E = Element<DTYPE>;
    using T = typename E::type;
    using R = Row<DTYPE>;
    constexpr int WAVES = THREADS / 64;
    constexpr uint32_t IN = R::kIn;
    __shared__ float parts[3][WAVES][2];
    extern __shared__ __attribute__((aligned(16))) char entries[]; // the teacher's: id, logit and then probability, z
    int* id = reinterpret_cast<int*>(entries);
    float* t = reinterpret_cast<float*>(id + whole_fours(a.top));
    float* at_id = t + whole_fours(a.top);
    __shared__ uint32_t seen[MODE == kForward ? 1 : kSeenBits / 32];
    const uint32_t block = linear_block(), tid = threadIdx.x, row = MODE == kBackward ? block / a.pieces : block;
    if (row >= a.rows) return;
    const T* z = static_cast<const T*>(a.z) + (uint64_t)row * a.ldz;
    const R lies(z, a.vocab);
    // this workgroup's vectors of the row, and with the first of them the loose elements
    const uint32_t piece = MODE == kBackward ? block - row * a.pieces : 0, per = MODE == kBackward ? (lies.vectors + a.pieces - 1) / a.pieces : 0;
    const uint32_t k_first = piece * per, k_end = MODE == kBackward ? min(k_first + per, lies.vectors) : lies.vectors;
    const float grad = MODE == kForward ? 0.0f : a.grad[row];
    const float c = a.inv_tau * kLog2e;

    u32x4 held[VECTORS > 0 ? VECTORS : 1];
#pragma unroll
    for (int i = 0; i < VECTORS; ++i) {
        held[i] = u32x4{R::kNothing, R::kNothing, R::kNothing, R::kNothing};
        if (tid + i * THREADS < lies.vectors) held[i] = lies.template load<true>(z, tid + i * THREADS);
    }
    const int64_t loose = piece == 0 ? lies.loose(tid) : -1;
    const float z_loose = loose >= 0 ? E::load(z[loose]) : -INFINITY;

    if constexpr (MODE != kForward) {
        for (uint32_t i = tid; i < kSeenBits / 32; i += THREADS) seen[i] = 0;
    }
    float t_peak = -INFINITY;
    bool bad = false, twice = false;
    for (uint32_t i = tid; i < a.top; i += THREADS) {
        const uint64_t at = (uint64_t)row * a.top + i;
        const int64_t w = a.wide_ids ? static_cast<const int64_t*>(a.ids)[at] : static_cast<const int32_t*>(a.ids)[at];
        const float v = a.t[at];
        const bool there = w >= 0 && w < (int64_t)a.vocab && v != -INFINITY;
        id[i] = there ? (int)w : -1;
        t[i] = v;
        // (another piece's elements may be gradients by now, where dz is z)
        at_id[i] = there && (MODE != kBackward || lies.within((uint32_t)w, k_first, k_end)) ? E::load(z[w]) : 0.0f;
        if (there) {
            t_peak = fmaxf(t_peak, v);
            bad |= !(v < INFINITY);
        }
    }
    if constexpr (MODE != kForward) {                              // whether an id occurs twice: those whose bit was set look closer
        __syncthreads();
        for (uint32_t i = tid; i < a.top; i += THREADS)
            if (id[i] >= 0 && (atomicOr(&seen[(id[i] & (kSeenBits - 1)) / 32], 1u << (id[i] & 31)) >> (id[i] & 31) & 1u))
                twice |= alike(id, t, a.top, i).any;
    }

    float top = z_loose, log_total = 0.0f;                         // the row's largest logit, ln sum exp((z - top) / tau)
    Softmax q;
    if constexpr (MODE != kBackward && VECTORS > 0) {
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) {
            float v[IN];
            R::unpack(held[i], v);
#pragma unroll
            for (uint32_t j = 0; j < IN; j += 2) top = max3(top, v[j], v[j + 1]);
        }
    } else if constexpr (MODE != kBackward) {
        const float first[1] = {z_loose};
        q.take(first, c);
#pragma unroll 4
        for (uint32_t k = tid; k < lies.vectors; k += THREADS) {
            float v[IN];
            R::unpack(lies.template load<false>(z, k), v);
            q.take(v, c);
        }
        top = q.m;
    }
    group_reduce<WAVES, true>(t_peak, top, parts[0]);
    float t_sum = 0.0f, total = 0.0f;
    for (uint32_t i = tid; i < a.top; i += THREADS)
        if (id[i] >= 0) t_sum += __builtin_amdgcn_exp2f((t[i] - t_peak) * c);
    if (bad) t_sum = NAN;
    if constexpr (MODE == kBackward) {
        top = a.stats_in[2 * (uint64_t)row];
        log_total = a.stats_in[2 * (uint64_t)row + 1];
    }
    const float low = top == -INFINITY ? 0.0f : top;               // -inf - -inf has no value
    auto power = [&](float v) { return __builtin_amdgcn_exp2f((v - low) * c); };
    if constexpr (MODE != kBackward && VECTORS > 0) {
        total = power(z_loose);
#pragma unroll
        for (int i = 0; i < VECTORS; ++i) {
            float v[IN];
            keep_packed(held[i]);
            R::unpack(held[i], v);
#pragma unroll
            for (uint32_t j = 0; j < IN; ++j) total += power(v[j]);
        }
    } else if constexpr (MODE != kBackward) {
        total = q.m == -INFINITY ? q.s : q.s * power(q.m);
    }
    group_reduce<WAVES, false>(t_sum, total, parts[1]);
    const bool empty = t_sum == 0.0f;
    const float t_log = empty ? 0.0f : logf(t_sum);
    if constexpr (MODE != kBackward) log_total = logf(total);
    // where nothing is left of the row every z is -inf and q is 0: any finite number does
    const float log_low = log_total == -INFINITY ? 0.0f : log_total;

    float loss = 0.0f, count = twice ? 1.0f : 0.0f;
    for (uint32_t i = tid; i < a.top; i += THREADS) {
        const float x = (t[i] - t_peak) * a.inv_tau - t_log, p = id[i] < 0 ? 0.0f : __builtin_amdgcn_exp2f(x * kLog2e);
        if (!(p <= 0.0f)) loss += p * (x - ((at_id[i] - low) * a.inv_tau - log_low));
        t[i] = p;
    }
    group_reduce<WAVES, false>(loss, count, parts[2]);
    if (MODE != kBackward && tid == 0) {
        a.loss[row] = empty ? 0.0f : loss * a.tau * a.tau;
        if (MODE == kForward) {
            a.stats[2 * (uint64_t)row] = top;
            a.stats[2 * (uint64_t)row + 1] = log_total;
        }
    }
    if constexpr (MODE != kForward) {
        T* dz = static_cast<T*>(a.dz) + (uint64_t)row * a.lddz;
        const bool counts = !empty && grad != 0.0f;
        const float g = t_sum != t_sum ? NAN : a.tau * grad;       // a teacher without a value leaves none to any element
        const float scale = counts ? g * __builtin_amdgcn_exp2f(-log_low * kLog2e) : 0.0f;
        // (the reductions' barriers: every z[id] is read where dz is z)
        if (loose >= 0) dz[loose] = E::store(counts ? scale * power(z_loose) : 0.0f);
        const float from = counts ? low : 0.0f;                    // of a row that does not count zeros are left: 0 * 2^0
        auto put = [&](uint32_t k, u32x4 w) {
            float v[IN];
            R::unpack(w, v);
#pragma unroll
            for (uint32_t j = 0; j < IN; ++j) v[j] = scale * __builtin_amdgcn_exp2f((v[j] - from) * c);
            lies.template store<(VECTORS > 0), WHOLE>(dz, k, v);
        };
        if constexpr (VECTORS > 0) {
            if (!counts) {
#pragma unroll
                for (int i = 0; i < VECTORS; ++i) held[i] = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < VECTORS; ++i) {
                keep_packed(held[i]);
                if (tid + i * THREADS < lies.vectors) put(tid + i * THREADS, held[i]);
            }
        } else if (counts) {
#pragma unroll 4
            for (uint32_t k = k_first + tid; k < k_end; k += THREADS) put(k, lies.template load<false>(z, k));
        } else {
            for (uint32_t k = k_first + tid; k < k_end; k += THREADS) put(k, u32x4{0, 0, 0, 0});
        }
        if (!counts) return;
        __syncthreads();                                           // the elements that the teacher names are written once more
        for (uint32_t i = tid; i < a.top; i += THREADS)
            if (id[i] >= 0 && lies.within(id[i], k_first, k_end)) {
                float p = t[i];
                if (count != 0.0f) {                               // an id's first entry takes the probabilities of all
                    const Alike others = alike(id, t, a.top, i);
                    if (others.before) continue;
                    p += others.sum;
                }
                dz[id[i]] = E::store(scale * power(at_id[i]) - g * p);
            }
    }
}

template <int DTYPE, int MODE, int THREADS, int VECTORS>
hipError_t launch(const DistillArgs& a, hipStream_t st)
{
    dim3 grid;
    if (!fold_grid((uint64_t)a.rows * a.pieces, THREADS, 1, grid)) return hipErrorInvalidValue;
    const size_t entries = 12 * (size_t)whole_fours(a.top);
    if constexpr (MODE != kForward) {
        const uint64_t size = DTYPE == TQ_F32 ? 4 : 2;
        if (((reinterpret_cast<uintptr_t>(a.dz) - reinterpret_cast<uintptr_t>(a.z)) | (a.lddz - a.ldz) * size) & 15u) {
            distill_kernel<DTYPE, MODE, THREADS, VECTORS, false><<<grid, THREADS, entries, st>>>(a);
            return hipGetLastError();
        }
    }
    distill_kernel<DTYPE, MODE, THREADS, VECTORS, true><<<grid, THREADS, entries, st>>>(a);
    return hipGetLastError();
}

template <int DTYPE, int MODE>
hipError_t launch(DistillArgs& a, hipStream_t st)
{
    const uint64_t vectors = (uint64_t)a.vocab / Row<DTYPE>::kIn;
    // The smallest workgroup whose registers hold the row, so that several share a compute unit and one computes while another waits for
    // memory (2048 x 50001 bf16 with the loss: 1024 threads with 8 vectors 124 us, 512 with 16 92); at 16 vectors of 1024 threads
    // one fills it.  Longer rows are read twice.  The forward pass has nothing to keep: long rows go past the registers (2048 x 131072:
    // kept 134 us, not kept 92), short ones are faster from them, since their maximum is known before their sum begins.
    if constexpr (MODE == kForward) {
        if (vectors <= 64 * 4) return launch<DTYPE, MODE, 64, 4>(a, st);
        if (vectors <= 256 * 4) return launch<DTYPE, MODE, 256, 4>(a, st);
        if (vectors <= 256 * 8) return launch<DTYPE, MODE, 256, 8>(a, st);
        if (vectors <= 512 * 8) return launch<DTYPE, MODE, 512, 8>(a, st);
        if (vectors <= 512 * 16) return launch<DTYPE, MODE, 512, 0>(a, st);
        return launch<DTYPE, MODE, 1024, 0>(a, st);
    } else if constexpr (MODE == kBoth) {
        if (vectors <= 64 * 4) return launch<DTYPE, MODE, 64, 4>(a, st);
        if (vectors <= 256 * 4) return launch<DTYPE, MODE, 256, 4>(a, st);
        if (vectors <= 256 * 8) return launch<DTYPE, MODE, 256, 8>(a, st);
        if (vectors <= 512 * 8) return launch<DTYPE, MODE, 512, 8>(a, st);
        if (vectors <= 512 * 16) return launch<DTYPE, MODE, 512, 16>(a, st);
        if (vectors <= 1024 * 16) return launch<DTYPE, MODE, 1024, 16>(a, st);
        return launch<DTYPE, MODE, 1024, 0>(a, st);
    } else {
        if (vectors <= 256) return launch<DTYPE, MODE, 64, 0>(a, st);
        const uint64_t wanted = 1024 / a.rows, most = vectors / 1024;      // a few workgroups for each compute unit, 4 vectors a thread
        a.pieces = (uint32_t)(most < wanted ? most : wanted);
        if (a.pieces < 1) a.pieces = 1;
        if (vectors <= 4096 || a.pieces > 1) return launch<DTYPE, MODE, 256, 0>(a, st);
        return launch<DTYPE, MODE, 1024, 0>(a, st);
    }
}

template <int MODE>
hipError_t launch(DistillArgs& a, int dtype, hipStream_t st)
{
    if (dtype == TQ_F32) return launch<TQ_F32, MODE>(a, st);
    return dtype == TQ_BF16 ? launch<TQ_BF16, MODE>(a, st) : launch<TQ_F16, MODE>(a, st);
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
    a.pieces = 1;
    a.wide_ids = ids_bytes == 8;
    a.tau = temperature;
    a.inv_tau = 1.0f / temperature;
    if (!dz) return launch<kForward>(a, dtype, st);
    return stats_in ? launch<kBackward>(a, dtype, st) : launch<kBoth>(a, dtype, st);
}
