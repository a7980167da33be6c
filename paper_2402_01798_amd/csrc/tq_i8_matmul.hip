// Products of matrices of 8-bit integers (tq_i8.h): out = A B^T (+ bias), and linear layers whose tokens are cast inside.
#include <type_traits>

#include "tq_i8_device.h"
#include "tq_tiles.h"

namespace tq {

using namespace i8;

namespace {

struct I8MatmulArgs {
    const void* x;                 // tokens that are not in 8-bit form yet, in place of a and sa
    const uint8_t *a, *b;
    const float *sa, *sb, *bias;
    void* out;
    uint64_t ldx, ldo;
    uint32_t m, n, k, groups;
    uint32_t tiles_x, tiles_y, tiles;
    uint32_t splits;               // of k, over workgroups
    int* partial;                  // [splits][m][n]
};

// Of 8 sums of a row from column `col` on.
template <int DTYPE>
__device__ __forceinline__ void store_scaled(const I8MatmulArgs& g, uint32_t row, uint32_t col, const int (&sums)[8])
{
    const int n = (int)min(g.n - col, 8u);
    const float sa = g.sa[row];
    float sb[8], bias[8], v[8];
    load8<TQ_F32>(g.sb + col, n, sb);
    if (g.bias) load8<TQ_F32>(g.bias + col, n, bias);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = (float)sums[e] * sa * sb[e];
        if (g.bias) v[e] += bias[e];
    }
    store8<DTYPE>(static_cast<typename Element<DTYPE>::type*>(g.out) + row * g.ldo + col, n, v);
}

// 8192^3 to bf16: 447 to 475 us (2.3 to 2.5 POP/s); a library's product to int32 of the same codes, in turn, 433 to 440.  The matrix units are busy 67 % of
// the clocks at 1.7 GHz: the low clock points to power.  The first calls after a pause take 580 to 720.  Four wavefronts of 128 x 128 with slices of
// 64 bytes, not tried apart: 506, units busy 61 %.
template <int DTYPE, class S>
__global__ __launch_bounds__(S::kThreads, S::kOnSimd) void i8_tile_kernel(I8MatmulArgs g)
{
    extern __shared__ char lds[];
    uint32_t tile, ty, tx;
    if (!tile_number(linear_block(), g.tiles * g.splits, tile)) return;
    const uint32_t split = tile / g.tiles, each = (g.groups + g.splits - 1) / g.splits, first = min(split * each, g.groups);
    tile_place(tile - split * g.tiles, g.tiles_y, g.tiles_x, ty, tx);
    typename S::Sums acc[S::kFragsM][S::kFragsN];
    tile_sums<S>(TileOperands{g.a, g.b, g.m, g.n, g.groups, first, min(each, g.groups - first)}, ty * S::BM, tx * S::BN, lds, acc);
    tile_chunks<S>(acc, ty * S::BM, tx * S::BN, [&](uint32_t row, uint32_t col, const int (&sums)[8]) {
        if (row >= g.m || col >= g.n) return;
        if (g.splits == 1) return store_scaled<DTYPE>(g, row, col, sums);
        float bits[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) bits[e] = __int_as_float(sums[e]);
        store8<TQ_F32>(reinterpret_cast<float*>(g.partial) + ((uint64_t)split * g.m + row) * g.n + col, (int)min(g.n - col, 8u), bits);
    });
}

// The splits' sums, joined: whole numbers, so in any order.
template <int DTYPE>
__global__ __launch_bounds__(256) void i8_join_kernel(I8MatmulArgs g)
{
    const uint32_t chunks = (g.n + 7) / 8;
    const uint64_t at = (uint64_t)linear_block() * 256 + threadIdx.x, row = at / chunks;
    if (row >= g.m) return;
    const uint32_t col = (uint32_t)(at - row * chunks) * 8;
    const int n = (int)min(g.n - col, 8u);
    int sums[8] = {};
#pragma unroll 8
    for (uint32_t s = 0; s < g.splits; ++s) {
        float bits[8];
        load8<TQ_F32>(reinterpret_cast<const float*>(g.partial) + (s * (uint64_t)g.m + row) * g.n + col, n, bits);
#pragma unroll
        for (int e = 0; e < 8; ++e) sums[e] += __float_as_int(bits[e]);
    }
    store_scaled<DTYPE>(g, (uint32_t)row, col, sums);
}

// Few rows of A, 32 at most, against 32 rows of B, WAVES wavefronts over parts of k: serving, where B is read once and bounds it.
// B comes through a ring of STAGES buffers for each wavefront, 128 bytes of k at a time.  A, by HOW: in the same ring (kStream); whole into
// LDS, where it is small (kKept); or cast there by every workgroup, from type HOW (0 ..).
enum { kStream = -2, kKept = -1 };

template <int HOW, int WAVES, int STAGES>
struct Few {
    static constexpr int kBlocksA = HOW == kStream ? 1 : 0;        // blocks of 32 rows in a buffer, A's before B's
    static constexpr int kStage = (kBlocksA + 1) * 4096, kLoads = (kBlocksA + 1) * 4;
    static constexpr int kRing = WAVES * STAGES * kStage, kSums = WAVES * 32 * 33 * 4;
    static_assert(kRing <= (int)kLdsBytes, "rings");
};

__host__ __device__ constexpr uint64_t kept_row(uint64_t groups) { return groups * 128 + 16; }    // 16 more: rows in different banks

template <class S>
constexpr uint64_t few_bytes(uint64_t kept) { return S::kRing + kept > (uint64_t)S::kSums ? S::kRing + kept : S::kSums; }

template <int DTYPE, int HOW, int WAVES, int STAGES>
__global__ __launch_bounds__(WAVES * 64) void i8_few_kernel(I8MatmulArgs g)
{
#ifdef __HIP_DEVICE_COMPILE__                                      // the host's pass does not know the type of a buffer
    using S = Few<HOW, WAVES, STAGES>;
    using P = TileProduct<kInt8>;
    extern __shared__ char lds[];
    const uint32_t tx = linear_block();
    if (tx >= g.tiles) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5;
    const uint32_t col0 = tx * 32, per = (g.groups + WAVES - 1) / WAVES, first = min(wave * per, g.groups), trips = min(per, g.groups - first);
    const uint64_t stride = (uint64_t)g.groups * 128;
    char* ring = lds + wave * (STAGES * S::kStage);
    char* kept = lds + S::kRing;
    float* kept_scales = reinterpret_cast<float*>(kept + g.m * kept_row(g.groups));
    // Rows past the end repeat the last.  A request covers 8 rows; pieces of 16 bytes lie as in tiles.
    uint32_t from[S::kLoads];
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const bool is_a = i < 4 * S::kBlocksA;
        const uint32_t row = (is_a ? i : i - 4 * S::kBlocksA) * 8 + lane / 8;
        from[i] = min(row, (is_a ? g.m : g.n - col0) - 1) * (uint32_t)stride + ((lane & 7) ^ tile_turn(i * 8 + lane / 8)) * 16;
    }
    const uint32_t turned = trips ? tx % trips : 0;                // workgroups begin at different places
    auto group_of = [&](uint32_t t) { return first + (t + turned < trips ? t + turned : t + turned - trips); };
    auto fetch = [&](uint32_t t, uint32_t stage) {
        const int some = __builtin_amdgcn_readfirstlane(t < trips ? -1 : 0);        // of length 0 behind the last
        const auto of_b = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.b) + col0 * stride, 0, some, 0x20000);
        const auto of_a = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(g.a), 0, some, 0x20000);
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(i < 4 * S::kBlocksA ? of_a : of_b, (tile_lds_bytes*)(ring + stage * S::kStage + i * 1024), 16,
                                                     from[i], group_of(t) * 128, 0, 0);
    };
#pragma unroll
    for (uint32_t t = 0; t < STAGES; ++t) fetch(t, t);

    if constexpr (HOW == kKept) {
        for (uint32_t row = wave; row < g.m; row += WAVES)
            for (uint32_t i = lane; i < g.groups * 8; i += 64)
                *reinterpret_cast<u32x4*>(kept + row * kept_row(g.groups) + i * 16) = *reinterpret_cast<const u32x4*>(g.a + row * stride + i * 16);
        __syncthreads();
    } else if constexpr (HOW >= 0) {                               // rows side by side, each by `team` wavefronts
        using T = typename Element<HOW>::type;
        constexpr int kAhead = HOW == TQ_F32 ? 8 : 16;             // requests of a lane on their way together
        __shared__ uint32_t part[2][WAVES];
        const uint32_t octs = g.groups * 16, team = g.m == 1 ? WAVES : g.m == 2 ? WAVES / 2 : g.m <= 4 ? WAVES / 4 : 1, at_once = WAVES / team;
        const uint32_t me = wave % team * 64 + lane, step = team * 64;
        for (uint32_t turn = 0; turn * at_once < g.m; ++turn) {
            const uint32_t row = turn * at_once + wave / team;
            const bool some = row < g.m;                           // wavefronts without a row meet the others at the barrier
            const T* x = static_cast<const T*>(g.x) + min(row, g.m - 1) * g.ldx;
            auto load = [&](Eight<HOW>& e, uint32_t oct) {
                const int64_t n = some ? (int64_t)g.k - (int64_t)oct * 8 : 0;
                if (n >= 8) e.load(x + (uint64_t)oct * 8);
                else if (n > 0) e.load(x + (uint64_t)oct * 8, (int)n);
                else e.clear();
            };
            Eight<HOW> w[kAhead];
            uint32_t largest = 0;
            for (uint32_t o = 0; o < octs; o += kAhead * step) {
#pragma unroll
                for (int i = 0; i < kAhead; ++i) load(w[i], o + i * step + me);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) largest = max(largest, w[i].largest());
            }
            largest = wave_largest(largest);
            if (lane == 0) part[turn & 1][wave] = largest;
            __syncthreads();
            for (uint32_t v = 0; v < team; ++v) largest = max(largest, part[turn & 1][wave / team * team + v]);
            const I8Row s(largest);
            if (some && me == 0) kept_scales[row] = s.scale;
            for (uint32_t o = 0; o < octs; o += kAhead * step) {
                if (octs > kAhead * step) {                        // a longer row is read again
#pragma unroll
                    for (int i = 0; i < kAhead; ++i) load(w[i], o + i * step + me);
                }
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const uint32_t oct = o + i * step + me;
                    if (!some || oct >= octs) continue;
                    float v[8];
                    w[i].unpack(v);
                    *reinterpret_cast<u32x2*>(kept + row * kept_row(g.groups) + oct * 8) = s.codes(v);
                }
            }
        }
        __syncthreads();
    }

    const char* mine = kept + min(r, g.m - 1) * kept_row(g.groups) + half * 16;
    P::Sums acc;
#pragma unroll
    for (int e = 0; e < 16; ++e) acc[e] = 0;
    uint32_t stage = 0;
    for (uint32_t t = 0; t < trips; ++t) {
        asm volatile("s_waitcnt vmcnt(%0)" ::"n"(S::kLoads * (STAGES - 1)) : "memory");
        const char* base = ring + stage * S::kStage;
        tile_i32x4 a[4], b[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint32_t at = r * 128 + ((2 * s + half) ^ tile_turn(r)) * 16;
            b[s] = *reinterpret_cast<const tile_i32x4*>(base + S::kBlocksA * 4096 + at);
            a[s] = *reinterpret_cast<const tile_i32x4*>(HOW == kStream ? base + at : mine + group_of(t) * 128 + s * 32);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the buffer is read: it may be filled again
        fetch(t + STAGES, stage);
#pragma unroll
        for (int s = 0; s < 4; ++s) acc = P::step(a[s], b[s], acc);
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    constexpr int kEach = 32 * 32 / (WAVES * 64);                  // outputs of a thread
    float scales[kEach];                                           // of the rows that it joins below
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const uint32_t row = min((threadIdx.x + u * WAVES * 64) / 32, g.m - 1);
        scales[u] = HOW >= 0 ? kept_scales[row] : g.sa[row];
    }
    __syncthreads();                                               // the rings and what is kept behind them are done with
    int* sums = reinterpret_cast<int*>(lds);
#pragma unroll
    for (int e = 0; e < 16; ++e) sums[(wave * 32 + (e / 4) * 8 + half * 4 + e % 4) * 33 + r] = acc[e];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const uint32_t i = threadIdx.x + u * WAVES * 64, row = i / 32, col = i & 31;
        if (row >= g.m || col0 + col >= g.n) continue;
        int sum = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum += sums[(w * 32 + row) * 33 + col];
        float v = (float)sum * scales[u] * g.sb[col0 + col];
        if (g.bias) v += g.bias[col0 + col];
        static_cast<typename Element<DTYPE>::type*>(g.out)[row * g.ldo + col0 + col] = Element<DTYPE>::store(v);
    }
#endif
}

template <int DTYPE, class S>
hipError_t launch_tiles(I8MatmulArgs& g, hipStream_t st)
{
    const uint64_t x = ((uint64_t)g.n + S::BN - 1) / S::BN, y = ((uint64_t)g.m + S::BM - 1) / S::BM;
    dim3 grid;
    if (x * y * g.splits > 0xFFFFFFF0ull || !fold_grid((x * y * g.splits + 7) / 8 * 8, S::kThreads, 1, grid)) return hipErrorInvalidValue;
    g.tiles_x = (uint32_t)x;
    g.tiles_y = (uint32_t)y;
    g.tiles = (uint32_t)(x * y);
    i8_tile_kernel<DTYPE, S><<<grid, S::kThreads, S::kBytes, st>>>(g);
    return hipGetLastError();
}

template <int DTYPE, int HOW, int WAVES, int STAGES>
hipError_t launch_few(I8MatmulArgs& g, hipStream_t st)
{
    using S = Few<HOW, WAVES, STAGES>;
    g.tiles = (g.n + 31) / 32;
    dim3 grid;
    if (!fold_grid(g.tiles, WAVES * 64, 1, grid)) return hipErrorInvalidValue;
    const uint64_t kept = HOW == kStream ? 0 : g.m * kept_row(g.groups) + g.m * 4;
    i8_few_kernel<DTYPE, HOW, WAVES, STAGES><<<grid, WAVES * 64, few_bytes<S>(kept), st>>>(g);
    return hipGetLastError();
}

constexpr uint64_t kKeptBytes = 30 << 10;      // of A in LDS, beside rings of 48 or 64 KiB

// Few rows, wavefronts x buffers, us of a linear layer in bf16 (the cast of A with it):
//   m x n x k            8 x 4    8 x 2    4 x 2    4 x 3    4 x 4
//   1 x 4096 x 4096        7.7      7.4      7.6      7.7      7.8
//   1 x 8192 x 8064       15.1     15.4     15.9     15.9     16.0
//   1 x 8192 x 8192       19.4     16.7     16.3     16.6     16.6     rows a power of two apart wait for each other: fewer of them are
//   1 x 4096 x 16384      17.9     16.3     16.9     16.9     17.1     asked for at a time
//   1 x 14336 x 4096               11.9     11.3     11.1     11.5     two workgroups or more on a unit
//   1 x 14336 x 8192               22.3     23.0     22.7     22.2
// and of rows that come with B:
//   24 x 4096 x 4096              10.2     10.2     10.1     10.2
//   24 x 14336 x 4096             16.8     14.0     15.5     15.9
//   24 x 8192 x 8192              21.7     17.4     17.8     18.0
// Requests of 1024 bytes of one row, with a barrier for every 32 rows of that, took as long or longer (8192 x 8192 19.4, 14336 x 4096 14.1).

template <int DTYPE>
hipError_t launch_matmul(I8MatmulArgs& g, hipStream_t st)
{
    g.splits = splits_of(g.m, g.n, g.groups);
    switch (shape_of(g.m, g.n, g.groups)) {
        case kFewShape:
            if (g.m * kept_row(g.groups) <= kKeptBytes)
                return g.n <= 32 * kComputeUnits ? launch_few<DTYPE, kKept, 8, 2>(g, st) : launch_few<DTYPE, kKept, 4, 3>(g, st);
            return launch_few<DTYPE, kStream, 4, 2>(g, st);
        case k256: return launch_tiles<DTYPE, TileShape<kInt8, 256, 256, 2, 4, 2>>(g, st);
        case k192: return launch_tiles<DTYPE, TileShape<kInt8, 192, 192, 2, 6, 3>>(g, st);
        case k256x128: return launch_tiles<DTYPE, TileShape<kInt8, 256, 128, 4, 2, 3>>(g, st);
        case k192x256: return launch_tiles<DTYPE, TileShape<kInt8, 192, 256, 2, 4, 2>>(g, st);
        case k128x320: return launch_tiles<DTYPE, TileShape<kInt8, 128, 320, 4, 2, 2>>(g, st);
        case k128x256: return launch_tiles<DTYPE, TileShape<kInt8, 128, 256, 2, 4, 3>>(g, st);
        case k128: return launch_tiles<DTYPE, TileShape<kInt8, 128, 128, 2, 4, 2>>(g, st);
        case k64: break;
    }
    const hipError_t e = launch_tiles<DTYPE, TileShape<kInt8, 64, 64, 2, 2, 3>>(g, st);
    if (e != hipSuccess || g.splits == 1) return e;
    dim3 grid;
    if (!fold_grid(((uint64_t)g.m * ((g.n + 7) / 8) + 255) / 256, 256, 1, grid)) return hipErrorInvalidValue;
    i8_join_kernel<DTYPE><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace
}  // namespace tq

uint64_t tq_i8_matmul_workspace_bytes_impl(uint64_t m, uint64_t n, uint64_t k)
{
    const uint32_t s = tq::splits_of(m, n, (k + 127) / 128);
    return s == 1 ? 0 : s * m * n * sizeof(int);
}

hipError_t tq_launch_i8_matmul(const void* a, const float* sa, const void* b, const float* sb, uint64_t m, uint64_t n, uint64_t k,
                               const float* bias, void* out, int dtype, uint64_t ldo, void* workspace, hipStream_t st)
{
    using namespace tq;
    I8MatmulArgs g = {};
    g.a = static_cast<const uint8_t*>(a);
    g.b = static_cast<const uint8_t*>(b);
    g.sa = sa;
    g.sb = sb;
    g.bias = bias;
    g.out = out;
    g.ldo = ldo;
    g.m = (uint32_t)m;
    g.n = (uint32_t)n;
    g.k = (uint32_t)k;
    g.groups = (uint32_t)((k + 127) / 128);
    g.partial = static_cast<int*>(workspace);
    if (dtype == TQ_F32) return launch_matmul<TQ_F32>(g, st);
    return dtype == TQ_BF16 ? launch_matmul<TQ_BF16>(g, st) : launch_matmul<TQ_F16>(g, st);
}

bool tq_i8_linear_in_one(uint64_t m, uint64_t n, uint64_t k)
{
    return m <= 8 && m * tq::kept_row((k + 127) / 128) <= tq::kKeptBytes;
}

hipError_t tq_launch_i8_linear_few(const void* x, int x_dtype, uint64_t m, uint64_t ldx, const void* w, const float* sw, uint64_t n, uint64_t k,
                                   const float* bias, void* out, int dtype, uint64_t ldo, hipStream_t st)
{
    using namespace tq;
    I8MatmulArgs g = {};
    g.x = x;
    g.ldx = ldx;
    g.b = static_cast<const uint8_t*>(w);
    g.sb = sw;
    g.bias = bias;
    g.out = out;
    g.ldo = ldo;
    g.m = (uint32_t)m;
    g.n = (uint32_t)n;
    g.k = (uint32_t)k;
    g.groups = (uint32_t)((k + 127) / 128);
    auto as = [&](auto D, auto X) {
        constexpr int T = decltype(D)::value, F = decltype(X)::value;
        return g.n <= 32 * kComputeUnits ? launch_few<T, F, 8, 2>(g, st) : launch_few<T, F, 4, 3>(g, st);
    };
    auto from = [&](auto D) {
        if (x_dtype == TQ_F32) return as(D, std::integral_constant<int, TQ_F32>{});
        return x_dtype == TQ_BF16 ? as(D, std::integral_constant<int, TQ_BF16>{}) : as(D, std::integral_constant<int, TQ_F16>{});
    };
    if (dtype == TQ_F32) return from(std::integral_constant<int, TQ_F32>{});
    return dtype == TQ_BF16 ? from(std::integral_constant<int, TQ_BF16>{}) : from(std::integral_constant<int, TQ_F16>{});
}
