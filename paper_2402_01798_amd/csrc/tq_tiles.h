// Tiles of products A B^T on the matrix cores, for operands whose rows lie as groups of 128 bytes of k: 8-bit integers, binary16
// numbers, or pairs of those.  The sums of a tile stay in registers; what becomes of them is the calling kernel's.
#pragma once

#include <type_traits>

#include "tq_mx_device.h"
#include "tq_shapes.h"

namespace tq {

constexpr uint64_t kLdsBytes = 160 << 10;
constexpr int kGroupBytes = 128;

typedef int tile_i32x4 __attribute__((ext_vector_type(4)));
typedef int tile_i32x16 __attribute__((ext_vector_type(16)));
typedef float tile_f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 tile_f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void tile_lds_bytes;

// 32 x 32 outputs += 16 bytes of k of 64 lanes: lane l holds row l % 32, half l / 32 of 32 bytes, of both operands.
template <int KIND>
struct TileProduct {
    using Sums = tile_f32x16;
    static __device__ __forceinline__ Sums step(tile_i32x4 a, tile_i32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(tile_f16x8, a), __builtin_bit_cast(tile_f16x8, b), c, 0, 0, 0);
    }
};
template <>
struct TileProduct<kInt8> {
    using Sums = tile_i32x16;
    static __device__ __forceinline__ Sums step(tile_i32x4 a, tile_i32x4 b, Sums c)
    {
        return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
    }
};

// BM x BN outputs by WM x WN wavefronts, a group of k at a time through a ring of STAGES buffers in LDS: BM rows of A, then BN of B.
template <int KIND_, int BM_, int BN_, int WM_, int WN_, int STAGES_>
struct TileShape {
    static constexpr int KIND = KIND_, BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_;
    using Product = TileProduct<KIND>;
    using Sums = typename Product::Sums;
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int kFragsM = BM / WM / 32, kFragsN = BN / WN / 32;
    static constexpr int kStage = (BM + BN) * kGroupBytes, kBytes = STAGES * kStage;
    static constexpr int kPieces = kGroupBytes / 16, kRows = 64 / kPieces;  // rows that a request of a wavefront covers
    static constexpr int kLoadsA = BM / kRows / kWaves, kLoads = (BM + BN) / kRows / kWaves;   // requests of a wavefront for a buffer
    static constexpr int kOnUnit = (int)kLdsBytes / kBytes;        // workgroups on a compute unit
    static constexpr int kOnSimd = kOnUnit * kWaves / 4 < 1 ? 1 : kOnUnit * kWaves / 4 > 4 ? 4 : kOnUnit * kWaves / 4;      // wavefronts
    static constexpr bool kPair = KIND == kHalfPair;
    static constexpr int kStep = kPair ? 64 : 32, kSteps = kGroupBytes / kStep; // bytes of a row that are multiplied at a time
    static constexpr int kReads = (kFragsM + kFragsN) * (kPair ? 2 : 1), kProducts = kFragsM * kFragsN * (kPair ? 3 : 1);     // of a step
    static_assert(kSteps % 2 == 0, "operands are read into two sets of registers in turn");
    static_assert(BM / kRows % kWaves == 0 && BN / kRows % kWaves == 0 && kRows * kWaves % 16 == 0 && kBytes <= (int)kLdsBytes && STAGES >= 2,
                  "requests in equal numbers");
};

struct TileOperands {
    const uint8_t *a, *b;          // rows of groups * 128 bytes; BM and BN of them and a row more within 2^32 bytes, which offsets are checked against
    uint32_t m, n, groups;
    uint32_t first, count;         // the groups of k that are summed
};

// A row's pieces of 16 bytes lie in a buffer in another order from row to row: piece p of row r in place p ^ tile_turn(r), so that
// 16 rows' pieces of the same k, which are read together, lie in 64 different banks.
__device__ __forceinline__ uint32_t tile_turn(uint32_t row) { return row >> 1 & 7; }

// A step's operands in a wavefront's registers; of pairs, their second numbers too.
template <class S>
struct TileFragments {
    tile_i32x4 a[S::kPair ? 2 : 1][S::kFragsM], b[S::kPair ? 2 : 1][S::kFragsN];

    // The R-th of kReads requests, first those of the first products.
    template <int R>
    __device__ __forceinline__ void read(const char* rows_a, const char* rows_b, uint32_t at)
    {
        constexpr int low = R / (S::kFragsM + S::kFragsN), r = R % (S::kFragsM + S::kFragsN);
        if constexpr (low) at ^= 32;
        if constexpr (r == 0) b[low][0] = *reinterpret_cast<const tile_i32x4*>(rows_b + at);
        else if constexpr (r <= S::kFragsM) a[low][r - 1] = *reinterpret_cast<const tile_i32x4*>(rows_a + (r - 1) * 32 * kGroupBytes + at);
        else b[low][r - S::kFragsM] = *reinterpret_cast<const tile_i32x4*>(rows_b + (r - S::kFragsM) * 32 * kGroupBytes + at);
    }
    // The P-th of kProducts.  Of pairs (a + a')(b + b') but for a' b', which is 2^-22 of it.
    template <int P>
    __device__ __forceinline__ void product(typename S::Sums (&acc)[S::kFragsM][S::kFragsN]) const
    {
        constexpr int which = P / (S::kFragsM * S::kFragsN), i = P % S::kFragsM, j = P / S::kFragsM % S::kFragsN;
        acc[i][j] = S::Product::step(b[which == 2][j], a[which == 1][i], acc[i][j]);
    }
};

template <int N, typename F>
__device__ __forceinline__ void repeat(F f)
{
    if constexpr (N > 0) {
        repeat<N - 1>(f);
        f(std::integral_constant<int, N - 1>{});
    }
}

// Sums of the tile at (row0, col0).  Rows past the end repeat the last: their sums mean nothing.  A lane holds of 32 x 32 outputs
// one row's: element e is column (e / 4) * 8 + (lane / 32) * 4 + e % 4 of row lane % 32.
// A step's operands are read while the step before it is multiplied, one request behind a product; the first ones of the next group in the
// second half of a group's last step, behind the barrier after which every wavefront is done with this group's buffer.
template <class S>
__device__ __forceinline__ void tile_sums(const TileOperands& g, uint32_t row0, uint32_t col0, char* lds,
                                          typename S::Sums (&acc)[S::kFragsM][S::kFragsN])
{
#ifdef __HIP_DEVICE_COMPILE__                                      // the host's pass does not know the type of a buffer
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 31, half = lane >> 5, wm = wave / S::WN, wn = wave % S::WN;
    row0 = __builtin_amdgcn_readfirstlane(row0);                   // the same in all lanes, which divisions hide from the compiler
    col0 = __builtin_amdgcn_readfirstlane(col0);
    const uint64_t stride = (uint64_t)g.groups * kGroupBytes;
    const uint32_t trips = g.count;
    uint32_t from[S::kLoads];
    const uint32_t piece = (lane % S::kPieces) ^ tile_turn(wave * S::kRows + lane / S::kPieces);       // in each of a wavefront's requests
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const bool is_a = i < S::kLoadsA;                          // A's rows first
        const uint32_t row = (i * S::kWaves + wave) * S::kRows - (is_a ? 0 : S::BM) + lane / S::kPieces;
        from[i] = min(row, (is_a ? g.m - row0 : g.n - col0) - 1) * (uint32_t)stride + piece * 16;
    }
    // The groups behind the last are requested with a length of 0 in place of the operands': nothing is read, and every trip is alike.
    auto fetch_one = [&](auto I, uint32_t t, uint32_t stage) {
        constexpr int i = decltype(I)::value;
        // buffer addressing: a lane's place in the tile is a 32-bit number, and what all lanes share a scalar
        const auto of = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(i < S::kLoadsA ? g.a + row0 * stride : g.b + col0 * stride), 0,
                                                          __builtin_amdgcn_readfirstlane(t < trips ? -1 : 0), 0x20000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(of, (tile_lds_bytes*)(lds + stage * S::kStage + (i * S::kWaves + wave) * 1024), 16, from[i],
                                                 (g.first + t) * kGroupBytes, 0, 0);
    };
#pragma unroll
    for (uint32_t t = 0; t < S::STAGES; ++t) repeat<S::kLoads>([&](auto I) { fetch_one(I, t, t); });
#pragma unroll
    for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
        for (int j = 0; j < S::kFragsN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const uint32_t rows_a = (wm * S::kFragsM * 32 + r) * kGroupBytes, rows_b = (S::BM + wn * S::kFragsN * 32 + r) * kGroupBytes;
    const uint32_t first_piece = (half ^ tile_turn(lane)) * 16;      // of step 0
    auto read = [&](TileFragments<S>& f, auto R, const char* base, int s) {
        f.template read<decltype(R)::value>(base + rows_a, base + rows_b, first_piece ^ (S::kStep * s));
    };
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(S::kLoads * (S::STAGES - 1)) : "memory");
    TileFragments<S> now[2];
    repeat<S::kReads>([&](auto R) { read(now[0], R, lds, 0); });
    constexpr int kHalfway = S::kProducts / 2, kLeft = S::kProducts - kHalfway;
    constexpr int kReadsEach = (2 * S::kReads + kLeft - 1) / kLeft, kLoadsEach = (S::kLoads + kLeft - 1) / kLeft;
    uint32_t stage = 0;
    for (uint32_t t = 0; t < trips; ++t) {
        const char* base = lds + stage * S::kStage;
        repeat<S::kSteps - 1>([&](auto I) {
            constexpr int s = decltype(I)::value;
            repeat<S::kProducts>([&](auto P) {
                now[s & 1].template product<decltype(P)::value>(acc);
                constexpr int each = (S::kReads + S::kProducts - 1) / S::kProducts;
                repeat<each>([&](auto R) {
                    constexpr int at = decltype(P)::value * each + decltype(R)::value;
                    if constexpr (at < S::kReads) read(now[~s & 1], std::integral_constant<int, at>{}, base, s + 1);
                });
                __builtin_amdgcn_sched_barrier(0);
            });
        });
        TileFragments<S>& last = now[(S::kSteps - 1) & 1];
        const uint32_t next = stage + 1 == S::STAGES ? 0 : stage + 1;
        repeat<kHalfway>([&](auto P) { last.template product<decltype(P)::value>(acc); });
        __builtin_amdgcn_sched_barrier(0);
        // the next group is there, and every wavefront has read this one
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(S::kLoads * (S::STAGES - 2)) : "memory");
        const char* after = lds + next * S::kStage;
        repeat<kLeft>([&](auto Q) {
            constexpr int q = decltype(Q)::value;
            last.template product<kHalfway + q>(acc);
            repeat<kReadsEach>([&](auto R) {
                constexpr int at = q * kReadsEach + decltype(R)::value;
                if constexpr (at < S::kReads) read(now[0], std::integral_constant<int, at>{}, after, 0);
            });
            repeat<kLoadsEach>([&](auto I) {
                constexpr int at = q * kLoadsEach + decltype(I)::value;
                if constexpr (at < S::kLoads) fetch_one(std::integral_constant<int, at>{}, t + S::STAGES, stage);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        stage = next;
    }
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");   // nothing is on its way to LDS any more
#endif
}

// f(row, column of the first, 8 sums side by side) for all of this lane's sums of the tile.
template <class S, typename F>
__device__ __forceinline__ void tile_chunks(const typename S::Sums (&acc)[S::kFragsM][S::kFragsN], uint32_t row0, uint32_t col0, F f)
{
    using Value = std::remove_reference_t<decltype(acc[0][0][0] + 0)>;
    uint32_t me = threadIdx.x & 63;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / S::WN, wn = wave % S::WN;
    asm volatile("" : "+v"(me));                                   // places are found here, not kept through the sums' loop
#pragma unroll
    for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
        for (int j = 0; j < S::kFragsN; ++j)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                Value v[8];
#pragma unroll
                for (int e = 0; e < 4; ++e) {                      // 4 columns changed for 4 with the other half make 8 in a row
                    const Value a = acc[i][j][q * 8 + e], b = acc[i][j][q * 8 + 4 + e];
                    const auto w = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b), false, false);
                    const uint32_t c = w[0], d = w[1];
                    v[e] = __builtin_bit_cast(Value, c);
                    v[4 + e] = __builtin_bit_cast(Value, d);
                }
                f(row0 + (wm * S::kFragsM + i) * 32 + (me & 31), col0 + (wn * S::kFragsN + j) * 32 + q * 16 + (me >> 5) * 8, v);
            }
}

// Which of `tiles` this workgroup takes.  Workgroups go to the 8 dies in turn; each die takes a run of tiles, so that what its tiles share
// is in its cache.  false: none.
__device__ __forceinline__ bool tile_number(uint32_t block, uint32_t tiles, uint32_t& tile)
{
    const uint32_t per = (tiles + 7) / 8;
    tile = (block & 7) * per + (block >> 3);
    return block < 8 * per && tile < tiles;
}
// Tile `tile` of tiles_y x tiles_x: a run goes down 4 tiles and then on to the next column.
__device__ __forceinline__ void tile_place(uint32_t tile, uint32_t tiles_y, uint32_t tiles_x, uint32_t& ty, uint32_t& tx)
{
    const uint32_t band = tile / (4 * tiles_x), rows = min(4u, tiles_y - band * 4), in = tile - band * 4 * tiles_x;
    ty = band * 4 + in % rows;
    tx = in / rows;
}
// Tile `tile` of those on and below the diagonal of `rows` x `rows`, in bands of 4 rows: down a band's rows and on to the next column, at its end
// what there is of the diagonal's columns.  8 b^2 + 2 b of them come before band b.
__device__ __forceinline__ void tile_place_below(uint32_t tile, uint32_t rows, uint32_t& ty, uint32_t& tx)
{
    uint32_t b = (uint32_t)(sqrtf((float)tile * 0.125f));          // within one of it
    while (b && 8 * b * b + 2 * b > tile) --b;
    while (8 * (b + 1) * (b + 1) + 2 * (b + 1) <= tile) ++b;
    uint32_t in = tile - (8 * b * b + 2 * b);
    const uint32_t high = min(4u, rows - 4 * b);
    if (in < 4 * b * high) {
        tx = in / high;
        ty = 4 * b + in % high;
        return;
    }
    in -= 4 * b * high;
    tx = 4 * b;
    for (uint32_t left = high; in >= left; --left) {
        in -= left;
        ++tx;
    }
    ty = tx + in;
}

}  // namespace tq
