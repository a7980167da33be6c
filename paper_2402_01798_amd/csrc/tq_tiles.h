// Tiles of products A B^T on the matrix cores, for operands whose rows lie as groups of 128 bytes of k: 8-bit integers, binary16
// numbers, or pairs of those.  The sums of a tile stay in registers; what becomes of them is the calling kernel's.
#pragma once

#include "tq_mx_device.h"

namespace tq {

constexpr uint64_t kComputeUnits = 256, kLdsBytes = 160 << 10;

// What a group of 128 bytes holds.  kHalfPair: 32 elements as the sum of two binary16 numbers, the 32 larger ones first.
enum { kInt8, kHalf, kHalfPair };

constexpr __host__ __device__ uint32_t in_group(int kind) { return kind == kInt8 ? 128u : kind == kHalf ? 64u : 32u; }

typedef int tile_i32x4 __attribute__((ext_vector_type(4)));
typedef int tile_i32x16 __attribute__((ext_vector_type(16)));
typedef float tile_f32x16 __attribute__((ext_vector_type(16)));
typedef _Float16 tile_f16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(1))) const void tile_global_bytes;
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
    static constexpr int kStage = (BM + BN) * 128, kBytes = STAGES * kStage;
    static constexpr int kLoads = (BM + BN) / 8 / kWaves;          // requests of a wavefront for a buffer, 8 rows each
    static constexpr int kOnUnit = kThreads > 512 ? 1 : (int)(kLdsBytes / kBytes) * kThreads > 2048 ? 2048 / kThreads : (int)(kLdsBytes / kBytes);
    static constexpr int kOnSimd = (kOnUnit * kThreads + 255) / 256 > 4 ? 4 : (kOnUnit * kThreads + 255) / 256;
    static_assert((BM + BN) / 8 % kWaves == 0 && kWaves % 2 == 0 && kBytes <= (int)kLdsBytes, "requests in equal numbers");
};

// Waits until the requests of all but the newest `newer` buffers (at most N) are there.
template <int PER, int N>
__device__ __forceinline__ void wait_for_buffers(uint32_t newer)
{
    if constexpr (N > 0) {
        if (newer < N) return wait_for_buffers<PER, N - 1>(newer);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PER * N) : "memory");
}

struct TileOperands {
    const uint8_t *a, *b;          // rows of groups * 128 bytes
    uint32_t m, n, groups;
    uint32_t first, trips;         // the groups of k that are summed
};

// A row's 8 pieces of 16 bytes lie in a buffer in another order from row to row: piece p of row r in place p ^ tile_turn(r), so that
// 16 rows' pieces of the same k, which are read together, lie in 64 different banks.
__device__ __forceinline__ uint32_t tile_turn(uint32_t row) { return row >> 1 & 7; }

// Sums of the tile at (row0, col0).  Rows past the end repeat the last: their sums mean nothing.  A lane holds of 32 x 32 outputs
// one row's: element e is column (e / 4) * 8 + (lane / 32) * 4 + e % 4 of row lane % 32.
template <class S>
__device__ __forceinline__ void tile_sums(const TileOperands& g, uint32_t row0, uint32_t col0, char* lds,
                                          typename S::Sums (&acc)[S::kFragsM][S::kFragsN])
{
    using P = typename S::Product;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t r = lane & 31, half = lane >> 5, wm = wave / S::WN, wn = wave % S::WN;
    const uint8_t* from[S::kLoads];
    const uint32_t piece = (lane % 8) ^ tile_turn(wave * 8 + lane / 8);        // the same in each of a wavefront's requests
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const uint32_t c = i * S::kWaves + wave;                   // A's rows first
        const bool is_a = c < S::BM / 8;
        const uint32_t row = (is_a ? c : c - S::BM / 8) * 8 + lane / 8;
        from[i] = (is_a ? g.a : g.b) + ((uint64_t)(is_a ? min(row0 + row, g.m - 1) : min(col0 + row, g.n - 1)) * g.groups + g.first) * 128 + piece * 16;
    }
    auto fetch = [&](uint32_t t, uint32_t stage) {
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i)
            __builtin_amdgcn_global_load_lds((tile_global_bytes*)(from[i] + (uint64_t)t * 128),
                                             (tile_lds_bytes*)(lds + stage * S::kStage + (i * S::kWaves + wave) * 1024), 16, 0, 0);
    };
#pragma unroll
    for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
        for (int j = 0; j < S::kFragsN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0;
    const uint32_t ra = wm * S::kFragsM * 32 + r, rb = S::BM + wn * S::kFragsN * 32 + r;
#pragma unroll
    for (uint32_t t = 0; t < S::STAGES - 1; ++t)
        if (t < g.trips) fetch(t, t);
    uint32_t stage = 0, free_stage = S::STAGES - 1;
    for (uint32_t t = 0; t < g.trips; ++t) {
        // this trip's requests are there, and every wavefront is done with the buffer that is filled next
        wait_for_buffers<S::kLoads, S::STAGES - 2>(g.trips - 1 - t);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + S::STAGES - 1 < g.trips) fetch(t + S::STAGES - 1, free_stage);
        const char* base = lds + stage * S::kStage;
        auto read = [&](uint32_t row, int s) {
            return *reinterpret_cast<const tile_i32x4*>(base + row * 128 + ((2 * s + half) ^ tile_turn(lane)) * 16);
        };
        constexpr int kSteps = S::KIND == kHalfPair ? 2 : 4;
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            tile_i32x4 a[S::kFragsM], b[S::kFragsN];
#pragma unroll
            for (int i = 0; i < S::kFragsM; ++i) a[i] = read(ra + i * 32, s);
#pragma unroll
            for (int j = 0; j < S::kFragsN; ++j) b[j] = read(rb + j * 32, s);
            if constexpr (S::KIND == kHalfPair) {                  // (a + a')(b + b') but for a' b', which is 2^-22 of it
                tile_i32x4 low[S::kFragsN > S::kFragsM ? S::kFragsN : S::kFragsM];
#pragma unroll
                for (int j = 0; j < S::kFragsN; ++j) low[j] = read(rb + j * 32, s + 2);
#pragma unroll
                for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
                    for (int j = 0; j < S::kFragsN; ++j) acc[i][j] = P::step(low[j], a[i], acc[i][j]);
#pragma unroll
                for (int i = 0; i < S::kFragsM; ++i) low[i] = read(ra + i * 32, s + 2);
#pragma unroll
                for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
                    for (int j = 0; j < S::kFragsN; ++j) acc[i][j] = P::step(b[j], low[i], acc[i][j]);
            }
#pragma unroll
            for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
                for (int j = 0; j < S::kFragsN; ++j) acc[i][j] = P::step(b[j], a[i], acc[i][j]);
        }
        free_stage = stage;
        stage = stage + 1 == S::STAGES ? 0 : stage + 1;
    }
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
// Tile `tile` of those on and below the diagonal, row after row.
__device__ __forceinline__ void tile_place_below(uint32_t tile, uint32_t& ty, uint32_t& tx)
{
    ty = (uint32_t)((sqrtf(8.0f * (float)tile + 1.0f) - 1.0f) * 0.5f);
    while ((uint64_t)(ty + 1) * (ty + 2) / 2 <= tile) ++ty;
    while ((uint64_t)ty * (ty + 1) / 2 > tile) --ty;
    tx = tile - (uint32_t)((uint64_t)ty * (ty + 1) / 2);
}

}  // namespace tq
