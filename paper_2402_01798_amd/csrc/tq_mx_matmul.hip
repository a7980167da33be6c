// Products of microscaled 4-bit matrices (tq_mx.h): out = A B^T (+ add).
#include <type_traits>

#include "tq_mx_device.h"

namespace tq {
namespace {

constexpr uint64_t kUnits = 256, kLds = 160 << 10;                 // compute units, and the LDS of one in bytes
constexpr uint64_t kSplitGroups = 16;                              // of a workgroup at least, where k is split over several
constexpr uint64_t kSplitSaves = 40;

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatmulArgs {
    const void* x;                 // tokens that are not in 4-bit form yet, in place of a and sa
    const uint8_t *a, *sa, *b, *sb;
    const float* add;
    void* out;
    uint64_t ldx, lda, ldo;
    uint32_t m, n, k, groups;
    uint32_t tiles_x;
    uint64_t tiles;                // of the output, times `splits`
    float* partial;                // [splits][m][n]: sums over parts of k that different workgroups take
    uint32_t splits;
};

// 32 x 32 outputs += 64 elements of k.  Lane l holds row l % 32 and block l / 32 of both operands: 32 codes and their scale, a byte
// of a word.
template <int BYTE>
__device__ __forceinline__ f32x16 mfma32(i32x4 a, i32x4 b, f32x16 c, int sa, int sb)
{
    const i32x8 wa = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1);
    const i32x8 wb = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(wa, wb, c, 4, 4, BYTE, sa, BYTE, sb);
}

template <int DTYPE>
__device__ __forceinline__ void store_one(const MatmulArgs& g, uint32_t row, uint32_t col, float v)
{
    using E = Element<DTYPE>;
    if (row >= g.m || col >= g.n) return;
    static_cast<typename E::type*>(g.out)[row * g.ldo + col] = E::store(v);
}

typedef __attribute__((address_space(1))) const void global_bytes;
typedef __attribute__((address_space(3))) void lds_bytes;

// Which tile this workgroup takes.  Workgroups go to the 8 dies in turn; each die takes a run of tiles, which goes down 4 tiles and
// then on to the next column, so that the tiles at work on a die at a time share their rows in its cache.
__device__ __forceinline__ bool find_tile(const MatmulArgs& g, uint32_t& ty, uint32_t& tx, uint32_t& split)
{
    const uint32_t block = linear_block(), per = (uint32_t)(g.tiles + 7) / 8;
    uint32_t tile = (block & 7) * per + (block >> 3);
    if (block >= 8 * per || tile >= g.tiles) return false;
    const uint32_t of_a_split = (uint32_t)g.tiles / g.splits, tiles_y = of_a_split / g.tiles_x;
    split = tile / of_a_split;
    tile -= split * of_a_split;
    const uint32_t band = tile / (4 * g.tiles_x), rows = min(4u, tiles_y - band * 4), in = tile - band * 4 * g.tiles_x;
    ty = band * 4 + in % rows;
    tx = in / rows;
    return true;
}

// BM x BN outputs by WM x WN wavefronts, GROUPS groups of 128 elements of k at a time through a ring of STAGES buffers in LDS.  A
// buffer holds BM rows of A and BN of B, 64 GROUPS bytes each, then the groups' scales, 4 bytes for each row.
template <int BM, int BN, int WM, int WN, int KS, int GROUPS, int STAGES>
struct Tile {
    static constexpr int kThreads = WM * WN * KS * 64, kWaves = WM * WN;     // wavefronts of a part
    static constexpr int kFragsM = BM / WM / 32, kFragsN = BN / WN / 32;
    static constexpr int kRow = 64 * GROUPS;                       // bytes
    static constexpr int kPieces = 4 * GROUPS;                     // of 16 bytes in a row
    static constexpr int kRows = 64 / kPieces;                     // that one request of a wavefront covers
    static constexpr int kScales = (BM + BN) * kRow;               // where a buffer's scales begin
    static constexpr int kStage = kScales + (BM + BN) * 4 * GROUPS;
    static constexpr int kRequests = (BM + BN) / kRows;            // of codes, shared by the wavefronts; some make one a second time
    static constexpr int kLoads = (kRequests + kWaves - 1) / kWaves;
    static constexpr int kScaleLoads = ((BM + BN) * GROUPS / 64 + kWaves - 1) / kWaves;
    static constexpr int kPerStage = kLoads + kScaleLoads;
    static constexpr int kRing = STAGES * kStage;
    static constexpr int kSums = KS > 1 ? BM * (BN + 1) * 4 : 0;   // a part's outputs, a row longer against bank conflicts
    static constexpr int kBytes = KS * (kRing > kSums ? kRing : kSums);
    static constexpr int kOnUnit = kThreads > 512 ? 1 : (int)(kLds / kBytes);  // workgroups on a compute unit
    static constexpr int kOnSimd = (kOnUnit * kThreads + 255) / 256;           // wavefronts on a SIMD, which share 512 registers
    static constexpr int kFrags = kFragsM * kFragsN;
    // registers that sums (16 a fragment), operands (8 a row and column of them) and some 38 others leave, and the fragments whose
    // addends they hold
    static constexpr int kRoom = (512 / kOnSimd < 256 ? 512 / kOnSimd : 256) - 16 * kFrags - 8 * (kFragsM + kFragsN) - 38;
    static constexpr int kEarly = kRoom < 16 ? 0 : kRoom / 16 < kFrags ? kRoom / 16 : kFrags, kAhead = kEarly ? kEarly : 1;
    static_assert(BM % 64 == 0 && BN % 64 == 0 && kBytes <= kLds, "requests of scales are of 64 rows");
};

// Waits until the requests of all but the newest `newer` stages (at most N) are there.
template <int PER, int N>
__device__ __forceinline__ void wait_for_stages(uint32_t newer)
{
    if constexpr (N > 0) {
        if (newer < N) return wait_for_stages<PER, N - 1>(newer);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PER * N) : "memory");
}

// Registers for as many wavefronts on a SIMD as LDS has room for workgroups on the compute unit.
template <int DTYPE, int BM, int BN, int WM, int WN, int KS, int GROUPS, int STAGES, bool ADD>
__global__ __launch_bounds__(WM * WN * KS * 64, (Tile<BM, BN, WM, WN, KS, GROUPS, STAGES>::kOnSimd)) void mx_matmul_tile_kernel(MatmulArgs g)
{
    using S = Tile<BM, BN, WM, WN, KS, GROUPS, STAGES>;
    extern __shared__ char lds[];
    uint32_t ty, tx, split;
    if (!find_tile(g, ty, tx, split)) return;
    const uint32_t lane = threadIdx.x & 63, wave_in_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t part = wave_in_all / S::kWaves, wave = wave_in_all % S::kWaves;
    const uint32_t r = lane & 31, half = lane >> 5, wm = wave / WN, wn = wave % WN;
    const uint32_t row0 = ty * BM, col0 = tx * BN;

    // A row's pieces lie in the buffer in another order from row to row: piece p of row n in place p ^ turn(n), so that 16 rows'
    // pieces of the same k, which are read together, lie in 64 different banks.
    constexpr auto turn = [](uint32_t n) { return GROUPS == 1 ? n >> 2 & 3 : n >> 1 & 7; };
    const uint8_t* from[S::kLoads];                                // rows past the end repeat the last
    uint32_t scale_row[S::kScaleLoads];
    static_assert(S::kRows * S::kWaves % 16 == 0 && (S::kRequests % S::kWaves == 0 || S::kRows == 16),
                  "turn, of period 16, is the same in each of a wavefront's requests");
    const uint32_t piece = (lane % S::kPieces) ^ turn(wave * S::kRows + lane / S::kPieces);
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
        const uint32_t c = (i * S::kWaves + wave) % S::kRequests;  // A's rows first
        const bool is_a = c < BM / S::kRows;
        const uint32_t row = (is_a ? c : c - BM / S::kRows) * S::kRows + lane / S::kPieces;
        from[i] = (is_a ? g.a : g.b) + (uint64_t)(is_a ? min(row0 + row, g.m - 1) : min(col0 + row, g.n - 1)) * g.groups * 64;
    }
#pragma unroll
    for (int i = 0; i < S::kScaleLoads; ++i) {
        const uint32_t c = (i * S::kWaves + wave) % ((BM + BN) * GROUPS / 64);     // group after group: A's rows, then B's
        const uint32_t row = c % ((BM + BN) / 64) * 64 + lane;
        scale_row[i] = row < BM ? min(row0 + row, g.m - 1) : min(col0 + row - BM, g.n - 1);
    }
    // this part of k, in trips of GROUPS groups, up to `end`; `most` is the longest part's
    const uint32_t all = (g.groups + GROUPS - 1) / GROUPS, of_a_split = KS == 1 ? all : (all + g.splits - 1) / g.splits;
    const uint32_t begin = KS == 1 ? 0 : split * of_a_split, end = min(begin + of_a_split, all);
    const uint32_t most = (of_a_split + KS - 1) / KS, first_trip = begin + part * most;
    const uint32_t trips = KS == 1 ? all : first_trip < end ? min(most, end - first_trip) : 0;
    char* ring = lds + part * S::kRing;
    auto fetch = [&](uint32_t t, uint32_t stage) {
        char* base = ring + stage * S::kStage;
        const uint32_t first = (first_trip + t) * GROUPS;
        // the second half of the last stage may not be there: the first again, which is not used
        const uint32_t at = (GROUPS == 1 || first + 1 < g.groups ? piece : piece & 3) * 16;
#pragma unroll
        for (int i = 0; i < S::kLoads; ++i) {
            const uint32_t c = (i * S::kWaves + wave) % S::kRequests;
            __builtin_amdgcn_global_load_lds((global_bytes*)(from[i] + (uint64_t)first * 64 + at), (lds_bytes*)(base + c * 1024), 16, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < S::kScaleLoads; ++i) {
            const uint32_t c = (i * S::kWaves + wave) % ((BM + BN) * GROUPS / 64), in_group = c % ((BM + BN) / 64);
            const uint64_t group = min(first + c / ((BM + BN) / 64), g.groups - 1);
            const uint32_t* q = in_group < BM / 64 ? reinterpret_cast<const uint32_t*>(g.sa) + group * g.m
                                                   : reinterpret_cast<const uint32_t*>(g.sb) + group * g.n;
            __builtin_amdgcn_global_load_lds((global_bytes*)(q + scale_row[i]), (lds_bytes*)(base + S::kScales + c * 256), 4, 0, 0);
        }
    };

    const uint32_t ra = wm * S::kFragsM * 32 + r, rb = BM + wn * S::kFragsN * 32 + r;
    f32x16 acc[S::kFragsM][S::kFragsN] = {};
    // Of 32 x 32 outputs a lane holds 16: with its row of B first in the instruction, of one row 4 columns of every 8, which make
    // whole 16-byte stores of 16-bit elements (bf16 2056 x 1000 x 1999 9.4 -> 8.7 us); else of one column 4 rows of every 8, 32 lanes
    // with 128 bytes of fp32 in a row (fp32 with an addend, the same size, 13.2 -> 10.0 us).
    constexpr bool kAlongRow = KS == 1 && DTYPE != TQ_F32;
    // The addend comes after the sums: they would be rounded to its bits at every step, and gradients that are accumulated over batches
    // are far larger than what one batch adds.  Fragment f's 16, as they are stored.  The first kEarly fragments' are requested before
    // the sums begin, one more when one is used; without registers for that each when it is wanted, while other workgroups work.
    // In the sums from the start / after them, us: 2056 x 1000 x 1999 fp32 10.1 / 10.1, 4096 x 4096 x 512 26.6 / 25.8, 8192 x 8192 x 8192
    // 364 / 357, as bf16 348 / 361, 1037 x 8192 x 4096 bf16 45 / 36.  A kernel for products with an addend and one for those without:
    // the registers that wait for it cost the others 1 % at 8192 x 8192 x 8192.
    auto addends = [&](int f, uint32_t me, float (&v)[2][8]) {
        const uint32_t row = row0 + (wm * S::kFragsM + f / S::kFragsN) * 32, col = col0 + (wn * S::kFragsN + f % S::kFragsN) * 32;
        if constexpr (kAlongRow) {
            const float* from_row = g.add + min(row + (me & 31), g.m - 1) * g.lda;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t at = col + q * 16 + (me >> 5) * 8;
                load8<TQ_F32>(from_row + at, (int)min((int64_t)g.n - (int64_t)at, (int64_t)8), v[q]);
            }
        } else {
            const float* from_col = g.add + min(col + (me & 31), g.n - 1);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e / 8][e % 8] = from_col[min(row + (e / 4) * 8 + (me >> 5) * 4 + e % 4, g.m - 1) * g.lda];
        }
    };
    constexpr int kEach = KS > 1 ? BM * BN / S::kThreads : 1;      // outputs of a thread where the parts are joined
    float extra[S::kAhead][2][8] = {}, extra_of[kEach] = {};
    if constexpr (ADD && KS == 1 && S::kEarly) {
#pragma unroll
        for (int f = 0; f < S::kAhead; ++f) addends(f, lane, extra[f]);
    } else if constexpr (ADD && KS > 1) {
        if (g.splits == 1) {
#pragma unroll
            for (int u = 0; u < kEach; ++u) {
                const uint32_t at = threadIdx.x + u * S::kThreads;
                extra_of[u] = g.add[min(row0 + at / BN, g.m - 1) * g.lda + min(col0 + at % BN, g.n - 1)];
            }
        }
    }
#pragma unroll
    for (uint32_t t = 0; t < STAGES - 1; ++t)
        if (t < trips) fetch(t, t);
    uint32_t stage = 0, free_stage = STAGES - 1;
    for (uint32_t t = 0; t < most; ++t) {
        // this trip's requests are there, and every wavefront is done with the buffer that is filled next
        wait_for_stages<S::kPerStage, STAGES - 2>(t < trips ? trips - 1 - t : 0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        if (t + STAGES - 1 < trips) fetch(t + STAGES - 1, free_stage);
        const char* base = ring + stage * S::kStage;
#pragma unroll
        for (int h = 0; h < GROUPS; ++h) {
            if (KS > 1 && h == 0 && t >= trips) break;             // a shorter part
            if (h && (first_trip + t) * GROUPS + h >= g.groups) break;
            int sa[S::kFragsM], sb[S::kFragsN];
            i32x4 a[2][S::kFragsM], b[2][S::kFragsN];
            const char* scales = base + S::kScales + h * (BM + BN) * 4;
#pragma unroll
            for (int i = 0; i < S::kFragsM; ++i) sa[i] = *reinterpret_cast<const int*>(scales + (ra + i * 32) * 4) >> (8 * half);
#pragma unroll
            for (int j = 0; j < S::kFragsN; ++j) sb[j] = *reinterpret_cast<const int*>(scales + (rb + j * 32) * 4) >> (8 * half);
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const uint32_t at = ((4 * h + 2 * s + half) ^ turn(lane)) * 16;
#pragma unroll
                for (int i = 0; i < S::kFragsM; ++i) a[s][i] = *reinterpret_cast<const i32x4*>(base + (ra + i * 32) * S::kRow + at);
#pragma unroll
                for (int j = 0; j < S::kFragsN; ++j) b[s][j] = *reinterpret_cast<const i32x4*>(base + (rb + j * 32) * S::kRow + at);
            }
#pragma unroll
            for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
                for (int j = 0; j < S::kFragsN; ++j)
                    acc[i][j] = kAlongRow ? mfma32<0>(b[0][j], a[0][i], acc[i][j], sb[j], sa[i]) : mfma32<0>(a[0][i], b[0][j], acc[i][j], sa[i], sb[j]);
#pragma unroll
            for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
                for (int j = 0; j < S::kFragsN; ++j)
                    acc[i][j] = kAlongRow ? mfma32<2>(b[1][j], a[1][i], acc[i][j], sb[j], sa[i]) : mfma32<2>(a[1][i], b[1][j], acc[i][j], sa[i], sb[j]);
        }
        free_stage = stage;
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    if constexpr (KS > 1) {                                        // the parts' sums, joined in their order
        __syncthreads();                                           // the rings are done with
        float* sums = reinterpret_cast<float*>(lds);
        const uint32_t at = (part * BM + wm * S::kFragsM * 32 + half * 4) * (BN + 1) + wn * S::kFragsN * 32 + r;
#pragma unroll
        for (int i = 0; i < S::kFragsM; ++i)
#pragma unroll
            for (int j = 0; j < S::kFragsN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) sums[at + (i * 32 + (e / 4) * 8 + e % 4) * (BN + 1) + j * 32] = acc[i][j][e];
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kEach; ++u) {
            const uint32_t i = threadIdx.x + u * S::kThreads, row = i / BN, col = i % BN;
            float v = 0.0f;
#pragma unroll
            for (int q = 0; q < KS; ++q) v += sums[(q * BM + row) * (BN + 1) + col];
            if constexpr (ADD) v += extra_of[u];
            if (g.splits == 1) store_one<DTYPE>(g, row0 + row, col0 + col, v);
            else if (row0 + row < g.m && col0 + col < g.n) g.partial[((uint64_t)split * g.m + row0 + row) * g.n + col0 + col] = v;
        }
        return;
    }
    uint32_t me = threadIdx.x & 63;
    asm volatile("" : "+v"(me));                                   // places in the output are found here, not kept through the loop
#pragma unroll
    for (int f = 0; f < S::kFrags; ++f) {
        const int i = f / S::kFragsN, j = f % S::kFragsN;
        const uint32_t row = row0 + (wm * S::kFragsM + i) * 32, col = col0 + (wn * S::kFragsN + j) * 32;
        if constexpr (ADD && !S::kEarly) addends(f, me, extra[0]);
        float v[2][8];
#pragma unroll
        for (int q = 0; q < 2; ++q)
#pragma unroll
            for (int e = 0; e < (kAlongRow ? 4 : 8); ++e) {
                if constexpr (kAlongRow) {                         // 4 columns changed for 4 with the other half make 8 in a row
                    const auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][q * 8 + e]),
                                                                    __float_as_uint(acc[i][j][q * 8 + 4 + e]), false, false);
                    v[q][e] = __uint_as_float(w[0]);
                    v[q][4 + e] = __uint_as_float(w[1]);
                } else {
                    v[q][e] = acc[i][j][q * 8 + e];
                }
            }
        if constexpr (ADD) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                v[e / 8][e % 8] += extra[f % S::kAhead][e / 8][e % 8];
                asm volatile("" : "+v"(v[e / 8][e % 8]));          // here: beside its store it would wait for the stores before it
            }
            if (S::kEarly && f + S::kAhead < S::kFrags) addends(f + S::kAhead, me, extra[f % S::kAhead]);
            asm volatile("" : "+v"(me));                           // nor from one fragment to the next, where addends wait as well
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (kAlongRow) {
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const uint32_t to_row = row + (me & 31), to_col = col + q * 16 + (me >> 5) * 8;
                if (to_row < g.m && to_col < g.n)
                    store8<DTYPE>(static_cast<typename Element<DTYPE>::type*>(g.out) + to_row * g.ldo + to_col, (int)min(g.n - to_col, 8u), v[q]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) store_one<DTYPE>(g, row + (e / 4) * 8 + (me >> 5) * 4 + e % 4, col + (me & 31), v[e / 8][e % 8]);
        }
    }
}

// Few rows of A, FRAGS x 32 at most, against 32 rows of B, WAVES wavefronts over parts of k: serving, where B is read once and bounds
// it.  B comes through a ring of STAGES buffers for each wavefront, 256 of k at a time, and rows of A in 4-bit form (X < 0) with it.
// Others, of type X, are cast here by every workgroup and stay in LDS; the rings' first requests are on their way meanwhile.
template <int X, int FRAGS, int WAVES, int STAGES>
struct Few {
    static constexpr int kRowsA = X < 0 ? FRAGS * 32 : 0;          // in a buffer, before the 32 of B
    static constexpr int kScales = (kRowsA + 32) * 128;            // then two groups' scales of 32 rows at a time
    static constexpr int kStage = kScales + (kRowsA + 32) * 8;
    static constexpr int kPerStage = 5 * (kRowsA + 32) / 32;       // requests: 4 of codes and one of scales for 32 rows
    static constexpr int kRing = WAVES * STAGES * kStage;
    static constexpr int kSums = WAVES * FRAGS * 32 * 33 * 4;
    static_assert(kRing <= kLds && kRing >= kSums, "the sums take the rings' place");
};
constexpr int kFewWaves = 8, kFewStages = 2;                       // where A is cast
using FewCast = Few<0, 1, kFewWaves, kFewStages>;

__host__ __device__ constexpr uint64_t few_row_bytes(uint64_t groups) { return groups * 64 + 16; }
__host__ __device__ constexpr uint64_t few_bytes(uint64_t m, uint64_t groups) { return FewCast::kRing + m * (few_row_bytes(groups) + groups * 4); }

// X: the type of g.x, or -1 for rows in 4-bit form.
template <int DTYPE, int X, int FRAGS, int WAVES, int STAGES>
__global__ __launch_bounds__(WAVES * 64) void mx_matmul_few_kernel(MatmulArgs g)
{
    using S = Few<X, FRAGS, WAVES, STAGES>;
    static_assert(X < 0 || FRAGS == 1, "rows that are cast here");
    constexpr int kBlocksA = S::kRowsA / 32;                       // blocks of 32 rows in a buffer, A's before B's
    extern __shared__ char lds[];
    const uint32_t tx = linear_block();
    if (tx >= g.tiles) return;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, half = lane >> 5;
    const uint32_t col0 = tx * 32, pairs = (g.groups + 1) / 2;
    const uint32_t per = (pairs + WAVES - 1) / WAVES, first = wave * per, trips = first < pairs ? min(per, pairs - first) : 0;
    char* ring = lds + wave * (STAGES * S::kStage);
    const uint32_t row_bytes = (uint32_t)few_row_bytes(g.groups);
    char* codes = lds + S::kRing;                                  // of rows cast here
    char* scales = codes + g.m * row_bytes;                        // [m][groups][4]

    const uint8_t* from[4 * (kBlocksA + 1)];
    const uint32_t piece[2] = {(lane & 7) ^ (lane >> 4), (lane & 7) ^ (4 + (lane >> 4))};      // of rows 8 i + lane / 8, i even and odd
    uint32_t scale_row[kBlocksA + 1];
#pragma unroll
    for (int i = 0; i < 4 * (kBlocksA + 1); ++i) {
        const uint32_t row = i % 4 * 8 + (lane >> 3);
        from[i] = i < 4 * kBlocksA ? g.a + (uint64_t)min(i / 4 * 32 + row, g.m - 1) * g.groups * 64
                                   : g.b + (uint64_t)min(col0 + row, g.n - 1) * g.groups * 64;
    }
#pragma unroll
    for (int i = 0; i <= kBlocksA; ++i) scale_row[i] = i < kBlocksA ? min(i * 32 + r, g.m - 1) : min(col0 + r, g.n - 1);
    auto fetch = [&](uint32_t t, uint32_t stage) {
        char* base = ring + stage * S::kStage;
        const uint32_t group = 2 * (first + t);
        const bool both = group + 1 < g.groups;                    // the second half of the last may not be there: the first again
#pragma unroll
        for (int i = 0; i < 4 * (kBlocksA + 1); ++i) {
            const uint32_t at = both ? piece[i & 1] : piece[i & 1] & 3;
            __builtin_amdgcn_global_load_lds((global_bytes*)(from[i] + (uint64_t)group * 64 + at * 16), (lds_bytes*)(base + i * 1024), 16, 0, 0);
        }
        const uint64_t mine = both ? group + half : group;
#pragma unroll
        for (int i = 0; i <= kBlocksA; ++i) {
            const uint8_t* q = i < kBlocksA ? g.sa + (mine * g.m + scale_row[i]) * 4 : g.sb + (mine * g.n + scale_row[i]) * 4;
            __builtin_amdgcn_global_load_lds((global_bytes*)q, (lds_bytes*)(base + S::kScales + i * 256), 4, 0, 0);
        }
    };
#pragma unroll
    for (uint32_t t = 0; t < STAGES; ++t)
        if (t < trips) fetch(t, t);

    if constexpr (X >= 0) {
        using T = typename Element<X>::type;
        const uint32_t octs = g.groups * 16, all = g.m * octs;     // of 8 elements in a row: four neighbouring lanes are a block
        auto from_x = [&](uint32_t i, uint32_t& row, uint32_t& oct) {
            row = i / octs;
            oct = i - row * octs;
            return static_cast<const T*>(g.x) + row * g.ldx + (uint64_t)oct * 8;
        };
        auto put = [&](uint32_t row, uint32_t oct, const float (&v)[8]) {
            uint32_t largest = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) largest = max(largest, magnitude_bits(v[j]));
            const uint32_t byte = mx_scale_byte<false>(quad_max(largest));
            *reinterpret_cast<uint32_t*>(codes + row * row_bytes + oct * 4) = mx_nearest(v, byte);
            if ((oct & 3) == 0) scales[row * octs / 4 + oct / 4] = (char)byte;
        };
        uint32_t i = threadIdx.x, row, oct;
        if (g.k % kMxGroup == 0) {                                 // 4 requests of a thread are on their way together
            for (; i + 3 * WAVES * 64 < all; i += 4 * WAVES * 64) {
                Eight<X> w[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) w[u].load(from_x(i + u * WAVES * 64, row, oct));
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    float v[8];
                    w[u].unpack(v);
                    from_x(i + u * WAVES * 64, row, oct);
                    put(row, oct, v);
                }
            }
        }
        for (; i < all; i += WAVES * 64) {
            float v[8];
            const T* p = from_x(i, row, oct);
            load8<X>(p, (int)min((int64_t)g.k - (int64_t)oct * 8, (int64_t)8), v);
            put(row, oct, v);
        }
        __syncthreads();
    }

    const char* my_codes = codes + min(r, g.m - 1) * row_bytes;
    const char* my_scales = scales + min(r, g.m - 1) * g.groups * 4;
    f32x16 acc[FRAGS] = {};
    uint32_t stage = 0;
    for (uint32_t t = 0; t < trips; ++t) {
        wait_for_stages<S::kPerStage, STAGES - 1>(trips - 1 - t);
        const char* base = ring + stage * S::kStage;
        const uint32_t group = 2 * (first + t);
        const bool both = group + 1 < g.groups;
        i32x4 a[FRAGS][4], b[4];
        int sa[FRAGS][2], sb[2];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint32_t at = r * 128 + ((2 * s + half) ^ (r >> 1 & 7)) * 16;
            b[s] = *reinterpret_cast<const i32x4*>(base + kBlocksA * 4096 + at);
#pragma unroll
            for (int f = 0; f < FRAGS; ++f)
                a[f][s] = *reinterpret_cast<const i32x4*>(X < 0 ? base + f * 4096 + at
                                                                : my_codes + (group + (both ? s / 2 : 0)) * 64 + (2 * (s & 1) + half) * 16);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const char* at = base + S::kScales + (h * 32 + r) * 4;
            sb[h] = *reinterpret_cast<const int*>(at + kBlocksA * 256) >> (8 * half);
#pragma unroll
            for (int f = 0; f < FRAGS; ++f)
                sa[f][h] = *reinterpret_cast<const int*>(X < 0 ? at + f * 256 : my_scales + (group + (both ? h : 0)) * 4) >> (8 * half);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");         // the buffer is read: it may be filled again
        if (t + STAGES < trips) fetch(t + STAGES, stage);
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) acc[f] = mfma32<0>(a[f][0], b[0], acc[f], sa[f][0], sb[0]);
#pragma unroll
        for (int f = 0; f < FRAGS; ++f) acc[f] = mfma32<2>(a[f][1], b[1], acc[f], sa[f][0], sb[0]);
        if (both) {
#pragma unroll
            for (int f = 0; f < FRAGS; ++f) acc[f] = mfma32<0>(a[f][2], b[2], acc[f], sa[f][1], sb[1]);
#pragma unroll
            for (int f = 0; f < FRAGS; ++f) acc[f] = mfma32<2>(a[f][3], b[3], acc[f], sa[f][1], sb[1]);
        }
        stage = stage + 1 == STAGES ? 0 : stage + 1;
    }
    __syncthreads();                                               // the rings are done with
    float* sums = reinterpret_cast<float*>(lds);
#pragma unroll
    for (int f = 0; f < FRAGS; ++f)
#pragma unroll
        for (int e = 0; e < 16; ++e) sums[((wave * FRAGS + f) * 32 + (e / 4) * 8 + half * 4 + e % 4) * 33 + r] = acc[f][e];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < g.m * 32; i += WAVES * 64) {
        const uint32_t row = i / 32, col = i & 31;
        float v = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += sums[(w * FRAGS * 32 + row) * 33 + col];
        if (g.add && col0 + col < g.n) v += g.add[row * g.lda + col0 + col];
        store_one<DTYPE>(g, row, col0 + col, v);
    }
}

// The splits' sums, joined in their order.
template <int DTYPE>
__global__ __launch_bounds__(256) void mx_join_kernel(MatmulArgs g)
{
    const uint64_t at = (uint64_t)linear_block() * 256 + threadIdx.x, size = (uint64_t)g.m * g.n;
    if (at >= size) return;
    float v = g.partial[at];
#pragma unroll 8
    for (uint32_t s = 1; s < g.splits; ++s) v += g.partial[s * size + at];
    const uint32_t row = (uint32_t)(at / g.n), col = (uint32_t)(at % g.n);
    if (g.add) v += g.add[row * g.lda + col];
    store_one<DTYPE>(g, row, col, v);
}

template <int DTYPE, int BM, int BN, int WM, int WN, int KS, int GROUPS, int STAGES>
hipError_t launch_tile(MatmulArgs& g, hipStream_t st)
{
    using S = Tile<BM, BN, WM, WN, KS, GROUPS, STAGES>;
    g.tiles_x = (g.n + BN - 1) / BN;
    g.tiles = (uint64_t)g.tiles_x * ((g.m + BM - 1) / BM) * g.splits;
    dim3 grid;
    if (!fold_grid((g.tiles + 7) / 8 * 8, S::kThreads, 1, grid)) return hipErrorInvalidValue;
    if (g.add) mx_matmul_tile_kernel<DTYPE, BM, BN, WM, WN, KS, GROUPS, STAGES, true><<<grid, S::kThreads, S::kBytes, st>>>(g);
    else mx_matmul_tile_kernel<DTYPE, BM, BN, WM, WN, KS, GROUPS, STAGES, false><<<grid, S::kThreads, S::kBytes, st>>>(g);
    return hipGetLastError();
}

template <int DTYPE, int X, int FRAGS, int WAVES, int STAGES>
hipError_t launch_few(MatmulArgs& g, hipStream_t st)
{
    using S = Few<X, FRAGS, WAVES, STAGES>;
    g.tiles = (g.n + 31) / 32;
    dim3 grid;
    if (!fold_grid(g.tiles, WAVES * 64, 1, grid)) return hipErrorInvalidValue;
    const uint32_t bytes = X < 0 ? (uint32_t)S::kRing : (uint32_t)few_bytes(g.m, g.groups);
    mx_matmul_few_kernel<DTYPE, X, FRAGS, WAVES, STAGES><<<grid, WAVES * 64, bytes, st>>>(g);
    return hipGetLastError();
}

// Which kernel.  Times in us of bf16 products, in turn, replayed from a graph; `64/4` are tiles of 64 with k in 4 parts, `few` is
// the kernel for few rows; the last seven rows are fp32:
//   m x n x k            256  256x128  128x320   192    128     64   64/4    few
//   8192 x 8192 x 8192   283    325      360     372    390    459    645          large tiles move least through the caches
//   4096 x 4096 x 4096  47.9   54.0     62.9    62.4   62.3   72.4    113
//   5000 x 5000 x 3000  63.1   67.2     71.2    70.1   73.7   80.5    143
//   2000 x 6000 x 4096  38.9   41.3     54.6    51.1   42.3   49.5   80.7          the others leave a last round with few tiles
//   1037 x 8192 x 4096  38.3   40.2     34.1    52.4   39.6   39.3   63.0
//   600 x 14336 x 4096  39.7   41.4     34.2    54.2   39.5
//   1800 x 5120 x 4096  38.2   40.6     33.8    52.4   39.2
//   3500 x 2816 x 4096  37.2   40.4     34.0    51.5   39.4
//   3000 x 3000 x 4096  37.2   39.0     34.2    32.0   39.1   39.5   62.2
//   1500 x 4000 x 8192  58.6   44.3     51.3    48.5   47.9   52.0   68.4
//   2048 x 2048 x 2048  20.2   14.2     16.5    16.1   11.7   11.4   20.0          256 leaves three quarters of the device without a tile
//   4096 x 1000 x 784   12.3    9.4     10.3    10.4    7.9    8.3   16.5
//   600 x 5000 x 3000   25.3   17.8     20.9    20.6   13.9   14.5   24.4
//   2056 x 1000 x 1999  18.3   12.6     15.2    14.7    9.8    8.6   15.2
//   512 x 4096 x 4096   31.5   20.7     25.8    25.0   15.5   11.4   14.5
//   256 x 4096 x 4096   30.3   19.9     25.0    24.0   14.4    9.0    8.1          64 too: the parts of k run beside each other
//   128 x 8192 x 8192   53.8   35.0     45.9    42.5   25.7   18.8   13.2
//   64 x 8192 x 8192                                                  12.8   11.0  4 wavefronts of 64 x 32
//   64 x 4096 x 4096                                                   8.4    7.1
//   64 x 32000 x 4096                                          18.0   16.7   27.6  1000 tiles, each with all of A to read
//   33 x 33000 x 4096                                          26.0   17.6   29.0  rows that are not there take half of a tile of 128
//   64 x 128256 x 4096                                         62.3   56.1  103
//   64 x 131001 x 1024                                         24.5   21.8   54
//   32 x 8192 x 8192                                                  12.0    8.9  8 wavefronts of 32 x 32
//   32 x 4096 x 4096                                                   8.1    4.6
//   32 x 32000 x 4096                                          16.5          18.7  (4 wavefronts, two workgroups on a unit, 16.0)
//   1 x 32000 x 4096                                                         16.9  (14.1)
//   32 x 1000 x 16384                                                 10.2    8.4  k over workgroups against one
//   32 x 300 x 32768                                                   9.6   13.0
//   784 x 1000 x 64      6.1    4.4      5.2     5.2    3.7    3.2    4.7          nothing to part
//   1 x 8192 x 8192     51.7   34.5     43.6    41.5   24.2   17.6   11.3    7.3
//   4096 x 4096 x 128   14.8   13.8                    13.3   16.6                 the stores, and requests that nothing overlaps
//   4096 x 4096 x 512   18.0   17.5                    16.9   20.4
//   4096 x 4096 x 1024  22.1   21.5                    21.9   26.3
//   8192 x 4096 x 256   27.6   25.8                    24.3   28.8
//   8192 x 8192 x 128   57.0   46.4                    44.4   55.5
//   8192 x 8192 x 512   70.3   71.7                    60.6   76.8
//   64 x 131001 x 1024                                 27.4   24.4   56
// Enough tiles of 128 for every compute unit: the shape whose rounds take least.  Where the sides leave little over this is 256.  The
// rounds are compared by their steps alone.  What a round costs beside them is left out, so up to 512 of k the rule takes tiles of
// 256 where those of 128 are 6 to 22 % faster (two or three of them share a compute unit); from 1024 on that is within 3 %.
// Few tiles and a long k: k is split over workgroups too, where at least 40 groups (5 steps of a workgroup, the second launch's
// price) are saved.  Not split / split, us: 64 x 64 x 8192 9.8 / 7.8, x 32768 28 / 9.5, x 131072 119 / 12, 256 x 256 x 32768 29 / 12,
// 700 x 700 x 32768 35 / 26; with fewer saved it loses (500 x 500 x 4096 7.3 / 8.6).
enum Shape { kFew, kFewOfMany, kFew64, k256, k256x128, k128x320, k192, k128, k64, k64InParts };

// A tile's sides, and the time in ns that 128 elements of k took while 1, 2, .. of them, as many as fit, were at work on every
// compute unit.
struct Pace {
    Shape shape;
    uint64_t bm, bn;
    uint32_t ns[3];
};
constexpr Pace kPaces[] = {{k256, 256, 256, {1010, 0, 0}}, {k256x128, 256, 128, {580, 1090, 0}}, {k128x320, 128, 320, {860, 0, 0}},
                           {k192, 192, 192, {740, 0, 0}},  {k128, 128, 128, {400, 700, 1080}}};

uint64_t tiles_of(uint64_t m, uint64_t n, uint64_t bm, uint64_t bn) { return (m + bm - 1) / bm * ((n + bn - 1) / bn); }

uint64_t pace(const Pace& p, uint64_t m, uint64_t n)
{
    const uint64_t fit = p.ns[2] ? 3 : p.ns[1] ? 2 : 1, each = (tiles_of(m, n, p.bm, p.bn) + kUnits - 1) / kUnits;
    return each / fit * p.ns[fit - 1] + (each % fit ? p.ns[each % fit - 1] : 0);
}

// Over how many workgroups k is split beside the few tiles of 64.
uint32_t splits_of_64(uint64_t m, uint64_t n, uint64_t groups)
{
    const uint64_t most = kUnits / tiles_of(m, n, 64, 64), wanted = groups / kSplitGroups, s = wanted < most ? wanted : most;
    return s > 1 && groups - groups / s >= kSplitSaves ? (uint32_t)s : 1;
}

Shape shape(uint64_t m, uint64_t n, uint64_t groups)
{
    const bool split = splits_of_64(m, n, groups) > 1;
    if (m <= 32 && (!split || groups <= 128)) return n <= kUnits * 32 ? kFew : kFewOfMany;
    if (m <= 64 && !split && n <= kUnits * 32) return kFew64;
    if (m <= 64 || tiles_of(m, n, 128, 128) < kUnits) return tiles_of(m, n, 64, 64) > kUnits || groups < 4 ? k64 : k64InParts;
    const Pace* best = kPaces;
    for (const Pace& p : kPaces)
        if (pace(p, m, n) < pace(*best, m, n)) best = &p;
    return best->shape;
}

uint32_t splits(uint64_t m, uint64_t n, uint64_t groups) { return shape(m, n, groups) == k64InParts ? splits_of_64(m, n, groups) : 1; }

template <int DTYPE>
hipError_t launch_matmul(MatmulArgs& g, hipStream_t st)
{
    g.splits = 1;
    switch (shape(g.m, g.n, g.groups)) {
        case kFew: return launch_few<DTYPE, -1, 1, 8, 2>(g, st);
        case kFewOfMany: return launch_few<DTYPE, -1, 1, 4, 2>(g, st);
        case kFew64: return launch_few<DTYPE, -1, 2, 4, 3>(g, st);
        // 8 wavefronts of 128 x 64, 256 of k a trip (whole lines of 128 bytes): 8192^3 289 us, by 16 wavefronts of 64 x 64 300, and with
        // 128 of k a trip and three buffers 310.  Tiles of which two are to fit have buffers of 128 of k.
        case k256: return launch_tile<DTYPE, 256, 256, 2, 4, 1, 2, 2>(g, st);
        case k256x128: return launch_tile<DTYPE, 256, 128, 4, 2, 1, 1, 3>(g, st);
        case k128x320: return launch_tile<DTYPE, 128, 320, 2, 5, 1, 1, 3>(g, st);
        case k192: return launch_tile<DTYPE, 192, 192, 3, 3, 1, 1, 3>(g, st);
        case k128: return launch_tile<DTYPE, 128, 128, 2, 4, 1, 1, 3>(g, st);
        case k64: return launch_tile<DTYPE, 64, 64, 2, 2, 1, 2, 2>(g, st);
        case k64InParts: break;
    }
    g.splits = splits(g.m, g.n, g.groups);
    const hipError_t e = launch_tile<DTYPE, 64, 64, 2, 2, 4, 2, 2>(g, st);
    if (e != hipSuccess || g.splits == 1) return e;
    dim3 grid;
    if (!fold_grid(((uint64_t)g.m * g.n + 255) / 256, 256, 1, grid)) return hipErrorInvalidValue;
    mx_join_kernel<DTYPE><<<grid, 256, 0, st>>>(g);
    return hipGetLastError();
}

}  // namespace
}  // namespace tq

uint64_t tq_mx_matmul_workspace_bytes_impl(uint64_t m, uint64_t n, uint64_t k)
{
    const uint32_t s = tq::splits(m, n, (k + tq::kMxGroup - 1) / tq::kMxGroup);
    return s == 1 ? 0 : s * m * n * sizeof(float);
}

hipError_t tq_launch_mx_matmul(const void* a, const void* sa, const void* b, const void* sb, uint64_t m, uint64_t n, uint64_t k,
                               const float* add, uint64_t lda, void* out, int dtype, uint64_t ldo, void* workspace, hipStream_t st)
{
    using namespace tq;
    MatmulArgs g = {};
    g.a = static_cast<const uint8_t*>(a);
    g.sa = static_cast<const uint8_t*>(sa);
    g.b = static_cast<const uint8_t*>(b);
    g.sb = static_cast<const uint8_t*>(sb);
    g.add = add;
    g.lda = lda;
    g.out = out;
    g.ldo = ldo;
    g.m = (uint32_t)m;
    g.n = (uint32_t)n;
    g.k = (uint32_t)k;
    g.groups = (uint32_t)((k + kMxGroup - 1) / kMxGroup);
    g.partial = static_cast<float*>(workspace);
    if (dtype == TQ_F32) return launch_matmul<TQ_F32>(g, st);
    return dtype == TQ_BF16 ? launch_matmul<TQ_BF16>(g, st) : launch_matmul<TQ_F16>(g, st);
}

// Rows cast by every workgroup of the product, or once in a launch before it.  Linear layers of n x k, in us (one launch / two), * where
// the rule takes one launch:
//                   1            2            3            4            5            8            16 tokens
//   4096 x 4096    *4.6 / 6.0   *5.0 / 6.1   *5.5 / 6.2   *5.4 / 6.2   *5.9 / 6.3   *6.6 / 6.3    9.0 / 6.5
//   8192 x 2048    *4.5 / 6.0   *4.5 / 6.2   *4.9 / 6.2   *4.9 / 6.3   *5.3 / 6.4   *5.3 / 6.4   *6.5 / 6.5
//   8192 x 8192    *8.7 / 10.4  *9.1 / 10.8  *9.8 / 10.5 *10.4 / 10.9 *11.1 / 10.6  13.0 / 11.0  18.0 / 11.2
//   4096 x 14336   *8.8 / 9.5   *9.9 / 9.5  *10.8 / 9.7   11.8 / 9.6   12.6 / 9.7   15.7 / 9.8   (beyond LDS)
//   32000 x 4096  *14.4 / 16.3 *16.0 / 16.1 *17.3 / 16.3  15.9 / 16.4  17.5 / 16.2  26.2 / 16.3  35.8 / 16.9   four rounds of workgroups
// At its edge the two are within 6 % of each other, with 4096 x 14336 and 32000 x 4096 11 and 6 % apart.
bool tq_mx_linear_in_one(uint64_t m, uint64_t n, uint64_t k)
{
    const uint64_t groups = (k + tq::kMxGroup - 1) / tq::kMxGroup, rounds = (n + 32 * tq::kUnits - 1) / (32 * tq::kUnits);
    return m <= 16 && (m - 1) * groups * rounds <= 256 && tq::few_bytes(m, groups) <= tq::kLds;
}

hipError_t tq_launch_mx_linear_few(const void* x, int x_dtype, uint64_t m, uint64_t ldx, const void* w, const void* sw, uint64_t n,
                                   uint64_t k, void* out, int dtype, uint64_t ldo, hipStream_t st)
{
    using namespace tq;
    MatmulArgs g = {};
    g.x = x;
    g.ldx = ldx;
    g.b = static_cast<const uint8_t*>(w);
    g.sb = static_cast<const uint8_t*>(sw);
    g.out = out;
    g.ldo = ldo;
    g.m = (uint32_t)m;
    g.n = (uint32_t)n;
    g.k = (uint32_t)k;
    g.groups = (uint32_t)((k + kMxGroup - 1) / kMxGroup);
    auto as = [&](auto D) {
        constexpr int T = decltype(D)::value;
        if (x_dtype == TQ_F32) return launch_few<T, TQ_F32, 1, kFewWaves, kFewStages>(g, st);
        return x_dtype == TQ_BF16 ? launch_few<T, TQ_BF16, 1, kFewWaves, kFewStages>(g, st) : launch_few<T, TQ_F16, 1, kFewWaves, kFewStages>(g, st);
    };
    if (dtype == TQ_F32) return as(std::integral_constant<int, TQ_F32>{});
    return dtype == TQ_BF16 ? as(std::integral_constant<int, TQ_BF16>{}) : as(std::integral_constant<int, TQ_F16>{});
}
