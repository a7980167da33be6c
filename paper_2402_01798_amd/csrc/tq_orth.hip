// Orthogonalised updates (tq_orth.h): momentum, the norm, Newton-Schulz steps, new parameters.
//
// X and the products' other operands are held in binary16, times 2^12: singular values stay within 3 (the entry point sees to it), so
// that no element passes 2^16, and elements down to 2^-26 of the largest singular value keep all their bits.  A step is three products, of
// rows along k in all of them:
//     A = X X^T (symmetric: the tiles on and below the diagonal),  B = a I + b A + c A A (symmetric too),  X' = B X
// the last against X^T, so X' is written both ways.  The last X' is written once, as the result or into the parameters.
#include <type_traits>

#include "tq_orth.h"
#include "tq_tiles.h"

namespace tq {

using namespace orth;

namespace {

constexpr float kUnit = 4096.0f;               // what elements in binary16 are held times
constexpr uint32_t kParts = 256;               // partial sums of a matrix's squares, at most

struct OrthPointers {
    const void* g[TQ_ORTH_MAX_COUNT];
    const float* v[TQ_ORTH_MAX_COUNT];
    float* v_out[TQ_ORTH_MAX_COUNT];
};

struct OrthArgs {
    char* workspace;
    uint64_t stride;                           // bytes of a matrix's part of the workspace
    uint64_t x, xt, a, b;                      // where in it they lie; the partial sums at 0
    uint64_t size;                             // elements
    uint32_t rows, cols, parts;
    uint32_t tiles_x, tiles;
    float momentum, eps;
    int nesterov, update, flip;
};

template <int DTYPE>
__device__ __forceinline__ void load_eight(const void* p, uint64_t at, int n, float (&v)[8])
{
    load8<DTYPE>(static_cast<const typename Element<DTYPE>::type*>(p) + at, n, v);
}

// Sums of squares in binary64, and the new momentum.  Memory: four of 1024 x 4096 fp32 48 us, 4.2 TB/s.
template <int DTYPE>
__global__ __launch_bounds__(256) void orth_norm_kernel(OrthPointers p, OrthArgs o)
{
    __shared__ double part[256];
    const uint32_t which = blockIdx.y, block = linear_block();
    if (block >= o.parts) return;
    double sum = 0.0;
    for (uint64_t at = ((uint64_t)block * 256 + threadIdx.x) * 8; at < o.size; at += (uint64_t)o.parts * 2048) {
        const int n = (int)min(o.size - at, (uint64_t)8);
        float g[8];
        load_eight<DTYPE>(p.g[which], at, n, g);
        if (o.update) {
            float v[8];
            load8<TQ_F32>(p.v[which] + at, n, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = o.momentum * v[j] + g[j];
                g[j] = o.nesterov ? g[j] + o.momentum * v[j] : v[j];
            }
            store8<TQ_F32>(p.v_out[which] + at, n, v);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (j < n) sum += (double)g[j] * (double)g[j];
    }
    part[threadIdx.x] = sum;
    __syncthreads();
    for (uint32_t half = 128; half; half /= 2) {
        if (threadIdx.x < half) part[threadIdx.x] += part[threadIdx.x + half];
        __syncthreads();
    }
    if (threadIdx.x == 0) reinterpret_cast<double*>(o.workspace + which * o.stride)[block] = part[0];
}

// Where 8 elements from column `col` on lie in a row.
template <int KIND>
__device__ __forceinline__ uint64_t in_row(uint32_t col)
{
    return KIND == kHalf ? (uint64_t)col * 2 : (uint64_t)(col / 16) * 64 + col % 16 * 2;
}

__device__ __forceinline__ float low_part(float v, _Float16 high) { return v - (float)high; }

template <int KIND>
__device__ __forceinline__ void put8(char* row, uint32_t col, const float (&v)[8])
{
    tile_f16x8 high, low;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        high[e] = (_Float16)v[e];
        low[e] = (_Float16)low_part(v[e], high[e]);
    }
    char* to = row + in_row<KIND>(col);
    *reinterpret_cast<tile_f16x8*>(to) = high;
    if constexpr (KIND == kHalfPair) *reinterpret_cast<tile_f16x8*>(to + 32) = low;
}

// 8 elements of a row in each lane to columns: lanes whose rows are 4 in a row change elements, after which a lane holds 4 rows of the
// two columns c and c + 4, c = its row % 4.  8 bytes at a time 32 rows of a column are stored by 8 lanes; element by element it took 64.
__device__ __forceinline__ void turn4(const tile_f16x8& v, uint32_t row, u32x2 (&out)[2])
{
    const u32x4 w = __builtin_bit_cast(u32x4, v);
    const uint32_t halves = row & 1 ? 0x03020706u : 0x05040100u;   // of two words: those of this lane's column, the lower row's first
    u32x4 t;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t other = dpp_move<0xB1>(w[k]);               // of lane ^ 1
        t[k] = __builtin_amdgcn_perm(other, w[k], halves);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t give = row & 2 ? t[2 * k] : t[2 * k + 1], keep = row & 2 ? t[2 * k + 1] : t[2 * k];
        const uint32_t got = dpp_move<0x4E>(give);                 // of lane ^ 2
        out[k] = row & 2 ? u32x2{got, keep} : u32x2{keep, got};
    }
}

// The same 8 elements of 64 lanes' rows at their places in the transposed matrix, whose rows are `to_row` bytes, `cols` of them there.
template <int KIND>
__device__ __forceinline__ void put_turned(char* to, uint64_t to_row, uint32_t row, uint32_t col, uint32_t cols, const tile_f16x8& high, const tile_f16x8& low)
{
    u32x2 h[2], l[2];
    turn4(high, row, h);
    if constexpr (KIND == kHalfPair) turn4(low, row, l);
    if (in_row<KIND>(row & ~3u) >= to_row) return;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const uint32_t c = col + (row & 3) + 4 * k;
        if (c >= cols) continue;
        char* at = to + c * to_row + in_row<KIND>(row & ~3u);
        *reinterpret_cast<u32x2*>(at) = h[k];
        if constexpr (KIND == kHalfPair) *reinterpret_cast<u32x2*>(at + 32) = l[k];
    }
}

template <int KIND>
__device__ __forceinline__ void get8(const char* row, uint32_t col, float (&v)[8])
{
    const char* from = row + in_row<KIND>(col);
    const tile_f16x8 high = *reinterpret_cast<const tile_f16x8*>(from);
    if constexpr (KIND == kHalfPair) {
        const tile_f16x8 low = *reinterpret_cast<const tile_f16x8*>(from + 32);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)high[e] + (float)low[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (float)high[e];
    }
}

constexpr __host__ __device__ uint32_t groups_of(int kind, uint32_t n) { return (n + in_group(kind) - 1) / in_group(kind); }

// U / (|U| + eps) both ways, 64 x 64 elements a workgroup, zeros behind the rows' ends.  Memory: four of 1024 x 4096 as pairs 57 us, 4.7 TB/s.
template <int DTYPE, int KIND>
__global__ __launch_bounds__(256) void orth_begin_kernel(OrthPointers p, OrthArgs o)
{
    __shared__ double part[256];
    __shared__ float square[64][65];
    const uint32_t which = blockIdx.y;
    uint32_t tile;
    if (!tile_number(linear_block(), o.tiles, tile)) return;
    char* ws = o.workspace + which * o.stride;
    part[threadIdx.x] = threadIdx.x < o.parts ? reinterpret_cast<const double*>(ws)[threadIdx.x] : 0.0;
    __syncthreads();
    for (uint32_t half = 128; half; half /= 2) {
        if (threadIdx.x < half) part[threadIdx.x] += part[threadIdx.x + half];
        __syncthreads();
    }
    const double factor = (double)kUnit / (sqrt(part[0]) + (double)o.eps);
    const uint32_t row0 = tile / o.tiles_x * 64, col0 = tile % o.tiles_x * 64;
    char* direct = ws + (o.flip ? o.xt : o.x);
    char* turned = ws + (o.flip ? o.x : o.xt);
    const uint64_t direct_row = (uint64_t)groups_of(KIND, o.cols) * 128, turned_row = (uint64_t)groups_of(KIND, o.rows) * 128;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t r = threadIdx.x / 8 + i * 32, c = threadIdx.x % 8 * 8, row = row0 + r, col = col0 + c;
        float u[8] = {};
        if (row < o.rows && col < o.cols) {
            const uint64_t at = (uint64_t)row * o.cols + col;
            const int n = (int)min(o.cols - col, 8u);
            if (o.update) load8<TQ_F32>(p.v_out[which] + at, n, u);
            if (!o.update || o.nesterov) {
                float g[8];
                load_eight<DTYPE>(p.g[which], at, n, g);
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = o.update ? g[j] + o.momentum * u[j] : g[j];
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) u[j] = j < n ? (float)((double)u[j] * factor) : 0.0f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) square[r][c + j] = u[j];
        if (row < o.rows && in_row<KIND>(col) < direct_row) put8<KIND>(direct + row * direct_row, col, u);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t r = threadIdx.x / 8 + i * 32, c = threadIdx.x % 8 * 8, row = col0 + r, col = row0 + c;
        float u[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) u[j] = square[c + j][r];
        if (row < o.cols && in_row<KIND>(col) < turned_row) put8<KIND>(turned + row * turned_row, col, u);
    }
}

enum { kGram, kPolynomial, kApply };

struct StepArgs {
    char* workspace;
    uint64_t stride, from_a, from_b, to, to_turned;    // places in a matrix's part of the workspace
    uint32_t m, n, k;                          // of this product
    uint32_t tiles_x, tiles_y, tiles, count;   // tiles of each of `count` matrices
    float a, b, c;
};

// This workgroup's matrix and tile.  A die takes a run of them, of one matrix after the other: spread over the dies each die's cache would hold
// something of all matrices (four of 1024 x 4096, pairs, X X^T).
__device__ __forceinline__ bool find_tile(const StepArgs& s, uint32_t& which, uint32_t& tile)
{
    if (!tile_number(linear_block(), s.tiles * s.count, tile)) return false;
    which = __builtin_amdgcn_readfirstlane(tile / s.tiles);
    tile -= which * s.tiles;
    return true;
}

// One of a step's first products, or its last where another step follows.  4096 x 4096 in binary16: 77 to 83, 80 to 85 and 126 to 141
// us, the matrix units busy 51, 49 and 56 % of the clocks; as pairs 192, 194 and 315 us, busy 67, 65 and 74 %.  Each is one round of tiles, so that nothing overlaps its first requests and last stores.
template <class S, int WHAT>
__global__ __launch_bounds__(S::kThreads, S::kOnSimd) void orth_step_kernel(StepArgs s)
{
    extern __shared__ char lds[];
    constexpr int KIND = S::KIND;
    uint32_t which, tile, ty, tx;
    if (!find_tile(s, which, tile)) return;
    if (WHAT == kApply) tile_place(tile, s.tiles_y, s.tiles_x, ty, tx);
    else tile_place_below(tile, s.tiles_y, ty, tx);
    char* ws = s.workspace + which * s.stride;
    const uint32_t groups = groups_of(KIND, s.k), row0 = ty * S::BM, col0 = tx * S::BN;
    typename S::Sums acc[S::kFragsM][S::kFragsN];
    const TileOperands operands = {reinterpret_cast<uint8_t*>(ws + s.from_a), reinterpret_cast<uint8_t*>(ws + s.from_b), s.m, s.n, groups, 0, groups};
    tile_sums<S>(operands, row0, col0, lds, acc);
    const uint64_t to_row = (uint64_t)groups_of(KIND, s.n) * 128, turned_row = (uint64_t)groups_of(KIND, s.m) * 128;
    const bool turn = WHAT == kApply || ty != tx;
    tile_chunks<S>(acc, row0, col0, [&](uint32_t row, uint32_t col, const float (&sums)[8]) {
        float v[8];
        const bool there = row < s.m && in_row<KIND>(col) < to_row;
        if constexpr (WHAT == kPolynomial) {
            float gram[8] = {};
            if (there) get8<KIND>(ws + s.from_a + row * to_row, col, gram);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf(s.c, sums[e] * (1.0f / kUnit), fmaf(s.b, gram[e], row == col + e ? s.a * kUnit : 0.0f));
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = sums[e] * (1.0f / kUnit);
        }
        tile_f16x8 high, low;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = row < s.m && col + e < s.n ? v[e] : 0.0f;
            high[e] = (_Float16)v[e];
            low[e] = (_Float16)low_part(v[e], high[e]);
        }
        if (there) {
            char* to = ws + s.to + row * to_row + in_row<KIND>(col);
            *reinterpret_cast<tile_f16x8*>(to) = high;
            if constexpr (KIND == kHalfPair) *reinterpret_cast<tile_f16x8*>(to + 32) = low;
        }
        if (turn) put_turned<KIND>(ws + s.to_turned, turned_row, row, col, s.n, high, low);
    });
}

struct EndArgs {
    void* out[TQ_ORTH_MAX_COUNT];              // or theta'
    const float* theta[TQ_ORTH_MAX_COUNT];
    StepArgs s;
    float eta, scale, weight_decay;
};

// The last product, rows x cols as the caller has them; theta in place of an output's type: the new parameters.
template <class S, int DTYPE, bool UPDATE>
__global__ __launch_bounds__(S::kThreads, S::kOnSimd) void orth_end_kernel(EndArgs a)
{
    extern __shared__ char lds[];
    const StepArgs& s = a.s;
    uint32_t which, tile, ty, tx;
    if (!find_tile(s, which, tile)) return;
    tile_place(tile, s.tiles_y, s.tiles_x, ty, tx);
    const uint32_t groups = groups_of(S::KIND, s.k);
    const char* ws = s.workspace + which * s.stride;
    typename S::Sums acc[S::kFragsM][S::kFragsN];
    const TileOperands operands = {reinterpret_cast<const uint8_t*>(ws + s.from_a), reinterpret_cast<const uint8_t*>(ws + s.from_b), s.m, s.n, groups, 0, groups};
    tile_sums<S>(operands, ty * S::BM, tx * S::BN, lds, acc);
    tile_chunks<S>(acc, ty * S::BM, tx * S::BN, [&](uint32_t row, uint32_t col, const float (&sums)[8]) {
        if (row >= s.m || col >= s.n) return;
        const int n = (int)min(s.n - col, 8u);
        const uint64_t at = (uint64_t)row * s.n + col;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = sums[e] * (1.0f / (kUnit * kUnit));
        if constexpr (UPDATE) {
            float theta[8];
            load8<TQ_F32>(a.theta[which] + at, n, theta);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = theta[e] - a.eta * (a.scale * v[e] + a.weight_decay * theta[e]);
        }
        store8<DTYPE>(static_cast<typename Element<DTYPE>::type*>(a.out[which]) + at, n, v);
    });
}

// Small matrices: a workgroup has X, X^T, A and B of one in its LDS and takes all steps in one launch, where the products of the kernels above
// would each be a launch of a few us.  Rows are 16 bytes longer than their elements, so that 16 of them lie in different banks; everything is
// padded to 32 with zeros.  Us, by the kernels above / this one: 64 x 256 61 / 31, 128 x 128 66 / 34, 128 x 160 67 / 40, 32 x 32 pairs 53 / 15,
// 64 x 128 pairs 78 / 29, 32 x 900 80 / 51 (the less of two runs), 16 updates of 64 x 128 120 / 83.  Chains of LDS reads and matrix instructions bound it: its wavefronts
// wait for half of the time.
struct SmallArgs {
    void* out[TQ_ORTH_MAX_COUNT];
    const float* theta[TQ_ORTH_MAX_COUNT];
    float coefficients[TQ_ORTH_MAX_STEPS][3];
    uint32_t rows, cols;
    int dtype, out_dtype, steps, nesterov;
    float momentum, eps, eta, scale, weight_decay;
};

typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
constexpr uint32_t kSmallWaves = 16, kSmallFrags = 2;              // 32 x 32 outputs that a wavefront may hold

struct SmallPlan {
    uint32_t r, c, row_x, row_t, xt, a, b, bytes;                  // row_t: of X^T, A and B; bytes: of all four, once for each number of a pair
};
__host__ __device__ inline SmallPlan small_plan(uint64_t rows, uint64_t cols)
{
    SmallPlan p;
    p.r = (uint32_t)(((rows < cols ? rows : cols) + 31) / 32 * 32);
    p.c = (uint32_t)(((rows < cols ? cols : rows) + 31) / 32 * 32);
    p.row_x = p.c * 2 + 16;
    p.row_t = p.r * 2 + 16;
    p.xt = p.r * p.row_x;
    p.a = p.xt + p.c * p.row_t;
    p.b = p.a + p.r * p.row_t;
    p.bytes = p.b + p.r * p.row_t;
    return p;
}
constexpr uint32_t kSmallBytes = (156 << 10);

bool is_small(uint64_t rows, uint64_t cols, int kind)
{
    const uint64_t r = rows < cols ? rows : cols, c = rows < cols ? cols : rows;
    if (r > 128 || c > 4096) return false;
    const SmallPlan p = small_plan(rows, cols);
    return p.bytes * (kind == kHalfPair ? 2u : 1u) <= kSmallBytes && p.r / 32 * (p.c / 32) <= kSmallWaves * kSmallFrags;
}

template <int KIND, bool UPDATE>
__global__ __launch_bounds__(kSmallWaves * 64) void orth_small_kernel(OrthPointers q, SmallArgs s)
{
    using P = TileProduct<KIND>;
    extern __shared__ char lds[];
    __shared__ double part[kSmallWaves];
    constexpr uint32_t kAll = kSmallWaves * 64;
    const uint32_t which = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t me = lane;
    if (blockIdx.x) return;
    const SmallPlan p = small_plan(s.rows, s.cols);
    const uint32_t size = s.rows * s.cols;
    const bool flip = s.rows > s.cols;
    char *x = lds, *xt = lds + p.xt, *a = lds + p.a, *b = lds + p.b;
    for (uint32_t i = threadIdx.x * 16; i < p.bytes * (KIND == kHalfPair ? 2 : 1); i += kAll * 16) *reinterpret_cast<u32x4*>(lds + i) = u32x4{0, 0, 0, 0};
    // 8 elements of U from `at` on, and of the new momentum
    auto load = [&](uint32_t at, float (&u)[8], float (&v)[8]) {
        const int n = (int)min(size - at, 8u);
        if (s.dtype == TQ_F32) load_eight<TQ_F32>(q.g[which], at, n, u);
        else if (s.dtype == TQ_BF16) load_eight<TQ_BF16>(q.g[which], at, n, u);
        else load_eight<TQ_F16>(q.g[which], at, n, u);
        if constexpr (UPDATE) {
            load8<TQ_F32>(q.v[which] + at, n, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                v[j] = s.momentum * v[j] + u[j];
                u[j] = s.nesterov ? u[j] + s.momentum * v[j] : v[j];
            }
        }
        return n;
    };
    auto put = [&](char* array, uint32_t stride, uint32_t row, uint32_t col, float v) {
        char* to = array + row * stride + col * 2;
        const _Float16 high = (_Float16)v;
        *reinterpret_cast<_Float16*>(to) = high;
        if constexpr (KIND == kHalfPair) *reinterpret_cast<_Float16*>(to + p.bytes) = (_Float16)low_part(v, high);
    };
    double sum = 0.0, factor = 0.0;                                // of squares, in binary64
#pragma nounroll
    for (int pass = 0; pass < 2; ++pass) {                         // one code for both: what is not in the instruction cache yet is waited for
#pragma nounroll
        for (uint32_t at = threadIdx.x * 8; at < size; at += kAll * 8) {
            float u[8], v[8];
            const int n = load(at, u, v);
            if (pass == 0) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j < n) sum += (double)u[j] * (double)u[j];
                continue;
            }
            if constexpr (UPDATE) store8<TQ_F32>(q.v_out[which] + at, n, v);
            uint32_t row = at / s.cols, col = at % s.cols;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j >= n) break;
                const float held = (float)((double)u[j] * factor);
                put(flip ? xt : x, flip ? p.row_t : p.row_x, row, col, held);
                put(flip ? x : xt, flip ? p.row_x : p.row_t, col, row, held);
                if (++col == s.cols) {
                    col = 0;
                    ++row;
                }
            }
        }
        if (pass == 0) {
#pragma unroll
            for (int d = 32; d; d /= 2) sum += __shfl_xor(sum, d);
            if (lane == 0) part[wave] = sum;
        }
        __syncthreads();
        if (pass == 0) {
            sum = 0.0;
#pragma unroll
            for (uint32_t w = 0; w < kSmallWaves; ++w) sum += part[w];
            factor = (double)kUnit / (sqrt(sum) + (double)s.eps);
        }
    }

    // 32 x 32 outputs of rows of two arrays; a lane's 16 as in tiles.  32 of k at a time, the next 32 on their way.
    auto product = [&](const char* from_a, const char* from_b, uint32_t stride, uint32_t row_a, uint32_t row_b, uint32_t k) {
        constexpr int kNumbers = KIND == kHalfPair ? 2 : 1;
        typename P::Sums acc;
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[e] = 0.0f;
        const char* pa = from_a + (row_a + (me & 31)) * stride + (me >> 5) * 16;
        const char* pb = from_b + (row_b + (me & 31)) * stride + (me >> 5) * 16;
        tile_i32x4 va[2][kNumbers], vb[2][kNumbers];
        auto load = [&](uint32_t i) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < kNumbers; ++n) {
                    va[h][n] = *reinterpret_cast<const tile_i32x4*>(pa + n * p.bytes + i + h * 32);
                    vb[h][n] = *reinterpret_cast<const tile_i32x4*>(pb + n * p.bytes + i + h * 32);
                }
        };
        load(0);
        for (uint32_t i = 0; i < k * 2; i += 64) {
            tile_i32x4 a[2][kNumbers], b[2][kNumbers];
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int n = 0; n < kNumbers; ++n) {
                    a[h][n] = va[h][n];
                    b[h][n] = vb[h][n];
                }
            load(i + 64 < k * 2 ? i + 64 : 0);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                acc = P::step(b[h][0], a[h][0], acc);
                if constexpr (KIND == kHalfPair) {
                    acc = P::step(b[h][0], a[h][1], acc);
                    acc = P::step(b[h][1], a[h][0], acc);
                }
            }
        }
        return acc;
    };
    auto row_of = [&](uint32_t row0) { return row0 + (me & 31); };
    auto col_of = [&](uint32_t col0, int e) { return col0 + (e / 4) * 8 + (me >> 5) * 4 + e % 4; };
    // Into an array, 4 columns at a time.
    auto place = [&](char* to, uint32_t stride, uint32_t row0, uint32_t col0, const typename P::Sums& v) {
#pragma unroll
        for (int e = 0; e < 16; e += 4) {
            f16x4 high, low;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                high[i] = (_Float16)v[e + i];
                low[i] = (_Float16)low_part(v[e + i], high[i]);
            }
            char* at = to + row_of(row0) * stride + col_of(col0, e) * 2;
            *reinterpret_cast<f16x4*>(at) = high;
            if constexpr (KIND == kHalfPair) *reinterpret_cast<f16x4*>(at + p.bytes) = low;
        }
    };
    const uint32_t down = p.r / 32, across = p.c / 32;
    for (int step = 0; step < s.steps; ++step) {
        const float fa = s.coefficients[step][0], fb = s.coefficients[step][1], fc = s.coefficients[step][2];
        for (uint32_t at = wave; at < down * down; at += kSmallWaves) {
            const uint32_t row0 = at % down * 32, col0 = at / down * 32;
            asm volatile("" : "+v"(me));
            typename P::Sums v = product(x, x, p.row_x, row0, col0, p.c);
#pragma unroll
            for (int e = 0; e < 16; ++e) v[e] *= 1.0f / kUnit;
            place(a, p.row_t, row0, col0, v);
        }
        __syncthreads();
        for (uint32_t at = wave; at < down * down; at += kSmallWaves) {
            const uint32_t row0 = at % down * 32, col0 = at / down * 32;
            asm volatile("" : "+v"(me));
            typename P::Sums v = product(a, a, p.row_t, row0, col0, p.r);
#pragma unroll
            for (int e = 0; e < 16; e += 4) {
                const char* from = a + row_of(row0) * p.row_t + col_of(col0, e) * 2;
                f16x4 high = *reinterpret_cast<const f16x4*>(from), low = {};
                if constexpr (KIND == kHalfPair) low = *reinterpret_cast<const f16x4*>(from + p.bytes);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float gram = KIND == kHalfPair ? (float)high[i] + (float)low[i] : (float)high[i];
                    v[e + i] = fmaf(fc, v[e + i] * (1.0f / kUnit), fb * gram);
                }
            }
            if (row0 == col0) {
#pragma unroll
                for (int e = 0; e < 16; ++e) v[e] += row_of(0) == col_of(0, e) ? fa * kUnit : 0.0f;
            }
            place(b, p.row_t, row0, col0, v);
        }
        __syncthreads();
        asm volatile("" : "+v"(me));                               // places are found where they are used, not kept from step to step
        typename P::Sums held[kSmallFrags];
#pragma unroll
        for (uint32_t f = 0; f < kSmallFrags; ++f) {
            const uint32_t at = wave + f * kSmallWaves;
            if (at < down * across) held[f] = product(b, xt, p.row_t, at % down * 32, at / down * 32, p.r);
        }
        __syncthreads();
        const bool end = step + 1 == s.steps;
#pragma unroll
        for (uint32_t f = 0; f < kSmallFrags; ++f) {
            const uint32_t at = wave + f * kSmallWaves, row0 = at % down * 32, col0 = at / down * 32;
            if (at >= down * across) continue;
            asm volatile("" : "+v"(me));
            if (end) {                                             // as binary32, in place of everything
#pragma unroll
                for (int e = 0; e < 16; ++e) reinterpret_cast<float*>(lds)[row_of(row0) * p.c + col_of(col0, e)] = held[f][e] * (1.0f / (kUnit * kUnit));
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) held[f][e] *= 1.0f / kUnit;
                place(x, p.row_x, row0, col0, held[f]);
#pragma unroll
                for (int e = 0; e < 16; ++e) put(xt, p.row_t, col_of(col0, e), row_of(row0), held[f][e]);
            }
        }
        __syncthreads();
    }
#pragma nounroll
    for (uint32_t at = threadIdx.x; at < size; at += kAll) {
        const uint32_t i = at / s.cols, j = at - i * s.cols;
        float o = reinterpret_cast<const float*>(lds)[flip ? j * p.c + i : i * p.c + j];
        if constexpr (UPDATE) {
            const float theta = s.theta[which][at];
            static_cast<float*>(s.out[which])[at] = theta - s.eta * (s.scale * o + s.weight_decay * theta);
        } else if (s.out_dtype == TQ_F32) {
            static_cast<float*>(s.out[which])[at] = o;
        } else {
            static_cast<uint16_t*>(s.out[which])[at] = s.out_dtype == TQ_BF16 ? Element<TQ_BF16>::store(o) : Element<TQ_F16>::store(o);
        }
    }
}

// A matrix's part of the workspace.
struct Layout {
    uint64_t x, xt[2], a, b, stride;
};
Layout layout(uint64_t rows, uint64_t cols, int kind)
{
    const uint64_t r = rows < cols ? rows : cols, c = rows < cols ? cols : rows;
    auto bytes = [&](uint64_t n, uint64_t k) { return n * ((k + in_group(kind) - 1) / in_group(kind)) * 128; };
    Layout l;
    l.x = kParts * sizeof(double);
    l.xt[0] = l.x + bytes(r, c);
    l.xt[1] = l.xt[0] + bytes(c, r);
    l.a = l.xt[1] + bytes(c, r);
    l.b = l.a + bytes(r, r);
    l.stride = l.b + bytes(r, r);
    return l;
}

struct OrthCall {
    const void* const* g;
    const float* const* v;
    float* const* v_out;
    const float* const* theta;
    void* const* out;
    int count, dtype, out_dtype, steps, nesterov;
    uint64_t rows, cols;
    const float* coefficients;
    float eps, eta, momentum, weight_decay, scale;
    char* workspace;
};

template <int KIND, typename F>
hipError_t by_shape(const StepArgs& s, bool below, int count, F f)
{
    switch (shape_of(KIND, s.m, s.n, s.k, below, (uint64_t)count)) {
        case k256: return f(TileShape<KIND, 256, 256, 2, 4, 2>{});
        case k192: return f(TileShape<KIND, 192, 192, 2, 6, 3>{});
        case k128: return f(TileShape<KIND, 128, 128, 2, 4, 2>{});
        case k128Alone: return f(TileShape<KIND, 128, 128, 2, 4, 5>{});
        case k64: return f(TileShape<KIND, 64, 64, 2, 2, 3>{});
    }
    return hipErrorInvalidValue;
}

template <class S>
bool set_tiles(StepArgs& s, bool below, int count, dim3& grid)
{
    const uint64_t tiles = tiles_of(s.m, s.n, S::BM, below);
    s.tiles_x = (s.n + S::BN - 1) / S::BN;
    s.tiles_y = (s.m + S::BM - 1) / S::BM;
    s.tiles = (uint32_t)tiles;
    s.count = (uint32_t)count;
    return tiles * count <= 0xFFFFFFF0ull && fold_grid((tiles * count + 7) / 8 * 8, S::kThreads, 1, grid);
}

template <int KIND, int WHAT>
hipError_t launch_step(StepArgs s, int count, hipStream_t st)
{
    return by_shape<KIND>(s, WHAT != kApply, count, [&](auto shape) -> hipError_t {
        using S = decltype(shape);
        dim3 grid;
        if (!set_tiles<S>(s, WHAT != kApply, count, grid)) return hipErrorInvalidValue;
        orth_step_kernel<S, WHAT><<<grid, S::kThreads, S::kBytes, st>>>(s);
        return hipGetLastError();
    });
}

template <int KIND, int DTYPE, bool UPDATE>
hipError_t launch_end(EndArgs& a, int count, hipStream_t st)
{
    return by_shape<KIND>(a.s, false, count, [&](auto shape) -> hipError_t {
        using S = decltype(shape);
        dim3 grid;
        if (!set_tiles<S>(a.s, false, count, grid)) return hipErrorInvalidValue;
        orth_end_kernel<S, DTYPE, UPDATE><<<grid, S::kThreads, S::kBytes, st>>>(a);
        return hipGetLastError();
    });
}

template <int KIND>
hipError_t launch_begin(const OrthCall& q, const OrthPointers& p, OrthArgs& o, hipStream_t st)
{
    dim3 norm_grid, grid;
    o.parts = (uint32_t)((o.size + 8191) / 8192 < kParts ? (o.size + 8191) / 8192 : kParts);
    const uint64_t x = ((uint64_t)o.cols + 63) / 64, tiles = x * (((uint64_t)o.rows + 63) / 64);
    o.tiles_x = (uint32_t)x;
    o.tiles = (uint32_t)tiles;
    if (!fold_grid(o.parts, 256, (unsigned)q.count, norm_grid) || tiles > 0xFFFFFFF0ull ||
        !fold_grid((tiles + 7) / 8 * 8, 256, (unsigned)q.count, grid))
        return hipErrorInvalidValue;
    auto as = [&](auto D) {
        constexpr int kD = decltype(D)::value;
        orth_norm_kernel<kD><<<norm_grid, 256, 0, st>>>(p, o);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        orth_begin_kernel<kD, KIND><<<grid, 256, 0, st>>>(p, o);
        return hipGetLastError();
    };
    if (q.dtype == TQ_F32) return as(std::integral_constant<int, TQ_F32>{});
    return q.dtype == TQ_BF16 ? as(std::integral_constant<int, TQ_BF16>{}) : as(std::integral_constant<int, TQ_F16>{});
}

constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};

template <int KIND>
hipError_t launch_small(const OrthCall& q, const OrthPointers& p, hipStream_t st)
{
    SmallArgs s = {};
    for (int i = 0; i < q.count; ++i) {
        s.out[i] = q.out[i];
        s.theta[i] = q.theta ? q.theta[i] : nullptr;
    }
    for (int i = 0; i < q.steps; ++i)
        for (int j = 0; j < 3; ++j) s.coefficients[i][j] = q.coefficients ? q.coefficients[3 * i + j] : kQuintic[j];
    s.rows = (uint32_t)q.rows;
    s.cols = (uint32_t)q.cols;
    s.dtype = q.dtype;
    s.out_dtype = q.out_dtype;
    s.steps = q.steps;
    s.nesterov = q.nesterov;
    s.momentum = q.momentum;
    s.eps = q.eps;
    s.eta = q.eta;
    s.scale = q.scale;
    s.weight_decay = q.weight_decay;
    const uint32_t bytes = small_plan(q.rows, q.cols).bytes * (KIND == kHalfPair ? 2 : 1);
    if (q.theta) orth_small_kernel<KIND, true><<<dim3(1, q.count), kSmallWaves * 64, bytes, st>>>(p, s);
    else orth_small_kernel<KIND, false><<<dim3(1, q.count), kSmallWaves * 64, bytes, st>>>(p, s);
    return hipGetLastError();
}

template <int KIND>
hipError_t launch_orth(const OrthCall& q, hipStream_t st)
{
    const Layout l = layout(q.rows, q.cols, KIND);
    const bool flip = q.rows > q.cols;
    const uint32_t r = (uint32_t)(flip ? q.cols : q.rows), c = (uint32_t)(flip ? q.rows : q.cols);
    OrthPointers p = {};
    for (int i = 0; i < q.count; ++i) {
        p.g[i] = q.g[i];
        p.v[i] = q.v ? q.v[i] : nullptr;
        p.v_out[i] = q.v ? q.v_out[i] : nullptr;
    }
    if (is_small(q.rows, q.cols, KIND)) return launch_small<KIND>(q, p, st);
    OrthArgs o = {};
    o.workspace = q.workspace;
    o.stride = l.stride;
    o.x = l.x;
    o.xt = l.xt[0];
    o.size = q.rows * q.cols;
    o.rows = (uint32_t)q.rows;
    o.cols = (uint32_t)q.cols;
    o.momentum = q.momentum;
    o.eps = q.eps;
    o.nesterov = q.nesterov;
    o.update = q.v != nullptr;
    o.flip = flip;
    hipError_t e = launch_begin<KIND>(q, p, o, st);
    StepArgs s = {};
    s.workspace = q.workspace;
    s.stride = l.stride;
    for (int step = 0; step < q.steps && e == hipSuccess; ++step) {
        const float* f = q.coefficients ? q.coefficients + 3 * step : kQuintic;
        s.a = f[0];
        s.b = f[1];
        s.c = f[2];
        const uint64_t xt = l.xt[step & 1];
        s.m = s.n = r;
        s.k = c;
        s.from_a = s.from_b = l.x;
        s.to = s.to_turned = l.a;
        if ((e = launch_step<KIND, kGram>(s, q.count, st)) != hipSuccess) return e;
        s.k = r;
        s.from_a = s.from_b = l.a;
        s.to = s.to_turned = l.b;
        if ((e = launch_step<KIND, kPolynomial>(s, q.count, st)) != hipSuccess) return e;
        if (step + 1 < q.steps) {
            s.n = c;
            s.from_a = l.b;
            s.from_b = xt;
            s.to = l.x;
            s.to_turned = l.xt[~step & 1];
            e = launch_step<KIND, kApply>(s, q.count, st);
            continue;
        }
        EndArgs a = {};
        for (int i = 0; i < q.count; ++i) {
            a.out[i] = q.out[i];
            a.theta[i] = q.theta ? q.theta[i] : nullptr;
        }
        a.s = s;
        a.s.m = o.rows;
        a.s.n = o.cols;
        a.s.from_a = flip ? xt : l.b;
        a.s.from_b = flip ? l.b : xt;
        a.eta = q.eta;
        a.scale = q.scale;
        a.weight_decay = q.weight_decay;
        if (q.theta) e = launch_end<KIND, TQ_F32, true>(a, q.count, st);
        else if (q.out_dtype == TQ_F32) e = launch_end<KIND, TQ_F32, false>(a, q.count, st);
        else if (q.out_dtype == TQ_BF16) e = launch_end<KIND, TQ_BF16, false>(a, q.count, st);
        else e = launch_end<KIND, TQ_F16, false>(a, q.count, st);
    }
    return e;
}

}  // namespace
}  // namespace tq

uint64_t tq_orth_workspace_bytes_impl(uint64_t rows, uint64_t cols, int count, int precision)
{
    return tq::layout(rows, cols, precision == TQ_ORTH_HALF ? tq::kHalf : tq::kHalfPair).stride * (uint64_t)count;
}

hipError_t tq_launch_orth(const void* const* g, int count, int dtype, uint64_t rows, uint64_t cols, float eta, float momentum, int nesterov,
                          float weight_decay, float scale, int steps, const float* coefficients, int precision, float eps,
                          const float* const* v, float* const* v_out, const float* const* theta, void* const* out, int out_dtype,
                          void* workspace, hipStream_t st)
{
    const tq::OrthCall q = {g, v, v_out, theta, out, count, dtype, out_dtype, steps, nesterov, rows, cols, coefficients,
                            eps, eta, momentum, weight_decay, scale, static_cast<char*>(workspace)};
    return precision == TQ_ORTH_HALF ? tq::launch_orth<tq::kHalf>(q, st) : tq::launch_orth<tq::kHalfPair>(q, st);
}
