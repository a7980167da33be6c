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

// Sums of squares in binary64, and the new momentum.
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

template <int KIND>
__device__ __forceinline__ void put1(char* row, uint32_t col, float v)
{
    char* to = row + in_row<KIND>(col);
    const _Float16 high = (_Float16)v;
    *reinterpret_cast<_Float16*>(to) = high;
    if constexpr (KIND == kHalfPair) *reinterpret_cast<_Float16*>(to + 32) = (_Float16)low_part(v, high);
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

// U / (|U| + eps) both ways, 64 x 64 elements a workgroup, zeros behind the rows' ends.
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
    uint32_t tiles_x, tiles_y, tiles;
    float a, b, c;
};

// One of a step's first products, or its last where another step follows.
template <class S, int WHAT>
__global__ __launch_bounds__(S::kThreads, S::kOnSimd) void orth_step_kernel(StepArgs s)
{
    extern __shared__ char lds[];
    constexpr int KIND = S::KIND;
    uint32_t tile, ty, tx;
    if (!tile_number(linear_block(), s.tiles, tile)) return;
    if (WHAT == kApply) tile_place(tile, s.tiles_y, s.tiles_x, ty, tx);
    else tile_place_below(tile, ty, tx);
    char* ws = s.workspace + blockIdx.y * s.stride;
    const uint32_t groups = groups_of(KIND, s.k), row0 = ty * S::BM, col0 = tx * S::BN;
    typename S::Sums acc[S::kFragsM][S::kFragsN];
    const TileOperands operands = {reinterpret_cast<uint8_t*>(ws + s.from_a), reinterpret_cast<uint8_t*>(ws + s.from_b), s.m, s.n, groups, 0, groups};
    if (!tile_sums<S>(operands, row0, col0, lds, acc)) return;
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
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = row < s.m && col + e < s.n ? v[e] : 0.0f;
        if (there) put8<KIND>(ws + s.to + row * to_row, col, v);
        if (turn && in_row<KIND>(row) < turned_row) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < s.n) put1<KIND>(ws + s.to_turned + (col + e) * turned_row, row, v[e]);
        }
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
    uint32_t tile, ty, tx;
    if (!tile_number(linear_block(), s.tiles, tile)) return;
    tile_place(tile, s.tiles_y, s.tiles_x, ty, tx);
    const uint32_t which = blockIdx.y, groups = groups_of(S::KIND, s.k);
    const char* ws = s.workspace + which * s.stride;
    typename S::Sums acc[S::kFragsM][S::kFragsN];
    const TileOperands operands = {reinterpret_cast<const uint8_t*>(ws + s.from_a), reinterpret_cast<const uint8_t*>(ws + s.from_b), s.m, s.n, groups, 0, groups};
    if (!tile_sums<S>(operands, ty * S::BM, tx * S::BN, lds, acc)) return;
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

// Tiles of a product: their sides, the time in ns that a group of k took while 1, 2, .. of them, as many as fit, were at work on every compute
// unit, and what a round of them costs beside that.
enum Shape { k256, k192, k128, k64, k64InParts };
struct Pace {
    Shape shape;
    uint64_t side;
    uint32_t ns[3], round;
};
constexpr Pace kPaces[2][5] = {
    {{k256, 256, {1553, 0, 0}, 12000}, {k192, 192, {943, 0, 0}, 9000}, {k128, 128, {580, 925, 0}, 8000}, {k64, 64, {262, 375, 560}, 4000}, {k64InParts, 64, {140, 0, 0}, 5000}},
    {{k256, 256, {2200, 0, 0}, 12000}, {k192, 192, {1300, 0, 0}, 9000}, {k128, 128, {700, 1200, 0}, 8000}, {k64, 64, {300, 420, 620}, 4000}, {k64InParts, 64, {160, 0, 0}, 5000}}};

uint64_t tiles_of(uint64_t m, uint64_t n, uint64_t side, bool below)
{
    const uint64_t y = (m + side - 1) / side, x = (n + side - 1) / side;
    return below ? y * (y + 1) / 2 : x * y;
}

Shape shape_of(int kind, uint64_t m, uint64_t n, uint64_t k, bool below, uint64_t count)
{
    const Pace* best = nullptr;
    uint64_t least = ~0ull;
    for (const Pace& p : kPaces[kind == kHalfPair]) {
        const uint64_t each = (tiles_of(m, n, p.side, below) * count + kComputeUnits - 1) / kComputeUnits, groups = (k + in_group(kind) - 1) / in_group(kind);
        const uint64_t fit = p.ns[2] ? 3 : p.ns[1] ? 2 : 1, rest = each % fit;
        const uint64_t t = each / fit * (p.ns[fit - 1] * groups + p.round) + (rest ? p.ns[rest - 1] * groups + p.round : 0);
        if (t < least) {
            least = t;
            best = &p;
        }
    }
    return best->shape;
}

template <int KIND, typename F>
hipError_t by_shape(const StepArgs& s, bool below, int count, F f)
{
    switch (shape_of(KIND, s.m, s.n, s.k, below, (uint64_t)count)) {
        case k256: return f(TileShape<KIND, 256, 256, 2, 4, 128, 2>{});
        case k192: return f(TileShape<KIND, 192, 192, 2, 6, 128, 3>{});
        case k128: return f(TileShape<KIND, 128, 128, 2, 4, 128, 2>{});
        case k64: return f(TileShape<KIND, 64, 64, 2, 2, 128, 3>{});
        case k64InParts: return f(TileShape<KIND, 64, 64, 2, 2, 128, 2, 4>{});
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
    return tiles <= 0xFFFFFFF0ull && fold_grid((tiles + 7) / 8 * 8, S::kThreads, (unsigned)count, grid);
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
        static const float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};
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
