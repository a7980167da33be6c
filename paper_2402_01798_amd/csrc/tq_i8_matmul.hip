// Products of matrices of 8-bit integers (tq_i8.h): out = A B^T (+ bias).
#include <type_traits>

#include "tq_i8_device.h"
#include "tq_tiles.h"

namespace tq {
namespace {

struct I8MatmulArgs {
    const uint8_t *a, *b;
    const float *sa, *sb, *bias;
    void* out;
    uint64_t ldo;
    uint32_t m, n, groups;
    uint32_t tiles_x, tiles_y, tiles;
};

template <int DTYPE, class S>
__global__ __launch_bounds__(S::kThreads, S::kOnSimd) void i8_tile_kernel(I8MatmulArgs g)
{
    extern __shared__ char lds[];
    uint32_t tile, ty, tx;
    if (!tile_number(linear_block(), g.tiles, tile)) return;
    tile_place(tile, g.tiles_y, g.tiles_x, ty, tx);
    typename S::Sums acc[S::kFragsM][S::kFragsN];
    tile_sums<S>(TileOperands{g.a, g.b, g.m, g.n, g.groups, 0, g.groups}, ty * S::BM, tx * S::BN, lds, acc);
    tile_chunks<S>(acc, ty * S::BM, tx * S::BN, [&](uint32_t row, uint32_t col, const int (&sums)[8]) {
        if (row >= g.m || col >= g.n) return;
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
    });
}

template <int DTYPE, class S>
hipError_t launch_tiles(I8MatmulArgs& g, hipStream_t st)
{
    const uint64_t x = ((uint64_t)g.n + S::BN - 1) / S::BN, y = ((uint64_t)g.m + S::BM - 1) / S::BM;
    dim3 grid;
    if (x * y > 0xFFFFFFF0ull || !fold_grid((x * y + 7) / 8 * 8, S::kThreads, 1, grid)) return hipErrorInvalidValue;
    g.tiles_x = (uint32_t)x;
    g.tiles_y = (uint32_t)y;
    g.tiles = (uint32_t)(x * y);
    i8_tile_kernel<DTYPE, S><<<grid, S::kThreads, S::kBytes, st>>>(g);
    return hipGetLastError();
}

template <int DTYPE>
hipError_t launch_matmul(I8MatmulArgs& g, hipStream_t st)
{
    return launch_tiles<DTYPE, TileShape<kInt8, 256, 256, 2, 2, 64, 5>>(g, st);
}

}  // namespace
}  // namespace tq

uint64_t tq_i8_matmul_workspace_bytes_impl(uint64_t, uint64_t, uint64_t) { return 0; }

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
    g.groups = (uint32_t)((k + 127) / 128);
    if (dtype == TQ_F32) return launch_matmul<TQ_F32>(g, st);
    return dtype == TQ_BF16 ? launch_matmul<TQ_BF16>(g, st) : launch_matmul<TQ_F16>(g, st);
}
