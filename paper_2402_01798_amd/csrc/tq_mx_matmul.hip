// Products of microscaled 4-bit matrices (tq_mx.h): out = A B^T (+ add).
#include "tq_mx_device.h"

namespace tq {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

struct MatmulArgs {
    const uint8_t *a, *sa, *b, *sb;
    const float* add;
    void* out;
    uint64_t lda, ldo;
    uint32_t m, n, groups;
    uint32_t tiles_x;
    uint64_t tiles;
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
    if (g.add) v += g.add[row * g.lda + col];
    static_cast<typename E::type*>(g.out)[row * g.ldo + col] = E::store(v);
}

// A wavefront's 32 x 32 outputs straight from memory.
template <int DTYPE>
__global__ __launch_bounds__(64) void mx_matmul_direct_kernel(MatmulArgs g)
{
    const uint32_t block = linear_block();
    if (block >= g.tiles) return;
    const uint32_t ty = block / g.tiles_x, tx = block - ty * g.tiles_x;
    const uint32_t lane = threadIdx.x, r = lane & 31, half = lane >> 5;
    const uint32_t ra = min(ty * 32 + r, g.m - 1), rb = min(tx * 32 + r, g.n - 1);      // rows past the end repeat the last
    const uint8_t* pa = g.a + (uint64_t)ra * g.groups * 64 + half * 16;
    const uint8_t* pb = g.b + (uint64_t)rb * g.groups * 64 + half * 16;
    f32x16 acc = {};
    for (uint32_t i = 0; i < g.groups; ++i) {
        const int sa = *reinterpret_cast<const int*>(g.sa + ((uint64_t)i * g.m + ra) * 4) >> (8 * half);
        const int sb = *reinterpret_cast<const int*>(g.sb + ((uint64_t)i * g.n + rb) * 4) >> (8 * half);
        const i32x4* qa = reinterpret_cast<const i32x4*>(pa + (uint64_t)i * 64);
        const i32x4* qb = reinterpret_cast<const i32x4*>(pb + (uint64_t)i * 64);
        acc = mfma32<0>(qa[0], qb[0], acc, sa, sb);
        acc = mfma32<2>(qa[2], qb[2], acc, sa, sb);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) store_one<DTYPE>(g, ty * 32 + (i / 4) * 8 + half * 4 + i % 4, tx * 32 + r, acc[i]);
}

}  // namespace
}  // namespace tq

uint64_t tq_mx_matmul_workspace_bytes_impl(uint64_t m, uint64_t n, uint64_t k) { return 0; }

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
    g.groups = (uint32_t)((k + kMxGroup - 1) / kMxGroup);
    g.tiles_x = (uint32_t)((n + 31) / 32);
    g.tiles = g.tiles_x * ((m + 31) / 32);
    dim3 grid;
    if (!fold_grid(g.tiles, 64, 1, grid)) return hipErrorInvalidValue;
    if (dtype == TQ_F32) mx_matmul_direct_kernel<TQ_F32><<<grid, 64, 0, st>>>(g);
    else if (dtype == TQ_BF16) mx_matmul_direct_kernel<TQ_BF16><<<grid, 64, 0, st>>>(g);
    else mx_matmul_direct_kernel<TQ_F16><<<grid, 64, 0, st>>>(g);
    return hipGetLastError();
}
