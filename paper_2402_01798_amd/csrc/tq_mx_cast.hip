// Matrices to microscaled 4-bit form and back (tq_mx.h).
#include <type_traits>

#include "tq_mx_device.h"

namespace tq {
namespace {

struct CastArgs {
    const void* x;
    uint8_t *codes, *scales, *codes_t, *scales_t;
    uint64_t ld;
    uint32_t rows, cols, groups, groups_t;     // groups of 128 along a row, along a column
    uint32_t k0, k1, worker, step;
    uint32_t tiles_x, log_lanes;               // rows kernel: workgroups along a row, lanes along a row
    uint64_t tiles;
    bool blocks;                               // by mx_cast_block_kernel
};

// Along the rows: a lane takes 8 elements, four lanes a block, 16 lanes a group.  A workgroup is 2^log_lanes lanes along a row
// times as many rows as fit.
template <int DTYPE, bool STOCHASTIC>
__global__ __launch_bounds__(256) void mx_cast_rows_kernel(CastArgs a)
{
    using T = typename Element<DTYPE>::type;
    const uint32_t block = linear_block();
    if (block >= a.tiles) return;
    const uint32_t lane = threadIdx.x & ((1u << a.log_lanes) - 1), sub = threadIdx.x >> a.log_lanes;
    const uint32_t by = block / a.tiles_x, bx = block - by * a.tiles_x;
    const uint64_t row = (uint64_t)by * (256u >> a.log_lanes) + sub;
    const uint32_t oct = (bx << a.log_lanes) + lane;             // which 8 elements of the row
    if (row >= a.rows || oct >= a.groups * 16) return;           // 16 lanes of a group leave together
    const int n = (int)min((int64_t)a.cols - (int64_t)oct * 8, (int64_t)8);
    float v[8];
    const T* x = static_cast<const T*>(a.x);
    if constexpr (STOCHASTIC) x += round_toward_zero();
    load8<DTYPE>(x + row * a.ld + (uint64_t)oct * 8, n, v);
    uint32_t draws[4] = {};
    if constexpr (STOCHASTIC) philox4x32_10(oct, (uint32_t)row, a.worker, a.step, a.k0, a.k1, draws);
    uint32_t largest = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) largest = max(largest, magnitude_bits(v[j]));
    largest = quad_max(largest);
    const uint32_t byte = mx_scale_byte<STOCHASTIC>(largest);
    uint32_t w = 0;
    if constexpr (STOCHASTIC) {
#pragma unroll
        for (int j = 7; j >= 0; --j) w = mx_push(w, v[j], byte, mx_draw(draws[j / 2], j & 1));
        if (byte == 255) w = 0;
    } else {
        w = mx_nearest(v, byte);
    }
    reinterpret_cast<uint32_t*>(a.codes)[row * (a.groups * 16) + oct] = w;
    if ((oct & 3) == 0) a.scales[((uint64_t)(oct / 16) * a.rows + row) * 4 + (oct / 4 & 3)] = (uint8_t)byte;
}

// Along the columns, or both ways: a workgroup takes 128 x 128 elements, a wavefront 32 rows of them, which are whole blocks in
// either direction.  Lane 4 c + r of a wavefront holds columns 8 c .. 8 c + 7 of rows 8 r .. 8 r + 7: a row's block is
// four lanes 4 apart, a column's four neighbouring lanes.  The transposed codes go through LDS, so that a column's 64 bytes are
// written at once.
template <int DTYPE, bool STOCHASTIC, bool ROWS>
__global__ __launch_bounds__(256) void mx_cast_tile_kernel(CastArgs a)
{
    using T = typename Element<DTYPE>::type;
    __shared__ uint32_t codes_t[128][17];                        // 16 words of a column; one more against bank conflicts
    __shared__ uint8_t scale_t[128][4], scale[128][4];
    const uint32_t block = linear_block();
    if (block >= a.tiles) return;
    const uint32_t ty = block / a.tiles_x, tx = block - ty * a.tiles_x;
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 2, r = lane & 3;
    const uint32_t row0 = ty * 128 + wave * 32 + r * 8, oct = tx * 16 + c;
    const int n = (int)max(min((int64_t)a.cols - (int64_t)oct * 8, (int64_t)8), (int64_t)0);
    const T* x = static_cast<const T*>(a.x);
    if constexpr (STOCHASTIC) x += round_toward_zero();
    Eight<DTYPE> held[8];
    x += (uint64_t)oct * 8;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) held[i].load(x + (uint64_t)min(row0 + i, a.rows - 1) * a.ld);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) held[i].load(x + (uint64_t)min(row0 + i, a.rows - 1) * a.ld, n);
    }
    if (row0 + 8 > a.rows) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (row0 + i >= a.rows) held[i].clear();
    }
    uint32_t byte_t[8], most[Eight<DTYPE>::kWords] = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) held[i].largest_of_columns(most);
#pragma unroll
    for (int j = 0; j < Eight<DTYPE>::kWords; ++j) {             // of four neighbouring lanes
        most[j] = Eight<DTYPE>::larger(most[j], dpp_move<0xB1>(most[j]));
        most[j] = Eight<DTYPE>::larger(most[j], dpp_move<0x4E>(most[j]));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        byte_t[j] = mx_scale_byte<STOCHASTIC>(Eight<DTYPE>::bits(most[j * Eight<DTYPE>::kWords / 8], j & 1));
        if (r == 0) scale_t[c * 8 + j][wave] = (uint8_t)byte_t[j];
    }
    uint32_t w_t[8] = {};
    auto along_the_row = [&](int i, const float (&v)[8]) {       // and, rounded stochastically, down the columns
        const uint32_t row = row0 + i;
        uint32_t byte = 0, w = 0;
        if constexpr (ROWS) byte = mx_scale_byte<STOCHASTIC>(stride4_max(held[i].largest()));
        if constexpr (STOCHASTIC) {
            uint32_t draws[4], o = oct;
            asm volatile("" : "+v"(o));                          // not all rows' draws first: they would wait in registers
            philox4x32_10(o, row, a.worker, a.step, a.k0, a.k1, draws);
#pragma unroll
            for (int j = 7; j >= 0; --j) {
                const uint32_t d = mx_draw(draws[j / 2], j & 1);
                w_t[j] = mx_push(w_t[j], v[j], byte_t[j], d);
                if constexpr (ROWS) w = mx_push(w, v[j], byte, d);
                asm volatile("" : "+v"(w_t[j]));                 // here and not where it is stored, for which what goes into it would
            }                                                    // have to be kept
            if (byte == 255) w = 0;
        } else if constexpr (ROWS) {
            w = mx_nearest(v, byte);
        }
        if constexpr (ROWS) {
            if (row < a.rows) reinterpret_cast<uint32_t*>(a.codes)[(uint64_t)row * (a.groups * 16) + oct] = w;
            if ((c & 3) == 0) scale[wave * 32 + r * 8 + i][c / 4] = (uint8_t)byte;
        }
    };
    auto two_rows = [&](auto P) {
        constexpr int p = decltype(P)::value;
        float even[8], odd[8];
        held[2 * p + 1].unpack(odd);
        along_the_row(2 * p + 1, odd);
        held[2 * p].unpack(even);
        along_the_row(2 * p, even);
        if constexpr (!STOCHASTIC) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                w_t[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w_t[j], even[j], odd[j], __uint_as_float(byte_t[j] << 23), p);
        }
        __builtin_amdgcn_sched_barrier(0);                       // one pair after the other: fewer registers
    };
    two_rows(std::integral_constant<int, 3>{});                  // downwards: mx_push puts the last one lowest
    two_rows(std::integral_constant<int, 2>{});
    two_rows(std::integral_constant<int, 1>{});
    two_rows(std::integral_constant<int, 0>{});
#pragma unroll
    for (int j = 0; j < 8; ++j) codes_t[c * 8 + j][wave * 4 + r] = byte_t[j] == 255 ? 0 : w_t[j];
    __syncthreads();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t column = h * 64 + threadIdx.x / 4, piece = threadIdx.x & 3;
        const uint64_t out = (uint64_t)tx * 128 + column;
        if (out < a.cols) {
            const uint32_t* p = &codes_t[column][piece * 4];
            *reinterpret_cast<u32x4*>(a.codes_t + (out * a.groups_t + ty) * 64 + piece * 16) = u32x4{p[0], p[1], p[2], p[3]};
        }
    }
    if (threadIdx.x < 128) {
        const uint64_t column = (uint64_t)tx * 128 + threadIdx.x;
        if (column < a.cols)
            *reinterpret_cast<uint32_t*>(a.scales_t + ((uint64_t)ty * a.cols + column) * 4) = *reinterpret_cast<const uint32_t*>(scale_t[threadIdx.x]);
    } else if (ROWS) {
        const uint64_t row = (uint64_t)ty * 128 + (threadIdx.x - 128);
        if (row < a.rows)
            *reinterpret_cast<uint32_t*>(a.scales + ((uint64_t)tx * a.rows + row) * 4) = *reinterpret_cast<const uint32_t*>(scale[threadIdx.x - 128]);
    }
}

// The same for small matrices, where the time is one wavefront's from its request to its store: a wavefront takes one block in
// either direction, 32 x 32, a quarter of the elements a lane.  Lane 16 c + r holds columns 8 c .. 8 c + 7 of rows 2 r and 2 r + 1.
template <int DTYPE, bool STOCHASTIC, bool ROWS>
__global__ __launch_bounds__(256) void mx_cast_block_kernel(CastArgs a)
{
    using T = typename Element<DTYPE>::type;
    __shared__ __attribute__((aligned(16))) uint8_t codes_t[4][32][16];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane >> 4, r = lane & 15;
    const uint64_t tile = (uint64_t)linear_block() * 4 + wave;
    if (tile >= a.tiles) return;
    const uint32_t rb = (uint32_t)(tile / a.tiles_x), cb = (uint32_t)(tile - (uint64_t)rb * a.tiles_x);
    const uint32_t row0 = rb * 32 + r * 2, oct = cb * 4 + c;
    const int n = (int)max(min((int64_t)a.cols - (int64_t)oct * 8, (int64_t)8), (int64_t)0);
    const T* x = static_cast<const T*>(a.x);
    if constexpr (STOCHASTIC) x += round_toward_zero();
    x += (uint64_t)oct * 8;
    float v[2][8];
#pragma unroll
    for (int i = 0; i < 2; ++i) load8<DTYPE>(x + (uint64_t)min(row0 + i, a.rows - 1) * a.ld, row0 + i < a.rows ? n : 0, v[i]);
    uint32_t draws[2][4] = {};
    if constexpr (STOCHASTIC) {
        philox4x32_10(oct, row0, a.worker, a.step, a.k0, a.k1, draws[0]);
        philox4x32_10(oct, row0 + 1, a.worker, a.step, a.k0, a.k1, draws[1]);
    }
    if constexpr (ROWS) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            uint32_t largest = 0, w = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) largest = max(largest, magnitude_bits(v[i][j]));
            const uint32_t byte = mx_scale_byte<STOCHASTIC>(stride16_max(largest));
            if constexpr (STOCHASTIC) {
#pragma unroll
                for (int j = 7; j >= 0; --j) w = mx_push(w, v[i][j], byte, mx_draw(draws[i][j / 2], j & 1));
                if (byte == 255) w = 0;
            } else {
                w = mx_nearest(v[i], byte);
            }
            if (row0 + i < a.rows) {
                reinterpret_cast<uint32_t*>(a.codes)[(uint64_t)(row0 + i) * (a.groups * 16) + oct] = w;
                if (c == 0) a.scales[((uint64_t)(cb / 4) * a.rows + row0 + i) * 4 + (cb & 3)] = (uint8_t)byte;
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t byte = mx_scale_byte<STOCHASTIC>(row16_max(max(magnitude_bits(v[0][j]), magnitude_bits(v[1][j]))));
        uint32_t w = 0;
        if constexpr (STOCHASTIC) {
            w = mx_push(w, v[1][j], byte, mx_draw(draws[1][j / 2], j & 1));
            w = mx_push(w, v[0][j], byte, mx_draw(draws[0][j / 2], j & 1));
        } else {
            w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0][j], v[1][j], __uint_as_float(byte << 23), 0);
        }
        codes_t[wave][c * 8 + j][r] = byte == 255 ? 0 : (uint8_t)w;
        const uint32_t column = oct * 8 + j;
        if (r == 0 && column < a.cols) a.scales_t[((uint64_t)(rb / 4) * a.cols + column) * 4 + (rb & 3)] = (uint8_t)byte;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // other lanes' bytes; a wavefront's LDS operations complete in order
    const uint64_t column = (uint64_t)cb * 32 + lane;
    if (lane < 32 && column < a.cols)
        *reinterpret_cast<u32x4*>(a.codes_t + (column * a.groups_t + rb / 4) * 64 + (rb & 3) * 16) = *reinterpret_cast<const u32x4*>(codes_t[wave][lane]);
}

// Back: a lane takes 8 elements, as in mx_cast_rows_kernel.
template <int DTYPE>
__global__ __launch_bounds__(256) void mx_dequantize_kernel(CastArgs a)
{
    using T = typename Element<DTYPE>::type;
    const uint32_t block = linear_block();
    if (block >= a.tiles) return;
    const uint32_t lane = threadIdx.x & ((1u << a.log_lanes) - 1), sub = threadIdx.x >> a.log_lanes;
    const uint32_t by = block / a.tiles_x, bx = block - by * a.tiles_x;
    const uint64_t row = (uint64_t)by * (256u >> a.log_lanes) + sub;
    const uint32_t oct = (bx << a.log_lanes) + lane;
    if (row >= a.rows || (uint64_t)oct * 8 >= a.cols) return;
    const uint32_t w = reinterpret_cast<const uint32_t*>(a.codes)[row * (a.groups * 16) + oct];
    const uint32_t byte = a.scales[((uint64_t)(oct / 16) * a.rows + row) * 4 + (oct / 4 & 3)];
    float v[8];
    // A power of two from its byte: the smallest is a subnormal number, 255 is NaN.
    const float scale = __uint_as_float(byte == 255 ? 0x7FC00000u : byte == 0 ? 0x00400000u : byte << 23);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        f32x2 p;
        if (j == 0) p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 0);
        else if (j == 1) p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 1);
        else if (j == 2) p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 2);
        else p = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.0f, 3);
        v[2 * j] = p.x * scale;
        v[2 * j + 1] = p.y * scale;
    }
    const int n = (int)min((int64_t)a.cols - (int64_t)oct * 8, (int64_t)8);
    store8<DTYPE>(static_cast<T*>(const_cast<void*>(a.x)) + row * a.ld + (uint64_t)oct * 8, n, v);
}

template <int DTYPE, bool STOCHASTIC>
void launch_cast(const CastArgs& a, dim3 grid, hipStream_t st)
{
    if (!a.codes_t) mx_cast_rows_kernel<DTYPE, STOCHASTIC><<<grid, 256, 0, st>>>(a);
    else if (a.blocks && a.codes) mx_cast_block_kernel<DTYPE, STOCHASTIC, true><<<grid, 256, 0, st>>>(a);
    else if (a.blocks) mx_cast_block_kernel<DTYPE, STOCHASTIC, false><<<grid, 256, 0, st>>>(a);
    else if (a.codes) mx_cast_tile_kernel<DTYPE, STOCHASTIC, true><<<grid, 256, 0, st>>>(a);
    else mx_cast_tile_kernel<DTYPE, STOCHASTIC, false><<<grid, 256, 0, st>>>(a);
}

template <int DTYPE>
void launch_cast(const CastArgs& a, bool stochastic, dim3 grid, hipStream_t st)
{
    if (stochastic) launch_cast<DTYPE, true>(a, grid, st);
    else launch_cast<DTYPE, false>(a, grid, st);
}

// Lanes along a row and workgroups of the kernels that go along the rows.
bool rows_grid(CastArgs& a, uint64_t octs, dim3& grid)
{
    a.log_lanes = 4;
    while (a.log_lanes < 8 && (1ull << a.log_lanes) < octs) ++a.log_lanes;
    a.tiles_x = (uint32_t)((octs + (1ull << a.log_lanes) - 1) >> a.log_lanes);
    const uint64_t per = 256u >> a.log_lanes;
    a.tiles = a.tiles_x * ((a.rows + per - 1) / per);
    return fold_grid(a.tiles, 256, 1, grid);
}

}  // namespace
}  // namespace tq

hipError_t tq_launch_mx_quantize(const void* x, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int rounding, uint64_t seed,
                                 uint32_t worker, uint32_t step, void* codes, void* scales, void* codes_t, void* scales_t,
                                 hipStream_t st)
{
    using namespace tq;
    CastArgs a = {};
    a.x = x;
    a.codes = static_cast<uint8_t*>(codes);
    a.scales = static_cast<uint8_t*>(scales);
    a.codes_t = static_cast<uint8_t*>(codes_t);
    a.scales_t = static_cast<uint8_t*>(scales_t);
    a.ld = ld;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.groups = (uint32_t)((cols + kMxGroup - 1) / kMxGroup);
    a.groups_t = (uint32_t)((rows + kMxGroup - 1) / kMxGroup);
    a.k0 = (uint32_t)seed;
    a.k1 = (uint32_t)(seed >> 32);
    a.worker = worker;
    a.step = step;
    dim3 grid;
    if (codes_t) {
        // Blocks of 32 x 32 a wavefront below 256 tiles of 128 x 128 (one for each compute unit).  Tiles / blocks, us, both forms of fp32
        // nearest and stochastic: 64 x 784 5.1 / 3.4 and 6.9 / 3.9, 1000 x 1000 6.3 / 3.6 and 8.2 / 4.1, 2048 x 2048 5.9 / 6.1 and 7.8 / 7.3,
        // 4096 x 4096 15.7 / 17.6 and 19.5 / 19.8 (bf16 11.7 / 14.6 and 17.7 / 19.9).
        a.blocks = (uint64_t)a.groups * a.groups_t < 256;
        a.tiles_x = a.blocks ? a.groups * 4 : a.groups;
        a.tiles = (uint64_t)a.tiles_x * (a.blocks ? a.groups_t * 4 : a.groups_t);
        if (!fold_grid(a.blocks ? (a.tiles + 3) / 4 : a.tiles, 256, 1, grid)) return hipErrorInvalidValue;
    } else if (!rows_grid(a, (uint64_t)a.groups * 16, grid)) {
        return hipErrorInvalidValue;
    }
    const bool stochastic = rounding == TQ_MX_STOCHASTIC;
    if (dtype == TQ_F32) launch_cast<TQ_F32>(a, stochastic, grid, st);
    else if (dtype == TQ_BF16) launch_cast<TQ_BF16>(a, stochastic, grid, st);
    else launch_cast<TQ_F16>(a, stochastic, grid, st);
    return hipGetLastError();
}

hipError_t tq_launch_mx_dequantize(const void* codes, const void* scales, uint64_t rows, uint64_t cols, void* out, int dtype,
                                   uint64_t ldo, hipStream_t st)
{
    using namespace tq;
    CastArgs a = {};
    a.x = out;
    a.codes = static_cast<uint8_t*>(const_cast<void*>(codes));
    a.scales = static_cast<uint8_t*>(const_cast<void*>(scales));
    a.ld = ldo;
    a.rows = (uint32_t)rows;
    a.cols = (uint32_t)cols;
    a.groups = (uint32_t)((cols + kMxGroup - 1) / kMxGroup);
    dim3 grid;
    if (!rows_grid(a, (cols + 7) / 8, grid)) return hipErrorInvalidValue;
    if (dtype == TQ_F32) mx_dequantize_kernel<TQ_F32><<<grid, 256, 0, st>>>(a);
    else mx_dequantize_kernel<TQ_BF16><<<grid, 256, 0, st>>>(a);
    return hipGetLastError();
}
