// Which tiles a product takes, by its sizes: rules on the host, of no device code, so that a host program may ask them too.
#pragma once

#include <cstdint>

namespace tq {

constexpr uint64_t kComputeUnits = 256;

// What a group of 128 bytes holds.  kHalfPair: elements as the sum of two binary16 numbers, 16 larger ones and the 16 smaller ones that go with
// them, twice.
enum { kInt8, kHalf, kHalfPair };

constexpr uint32_t in_group(int kind) { return kind == kInt8 ? 128u : kind == kHalf ? 64u : 32u; }

// ---- products of 8-bit integers (tq_i8_matmul.hip)

namespace i8 {

enum Shape { kFewShape, k256, k192, k192x256, k256x128, k128x256, k128x320, k128, k64 };

// A tile's sides, the time in ns that a group of k took while 1, 2, .. of them, as many as fit, were at work on every compute unit, and what
// a round of them costs beside that.  Us of bf16 products by shape:
//                         256   192x256  192   256x128  128x256  128x320   128     rule
//   1037 x 8192 x 4096    54.9   48.1    63.9   62.6     61.1     48.3    58.6     47.5
//   600 x 14336 x 4096    55.0   49.6    63.4   62.5     60.9     47.2    59.5     47.4
//   1500 x 4000 x 8192    82.6   72.6    62.3   62.7     63.4     68.0    64.9     62.4
//   2000 x 6000 x 4096    59.5   83.4    66.7   65.0     66.3     74.9    64.5     59.3
//   3500 x 2816 x 4096    55.5   52.7    64.2   61.9     62.2     49.9    60.6     50.6
//   5000 x 5000 x 3000    92.3  104      92.6  103      106       97.4   102       91.7
//   2056 x 1000 x 1999    28.4   22.4    17.8   17.5     17.4     20.4    12.1     13.2
struct Pace {
    Shape shape;
    uint64_t bm, bn;
    uint32_t ns[3], round;
};
constexpr Pace kPaces[] = {{k256, 256, 256, {1553, 0, 0}, 12000},   {k192, 192, 192, {943, 0, 0}, 9000},      {k256x128, 256, 128, {853, 0, 0}, 9000},
                           {k128x256, 128, 256, {870, 0, 0}, 9000}, {k192x256, 192, 256, {1200, 0, 0}, 10000},
                           {k128x320, 128, 320, {1030, 0, 0}, 9000}, {k128, 128, 128, {580, 925, 0}, 8000}, {k64, 64, 64, {262, 375, 560}, 3500}};

inline uint64_t pace(const Pace& p, uint64_t m, uint64_t n, uint64_t groups)
{
    const uint64_t tiles = (m + p.bm - 1) / p.bm * ((n + p.bn - 1) / p.bn), each = (tiles + kComputeUnits - 1) / kComputeUnits;
    const uint64_t fit = p.ns[2] ? 3 : p.ns[1] ? 2 : 1, rest = each % fit;
    return each / fit * (p.ns[fit - 1] * groups + p.round) + (rest ? p.ns[rest - 1] * groups + p.round : 0);
}

inline Shape shape_of(uint64_t m, uint64_t n, uint64_t groups)
{
    if (m <= 32) return kFewShape;
    const Pace* best = kPaces;
    for (const Pace& p : kPaces)
        if (pace(p, m, n, groups) < pace(*best, m, n, groups)) best = &p;
    return best->shape;
}

// Over how many workgroups k is split where few tiles of 64 leave compute units idle: as many as take least with the second launch and the partial
// sums' way through memory.  Not split / split, us: 40 x 1000 x 16384 31.3 / 11.5, 128 x 1024 x 16384 31.5 / 12.6, 64 x 64 x 65536 112 / 14.9,
// 256 x 512 x 8192 17.6 / 11.1, 64 x 4096 x 8192 18.0 / 12.5; 100 x 4096 x 4096 stays whole, 10.7 (in 4 parts 13.4).
inline uint32_t splits_of(uint64_t m, uint64_t n, uint64_t groups)
{
    if (shape_of(m, n, groups) != k64) return 1;
    const uint64_t tiles = (m + 63) / 64 * ((n + 63) / 64);
    uint64_t best = 1, least = 0;
    for (uint64_t s = 1; s <= 64 && s * 4 <= groups && tiles * s <= 2 * kComputeUnits; ++s) {
        const uint64_t ns = (groups + s - 1) / s * (tiles * s <= kComputeUnits ? 262 : 375) + (s > 1 ? 5000 + s * m * n * 8 / 5000 : 0);
        if (s > 1 && ns >= least) continue;
        least = ns;
        best = s;
    }
    return (uint32_t)best;
}

}  // namespace i8

// ---- products of orthogonalised updates (tq_orth.hip)

namespace orth {

// Tiles of a product: their sides, the time in ns that a group of k took while 1, 2, .. of them, as many as fit, were at work on every compute
// unit, and what a round of them costs beside that (both transposes are written).  `alone`: five buffers in place of two, one workgroup on a
// unit.  Kernel times of products, us, * the rule's:
//                                                        256     192     128   128 alone   64
//   binary16  4096^3, symmetric                         110    * 92     122     127       160
//   binary16  4096^3                                  * 131     177     164     180       235
//   binary16  512 x 512 x 2048, symmetric                46      26      21      18     * 11.5
//   binary16  512 x 2048 x 512                           23      15      11      11     *  8.5
//   pairs     2048^3, symmetric                         111      71      55    * 52        55
//   pairs     2048^3                                    117      78      63    * 62        82
//   pairs     4 of 1024 x 1024 x 4096, symmetric        213     140     108    * 95       102
//   pairs     4 of 1024 x 4096 x 1024                 * 104     156     117     137       166
//   pairs     784 x 1000 x 784                           56      34      23      20     * 11
// k in two or four parts by more wavefronts of a workgroup took longer than tiles of 64 by one set of them everywhere (784 x 1000: 13).
enum Shape { k256, k192, k128, k128Alone, k64 };
struct Pace {
    Shape shape;
    uint64_t side;
    uint32_t ns[3], round;
};
constexpr Pace kPaces[2][5] = {
    {{k256, 256, {1553, 0, 0}, 25000}, {k192, 192, {943, 0, 0}, 20000}, {k128, 128, {580, 925, 0}, 12000}, {k128Alone, 128, {540, 0, 0}, 12000}, {k64, 64, {262, 375, 560}, 5000}},
    {{k256, 256, {1900, 0, 0}, 40000}, {k192, 192, {1100, 0, 0}, 24000}, {k128, 128, {800, 1200, 0}, 15000}, {k128Alone, 128, {730, 0, 0}, 12000}, {k64, 64, {270, 450, 770}, 5000}}};

inline uint64_t tiles_of(uint64_t m, uint64_t n, uint64_t side, bool below)
{
    const uint64_t y = (m + side - 1) / side, x = (n + side - 1) / side;
    return below ? y * (y + 1) / 2 : x * y;
}

inline Shape shape_of(int kind, uint64_t m, uint64_t n, uint64_t k, bool below, uint64_t count)
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

}  // namespace orth

}  // namespace tq
