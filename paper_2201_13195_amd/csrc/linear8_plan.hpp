// Which kernel a product of 8-bit operands takes (plain C++).
#pragma once
#include <stdint.h>

namespace rmm {

// Tokens x outputs of a work-group.  FEW: eight waves share the contraction (linear8_few.hpp); MANY: four, where there are
// more work-groups than compute units; TILE: linear8_tile.hpp.
enum {
    LINEAR8_FEW_16x16 = 0,
    LINEAR8_FEW_16x32 = 1,
    LINEAR8_FEW_32x32 = 2,
    LINEAR8_FEW_64x32 = 3,
    LINEAR8_MANY_16x64 = 4,
    LINEAR8_MANY_32x32 = 5,
    LINEAR8_MANY_64x32 = 6,
    LINEAR8_TILE_64x128 = 7,
    LINEAR8_TILE_128_SPLIT = 8,
    LINEAR8_TILE_128 = 9,
    LINEAR8_TILE_256 = 10
};

// A row per rule, times in us of bf16 results measured on both sides of it (256 compute units):
//   - the smallest FEW kernel with no more work-groups than compute units: its time is one round of a latency and the contraction.
//       24 x 4096 -> 1024 16x16 4.3, 16x32 4.5, 128 x 128 tiles 20;   128 x 768 -> 768 16x16 3.9 (384 work-groups), 16x32 3.4, 32x32 3.8;
//       64 x 4096 -> 4096 16x32 8.7 (512), 32x32 7.0, 64x32 7.5;   128 x 4096 -> 4096 32x32 10.1 (512), 64x32 8.0, MANY 32x32 8.8
//   - instead of 64x32 MANY 32x32, two work-groups to a compute unit, where its four waves have no more than two blocks each (traced
//     launches, fp32 scales, 64x32 in brackets):  128 x 256 -> 4096 4.2 (4.5), 1000 x 256 -> 400 4.3 (4.5), 500 x 384 -> 900 4.4 (4.6),
//       64 x 512 -> 6000 4.4 (4.6), 200 x 512 -> 2048 4.4 (4.7), 2000 x 640 -> 256 4.7 (5.1), 256 x 768 -> 2048 4.8 (5.0), 400 x 900 -> 1000 5.3 (5.7),
//       500 x 1024 -> 768 5.0 (5.1), 128 x 1024 -> 4000 5.3 (5.3);   twelve blocks:  200 x 1536 -> 2048 5.8 (5.6), 500 x 1536 -> 768 5.7 (5.5)
//   - up to 64 tokens and more outputs than that: the weights are read once, whatever the tile, and four waves of more outputs keep more of
//     them in flight.  1 x 4096 -> 32000 (131 MB) 16x32 23.9, MANY 16x64 20.2, 128 x 128 tiles 27.9;  32 x 4096 -> 16384 MANY 32x32 12.8,
//     64x32 13.5, 64 x 128 tiles 15.1;  48 x 4096 -> 16384 MANY 32x32 20.8, 64x32 14.1, 64 x 128 tiles 15.6
//   - MANY 64x32 for up to two work-groups a compute unit too:  1024 x 1024 -> 1024 5.8 (64 x 128 tiles 7.1);  256 x 4096 -> 4096 11.8 (14.5),
//     but 400 x 768 -> 3000 (658) 8.1 (7.1) and 512 x 4096 -> 4096 (1024) 22.5 (15.2)
//   - tiles otherwise, up to a compute unit's one by two groups of waves that share the contraction, where it is long enough:
//     64 x 128 from six blocks of it on (three for fp32 results, whose every block is four times the work), 128 x 128 from twenty.
//       512 x 4096 -> 4096 64 x 128 16.9, 128 x 128 split 22.0, as below 26.6;   512 x 1024 -> 4096 8.1, 9.3, 8.6;   512 x 640 -> 4096 7.3, 8.5, 7.1;
//       1024 x 4096 -> 4096 (512 of 64 x 128) 31.4, 25.1, 28.9;   1024 x 2560 -> 4096 22.9, 17.3, 18.3;   1024 x 2048 -> 4096 20.1, 14.6, 14.6
//   - as many as there are, one group of waves each.  A 256 x 256 tile has a compute unit to itself, two 128 x 128 tiles share one.  The model
//     below counts, in hundredths of us, 1.2 us for a step of 128 (0.95 for both small ones) and 3 (2) more for a round of tiles. Measured, a step
//     of the large tile is 1.3 to 1.5 up to 16 of them and 1.6 beyond (8192 x 1024, 2048, 4096 -> 2048, one round: 22.2, 34.1, 59.8), so that
//     near the break-even the large tile is taken where the small one would do better (bf16 results, fp32 scales, the same operands again and again):
//       256 taken:  4096 x 1024 -> 4096 256 21.9, 128 23.9;   8192 x 512 -> 4096 25.7, 27.3;   8192 x 1024 -> 2048 22.2, 23.9;   16384 x 1024 -> 1024 22.4, 24.0;
//         7000 x 2048 -> 4096 59.5, 67.1;   16384 x 1024 -> 4096 72, 85;   8192 x 4096 -> 4096 115, 143;   16384 x 4096 -> 4096 225, 282 (powers of two 211, 262)
//       256 taken, and 128 would be faster:  16384 x 768 -> 768 17.5, 17.1;   4096 x 1024 -> 2560 19.2, 18.9;   6000 x 1024 -> 4096 34.4, 33.8;
//         3000 x 1500 -> 6000 48.3, 43.0;   5000 x 1024 -> 4096 33.1, 29.0
//       128 taken:  8192 x 1024 -> 1024 18.7, 14.1;   4096 x 2048 -> 2048 28.6, 22.1
//     fp32 results have no 256 x 256 tiles (the exact way needs the registers).
inline int64_t linear8_groups(int64_t n, int64_t d_out, int64_t tokens, int64_t outputs) {
    return ((n + tokens - 1) / tokens) * ((d_out + outputs - 1) / outputs);
}
inline int linear8_plan(int64_t n, int64_t d_in, int64_t d_out, int64_t ld_x, int64_t ld_w, bool exact) {
    constexpr int64_t kUnits = 256;
    if (linear8_groups(n, d_out, 16, 16) <= kUnits) return LINEAR8_FEW_16x16;
    if (linear8_groups(n, d_out, 16, 32) <= kUnits) return LINEAR8_FEW_16x32;
    if (linear8_groups(n, d_out, 32, 32) <= kUnits) return LINEAR8_FEW_32x32;
    const int64_t steps = (d_in + 127) / 128;
    if (n > 16 && steps <= 8 && linear8_groups(n, d_out, 32, 32) <= 2 * kUnits) return LINEAR8_MANY_32x32;
    if (linear8_groups(n, d_out, 64, 32) <= kUnits) return LINEAR8_FEW_64x32;
    if (n <= 16) return LINEAR8_MANY_16x64;
    const int64_t small = linear8_groups(n, d_out, 128, 128), large = linear8_groups(n, d_out, 256, 256);
    const bool fits = ld_x < (1 << 23) && ld_w < (1 << 23) && small < (1 << 23);  // (offsets within a tile, and the grid, in 32 bits)
    if (n <= 32 || !fits) return LINEAR8_MANY_32x32;
    if (n <= 64 || linear8_groups(n, d_out, 64, 32) <= 2 * kUnits) return LINEAR8_MANY_64x32;
    if (linear8_groups(n, d_out, 64, 128) <= kUnits && steps >= (exact ? 3 : 6)) return LINEAR8_TILE_64x128;
    if (small <= kUnits && steps >= 20) return LINEAR8_TILE_128_SPLIT;
    if (exact) return LINEAR8_TILE_128;
    const int64_t t256 = 600 + (large + kUnits - 1) / kUnits * (120 * steps + 300);
    const int64_t t128 = 300 + (small + 2 * kUnits - 1) / (2 * kUnits) * (95 * steps + 200);
    return t256 <= t128 ? LINEAR8_TILE_256 : LINEAR8_TILE_128;
}

}  // namespace rmm
