// How a product with weights in 4 bits is cut up.  Host code alone: tests build it without a GPU.
#pragma once

#include <stdint.h>

#include "oz_scaled_plan.h"

namespace oz {

constexpr int kPackedBlock = 128;        // of k

struct PackedPlan {
    int rows, strips;      // 16s of rows of x and of W to a workgroup
    int waves;             // that share k
};

// Pieces of `size` rows of x; groups 0: all are one's.
inline int64_t packed_tiles(int64_t m, int64_t groups, int64_t size) { return groups ? group_pieces(m, groups, size) : (m + size - 1) / size; }

// shift: of W's groups, log2 of 32, 64 or 128; bytes: of an element of x.
inline PackedPlan packed_plan(int64_t m, int64_t n, int64_t k, int64_t groups, int bytes, int shift, int num_cu) {
    const int64_t avg = groups ? (m + groups - 1) / groups : m;      // rows of a group on average
    const int64_t blocks = std::max<int64_t>((k + kPackedBlock - 1) / kPackedBlock, 1);
    auto tiles_of = [&](int rows) { return packed_tiles(m, groups, rows * 16) * ((n + 15) / 16); };
    PackedPlan p{avg <= 16 ? 1 : avg <= 32 ? 2 : 4, 1, 1};
    // as many rows of x as there are, up to 64, but fewer where that leaves the chip idle: W is read more often then, by more (33 x 1300 x 777, groups of
    // 64: 11.6 us with 64, 6.4 with 16 and two scales to a block)
    while (p.rows > 1 && tiles_of(p.rows / 2) <= 2 * num_cu) p.rows /= 2;
    const int64_t tiles = tiles_of(p.rows);
    // Rows of W, and waves that share k: what fills the chip with 16 waves to a CU that have two blocks each, with as much of W to a wave as that leaves,
    // since all of it shares the wave's x (64 x 8192 x 8192: 66 us with one strip, 42 with two).
    auto waves_of = [&](int strips, int most) {
        int w = 1;
        while (w < most && w < blocks && tiles / strips * w < 16 * num_cu) w *= 2;
        return w;
    };
    // more rows of W for each x take more registers: groups of 32 with their scales leave room for two strips, small groups and 64 rows of x, and float32
    // beside more than 16, for one
    const int most = p.rows == 1 ? (shift == 5 ? 2 : 4) : bytes == 2 && (p.rows == 2 || shift == 7) ? 2 : 1;
    p.waves = waves_of(1, p.rows == 1 ? 16 : 8);
    for (int more = 2; more <= most; more *= 2) {
        const int w = waves_of(more, p.rows == 1 && more * bytes <= 4 ? 16 : 8);
        if (tiles / more * w < (p.rows == 4 ? 8 : 16) * num_cu) break;
        p.strips = more;
        p.waves = w;
    }
    return p;
}

}  // namespace oz
