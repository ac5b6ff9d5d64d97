// How a product with weights in 4 bits is cut up.  Host code alone: tests build it without a GPU.
#pragma once

#include <stdint.h>

#include "oz_scaled_plan.h"

namespace oz {

constexpr int kPackedBlock = 128;        // of k

struct PackedPlan {
    bool staged;           // x through LDS
    int rows, strips;      // 16s of rows of x and of W to a workgroup
    int waves;             // that share k
};

// Pieces of `size` rows of x; groups 0: all are one's.
inline int64_t packed_tiles(int64_t m, int64_t groups, int64_t size) { return groups ? group_pieces(m, groups, size) : (m + size - 1) / size; }

// shift: of W's groups, log2 of 32, 64 or 128; bytes: of an element of x.  Times below: us of one product on 256 CUs.
inline PackedPlan packed_plan(int64_t m, int64_t n, int64_t k, int64_t groups, int bytes, int shift, int num_cu) {
    const int64_t avg = groups ? (m + groups - 1) / groups : m;      // rows of a group on average
    const int64_t blocks = std::max<int64_t>((k + kPackedBlock - 1) / kPackedBlock, 1);
    auto workgroups = [&](int rows, int strips) { return packed_tiles(m, groups, rows * 16) * ((n + 16 * strips - 1) / (16 * strips)); };
    // waves that share k: what fills the chip with so many of them; more than four have `least` blocks each
    auto waves_of = [&](int64_t of, int64_t want, int most, int least) {
        int w = 1;
        while (w < most && (w < 4 ? w : w * least) < blocks && of * w < want) w *= 2;
        return w;
    };
    // x through LDS where its loads count, which four rows' do not (bfloat16, 4096 x 4096, groups of 32: 1 row 5.9 without, 6.7 with; 16 rows 8.3, 7.0; 64 rows
    // 21, 13); of float32 eight (8 rows 11.6, 12.7; 12 rows of 8192 x 8192 37, 26)
    if (avg > (bytes == 4 ? 8 : 4)) {
        // The largest tile of which there are enough.  64 x 32 W by x with groups of 128 alone: registers (bfloat16 128 x 8192 x 8192: 37, with 32 x 32 46;
        // 512 rows of 32 groups, 2048 x 2048: 25, with 32 x 16 25, float32 54 and 64).  Fewer tiles than CUs are worse than smaller ones
        // (64 x 4096 x 4096: 64 x 32 18, 32 x 32 10.6; 24 x 4096 x 4096: 32 x 32 9.5, 32 x 16 7.6; 32 x 1536 x 2048: 5.8 with 32 x 16, 4.9 with 16 x 16).
        // Eight waves to a CU, of groups twice as many, whose last tiles are not full (512 rows of 8 groups, 4096 x 2048, groups of 32: 67 us, 53).
        const int64_t want = (avg > 24 && groups ? 16 : 8) * num_cu;
        if (shift == 7 && avg > (groups ? 12 : 16) && workgroups(2, 4) * bytes >= 4 * num_cu) return {true, 2, 4, waves_of(workgroups(2, 4), want, 8, 2)};
        if (avg > 16 && workgroups(2, 2) >= num_cu) return {true, 2, 2, waves_of(workgroups(2, 2), want, 8, 2)};
        if (workgroups(1, 2) * 4 >= 3 * num_cu) return {true, 1, 2, waves_of(workgroups(1, 2), want, 8, 2)};
        // float32 is the same without (33 x 1300 x 777: 6.3, 6.8)
        if (bytes == 2) return {true, 1, 1, waves_of(workgroups(1, 1), want, 8, 2)};
    }
    // 16 waves to a CU that have two blocks each, with as much of W to a wave as that leaves, since all of it shares the wave's x; groups of 32 with
    // their scales leave registers for two strips
    PackedPlan p{false, 1, 1, 1};
    const int64_t tiles = workgroups(1, 1);
    p.waves = waves_of(tiles, 16 * num_cu, 16, 1);
    for (int more = 2; more <= (shift == 5 ? 2 : 4); more *= 2) {
        const int w = waves_of(tiles / more, 16 * num_cu, more * bytes <= 4 ? 16 : 8, 1);
        if (tiles / more * w < 16 * num_cu) break;
        p.strips = more;
        p.waves = w;
    }
    return p;
}

}  // namespace oz
