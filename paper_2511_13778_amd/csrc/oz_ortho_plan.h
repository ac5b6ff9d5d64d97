// Which tiles the products of an orthogonal update take.  Host code alone: tests build it without a GPU.
#pragma once

#include <stdint.h>

#include <algorithm>

namespace oz {

struct OrthoTiles { int square, apply; };      // sides of the tiles of A and A^2, and of P X

// Time of one product, in us: `tiles` of `steps` times 64 of k on 256 CUs, in rounds of as many as a CU holds.  Constants fitted to 840 products of 40
// shapes from 48 to 4096 (7 to 13 % off; the choice made with them costs 0.6 % over the best of each, 10 % at most).
struct OrthoCost {
    int side, held;
    double latency, busy;              // a step: of one tile alone, of each tile that shares the CU
    double end, end_apply, end_more;   // what a tile's sums become; of P X; for each further tile on the CU
    double base;
};
inline double ortho_time(const OrthoCost& c, int64_t tiles, int64_t steps, bool apply, int num_cu) {
    const int64_t per = (tiles + num_cu - 1) / num_cu, full = per / c.held, rest = per % c.held;
    auto round = [&](int64_t n) { return double(steps) * std::max(c.latency, double(n) * c.busy) + (apply ? c.end_apply : c.end) + double(n - 1) * c.end_more; };
    return c.base + double(full) * round(c.held) + (rest ? round(rest) : 0.0);
}

// parts: 16-bit parts of an operand.  m <= n.
inline OrthoTiles ortho_tiles(int64_t batch, int64_t m, int64_t n, int parts, int num_cu) {
    static const OrthoCost costs[2][4] = {{{64, 2, 0.273, 0.198, 0.71, 1.91, 1.95, 2.23}, {128, 2, 0.02, 0.402, 4.2, 7.9, 6.3, 0.0},
                                           {192, 1, 0.786, 0.636, 6.7, 13.1, 0.0, 0.0}, {256, 1, 1.25, 0.87, 9.7, 21.1, 0.0, 0.0}},
                                          {{64, 1, 0.185, 0.545, 2.9, 4.3, 0.0, 0.7}, {128, 2, 0.431, 0.356, 6.4, 10.7, 19.8, 0.0},
                                           {192, 1, 0.755, 0.338, 10.9, 19.4, 0.0, 0.0}, {256, 1, 0.643, 1.171, 19.3, 31.9, 0.0, 0.0}}};
    OrthoTiles best{64, 64};
    double square = 1e30, apply = 1e30;
    for (const OrthoCost& c : costs[parts - 1]) {
        const int64_t tm = (m + c.side - 1) / c.side, tn = (n + c.side - 1) / c.side, half = tm * (tm + 1) / 2 * batch;
        // large tiles walk through two parts' three products one after the other
        const int64_t passes = parts == 2 && c.side > 64 ? 3 : 1, steps_m = (m + 63) / 64 * passes, steps_n = (n + 63) / 64 * passes;
        const double s = ortho_time(c, half, steps_n, false, num_cu) + ortho_time(c, half, steps_m, false, num_cu);
        const double a = ortho_time(c, tm * tn * batch, steps_m, true, num_cu);
        if (s < square) square = s, best.square = c.side;
        if (a < apply) apply = a, best.apply = c.side;
    }
    return best;
}

}  // namespace oz
