// Which kernel computes a product of 8-bit block-scaled matrices, by sizes and types alone; host code.
//
// Time of a route, in us:  3 + steps * (rounds of a full CU, and what is left) + each * c,  c = tiles / compute units, rounded up: a step of
// 128 of k takes `per` for each of the tiles that a CU has at a time (its matrix unit and LDS are shared), but no less than a lone
// tile takes, and a tile's first loads and its results cost `each`.  The constants are fits to times measured at twelve sizes from 256 x 1000 x 1000 to 8192^3: where a route
// is the best one within 13 % from 17 us on, up to 28 % too long for calls under 10 us, where the choice loses 3 %.  Tiles of 256 x 256 need the fewest bytes per operation and win on large outputs (8192^3 402 us, 256 x 128 462,
// 128 x 128 556), those of 128 x 128 and 64 x 64, several to a CU, overlap one's results with another's products and win on
// short k and where larger ones leave CUs idle (8192 x 8192 x 512 56 us, 256 x 256 62; 1024^3 6.2 us in 64 x 64, 9.6 in 128 x 128).
// 64 x 64 tiles that are alone on their CU take four stages: from memory two wait for each step's loads (200 x 2048 x 2048 15.2 us, with four 9.8,
// widened 15.4 and 12.3), from the caches two are ahead (9.0, 9.5), and `alone` of two stages is what they take from memory.  The launch
// gives them to parts of a k that is cut as well.
#pragma once

#include <algorithm>
#include <stddef.h>
#include <stdint.h>

namespace oz {

// Pieces of `size` that groups of `total` rows can be cut into at most, each group for itself (a group of its own for rows behind the last).
inline int64_t group_pieces(int64_t total, int64_t groups, int64_t size) {
    const int64_t g = groups + 1 < total ? groups + 1 : total;
    return (total + (size - 1) * g) / size;
}

enum class ScaledRoute { kFew, kTiles64, kTiles64Deep, kTiles128, kTall, kBig };

struct ScaledPlan {
    ScaledRoute route;
    int parts;         // of k
    int waves;         // kFew: of a workgroup
};

struct RouteCost { double alone, per, each; };

// [E8M0 scales, float32 scales, E8M0 widened, float32 widened][64 x 64, 64 x 64 with four stages, 128 x 128, 256 x 128, 256 x 256]
constexpr RouteCost kRouteCost[4][5] = {
    {{.49, .197, .40}, {.39, .25, .40}, {.785, .54, 1.2}, {.81, .81, 5.5}, {1.42, 1.42, 9.1}},
    {{.52, .226, .45}, {.48, .29, .45}, {.93, .675, 1.3}, {1.09, 1.09, 5.7}, {0, 0, 0}},
    {{.66, .298, .51}, {.575, .352, .51}, {1.14, .893, 1.8}, {0, 0, 0}, {0, 0, 0}},
    {{.70, .34, .51}, {.645, .40, .51}, {1.24, 1.09, 1.8}, {0, 0, 0}, {0, 0, 0}},
};

inline int64_t div_up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// m rows in `groups` groups (1: no groups) that tiles do not cross, each of about the same size; repeats: products of this size in the call.
inline double route_time(int kind, int route, int64_t m, int64_t n, int64_t blocks, int64_t groups, int64_t repeats, int num_cu) {
    static const int rows[5] = {64, 64, 128, 256, 256}, cols[5] = {64, 64, 128, 128, 256};
    const RouteCost& c = kRouteCost[kind][route];
    if (c.per == 0) return 1e30;
    // groups end inside a tile, and are not equally large: a tile more for each (16384 rows in 16 uneven groups, float32 scales: 256 x 128 tiles
    // 231 us and 234 by this count, 128 x 128 220 and 221)
    const double tiles_m = groups > 1 ? std::min(double(m) / rows[route] + double(groups), double(m)) : double(div_up(m, rows[route]));
    const double per_cu = double(div_up(int64_t(tiles_m * double(div_up(n, cols[route])) * double(repeats) + 0.5), num_cu));
    static const int together[5] = {4, 2, 2, 1, 1};
    const double full = double(int64_t(per_cu) / together[route] * together[route]), left = per_cu - full;
    return 3.0 + double(blocks) * (full * c.per + (left > 0 ? std::max(c.alone, left * c.per) : 0.0)) + c.each * per_cu;
}

// Rows of A that share a read of B, on average, up to which that read is what counts.
// (With groups the average decides: a group with many more rows reads its B once per 16, 32 or 64 of them.)
constexpr int kFewRows = 64;

// A product without groups may be cut along k: into how many parts is decided by its sizes alone, because the workspace is.
inline ScaledPlan cut_plan(int64_t m, int64_t n, int64_t k, int num_cu) {
    const int64_t blocks = div_up(k, 128), fours = div_up(blocks, 4);
    if (m <= kFewRows) {
        const int64_t strips = div_up(n, 16);
        const int64_t parts = std::max<int64_t>(1, std::min<int64_t>({num_cu / strips, fours / 8, 16}));
        const int64_t each = div_up(fours, parts);
        return ScaledPlan{ScaledRoute::kFew, int(parts), each <= 4 ? 4 : each <= 8 ? 8 : 16};
    }
    double best = 1e30;
    for (int r = 0; r < 5; ++r) best = std::min(best, route_time(0, r, m, n, blocks, 1, 1, num_cu));
    int parts = 1;
    for (int64_t p = 2; p <= 16 && p <= blocks / 4; p *= 2) {
        // a launch more, and the planes written and read
        const double t = route_time(0, 0, m, n, div_up(blocks, p), 1, p, num_cu) + 2.5 + double(p) * double(m) * double(n) * 8 / 5e6;
        if (t < 0.9 * best) {
            best = t / 0.9;
            parts = int(p);
        }
    }
    return ScaledPlan{ScaledRoute::kTiles64, parts, 0};
}

// kind: row of kRouteCost.  by_rows: m rows in `groups` groups; by_k: `groups` products of m x n, k their rows together.
inline ScaledPlan scaled_plan(int kind, int64_t m, int64_t n, int64_t k, int64_t groups, bool by_rows, bool by_k, int num_cu) {
    const int64_t rows = by_rows ? div_up(m, groups) : m;
    if (!by_k && rows <= kFewRows) {
        ScaledPlan p = cut_plan(rows, n, k, num_cu);
        if (by_rows) {
            p.parts = 1;
            p.waves = div_up(k, 512) <= 4 ? 4 : div_up(k, 512) <= 8 ? 8 : 16;
        }
        return p;
    }
    if (!by_rows && !by_k) {
        const ScaledPlan p = cut_plan(m, n, k, num_cu);
        if (p.parts > 1) return p;
    }
    const int64_t blocks = by_k ? div_up(div_up(k, 128), groups) : div_up(k, 128);
    int best = 0;
    for (int r = 1; r < 5; ++r)
        if (route_time(kind, r, m, n, blocks, by_rows ? groups : 1, by_k ? groups : 1, num_cu) <
            route_time(kind, best, m, n, blocks, by_rows ? groups : 1, by_k ? groups : 1, num_cu))
            best = r;
    return ScaledPlan{ScaledRoute(int(ScaledRoute::kTiles64) + best), 1, 0};
}

}  // namespace oz
