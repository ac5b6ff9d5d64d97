// plan KIND M N K GROUPS BY_ROWS BY_K: route, parts, waves, and the fitted time of each route
#include <cstdio>
#include <cstdlib>

#include "oz_scaled_plan.h"

int main(int argc, char** argv) {
    for (int i = 1; i + 6 < argc; i += 7) {
        long v[7];
        for (int j = 0; j < 7; ++j) v[j] = std::atol(argv[i + j]);
        const oz::ScaledPlan p = oz::scaled_plan(int(v[0]), v[1], v[2], v[3], v[4], v[5] != 0, v[6] != 0, 256);
        std::printf("%d %d %d", int(p.route), p.parts, p.waves);
        for (int r = 0; r < 5; ++r) std::printf(" %.3f", oz::route_time(int(v[0]), r, v[1], v[2], oz::div_up(v[3], 128), 1, 1, 256));
        std::printf("\n");
    }
    return 0;
}
