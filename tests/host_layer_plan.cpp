// packed M N K GROUPS BYTES SHIFT: staged, rows, strips, waves.  ortho BATCH M N PARTS: tiles of the square products and of P X.
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "oz_ortho_plan.h"
#include "oz_packed_plan.h"

int main(int argc, char** argv) {
    long v[6] = {};
    for (int i = 2; i < argc && i < 8; ++i) v[i - 2] = std::atol(argv[i]);
    if (argc == 8 && !std::strcmp(argv[1], "packed")) {
        const oz::PackedPlan p = oz::packed_plan(v[0], v[1], v[2], v[3], int(v[4]), int(v[5]), 256);
        std::printf("%d %d %d %d\n", int(p.staged), p.rows, p.strips, p.waves);
        return 0;
    }
    if (argc == 6 && !std::strcmp(argv[1], "ortho")) {
        const oz::OrthoTiles t = oz::ortho_tiles(v[0], v[1], v[2], int(v[3]), 256);
        std::printf("%d %d\n", t.square, t.apply);
        return 0;
    }
    return 1;
}
