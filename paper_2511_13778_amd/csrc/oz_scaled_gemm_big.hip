// Large products with E8M0 scales: 256 x 256 and 256 x 128 tiles, sums in the accumulation registers.
#include "oz_scaled_gemm_big.h"

namespace oz {

bool prepare_scaled_gemm() { return prepare<4, Scales::kE8M0>() && prepare<2, Scales::kE8M0>() && prepare_scaled_gemm_f32(); }

void launch_scaled_gemm_big(hipStream_t st, const ScaledGemm& g, bool square) {
    if (!g.e8m0) launch_scaled_gemm_big_f32(st, g);
    else if (square) launch<4, Scales::kE8M0>(st, g);
    else launch<2, Scales::kE8M0>(st, g);
}

}  // namespace oz
