// Large products with float32 scales: 256 x 128 tiles, results of the matrix instruction and sums in ordinary registers.
#include "oz_scaled_gemm_big.h"

namespace oz {

bool prepare_scaled_gemm_f32() { return prepare<2, Scales::kBlocks>() && prepare<2, Scales::kRows>(); }

void launch_scaled_gemm_big_f32(hipStream_t st, const ScaledGemm& g) {
    if (g.b.shift == 7) launch<2, Scales::kBlocks>(st, g);
    else launch<2, Scales::kRows>(st, g);
}

}  // namespace oz
