// Product of float16 rows with weights in 4 bits.
#include "oz_packed_gemm.h"

namespace oz {

void launch_packed_gemm_f16(hipStream_t st, const PackedGemm& g, int num_cu) { launch_typed<f16_t>(st, g, num_cu); }
bool prepare_packed_gemm_f16() { return allow_staged<f16_t, true>(); }

}  // namespace oz
