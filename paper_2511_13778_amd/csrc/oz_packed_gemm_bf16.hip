// Product of bfloat16 rows with weights in 4 bits.
#include "oz_packed_gemm.h"

namespace oz {

void launch_packed_gemm_bf16(hipStream_t st, const PackedGemm& g, int num_cu) { launch_typed<bf16_t>(st, g, num_cu); }
bool prepare_packed_gemm_bf16() { return allow_staged<bf16_t, true>() && allow_staged<bf16_t, false>(); }

}  // namespace oz
