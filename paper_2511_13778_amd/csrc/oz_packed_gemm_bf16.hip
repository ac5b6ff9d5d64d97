// Product of bfloat16 rows with weights in 4 bits.
#include "oz_packed_gemm.h"

namespace oz {

void launch_packed_gemm_bf16(hipStream_t st, const PackedGemm& g, int num_cu) { launch_typed<bf16_t>(st, g, num_cu); }

}  // namespace oz
