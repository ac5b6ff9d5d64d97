// Product of float32 rows with weights in 4 bits.
#include "oz_packed_gemm.h"

namespace oz {

void launch_packed_gemm_f32(hipStream_t st, const PackedGemm& g, int num_cu) { launch_typed<float>(st, g, num_cu); }
bool prepare_packed_gemm_f32() { return allow_staged<float, true>(); }

}  // namespace oz
