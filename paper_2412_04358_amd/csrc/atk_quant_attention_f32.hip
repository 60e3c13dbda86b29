#include "atk_quant_attention_kernel.h"

namespace atk {
hipError_t launch_quant_f32(const QuantAttnDev &d, int bits, int dp, int rt, bool join, hipStream_t stream) { return launch_quant_elt<ATK_F32>(d, bits, dp, rt, join, stream); }
}  // namespace atk
