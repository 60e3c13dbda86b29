#include "atk_quant_attention_kernel.h"

namespace atk {
hipError_t launch_quant_f32(const QuantAttnDev &d, int bits, int dp, int rt, int mode, hipStream_t stream) { return launch_quant_elt<ATK_F32>(d, bits, dp, rt, mode, stream); }
}  // namespace atk
