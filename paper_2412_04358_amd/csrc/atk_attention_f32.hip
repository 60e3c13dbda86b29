// Instances of the attention kernels for f32.
#include "atk_attention_kernel.h"

namespace atk {
hipError_t launch_attn_f32(const AttnDev &a, int dp, int rt, int waves, hipStream_t stream) { return launch_attn<ATK_F32>(a, dp, rt, waves, stream); }
}  // namespace atk
