// Instances of the attention kernels for bf16.
#include "atk_attention_kernel.h"

namespace atk {
hipError_t launch_attn_bf16(const AttnDev &a, int dp, int rt, int waves, hipStream_t stream) { return launch_attn<ATK_BF16>(a, dp, rt, waves, stream); }
}  // namespace atk
