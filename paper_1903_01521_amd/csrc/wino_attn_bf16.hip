// Attention kernels of bfloat16 tensors.
#include "wino_attn_device.h"

namespace wino {

hipError_t attn_bf16(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    return attn_run_any<__bf16>(g, p, backward, st);
}

}  // namespace wino
