// Attention kernels of 32-bit floating point tensors.
#include "wino_attn_device.h"

namespace wino {

hipError_t attn_f32(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    return attn_run_any<float>(g, p, backward, st);
}

}  // namespace wino
