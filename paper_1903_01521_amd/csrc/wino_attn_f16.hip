// Attention kernels of 16-bit floating point tensors.
#include "wino_attn_device.h"

namespace wino {

hipError_t attn_f16(const AttnK& g, const AttnPlan& p, bool backward, hipStream_t st) {
    return attn_run_any<_Float16>(g, p, backward, st);
}

}  // namespace wino
