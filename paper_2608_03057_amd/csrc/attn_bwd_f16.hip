// Backward attention of half heads.
#include "attn_bwd.h"

namespace tasq {
hipError_t attn_backward_f16(const AttnCall &a, hipStream_t stream)
{
    return attn_backward_typed<f16_t>(a, stream);
}
}  // namespace tasq
