// Backward attention of bfloat16 heads.
#include "attn_bwd.h"

namespace tasq {
hipError_t attn_backward_bf16(const AttnCall &a, hipStream_t stream)
{
    return attn_backward_typed<bf16_t>(a, stream);
}
}  // namespace tasq
