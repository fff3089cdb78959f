// Forward attention of bfloat16 heads.
#include "attn_fwd.h"

namespace tasq {
hipError_t attn_forward_bf16(const AttnCall &a, hipStream_t stream)
{
    return attn_forward_typed<bf16_t>(a, stream);
}
}  // namespace tasq
