// Forward attention of half heads.
#include "attn_fwd.h"

namespace tasq {
hipError_t attn_forward_f16(const AttnCall &a, hipStream_t stream)
{
    return attn_forward_typed<f16_t>(a, stream);
}
}  // namespace tasq
