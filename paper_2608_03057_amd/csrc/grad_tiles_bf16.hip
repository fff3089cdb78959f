// The token-scaled linear's gradient over many tokens in bfloat16 (grad_tiles.h).
#include "grad_tiles.h"

namespace tasq {

hipError_t grad_values_bf16(const GradValues &v, hipStream_t stream)
{
    return write_values<bf16_t>(v, stream);
}

hipError_t grad_gemm_bf16(const GradGemm &g, bool turned_a, hipStream_t stream)
{
    return run_gemm<bf16_t>(g, turned_a, stream);
}

}  // namespace tasq
