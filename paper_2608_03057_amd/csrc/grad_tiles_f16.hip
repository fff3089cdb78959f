// The token-scaled linear's gradient over many tokens in half (grad_tiles.h).
#include "grad_tiles.h"

namespace tasq {

hipError_t grad_values_f16(const GradValues &v, hipStream_t stream)
{
    return write_values<f16_t>(v, stream);
}

hipError_t grad_gemm_f16(const GradGemm &g, bool turned_a, hipStream_t stream)
{
    return run_gemm<f16_t>(g, turned_a, stream);
}

}  // namespace tasq
