// The token-scaled linear's gradient in bfloat16 (token_grad.h).
#include "token_grad.h"

namespace tasq {

hipError_t token_grad_bf16(const GradJob &g, bool turned_a, bool whole, hipStream_t stream)
{
    return run_product<bf16_t>(g, turned_a, whole, stream);
}

hipError_t token_grads_bf16(const GradJob *x, const GradJob *w, int groups, bool whole,
                            hipStream_t stream)
{
    return run_products<bf16_t>(x, w, groups, whole, stream);
}

}  // namespace tasq
