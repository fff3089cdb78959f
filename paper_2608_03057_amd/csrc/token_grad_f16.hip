// The token-scaled linear's gradient in half (token_grad.h).
#include "token_grad.h"

namespace tasq {

hipError_t token_grad_f16(const GradJob &g, bool turned_a, bool whole, hipStream_t stream)
{
    return run_product<f16_t>(g, turned_a, whole, stream);
}

hipError_t token_grads_f16(const GradJob *x, const GradJob *w, int groups, bool whole,
                           hipStream_t stream)
{
    return run_products<f16_t>(x, w, groups, whole, stream);
}

}  // namespace tasq
