// C ABI of the attention half of a block (include/tasq.h): argument checks,
// then one launcher each.
#include <math.h>

#include "block_internal.h"
#include "floats.h"

namespace {

bool type_known(int t)
{
    return t == TASQ_TYPE_F32 || t == TASQ_TYPE_BF16 || t == TASQ_TYPE_F16;
}

bool aligned_to(const void *p, size_t bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0;
}

int status(hipError_t e) { return e == hipSuccess ? TASQ_OK : TASQ_ERR_HIP; }

int check_heads(const tasq_heads &h, int type, int dim, bool grad)
{
    if (h.batch < 0 || h.tokens < 0 || h.heads < 0 || h.positions < 0 || h.rot < 0 ||
        h.rot > dim || h.rot % 2)
        return TASQ_ERR_DIM;
    for (int i = 0; i < 3; ++i)
        if (h.x_stride[i] < 0 || (grad && h.dy_stride[i] < 0))
            return TASQ_ERR_DIM;
    // Units of a launch are counted in 32 bits, and so are tokens.
    if ((long long)h.batch * h.tokens > (1LL << 30) ||
        (long long)h.batch * h.tokens * ((h.heads + 3LL) / 4) > (1LL << 30))
        return TASQ_ERR_DIM;
    if (!aligned_to(h.weight, 4) || !aligned_to(h.dweight, 4))
        return TASQ_ERR_ALIGN;
    if ((long long)h.batch * h.tokens * h.heads == 0)
        return TASQ_OK;
    if (!h.x || !h.out || (grad && !h.dy) || (h.rot && (!h.cos || !h.sin)))
        return TASQ_ERR_NULL;
    const size_t es = (size_t)tasq::type_bytes(type);
    if (!aligned_to(h.x, es) || !aligned_to(h.out, es) || (grad && !aligned_to(h.dy, es)) ||
        !aligned_to(h.cos, 4) || !aligned_to(h.sin, 4) || !aligned_to(h.position, 4))
        return TASQ_ERR_ALIGN;
    return TASQ_OK;
}

int norm_rotate(const tasq_heads *jobs, int n, int type, int dim, float eps, int interleaved,
                bool grad, void *workspace, size_t workspace_bytes, void *stream)
{
    if (n < 0 || n > TASQ_MAX_NORM_JOBS || !(eps >= 0.0f) || isinf(eps))
        return TASQ_ERR_RANGE;
    if (!type_known(type))
        return TASQ_ERR_KIND;
    if (dim < 2 || dim > TASQ_MAX_NORM_DIM || dim % 2)
        return TASQ_ERR_DIM;
    if (n == 0)
        return TASQ_OK;
    if (!jobs)
        return TASQ_ERR_NULL;
    tasq::HeadCall call{};
    call.n = n;
    call.type = type;
    call.dim = dim;
    call.interleaved = interleaved != 0;
    call.eps = eps;
    for (int i = 0; i < n; ++i) {
        const tasq_heads &h = jobs[i];
        if (int rc = check_heads(h, type, dim, grad))
            return rc;
        tasq::HeadJob &j = call.job[i];
        j.x = h.x;
        j.dy = h.dy;
        j.out = h.out;
        j.weight = h.weight;
        j.dweight = h.dweight;
        j.cos = h.cos;
        j.sin = h.sin;
        j.position = h.position;
        const int extent[3] = {h.batch, h.tokens, h.heads};
        for (int k = 0; k < 3; ++k) {
            j.x_stride[k] = extent[k] > 1 ? h.x_stride[k] : 0;
            j.dy_stride[k] = grad && extent[k] > 1 ? h.dy_stride[k] : 0;
        }
        j.batch = h.batch;
        j.tokens = h.tokens;
        j.heads = h.heads;
        j.positions = h.positions;
        j.rot = h.rot;
    }
    if (grad) {
        if (!aligned_to(workspace, 256))
            return TASQ_ERR_ALIGN;
        if (!workspace || workspace_bytes < tasq_norm_rotate_workspace_bytes(n, dim))
            return TASQ_ERR_WORKSPACE;
    }
    return status(tasq::launch_norm_rotate(call, grad, static_cast<float *>(workspace),
                                           static_cast<hipStream_t>(stream)));
}

}  // namespace

extern "C" {

int tasq_quantize_tokens(const void *x, int x_type, int M, int K, long long x_stride,
                         int8_t *X_out, float *sx_out, void *stream)
{
    if (!type_known(x_type))
        return TASQ_ERR_KIND;
    if (M < 0 || K < 0 || (M > 1 && x_stride < K))
        return TASQ_ERR_DIM;
    if (K > TASQ_MAX_K)
        return TASQ_ERR_OVERFLOW;
    if (M == 0)
        return TASQ_OK;
    if (!sx_out || (K > 0 && (!x || !X_out)))
        return TASQ_ERR_NULL;
    if (!aligned_to(x, (size_t)tasq::type_bytes(x_type)) || !aligned_to(sx_out, 4))
        return TASQ_ERR_ALIGN;
    return status(tasq::launch_quantize_tokens(x, x_type, M, K, M > 1 ? x_stride : K, X_out,
                                               sx_out, static_cast<hipStream_t>(stream)));
}

int tasq_masked_linear_tokens(const int8_t *X, const float *sx, const int8_t *W, const float *sw,
                              const float *bias, int M, int N, int K, int b, void *y_out,
                              int y_type, void *stream)
{
    if (!type_known(y_type))
        return TASQ_ERR_KIND;
    if (M < 0 || N < 0 || K < 0)
        return TASQ_ERR_DIM;
    if (K > TASQ_MAX_K)
        return TASQ_ERR_OVERFLOW;
    if (b < 1 || b > 8)
        return TASQ_ERR_BITS;
    if (M == 0 || N == 0)
        return TASQ_OK;
    if (!sx || !sw || !y_out || (K > 0 && (!X || !W)))
        return TASQ_ERR_NULL;
    if (!aligned_to(sx, 4) || !aligned_to(sw, 4) || !aligned_to(bias, 4) ||
        !aligned_to(y_out, (size_t)tasq::type_bytes(y_type)))
        return TASQ_ERR_ALIGN;
    tasq::TokenLinear t{X, W, sx, sw, bias, y_out, M, N, K, b, y_type};
    return status(tasq::launch_linear_tokens(t, static_cast<hipStream_t>(stream)));
}

size_t tasq_norm_rotate_workspace_bytes(int n, int dim)
{
    if (n <= 0 || n > TASQ_MAX_NORM_JOBS || dim <= 0 || dim > TASQ_MAX_NORM_DIM)
        return 0;
    return (size_t)n * tasq::kHeadGroups * (size_t)dim * sizeof(float);
}

int tasq_norm_rotate(const tasq_heads *jobs, int n, int type, int dim, float eps,
                     int interleaved, void *stream)
{
    return norm_rotate(jobs, n, type, dim, eps, interleaved, false, nullptr, 0, stream);
}

int tasq_norm_rotate_backward(const tasq_heads *jobs, int n, int type, int dim, float eps,
                              int interleaved, void *workspace, size_t workspace_bytes,
                              void *stream)
{
    return norm_rotate(jobs, n, type, dim, eps, interleaved, true, workspace, workspace_bytes,
                       stream);
}

}  // extern "C"
