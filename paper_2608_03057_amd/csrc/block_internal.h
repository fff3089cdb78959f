// Internal declarations of the attention half of a block: token-scaled
// linears, the norm and rotation of heads, and attention.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tasq.h"
#include "tasq_internal.h"

namespace tasq {

// Symmetric 8-bit codes with one scale per row (token_quant.hip).
hipError_t launch_quantize_tokens(const void *x, int type, int M, int K, long long stride,
                                  int8_t *q, float *sx, hipStream_t stream);

// y = (X W_b^T) sx[m] sw[n] + bias[n] (token_gemm.hip).
struct TokenLinear {
    const int8_t *X, *W;
    const float *sx, *sw, *bias;
    void *y;
    int M, N, K, bits, type;
};
hipError_t launch_linear_tokens(const TokenLinear &t, hipStream_t stream);

// The norm and rotation of heads (head_norm.hip).
constexpr int kMaxHeadDim = TASQ_MAX_NORM_DIM;
// Most workgroups of the gradient, each with one partial dw per job.
constexpr int kHeadGroups = 1024;

struct HeadJob {
    const void *x, *dy;
    void *out;
    const float *weight;
    float *dweight;
    const float *cos, *sin;
    const int32_t *position;
    long long x_stride[3], dy_stride[3];
    int batch, tokens, heads, positions, rot;
    int units;                  // set by launch_norm_rotate
};
struct HeadCall {
    HeadJob job[2];
    int n, type, dim, interleaved;
    float eps;
    float inv_dim;              // set by launch_norm_rotate
};
// part: n * kHeadGroups * dim floats (grad only).
hipError_t launch_norm_rotate(const HeadCall &call, bool grad, float *part, hipStream_t stream);

}  // namespace tasq
