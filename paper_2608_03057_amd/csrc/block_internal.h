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
    int first_block;            // of the launch
};
// part: n * kHeadGroups * dim floats (grad only).
hipError_t launch_norm_rotate(const HeadCall &call, bool grad, float *part, hipStream_t stream);

// Attention (attn_fwd.h, attn_bwd.h).  Rows are (query head of the group,
// query) pairs of one key head; a workgroup has 128 rows (256 in the forward
// pass with row_blocks 2), or 128 keys in k_attn_dkdv.  plan_attention sets
// the launch's shape.
// 16-element steps of a head that row_blocks 2 takes.
constexpr int kAttnWideFrom = 3, kAttnWideSteps = 5;
struct AttnCall {
    const void *q, *k, *v;
    const int32_t *kv_lengths;  // [batch] or null
    const uint8_t *key_mask;    // [batch][kv_len] or null
    void *out;                  // [batch][q_len][heads][dim]
    float *lse;                 // [batch][heads][q_len], null if not wanted
    const void *dout;           // backward
    void *dq, *dk, *dv;
    long long q_stride[3], k_stride[3], v_stride[3], dout_stride[3];    // batch, token, head
    int type, batch, heads, kv_heads, q_len, kv_len, dim;
    float scale, scale_log2;    // scale, and scale * log2(e)
    int row_blocks;                                 // blocks of 32 rows of a wave
    int row_tiles, splits, split_tiles;             // ranges of the keys, in tiles of 64
    int key_tiles, kv_splits, kv_split_tiles;       // ranges of the rows (k_attn_dkdv)
    float *part, *part_lse;     // [splits][batch][..] parts of out (or dq) and lse
    float *kv_part;             // [kv_splits][2][batch][kv_len][kv_heads][dim]
    float *delta;               // [batch][heads][q_len]
    int first_unit;             // of the launch
};

// The kernel in launches of at most 2^22 workgroups: one has fewer than 2^32
// threads.
inline hipError_t launch_units(void (*kernel)(AttnCall), AttnCall a, long long units,
                               hipStream_t stream)
{
    constexpr long long MOST = 1 << 22;
    hipError_t e = hipSuccess;
    for (long long u = 0; u < units && e == hipSuccess; u += MOST) {
        a.first_unit = (int)u;
        kernel<<<(unsigned)(units - u < MOST ? units - u : MOST), 256, 0, stream>>>(a);
        e = hipGetLastError();
    }
    return e;
}

hipError_t attn_forward_bf16(const AttnCall &a, hipStream_t stream);
hipError_t attn_forward_f16(const AttnCall &a, hipStream_t stream);
hipError_t attn_backward_bf16(const AttnCall &a, hipStream_t stream);
hipError_t attn_backward_f16(const AttnCall &a, hipStream_t stream);

}  // namespace tasq
