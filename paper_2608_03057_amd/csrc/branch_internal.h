// Internal declarations of what stands around a block's quantized linears: the
// norm of the residual stream, 4-bit microscaled linears, and the gradient of the
// token-scaled linear.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tasq.h"
#include "tasq_internal.h"

namespace tasq {

// The residual stream's norm and its gradient (residual_norm.hip).
struct Modulation {             // of entry b at p + b * stride
    const void *p;
    long long stride;
};
struct NormCall {
    const void *x, *y, *dh, *dr;
    long long x_stride[2], y_stride[2], dh_stride[2], dr_stride[2];     // batch, token
    Modulation gate, scale, shift;
    const float *weight, *post_weight;
    void *r, *h, *dx, *dy;
    float *dgate, *dscale, *dshift, *dweight, *dpost;
    int type, wide_mods;        // wide_mods: modulations are fp32, else of `type`
    int layer, batch, tokens, width, shared;
    float eps, alpha, inv_width;
    int rows, chunks;           // rows of a team's run; runs (backward: workgroups) an entry
    int waves, groups;          // of a row; rows of a workgroup at a time (backward)
    long long first_unit;       // of the launch
    float *part;                // backward: [batch][chunks][3][width]
    bool sums;                  // backward: some of dgate .. dpost are wanted
};
hipError_t launch_residual_norm(const NormCall &c, hipStream_t stream);
hipError_t launch_residual_norm_backward(const NormCall &c, hipStream_t stream);
// Waves of a row, rows at a time and workgroups for each batch entry of the gradient.
struct NormTeams {
    int waves, groups, chunks;
};
NormTeams residual_norm_teams(int type, int batch, int tokens, int width);

// 4-bit microscaled codes (mx4_quant.hip) and the linear on them (mx4_gemm.hip): rows
// of K128 * 128 elements, 64 bytes of codes and four scales each 128.
hipError_t launch_quantize_mx4(const void *x, int type, int M, int K, long long stride,
                               uint8_t *codes, uint8_t *scales, hipStream_t stream);
struct Mx4Linear {
    const uint8_t *X, *sx, *W, *sw;
    const float *bias;
    void *y;
    int M, N, K128, type;
};
hipError_t launch_mx4_linear(const Mx4Linear &a, hipStream_t stream);

// One product of the token-scaled linear's gradient (token_grad.h):
// out[r][c] = sum_z A(r, z) s[z] Q[z][c], A [R][Z], or [Z][R] turned.
struct GradJob {
    const void *A;
    long long a_stride;
    const int8_t *Q;            // [Z][C]
    const float *s;             // [Z]
    uint32_t mask;              // of four codes
    void *out;                  // [R][C]
    float *dbias;               // [R], turned only, or null
    int R, Z, C;
    int tile, tiles_r, tiles_c;         // 64, 128 or 256 rows and columns
    int splits, split_steps;            // ranges of Z, in steps of 64
    float *part, *bias_part;            // [splits][R][C], [splits][R]
};
// The same over many tokens (grad_tiles.h): Q's values in A's type.
struct GradGemm {
    const void *A, *Q;          // rows of whole 16-byte chunks; Q [Z][q_stride]
    long long a_stride;
    int q_stride;
    const float *back;          // factor of the sums, or null
    void *out;
    float *dbias;
    int R, Z, C;
    int tile_c, tiles_r, tiles_c;       // 256 rows by 256 or 192 columns
    int splits, split_steps;            // ranges of Z, in steps of 32
    float *part, *bias_part;
};
// Rows to be written as whole chunks of values: codes times factors, or values.
struct GradValues {
    struct Job {
        const int8_t *q;        // [rows][width], or null: from
        const float *s;         // [rows]
        uint32_t mask;
        float *back;            // receives the factor of the sums (half)
        const void *from;
        long long from_stride;
        void *to;               // [rows][to_stride]
        int rows, width, to_stride;
    } job[3];
    int n;
};
hipError_t grad_values_bf16(const GradValues &v, hipStream_t stream);
hipError_t grad_values_f16(const GradValues &v, hipStream_t stream);
hipError_t grad_gemm_bf16(const GradGemm &g, bool turned_a, hipStream_t stream);
hipError_t grad_gemm_f16(const GradGemm &g, bool turned_a, hipStream_t stream);

hipError_t token_grad_bf16(const GradJob &g, bool turned_a, bool whole, hipStream_t stream);
hipError_t token_grad_f16(const GradJob &g, bool turned_a, bool whole, hipStream_t stream);
// Products in one launch: dx's x, dw's w or (neither null) both, of one tile size: 64,
// with the range of a workgroup in 1 or 2 parts side by side, or both of 128.
hipError_t token_grads_bf16(const GradJob *x, const GradJob *w, int groups, bool whole,
                            hipStream_t stream);
hipError_t token_grads_f16(const GradJob *x, const GradJob *w, int groups, bool whole,
                           hipStream_t stream);

}  // namespace tasq
