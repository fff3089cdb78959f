// C ABI of what stands around a block's quantized linears (include/tasq.h):
// argument checks, then one launcher each.
#include <math.h>

#include "branch_internal.h"
#include "floats.h"

namespace {

constexpr int kMostRows = 1 << 30;  // rounded up to tiles in 32 bits

bool type_known(int t)
{
    return t == TASQ_TYPE_F32 || t == TASQ_TYPE_BF16 || t == TASQ_TYPE_F16;
}

bool aligned_to(const void *p, size_t bytes)
{
    return reinterpret_cast<uintptr_t>(p) % bytes == 0;
}

int status(hipError_t e) { return e == hipSuccess ? TASQ_OK : TASQ_ERR_HIP; }

bool finite(float v) { return !isnan(v) && !isinf(v); }

// Sizes that tasq_residual_norm_workspace_bytes needs to be valid.
bool residual_sizes(int batch, int tokens, int width)
{
    return batch >= 0 && batch <= TASQ_MAX_RESIDUAL_BATCH && tokens >= 0 && width >= 0 &&
           width <= TASQ_MAX_RESIDUAL_WIDTH && (long long)batch * tokens <= kMostRows;
}

int residual_norm(const tasq_residual *a, bool grad, void *stream)
{
    if (!a)
        return TASQ_ERR_NULL;
    if (!type_known(a->type) || (a->mod_type != TASQ_TYPE_F32 && a->mod_type != a->type) ||
        (a->kind != TASQ_NORM_LAYER && a->kind != TASQ_NORM_RMS))
        return TASQ_ERR_KIND;
    if (!(a->eps >= 0.0f) || !finite(a->eps) || !finite(a->residual_scale) ||
        (a->shared & ~(TASQ_SHARED_GATE | TASQ_SHARED_SCALE | TASQ_SHARED_SHIFT)))
        return TASQ_ERR_RANGE;
    if (!residual_sizes(a->batch, a->tokens, a->width))
        return TASQ_ERR_DIM;
    tasq::NormCall c{};
    const int extent[2] = {a->batch, a->tokens};
    const long long *in[4] = {a->x_stride, a->y_stride, a->dh_stride, a->dr_stride};
    long long *out[4] = {c.x_stride, c.y_stride, c.dh_stride, c.dr_stride};
    const bool used[4] = {true, a->y != nullptr, grad, grad && a->dr};
    for (int t = 0; t < 4; ++t)
        for (int i = 0; i < 2; ++i) {
            if (!used[t] || extent[i] < 2)
                continue;
            if (in[t][i] < 0)
                return TASQ_ERR_DIM;
            out[t][i] = in[t][i];
        }
    // A factor of the branch does nothing without one.
    const void *gate = a->y ? a->gate : nullptr;
    const float *post = a->y ? a->post_weight : nullptr;
    const void *mods[3] = {gate, a->scale, a->shift};
    const long long strides[3] = {a->gate_stride, a->scale_stride, a->shift_stride};
    tasq::Modulation *to[3] = {&c.gate, &c.scale, &c.shift};
    for (int i = 0; i < 3; ++i) {
        const bool each = a->batch > 1 && !(a->shared & (1 << i));
        if (mods[i] && each && strides[i] < 0)
            return TASQ_ERR_DIM;
        *to[i] = {mods[i], each ? strides[i] : 0};
    }
    const bool none = (long long)a->batch * a->tokens * a->width == 0;
    float *sums[5] = {a->dgate, a->dscale, a->dshift, a->dweight, a->dpost_weight};
    if (!a->y && !none)         // (an empty y may be NULL: its gate's gradient is zeros)
        sums[0] = sums[4] = nullptr;
    bool some_sum = false;
    for (int i = 0; grad && i < 5; ++i) {
        if (!aligned_to(sums[i], 4))
            return TASQ_ERR_ALIGN;
        some_sum = some_sum || sums[i];
    }
    if (none && !(some_sum && a->width))
        return TASQ_OK;
    const size_t es = (size_t)tasq::type_bytes(a->type), ms = (size_t)tasq::type_bytes(a->mod_type);
    if (!none) {
        if (!a->x || (grad ? !a->dh || !a->dx || (a->y && !a->dy) : !a->h || (a->y && !a->r)))
            return TASQ_ERR_NULL;
        const void *wide[] = {a->x, a->y, grad ? a->dh : a->h, grad ? a->dr : a->r,
                              grad ? a->dx : nullptr, grad ? a->dy : nullptr};
        for (const void *p : wide)
            if (!aligned_to(p, es))
                return TASQ_ERR_ALIGN;
    }
    if (!aligned_to(gate, ms) || !aligned_to(a->scale, ms) || !aligned_to(a->shift, ms) ||
        !aligned_to(a->weight, 4) || !aligned_to(post, 4))
        return TASQ_ERR_ALIGN;
    if (some_sum) {
        if (!aligned_to(a->workspace, 256))
            return TASQ_ERR_ALIGN;
        const size_t need = tasq_residual_norm_workspace_bytes(a->batch, a->tokens, a->width);
        if (need && (!a->workspace || a->workspace_bytes < need))
            return TASQ_ERR_WORKSPACE;
        c.part = static_cast<float *>(a->workspace);
    }
    c.x = a->x;
    c.y = a->y;
    c.dh = a->dh;
    c.dr = a->dr;
    c.weight = a->weight;
    c.post_weight = post;
    c.r = a->r;
    c.h = a->h;
    c.dx = a->dx;
    c.dy = a->dy;
    c.dgate = sums[0];
    c.dscale = sums[1];
    c.dshift = sums[2];
    c.dweight = sums[3];
    c.dpost = sums[4];
    c.sums = some_sum;
    c.type = a->type;
    c.wide_mods = a->mod_type == TASQ_TYPE_F32;
    c.layer = a->kind == TASQ_NORM_LAYER;
    c.batch = a->batch;
    c.tokens = a->tokens;
    c.width = a->width;
    c.shared = a->shared;
    c.eps = a->eps;
    c.alpha = a->y ? a->residual_scale : 1.0f;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return status(grad ? tasq::launch_residual_norm_backward(c, st)
                       : tasq::launch_residual_norm(c, st));
}

constexpr size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// Tiles and ranges of a product [R][C] over Z, and the bytes of its workspace.
size_t plan_grad(tasq::GradJob &g, bool bias, bool cut)
{
    const int steps = (int)((g.Z + 63LL) / 64);
    auto tiles = [&](int t) { return ((g.R + t - 1LL) / t) * ((g.C + t - 1LL) / t); };
    g.tile = 64;
    g.splits = 1;
    for (const int t : {256, 128, 64}) {
        const long long n = tiles(t);
        long long s = n > 0 && cut ? 256 / n : 1;
        s = s < 1 ? 1 : s > steps / 8 ? (steps / 8 > 1 ? steps / 8 : 1) : s;
        g.tile = t;
        g.splits = (int)s;
        if (n * s >= 128)
            break;
    }
    g.tiles_r = (int)((g.R + g.tile - 1LL) / g.tile);
    g.tiles_c = (int)((g.C + g.tile - 1LL) / g.tile);
    if (bias && g.tiles_c == 0)
        g.tiles_c = 1;          // the rows' sums alone
    g.split_steps = (steps + g.splits - 1) / g.splits;
    if (g.split_steps > 0)
        g.splits = (steps + g.split_steps - 1) / g.split_steps;
    if (g.splits <= 1)
        return 0;
    return round256((size_t)g.splits * g.R * g.C * sizeof(float)) +
           round256((size_t)g.splits * g.R * sizeof(float));
}

// The two products: of dx (turned false) and of dw.
tasq::GradJob grad_job(int M, int N, int K, bool turned)
{
    tasq::GradJob g{};
    g.R = turned ? N : M;
    g.Z = turned ? M : N;
    g.C = K;
    return g;
}

bool grad_sizes(int M, int N, int K)
{
    return M >= 0 && M <= kMostRows && N >= 0 && N <= kMostRows && K >= 0;
}

}  // namespace

extern "C" {

int tasq_residual_norm(const tasq_residual *a, void *stream)
{
    return residual_norm(a, false, stream);
}

int tasq_residual_norm_backward(const tasq_residual *a, void *stream)
{
    return residual_norm(a, true, stream);
}

size_t tasq_residual_norm_workspace_bytes(int batch, int tokens, int width)
{
    if (!residual_sizes(batch, tokens, width) || (long long)batch * tokens == 0)
        return 0;
    return (size_t)batch * (size_t)tasq::residual_norm_chunks(batch, tokens, width) * 3 *
           (size_t)width * sizeof(float);
}

int tasq_quantize_mx4(const void *x, int x_type, int M, int K, long long x_stride,
                      uint8_t *codes_out, uint8_t *scales_out, void *stream)
{
    if (!type_known(x_type))
        return TASQ_ERR_KIND;
    if (M < 0 || M > kMostRows || K < 0 || (M > 1 && x_stride < K))
        return TASQ_ERR_DIM;
    if (K > TASQ_MAX_K)
        return TASQ_ERR_OVERFLOW;
    if (M == 0 || K == 0)
        return TASQ_OK;
    if (!x || !codes_out || !scales_out)
        return TASQ_ERR_NULL;
    if (!aligned_to(x, (size_t)tasq::type_bytes(x_type)) || !aligned_to(codes_out, 16) ||
        !aligned_to(scales_out, 4))
        return TASQ_ERR_ALIGN;
    return status(tasq::launch_quantize_mx4(x, x_type, M, K, M > 1 ? x_stride : K, codes_out,
                                            scales_out, static_cast<hipStream_t>(stream)));
}

int tasq_linear_mx4(const uint8_t *X, const uint8_t *sx, const uint8_t *W, const uint8_t *sw,
                    const float *bias, int M, int N, int K, void *y_out, int y_type, void *stream)
{
    if (!type_known(y_type))
        return TASQ_ERR_KIND;
    if (M < 0 || M > kMostRows || N < 0 || N > kMostRows || K < 0 || K % 128)
        return TASQ_ERR_DIM;
    if (K > TASQ_MAX_K + 1)
        return TASQ_ERR_OVERFLOW;
    if (M == 0 || N == 0)
        return TASQ_OK;
    if (!y_out || (K > 0 && (!X || !sx || !W || !sw)))
        return TASQ_ERR_NULL;
    if (!aligned_to(X, 16) || !aligned_to(W, 16) || !aligned_to(sx, 4) || !aligned_to(sw, 4) ||
        !aligned_to(bias, 4) || !aligned_to(y_out, (size_t)tasq::type_bytes(y_type)))
        return TASQ_ERR_ALIGN;
    tasq::Mx4Linear a{X, sx, W, sw, bias, y_out, M, N, K / 128, y_type};
    return status(tasq::launch_mx4_linear(a, static_cast<hipStream_t>(stream)));
}

size_t tasq_masked_linear_tokens_backward_workspace_bytes(int M, int N, int K)
{
    if (!grad_sizes(M, N, K) || K > TASQ_MAX_K)
        return 0;
    size_t most = 0;
    for (const bool turned : {false, true}) {
        tasq::GradJob g = grad_job(M, N, K, turned);
        const size_t bytes = plan_grad(g, turned, true);
        most = bytes > most ? bytes : most;
    }
    return most;
}

int tasq_masked_linear_tokens_backward(const void *dy, int type, long long dy_stride,
                                       const int8_t *X, const float *sx, const int8_t *W,
                                       const float *sw, int M, int N, int K, int b, void *dx,
                                       void *dw, float *dbias, void *workspace,
                                       size_t workspace_bytes, void *stream)
{
    if (type != TASQ_TYPE_BF16 && type != TASQ_TYPE_F16)
        return TASQ_ERR_KIND;
    if (!grad_sizes(M, N, K) || (M > 1 && dy_stride < N))
        return TASQ_ERR_DIM;
    if (K > TASQ_MAX_K)
        return TASQ_ERR_OVERFLOW;
    if (b < 1 || b > 8)
        return TASQ_ERR_BITS;
    if (!dw && dbias && N > 0 && K > 0)
        return TASQ_ERR_NULL;
    const bool want_x = dx && M > 0 && K > 0, want_w = (dw && N > 0 && K > 0) || (dbias && N > 0);
    if (!want_x && !want_w)
        return TASQ_OK;
    if (M > 0 && N > 0 && (!dy || (want_x && (!W || !sw)) || (want_w && K > 0 && (!X || !sx))))
        return TASQ_ERR_NULL;
    if (!aligned_to(dy, 2) || !aligned_to(dx, 2) || !aligned_to(dw, 2) || !aligned_to(dbias, 4) ||
        !aligned_to(sx, 4) || !aligned_to(sw, 4) || !aligned_to(workspace, 256))
        return TASQ_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const size_t have = workspace ? workspace_bytes : 0;
    for (const bool turned : {false, true}) {
        if (!(turned ? want_w : want_x))
            continue;
        tasq::GradJob g = grad_job(M, N, K, turned);
        g.A = dy;
        g.a_stride = M > 1 ? dy_stride : N;
        g.Q = turned ? X : W;
        g.s = turned ? sx : sw;
        g.mask = turned ? 0xffffffffu : tasq::keep_mask_dword(b);
        g.out = turned ? dw : dx;
        g.dbias = turned ? dbias : nullptr;
        if (plan_grad(g, g.dbias, true) > have)
            plan_grad(g, g.dbias, false);
        if (g.splits > 1) {
            g.part = static_cast<float *>(workspace);
            g.bias_part = g.part + round256((size_t)g.splits * g.R * g.C * sizeof(float)) / 4;
        }
        // (Offsets within a tile of A are 32-bit.)
        const bool whole = N % 8 == 0 && g.a_stride % 8 == 0 && K % 16 == 0 &&
                           aligned_to(dy, 16) && aligned_to(g.Q, 16) && g.a_stride < (1 << 22);
        const hipError_t e = type == TASQ_TYPE_BF16 ? tasq::token_grad_bf16(g, turned, whole, st)
                                                    : tasq::token_grad_f16(g, turned, whole, st);
        if (e != hipSuccess)
            return TASQ_ERR_HIP;
    }
    return TASQ_OK;
}

}  // extern "C"
