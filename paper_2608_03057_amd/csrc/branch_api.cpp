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
        const size_t need =
            tasq_residual_norm_workspace_bytes(a->type, a->batch, a->tokens, a->width);
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

// One product of the gradient, [R][C] over Z, and how it runs: of values over 256-row
// tiles, or of codes as they are.
struct GradPlan {
    int R, Z, C;
    int tile, tile_c;           // rows and columns of a tile
    int tiles_r, tiles_c, splits, split_steps;
    size_t parts;               // bytes of the ranges' parts
};

// Floats of a product's parts, before the bias'.
size_t part_floats(const GradPlan &p)
{
    return round256((size_t)p.splits * p.R * p.C * sizeof(float)) / sizeof(float);
}

long long units_of(const GradPlan &p) { return (long long)p.tiles_r * p.tiles_c * p.splits; }

int tiles_of(int n, int t) { return (int)((n + t - 1LL) / t); }

// Ranges of the sum: as many as give `units` workgroups, of at least `least` steps.
void cut_sum(GradPlan &p, int steps, int units, int least, bool cut)
{
    const long long n = (long long)p.tiles_r * p.tiles_c;
    long long s = n > 0 && cut ? units / n : 1;
    const int most = steps / least;
    s = s > most ? most : s;
    p.splits = s < 1 ? 1 : (int)s;
    p.split_steps = (steps + p.splits - 1) / p.splits;
    if (p.split_steps > 0)
        p.splits = (steps + p.split_steps - 1) / p.split_steps;
    if (p.splits < 1)
        p.splits = 1;
    p.parts = p.splits == 1 ? 0
                            : part_floats(p) * sizeof(float) +
                                  round256((size_t)p.splits * p.R * sizeof(float));
}

// Of codes.  Counted in tiles of 64 x 64 and their steps of 64, with three more for a
// tile's first loads and its result, small work is spread wide and large work kept in
// tiles that read less.  (Measured at tiles of 64 / 128 / 256, us with the joins: 576
// steps of 256 x 1152, 700 tokens, for dx 13 / 18 / 24; 1152 x 1152 over 2000 tokens
// 22 / 22 / 28; 9280 x 2288 over 400 tokens 48 / 38 / 37; 11144 x 2400 over 868 tokens
// 110 / 81 / 66.  Rows that are no whole chunks pass through registers, and a tile of 256
// is alone on its compute unit with that: 9273 x 2278 over 405 tokens 48 at 128, 93 at
// 256.)  Ranges of the sum: for 6 tokens of 10536 x 3344 tiles of 64 in 212 / 477 / 1007
// workgroups take 26 / 19 / 17 us for dx; tiles of 128 for 2000 tokens of 1152 x 1152 in up
// to 256 / 512 of each product 29 / 38 for both; below 24 steps the join's launch is more
// than the ranges save (700 x 1152 x 1152 17.3 / 12.5 without).
void plan_codes(GradPlan &p, bool bias, bool whole, bool cut, int groups = 1)
{
    const int steps = (int)((p.Z + 63LL) / 64);
    const long long work = (long long)tiles_of(p.R, 64) * tiles_of(p.C, 64) * (steps + 3);
    const int t = work < 9500 ? 64 : work < 36000 || !whole ? 128 : 256;
    p.tile = p.tile_c = t;
    p.tiles_r = tiles_of(p.R, t);
    p.tiles_c = tiles_of(p.C, t);
    if (bias && p.tiles_c == 0)
        p.tiles_c = 1;          // the rows' sums alone
    if (t == 64 && groups == 1)
        cut_sum(p, steps, 512, 4, cut && steps >= 24);
    else
        cut_sum(p, steps, 256, 8 * groups, cut);
}

// Both products of codes, and in how many parts side by side workgroups of tiles of 64
// have their range (alike for one product alone: the sums are the same).  Two where there
// are few workgroups: with ranges of their own instead they need a launch more.  (One / two
// parts, us a call: 1200 x 1152 x 640, 370 workgroups, 16.0 / 14.2; 1500 x 640 x 640, 340,
// 15.9 / 13.7; 700 x 1152 x 1152, 522, 12.5 / 15.4.  Four parts: 8000 x 128 x 128 21.5 for
// 15.8 of two.)
int plan_both(GradPlan (&plan)[2], bool bias, const bool (&whole)[2], bool cut)
{
    long long small = 0;
    for (const bool turned : {false, true}) {
        plan_codes(plan[turned], turned && bias, whole[turned], false);
        small += plan[turned].tile == 64 ? units_of(plan[turned]) : 0;
    }
    const int groups = small <= 416 ? 2 : 1;
    for (const bool turned : {false, true})
        plan_codes(plan[turned], turned && bias, whole[turned], cut,
                   plan[turned].tile == 64 ? groups : 1);
    return groups;
}

// Of values: tiles of 256 rows by the width that takes the least time, counted in
// rounds of one workgroup a compute unit.  (0.6 us a step of 256 x 256 x 32 and 4 for a
// tile's ends, parts at 4 TB/s.  192 / 256 columns: 8192 tokens, 1152 -> 3456, 72 / 85
// for dx and 92 / 102 for dw; 4096 tokens, 2240 -> 11200, 208 / 245 and 244 / 219.)
void plan_values(GradPlan &p, bool bias)
{
    const int steps = (int)((p.Z + 31LL) / 32);
    GradPlan best{};
    double least = 0;
    for (const int c : {256, 192}) {
        GradPlan q = p;
        q.tile = 256;
        q.tile_c = c;
        q.tiles_r = tiles_of(q.R, 256);
        q.tiles_c = tiles_of(q.C, c);
        if (bias && q.tiles_c == 0)
            q.tiles_c = 1;
        for (const int units : {256, 512}) {
            cut_sum(q, steps, units, 16, true);
            const long long n = (long long)q.tiles_r * q.tiles_c * q.splits;
            const double us = (double)((n + 255) / 256) * (q.split_steps * 0.6 * c / 256.0 + 4.0) +
                              (q.splits > 1 ? 2.0 + 2.0 * q.parts / 4e6 : 0.0);
            if (least == 0 || us < least) {
                least = us;
                best = q;
            }
        }
    }
    p = best;
}

// Values pay where there is work enough to fill such tiles and to make up for the pass
// that writes them.  (Codes / values, us of all kernels: 2000 x 1152 x 1152 52 / 52, 4096
// tokens of it 55 / 64, 8192 tokens 81 / 73; 2048 x 2240 x 2240 87 / 84; 512 x 4608 x 4608
// 82 / 80; 3001 x 4447 x 982 143 / 128.  With a copy of dy before it, rows at odd
// addresses: 520 x 4456 x 4408 78 / 90, 2048 x 2240 x 2400 87 / 90, 3000 x 2240 x 2400
// 114 / 102, 8192 x 3456 x 1152 259 / 169, 4096 x 11200 x 2240 581 / 439.)
bool values_pay(int M, int N, int K)
{
    return M >= 512 && N >= 256 && K >= 256 && (double)M * N * K >= 1e10;
}

// The two products: of dx (turned false) and of dw.
GradPlan grad_plan(int M, int N, int K, bool turned)
{
    GradPlan p{};
    p.R = turned ? N : M;
    p.Z = turned ? M : N;
    p.C = K;
    return p;
}

// Elements of a row of values: whole cache lines.
constexpr int value_row(int n) { return (n + 63) / 64 * 64; }

// Bytes of the values of both 8-bit operands and (copy) of dy, and of the two factors.
struct ValueBytes {
    size_t w, x, dy, back;
    size_t all() const { return w + x + dy + back; }
};

ValueBytes value_bytes(int M, int N, int K, bool want_x, bool want_w, bool copy)
{
    const size_t row = 2 * (size_t)value_row(K);
    return {want_x ? round256(N * row) : 0, want_w ? round256(M * row) : 0,
            copy ? round256((size_t)M * 2 * value_row(N)) : 0, 256};
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

size_t tasq_residual_norm_workspace_bytes(int type, int batch, int tokens, int width)
{
    if (!type_known(type) || !residual_sizes(batch, tokens, width) ||
        (long long)batch * tokens == 0)
        return 0;
    return (size_t)batch * (size_t)tasq::residual_norm_teams(type, batch, tokens, width).chunks *
           3 * (size_t)width * sizeof(float);
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
    // For rows of dy and of codes wherever they lie.  Of values one product's parts after
    // the other's, and a copy of dy; of codes the parts of both, each of the larger tile.
    GradPlan plan[2] = {grad_plan(M, N, K, false), grad_plan(M, N, K, true)};
    if (values_pay(M, N, K)) {
        plan_values(plan[0], false);
        plan_values(plan[1], true);
        const size_t parts = plan[0].parts > plan[1].parts ? plan[0].parts : plan[1].parts;
        return parts + value_bytes(M, N, K, true, true, true).all();
    }
    size_t most[2] = {};
    for (const bool whole : {false, true}) {
        plan_both(plan, true, {whole, whole}, true);
        for (int i = 0; i < 2; ++i)
            most[i] = plan[i].parts > most[i] ? plan[i].parts : most[i];
    }
    return most[0] + most[1];
}

int tasq_masked_linear_tokens_backward(const void *dy, int type, long long dy_stride,
                                       const int8_t *X, const float *sx, const int8_t *W,
                                       const float *sw, int M, int N, int K, int b, void *dx,
                                       void *dw, float *dbias, void *workspace,
                                       size_t workspace_bytes, void *stream)
{
    if (type != TASQ_TYPE_BF16 && type != TASQ_TYPE_F16)
        return TASQ_ERR_KIND;
    if (!grad_sizes(M, N, K) || (M > 1 && (dy_stride < N || dy_stride >= TASQ_MAX_GRAD_STRIDE)))
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
    const bool bf16 = type == TASQ_TYPE_BF16;
    // (One row has any; 32-bit offsets within a tile.)
    const long long stride = M > 1 ? dy_stride : N < 4096 ? (N + 7) / 8 * 8 : 4096;
    size_t have = workspace ? workspace_bytes : 0;
    char *at = static_cast<char *>(workspace);
    GradPlan plan[2];
    for (const bool turned : {false, true})
        plan[turned] = grad_plan(M, N, K, turned);

    // Values, where they pay and there is room for them.
    const bool dy_whole = N % 8 == 0 && stride % 8 == 0 && aligned_to(dy, 16);
    const ValueBytes vb = value_bytes(M, N, K, want_x, want_w, !dy_whole);
    bool values = values_pay(M, N, K);
    if (values) {
        size_t parts = 0;
        for (const bool turned : {false, true}) {
            plan_values(plan[turned], turned && dbias);
            const bool wanted = turned ? want_w : want_x;
            parts = wanted && plan[turned].parts > parts ? plan[turned].parts : parts;
        }
        values = vb.all() + parts <= have;
    }
    tasq::GradGemm gemm[2] = {};
    if (values) {
        tasq::GradValues v{};
        auto take = [&](size_t bytes) {
            char *p = at;
            at += bytes;
            return p;
        };
        float *back = reinterpret_cast<float *>(take(vb.back));
        const void *A = dy;
        long long a_stride = stride;
        if (!dy_whole) {
            auto &j = v.job[v.n++];
            j = {};
            j.from = dy;
            j.from_stride = stride;
            j.to = take(vb.dy);
            j.rows = M;
            j.width = N;
            j.to_stride = value_row(N);
            A = j.to;
            a_stride = j.to_stride;
        }
        for (const bool turned : {false, true}) {
            if (!(turned ? want_w : want_x))
                continue;
            auto &j = v.job[v.n++];
            j = {};
            j.q = turned ? X : W;
            j.s = turned ? sx : sw;
            j.mask = turned ? 0xffffffffu : tasq::keep_mask_dword(b);
            j.back = back + turned;
            j.to = take(turned ? vb.x : vb.w);
            j.rows = plan[turned].Z;
            j.width = K;
            j.to_stride = value_row(K);
            tasq::GradGemm &g = gemm[turned];
            g.A = A;
            g.a_stride = a_stride;
            g.Q = j.to;
            g.q_stride = j.to_stride;
            g.back = bf16 ? nullptr : j.back;
        }
        if ((bf16 ? tasq::grad_values_bf16(v, st) : tasq::grad_values_f16(v, st)) != hipSuccess)
            return TASQ_ERR_HIP;
    }
    if (values) {
        for (const bool turned : {false, true}) {
            if (!(turned ? want_w : want_x))
                continue;
            const GradPlan &p = plan[turned];
            tasq::GradGemm &g = gemm[turned];
            g.out = turned ? dw : dx;
            g.dbias = turned ? dbias : nullptr;
            g.R = p.R;
            g.Z = p.Z;
            g.C = p.C;
            g.tile_c = p.tile_c;
            g.tiles_r = p.tiles_r;
            g.tiles_c = p.tiles_c;
            g.splits = p.splits;
            g.split_steps = p.split_steps;
            if (p.splits > 1) {
                g.part = reinterpret_cast<float *>(at);
                g.bias_part = g.part + part_floats(p);
            }
            if ((bf16 ? tasq::grad_gemm_bf16(g, turned, st) : tasq::grad_gemm_f16(g, turned, st)) !=
                hipSuccess)
                return TASQ_ERR_HIP;
        }
        return TASQ_OK;
    }
    tasq::GradJob job[2] = {};
    const bool whole[2] = {dy_whole && K % 16 == 0 && aligned_to(W, 16),
                           dy_whole && K % 16 == 0 && aligned_to(X, 16)};
    const bool want[2] = {want_x, want_w};
    int groups = plan_both(plan, dbias, whole, true);
    if ((want_x ? plan[0].parts : 0) + (want_w ? plan[1].parts : 0) > have)
        groups = plan_both(plan, dbias, whole, false);
    for (const bool turned : {false, true}) {
        const GradPlan &p = plan[turned];
        tasq::GradJob &g = job[turned];
        g.A = dy;
        g.a_stride = stride;
        g.Q = turned ? X : W;
        g.s = turned ? sx : sw;
        g.mask = turned ? 0xffffffffu : tasq::keep_mask_dword(b);
        g.out = turned ? dw : dx;
        g.dbias = turned ? dbias : nullptr;
        g.R = p.R;
        g.Z = p.Z;
        g.C = p.C;
        g.tile = p.tile;
        g.tiles_r = p.tiles_r;
        g.tiles_c = p.tiles_c;
        g.splits = p.splits;
        g.split_steps = p.split_steps;
        if (want[turned] && p.splits > 1) {
            g.part = reinterpret_cast<float *>(at);
            g.bias_part = g.part + part_floats(p);
            at += p.parts;
        }
    }
    // Small products share a launch (on its own each takes 3 us of the host's, and fills
    // less of the card).
    const auto run = [&](const tasq::GradJob *x, const tasq::GradJob *w) {
        const bool chunks = whole[x ? 0 : 1];
        if (x && w ? x->tile <= 128 : (x ? x : w)->tile == 64)
            return bf16 ? tasq::token_grads_bf16(x, w, groups, chunks, st)
                        : tasq::token_grads_f16(x, w, groups, chunks, st);
        return bf16 ? tasq::token_grad_bf16(x ? *x : *w, !x, chunks, st)
                    : tasq::token_grad_f16(x ? *x : *w, !x, chunks, st);
    };
    if (want_x && want_w && plan[0].tile == plan[1].tile && plan[0].tile <= 128 &&
        whole[0] == whole[1])
        return status(run(&job[0], &job[1]));
    if (want_x && run(&job[0], nullptr) != hipSuccess)
        return TASQ_ERR_HIP;
    return want_w ? status(run(nullptr, &job[1])) : TASQ_OK;
}

}  // extern "C"
