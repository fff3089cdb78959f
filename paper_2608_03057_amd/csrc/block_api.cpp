// C ABI of the attention half of a block (include/tasq.h): argument checks,
// then one launcher each.
#include <math.h>

#include "block_internal.h"
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

int check_heads(const tasq_heads &h, int type, int dim, bool grad)
{
    if (h.batch < 0 || h.tokens < 0 || h.heads < 0 || h.positions < 0 || h.rot < 0 ||
        h.rot > dim || h.rot % 2)
        return TASQ_ERR_DIM;
    for (int i = 0; i < 3; ++i)
        if (h.x_stride[i] < 0 || (grad && h.dy_stride[i] < 0))
            return TASQ_ERR_DIM;
    // Units of a call are counted in 32 bits, and so are tokens and heads.
    if (h.heads > (1 << 30) || (long long)h.batch * h.tokens > (1LL << 30) ||
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

// A pass: microseconds that a workgroup takes for a tile of heads of dim when it
// has a compute unit to itself (measured at 16 to 128; from 64 on registers run
// short in dK and dV), and fp32 results for each of its resident elements.
struct Pass {
    double slope, base, wide_slope, wide_base;
    int results;
    double tile(int dim) const { return fmax(slope * dim + base, wide_slope * dim + wide_base); }
};
constexpr Pass kForward = {0.0087, 0.35, 0, 0, 1}, kQueryGrad = {0.0161, 0.48, 0, 0, 1},
               kKeyGrad = {0.02, 0.5, 0.05, -1.3, 2};

// Ranges that `tiles` streamed tiles of a pass are cut into when `base` workgroups
// would run uncut: none, or as many as make half a workgroup, one or two for each
// compute unit, at least two tiles each, whichever takes the shortest by the model
//   tiles of a range * tile time * (1.2 where two share a compute unit)
//     + 6 us for the launch that joins the parts + their bytes, written and read,
//       at 4 TB/s.
// Of 224 shapes of 32 to 256 workgroups and 8 to 64 tiles its choice takes 2.1%
// more forward than the best of one to twelve ranges in the geometric mean, 28% at
// most (13.2 us against 10.3), and 83% of uncut; of 96 each 1 to 2% and up to 17% in
// the gradients.
// us uncut and cut (ranges): forward, heads of 72, 32 workgroups of 64 tiles 63.6
// and 20.8 (8), 160 of 64 67.9 and 45.8 (3), 160 of 16 20.2 and 26.0 (3); one query
// over 8191 keys of 128 160 and 12 (64); both gradients with dK and dV cut, heads
// of 72, 96 of 64 157 and 87 (5), 160 of 64 176 and 130 (3), 256 of 16 62.1 and 67.5
// (2); with dQ cut, 160 of 64 159 and 134 (3), 160 of 16 52.0 and 53.2 (3).
void plan_ranges(long long base, int tiles, int dim, size_t rows, const Pass &pass, int *ranges,
                 int *range_tiles)
{
    *ranges = 1;
    *range_tiles = tiles > 0 ? tiles : 1;
    if (base <= 0 || base > 256 || tiles < 8)
        return;
    double best = tiles * pass.tile(dim);
    for (const int units : {128, 256, 512}) {
        const int most = tiles / 2, want = (int)(units / base);
        if (want < 2)
            continue;
        const int cut = want < most ? want : most;
        const int t = (tiles + cut - 1) / cut, r = (tiles + t - 1) / t;
        const double us = t * pass.tile(dim) * (r * base > 256 ? 1.2 : 1.0) + 6.0 +
                          8.0 * pass.results * r * (double)rows * dim / 4e6;
        if (us < best) {
            best = us;
            *ranges = r;
            *range_tiles = t;
        }
    }
}

constexpr size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// The launch's shape (with cuts if `cut`), and the bytes of its workspace.
size_t plan_attention(tasq::AttnCall &c, bool backward, bool cut)
{
    const int group = c.kv_heads ? c.heads / c.kv_heads : 0;
    const long long pairs = (long long)c.batch * c.kv_heads;
    const int key_tiles = (c.kv_len + 63) / 64;
    const long long pair_rows = (long long)group * c.q_len;
    // Two blocks of rows to a wave halve what a row reads of LDS, but take registers:
    // two workgroups of 256 rows to a compute unit where three of 128 fit.  So they
    // run where one round of them replaces two of the smaller, and where rounds
    // are many for dims up to 64.  us with one block and two, by workgroups of 256
    // rows: heads of 64 over 1024 keys 384 34.8 and 38.8, 400 45.2 and 39.6, 512 46.5
    // and 41.9, 544 52.2 and 59.5, 704 61.1 and 61.1, 1024 81.8 and 77.0; of 72 384
    // 42.7 and 53.7, 512 56.5 and 57.1, over 4096 512 191.7 and 186.7, 544 214 and 299,
    // 1024 361 and 384.  (Heads of 72 lose 4% over 300 keys, 26.7 and 28.3, and heads up
    // to 32 gain nothing: 512 34.8 and 33.1, 704 45.2 and 44.9.)
    const int steps = (c.dim + 15) / 16;
    const long long wide = pairs * ((pair_rows + 255) / 256);
    const bool fits = steps >= tasq::kAttnWideFrom && steps <= tasq::kAttnWideSteps;
    c.row_blocks = !backward && fits &&
                           ((wide > 384 && wide <= 512) || (steps <= 4 && wide >= 704))
                       ? 2
                       : 1;
    c.row_tiles = (int)((pair_rows + 128 * c.row_blocks - 1) / (128 * c.row_blocks));
    const size_t rows = (size_t)c.batch * c.heads * c.q_len;
    plan_ranges(cut ? pairs * c.row_tiles : 0, key_tiles, c.dim, rows,
                backward ? kQueryGrad : kForward, &c.splits, &c.split_tiles);
    size_t bytes = 0;
    if (c.splits > 1) {
        bytes += round256(c.splits * rows * c.dim * sizeof(float));
        bytes += backward ? 0 : round256(c.splits * rows * sizeof(float));
    }
    if (backward) {
        c.key_tiles = (c.kv_len + 127) / 128;
        plan_ranges(cut ? pairs * c.key_tiles : 0, group * ((c.q_len + 63) / 64), c.dim,
                    (size_t)c.batch * c.kv_heads * c.kv_len, kKeyGrad, &c.kv_splits,
                    &c.kv_split_tiles);
        bytes += round256(rows * sizeof(float));
        if (c.kv_splits > 1)
            bytes += round256((size_t)c.kv_splits * 2 * c.batch * c.kv_len * c.kv_heads * c.dim *
                              sizeof(float));
    }
    return bytes;
}

void lay_out_workspace(tasq::AttnCall &c, bool backward, void *workspace)
{
    char *p = static_cast<char *>(workspace);
    const size_t rows = (size_t)c.batch * c.heads * c.q_len;
    auto take = [&](size_t floats) {
        float *r = reinterpret_cast<float *>(p);
        p += round256(floats * sizeof(float));
        return r;
    };
    if (c.splits > 1) {
        c.part = take(c.splits * rows * c.dim);
        if (!backward)
            c.part_lse = take(c.splits * rows);
    }
    if (backward) {
        c.delta = take(rows);
        if (c.kv_splits > 1)
            c.kv_part = take((size_t)c.kv_splits * 2 * c.batch * c.kv_len * c.kv_heads * c.dim);
    }
}

// Strides of a [batch][tokens][heads][dim] operand, those of extents below 2
// as zero.
int take_strides(const long long *in, int batch, int tokens, int heads, long long *out)
{
    const int extent[3] = {batch, tokens, heads};
    for (int i = 0; i < 3; ++i) {
        out[i] = extent[i] > 1 ? in[i] : 0;
        // A tile of 64 rows is addressed with 32-bit byte offsets.
        if (out[i] < 0 || (i == 1 && out[i] >= (1LL << 23)))
            return TASQ_ERR_DIM;
        if (out[i] % 8)
            return TASQ_ERR_ALIGN;
    }
    return TASQ_OK;
}

// Sizes and types: what tasq_attention_workspace_bytes needs to be valid.
int check_attention_sizes(const tasq_attention *a, tasq::AttnCall &c)
{
    if (!a)
        return TASQ_ERR_NULL;
    if (a->type != TASQ_TYPE_BF16 && a->type != TASQ_TYPE_F16)
        return TASQ_ERR_KIND;
    if (a->batch < 0 || a->heads < 0 || a->kv_heads < 0 || a->q_len < 0 || a->kv_len < 0 ||
        a->dim < 8 || a->dim > TASQ_MAX_ATTENTION_DIM || a->dim % 8 ||
        (a->kv_heads ? a->heads % a->kv_heads : a->heads) != 0)
        return TASQ_ERR_DIM;
    // Rows, keys and workgroups are counted in 32 bits.
    const long long most = 1LL << 30;
    if (a->kv_len > most || (long long)a->heads * a->q_len > most ||
        (long long)a->batch * a->kv_heads > (1 << 20) ||
        (long long)a->batch * a->heads * (a->q_len / 32 + 1LL) > most ||
        (long long)a->batch * a->kv_heads * (a->kv_len / 32 + 1LL) > most)
        return TASQ_ERR_DIM;
    c.type = a->type;
    c.batch = a->batch;
    c.heads = a->heads;
    c.kv_heads = a->kv_heads;
    c.q_len = a->q_len;
    c.kv_len = a->kv_len;
    c.dim = a->dim;
    return TASQ_OK;
}

int attention(const tasq_attention *a, bool backward, void *stream)
{
    tasq::AttnCall c{};
    if (int rc = check_attention_sizes(a, c))
        return rc;
    if (!(a->scale > 0.0f) || isinf(a->scale))
        return TASQ_ERR_RANGE;
    const bool queries = c.batch && c.heads && c.q_len, keys = c.batch && c.kv_heads && c.kv_len;
    if (!queries && !(backward && keys))
        return TASQ_OK;
    if ((queries && (!a->q || !a->out)) || (keys && (!a->k || !a->v)))
        return TASQ_ERR_NULL;
    if (backward && ((queries && (!a->dout || !a->lse || !a->dq)) || (keys && (!a->dk || !a->dv))))
        return TASQ_ERR_NULL;
    const void *wide[] = {a->q, a->k, a->v, a->out, a->dout, a->dq, a->dk, a->dv};
    for (int i = 0; i < (backward ? 8 : 4); ++i)
        if (!aligned_to(wide[i], 16))
            return TASQ_ERR_ALIGN;
    if (!aligned_to(a->kv_lengths, 4) || !aligned_to(a->lse, 4) ||
        !aligned_to(a->workspace, 256))
        return TASQ_ERR_ALIGN;
    int rc = take_strides(a->q_stride, c.batch, c.q_len, c.heads, c.q_stride);
    if (!rc)
        rc = take_strides(a->k_stride, c.batch, c.kv_len, c.kv_heads, c.k_stride);
    if (!rc)
        rc = take_strides(a->v_stride, c.batch, c.kv_len, c.kv_heads, c.v_stride);
    if (!rc && backward)
        rc = take_strides(a->dout_stride, c.batch, c.q_len, c.heads, c.dout_stride);
    if (rc)
        return rc;
    c.q = a->q;
    c.k = a->k;
    c.v = a->v;
    c.kv_lengths = a->kv_lengths;
    c.key_mask = a->key_mask;
    c.out = a->out;
    c.lse = a->lse;
    c.dout = a->dout;
    c.dq = a->dq;
    c.dk = a->dk;
    c.dv = a->dv;
    c.scale = a->scale;
    c.scale_log2 = a->scale * 1.4426950408889634f;
    const size_t have = a->workspace ? a->workspace_bytes : 0;
    if (plan_attention(c, backward, true) > have && plan_attention(c, backward, false) > have)
        return TASQ_ERR_WORKSPACE;
    lay_out_workspace(c, backward, a->workspace);
    const bool bf16 = c.type == TASQ_TYPE_BF16;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (backward)
        return status(bf16 ? tasq::attn_backward_bf16(c, st) : tasq::attn_backward_f16(c, st));
    return status(bf16 ? tasq::attn_forward_bf16(c, st) : tasq::attn_forward_f16(c, st));
}

}  // namespace

extern "C" {

int tasq_quantize_tokens(const void *x, int x_type, int M, int K, long long x_stride,
                         int8_t *X_out, float *sx_out, void *stream)
{
    if (!type_known(x_type))
        return TASQ_ERR_KIND;
    if (M < 0 || M > kMostRows || K < 0 || (M > 1 && x_stride < K))
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
    if (M < 0 || M > kMostRows || N < 0 || N > kMostRows || K < 0)
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

size_t tasq_attention_workspace_bytes(const tasq_attention *a, int backward)
{
    tasq::AttnCall c{};
    if (check_attention_sizes(a, c))
        return 0;
    return plan_attention(c, backward != 0, true);
}

int tasq_attention_forward(const tasq_attention *a, void *stream)
{
    return attention(a, false, stream);
}

int tasq_attention_backward(const tasq_attention *a, void *stream)
{
    return attention(a, true, stream);
}

}  // extern "C"
