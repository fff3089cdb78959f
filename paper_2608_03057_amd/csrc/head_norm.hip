// Root-mean-square norm of every head of q and k with the position rotation
// in the same pass, and its gradient.
//
//   r = 1 / sqrt(mean_d x[d]^2 + eps),   n[d] = x[d] r w[d],
//   (y1, y2) = (n1 c - n2 s, n1 s + n2 c)  for each of the R / 2 rotated pairs,
//   y[d] = n[d] from R on,
// a pair being (i, i + R/2) or, interleaved, (2 i, 2 i + 1), c and s the
// table's cosine and sine of frequency i at the token's position.  Backward,
// with g the inverse rotation of dy:
//   dx[d] = r (g[d] w[d] - x[d] r^2 mean_d(g w x)),   dw[d] = sum g[d] x[d] r
// over all heads of all tokens.  Everything between the loads and the stores
// is fp32.
//
// Bound by memory: x (and dy) are read once, y (dx) is written once.  q and k of
// 8192 tokens, 16 heads of 72 each in bfloat16: 16.1 us, 4.7 TB/s; the gradient of
// 4096 tokens, 20 heads of 112 each in half: 27.1 us, 4.1 TB/s, and 3.9 us for the
// weights' sums.  A head belongs to a group of lanes of a wave with eight elements
// each, four pairs that meet the same four frequencies, so the norm's sum is a
// few lane exchanges and the rotation needs none; a group takes kHeads heads of
// one token in turn, which share its cosines and sines.
#include "block_internal.h"
#include "floats.h"

namespace tasq {

namespace {

constexpr int kHeads = 4;       // heads of a token that a lane group takes

struct Unit {
    int b, s, h;                // h: the first head
    unsigned token;
};

// Unit v of a job: its token and the first of its heads.
__device__ __forceinline__ Unit unit_of(const HeadJob &j, unsigned v)
{
    Unit r;
    const unsigned blocks = (unsigned)(j.heads + kHeads - 1) / kHeads;
    r.token = v / blocks;
    r.h = (int)(v - r.token * blocks) * kHeads;
    r.b = (int)(r.token / (unsigned)j.tokens);
    r.s = (int)(r.token - (unsigned)r.b * (unsigned)j.tokens);
    return r;
}

// The table's row of a token, or -1 where it has no position in the table.
__device__ __forceinline__ int position_of(const HeadJob &j, const Unit &u)
{
    const int p = j.position ? j.position[u.token] : u.s;
    return j.rot && (unsigned)p < (unsigned)j.positions ? p : -1;
}

// Lane l's eight elements of a head as pairs (x1[i], x2[i]), i < 4: pairs 4 l .. of
// the rotated ones and, behind them, of neighbours that nothing turns.
// (kSplit: as kHalves, where a lane has pairs of both kinds, R / 2 not a multiple of
// four; the lanes that do take their elements one by one.  8192 tokens, 32 heads of
// 72 of which 36 rotate, in bfloat16 29 us a call and 48 backward, against 60 and
// 104 of a wave to each head; 17.4 and 30.7 where all 72 rotate.)
enum Form { kHalves, kInterleaved, kSplit };

template <Form FORM> struct Pairs {
    static constexpr bool INTERLEAVED = FORM == kInterleaved;
    int o1, o2;                 // first elements of x1 and x2 (interleaved: o1 alone)
    int turned;                 // of the four pairs, those that rotate
    int rot;
    bool mixed;                 // some of the four rotate and some do not

    template <class P> struct Raw {
        Packed<P, 4> a, b;
    };

    __device__ __forceinline__ void init(int l, int rot_)
    {
        rot = rot_;
        turned = min(max(rot / 2 - 4 * l, 0), 4);
        mixed = FORM == kSplit && (turned & 3) != 0;
        o1 = INTERLEAVED || turned == 0 ? 8 * l : 4 * l;
        o2 = INTERLEAVED || turned == 0 ? o1 + 4 : o1 + rot / 2;
    }
    // Element of x1[i] (second: of x2[i]).
    __device__ __forceinline__ int element(int i, bool second) const
    {
        if (INTERLEAVED)
            return o1 + 2 * i + second;
        if (mixed && i >= turned)
            return rot + 2 * (i - turned) + second;
        return (second ? o2 : o1) + i;
    }
    template <class P> __device__ __forceinline__ Raw<P> fetch(const P *p) const
    {
        if (!mixed) {
            if constexpr (INTERLEAVED)
                return *reinterpret_cast<const Raw<P> *>(p + o1);
            else
                return {*reinterpret_cast<const Packed<P, 4> *>(p + o1),
                        *reinterpret_cast<const Packed<P, 4> *>(p + o2)};
        }
        P e[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = p[element(i, false)];
            e[4 + i] = p[element(i, true)];
        }
        return __builtin_bit_cast(Raw<P>, e);
    }
    template <class P>
    static __device__ __forceinline__ void pairs(Raw<P> r, float (&x1)[4], float (&x2)[4])
    {
        // Here, and not for all heads at once, which takes twice the registers.
#pragma unroll
        for (int i = 0; i < Packed<P, 4>::kWords; ++i) {
            uint32_t u = r.a.w[i], v = r.b.w[i];
            asm volatile("" : "+v"(u), "+v"(v));
            r.a.w[i] = u;
            r.b.w[i] = v;
        }
        if constexpr (INTERLEAVED) {
            float e[8];
            __builtin_bit_cast(Packed<P, 8>, r).floats(e);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x1[i] = e[2 * i];
                x2[i] = e[2 * i + 1];
            }
        } else {
            r.a.floats(x1);
            r.b.floats(x2);
        }
    }
    template <class P>
    __device__ __forceinline__ void store(P *p, const float (&x1)[4], const float (&x2)[4]) const
    {
        if constexpr (INTERLEAVED) {
            float e[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                e[2 * i] = x1[i];
                e[2 * i + 1] = x2[i];
            }
            reinterpret_cast<Packed<P, 8> *>(p + o1)->set(e);
        } else if (!mixed) {
            reinterpret_cast<Packed<P, 4> *>(p + o1)->set(x1);
            reinterpret_cast<Packed<P, 4> *>(p + o2)->set(x2);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[element(i, false)] = (P)x1[i];
                p[element(i, true)] = (P)x2[i];
            }
        }
    }
    __device__ __forceinline__ void weights(const float *w, float (&w1)[4], float (&w2)[4]) const
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w1[i] = w2[i] = 1.0f;
        if (w)
            pairs(fetch(w), w1, w2);
    }
};

// Sum over the LPR lanes of a group.
template <int LPR> __device__ __forceinline__ float group_sum(float v)
{
    return group_reduce<LPR>(v, [](float a, float b) { return a + b; });
}

// Cosines and sines of lane l's pairs at row p of the tables, of which `turned`
// rotate.
__device__ __forceinline__ void cos_sin(const HeadJob &j, int p, int l, int turned, float (&c)[4],
                                        float (&s)[4])
{
    const size_t at = (size_t)p * (j.rot / 2) + 4 * l;
    if (p >= 0 && turned == 4) {
        reinterpret_cast<const Packed<float, 4> *>(j.cos + at)->floats(c);
        reinterpret_cast<const Packed<float, 4> *>(j.sin + at)->floats(s);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bool turn = p >= 0 && i < turned;
            c[i] = turn ? j.cos[at + i] : 1.0f;
            s[i] = turn ? j.sin[at + i] : 0.0f;
        }
    }
}

template <class T, Form FORM, int LPR>
__global__ void __launch_bounds__(256) k_norm_rotate(HeadCall call)
{
    constexpr int GROUPS = 256 / LPR;
    // The first blocks are the first job's, so that a workgroup's job is one.
    const int first = (call.job[0].units + GROUPS - 1) / GROUPS;
    const int block = call.first_block + (int)blockIdx.x;
    const int job = block >= first;
    const HeadJob &j = call.job[job];
    const int u = (block - (job ? first : 0)) * GROUPS + (int)threadIdx.x / LPR;
    if (u >= j.units)
        return;                 // whole groups, which exchange among themselves only
    const int l = threadIdx.x % LPR;
    const Unit un = unit_of(j, (unsigned)u);
    const bool live = 8 * l < call.dim;
    Pairs<FORM> at;
    at.init(live ? l : 0, j.rot);
    const T *x = static_cast<const T *>(j.x) + un.b * j.x_stride[0] + un.s * j.x_stride[1];
    typename Pairs<FORM>::template Raw<T> raw[kHeads];
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        raw[k] = {};
        if (live && un.h + k < j.heads)
            raw[k] = at.fetch(x + (un.h + k) * j.x_stride[2]);
    }
    float c[4], s[4], w1[4], w2[4];
    cos_sin(j, position_of(j, un), live ? l : 0, at.turned, c, s);
    at.weights(j.weight, w1, w2);
    T *y = static_cast<T *>(j.out) + (size_t)un.token * j.heads * call.dim;
#pragma unroll
    for (int k = 0; k < kHeads; ++k) {
        float sum = 0.0f, x1[4], x2[4];
        at.pairs(raw[k], x1, x2);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            sum += x1[i] * x1[i] + x2[i] * x2[i];
        const float r = rsqrtf(group_sum<LPR>(sum) * call.inv_dim + call.eps);
        float y1[4], y2[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float n1 = x1[i] * r * w1[i], n2 = x2[i] * r * w2[i];
            y1[i] = n1 * c[i] - n2 * s[i];
            y2[i] = n1 * s[i] + n2 * c[i];
        }
        if (live && un.h + k < j.heads)
            at.store(y + (size_t)(un.h + k) * call.dim, y1, y2);
    }
}

// Head dimensions that are not a multiple of eight: one wave per head, pairs p,
// p + 64, .. of lane p.  The gradient's dw meets in `part` as below.
template <class T, bool GRAD>
__global__ void __launch_bounds__(256) k_norm_rotate_any(HeadCall call, float *part)
{
    constexpr int NP = kMaxHeadDim / 2 / 64;    // pairs of a lane
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int half = call.dim / 2;
    __shared__ float total[4][kMaxHeadDim];
    for (int job = 0; job < call.n; ++job) {
        const HeadJob &j = call.job[job];
        int o1[NP], o2[NP];
        float w1[NP], w2[NP], dw1[NP] = {}, dw2[NP] = {};
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = lane + 64 * i;
            const bool halves = !call.interleaved && 2 * p < j.rot;
            o1[i] = halves ? p : 2 * p;
            o2[i] = halves ? p + j.rot / 2 : 2 * p + 1;
            w1[i] = w2[i] = 1.0f;
            if (p < half && j.weight) {
                w1[i] = j.weight[o1[i]];
                w2[i] = j.weight[o2[i]];
            }
        }
        for (int u = blockIdx.x * 4 + wave; u < j.units; u += gridDim.x * 4) {
            const Unit un = unit_of(j, (unsigned)u);
            const int pos = position_of(j, un);
            float c[NP], s[NP];
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                const int p = lane + 64 * i;
                const bool turned = p < half && 2 * p < j.rot && pos >= 0;
                c[i] = turned ? j.cos[(size_t)pos * (j.rot / 2) + p] : 1.0f;
                s[i] = turned ? j.sin[(size_t)pos * (j.rot / 2) + p] : 0.0f;
            }
            for (int h = un.h; h < min(un.h + kHeads, j.heads); ++h) {
                const T *x = static_cast<const T *>(j.x) + un.b * j.x_stride[0] +
                             un.s * j.x_stride[1] + h * j.x_stride[2];
                T *out = static_cast<T *>(j.out) + ((size_t)un.token * j.heads + h) * call.dim;
                float a[NP], b[NP], sq = 0.0f;
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const bool live = lane + 64 * i < half;
                    a[i] = live ? (float)x[o1[i]] : 0.0f;
                    b[i] = live ? (float)x[o2[i]] : 0.0f;
                    sq += a[i] * a[i] + b[i] * b[i];
                }
                const float r = rsqrtf(group_sum<64>(sq) * call.inv_dim + call.eps);
                float y1[NP], y2[NP];
                if constexpr (!GRAD) {
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const float n1 = a[i] * r * w1[i], n2 = b[i] * r * w2[i];
                        y1[i] = n1 * c[i] - n2 * s[i];
                        y2[i] = n1 * s[i] + n2 * c[i];
                    }
                } else {
                    const T *dy = static_cast<const T *>(j.dy) + un.b * j.dy_stride[0] +
                                  un.s * j.dy_stride[1] + h * j.dy_stride[2];
                    float inner = 0.0f;
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        const bool live = lane + 64 * i < half;
                        const float d1 = live ? (float)dy[o1[i]] : 0.0f;
                        const float d2 = live ? (float)dy[o2[i]] : 0.0f;
                        y1[i] = d1 * c[i] + d2 * s[i];
                        y2[i] = d2 * c[i] - d1 * s[i];
                        inner += y1[i] * w1[i] * a[i] + y2[i] * w2[i] * b[i];
                    }
                    const float t = group_sum<64>(inner) * call.inv_dim * r * r;
#pragma unroll
                    for (int i = 0; i < NP; ++i) {
                        dw1[i] += y1[i] * a[i] * r;
                        dw2[i] += y2[i] * b[i] * r;
                        y1[i] = r * (y1[i] * w1[i] - a[i] * t);
                        y2[i] = r * (y2[i] * w2[i] - b[i] * t);
                    }
                }
#pragma unroll
                for (int i = 0; i < NP; ++i)
                    if (lane + 64 * i < half) {
                        out[o1[i]] = (T)y1[i];
                        out[o2[i]] = (T)y2[i];
                    }
            }
        }
        if constexpr (GRAD) {
            __syncthreads();            // the job before has been summed
#pragma unroll
            for (int i = 0; i < NP; ++i)
                if (lane + 64 * i < half) {
                    total[wave][o1[i]] = dw1[i];
                    total[wave][o2[i]] = dw2[i];
                }
            __syncthreads();
            for (int d = threadIdx.x; d < call.dim; d += 256)
                part[((size_t)job * gridDim.x + blockIdx.x) * call.dim + d] =
                    (total[0][d] + total[1][d]) + (total[2][d] + total[3][d]);
        }
    }
}

// The gradient.  A workgroup's lane groups take every gridDim.x-th unit; each
// keeps its part of dw in registers, the workgroup's parts meet in LDS and
// its sum goes to part[job][workgroup][dim], which k_sum_dweight adds up in
// order.  (No atomics: their order would change dw from run to run.)
template <class T, Form FORM, int LPR>
__global__ void __launch_bounds__(256, FORM == kSplit && sizeof(T) == 4 ? 3 : 4)
    k_norm_rotate_backward(HeadCall call, float *part)
{
    constexpr int GROUPS = 256 / LPR;
    const int l = threadIdx.x % LPR, group = threadIdx.x / LPR;
    const bool live = 8 * l < call.dim;
    __shared__ float sum[GROUPS][8 * LPR + 1];
    for (int job = 0; job < call.n; ++job) {
        const HeadJob &j = call.job[job];
        Pairs<FORM> at;
        at.init(live ? l : 0, j.rot);
        float w1[4], w2[4], dw1[4] = {}, dw2[4] = {};
        at.weights(j.weight, w1, w2);
        for (int u = blockIdx.x * GROUPS + group; u < j.units; u += gridDim.x * GROUPS) {
            const Unit un = unit_of(j, (unsigned)u);
            const T *x =
                static_cast<const T *>(j.x) + un.b * j.x_stride[0] + un.s * j.x_stride[1];
            const T *dy =
                static_cast<const T *>(j.dy) + un.b * j.dy_stride[0] + un.s * j.dy_stride[1];
            typename Pairs<FORM>::template Raw<T> xs[kHeads], ds[kHeads];
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                xs[k] = ds[k] = {};
                if (live && un.h + k < j.heads) {
                    xs[k] = at.fetch(x + (un.h + k) * j.x_stride[2]);
                    ds[k] = at.fetch(dy + (un.h + k) * j.dy_stride[2]);
                }
            }
            float c[4], s[4];
            cos_sin(j, position_of(j, un), live ? l : 0, at.turned, c, s);
            T *dx = static_cast<T *>(j.out) + (size_t)un.token * j.heads * call.dim;
#pragma unroll
            for (int k = 0; k < kHeads; ++k) {
                float sq = 0.0f, inner = 0.0f, g1[4], g2[4], x1[4], x2[4], d1[4], d2[4];
                at.pairs(xs[k], x1, x2);
                at.pairs(ds[k], d1, d2);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    g1[i] = d1[i] * c[i] + d2[i] * s[i];
                    g2[i] = d2[i] * c[i] - d1[i] * s[i];
                    sq += x1[i] * x1[i] + x2[i] * x2[i];
                    inner += g1[i] * w1[i] * x1[i] + g2[i] * w2[i] * x2[i];
                }
                // (A head past the last one is zeros, whose r without eps is infinite:
                // none of it may reach dw.)
                const float norm = rsqrtf(group_sum<LPR>(sq) * call.inv_dim + call.eps);
                const float r = un.h + k < j.heads ? norm : 0.0f;
                const float t = group_sum<LPR>(inner) * call.inv_dim * r * r;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    dw1[i] += g1[i] * x1[i] * r;
                    dw2[i] += g2[i] * x2[i] * r;
                    g1[i] = r * (g1[i] * w1[i] - x1[i] * t);
                    g2[i] = r * (g2[i] * w2[i] - x2[i] * t);
                }
                if (live && un.h + k < j.heads)
                    at.store(dx + (size_t)(un.h + k) * call.dim, g1, g2);
            }
        }
        __syncthreads();            // the job before has been summed
        if (live) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[group][at.element(i, false)] = dw1[i];
                sum[group][at.element(i, true)] = dw2[i];
            }
        }
        __syncthreads();
        for (int d = threadIdx.x; d < call.dim; d += 256) {
            float v = 0.0f;
            for (int g = 0; g < GROUPS; ++g)
                v += sum[g][d];
            part[((size_t)job * gridDim.x + blockIdx.x) * call.dim + d] = v;
        }
    }
}

// dw[d] = sum of `groups` workgroups' parts: 8 columns to a workgroup, 32 slices
// of the parts side by side.
__global__ void __launch_bounds__(256) k_sum_dweight(HeadCall call, const float *part, int groups)
{
    const int job = blockIdx.y, d = blockIdx.x * 8 + (threadIdx.x & 7);
    const int slice = threadIdx.x >> 3;
    __shared__ float sum[32][9];
    float v = 0.0f;
    if (d < call.dim) {
        const float *p = part + (size_t)job * groups * call.dim + d;
#pragma unroll 8
        for (int g = slice; g < groups; g += 32)
            v += p[(size_t)g * call.dim];
    }
    sum[slice][threadIdx.x & 7] = v;
    __syncthreads();
    if (threadIdx.x < 8 && d < call.dim && call.job[job].dweight) {
        v = 0.0f;
#pragma unroll
        for (int g = 0; g < 32; ++g)
            v += sum[g][threadIdx.x];
        call.job[job].dweight[d] = v;
    }
}

// Workgroups of the gradient: enough to fill the GPU, few enough that their
// partial sums stay small.
int grad_groups(const HeadCall &c, int units_per_group)
{
    const int most = c.job[0].units > c.job[1].units ? c.job[0].units : c.job[1].units;
    const int all = (most + units_per_group - 1) / units_per_group;
    return all < kHeadGroups ? all : kHeadGroups;
}

// (Workgroups of the forward pass go out 2^22 at a time: a launch has fewer than 2^32
// threads.)
template <class T, Form FORM, int LPR>
void launch_vectors(HeadCall c, bool grad, float *part, int *groups, hipStream_t stream)
{
    constexpr int GROUPS = 256 / LPR;
    if (grad) {
        *groups = grad_groups(c, GROUPS);
        k_norm_rotate_backward<T, FORM, LPR><<<*groups, 256, 0, stream>>>(c, part);
    } else {
        const int blocks = (c.job[0].units + GROUPS - 1) / GROUPS +
                           (c.job[1].units + GROUPS - 1) / GROUPS;
        constexpr int MOST = 1 << 22;
        for (c.first_block = 0; c.first_block < blocks; c.first_block += MOST) {
            const int left = blocks - c.first_block;
            k_norm_rotate<T, FORM, LPR><<<left < MOST ? left : MOST, 256, 0, stream>>>(c);
        }
    }
}

template <class T, Form FORM>
void launch_lanes(const HeadCall &c, bool grad, float *part, int *groups, hipStream_t stream)
{
    if (c.dim <= 32)
        launch_vectors<T, FORM, 4>(c, grad, part, groups, stream);
    else if (c.dim <= 64)
        launch_vectors<T, FORM, 8>(c, grad, part, groups, stream);
    else if (c.dim <= 128)
        launch_vectors<T, FORM, 16>(c, grad, part, groups, stream);
    else
        launch_vectors<T, FORM, 32>(c, grad, part, groups, stream);
}

}  // namespace

hipError_t launch_norm_rotate(const HeadCall &in, bool grad, float *part, hipStream_t stream)
{
    HeadCall c = in;
    c.inv_dim = 1.0f / (float)c.dim;
    bool plain = true;          // nothing rotates: pairs may lie as loads like them
    for (int i = 0; i < 2; ++i) {
        HeadJob &j = c.job[i];
        if (i >= c.n)
            j = HeadJob{};
        j.units = j.batch * j.tokens * ((j.heads + kHeads - 1) / kHeads);
        plain = plain && !j.rot;
    }
    if (plain)
        c.interleaved = 1;
    int groups = 0;
    hipError_t e = c.job[0].units == 0 && c.job[1].units == 0 ? hipSuccess : with_type(c.type, [&](auto zero) {
        using T = decltype(zero);
        if (c.dim % 8 == 0 && c.interleaved) {
            launch_lanes<T, kInterleaved>(c, grad, part, &groups, stream);
        } else if (c.dim % 8 == 0 && c.job[0].rot % 8 == 0 && c.job[1].rot % 8 == 0) {
            launch_lanes<T, kHalves>(c, grad, part, &groups, stream);
        } else if (c.dim % 8 == 0) {
            launch_lanes<T, kSplit>(c, grad, part, &groups, stream);
        } else {
            groups = grad_groups(c, 4);
            if (grad)
                k_norm_rotate_any<T, true><<<groups, 256, 0, stream>>>(c, part);
            else
                k_norm_rotate_any<T, false><<<groups, 256, 0, stream>>>(c, nullptr);
        }
        return hipGetLastError();
    });
    if (e != hipSuccess || !grad || c.n == 0)
        return e;
    k_sum_dweight<<<dim3((c.dim + 7) / 8, c.n), 256, 0, stream>>>(c, part, groups);
    return hipGetLastError();
}

}  // namespace tasq
