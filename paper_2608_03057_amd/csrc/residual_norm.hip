// The residual stream between two branches of a block, and its gradient:
//
//   r = alpha x + g P(y),     P(y) = y or N(y) wp,
//   h = N(r) w (1 + scale) + shift,
//   N(v) = (v - mean v) / sqrt(var v + eps)  or  v / sqrt(mean v^2 + eps),
//
// g, scale and shift per channel and batch entry (or shared), w and wp per
// channel.  Backward, with n = N(r), u = dh w (1 + scale), 1/s the factor of N:
//   D = dr + (u - [mean u] - n mean(u n)) / s,   dx = alpha D,
//   p = D g [wp],   dy = p  or  the same Jacobian of N at y applied to p,
// and sums over tokens: dshift = sum dh, P = sum dh n, Q = sum D N(y) (or D y), of
// which dscale = w P, dw = sum_b (1 + scale) P, dgate = wp Q, dwp = sum_b g Q.
// The bracketed means are the layer kind's.  Everything between the loads and the
// stores is fp32; the variance is that of the centred row, which two passes over
// registers give without cancellation.
//
// Bound by memory: every operand is read once and every result written once.  A
// row belongs to a wave (or a workgroup), which holds it in registers, eight
// channels to a lane and vector, between its sums and its stores.  8192 rows of 1152 in
// bfloat16 take 14.3 us (75 MB at the rate of a copy), their gradient 28 (113 MB at 4.1
// TB/s) and 4 for the sums over tokens.
#include "branch_internal.h"
#include "floats.h"

namespace tasq {

namespace {

__device__ __forceinline__ float add(float a, float b) { return a + b; }

// The threads of a row: a wave, or as many waves as its width takes.
template <bool WAVE> struct Team {
    int waves, first, group, t;         // first: the row's first wave; t: of its threads
    __device__ __forceinline__ explicit Team(int waves_) : waves(WAVE ? 1 : waves_)
    {
        const int wave = threadIdx.x >> 6;
        group = wave / waves;
        first = group * waves;
        t = (int)threadIdx.x - 64 * first;
    }
};

// Sums over the threads of a row, K at a time.  (Several waves a row: all rows of the
// workgroup together; two buffers in turn, so that one barrier a call is enough.)
constexpr int kMostWaves = 16;
template <bool WAVE, int K>
__device__ __forceinline__ void row_sums(const Team<WAVE> &team, float (&v)[K], int &turn)
{
#pragma unroll
    for (int i = 0; i < K; ++i)
        v[i] = group_reduce<64>(v[i], add);
    if constexpr (!WAVE) {
        __shared__ float part[2][kMostWaves][K];
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < K; ++i)
                part[turn][threadIdx.x >> 6][i] = v[i];
        }
        __syncthreads();
        // A lane a wave's part, the rest zeros.
        const int w = (int)(threadIdx.x & 15);
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const float p = part[turn][min(team.first + w, kMostWaves - 1)][i];
            v[i] = group_reduce<kMostWaves>(w < team.waves ? p : 0.0f, add);
        }
        turn ^= 1;
    }
}

// Where a thread's vectors of eight channels lie.  FULL: the width is a multiple of
// eight, so that a vector is whole or nothing.
template <int NV, bool FULL> struct Columns {
    int width, t, threads;
    __device__ __forceinline__ int k(int i) const { return 8 * (t + i * threads); }
    __device__ __forceinline__ bool some(int i) const { return k(i) < width; }
    __device__ __forceinline__ bool live(int i, int e) const
    {
        return FULL ? some(i) : k(i) + e < width;
    }
    // The vector's elements, zeros past the width.
    template <class T> __device__ __forceinline__ Packed<T, 8> load(const T *row, int i) const
    {
        const int at = k(i);
        Packed<T, 8> p = {};
        if (FULL ? at < width : at + 8 <= width) {
            p = *reinterpret_cast<const Packed<T, 8> *>(row + at);
        } else if (!FULL && at < width) {
            T e[8] = {};
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at + j < width)
                    e[j] = row[at + j];
            p = __builtin_bit_cast(Packed<T, 8>, e);
        }
        return p;
    }
    template <class T>
    __device__ __forceinline__ void store(T *row, int i, const float (&v)[8]) const
    {
        const int at = k(i);
        if (FULL ? at < width : at + 8 <= width) {
            Packed<T, 8> p;
            p.set(v);
            *reinterpret_cast<Packed<T, 8> *>(row + at) = p;
        } else if (!FULL && at < width) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (at + j < width)
                    row[at + j] = (T)v[j];
        }
    }
    // The same past the caches, for results that are larger than them.  (The gradient of
    // 8192 rows of 1152 in bfloat16: 30.0 us, 27.9 so; the forward pass 14.9 and 14.7, and
    // its results are read next.)
    template <class T>
    __device__ __forceinline__ void stream(T *row, int i, const float (&v)[8]) const
    {
        const int at = k(i);
        if (FULL ? at < width : at + 8 <= width) {
            typedef u32x4 __attribute__((aligned(2))) chunk_t;      // at any element
            constexpr int CHUNKS = 8 * (int)sizeof(T) / 16;
            struct Chunks {
                u32x4 c[CHUNKS];
            };
            Packed<T, 8> p;
            p.set(v);
            const Chunks u = __builtin_bit_cast(Chunks, p);
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
                __builtin_nontemporal_store(u.c[j], reinterpret_cast<chunk_t *>(row + at) + j);
        } else if (!FULL) {
            store(row, i, v);
        }
    }
    // Eight factors of a per-channel vector: `none` where there is none.
    template <class T>
    __device__ __forceinline__ void factors(const T *p, int i, float none, float (&v)[8]) const
    {
        if (p) {
            load(p, i).floats(v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = none;
        }
    }
    template <class T>
    __device__ __forceinline__ void modulation(const Modulation &m, bool wide, int b, int i,
                                               float none, float (&v)[8]) const
    {
        if (wide)
            factors(m.p ? static_cast<const float *>(m.p) + b * m.stride : nullptr, i, none, v);
        else
            factors(m.p ? static_cast<const T *>(m.p) + b * m.stride : nullptr, i, none, v);
    }
    // v less the mean, zeros past the width.
    __device__ __forceinline__ void centre(float (&v)[NV][8], float mean) const
    {
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] -= live(i, e) ? mean : 0.0f;
    }
};

// v centred (layer kind), and 1 / deviation.
template <bool WAVE, class Cols, int NV>
__device__ __forceinline__ float normalise(const NormCall &c, const Team<WAVE> &team,
                                           const Cols &at, float (&v)[NV][8], int &turn)
{
    if (c.layer) {
        float s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                s[0] += v[i][e];
        row_sums(team, s, turn);
        at.centre(v, s[0] * c.inv_width);
    }
    float q[1] = {0.0f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            q[0] += v[i][e] * v[i][e];
    row_sums(team, q, turn);
    return rsqrtf(q[0] * c.inv_width + c.eps);
}

// WAVE: rows of a wave each, four to a workgroup; else a row at a time.
template <class T, int NV, bool FULL, bool WAVE>
__global__ void __launch_bounds__(WAVE ? 256 : NV == 1 ? 512 : 1024) k_residual_norm(NormCall c)
{
    const Team<WAVE> team(c.waves);
    const long long unit = c.first_unit + (long long)blockIdx.x * (WAVE ? 4 : 1) + team.group;
    if (unit >= (long long)c.batch * c.chunks)
        return;                 // whole waves (WAVE), or nobody
    const int b = (int)(unit / c.chunks), s0 = (int)(unit % c.chunks) * c.rows;
    const int s1 = min(c.tokens, s0 + c.rows);
    const Columns<NV, FULL> at{c.width, team.t, 64 * team.waves};
    int turn = 0;
    float factor[NV][8], shift[NV][8], gate[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float w[8];
        at.factors(c.weight, i, 1.0f, w);
        at.template modulation<T>(c.scale, c.wide_mods, b, i, 0.0f, factor[i]);
        at.template modulation<T>(c.shift, c.wide_mods, b, i, 0.0f, shift[i]);
        at.template modulation<T>(c.gate, c.wide_mods, b, i, 1.0f, gate[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            factor[i][e] = w[e] * (1.0f + factor[i][e]);
    }
    const T *x = static_cast<const T *>(c.x) + b * c.x_stride[0];
    const T *y = static_cast<const T *>(c.y) + (c.y ? b * c.y_stride[0] : 0);
    const size_t out = (size_t)b * c.tokens;
    Packed<T, 8> xn[NV], yn[NV] = {};           // the next row, on its way
    auto fetch = [&](int s) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            xn[i] = at.load(x + s * c.x_stride[1], i);
            if (c.y)
                yn[i] = at.load(y + s * c.y_stride[1], i);
        }
    };
    fetch(s0);
    for (int s = s0; s < s1; ++s) {
        Packed<T, 8> xr[NV], yr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            xr[i] = xn[i];
            yr[i] = yn[i];
        }
        if (s + 1 < s1)
            fetch(s + 1);
        float v[NV][8];
        if (c.y) {
            float p[NV][8];
#pragma unroll
            for (int i = 0; i < NV; ++i)
                yr[i].floats(p[i]);
            if (c.post_weight) {
                const float d = normalise(c, team, at, p, turn);
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float w[8];
                    at.factors(c.post_weight, i, 1.0f, w);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        p[i][e] = p[i][e] * d * w[e];
                }
            }
            T *r = static_cast<T *>(c.r) + (out + s) * c.width;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                xr[i].floats(v[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[i][e] = c.alpha * v[i][e] + gate[i][e] * p[i][e];
                at.store(r, i, v[i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < NV; ++i)
                xr[i].floats(v[i]);
        }
        const float d = normalise(c, team, at, v, turn);
        T *h = static_cast<T *>(c.h) + (out + s) * c.width;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = v[i][e] * d * factor[i][e] + shift[i][e];
            at.store(h, i, v[i]);
        }
    }
}

// Most threads of a workgroup of the gradient: three waves a SIMD, whose registers
// hold a row of 16-bit values and its sums, or two for fp32.  Wider rows have sixteen
// channels a lane and the registers of 1024 threads, which are too few: they spill, one
// row at a time on a compute unit.  (Gradients of 33.5 M elements, channels: bfloat16,
// 403 MB, 76 us at 4096, 79 at 6144, 557 at 8192, 432 at 16384; fp32, 805 MB, 191 at 4096,
// 905 at 5120, 648 at 8192, 496 at 16384.)
template <class T, int NV> constexpr int kBackThreads = NV > 1 ? 1024 : sizeof(T) == 4 ? 512 : 768;

// A workgroup takes rows of one batch entry, every (chunks * groups)-th for each of
// its groups, with the sums over tokens in registers; the groups' meet in LDS and
// the workgroup's go to part[b][chunk], which k_norm_sums adds up in order.  (No
// atomics: their order would change the sums from run to run.)
template <class T, int NV, bool FULL, bool WAVE>
__global__ void __launch_bounds__((kBackThreads<T, NV>)) k_residual_norm_backward(NormCall c)
{
    constexpr bool AHEAD = NV == 1;
    const Team<WAVE> team(c.waves);
    const int groups = c.groups;
    const int b = (int)(blockIdx.x / (unsigned)c.chunks), chunk = blockIdx.x % (unsigned)c.chunks;
    const int group = team.group;
    const Columns<NV, FULL> at{c.width, team.t, 64 * team.waves};
    int turn = 0;
    float factor[NV][8], gate[NV][8];
    float dshift[NV][8] = {}, sum_p[NV][8] = {}, sum_q[NV][8] = {};
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        float w[8];
        at.factors(c.weight, i, 1.0f, w);
        at.template modulation<T>(c.scale, c.wide_mods, b, i, 0.0f, factor[i]);
        at.template modulation<T>(c.gate, c.wide_mods, b, i, 1.0f, gate[i]);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            factor[i][e] = w[e] * (1.0f + factor[i][e]);
        at.factors(c.post_weight, i, 1.0f, w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            gate[i][e] *= w[e];
    }
    const T *r = static_cast<const T *>(c.x) + b * c.x_stride[0];
    const T *y = static_cast<const T *>(c.y) + (c.y ? b * c.y_stride[0] : 0);
    const T *dh = static_cast<const T *>(c.dh) + b * c.dh_stride[0];
    const T *dr = static_cast<const T *>(c.dr) + (c.dr ? b * c.dr_stride[0] : 0);
    const size_t out = (size_t)b * c.tokens;
    const int step = c.chunks * groups;
    struct Rows {
        Packed<T, 8> r[NV], y[NV], dh[NV], dr[NV];
    } row = {}, next = {};
    // (A group past the last row has zeros.)
    auto fetch = [&](Rows &to, int s) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            to.r[i] = to.y[i] = to.dh[i] = to.dr[i] = {};
            if (s >= c.tokens)
                continue;
            to.r[i] = at.load(r + s * c.x_stride[1], i);
            to.dh[i] = at.load(dh + s * c.dh_stride[1], i);
            if (c.y)
                to.y[i] = at.load(y + s * c.y_stride[1], i);
            if (c.dr)
                to.dr[i] = at.load(dr + s * c.dr_stride[1], i);
        }
    };
    if constexpr (AHEAD)
        fetch(next, chunk * groups + group);
    // All groups of a workgroup together: they meet at its barriers.
    for (int s0 = chunk * groups; s0 < c.tokens; s0 += step) {
        const int s = s0 + group;
        const bool real = s < c.tokens;
        if constexpr (AHEAD) {
            row = next;
            fetch(next, s + step);
        } else {
            fetch(row, s);
        }
        float mean = 0.0f, mean_u = 0.0f;
        if (c.layer) {
            float m[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float n[8], u[8];
                row.r[i].floats(n);
                row.dh[i].floats(u);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    m[0] += n[e];
                    m[1] += u[e] * factor[i][e];
                }
            }
            row_sums(team, m, turn);
            mean = m[0] * c.inv_width;
            mean_u = m[1] * c.inv_width;
        }
        float q[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float n[8], u[8];
            row.r[i].floats(n);
            row.dh[i].floats(u);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                n[e] -= at.live(i, e) ? mean : 0.0f;
                q[0] += n[e] * n[e];
                q[1] += u[e] * factor[i][e] * n[e];
            }
        }
        row_sums(team, q, turn);
        const float d = real ? rsqrtf(q[0] * c.inv_width + c.eps) : 0.0f;
        const float inner = q[1] * d * c.inv_width;
        // D of vector i (and its part of the sums).
        auto back = [&](int i, float (&D)[8]) {
            float n[8], u[8];
            row.r[i].floats(n);
            row.dh[i].floats(u);
            row.dr[i].floats(D);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float ne = (n[e] - (at.live(i, e) ? mean : 0.0f)) * d;
                dshift[i][e] += u[e];
                sum_p[i][e] += u[e] * ne;
                D[e] += d * (u[e] * factor[i][e] - mean_u - ne * inner);
            }
        };
        T *dx = static_cast<T *>(c.dx) + (out + s) * c.width;
        T *dy = static_cast<T *>(c.dy) + (out + s) * c.width;
        if (!c.y) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float D[8];
                back(i, D);
                if (real)
                    at.stream(dx, i, D);
            }
        } else if (!c.post_weight) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float D[8], o[8], p[8];
                back(i, D);
                row.y[i].floats(p);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = c.alpha * D[e];
                    sum_q[i][e] += D[e] * p[e];
                    D[e] *= gate[i][e];
                }
                if (real)
                    at.stream(dx, i, o);
                if (real)
                    at.stream(dy, i, D);
            }
        } else {
            float p[NV][8], g[NV][8];
#pragma unroll
            for (int i = 0; i < NV; ++i)
                row.y[i].floats(p[i]);
            const float factor_y = normalise(c, team, at, p, turn);
            const float dev = real ? factor_y : 0.0f;
            float m[2] = {0.0f, 0.0f};
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float o[8];
                back(i, g[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    o[e] = c.alpha * g[i][e];
                    p[i][e] *= dev;
                    sum_q[i][e] += g[i][e] * p[i][e];
                    g[i][e] *= gate[i][e];
                    m[0] += at.live(i, e) ? g[i][e] : 0.0f;
                    m[1] += g[i][e] * p[i][e];
                }
                if (real)
                    at.stream(dx, i, o);
            }
            row_sums(team, m, turn);
            const float mean_g = c.layer ? m[0] * c.inv_width : 0.0f, in = m[1] * c.inv_width;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    p[i][e] = dev * (g[i][e] - mean_g - p[i][e] * in);
                if (real)
                    at.stream(dy, i, p[i]);
            }
        }
    }
    if (!c.sums)
        return;
    float *part = c.part + (size_t)blockIdx.x * 3 * c.width;
    if (groups == 1) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            at.store(part, i, dshift[i]);
            at.store(part + c.width, i, sum_p[i]);
            at.store(part + 2 * c.width, i, sum_q[i]);
        }
    } else {
        // (Groups of one row each have at most a workgroup's eight channels a thread.)
        __shared__ __attribute__((aligned(16))) float sum[8 * kBackThreads<T, 1>];
        const int channels = 8 * 64 * team.waves;
#pragma unroll
        for (int j = 0; j < 3; ++j) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const float *v = &(j == 0 ? dshift : j == 1 ? sum_p : sum_q)[0][e];
                *reinterpret_cast<float4 *>(&sum[group * channels + 8 * team.t + e]) =
                    make_float4(v[0], v[1], v[2], v[3]);
            }
            __syncthreads();
            for (int k = threadIdx.x; k < c.width; k += 64 * team.waves * groups) {
                float v = 0.0f;
                for (int g = 0; g < groups; ++g)
                    v += sum[g * channels + k];
                part[j * c.width + k] = v;
            }
        }
    }
}

// Adds the workgroups' parts up: a workgroup has 16 channels, 16 slices of the parts
// side by side, of one batch entry, or (sums.entries of them further) of all entries
// for what they share.
constexpr int kSumColumns = 16, kSumSlices = 16;

struct NormSums {
    int entries;                // with sums of their own: the batch, or 0
    int blocks;                 // of 16 channels
    int first;                  // workgroup of the launch
};

template <class T>
__global__ void __launch_bounds__(256) k_norm_sums(NormCall c, NormSums sums)
{
    const int col = threadIdx.x % kSumColumns, slice = threadIdx.x / kSumColumns;
    const int unit = sums.first + (int)blockIdx.x, entry = unit / sums.blocks;
    const int k = unit % sums.blocks * kSumColumns + col;
    __shared__ float sum[5][kSumSlices][kSumColumns + 1];
    const bool all = entry == sums.entries, on = k < c.width;
    const int b0 = all ? 0 : entry, b1 = all ? c.batch : b0 + 1;
    auto mod = [&](const Modulation &m, int b, float none) {
        if (!m.p)
            return none;
        return c.wide_mods ? static_cast<const float *>(m.p)[b * m.stride + k]
                           : (float)static_cast<const T *>(m.p)[b * m.stride + k];
    };
    // dshift, P, Q, sum_b (1 + scale) P, sum_b g Q
    float v[5] = {};
    if (on && c.chunks) {
        // Entries in turn, or with fewer chunks than slices several side by side.
        const int step = c.chunks >= kSumSlices ? 1 : kSumSlices / c.chunks;
        const int per = kSumSlices / step;
        const int eb = slice / per, first = slice % per;
        for (int b = eb < step ? b0 + eb : b1; b < b1; b += step) {
            const float *p = c.part + (size_t)b * c.chunks * 3 * c.width + k;
            float w[3] = {};
#pragma unroll 4
            for (int g = first; g < c.chunks; g += per)
#pragma unroll
                for (int j = 0; j < 3; ++j)
                    w[j] += p[((size_t)g * 3 + j) * c.width];
#pragma unroll
            for (int j = 0; j < 3; ++j)
                v[j] += w[j];
            if (all) {
                v[3] += w[1] * (1.0f + mod(c.scale, b, 0.0f));
                v[4] += w[2] * mod(c.gate, b, 1.0f);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 5; ++j)
        sum[j][slice][col] = v[j];
    __syncthreads();
    if (slice || !on)
        return;
#pragma unroll
    for (int j = 0; j < 5; ++j) {
        v[j] = 0.0f;
#pragma unroll
        for (int g = 0; g < kSumSlices; ++g)
            v[j] += sum[j][g][col];
    }
    const float w = c.weight ? c.weight[k] : 1.0f, wp = c.post_weight ? c.post_weight[k] : 1.0f;
    const size_t o = all ? (size_t)k : (size_t)b0 * c.width + k;
    if (c.dgate && all == ((c.shared & TASQ_SHARED_GATE) != 0))
        c.dgate[o] = wp * v[2];
    if (c.dscale && all == ((c.shared & TASQ_SHARED_SCALE) != 0))
        c.dscale[o] = w * v[1];
    if (c.dshift && all == ((c.shared & TASQ_SHARED_SHIFT) != 0))
        c.dshift[o] = v[0];
    if (all && c.dweight)
        c.dweight[k] = v[3];
    if (all && c.dpost)
        c.dpost[k] = v[4];
}

hipError_t launch_sums(const NormCall &c, hipStream_t stream)
{
    auto of_all = [&](int bit) { return (c.shared & bit) != 0; };
    const bool each = (c.dgate && !of_all(TASQ_SHARED_GATE)) ||
                      (c.dscale && !of_all(TASQ_SHARED_SCALE)) ||
                      (c.dshift && !of_all(TASQ_SHARED_SHIFT));
    const bool all = c.dweight || c.dpost || (c.dgate && of_all(TASQ_SHARED_GATE)) ||
                     (c.dscale && of_all(TASQ_SHARED_SCALE)) ||
                     (c.dshift && of_all(TASQ_SHARED_SHIFT));
    NormSums s;
    s.entries = each ? c.batch : 0;
    s.blocks = (c.width + kSumColumns - 1) / kSumColumns;
    const int units = (s.entries + (all ? 1 : 0)) * s.blocks;
    constexpr int MOST = 1 << 22;
    for (s.first = 0; s.first < units; s.first += MOST) {
        const unsigned grid = (unsigned)(units - s.first < MOST ? units - s.first : MOST);
        const hipError_t e = with_type(c.type, [&](auto zero) {
            k_norm_sums<decltype(zero)><<<grid, 256, 0, stream>>>(c, s);
            return hipGetLastError();
        });
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

// Waves of a row with NV vectors of eight channels a lane.
int waves_of(int width, int nv) { return (width + 512 * nv - 1) / (512 * nv); }

// Rows of a run in the forward pass: the modulations are read once for each run, and a
// row is requested while the one before is worked on.  Of more rows where there are
// enough to fill the card so.  (Runs of 1 / 2 / 4, us: 8192 rows of 1152 17.5 / 16.2 /
// 14.4, 4096 rows of 2240 18.0 / 15.9 / 14.1, 4096 of 1152 10.9 / 9.7 / 10.3, of 640 9.2
// / 9.3 / 9.5.)
int run_of(const NormCall &c)
{
    const long long rows = (long long)c.batch * c.tokens;
    const long long n = rows * c.width;
    return n >= 1 << 23 && rows >= 4096 ? 4 : n >= 1 << 22 && rows >= 2048 ? 2 : 1;
}

template <class T, int NV, bool FULL, bool WAVE> hipError_t forward(NormCall c, hipStream_t stream)
{
    constexpr int GROUPS = WAVE ? 4 : 1;
    c.waves = waves_of(c.width, NV);
    const long long units = (long long)c.batch * c.chunks;
    constexpr long long MOST = 1 << 20;         // workgroups of a launch
    for (c.first_unit = 0; c.first_unit < units; c.first_unit += MOST * GROUPS) {
        const long long left = (units - c.first_unit + GROUPS - 1) / GROUPS;
        k_residual_norm<T, NV, FULL, WAVE><<<(unsigned)(left < MOST ? left : MOST),
                                             64 * GROUPS * c.waves, 0, stream>>>(c);
        if (hipError_t e = hipGetLastError())
            return e;
    }
    return hipSuccess;
}

template <class T, int NV, bool FULL, bool WAVE>
hipError_t backward(const NormCall &c, hipStream_t stream)
{
    k_residual_norm_backward<T, NV, FULL, WAVE>
        <<<(unsigned)(c.batch * c.chunks), 64 * c.waves * c.groups, 0, stream>>>(c);
    return hipGetLastError();
}

// Eight channels a lane up to the workgroups' most, and sixteen.  (Rows of 1152 in
// bfloat16 with 24 channels a lane, a wave to a row: 17.5 us for 8192, 14.7 with three
// waves.  Sixteen spill a little: 33.5 M elements of bfloat16, 268 MB, 45 us at 4096
// channels, 73 at 5120, 51 at 8192, 65 at 16384; fp32 88, 189, 148, 175.)
constexpr int kWideForward = 8 * 512;

template <class T, bool FULL> hipError_t forward_width(const NormCall &c, hipStream_t stream)
{
    if (c.width <= 512)
        return forward<T, 1, FULL, true>(c, stream);
    if (c.width <= kWideForward)
        return forward<T, 1, FULL, false>(c, stream);
    return forward<T, 2, FULL, false>(c, stream);
}

template <class T, bool FULL> hipError_t backward_width(const NormCall &c, hipStream_t stream)
{
    if (c.width <= 512)
        return backward<T, 1, FULL, true>(c, stream);
    if (c.width <= 8 * kBackThreads<T, 1>)
        return backward<T, 1, FULL, false>(c, stream);
    return backward<T, 2, FULL, false>(c, stream);
}

}  // namespace

NormTeams residual_norm_teams(int type, int batch, int tokens, int width)
{
    const int threads = type == TASQ_TYPE_F32 ? kBackThreads<float, 1> : kBackThreads<bf16_t, 1>;
    const int nv = width <= 8 * threads ? 1 : 2;
    NormTeams n;
    n.waves = waves_of(width, nv);
    n.groups = nv == 1 && n.waves ? threads / 64 / n.waves : 1;
    n.groups = tokens < n.groups ? (tokens > 1 ? tokens : 1) : n.groups;
    const int want = (256 + batch - 1) / (batch > 0 ? batch : 1);
    const int most = (tokens + n.groups - 1) / n.groups;
    n.chunks = most < 1 ? 1 : want < most ? want : most;
    return n;
}

hipError_t launch_residual_norm(const NormCall &in, hipStream_t stream)
{
    NormCall c = in;
    c.inv_width = 1.0f / (float)c.width;
    c.rows = run_of(c);
    c.chunks = (c.tokens + c.rows - 1) / c.rows;
    return with_type(c.type, [&](auto zero) {
        using T = decltype(zero);
        return c.width % 8 == 0 ? forward_width<T, true>(c, stream)
                                : forward_width<T, false>(c, stream);
    });
}

hipError_t launch_residual_norm_backward(const NormCall &in, hipStream_t stream)
{
    NormCall c = in;
    c.inv_width = 1.0f / (float)c.width;
    if (c.batch && c.tokens) {
        const NormTeams n = residual_norm_teams(c.type, c.batch, c.tokens, c.width);
        c.chunks = n.chunks;
        c.waves = n.waves;
        c.groups = n.groups;
        const hipError_t e = with_type(c.type, [&](auto zero) {
            using T = decltype(zero);
            return c.width % 8 == 0 ? backward_width<T, true>(c, stream)
                                    : backward_width<T, false>(c, stream);
        });
        if (e != hipSuccess)
            return e;
    } else {
        c.chunks = 0;           // sums of nothing
    }
    return c.sums ? launch_sums(c, stream) : hipSuccess;
}

}  // namespace tasq
