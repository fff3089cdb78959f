// Attention, forward: O = softmax(scale Q K^T) V and its log-sum-exp, one pass
// over the keys with a running base and sum (the statistics, S and O in fp32; P
// is rounded to the inputs' type for the second product, as V is of that type;
// the sum takes the weights before that rounding).
//
// A workgroup of four waves has QB * 128 rows of one key head: (query head of
// the group, query) pairs, so that query heads which share keys share their
// loads; a wave has QB blocks of 32.  Tiles of 64 keys and values are staged in
// two LDS buffers, the next tile in flight while one is worked on.  With few rows the
// keys are cut into ranges, one workgroup each, whose partial results
// k_attn_join brings together.
//
// Bound by the products and the weights' vector instructions (a fused
// multiply-add, an exponential, an addition and half a conversion each), which
// take about as long, hardly overlap between the waves of a SIMD, and together
// leave it idle for 7% of the time at the 2.1 GHz that the power allows: 4096
// tokens among themselves, batch 2, 16 heads of 72 in bfloat16 (155 GFLOP) 186 us,
// 0.83 PFLOP/s, 8 heads of 128 137 us, 1.0; over texts of up to 300 words 21.
// One query over 8191 keys, 4 key heads of 128, batch 2 (a stream of 34 MB): 10.5
// and 3.7 for the join.
#pragma once

#include "attn.h"

namespace tasq {

// A row's weights are 2^(z - base), z in units of log2.  Floating-point weights
// keep their precision whatever the base, which only has to keep them and their
// products with values inside the range.  So it starts at 0 and no maximum is
// computed, unless a lane's sum over the first tile is outside [kLeast, kFirst) or
// over a later one reaches kMost: the tile's weights are then computed again with
// the base kRoom above the row's maximum, and its sums so far are rescaled.  In
// bfloat16 the sums thus hold values from 2^-100 to 2^105 over a hundred keys, and
// a base serves for scores that rise by 25 above the maximum it was taken from.
// (4096 tokens among themselves, 16 heads of 72, scores with a deviation of 1, 4, 8
// and 20: 192, 186, 186 and 210 us; with kFirst at 2^16 and no room 195, 212, 210 and
// 230.)
template <class T> struct Weights;
template <> struct Weights<bf16_t> {
    static constexpr float kLeast = 0x1p-16f, kFirst = 0x1p8f, kMost = 0x1p16f, kRoom = 20.0f;
};
template <> struct Weights<f16_t> {     // the largest half is 65504
    static constexpr float kLeast = 1.0f, kFirst = 0x1p15f, kMost = 0x1p15f, kRoom = 0.0f;
};

// What a wave holds of its QB blocks of 32 rows.
template <class T, int KS, int QB> struct Rows {
    static constexpr int DB = Tile<KS>::DB;
    u32x4 q[QB][KS];
    v16f_t o[QB][DB];
    float base[QB], sum[QB];

    // Lane l's row of block qb, l%32 of it: head and query of row m of the
    // (query head, query) pairs of key head hk.
    struct Row {
        bool ok;
        int head, s;
        __device__ __forceinline__ Row(const AttnCall &a, int hk, int first, int qb)
        {
            const int group = a.heads / a.kv_heads;
            const int m = first + 32 * qb + (int)(threadIdx.x & 31);
            ok = m < group * a.q_len;
            const int g = ok ? m / a.q_len : 0;
            s = ok ? m - g * a.q_len : 0;
            head = hk * group + g;
        }
    };

    __device__ __forceinline__ void init(const AttnCall &a, int b, int hk, int first)
    {
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const Row r(a, hk, first, qb);
            load_columns<KS>(static_cast<const T *>(a.q) + b * a.q_stride[0] +
                                 r.s * a.q_stride[1] + r.head * a.q_stride[2],
                             r.ok, a.dim, q[qb]);
            base[qb] = 0.0f;
            sum[qb] = 0.0f;
#pragma unroll
            for (int db = 0; db < DB; ++db)
                o[qb][db] = v16f_t{};
        }
    }

    // Sums of a tile that leave the base as it is, as bits: of the first tile and
    // of a later one.
    struct Sums {
        uint32_t least = __float_as_uint(Weights<T>::kLeast);
        uint32_t span = __float_as_uint(Weights<T>::kFirst) - __float_as_uint(Weights<T>::kLeast);
        __device__ __forceinline__ void later()
        {
            least = 0;
            span = __float_as_uint(Weights<T>::kMost);
        }
    };

    // 32 NR keys of a tile from row 32 rb on: x = K Q^T, the weights p,
    // o += V^T P^T.
    template <int NR>
    __device__ __forceinline__ void keys(const Tile<KS> &tile, const char *kt, const char *vt,
                                         int rb, float scale_log2, uint64_t live, Sums in)
    {
        v16f_t x[QB][NR];
        u32x4 p[QB][NR][2];
#pragma unroll
        for (int r = 0; r < NR; ++r)
            scores(tile, kt, rb + r, x, r);
        if (live != ~0ull) {
#pragma unroll
            for (int r = 0; r < NR; ++r)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float dead = dead_row(live, rb + r, i);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb)
                        x[qb][r][i] += dead;
                }
        }
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            float part = weights(scale_log2, base[qb], x[qb], p[qb]);
            // As bits, where NaN is above everything and less than least wraps.
            const bool out = __float_as_uint(part) - in.least >= in.span;
            if (__ballot(out)) {
                // The other rows keep their base, so that no row's result depends
                // on those beside it.
                const bool row_out =
                    across_halves(out ? 1.0f : 0.0f, [](float u, float v) { return u + v; }) != 0;
                const bool first = in.least != 0;
                float to = first ? -__builtin_huge_valf() : base[qb];
                float room = Weights<T>::kRoom;
                asm volatile("" : "+s"(room));      // or it holds a register all the time
#pragma unroll
                for (int r = 0; r < NR; ++r)
                    to = fmaxf(to, maximum(x[qb][r]) * scale_log2 + room);
                to = row_out ? to : base[qb];
                // No score above -inf: weights of zero.
                const float from = to == -__builtin_huge_valf() ? 0.0f : to;
                const float f = first ? 1.0f : __builtin_amdgcn_exp2f(base[qb] - from);
                base[qb] = to;
                sum[qb] *= f;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[qb][db][i] *= f;
                part = weights(scale_log2, from, x[qb], p[qb]);
            }
            sum[qb] += part;
        }
#pragma unroll
        for (int r = 0; r < NR; ++r)
            values(tile, vt, rb + r, p, r);
    }

    // x[..][at] = K Q^T for 32 keys of a tile, rows rb.
    template <int NR>
    __device__ __forceinline__ void scores(const Tile<KS> &tile, const char *kt, int rb,
                                           v16f_t (&x)[QB][NR], int at) const
    {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const u32x4 f = tile.rows(kt, rb, ks);
#pragma unroll
            for (int qb = 0; qb < QB; ++qb)
                x[qb][at] = mfma(T{}, f, q[qb][ks], ks ? x[qb][at] : v16f_t{});
        }
    }

    // o += V^T P^T for 32 keys of a tile, rows rb.
    template <int NR>
    __device__ __forceinline__ void values(const Tile<KS> &tile, const char *vt, int rb,
                                           const u32x4 (&p)[QB][NR][2], int at)
    {
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int db = 0; db < DB; ++db) {
                const u32x4 f = tile.columns(vt, 32 * rb + 16 * r, db);
#pragma unroll
                for (int qb = 0; qb < QB; ++qb)
                    o[qb][db] = mfma(T{}, f, p[qb][at][r], o[qb][db]);
            }
    }

    // Maximum of 32 scores of this lane's row.  (Four chains, here and below: a
    // result takes twice an instruction's time to be there for the next.)
    static __device__ __forceinline__ float maximum(const v16f_t &x)
    {
        float m[4];
#pragma unroll
        for (int i = 0; i < 16; ++i)
            m[i % 4] = i < 4 ? x[i] : fmaxf(m[i % 4], x[i]);
        return across_halves(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])),
                             [](float u, float v) { return fmaxf(u, v); });
    }

    // p = 2^(x scale - from), rounded as the next product's operand; returns the
    // lane's sum.
    template <int NR>
    static __device__ __forceinline__ float weights(float scale_log2, float from,
                                                    const v16f_t (&x)[NR], u32x4 (&p)[NR][2])
    {
        float s[4] = {};
#pragma unroll
        for (int r = 0; r < NR; ++r) {
            float e[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                e[i] = __builtin_amdgcn_exp2f(x[r][i] * scale_log2 - from);
                s[i % 4] += e[i];
            }
            p[r][0] = pack_rows<T>(e, 0);
            p[r][1] = pack_rows<T>(e, 1);
        }
        return (s[0] + s[1]) + (s[2] + s[3]);
    }

    // Writes the rows' results, or those of range sp of the keys.
    __device__ __forceinline__ void store(const AttnCall &a, int b, int hk, int first,
                                          int sp) const
    {
        const bool first_half = (threadIdx.x & 63) < 32;
#pragma unroll
        for (int qb = 0; qb < QB; ++qb) {
            const Row r(a, hk, first, qb);
            const float l = across_halves(sum[qb], [](float u, float v) { return u + v; });
            const bool none = __float_as_uint(l) == 0;
            const float inv = none ? 0.0f : 1.0f / l;
            const float lse = none ? -__builtin_huge_valf() : (base[qb] + __log2f(l)) * kLn2;
            const size_t row = ((size_t)b * a.heads + r.head) * a.q_len + r.s;
            if (a.splits > 1) {
                const size_t all = (size_t)a.batch * a.heads * a.q_len;
                store_columns_f32<DB>(a.part + (sp * all + row) * a.dim, r.ok, a.dim, o[qb],
                                      inv);
                if (r.ok && first_half)
                    a.part_lse[sp * all + row] = lse;
            } else {
                store_columns<T, DB>(static_cast<T *>(a.out) +
                                         (((size_t)b * a.q_len + r.s) * a.heads + r.head) *
                                             a.dim,
                                     r.ok, a.dim, o[qb], inv);
                if (a.lse && r.ok && first_half)
                    a.lse[row] = lse;
            }
        }
    }
};

template <class T, int KS, int QB>
__global__ void __launch_bounds__(256, QB == 1 && KS <= 5 ? 3 : 2) k_attn_forward(AttnCall a)
{
    constexpr int BM = 128 * QB, SIZE = Tile<KS>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[2][2 * SIZE];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int u = attn_unit(a);
    const int mt = u % a.row_tiles;
    u /= a.row_tiles;
    const int sp = u % a.splits;
    u /= a.splits;
    int hk, b;
    head_and_entry(a, u, hk, b);
    const int first = mt * BM + wave * 32 * QB;
    const bool busy = first < a.heads / a.kv_heads * a.q_len;   // the wave has rows
    Rows<T, KS, QB> rows;
    rows.init(a, b, hk, first);

    const int n = key_count(a, b);
    int t0, t1;
    key_range(a, n, sp, t0, t1);
    const long long *stride = wave < 2 ? a.k_stride : a.v_stride;
    const T *kv = static_cast<const T *>(wave < 2 ? a.k : a.v) + b * stride[0] + hk * stride[2];
    const long long step = kAttnTile * stride[1];
    const Tile<KS> tile;
    Stager<KS> stager;
    stager.init(wave, 2u * (uint32_t)stride[1], a.dim);
    uint64_t live = 0, now = 0;
    int next_byte = 0;
    typename Rows<T, KS, QB>::Sums in;
    if (t0 < t1) {
        now = live = live_keys(a, n, t0, mask_byte(a, b, n, t0));
        stager.request(kv + t0 * step, live, lds[0]);
        next_byte = mask_byte(a, b, n, t0 + 1);
        stager.wait();
        __syncthreads();
    }
    for (int t = t0; t < t1; ++t) {
        const char *kt = lds[(t - t0) & 1], *vt = kt + SIZE;
        if (t + 1 < t1) {
            live = live_keys(a, n, t + 1, next_byte);
            stager.request(kv + (t + 1) * step, live, lds[(t + 1 - t0) & 1]);
            next_byte = mask_byte(a, b, n, t + 2);
        }
        if (busy && now) {
            rows.template keys<2>(tile, kt, vt, 0, a.scale_log2, now, in);
            in.later();
        }
        now = live;
        stager.wait();
        __syncthreads();
    }
    rows.store(a, b, hk, first, sp);
}

// Brings the ranges of keys together: 32 lanes with four elements each have
// every SLICES-th range of a row, whose parts meet in LDS.
template <class T, int SLICES> __global__ void __launch_bounds__(256) k_attn_join(AttnCall a)
{
    constexpr int ROWS = 8 / SLICES;
    const int l = threadIdx.x & 31, slice = (threadIdx.x >> 5) % SLICES;
    const size_t all = (size_t)a.batch * a.heads * a.q_len;
    const size_t row = (size_t)blockIdx.x * ROWS + (threadIdx.x >> 5) / SLICES;
    const bool ok = row < all, has = ok && 4 * l < a.dim;
    float top = -__builtin_huge_valf(), sum = 0.0f, v[4] = {};
    if (ok)
        for (int sp = l; sp < a.splits; sp += 32)
            top = fmaxf(top, a.part_lse[sp * all + row]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1)
        top = fmaxf(top, __shfl_xor(top, off));
    const float base = top == -__builtin_huge_valf() ? 0.0f : top;
    if (ok) {
#pragma unroll 4
        for (int sp = slice; sp < a.splits; sp += SLICES) {
            const float w = __builtin_amdgcn_exp2f((a.part_lse[sp * all + row] - base) * kLog2e);
            float p[4] = {};
            if (has)
                load_vec(a.part + (sp * all + row) * a.dim + 4 * l, p);
            sum += w;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                v[i] += w * p[i];
        }
    }
    if constexpr (SLICES > 1) {
        __shared__ float sums[SLICES], vals[SLICES][TASQ_MAX_ATTENTION_DIM];
        store_vec(&vals[slice][4 * l], v);
        if (l == 0)
            sums[slice] = sum;
        __syncthreads();
        if (slice != 0)
            return;
#pragma unroll
        for (int i = 1; i < SLICES; ++i) {
            float p[4];
            load_vec(&vals[i][4 * l], p);
            sum += sums[i];
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] += p[e];
        }
    }
    const bool none = __float_as_uint(sum) == 0;
    const float inv = none ? 0.0f : 1.0f / sum;
    const int s = (int)(row % a.q_len);
    const size_t bh = row / a.q_len;
    const size_t head = bh % a.heads, b = bh / a.heads;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        v[i] *= inv;
    if (has)
        store_vec(static_cast<T *>(a.out) + ((b * a.q_len + s) * a.heads + head) * a.dim + 4 * l,
                  v);
    if (a.lse && ok && l == 0)
        a.lse[row] = none ? -__builtin_huge_valf() : base + __log2f(sum) * kLn2;
}

template <class T, int KS> hipError_t attn_forward_ks(const AttnCall &a, hipStream_t stream)
{
    const long long grid = (long long)a.batch * a.kv_heads * a.splits * a.row_tiles;
    void (*kernel)(AttnCall) = k_attn_forward<T, KS, 1>;
    if constexpr (KS >= kAttnWideFrom && KS <= kAttnWideSteps)
        if (a.row_blocks == 2)
            kernel = k_attn_forward<T, KS, 2>;
    return launch_units(kernel, a, grid, stream);
}

template <class T> hipError_t attn_forward_typed(const AttnCall &a, hipStream_t stream)
{
    hipError_t e;
    switch ((a.dim + 15) / 16) {
    case 1:
    case 2: e = attn_forward_ks<T, 2>(a, stream); break;
    case 3: e = attn_forward_ks<T, 3>(a, stream); break;
    case 4: e = attn_forward_ks<T, 4>(a, stream); break;
    case 5: e = attn_forward_ks<T, 5>(a, stream); break;
    case 6: e = attn_forward_ks<T, 6>(a, stream); break;
    case 7: e = attn_forward_ks<T, 7>(a, stream); break;
    default: e = attn_forward_ks<T, 8>(a, stream); break;
    }
    if (e != hipSuccess || a.splits == 1)
        return e;
    const size_t rows = (size_t)a.batch * a.heads * a.q_len;
    if (a.splits < 16)
        k_attn_join<T, 1><<<(unsigned)((rows + 7) / 8), 256, 0, stream>>>(a);
    else
        k_attn_join<T, 8><<<(unsigned)rows, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace tasq
