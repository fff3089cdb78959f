// Attention, backward, from the kept O and log-sum-exp:
//   P = exp(scale Q K^T - lse),   dS = P (dO V^T - delta),
//   delta = rowsum(dO O),
//   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO.
// Two kernels, both recomputing S and dP, so that every gradient is summed in
// registers in a fixed order: k_attn_dq has the queries resident and streams
// keys and values, k_attn_dkdv has the keys resident and streams queries and
// output gradients (over all query heads that share the key head).  S, P, dP,
// dS and the sums are fp32; P and dS are rounded to the inputs' type as the
// operands of the products.
//
// A weight of a long row is small, and as fp32 or half it would lose bits or
// vanish, so the kernels hold P' = 2^kShift P (kShift is taken off the exponent's
// lse) and dS' = 2^at P (dO V^T - delta), and take the factors out of the sums at
// the end.  bfloat16 has fp32's range: both carry 2^12, so that weights down to 2^-138
// count and score gradients up to 2^115 do.  Half ends at 65504: P carries 2^14; dS, which is as large or small as the
// gradients are, has a power of two of its own (score_shift).
//
// Where there are few resident tiles the streamed axis is cut into ranges
// whose fp32 parts k_attn_sum adds up in order.
//
// Bound by chains of products and vector instructions with two waves to a SIMD
// (matrix units busy for a quarter to a third of the time, vector units for a
// third to a half): 4096 queries over 300 masked keys, batch 2, 16 heads of 72 in
// bfloat16 41 us for dQ and 45 for dK and dV; 4096 tokens among themselves, 10
// heads of 64 in half 114 and 138 (320 workgroups on 256 compute units); batch 2,
// 8 heads of 128 in bfloat16 489 together, 0.70 PFLOP/s of the five products that
// a gradient cannot do without.
#pragma once

#include "attn.h"

namespace tasq {

template <class T> struct Range;
template <> struct Range<bf16_t> {
    static constexpr int kShift = 12;
    static constexpr bool kFits = false;            // dS' needs no power of its own
};
template <> struct Range<f16_t> {
    static constexpr int kShift = 14;
    static constexpr bool kFits = true;
};

// Largest magnitude of eight packed elements.
template <class T> __device__ __forceinline__ float largest(u32x4 v)
{
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x2 f = unpack2<T>(v[i]);
        m = fmaxf(m, fmaxf(fabsf(f.x), fabsf(f.y)));
    }
    return m;
}

// The exponent that dS' of a column (a query of dQ, a key of dK) carries in half.
// It follows `top`, the largest of the upstream gradients that a kernel sees first
// (its query's, or its first tile's), to 2^8, which leaves room for |V| of 64 and
// more where one key has all the weight: a dS is off by its own rounding or by
// 2^-33 top.  Where that is too little room, sums come out infinite or NaN, and the
// workgroup runs again with those columns' exponents kLess lower.  |dS'| is below
// 2^55, so kRuns are enough for inputs that are finite themselves.
// (us against dS without a power of its own, which lost up to all of its bits below
// 2^-24 and overflowed above 65504: heads of 64, 4096 among themselves 231 and 224;
// of 72 675 and 657, over 300 words 97 and 90; of 128, 2048 191 and 175.  A check of
// every block with a branch instead took 248, 728, 97 and 193.)
constexpr int kRuns = 4, kLess = 15;

__device__ __forceinline__ int score_shift(float top)
{
    const uint32_t u = __float_as_uint(top);
    const bool some = u - 1 < 0x7f800000u - 1;      // not zero, finite
    return some ? min(8 + 127 - (int)(u >> 23), Range<f16_t>::kShift) : Range<f16_t>::kShift;
}

// Whether a column's sums, rows d below dim, hold an infinity or NaN.
template <int DB> __device__ __forceinline__ bool not_finite(const v16f_t (&sum)[DB], int dim)
{
    const int h = (threadIdx.x & 63) >> 5;
    float zero = 0.0f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i)
            if (32 * db + 8 * (i / 4) + 4 * h < dim)
                zero = fmaf(sum[db][i], 0.0f, zero);
    zero = across_halves(zero, [](float a, float b) { return a + b; });
    return zero != zero;
}

template <class T, int KS> __global__ void __launch_bounds__(256, 2) k_attn_dq(AttnCall a)
{
    constexpr int DB = Tile<KS>::DB, SIZE = Tile<KS>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[2][2 * SIZE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int u = attn_unit(a);
    const int mt = u % a.row_tiles;
    u /= a.row_tiles;
    const int sp = u % a.splits;
    u /= a.splits;
    int hk, b;
    head_and_entry(a, u, hk, b);
    const int group = a.heads / a.kv_heads;

    const int rows = group * a.q_len;
    const int m = mt * 128 + wave * 32 + (lane & 31);
    const bool ok = m < rows;
    const int g = ok ? m / a.q_len : 0, s = ok ? m - g * a.q_len : 0;
    const int head = hk * group + g;
    const bool busy = mt * 128 + wave * 32 < rows;
    const size_t at = (((size_t)b * a.q_len + s) * a.heads + head) * a.dim;
    const size_t row = ((size_t)b * a.heads + head) * a.q_len + s;
    u32x4 qf[KS], gf[KS];
    load_columns<KS>(static_cast<const T *>(a.q) + b * a.q_stride[0] + s * a.q_stride[1] +
                         head * a.q_stride[2],
                     ok, a.dim, qf);
    load_columns<KS>(static_cast<const T *>(a.dout) + b * a.dout_stride[0] +
                         s * a.dout_stride[1] + head * a.dout_stride[2],
                     ok, a.dim, gf);
    u32x4 of[KS];
    load_columns<KS>(static_cast<const T *>(a.out) + at, ok, a.dim, of);
    const float lse = ok ? a.lse[row] : 0.0f;

    const int n = key_count(a, b);
    int t0, t1;
    key_range(a, n, sp, t0, t1);
    const long long *stride = wave < 2 ? a.k_stride : a.v_stride;
    const T *kv = static_cast<const T *>(wave < 2 ? a.k : a.v) + b * stride[0] + hk * stride[2];
    const long long step = kAttnTile * stride[1];

    v16f_t dq[DB];
    const Tile<KS> tile;
    Stager<KS> stager;
    stager.init(wave, 2u * (uint32_t)stride[1], a.dim);
    uint64_t live = 0, now = 0;
    int next_byte = 0;
    auto begin = [&] {
#pragma unroll
        for (int db = 0; db < DB; ++db)
            dq[db] = v16f_t{};
        if (t0 < t1) {
            now = live = live_keys(a, n, t0, mask_byte(a, b, n, t0));
            stager.request(kv + t0 * step, live, lds[0]);
            next_byte = mask_byte(a, b, n, t0 + 1);
        }
    };
    begin();
    // While the first tile is on its way.
    float delta = 0.0f;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 x = unpack2<T>(of[ks][i]), y = unpack2<T>(gf[ks][i]);
            delta += x.x * y.x + x.y * y.y;
        }
    delta = across_halves(delta, [](float p, float q) { return p + q; });
    if (ok && lane < 32 && sp == 0)
        a.delta[row] = delta;
    int carried = Range<T>::kShift;
    if constexpr (Range<T>::kFits) {
        float top = 0.0f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
            top = fmaxf(top, largest<T>(gf[ks]));
        carried = score_shift(
            across_halves(top, [](float p, float q) { return fmaxf(p, q); }));
    }
    for (int run = 1;; ++run) {
        // A row without keys (lse = -inf) has P = 0.
        float lse2 = lse * kLog2e - (float)carried;
        if (lse2 == -__builtin_huge_valf())
            lse2 = __builtin_huge_valf();
        if (t0 < t1) {
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
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    v16f_t sa = {}, pa = {};
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        sa = mfma(T{}, tile.rows(kt, rb, ks), qf[ks], sa);
                        pa = mfma(T{}, tile.rows(vt, rb, ks), gf[ks], pa);
                    }
                    float x[16];
                    if (now != ~0ull) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            sa[i] += dead_row(now, rb, i);
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float p = __builtin_amdgcn_exp2f(sa[i] * a.scale_log2 - lse2);
                        x[i] = p * (pa[i] - delta);
                    }
#pragma unroll
                    for (int s2 = 0; s2 < 2; ++s2) {
                        const u32x4 ds = pack_rows<T>(x, s2);
#pragma unroll
                        for (int db = 0; db < DB; ++db)
                            dq[db] =
                                mfma(T{}, tile.columns(kt, 32 * rb + 16 * s2, db), ds, dq[db]);
                    }
                }
            }
            now = live;
            stager.wait();
            __syncthreads();
        }
        if (!Range<T>::kFits || run == kRuns)
            break;
        const bool over = ok && not_finite(dq, a.dim);
        if (!__syncthreads_or(over))
            break;
        carried -= over ? kLess : 0;
        begin();
    }
    const float back = ldexpf(a.scale, -carried);
    if (a.splits > 1)
        store_columns_f32<DB>(a.part + (size_t)sp * a.batch * a.q_len * a.heads * a.dim + at, ok,
                              a.dim, dq, back);
    else
        store_columns<T, DB>(static_cast<T *>(a.dq) + at, ok, a.dim, dq, back);
}

template <class T, int KS> __global__ void __launch_bounds__(256, 2) k_attn_dkdv(AttnCall a)
{
    constexpr int DB = Tile<KS>::DB, SIZE = Tile<KS>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[2][2 * SIZE];
    __shared__ __attribute__((aligned(16))) float stat[2][2][kAttnTile];    // lse, delta
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int u = attn_unit(a);
    const int kt_ = u % a.key_tiles;
    u /= a.key_tiles;
    const int sp = u % a.kv_splits;
    u /= a.kv_splits;
    int hk, b;
    head_and_entry(a, u, hk, b);
    const int group = a.heads / a.kv_heads;

    const int n = key_count(a, b);
    const int key = kt_ * 128 + wave * 32 + (lane & 31);
    const bool ok = key < a.kv_len;
    const bool counts =
        key < n && (!a.key_mask || a.key_mask[(size_t)b * a.kv_len + key] != 0);
    const bool busy = __ballot(counts) != 0;
    u32x4 kf[KS], vf[KS];
    load_columns<KS>(static_cast<const T *>(a.k) + b * a.k_stride[0] + key * a.k_stride[1] +
                         hk * a.k_stride[2],
                     counts, a.dim, kf);
    load_columns<KS>(static_cast<const T *>(a.v) + b * a.v_stride[0] + key * a.v_stride[1] +
                         hk * a.v_stride[2],
                     counts, a.dim, vf);

    v16f_t dk[DB], dv[DB];
    // Tiles of 64 queries, the group's heads one after the other.
    const int per_head = (a.q_len + kAttnTile - 1) / kAttnTile;
    const int t0 = sp * a.kv_split_tiles;
    const int t1 = kt_ * 128 < n ? min(group * per_head, t0 + a.kv_split_tiles) : t0;
    const Tile<KS> tile;
    const long long *stride = wave < 2 ? a.q_stride : a.dout_stride;
    const T *from = static_cast<const T *>(wave < 2 ? a.q : a.dout) + b * stride[0];
    Stager<KS> stager;
    stager.init(wave, 2u * (uint32_t)stride[1], a.dim);
    float st = 0.0f;
    int g = 0, s0 = 0;          // head and first row of the next tile
    auto fetch = [&](int i) {
        const int left = a.q_len - s0, head = hk * group + g;
        const uint64_t live = left >= kAttnTile ? ~0ull : (1ull << left) - 1;
        stager.request(from + s0 * stride[1] + head * stride[2], live, lds[i]);
        if (wave < 2) {         // wave 0 has the rows' lse, wave 1 their delta
            const float *p = wave == 0 ? a.lse : a.delta;
            st = wave == 0 ? -__builtin_huge_valf() : 0.0f;
            if (lane < left)
                st = p[((size_t)b * a.heads + head) * a.q_len + s0 + lane];
        }
        s0 += kAttnTile;
        if (s0 >= a.q_len) {
            s0 = 0;
            ++g;
        }
    };
    // The rows' statistics are looked at here, when they have arrived, and not
    // where they are requested (4096 tokens among themselves, 16 heads of 64: two of
    // four waves waited 800 of 4100 cycles a tile there).
    auto put = [&](int i) {
        stager.wait();
        if (wave == 0) {        // rows past the end and rows without keys have P = 0
            const float l = st * kLog2e - (float)Range<T>::kShift;
            stat[i][0][lane] = l == -__builtin_huge_valf() ? __builtin_huge_valf() : l;
        } else if (wave == 1) {
            stat[i][1][lane] = Range<T>::kFits ? -st : st;
        }
    };
    auto begin = [&] {
#pragma unroll
        for (int db = 0; db < DB; ++db)
            dk[db] = dv[db] = v16f_t{};
        g = per_head ? t0 / per_head : 0;
        s0 = (t0 - g * per_head) * kAttnTile;
        if (t0 < t1) {
            fetch(0);
            put(0);
            __syncthreads();
        }
    };
    begin();
    int carried = Range<T>::kShift;
    if constexpr (Range<T>::kFits) {
        float top = 0.0f;
        if (t0 < t1) {
#pragma unroll
            for (int i = 0; i < 2 * KS; ++i)
                top = fmaxf(top, largest<T>(*reinterpret_cast<const u32x4 *>(
                                     lds[0] + SIZE + 16 * (64 * i + lane))));
        }
        carried = score_shift(
            group_reduce<64>(top, [](float p, float q) { return fmaxf(p, q); }));
    }
    for (int run = 1;; ++run) {
        const float lift = ldexpf(1.0f, carried - Range<T>::kShift);     // dS' over P' (..)
        for (int t = t0; t < t1; ++t) {
            const int cur = (t - t0) & 1;
            const char *qt = lds[cur], *gt = qt + SIZE;
            if (t + 1 < t1)
                fetch(cur ^ 1);
            if (busy) {
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    v16f_t sa = {}, pa = {};
                    if constexpr (Range<T>::kFits) {    // minus delta to begin with
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const float4 d = *reinterpret_cast<const float4 *>(
                                &stat[cur][1][32 * rb + 8 * q + 4 * (lane >> 5)]);
                            pa[4 * q] = d.x;
                            pa[4 * q + 1] = d.y;
                            pa[4 * q + 2] = d.z;
                            pa[4 * q + 3] = d.w;
                        }
                    }
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        sa = mfma(T{}, tile.rows(qt, rb, ks), kf[ks], sa);
                        pa = mfma(T{}, tile.rows(gt, rb, ks), vf[ks], pa);
                    }
                    float p[16], x[16];
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const int r = 32 * rb + 8 * q + 4 * (lane >> 5);
                        const float4 l = *reinterpret_cast<const float4 *>(&stat[cur][0][r]);
                        const float ls[4] = {l.x, l.y, l.z, l.w};
                        float de[4] = {};
                        if constexpr (!Range<T>::kFits) {
                            const float4 d = *reinterpret_cast<const float4 *>(&stat[cur][1][r]);
                            de[0] = d.x;
                            de[1] = d.y;
                            de[2] = d.z;
                            de[3] = d.w;
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            p[4 * q + i] =
                                __builtin_amdgcn_exp2f(sa[4 * q + i] * a.scale_log2 - ls[i]);
                            x[4 * q + i] = p[4 * q + i] * (pa[4 * q + i] - de[i]);
                            if constexpr (Range<T>::kFits)
                                x[4 * q + i] *= lift;
                        }
                    }
#pragma unroll
                    for (int s2 = 0; s2 < 2; ++s2) {
                        const u32x4 pf = pack_rows<T>(p, s2), ds = pack_rows<T>(x, s2);
#pragma unroll
                        for (int db = 0; db < DB; ++db) {
                            dv[db] =
                                mfma(T{}, tile.columns(gt, 32 * rb + 16 * s2, db), pf, dv[db]);
                            dk[db] =
                                mfma(T{}, tile.columns(qt, 32 * rb + 16 * s2, db), ds, dk[db]);
                        }
                    }
                }
            }
            if (t + 1 < t1)
                put(cur ^ 1);
            __syncthreads();
        }
        if (!Range<T>::kFits || run == kRuns)
            break;
        const bool over = counts && not_finite(dk, a.dim);
        if (!__syncthreads_or(over))
            break;
        carried -= over ? kLess : 0;
        begin();
    }
    // Keys that do not count have gradients of zero.
    if (!counts) {
#pragma unroll
        for (int db = 0; db < DB; ++db)
            dk[db] = dv[db] = v16f_t{};
    }
    const size_t at = (((size_t)b * a.kv_len + key) * a.kv_heads + hk) * a.dim;
    const float back = ldexpf(a.scale, -carried), back_v = ldexpf(1.0f, -Range<T>::kShift);
    if (a.kv_splits > 1) {
        const size_t all = (size_t)a.batch * a.kv_len * a.kv_heads * a.dim;
        store_columns_f32<DB>(a.kv_part + 2 * sp * all + at, ok, a.dim, dk, back);
        store_columns_f32<DB>(a.kv_part + (2 * sp + 1) * all + at, ok, a.dim, dv, back_v);
    } else {
        store_columns<T, DB>(static_cast<T *>(a.dk) + at, ok, a.dim, dk, back);
        store_columns<T, DB>(static_cast<T *>(a.dv) + at, ok, a.dim, dv, back_v);
    }
}

// out[i] = sum of `parts` fp32 parts, `step` elements apart, in order and four
// elements at a time (a head has a multiple of eight).  The gradients that were
// cut into ranges share a launch, one row of workgroups each: for dK and dV of
// 300 keys in 5 ranges two launches took 4.7 us each.
struct Sums {
    const float *part[3];
    void *out[3];
    size_t n[3], step[3];
    int parts[3], count;
};

template <class T> __global__ void __launch_bounds__(256) k_attn_sum(Sums sums)
{
    const int j = blockIdx.y;
    const size_t i = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
    if (i >= sums.n[j])
        return;
    const float *from = sums.part[j] + i;
    const size_t step = sums.step[j];
    const int parts = sums.parts[j];
    float s[4] = {};
#pragma unroll 4
    for (int p = 0; p < parts; ++p) {
        float v[4];
        load_vec(from + p * step, v);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            s[e] += v[e];
    }
    store_vec(static_cast<T *>(sums.out[j]) + i, s);
}

template <class T, int KS> hipError_t attn_backward_ks(const AttnCall &a, hipStream_t stream)
{
    const long long rows = (long long)a.batch * a.kv_heads * a.splits * a.row_tiles;
    const long long keys = (long long)a.batch * a.kv_heads * a.kv_splits * a.key_tiles;
    hipError_t e = launch_units(k_attn_dq<T, KS>, a, rows, stream);
    if (e == hipSuccess)
        e = launch_units(k_attn_dkdv<T, KS>, a, keys, stream);
    const size_t nq = (size_t)a.batch * a.q_len * a.heads * a.dim;
    const size_t nk = (size_t)a.batch * a.kv_len * a.kv_heads * a.dim;
    Sums sums{};
    size_t most = 0;
    auto add = [&](const float *part, size_t n, size_t step, int parts, void *out) {
        const int j = sums.count++;
        sums.part[j] = part;
        sums.out[j] = out;
        sums.n[j] = n;
        sums.step[j] = step;
        sums.parts[j] = parts;
        most = n > most ? n : most;
    };
    if (a.splits > 1)
        add(a.part, nq, nq, a.splits, a.dq);
    if (a.kv_splits > 1) {
        add(a.kv_part, nk, 2 * nk, a.kv_splits, a.dk);
        add(a.kv_part + nk, nk, 2 * nk, a.kv_splits, a.dv);
    }
    if (e == hipSuccess && most > 0) {
        k_attn_sum<T><<<dim3((unsigned)((most / 4 + 255) / 256), (unsigned)sums.count), 256, 0,
                        stream>>>(sums);
        e = hipGetLastError();
    }
    return e;
}

template <class T> hipError_t attn_backward_typed(const AttnCall &a, hipStream_t stream)
{
    switch ((a.dim + 15) / 16) {
    case 1:
    case 2: return attn_backward_ks<T, 2>(a, stream);
    case 3: return attn_backward_ks<T, 3>(a, stream);
    case 4: return attn_backward_ks<T, 4>(a, stream);
    case 5: return attn_backward_ks<T, 5>(a, stream);
    case 6: return attn_backward_ks<T, 6>(a, stream);
    case 7: return attn_backward_ks<T, 7>(a, stream);
    default: return attn_backward_ks<T, 8>(a, stream);
    }
}

}  // namespace tasq
