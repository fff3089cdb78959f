// Attention, forward: O = softmax(scale Q K^T) V and its log-sum-exp, one pass
// over the keys with a running maximum and sum (the statistics, S and O in
// fp32; P is rounded to the inputs' type for the second product, as V is of
// that type, after the running maximum has been taken off, so that its
// largest value is 1).
//
// A workgroup of four waves has QB * 128 rows of one key head: (query head of
// the group, query) pairs, so that query heads which share keys share their
// loads; a wave has QB blocks of 32.  Tiles of 64 keys and values are staged in
// two LDS buffers, the next tile in flight while one is worked on.  With few rows the
// keys are cut into ranges, one workgroup each, whose partial results
// k_attn_join brings together.
#pragma once

#include "attn.h"

namespace tasq {

// The running maximum (in units of log2) follows the row's true maximum only
// when that has risen by more than this: weights are then at most 2^kSlack,
// far inside the range of either type and of the sums, and most tiles leave
// the accumulators alone.
constexpr float kSlack = 8.0f;

template <class T, int KS, int QB>
__global__ void __launch_bounds__(256, QB == 1 && KS <= 5 ? 3 : 2) k_attn_forward(AttnCall a)
{
    constexpr int DB = Tile<KS>::DB, BM = 128 * QB, SIZE = Tile<KS>::kBytes;
    __shared__ __attribute__((aligned(16))) char lds[2][2 * SIZE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int u = attn_unit(blockIdx.x, gridDim.x);
    const int mt = u % a.row_tiles;
    u /= a.row_tiles;
    const int sp = u % a.splits;
    u /= a.splits;
    const int hk = u % a.kv_heads, b = u / a.kv_heads;
    const int group = a.heads / a.kv_heads;

    // This lane's rows.
    const int rows = group * a.q_len;
    const int first = mt * BM + wave * 32 * QB;
    const bool busy = first < rows;             // the wave has rows
    bool ok[QB];
    int head[QB], s[QB];
    u32x4 qf[QB][KS];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const int m = first + 32 * qb + (lane & 31);
        ok[qb] = m < rows;
        const int g = ok[qb] ? m / a.q_len : 0;
        s[qb] = ok[qb] ? m - g * a.q_len : 0;
        head[qb] = hk * group + g;
        load_columns<KS>(static_cast<const T *>(a.q) + b * a.q_stride[0] +
                             s[qb] * a.q_stride[1] + head[qb] * a.q_stride[2],
                         ok[qb], a.dim, qf[qb]);
    }

    const int n = key_count(a, b);
    const int t0 = sp * a.split_tiles;
    const int t1 = min((n + kAttnTile - 1) / kAttnTile, t0 + a.split_tiles);
    const long long *stride = wave < 2 ? a.k_stride : a.v_stride;
    const T *kv = static_cast<const T *>(wave < 2 ? a.k : a.v) + b * stride[0] + hk * stride[2];
    const long long step = kAttnTile * stride[1];

    v16f_t o[QB][DB];
    float top[QB], sum[QB];
#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        top[qb] = -__builtin_huge_valf();
        sum[qb] = 0.0f;
#pragma unroll
        for (int db = 0; db < DB; ++db)
            o[qb][db] = v16f_t{};
    }

    const Tile<KS> tile;
    Stager<KS> stager;
    stager.init(wave, 2u * (uint32_t)stride[1], a.dim);
    uint64_t live = 0, now = 0;
    int next_byte = 0;
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
            u32x4 p[QB][4];
            v16f_t x[QB][2];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const u32x4 f = tile.rows(kt, rb, ks);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb)
                        x[qb][rb] = mfma(T{}, f, qf[qb][ks], ks ? x[qb][rb] : v16f_t{});
                }
            if (now != ~0ull) {
#pragma unroll
                for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float dead = dead_row(now, rb, i);
#pragma unroll
                        for (int qb = 0; qb < QB; ++qb)
                            x[qb][rb][i] += dead;
                    }
            }
#pragma unroll
            for (int qb = 0; qb < QB; ++qb) {
                float mx = fmaxf(x[qb][0][0], x[qb][1][0]);
#pragma unroll
                for (int i = 1; i < 16; ++i)
                    mx = fmaxf(mx, fmaxf(x[qb][0][i], x[qb][1][i]));
                mx = across_halves(mx, [](float p, float q) { return fmaxf(p, q); });
                mx *= a.scale_log2;
                if (__ballot(mx > top[qb] + kSlack)) {
                    const float newtop = fmaxf(top[qb], mx);
                    // A row without a key so far has nothing to rescale.
                    const float f = newtop == -__builtin_huge_valf()
                                        ? 0.0f
                                        : __builtin_amdgcn_exp2f(top[qb] - newtop);
                    top[qb] = newtop;
                    sum[qb] *= f;
#pragma unroll
                    for (int db = 0; db < DB; ++db)
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            o[qb][db][i] *= f;
                }
                const float base = top[qb] == -__builtin_huge_valf() ? 0.0f : top[qb];
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    float e[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        e[i] = __builtin_amdgcn_exp2f(x[qb][rb][i] * a.scale_log2 - base);
                        sum[qb] += e[i];
                    }
                    p[qb][2 * rb] = pack_rows<T>(e, 0);
                    p[qb][2 * rb + 1] = pack_rows<T>(e, 1);
                }
            }
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    const u32x4 f = tile.columns(vt, 16 * r, db);
#pragma unroll
                    for (int qb = 0; qb < QB; ++qb)
                        o[qb][db] = mfma(T{}, f, p[qb][r], o[qb][db]);
                }
        }
        now = live;
        stager.wait();
        __syncthreads();
    }

#pragma unroll
    for (int qb = 0; qb < QB; ++qb) {
        const float l = across_halves(sum[qb], [](float p, float q) { return p + q; });
        const bool none = __float_as_uint(l) == 0;
        const float inv = none ? 0.0f : 1.0f / l;
        const float lse = none ? -__builtin_huge_valf() : (top[qb] + __log2f(l)) * kLn2;
        const size_t row = ((size_t)b * a.heads + head[qb]) * a.q_len + s[qb];
        if (a.splits > 1) {
            const size_t all = (size_t)a.batch * a.heads * a.q_len;
            store_columns_f32<DB>(a.part + (sp * all + row) * a.dim, ok[qb], a.dim, o[qb], inv);
            if (ok[qb] && lane < 32)
                a.part_lse[sp * all + row] = lse;
        } else {
            store_columns<T, DB>(static_cast<T *>(a.out) +
                                     (((size_t)b * a.q_len + s[qb]) * a.heads + head[qb]) *
                                         a.dim,
                                 ok[qb], a.dim, o[qb], inv);
            if (a.lse && ok[qb] && lane < 32)
                a.lse[row] = lse;
        }
    }
}

// Brings the ranges of keys together.  A workgroup has one row; its four waves
// take every fourth range, two elements to a lane, and meet in LDS.
template <class T> __global__ void __launch_bounds__(256) k_attn_join(AttnCall a)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const size_t all = (size_t)a.batch * a.heads * a.q_len, row = blockIdx.x;
    __shared__ float sums[4], vals[4][TASQ_MAX_ATTENTION_DIM];
    float top = -__builtin_huge_valf();
    for (int sp = lane; sp < a.splits; sp += 64)
        top = fmaxf(top, a.part_lse[sp * all + row]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        top = fmaxf(top, __shfl_xor(top, off));
    const float base = top == -__builtin_huge_valf() ? 0.0f : top;
    float sum = 0.0f, v0 = 0.0f, v1 = 0.0f;
    const bool ok = 2 * lane < a.dim;
#pragma unroll 4
    for (int sp = wave; sp < a.splits; sp += 4) {
        const float w = __builtin_amdgcn_exp2f((a.part_lse[sp * all + row] - base) * kLog2e);
        const float2 p = ok ? *reinterpret_cast<const float2 *>(
                                  a.part + (sp * all + row) * a.dim + 2 * lane)
                            : make_float2(0.0f, 0.0f);
        sum += w;
        v0 += w * p.x;
        v1 += w * p.y;
    }
    if (ok) {
        vals[wave][2 * lane] = v0;
        vals[wave][2 * lane + 1] = v1;
    }
    if (lane == 0)
        sums[wave] = sum;
    __syncthreads();
    if (wave != 0)
        return;
    sum = (sums[0] + sums[1]) + (sums[2] + sums[3]);
    const bool none = __float_as_uint(sum) == 0;
    const float inv = none ? 0.0f : 1.0f / sum;
    const int s = (int)(row % a.q_len), bh = (int)(row / a.q_len);
    const int head = bh % a.heads, b = bh / a.heads;
    if (ok) {
        float y[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            y[i] = ((vals[0][2 * lane + i] + vals[1][2 * lane + i]) +
                    (vals[2][2 * lane + i] + vals[3][2 * lane + i])) *
                   inv;
        *reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) +
                                      (((size_t)b * a.q_len + s) * a.heads + head) * a.dim +
                                      2 * lane) = pack2<T>(y[0], y[1]);
    }
    if (a.lse && lane == 0)
        a.lse[row] = none ? -__builtin_huge_valf() : base + __log2f(sum) * kLn2;
}

template <class T, int KS> hipError_t attn_forward_ks(const AttnCall &a, hipStream_t stream)
{
    const long long grid = (long long)a.batch * a.kv_heads * a.splits * a.row_tiles;
    if (grid == 0)
        return hipSuccess;
    void (*kernel)(AttnCall) = k_attn_forward<T, KS, 1>;
    if constexpr (KS <= kAttnWideSteps)
        if (a.row_blocks == 2)
            kernel = k_attn_forward<T, KS, 2>;
    kernel<<<(unsigned)grid, 256, 0, stream>>>(a);
    return hipGetLastError();
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
    const long long rows = (long long)a.batch * a.heads * a.q_len;
    k_attn_join<T><<<(unsigned)rows, 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace tasq
