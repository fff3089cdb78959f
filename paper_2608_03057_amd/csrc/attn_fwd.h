// Attention, forward: O = softmax(scale Q K^T) V and its log-sum-exp, one pass
// over the keys with a running maximum and sum (the statistics, S and O in
// fp32; P is rounded to the inputs' type for the second product, as V is of
// that type, after the running maximum has been taken off, so that its
// largest value is 1).
//
// A workgroup has 128 rows of one key head: (query head of the group, query)
// pairs, so that query heads which share keys share their loads; a wave has 32
// of them.  Tiles of 64 keys and values are staged in two LDS buffers, the
// next tile in flight in registers.  With few rows the keys are cut into
// ranges, one workgroup each, whose partial results k_attn_join brings
// together.
#pragma once

#include "attn.h"

namespace tasq {

template <class T, int KS>
__global__ void __launch_bounds__(256, KS <= 6 ? 3 : 2) k_attn_forward(AttnCall a)
{
    constexpr int NT = 256, DB = Tile<KS>::DB;
    __shared__ __attribute__((aligned(16))) char lds[2][2][Tile<KS>::kBytes];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int u = attn_unit(blockIdx.x, gridDim.x);
    const int mt = u % a.row_tiles;
    u /= a.row_tiles;
    const int sp = u % a.splits;
    u /= a.splits;
    const int hk = u % a.kv_heads, b = u / a.kv_heads;
    const int group = a.heads / a.kv_heads;

    // This lane's row.
    const int rows = group * a.q_len;
    const int m = mt * 128 + wave * 32 + (lane & 31);
    const bool ok = m < rows;
    const int g = ok ? m / a.q_len : 0, s = ok ? m - g * a.q_len : 0;
    const int head = hk * group + g;
    const bool busy = mt * 128 + wave * 32 < rows;      // the wave has rows
    u32x4 qf[KS];
    load_columns<KS>(static_cast<const T *>(a.q) + b * a.q_stride[0] + s * a.q_stride[1] +
                         head * a.q_stride[2],
                     ok, a.dim, qf);

    const int n = key_count(a, b);
    const int t0 = sp * a.split_tiles;
    const int t1 = min((n + kAttnTile - 1) / kAttnTile, t0 + a.split_tiles);
    const T *k = static_cast<const T *>(a.k) + b * a.k_stride[0] + hk * a.k_stride[2];
    const T *v = static_cast<const T *>(a.v) + b * a.v_stride[0] + hk * a.v_stride[2];
    const uint32_t kb = 2u * (uint32_t)a.k_stride[1], vb = 2u * (uint32_t)a.v_stride[1];

    v16f_t o[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
        o[db] = v16f_t{};
    float top = -__builtin_huge_valf(), sum = 0.0f;

    Stage<KS, NT> kst, vst;
    uint64_t live = 0;
    int next_byte = 0;
    auto fetch = [&](int t) {
        kst.load(k + (size_t)t * kAttnTile * a.k_stride[1], kb, a.dim, live);
        vst.load(v + (size_t)t * kAttnTile * a.v_stride[1], vb, a.dim, live);
    };
    uint64_t now = 0;
    if (t0 < t1) {
        now = live = live_keys(a, n, t0, mask_byte(a, b, n, t0));
        fetch(t0);
        next_byte = mask_byte(a, b, n, t0 + 1);
        kst.store(lds[0][0]);
        vst.store(lds[0][1]);
        __syncthreads();
    }
    for (int t = t0; t < t1; ++t) {
        const char *kt = lds[(t - t0) & 1][0], *vt = lds[(t - t0) & 1][1];
        if (t + 1 < t1) {
            live = live_keys(a, n, t + 1, next_byte);
            fetch(t + 1);
            next_byte = mask_byte(a, b, n, t + 2);
        }
        if (busy && now) {
            float x[2][16];
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) {
                v16f_t acc = {};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks)
                    acc = mfma(T{}, Tile<KS>::rows(kt, rb, ks), qf[ks], acc);
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    x[rb][i] = acc[i];
            }
            if (now != ~0ull) {
#pragma unroll
                for (int rb = 0; rb < 2; ++rb) {
                    const uint32_t bits = (uint32_t)(now >> (32 * rb)) >> (4 * (lane >> 5));
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        if (!((bits >> (8 * (i / 4) + i % 4)) & 1))
                            x[rb][i] = -__builtin_huge_valf();
                }
            }
            float mx = x[0][0];
#pragma unroll
            for (int i = 0; i < 16; ++i)
                mx = fmaxf(mx, fmaxf(x[0][i], x[1][i]));
            mx = across_halves(mx, [](float p, float q) { return fmaxf(p, q); });
            const float newtop = fmaxf(top, mx * a.scale_log2);
            // A row without a key so far keeps exponents of -inf.
            const float base = newtop == -__builtin_huge_valf() ? 0.0f : newtop;
            if (__ballot(newtop != top)) {
                const float f = __builtin_amdgcn_exp2f(top - base);
                sum *= f;
#pragma unroll
                for (int db = 0; db < DB; ++db)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        o[db][i] *= f;
            }
            top = newtop;
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    x[rb][i] = __builtin_amdgcn_exp2f(x[rb][i] * a.scale_log2 - base);
                    sum += x[rb][i];
                }
#pragma unroll
            for (int rb = 0; rb < 2; ++rb)
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2) {
                    const u32x4 p = pack_rows<T>(x[rb], s2);
#pragma unroll
                    for (int db = 0; db < DB; ++db)
                        o[db] = mfma(T{}, Tile<KS>::columns(vt, 32 * rb + 16 * s2, db), p, o[db]);
                }
        }
        now = live;
        if (t + 1 < t1) {
            kst.store(lds[(t + 1 - t0) & 1][0]);
            vst.store(lds[(t + 1 - t0) & 1][1]);
        }
        __syncthreads();
    }

    sum = across_halves(sum, [](float p, float q) { return p + q; });
    const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
    const float lse = sum == 0.0f ? -__builtin_huge_valf() : (top + __log2f(sum)) * kLn2;
    const size_t row = ((size_t)b * a.heads + head) * a.q_len + s;
    if (a.splits > 1) {
        const size_t all = (size_t)a.batch * a.heads * a.q_len;
        store_columns_f32<DB>(a.part + (sp * all + row) * a.dim, ok, a.dim, o, inv);
        if (ok && lane < 32)
            a.part_lse[sp * all + row] = lse;
        return;
    }
    store_columns<T, DB>(static_cast<T *>(a.out) +
                             (((size_t)b * a.q_len + s) * a.heads + head) * a.dim,
                         ok, a.dim, o, inv);
    if (a.lse && ok && lane < 32)
        a.lse[row] = lse;
}

// Brings the ranges of keys together: a wave per row, two elements to a lane.
template <class T> __global__ void __launch_bounds__(256) k_attn_join(AttnCall a)
{
    const int lane = threadIdx.x & 63;
    const long long all = (long long)a.batch * a.heads * a.q_len;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= all)
        return;
    float top = -__builtin_huge_valf();
    for (int sp = lane; sp < a.splits; sp += 64)
        top = fmaxf(top, a.part_lse[sp * all + row]);
#pragma unroll
    for (int off = 32; off > 0; off >>= 1)
        top = fmaxf(top, __shfl_xor(top, off));
    const float base = top == -__builtin_huge_valf() ? 0.0f : top;
    float sum = 0.0f, v0 = 0.0f, v1 = 0.0f;
    const bool ok = 2 * lane < a.dim;
    for (int sp = 0; sp < a.splits; ++sp) {
        const float w = __builtin_amdgcn_exp2f((a.part_lse[sp * all + row] - base) * kLog2e);
        sum += w;
        if (ok) {
            const float2 p =
                *reinterpret_cast<const float2 *>(a.part + (sp * all + row) * a.dim + 2 * lane);
            v0 += w * p.x;
            v1 += w * p.y;
        }
    }
    const float inv = sum > 0.0f ? 1.0f / sum : sum == 0.0f ? 0.0f : sum;
    const int s = (int)(row % a.q_len), bh = (int)(row / a.q_len);
    const int head = bh % a.heads, b = bh / a.heads;
    if (ok)
        *reinterpret_cast<uint32_t *>(static_cast<T *>(a.out) +
                                      (((size_t)b * a.q_len + s) * a.heads + head) * a.dim +
                                      2 * lane) = pack2<T>(v0 * inv, v1 * inv);
    if (a.lse && lane == 0)
        a.lse[row] = sum == 0.0f ? -__builtin_huge_valf() : base + __log2f(sum) * kLn2;
}

template <class T, int KS> hipError_t attn_forward_ks(const AttnCall &a, hipStream_t stream)
{
    const long long grid = (long long)a.batch * a.kv_heads * a.splits * a.row_tiles;
    if (grid == 0)
        return hipSuccess;
    k_attn_forward<T, KS><<<(unsigned)grid, 256, 0, stream>>>(a);
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
    k_attn_join<T><<<(unsigned)((rows + 3) / 4), 256, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace tasq
