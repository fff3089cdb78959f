// The token-scaled linear's gradient over many tokens: both operands in dy's type.
//
// Turning codes into values costs the K loop of token_grad.h as much as it can hide (88
// vector instructions a wave and 64 rows beside 32 products), and every tile of rows
// does it again.  Here a pass of its own writes s[z] q[z][c] once, rounded to dy's type
// (rows filled up to whole 16-byte chunks; dy too, where its own are not), and the
// product is one of two 16-bit matrices whose rows go to LDS directly: no registers and
// no vector instructions but addresses between memory and the matrix unit.  Bound by the
// matrix unit at the clock that the power allows it (2.0 to 2.2 GHz, busy 0.42 to 0.48):
// medians, 8192 tokens of 1152 -> 3456 77 us a product (the least 70) and 10 for the
// values, 4096 of 2240 -> 11200 206 (by card up to 245) and 19.
#pragma once

#include "token_grad.h"

namespace tasq {

namespace {

constexpr int kTileStep = 32;   // of the summed axis

// Tiles of BC columns by BR rows, WC x WR waves.  Rows of Q, and of A turned, are a
// step's stage in a ring of NS; of A as it lies a stage has two steps, so that a row's
// part is a whole cache line.  (With one step to a stage, half lines, 4096x2240 ->
// 11200 took 231 us for dx.)
template <int BC_, int BR_, int WC_, int WR_, int NS_, int NA_, bool TURNED_> struct TileCfg {
    static constexpr int BC = BC_, BR = BR_, WC = WC_, WR = WR_, NT = 64 * WC * WR;
    static constexpr bool TURNED = TURNED_;
    static constexpr int FC = BC / WC / 32, FR = BR / WR / 32;
    static constexpr int SPAN = TURNED ? 1 : 2;                 // steps of a stage of A
    static constexpr int NS = NS_, NA = TURNED ? NS_ : NA_;     // stages of Q and A
    static_assert(NS - 2 < SPAN * (NA - 1), "rows of A are asked for before those of Q");
    static constexpr int A_BYTES = BR * SPAN * kTileStep * 2, Q_BYTES = BC * kTileStep * 2;
    static constexpr int A_LOADS = A_BYTES / 16 / NT;           // of a thread
    static constexpr int Q_LOADS = (Q_BYTES / 16 + NT - 1) / NT;
    static_assert(A_BYTES % (16 * NT) == 0, "whole loads of A");
    // Threads without a chunk of Q in the last load write zeros behind the stages.
    static constexpr int Q0 = NA * A_BYTES, SPARE0 = Q0 + NS * Q_BYTES;
    static constexpr int LDS = SPARE0 + Q_LOADS * 16 * NT - Q_BYTES;
    // Requests of a wave that follow those of step t + 1 (and of its rows of A) when
    // step t, part `half` of a stage of A, ends: of NS - 2 steps.
    static constexpr int ahead(int half)
    {
        int n = 0;
        for (int d = 0; d < NS - 2; ++d)
            n += Q_LOADS + ((half + SPAN * NS - d) % SPAN == 0 ? A_LOADS : 0);
        return n;
    }
};

template <class T, class C>
__device__ __forceinline__ void grad_gemm_tile(const GradGemm &g, int tr, int tc, int split,
                                               char *sm)
{
    constexpr bool TURNED = C::TURNED;
    constexpr int A_PITCH = TURNED ? 2 * C::BR : 2 * C::SPAN * kTileStep;
    constexpr int Q_PITCH = 2 * C::BC;
    const int lane = threadIdx.x & 63;
    const int wave = (int)uniform(threadIdx.x >> 6);
    const int wc = wave % C::WC, wr = wave / C::WC;
    const int r0 = tr * C::BR, c0 = tc * C::BC;
    const int z0 = split * g.split_steps * kTileStep;
    const int z1 = min(g.Z, z0 + g.split_steps * kTileStep);
    const int steps = (z1 - z0 + kTileStep - 1) / kTileStep;
    const T *A = static_cast<const T *>(g.A), *Q = static_cast<const T *>(g.Q);
    const uint32_t lds0 = lds_offset(sm);

    // This lane's chunks: of A one column in all its rows, of Q each its own.
    constexpr int A_CH = A_PITCH / 16, Q_CH = Q_PITCH / 16;
    constexpr int A_NEXT = C::NT / A_CH;            // rows between a thread's chunks
    static_assert(C::NT % A_CH == 0 && A_NEXT % 16 == 0, "one column a lane");
    const int a_row = (int)threadIdx.x / A_CH, a_place = (int)threadIdx.x % A_CH;
    const int a_col = 8 * (TURNED ? a_place ^ (4 * turn_key<A_PITCH>(a_row))
                                  : a_place ^ ((a_row >> 1) & 7));
    const uint32_t a_pitch = 2u * (uint32_t)g.a_stride, q_pitch = 2u * (uint32_t)g.q_stride;
    const uint32_t a_off = TURNED && a_col >= g.R - r0
                               ? kOOB
                               : (uint32_t)a_row * a_pitch + 2u * (uint32_t)a_col;
    const uint32_t a_rows = uniform(min(g.R - r0, C::BR));
    uint32_t q_off[C::Q_LOADS];
#pragma unroll
    for (int i = 0; i < C::Q_LOADS; ++i) {
        const int p = i * C::NT + (int)threadIdx.x, row = p / Q_CH;
        const int c = 8 * ((p % Q_CH) ^ (4 * turn_key<Q_PITCH>(row)));
        q_off[i] = row < kTileStep && c0 + c < g.C
                       ? (uint32_t)row * q_pitch + 2u * (uint32_t)(c0 + c)
                       : kOOB;
    }
    // Rows of A of step t (and the next, C::SPAN of them), and of Q, to a stage; zeros
    // past the range.  A buffer ends with a whole chunk of its last row (a dword that
    // reaches past the end would be dropped, with its first element): rows have them.
    auto fetch_a = [&](uint32_t stage, int t) {
        const int zt = z0 + kTileStep * t;
        const int left = (int)uniform(max(z1 - zt, 0));
        rsrc_t ra;
        uint32_t off = a_off;
        if constexpr (TURNED) {
            const uint32_t n = (uint32_t)min(left, kTileStep);
            ra = make_rsrc(A + (size_t)zt * g.a_stride + r0,
                           n ? (n - 1) * a_pitch + 2u * ((a_rows + 7) & ~7u) : 0u);
        } else {
            // (From column zt on: the last row ends with the range.)
            ra = make_rsrc(A + (size_t)r0 * g.a_stride + zt,
                           left ? (a_rows - 1) * a_pitch + 2u * (((uint32_t)left + 7) & ~7u) : 0u);
            off = a_col < left ? off : kOOB;
        }
#pragma unroll
        for (int i = 0; i < C::A_LOADS; ++i)
            load_chunk_unseen(ra, lds0 + stage + (uint32_t)(i * C::NT + 64 * wave) * 16u,
                              off + (uint32_t)(i * A_NEXT) * a_pitch);
    };
    auto fetch_q = [&](uint32_t stage, int t) {
        const int zt = z0 + kTileStep * t;
        const uint32_t n = uniform(min(max(z1 - zt, 0), kTileStep));
        const rsrc_t rq = make_rsrc(Q + (size_t)zt * g.q_stride, n * q_pitch);
#pragma unroll
        for (int i = 0; i < C::Q_LOADS; ++i) {
            const uint32_t at = (uint32_t)(i * C::NT + 64 * wave) * 16u;
            const uint32_t to = at < C::Q_BYTES ? stage + at : C::SPARE0 + at - C::Q_BYTES;
            load_chunk_unseen(rq, lds0 + to, q_off[i]);
        }
    };

    uint32_t qa[C::FC], aa[C::FR];
#pragma unroll
    for (int i = 0; i < C::FC; ++i)
        qa[i] = turn_lane<Q_PITCH>(wc * C::FC + i);
#pragma unroll
    for (int j = 0; j < C::FR; ++j)
        aa[j] = TURNED ? turn_lane<A_PITCH>(wr * C::FR + j) : 0;
    uint32_t rows[2 * C::SPAN]; // of A as it lies: this lane's place in steps of 16
#pragma unroll
    for (int ks = 0; ks < 2 * C::SPAN; ++ks)
        rows[ks] = (uint32_t)((wr * C::FR * 32 + (lane & 31)) * A_PITCH +
                              16 * ((2 * ks + (lane >> 5)) ^ ((lane >> 1) & 7)));
    v16f_t acc[C::FC][C::FR];
#pragma unroll
    for (int i = 0; i < C::FC; ++i)
#pragma unroll
        for (int j = 0; j < C::FR; ++j)
            acc[i][j] = v16f_t{};
    const bool sums = TURNED && g.dbias && tc == 0;
    float bias[C::FR] = {};

    struct Operands {
        u32x4 a[C::FR], b[C::FC];
    } f[2];
    // Half ks of a step: of Q's stage, and of A's from its part `half` on.
    auto read = [&](uint32_t a_stage, int half, uint32_t q_stage, int ks, Operands &o) {
#pragma unroll
        for (int i = 0; i < C::FC; ++i)
            o.b[i] = turned<Q_PITCH>(sm + q_stage, qa[i], ks);
#pragma unroll
        for (int j = 0; j < C::FR; ++j) {
            if constexpr (TURNED)
                o.a[j] = turned<A_PITCH>(sm + a_stage, aa[j], ks);
            else
                o.a[j] = *reinterpret_cast<const u32x4 *>(sm + a_stage + rows[2 * half + ks] +
                                                          j * 32 * A_PITCH);
        }
    };
    auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int i = 0; i < C::FC; ++i)
#pragma unroll
            for (int j = 0; j < C::FR; ++j)
                acc[i][j] = mfma_grad(T{}, o.b[i], o.a[j], acc[i][j]);
    };
    // Reads and products in turn.
    auto in_turn = [&] {
        constexpr int PRODUCTS = C::FC * C::FR, READS = 2 * C::FC + (TURNED ? 2 : 1) * C::FR;
        constexpr int EACH = (READS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);          // a product
            if (i * EACH < READS)
                __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);   // LDS reads
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    if (steps > 0) {
        // (Steps past the last are fetched as zeros, so that the loop and its counts
        // are the same each time.)
        constexpr int PAIRS = C::NA - 1;        // stages of A that are filled at first
#pragma unroll
        for (int t = 0; t < C::NS - 1 || t < PAIRS * C::SPAN; ++t) {
            if (t % C::SPAN == 0 && t / C::SPAN < PAIRS)
                fetch_a((uint32_t)(t / C::SPAN * C::A_BYTES), t);
            if (t < C::NS - 1)
                fetch_q((uint32_t)(C::Q0 + t * C::Q_BYTES), t);
        }
        pers::wait_vm_lgkm0<0>();
        pers::barrier();
        // Stages of step t, and those that its requests go to: step t - 1's, which every
        // wave had read before the last barrier.
        uint32_t sa = 0, qs = C::Q0;
        uint32_t next_a = PAIRS * C::A_BYTES, next_q = C::Q0 + (C::NS - 1) * C::Q_BYTES;
        read(sa, 0, qs, 0, f[0]);
        auto step = [&](auto part, int t) {
            constexpr int half = decltype(part)::value;         // of A's stage
            constexpr bool last = half == C::SPAN - 1;
            if constexpr (half == 0)
                fetch_a(next_a, t + PAIRS * C::SPAN);
            fetch_q(next_q, t + C::NS - 1);
            if constexpr (TURNED) {
                // (The waves that read the same rows of A take the steps of 16 in
                // turn.)
#pragma unroll
                for (int ks = 0; ks < 2; ++ks) {
                    if (!sums || (2 * t + ks) % C::WC != wc)
                        continue;
#pragma unroll
                    for (int j = 0; j < C::FR; ++j) {
                        const u32x4 u = turned<A_PITCH>(sm + sa, aa[j], ks);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f32x2 v = unpack2<T>(u[k]);
                            bias[j] += v.x + v.y;
                        }
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            read(sa, half, qs, 1, f[1]);
            multiply(f[0]);
            in_turn();
            // Step t + 1's rows have landed, and this wave has read all of step t.
            pers::wait_vm_lgkm0<C::ahead(half)>();
            pers::barrier();
            next_q = qs;
            qs = qs == C::Q0 + (C::NS - 1) * C::Q_BYTES ? C::Q0 : qs + C::Q_BYTES;
            if constexpr (last) {
                next_a = sa;
                sa = sa == (C::NA - 1) * C::A_BYTES ? 0 : sa + C::A_BYTES;
            }
            read(sa, last ? 0 : half + 1, qs, 0, f[0]);
            multiply(f[1]);
            in_turn();
        };
        for (int t = 0; t < steps; t += C::SPAN) {
            step(std::integral_constant<int, 0>{}, t);
            if constexpr (C::SPAN == 2)
                step(std::integral_constant<int, 1>{}, t + 1);
        }
        pers::wait_vm_lgkm0<0>();
    }
    pers::barrier();            // the stages are free
    if (TURNED && sums)
        store_row_sums<C, C::WC>(bias, wr, wc, r0, g.R, g.dbias + (size_t)split * g.R, sm);
    const int row0 = r0 + wr * C::FR * 32, col0 = c0 + wc * C::FC * 32;
    const float back = g.back ? *g.back : 1.0f;
    auto scaled = [&](int, int, float (&v)[4]) {
        if constexpr (__is_same(T, f16_t)) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] *= back;
        }
    };
    if (g.splits > 1)
        store_tile<float>(g.part + (size_t)split * g.R * g.C, g.R, g.C, row0, col0,
                          sm + wave * kOutBytes<float, C::FC>, acc, scaled);
    else
        store_tile<T>(static_cast<T *>(g.out), g.R, g.C, row0, col0,
                      sm + wave * kOutBytes<T, C::FC>, acc, scaled);
}

template <class T, class C>
__global__ void __launch_bounds__(C::NT) k_grad_gemm(GradGemm g, int first)
{
    constexpr int OUT = C::WC * C::WR * kOutBytes<float, C::FC>;
    __shared__ __attribute__((aligned(1024))) char sm[C::LDS > OUT ? C::LDS : OUT];
    const int unit = first + xcd_remap(blockIdx.x, gridDim.x);
    const int tiles = g.tiles_r * g.tiles_c, split = unit / tiles;
    int tr, tc;
    tile_coords(unit - split * tiles, g.tiles_r, g.tiles_c, tr, tc);
    grad_gemm_tile<T, C>(g, (int)uniform(tr), (int)uniform(tc), (int)uniform(split), sm);
}

// Writes codes times their rows' factors as rows of T, and copies rows of T, into rows
// of whole 16-byte chunks (zeros past the width).
template <class T> __global__ void __launch_bounds__(256) k_grad_values(GradValues v)
{
    __shared__ float part[4];
    const int job = blockIdx.y;
    const GradValues::Job &j = v.job[job];
    const int chunks = (j.width + 7) / 8;
    const size_t n = (size_t)j.rows * chunks;
    int shift = 0;
    if constexpr (__is_same(T, f16_t)) {
        if (j.q) {
            shift = range_exponent<256>(j.s, 0, j.rows, part);
            if (blockIdx.x == 0 && threadIdx.x == 0)
                *j.back = ldexpf(1.0f, -shift);
        }
    }
    for (size_t at = (size_t)blockIdx.x * 256 + threadIdx.x; at < n; at += (size_t)gridDim.x * 256) {
        const int row = (int)(at / chunks), c = 8 * (int)(at - (size_t)row * chunks);
        u32x4 o = {0, 0, 0, 0};
        if (j.q) {
            const int8_t *p = j.q + (size_t)row * j.width + c;
            u32x2 w = {0, 0};
            if (c + 8 <= j.width) {
                const Packed<int8_t, 8> e = *reinterpret_cast<const Packed<int8_t, 8> *>(p);
                w = u32x2{e.w[0], e.w[1]};
            } else {
                uint64_t u = 0;
                for (int e = 0; e < j.width - c; ++e)
                    u |= (uint64_t)(uint8_t)p[e] << (8 * e);
                w = u32x2{(uint32_t)u, (uint32_t)(u >> 32)};
            }
            const float s = __is_same(T, f16_t) ? ldexpf(j.s[row], shift) : j.s[row];
            // (Zeros past the width, also where the factor is not finite.)
            o = dequantize<T>(u32x2{w.x & j.mask, w.y & j.mask}, s);
            if (c + 8 > j.width) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e >= j.width)
                        o[e / 2] &= e % 2 ? 0x0000ffffu : 0xffff0000u;
            }
        } else {
            const T *p = static_cast<const T *>(j.from) + (size_t)row * j.from_stride + c;
            if (c + 8 <= j.width) {
                o = __builtin_bit_cast(u32x4, *reinterpret_cast<const Packed<T, 8> *>(p));
            } else {
                T e[8] = {};
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (c + k < j.width)
                        e[k] = p[k];
                o = __builtin_bit_cast(u32x4, e);
            }
        }
        *reinterpret_cast<u32x4 *>(static_cast<T *>(j.to) + (size_t)row * j.to_stride + c) = o;
    }
}

template <class T> hipError_t write_values(const GradValues &v, hipStream_t stream)
{
    size_t most = 0;
    for (int i = 0; i < v.n; ++i) {
        const size_t n = (size_t)v.job[i].rows * ((v.job[i].width + 7) / 8);
        most = n > most ? n : most;
    }
    const size_t blocks = (most + 255) / 256;
    k_grad_values<T><<<dim3((unsigned)(blocks < 2048 ? blocks : 2048), v.n), 256, 0, stream>>>(v);
    return hipGetLastError();
}

template <class T, class C> hipError_t launch_gemm(const GradGemm &g, hipStream_t stream)
{
    constexpr long long MOST = 1 << 22;
    const long long units = (long long)g.tiles_r * g.tiles_c * g.splits;
    for (long long u = 0; u < units; u += MOST) {
        const unsigned grid = (unsigned)(units - u < MOST ? units - u : MOST);
        k_grad_gemm<T, C><<<grid, C::NT, 0, stream>>>(g, (int)u);
        if (hipError_t e = hipGetLastError())
            return e;
    }
    return hipSuccess;
}

template <class T, bool TURNED> hipError_t launch_gemm_tile(const GradGemm &g, hipStream_t stream)
{
    if (g.tile_c == 256)
        return launch_gemm<T, TileCfg<256, 256, 4, 2, TURNED ? 5 : 4, 3, TURNED>>(g, stream);
    return launch_gemm<T, TileCfg<192, 256, 2, 4, TURNED ? 5 : 4, 3, TURNED>>(g, stream);
}

template <class T> hipError_t run_gemm(GradGemm g, bool turned_a, hipStream_t stream)
{
    const GradParts p = {g.part, g.out, (size_t)g.R * g.C, g.splits,
                         g.dbias ? g.bias_part : nullptr, g.dbias, g.R};
    if (g.splits > 1 && g.dbias)
        g.dbias = g.bias_part;
    const hipError_t e = turned_a ? launch_gemm_tile<T, true>(g, stream)
                                  : launch_gemm_tile<T, false>(g, stream);
    return e != hipSuccess || g.splits == 1 ? e : join_parts<T>(&p, 1, stream);
}

}  // namespace

}  // namespace tasq
