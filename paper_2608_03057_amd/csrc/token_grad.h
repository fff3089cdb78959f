// Gradient of the token-scaled masked linear, y = (X W_b^T) sx[m] sw[n] + bias[n],
// from the 8-bit codes that the forward pass took:
//
//   dx[m][k] = sum_n dy[m][n] (sw[n] W_b[n][k]),
//   dw[n][k] = sum_m dy[m][n] (sx[m] X[m][k]),     dbias[n] = sum_m dy[m][n].
//
// Both are products of dy (or its transpose) with an 8-bit matrix Q [Z][C] whose rows,
// the summed axis, have a factor each: out[r][c] = sum_z A(r, z) s[z] Q[z][c].  The
// 8-bit operand becomes one of dy's type on its way to LDS, s[z] q rounded once: codes
// are exact in either type, so that this is the one rounding before the fp32 sums of
// the matrix unit.  In half it is kept in the middle of the type's range: the factors
// are divided by a power of two near the largest of a workgroup's and the sums are
// multiplied by it again; a factor below 2^-21 of the largest loses bits, to values that
// are below 2^-24 of the largest's.
//
// Bound by latency: 300 tokens of 640 -> 1288 (1 GFLOP) take 10 us for both products,
// eleven steps of loads, values, LDS and products after one another (1283 13); large products by
// the vector instructions that turn codes into values, of which a wave has 88 beside 32
// products, and which every tile of rows does again (grad_tiles.h).
//
// The matrix instruction takes Q's columns as its first operand, so that a lane has
// four neighbouring columns of an output row (tile_out.h), and eight values of the
// summed axis at a time: rows of dy give them as they lie, rows of Q and of dy's
// transpose through the transposing LDS load (four rows of 16 columns per 16 lanes).
#pragma once

#include "branch_internal.h"
#include "gemm_pers.h"
#include "tile_out.h"

namespace tasq {

namespace {

typedef bf16_t v8bf_t __attribute__((ext_vector_type(8)));
typedef f16_t v8h_t __attribute__((ext_vector_type(8)));
typedef short v4s_t __attribute__((ext_vector_type(4)));

__device__ __forceinline__ v16f_t mfma_grad(bf16_t, u32x4 a, u32x4 b, v16f_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf_t, a),
                                                   __builtin_bit_cast(v8bf_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ v16f_t mfma_grad(f16_t, u32x4 a, u32x4 b, v16f_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h_t, a),
                                                  __builtin_bit_cast(v8h_t, b), c, 0, 0, 0);
}

constexpr int kGradStep = 64;   // of the summed axis

// Tiles of BC columns of Q by BR rows of the output, WC x WR waves; G groups of them
// have a part of the tile's range each, with stages of their own, and add up at its end.
template <int BC_, int BR_, int WC_, int WR_, int G_ = 1> struct GradCfg {
    static constexpr int BC = BC_, BR = BR_, WC = WC_, WR = WR_, G = G_;
    static constexpr int NT = 64 * WC * WR, ALL = G * NT;       // threads of a group, and all
    static constexpr int FC = BC / WC / 32, FR = BR / WR / 32;
    static constexpr int A_BYTES = BR * kGradStep * 2, Q_BYTES = BC * kGradStep * 2;
    // Three stages of A, two of Q.
    static_assert(NT >= BR && 4 % WC == 0, "a thread to a row's sum");
    static constexpr int LDS = 3 * A_BYTES + 2 * Q_BYTES;
    static constexpr int Q_TASKS = kGradStep * BC / 8 / NT;     // 8 codes each
    static constexpr int A_TASKS = kGradStep * BR / 8 / NT;     // 16 bytes each
};

// Place of 16-byte chunk c of row z of a tile with PITCH bytes a row that the
// transposing load reads: the rows that it spans fall in distinct banks.
template <int PITCH> __device__ __forceinline__ int turn_key(int z)
{
    return PITCH % 256 == 0 ? z & 3 : (z >> 1) & 1;
}

template <int PITCH> __device__ __forceinline__ uint32_t turn_place(int z, int c)
{
    return (uint32_t)(z * PITCH + 16 * (c ^ (4 * turn_key<PITCH>(z))));
}

// Eight values z .. z + 7 of column `block * 32 + lane % 32` of such a tile, for lane
// half h rows 8 h on, from `lds` at row 16 ks: `at` is this lane's part of the address
// (turn_lane).
template <int PITCH> __device__ __forceinline__ uint32_t turn_lane(int block)
{
    const int lane = threadIdx.x & 63, z = 8 * (lane >> 5) + ((lane & 15) >> 2);
    const int c = 4 * block + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    return turn_place<PITCH>(z, c) + 8 * (lane & 1);
}

template <int PITCH>
__device__ __forceinline__ u32x4 turned(const char *lds, uint32_t at, int ks)
{
    typedef __attribute__((address_space(3))) v4s_t lds_t;
    const char *p = lds + at + 16 * ks * PITCH;
    static_assert(PITCH % 128 == 0, "rows z and z + 4 have the same key");
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)p));
    const u32x2 hi = __builtin_bit_cast(
        u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p + 4 * PITCH)));
    return u32x4{lo.x, lo.y, hi.x, hi.y};
}

// Eight codes times their row's factor as eight values of T.
template <class T> __device__ __forceinline__ u32x4 dequantize(u32x2 q, float s)
{
    u32x4 o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t w = q[i / 2] >> (16 * (i & 1));
        o[i] = pack2<T>((float)(int8_t)w * s, (float)(int8_t)(w >> 8) * s);
    }
    return o;
}

// The power of two that brings the largest finite factor of [z0, z1) to 2^7: with
// codes of up to 2^7 in magnitude a product stays below 2^15.  NT threads.
template <int NT>
__device__ __forceinline__ int range_exponent(const float *s, int z0, int z1, float *part)
{
    float top = 0.0f;
    for (int z = z0 + (int)threadIdx.x; z < z1; z += 8 * NT) {
        float f[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)     // (on their way together)
            f[i] = fabsf(s[min(z + i * NT, z1 - 1)]);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            top = f[i] < __builtin_inff() ? fmaxf(top, f[i]) : top;
    }
    top = group_reduce<64>(top, [](float a, float b) { return fmaxf(a, b); });
    if ((threadIdx.x & 63) == 0)
        part[threadIdx.x >> 6] = top;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < NT / 64; ++w)
        top = fmaxf(top, part[w]);
    __syncthreads();
    int e = 0;
    if (top > 0.0f)
        (void)frexpf(top, &e);          // top < 2^e
    return 8 - e;
}

// The sums of a tile's rows that its waves hold, a row to the lanes l and l + 32 and to
// N waves, of which this is the n-th, added up in order into out[r0 ..]; LDS is free
// before and after.
template <class C, int N>
__device__ __forceinline__ void store_row_sums(const float (&sum)[C::FR], int wr, int n, int r0,
                                               int R, float *out, char *sm)
{
    const int lane = threadIdx.x & 63;
    float *part = reinterpret_cast<float *>(sm);
#pragma unroll
    for (int j = 0; j < C::FR; ++j) {
        const uint32_t u = __float_as_uint(sum[j]);
        const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        if (lane < 32)
            part[n * C::BR + (wr * C::FR + j) * 32 + lane] =
                __uint_as_float(p[0]) + __uint_as_float(p[1]);
    }
    __syncthreads();
    const int r = (int)threadIdx.x;
    if (r < C::BR && r0 + r < R) {
        float v = part[r];
#pragma unroll
        for (int w = 1; w < N; ++w)
            v += part[w * C::BR + r];
        out[r0 + r] = v;
    }
    __syncthreads();
}

// out[r][c] of one tile and range of the summed axis.  TURNED: A is [Z][R], else
// [R][Z].  WHOLE: rows of both operands are whole 16-byte chunks at 16-byte addresses,
// and those of A go to LDS directly.
template <class T, class C, bool TURNED, bool WHOLE>
__device__ __forceinline__ void grad_tile(const GradJob &g, int tr, int tc, int split, char *all)
{
    constexpr int A_PITCH = TURNED ? 2 * C::BR : 2 * kGradStep;
    constexpr int Q_PITCH = 2 * C::BC;
    const int lane = threadIdx.x & 63;
    const int tid = (int)(threadIdx.x % C::NT), group = (int)uniform(threadIdx.x / C::NT);
    const int wave = (int)uniform(tid >> 6);
    const int wc = wave % C::WC, wr = wave / C::WC;
    const int r0 = tr * C::BR, c0 = tc * C::BC;
    const int first = split * g.split_steps * kGradStep;
    const int end = min(g.Z, first + g.split_steps * kGradStep);
    // A group's part of the range: as many steps for each, so that they meet at barriers.
    const int steps = ((end - first + kGradStep - 1) / kGradStep + C::G - 1) / C::G;
    const int z0 = first + group * steps * kGradStep, z1 = min(end, z0 + steps * kGradStep);
    char *const sm = all + group * C::LDS;
    const T *A = static_cast<const T *>(g.A);
    const int8_t *const q_end = g.Q + (size_t)g.Z * g.C;
    const bool factors = g.C > 0;       // (the rows' sums alone have none to read)
    int shift = 0;
    if constexpr (sizeof(T) == 2 && __is_same(T, f16_t))
        shift = range_exponent<C::ALL>(g.s, first, factors ? end : first,
                                       reinterpret_cast<float *>(all));

    // A step's codes and factors (and A's chunks, where they pass through registers)
    // on their way.
    struct Raw {
        u32x2 q[C::Q_TASKS];
        float s[C::Q_TASKS];
        u32x4 a[WHOLE ? 1 : C::A_TASKS];
    };
    // Offsets in LDS of a step's stage of A, and of Q.
    struct Stage {
        uint32_t a, q;
    };
    const uint32_t lds0 = lds_offset(sm);
    // This thread's first eight codes of a step: row qz, column c0 + qc, in every part.
    // (Neighbouring lanes write neighbouring chunks.)
    constexpr int Q_ROWS = C::NT / (C::BC / 8);     // between a thread's parts
    const int qz = tid / (C::BC / 8), qc = 8 * (tid % (C::BC / 8));
    const uint32_t q_off =
        c0 + qc < g.C ? (uint32_t)qz * (uint32_t)g.C + (uint32_t)(c0 + qc) : kOOB;
    // Where rows that are no whole chunks lie, a chunk reaches past its row: into the
    // next, or, of the last ones, past the operand's end.  The dword across that end is
    // dropped, and its first bytes are loaded one by one.
    const uint32_t a_pitch = 2u * (uint32_t)g.a_stride;
    const T *const a_end = A + (TURNED ? (size_t)(g.Z - 1) * g.a_stride + g.R
                                       : (size_t)(g.R - 1) * g.a_stride + g.Z);
    // Step t's, zeros past the range.
    auto request = [&](Raw &raw, int t) {
        const int zt = z0 + kGradStep * t;
        const uint32_t n = uniform(max(min(z1 - zt, kGradStep), 0));
        const rsrc_t rs = make_rsrc(g.s + zt, factors ? 4u * n : 0u);
        const int8_t *const q0 = g.Q + (size_t)zt * g.C;
        uint32_t bytes = n * (uint32_t)g.C;
        bool cut = false;       // some chunk of this step reaches past Q's end
        if (!WHOLE && n) {
            const long long rest = q_end - q0;
            cut = rest < bytes + 7;
            bytes = cut ? (uint32_t)rest : bytes + 7;
        }
        const rsrc_t rq = make_rsrc(q0, bytes);
#pragma unroll
        for (int i = 0; i < C::Q_TASKS; ++i) {
            raw.s[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(
                                                     rs, 4u * (uint32_t)(qz + i * Q_ROWS), 0, 0));
            raw.q[i] = __builtin_bit_cast(
                u32x2, __builtin_amdgcn_raw_buffer_load_b64(
                           rq, q_off + (uint32_t)(i * Q_ROWS) * (uint32_t)g.C, 0, 0));
        }
        if constexpr (!WHOLE) {
            const T *const a0 =
                A + (TURNED ? (size_t)zt * g.a_stride + r0 : (size_t)r0 * g.a_stride + zt);
            uint32_t a_bytes = 0;
            if (n) {
                const uint32_t rows = TURNED ? n : (uint32_t)min(g.R - r0, C::BR);
                const uint32_t cols = TURNED ? (uint32_t)min(g.R - r0, C::BR) : n;
                const long long want = (long long)(rows - 1) * a_pitch + 2 * cols + 14;
                const long long rest = 2 * (a_end - a0);
                a_bytes = (uint32_t)(rest < want ? rest : want);
            }
            const rsrc_t ra = make_rsrc(a0, uniform(a_bytes));
#pragma unroll
            for (int i = 0; i < C::A_TASKS; ++i) {
                const int task = tid + i * C::NT;
                const int row = task / (A_PITCH / 16), first = 8 * (task % (A_PITCH / 16));
                const bool in = TURNED ? row < (int)n && first < g.R - r0
                                       : r0 + row < g.R && first < (int)n;
                const uint32_t off = (uint32_t)row * a_pitch + 2u * (uint32_t)first;
                raw.a[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(
                                                         ra, in ? off : kOOB, 0, 0));
            }
            // The last dword of either operand.  (Chunks of A reach its end from the last
            // step only, which cuts Q short as well; those of Q, with rows of one code,
            // from the last rows of the step before too.)
            if (cut) {
#pragma unroll
                for (int i = 0; i < C::Q_TASKS; ++i) {
                    const int z = qz + i * Q_ROWS, c = c0 + qc;
                    const int8_t *p = q0 + (size_t)z * g.C + c;
                    const int left = z < (int)n && c < g.C && q_end - p < 8 ? (int)(q_end - p) : 0;
                    uint32_t u = 0;
#pragma unroll 1
                    for (int e = left & ~3; e < left; ++e)
                        u |= (uint32_t)(uint8_t)p[e] << (8 * (e & 3));
                    if (left & 3)
                        raw.q[i] = left < 4 ? u32x2{u, 0} : u32x2{raw.q[i].x, u};
                }
#pragma unroll
                for (int i = 0; i < C::A_TASKS; ++i) {
                    const int task = tid + i * C::NT;
                    const int row = task / (A_PITCH / 16), first = 8 * (task % (A_PITCH / 16));
                    const bool in = TURNED ? row < (int)n && first < g.R - r0
                                           : r0 + row < g.R && first < (int)n;
                    const T *p = a0 + (size_t)row * g.a_stride + first;
                    const int left = in && a_end - p < 8 ? (int)(a_end - p) : 0;
                    if (left & 1) {
                        const uint32_t u = __builtin_bit_cast(uint16_t, p[left - 1]);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            raw.a[i][k] = k == left / 2 ? u : raw.a[i][k];
                    }
                }
            }
        }
    };
    // This lane's first chunk of a step's rows of A: A_ROWS rows an instruction, every
    // A_NEXT-th of a wave's.  Its column is the same in all of them.
    constexpr int CH = A_PITCH / 16, A_ROWS = 64 / CH, A_NEXT = C::NT / 64 * A_ROWS;
    static_assert(TURNED ? A_NEXT % 4 == 0 : A_NEXT % 16 == 0, "one column a lane");
    const int a_row = wave * A_ROWS + lane / CH;
    const int a_col = 8 * (TURNED ? (lane % CH) ^ (4 * turn_key<A_PITCH>(a_row))
                                  : (lane % CH) ^ ((a_row >> 1) & 7));
    const uint32_t a_off = TURNED && a_col >= g.R - r0
                               ? kOOB
                               : (uint32_t)a_row * a_pitch + 2u * (uint32_t)a_col;
    const uint32_t a_last = 2u * uniform(min(g.R - r0, C::BR));
    // Step t's rows of A straight to LDS, zeros past the range.
    auto direct = [&](uint32_t stage, int t) {
        if constexpr (WHOLE) {
            const int zt = z0 + kGradStep * t;
            const int left = (int)uniform(max(z1 - zt, 0));
            rsrc_t rsrc;
            uint32_t off = a_off;
            if constexpr (TURNED) {
                const uint32_t n = (uint32_t)min(left, kGradStep);
                rsrc = make_rsrc(A + (size_t)zt * g.a_stride + r0,
                                 n ? (n - 1) * a_pitch + a_last : 0u);
            } else {
                // (From column zt on: the last row ends with the range.)
                rsrc = make_rsrc(A + (size_t)r0 * g.a_stride + zt,
                                 left ? (a_last / 2 - 1) * a_pitch + 2u * (uint32_t)left : 0u);
                off = a_col < left ? off : kOOB;
            }
#pragma unroll
            for (int i = 0; i < C::A_TASKS; ++i)
                load_chunk_unseen(
                    rsrc, lds0 + stage + (uint32_t)((wave * A_ROWS + i * A_NEXT) * A_PITCH),
                    off + (uint32_t)(i * A_NEXT) * a_pitch);
        }
    };
    // What request() gave, into its stage: Q's parts i0 .. i1 - 1; A's chunks.
    const uint32_t q_to = turn_place<Q_PITCH>(qz, qc / 8);
    static_assert(Q_ROWS % 4 == 0, "rows of a thread have one key");
    auto put = [&](const Raw &raw, Stage st, int i0, int i1) {
        char *to = sm + st.q;
#pragma unroll
        for (int i = 0; i < C::Q_TASKS; ++i) {
            if (i < i0 || i >= i1)
                continue;
            const float s = __is_same(T, f16_t) ? ldexpf(raw.s[i], shift) : raw.s[i];
            *reinterpret_cast<u32x4 *>(to + q_to + i * Q_ROWS * Q_PITCH) =
                dequantize<T>(u32x2{raw.q[i].x & g.mask, raw.q[i].y & g.mask}, s);
        }
    };
    auto put_chunks = [&](Raw &raw, Stage st, int t) {
        if constexpr (!WHOLE) {
            const int n = (int)uniform(z1 - z0 - kGradStep * t);    // rows of step t
            if (!TURNED && n < kGradStep) {     // zeros past the range within a chunk
#pragma unroll
                for (int i = 0; i < C::A_TASKS; ++i) {
                    const int left = n - 8 * ((tid + i * C::NT) % (A_PITCH / 16));
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        raw.a[i][k] &= left >= 2 * k + 2 ? ~0u : left == 2 * k + 1 ? 0xffffu : 0u;
                }
            }
#pragma unroll
            for (int i = 0; i < C::A_TASKS; ++i) {
                const int task = tid + i * C::NT;
                const int row = task / (A_PITCH / 16), c = task % (A_PITCH / 16);
                const uint32_t at = TURNED ? turn_place<A_PITCH>(row, c)
                                           : (uint32_t)(row * A_PITCH + 16 * (c ^ ((row >> 1) & 7)));
                *reinterpret_cast<u32x4 *>(sm + st.a + at) = raw.a[i];
            }
        }
    };

    uint32_t qa[C::FC], aa[C::FR];
#pragma unroll
    for (int i = 0; i < C::FC; ++i)
        qa[i] = turn_lane<Q_PITCH>(wc * C::FC + i);
#pragma unroll
    for (int j = 0; j < C::FR; ++j)
        aa[j] = TURNED ? turn_lane<A_PITCH>(wr * C::FR + j) : 0;
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
    auto read = [&](Stage st, int ks, Operands &o) {
        const char *A = sm + st.a, *Q = sm + st.q;
#pragma unroll
        for (int i = 0; i < C::FC; ++i)
            o.b[i] = turned<Q_PITCH>(Q, qa[i], ks);
#pragma unroll
        for (int j = 0; j < C::FR; ++j) {
            if constexpr (TURNED) {
                o.a[j] = turned<A_PITCH>(A, aa[j], ks);
            } else {
                const int row = (wr * C::FR + j) * 32 + (lane & 31);
                o.a[j] = *reinterpret_cast<const u32x4 *>(
                    A + row * A_PITCH + 16 * ((2 * ks + (lane >> 5)) ^ ((lane >> 1) & 7)));
            }
        }
    };
    auto multiply = [&](const Operands &o) {
#pragma unroll
        for (int i = 0; i < C::FC; ++i)
#pragma unroll
            for (int j = 0; j < C::FR; ++j)
                acc[i][j] = mfma_grad(T{}, o.b[i], o.a[j], acc[i][j]);
    };
    // Reads and products in turn, `valu` vector instructions to a product.
    auto in_turn = [&](auto valu) {
        constexpr int PRODUCTS = C::FC * C::FR, READS = 2 * C::FC + (TURNED ? 2 : 1) * C::FR;
        constexpr int EACH = (READS + PRODUCTS - 1) / PRODUCTS;
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);          // a product
            if (i * EACH < READS)
                __builtin_amdgcn_sched_group_barrier(0x100, EACH, 0);   // LDS reads
            if constexpr (decltype(valu)::value > 0)
                __builtin_amdgcn_sched_group_barrier(0x002, decltype(valu)::value, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> NO_VALU{};
    constexpr int HALF = (C::Q_TASKS + 1) / 2;
    constexpr std::integral_constant<int, (23 * HALF + C::FC * C::FR - 1) / (C::FC * C::FR)>
        PUT_VALU{};
    if (steps > 0) {
        // (Steps past the last are requested and put as zeros, so that the loop is
        // the same each time.)
        constexpr uint32_t Q0 = 3 * C::A_BYTES, A1 = C::A_BYTES, Q1 = C::Q_BYTES;
        Stage st = {0, Q0}, after = {A1, Q0 + Q1};      // of steps t and t + 1
        uint32_t free_a = 2 * A1;                       // of step t + 2
        Raw now, next;
        direct(st.a, 0);
        request(now, 0);
        put(now, st, 0, C::Q_TASKS);
        put_chunks(now, st, 0);
        direct(after.a, 1);
        request(next, 1);
        pers::wait_vm_lgkm0<0>();
        pers::barrier();
        read(st, 0, f[0]);
        for (int t = 0; t < steps; ++t) {
            if (TURNED && sums) {
                // (The WC waves that read the same rows of A take 16 of the step's
                // 64 values each, or 32.)
#pragma unroll
                for (int ks = 0; ks < 4; ks += C::WC)
#pragma unroll
                    for (int j = 0; j < C::FR; ++j) {
                        const u32x4 u = turned<A_PITCH>(sm + st.a, aa[j], ks + wc);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const f32x2 v = unpack2<T>(u[k]);
                            bias[j] += v.x + v.y;
                        }
                    }
            }
            // What the step before requested has landed: Q's rows of step t + 1, which
            // go to their stage now, and A's.  Those of t + 2 are requested: their
            // stage of A was read in step t - 1, before the last barrier.
            read(st, 1, f[1]);
            __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0)
            now = next;
            direct(free_a, t + 2);
            request(next, t + 2);
            put(now, after, 0, HALF);
            multiply(f[0]);
            in_turn(PUT_VALU);
            read(st, 2, f[0]);
            put(now, after, HALF, C::Q_TASKS);
            multiply(f[1]);
            in_turn(PUT_VALU);
            read(st, 3, f[1]);
            put_chunks(now, after, t + 1);
            multiply(f[0]);
            in_turn(NO_VALU);
            // This wave has read all of step t and written its part of t + 1.
            pers::wait_lgkm0();
            pers::barrier();
            const uint32_t done = st.a;
            st = after;
            after = {free_a, 2 * Q0 + Q1 - st.q};
            free_a = done;
            read(st, 0, f[0]);
            multiply(f[1]);
            in_turn(NO_VALU);
        }
        pers::wait_vm_lgkm0<0>();
    }
    pers::barrier();            // the stages are free
    if (TURNED && sums)
        store_row_sums<C, C::G * C::WC>(bias, wr, group * C::WC + wc, r0, g.R,
                                        g.dbias + (size_t)split * g.R, all);
    if constexpr (C::G > 1) {
        // The other groups' sums, behind where the first's results go out.
        constexpr int HELD = C::FC * C::FR * 16, OUT = C::NT / 64 * kOutBytes<float, C::FC>;
        static_assert(OUT + (C::G - 1) * C::NT * HELD * 4 <= C::G * C::LDS, "room in the stages");
        float *const part = reinterpret_cast<float *>(all + OUT);
        if (group > 0) {
#pragma unroll
            for (int v = 0; v < HELD; ++v)
                part[((group - 1) * HELD + v) * C::NT + tid] =
                    acc[v / 16 / C::FR][v / 16 % C::FR][v % 16];
        }
        __syncthreads();
        if (group > 0)
            return;
#pragma unroll
        for (int o = 0; o < C::G - 1; ++o)
#pragma unroll
            for (int v = 0; v < HELD; ++v)
                acc[v / 16 / C::FR][v / 16 % C::FR][v % 16] += part[(o * HELD + v) * C::NT + tid];
    }
    const int row0 = r0 + wr * C::FR * 32, col0 = c0 + wc * C::FC * 32;
    const float back = ldexpf(1.0f, -shift);
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

template <class T, class C, bool TURNED, bool WHOLE>
__global__ void __launch_bounds__(C::NT) k_token_grad(GradJob g, int first)
{
    constexpr int OUT = C::WC * C::WR * kOutBytes<float, C::FC>;
    __shared__ __attribute__((aligned(1024))) char sm[C::LDS > OUT ? C::LDS : OUT];
    const int unit = first + xcd_remap(blockIdx.x, gridDim.x);
    const int tiles = g.tiles_r * g.tiles_c, split = unit / tiles;
    int tr, tc;
    tile_coords(unit - split * tiles, g.tiles_r, g.tiles_c, tr, tc);
    grad_tile<T, C, TURNED, WHOLE>(g, (int)uniform(tr), (int)uniform(tc), (int)uniform(split), sm);
}

// Both products of a small gradient in one launch, from workgroup `from` on: dx's
// `first` workgroups, then dw's.
template <class T, class C, bool WHOLE>
__global__ void __launch_bounds__(C::ALL) k_token_grads(GradJob x, GradJob w, int first, int from)
{
    constexpr int OUT = C::WC * C::WR * kOutBytes<float, C::FC>, STAGES = C::G * C::LDS;
    __shared__ __attribute__((aligned(1024))) char sm[STAGES > OUT ? STAGES : OUT];
    // (Each XCD has its share of both.)
    const int block = from + (int)blockIdx.x, end = from + (int)gridDim.x;
    const bool turned_a = block >= first;
    const int low = turned_a ? max(first, from) : from, high = turned_a ? end : min(first, end);
    const int u = low - (turned_a ? first : 0) + xcd_remap(block - low, high - low);
    const int tiles_r = turned_a ? w.tiles_r : x.tiles_r;
    const int tiles_c = turned_a ? w.tiles_c : x.tiles_c;
    const int tiles = tiles_r * tiles_c, split = u / tiles;
    int tr, tc;
    tile_coords(u - split * tiles, tiles_r, tiles_c, tr, tc);
    tr = (int)uniform(tr);
    tc = (int)uniform(tc);
    if (turned_a)
        grad_tile<T, C, true, WHOLE>(w, tr, tc, (int)uniform(split), sm);
    else
        grad_tile<T, C, false, WHOLE>(x, tr, tc, (int)uniform(split), sm);
}

// Parts of a result that its ranges left, and of the bias'.
struct GradParts {
    const float *part;
    void *out;
    size_t n;
    int splits;
    const float *bias_part;
    float *dbias;
    int bias_n;
};

// Adds the ranges' parts up in order and rounds, of one result or two: four values a
// thread, and after the last of them the bias'.
template <class T>
__global__ void __launch_bounds__(256) k_join_grad(GradParts one, GradParts two)
{
    const GradParts &j = blockIdx.y ? two : one;
    const float *const part = j.part;
    T *const out = static_cast<T *>(j.out);
    const size_t n = j.n;
    const int splits = j.splits;
    const size_t at = 4 * ((size_t)blockIdx.x * 256 + threadIdx.x);
    if (at < n) {
        float v[4] = {};
        const int live = n - at < 4 ? (int)(n - at) : 4;
        if (live == 4) {
            for (int s = 0; s < splits; s += 8) {       // (eight on their way together)
                Packed<float, 4> p[8];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    p[i] = *reinterpret_cast<const Packed<float, 4> *>(
                        part + (size_t)min(s + i, splits - 1) * n + at);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    float f[4];
                    p[i].floats(f);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] += s + i < splits ? f[e] : 0.0f;
                }
            }
            Packed<T, 4> o;
            o.set(v);
            *reinterpret_cast<Packed<T, 4> *>(out + at) = o;
        } else {
            for (int e = 0; e < live; ++e) {
                float f = 0.0f;
                for (int s = 0; s < splits; ++s)
                    f += part[(size_t)s * n + at + e];
                out[at + e] = (T)f;
            }
        }
        return;
    }
    const size_t b = (size_t)blockIdx.x * 256 + threadIdx.x - (n + 3) / 4;
    if (j.bias_part && b < (size_t)j.bias_n) {
        float f = 0.0f;
        for (int s = 0; s < splits; ++s)
            f += j.bias_part[(size_t)s * j.bias_n + b];
        j.dbias[b] = f;
    }
}

template <class T, class C, bool TURNED, bool WHOLE>
hipError_t launch_cfg(const GradJob &g, hipStream_t stream)
{
    constexpr long long MOST = 1 << 22;
    const long long units = (long long)g.tiles_r * g.tiles_c * g.splits;
    for (long long u = 0; u < units; u += MOST) {
        const unsigned grid = (unsigned)(units - u < MOST ? units - u : MOST);
        k_token_grad<T, C, TURNED, WHOLE><<<grid, C::NT, 0, stream>>>(g, (int)u);
        if (hipError_t e = hipGetLastError())
            return e;
    }
    return hipSuccess;
}

// (Tiles of 256 are of whole chunks only: passing rows through registers as well, they
// spill, and are slower than tiles of 128.)
template <class T, bool TURNED>
hipError_t launch_product(const GradJob &g, bool whole, hipStream_t stream)
{
    if (g.tile == 256)
        return whole ? launch_cfg<T, GradCfg<256, 256, 4, 2>, TURNED, true>(g, stream)
                     : hipErrorInvalidValue;
    return whole ? launch_cfg<T, GradCfg<128, 128, 2, 2>, TURNED, true>(g, stream)
                 : launch_cfg<T, GradCfg<128, 128, 2, 2>, TURNED, false>(g, stream);
}

// What is left to add up of a product whose range is cut.
inline GradParts parts_of(const GradJob &g, float *dbias)
{
    return {g.part, g.out, (size_t)g.R * g.C, g.splits, dbias ? g.bias_part : nullptr, dbias, g.R};
}

template <class T> hipError_t join_parts(const GradParts *p, int n, hipStream_t stream)
{
    size_t most = 0;
    for (int i = 0; i < n; ++i) {
        const size_t threads = (p[i].n + 3) / 4 + (p[i].dbias ? p[i].bias_n : 0);
        most = threads > most ? threads : most;
    }
    k_join_grad<T><<<dim3((unsigned)((most + 255) / 256), n), 256, 0, stream>>>(p[0], p[n - 1]);
    return hipGetLastError();
}

// One of the two products, in tiles of 128 or 256, and, where its range is cut, the sum
// of its parts.
template <class T> hipError_t run_product(GradJob g, bool turned_a, bool whole, hipStream_t stream)
{
    const GradParts p = parts_of(g, g.dbias);
    if (g.splits > 1 && g.dbias)
        g.dbias = g.bias_part;
    hipError_t e = turned_a ? launch_product<T, true>(g, whole, stream)
                            : launch_product<T, false>(g, whole, stream);
    return e != hipSuccess || g.splits == 1 ? e : join_parts<T>(&p, 1, stream);
}

// In as many launches as keep one below 2^22 workgroups, as launch_cfg.
template <class T, class C>
hipError_t launch_small(const GradJob &x, const GradJob &w, bool whole, hipStream_t stream)
{
    constexpr long long MOST = 1 << 22;
    const long long first = (long long)x.tiles_r * x.tiles_c * x.splits;
    const long long units = first + (long long)w.tiles_r * w.tiles_c * w.splits;
    for (long long u = 0; u < units; u += MOST) {
        const unsigned grid = (unsigned)(units - u < MOST ? units - u : MOST);
        if (whole)
            k_token_grads<T, C, true><<<grid, C::ALL, 0, stream>>>(x, w, (int)first, (int)u);
        else
            k_token_grads<T, C, false><<<grid, C::ALL, 0, stream>>>(x, w, (int)first, (int)u);
        if (hipError_t e = hipGetLastError())
            return e;
    }
    return hipSuccess;
}

// Products of one tile size of 64 (in 1 or 2 groups) or 128.
template <class T>
hipError_t run_products(const GradJob *px, const GradJob *pw, int groups, bool whole,
                        hipStream_t stream)
{
    GradJob x = px ? *px : GradJob{}, w = pw ? *pw : GradJob{};     // (of no workgroups)
    const int tile = px ? x.tile : w.tile;
    GradParts p[2];
    int n = 0;
    if (x.splits > 1)
        p[n++] = parts_of(x, nullptr);
    if (w.splits > 1) {
        p[n++] = parts_of(w, w.dbias);
        if (w.dbias)
            w.dbias = w.bias_part;
    }
    const hipError_t e =
        tile == 128   ? launch_small<T, GradCfg<128, 128, 2, 2>>(x, w, whole, stream)
        : groups == 2 ? launch_small<T, GradCfg<64, 64, 2, 2, 2>>(x, w, whole, stream)
                      : launch_small<T, GradCfg<64, 64, 2, 2>>(x, w, whole, stream);
    return e != hipSuccess || n == 0 ? e : join_parts<T>(p, n, stream);
}

}  // namespace

}  // namespace tasq
