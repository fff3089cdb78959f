// Linear on 4-bit microscaled codes (mx4_quant.hip) of activations and weight:
//
//   y[m][n] = sum_blocks 2^(ex + ew) sum_32 x w (+ bias[n]),
//
// products of codes exact, sums fp32 in the matrix unit, y rounded once.  A lane's
// operand of the scaled matrix instruction is 32 elements of a row, 16 bytes, with
// one scale byte of four in a register: a block of the format.
//
// The weight's rows are the first operand, so that a lane's accumulators are four
// neighbouring channels of one token: they cross LDS as whole dwords on their way to
// rows of 16-byte stores.
//
// Bound, where there are many tokens, by what the products wait for: their share of the
// matrix units' time is 0.45 over long sums (8192^3 in 278 us where calls follow for
// long, 296 to 375 in a first dozen, whose clock is still settling), 0.27 for 4096x2240 ->
// 11200 (77 us, 81 by card) and 0.2 for 8192x1152 -> 4608 (41 us), where a tile's results
// take as long as two steps and 2.25 rounds of tiles the time of three.  With few tokens
// it is the launch and one round of loads.
#include "branch_internal.h"
#include "floats.h"
#include "gemm_pers.h"
#include "tile_out.h"

namespace tasq {

namespace {

typedef int v8i_t __attribute__((ext_vector_type(8)));
typedef float v4f_t __attribute__((ext_vector_type(4)));

constexpr int kFp4 = 4;         // the instruction's name for e2m1

__device__ __forceinline__ v8i_t operand(v4i v)
{
    return v8i_t{v.x, v.y, v.z, v.w, 0, 0, 0, 0};
}

template <int STEP>
__device__ __forceinline__ v16f_t mfma_mx4(v4i a, v4i b, v16f_t c, uint32_t sa, uint32_t sb)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(operand(a), operand(b), c, kFp4, kFp4,
                                                           STEP, (int)sa, STEP, (int)sb);
}

// Tiles of BN channels by BM tokens, WN x WM waves of 32x32 blocks.  A step is 256
// elements: 128 bytes of codes a row and eight scales.
template <int BN_, int BM_, int WN_, int WM_> struct Mx4Cfg {
    static constexpr int BN = BN_, BM = BM_, WN = WN_, WM = WM_;
    static constexpr int NT = 64 * WN * WM;
    static constexpr int FN = BN / WN / 32, FM = BM / WM / 32;
    static constexpr int ROWS = BN + BM;            // of a stage
    static constexpr int STAGE = ROWS * 128;
    static constexpr int LOADS = ROWS * 8 / NT;     // 16-byte chunks a thread and stage
    static_assert(ROWS * 8 % NT == 0, "whole loads");
};

// Rows of codes and scales of one operand's tile.
struct Mx4Rows {
    rsrc_t codes, scales;
    uint32_t pitch, scale_pitch;

    __device__ __forceinline__ void init(const uint8_t *c, const uint8_t *s, int rows, int first,
                                         int count, int K128)
    {
        pitch = 64u * (uint32_t)K128;
        scale_pitch = 4u * (uint32_t)K128;
        const uint32_t n = uniform(min(rows - first, count));
        codes = make_rsrc(c + (size_t)first * pitch, n * pitch);
        scales = make_rsrc(s + (size_t)first * scale_pitch, n * scale_pitch);
    }
    // Scales of row r for steps 2 p (lane half 0) and 2 p + 1 (half 1), eight blocks
    // each: one request a row and two steps.  The last four are the next row's, whose
    // blocks are not these, where `whole` is zero.
    __device__ __forceinline__ u32x2 request(int r, int p) const
    {
        const uint32_t at = 16u * (uint32_t)p + 8u * ((threadIdx.x & 63) >> 5);
        return __builtin_bit_cast(
            u32x2, __builtin_amdgcn_raw_buffer_load_b64(
                       scales, at < scale_pitch ? (uint32_t)r * scale_pitch + at : kOOB, 0, 0));
    }
    __device__ __forceinline__ uint32_t whole(int p) const
    {
        const uint32_t at = 16u * (uint32_t)p + 8u * ((threadIdx.x & 63) >> 5);
        return at + 4 < scale_pitch ? ~0u : 0u;
    }
};

// The scales that lane half h meets, one a byte: blocks 2 i + h of the eight of step
// 2 p (s[0]) and of 2 p + 1, from what request() gave.
__device__ __forceinline__ void half_scales(u32x2 u, uint32_t whole, uint32_t (&s)[2])
{
    u.y &= whole;
    const uint32_t sel = 0x06040200u + ((threadIdx.x & 63) >> 5) * 0x01010101u;
    const auto lo = __builtin_amdgcn_permlane32_swap(u.x, u.x, false, false);
    const auto hi = __builtin_amdgcn_permlane32_swap(u.y, u.y, false, false);
    s[0] = __builtin_amdgcn_perm(hi[0], lo[0], sel);
    s[1] = __builtin_amdgcn_perm(hi[1], lo[1], sel);
}

template <class C, class T> __global__ void __launch_bounds__(C::NT) k_mx4_gemm(Mx4Linear a)
{
    constexpr int OUT = C::WN * C::WM * kOutBytes<T, C::FN>;
    __shared__ __attribute__((aligned(1024))) char sm[2 * C::STAGE > OUT ? 2 * C::STAGE : OUT];
    const int lane = threadIdx.x & 63;
    const int wave = (int)uniform(threadIdx.x >> 6);
    const int wn = wave % C::WN, wm = wave / C::WN;
    const int r32 = lane & 31, h = lane >> 5;
    const int tiles_m = (a.M + C::BM - 1) / C::BM, tiles_n = (a.N + C::BN - 1) / C::BN;
    int tm, tn;
    tile_coords(xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, tm, tn);
    const int m0 = (int)uniform(tm * C::BM), n0 = (int)uniform(tn * C::BN);
    Mx4Rows W, X;
    W.init(a.W, a.sw, a.N, n0, C::BN, a.K128);
    X.init(a.X, a.sx, a.M, m0, C::BM, a.K128);
    // Chunk i of this thread: row 8 (i NW + wave) + lane / 8 of the stage, place
    // lane % 8, holding the row's chunk place ^ (row / 2 % 8), so that 16 rows of an
    // operand read fall in distinct banks.
    constexpr int NW = C::NT / 64;
    static_assert(NW % 2 == 0, "rows of a wave differ by multiples of 16");
    const uint32_t chunk = 16u * (uint32_t)((lane & 7) ^ (4 * (wave & 1) + (lane >> 4)));
    auto stage = [&](int t) {
        char *to = sm + (t & 1) * C::STAGE;
        const uint32_t at = 128u * (uint32_t)t + chunk;
#pragma unroll
        for (int i = 0; i < C::LOADS; ++i) {
            const bool w = i < C::BN / (8 * NW);                // known when unrolled
            const int first = 8 * (i * NW + wave);              // of the wave's eight rows
            const uint32_t row = (uint32_t)(first - (w ? 0 : C::BN) + (lane >> 3));
            load_chunk_to_lds(w ? W.codes : X.codes, to + first * 128,
                        at < W.pitch ? row * W.pitch + at : kOOB);
        }
    };
    v16f_t acc[C::FN][C::FM];
#pragma unroll
    for (int i = 0; i < C::FN; ++i)
#pragma unroll
        for (int j = 0; j < C::FM; ++j)
            acc[i][j] = v16f_t{};
    u32x2 sw[C::FN], sx[C::FM];
    uint32_t whole = 0;
    auto scales = [&](int p) {
        whole = W.whole(p);
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
            sw[i] = W.request((wn * C::FN + i) * 32 + r32, p);
#pragma unroll
        for (int j = 0; j < C::FM; ++j)
            sx[j] = X.request((wm * C::FM + j) * 32 + r32, p);
    };
    const int steps = (a.K128 + 1) / 2;
    uint32_t cw[C::FN][2], cx[C::FM][2];
    // Step t, an even one (part 0) or an odd one.
    auto multiply = [&](auto part, int t) {
        constexpr int odd = decltype(part)::value;
        const char *at = sm + odd * C::STAGE;
        auto read = [&](int row, int ks) {
            return *reinterpret_cast<const v4i *>(at + (row + r32) * 128 +
                                                  16 * ((2 * ks + h) ^ ((r32 >> 1) & 7)));
        };
        auto step = [&](auto tag) {
            constexpr int ks = decltype(tag)::value;
            v4i w[C::FN], x[C::FM];
#pragma unroll
            for (int i = 0; i < C::FN; ++i)
                w[i] = read((wn * C::FN + i) * 32, ks);
#pragma unroll
            for (int j = 0; j < C::FM; ++j)
                x[j] = read(C::BN + (wm * C::FM + j) * 32, ks);
#pragma unroll
            for (int i = 0; i < C::FN; ++i)
#pragma unroll
                for (int j = 0; j < C::FM; ++j)
                    acc[i][j] = mfma_mx4<ks>(w[i], x[j], acc[i][j], cw[i][odd], cx[j][odd]);
        };
        // Landed: this step's rows, and in even steps the scales; every wave has read
        // the other stage.
        __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0)
        if constexpr (!odd) {
#pragma unroll
            for (int i = 0; i < C::FN; ++i)
                half_scales(sw[i], whole, cw[i]);
#pragma unroll
            for (int j = 0; j < C::FM; ++j)
                half_scales(sx[j], whole, cx[j]);
        }
        __syncthreads();
        if (t + 1 < steps)
            stage(t + 1);
        if (odd && t + 1 < steps)
            scales((t + 1) / 2);
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
    };
    stage(0);
    scales(0);
    for (int t = 0; t < steps; t += 2) {
        multiply(std::integral_constant<int, 0>{}, t);
        if (t + 1 < steps)
            multiply(std::integral_constant<int, 1>{}, t + 1);
    }
    __syncthreads();            // the stages are free
    const int nw = n0 + wn * C::FN * 32;
    float bias[C::FN][16];
    const rsrc_t rb = make_rsrc(a.bias + n0, a.bias ? 4u * uniform(min(a.N - n0, C::BN)) : 0u);
#pragma unroll
    for (int i = 0; i < C::FN; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                bias[i][4 * q + e] = __builtin_bit_cast(
                    float, __builtin_amdgcn_raw_buffer_load_b32(
                               rb, 4u * (uint32_t)(nw - n0 + 32 * i + 8 * q + 4 * h + e), 0, 0));
    store_tile<T>(static_cast<T *>(a.y), a.M, a.N, m0 + wm * C::FM * 32, nw,
                  sm + wave * kOutBytes<T, C::FN>, acc, [&](int i, int q, float (&v)[4]) {
#pragma unroll
                      for (int e = 0; e < 4; ++e)
                          v[e] += bias[i][4 * q + e];
                  });
}

// One workgroup a compute unit walks the tiles of its XCD's run, two steps' operands
// ahead of its products across tiles: those of a tile's first steps are asked for
// before the stores of the tile before, which nothing waits for but the step after the
// next (one in-order counter covers loads and stores).  Outputs cross 4 KB of LDS a
// wave, whole lines of rows at a time.  (8192x1152 -> 4608 in bfloat16: 41 us, a
// workgroup a tile 45; 4096x2240 -> 11200 into fp32 77 and 88.  In tiles of 128, 45 and
// 107; two workgroups of 128 x 256 a compute unit in steps of half cache lines 47 and
// more, bound by requests to L2.)
template <class C, class T> struct Mx4Walk {
    static constexpr int OUT = 4096;                            // of a wave
    static constexpr int LDS = 2 * C::STAGE + C::NT / 64 * OUT;
    static constexpr int PER = 16 / (int)sizeof(T);             // values of a chunk
    static constexpr int COLS = 128 / (int)sizeof(T);           // of a row in LDS
    static constexpr int BLOCKS = COLS / 32;                    // of 32 channels
    // fp32 outputs leave L2 to the operands (4096x2240 -> 11200 80.5 us, 75.5 so; 16-bit
    // ones, half as many bytes, 41 and 42.5 at 8192x1152 -> 4608).
    static constexpr int STREAM = sizeof(T) == 4 ? 2 : 0;
    static constexpr int STORES = C::FM * (C::FN / BLOCKS) * 4; // of a wave and tile
    static_assert(C::FN % BLOCKS == 0 && STORES < 64, "whole rows; the counter's range");
};

template <class C, class T>
__global__ void __launch_bounds__(C::NT) k_mx4_walk(Mx4Linear a, int tiles_m, int tiles_n)
{
    using Walk = Mx4Walk<C, T>;
    __shared__ __attribute__((aligned(1024))) char sm[Walk::LDS];
    const int lane = threadIdx.x & 63;
    const int wave = (int)uniform(threadIdx.x >> 6);
    const int wn = wave % C::WN, wm = wave / C::WN;
    const int r32 = lane & 31, h = lane >> 5;
    // An eighth of the tiles to each XCD, every (workgroups of an XCD)-th to each of
    // its workgroups.
    const int tiles = tiles_m * tiles_n, x = blockIdx.x % 8, wgs = gridDim.x / 8;
    const int end = (int)((long long)tiles * (x + 1) / 8);
    int u = (int)((long long)tiles * x / 8) + blockIdx.x / 8;
    if (u >= end)
        return;
    const int steps = (a.K128 + 1) / 2;
    auto place = [&](int unit, int &m0, int &n0) {
        int tm, tn;
        tile_coords(unit, tiles_m, tiles_n, tm, tn);
        m0 = (int)uniform(tm * C::BM);
        n0 = (int)uniform(tn * C::BN);
    };

    // What is asked for next: step k of tile `ahead` (past the last tile, nothing).
    Mx4Rows W, X;
    int ahead = u, k = 0, am, an;
    auto aim = [&] {
        place(ahead < end ? ahead : u, am, an);
        const bool live = ahead < end;
        W.init(a.W, a.sw, live ? a.N : 0, live ? an : 0, C::BN, a.K128);
        X.init(a.X, a.sx, live ? a.M : 0, live ? am : 0, C::BM, a.K128);
    };
    aim();
    constexpr int NW = C::NT / 64;
    const uint32_t chunk = 16u * (uint32_t)((lane & 7) ^ (4 * (wave & 1) + (lane >> 4)));
    const uint32_t lds0 = lds_offset(sm);
    // Load i of step k's rows to a stage; the scales of operand i of step k and the next.
    uint32_t base = 0;          // this lane's place in the first rows of step k
    auto aim_rows = [&] {
        const uint32_t at = 128u * (uint32_t)k + chunk;
        uint32_t row = (uint32_t)(8 * wave + (lane >> 3));
        asm volatile("" : "+v"(row));
        base = at < W.pitch ? row * W.pitch + at : kOOB;
    };
    auto load = [&](uint32_t stage, int i) {
        const bool w = i < C::BN / (8 * NW);                // known when unrolled
        const int rows = 8 * NW * (w ? i : i - C::BN / (8 * NW));
        load_chunk_unseen(w ? W.codes : X.codes, lds0 + stage + (uint32_t)(i * NW + wave) * 1024u,
                          base + (uint32_t)rows * W.pitch);
    };
    auto advance = [&] {
        if (++k == steps) {
            k = 0;
            ahead += wgs;
            aim();
        }
    };
    constexpr int OPERANDS = C::FN + C::FM;
    u32x2 raw[OPERANDS];
    uint32_t whole = 0;
    auto ask_scales = [&](int i, int p) {
        raw[i] = i < C::FN ? W.request((wn * C::FN + i) * 32 + r32, p)
                           : X.request((wm * C::FM + i - C::FN) * 32 + r32, p);
    };
    // Scales of the step at work, and of the next one: of an even step, or of the odd
    // one after it.
    uint32_t now[OPERANDS], next[OPERANDS];
    auto take_scales = [&](int i, bool odd) {
        uint32_t s[2];
        half_scales(raw[i], whole, s);
        next[i] = odd ? s[1] : s[0];
    };
    // The bias of channel `lane` of this wave's, of the tile at n.
    static_assert(C::FN == 2, "a lane to a channel of the wave");
    auto ask_bias = [&](int n) {
        const rsrc_t rb = make_rsrc(a.bias + n, a.bias ? 4u * uniform(min(a.N - n, C::BN)) : 0u);
        return __builtin_amdgcn_raw_buffer_load_b32(rb, 4u * (uint32_t)(wn * 64 + lane), 0, 0);
    };
    struct Operands {
        v4i w[C::FN], x[C::FM];
    } f[2];
    v16f_t acc[C::FN][C::FM];
    constexpr int PRODUCTS = C::FN * C::FM;
    // Part ks of a step, with work(i) beside product i.
    auto multiply = [&](auto tag, const Operands &o, auto work) {
        constexpr int ks = decltype(tag)::value;
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
#pragma unroll
            for (int j = 0; j < C::FM; ++j) {
                acc[i][j] = mfma_mx4<ks>(o.w[i], o.x[j], acc[i][j], now[i], now[C::FN + j]);
                // (Here, and not behind all that is read in the step.)
                asm volatile("" : "+v"(acc[i][j]));
                work(i * C::FM + j);
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    // LDS read i of part ks: the operands in the order in which products take them.
    const uint32_t place0 = (uint32_t)(r32 * 128 + 16 * (h ^ ((r32 >> 1) & 7)));
    auto read = [&](uint32_t stage, int ks, int i, Operands &o) {
        uint32_t at = place0;           // (formed here, not kept for each ks)
        asm volatile("" : "+v"(at));
        const char *p = sm + stage + (at ^ (uint32_t)(32 * ks));
        if (i == 0 || i > C::FM)
            o.w[i ? i - C::FM : 0] = *reinterpret_cast<const v4i *>(
                p + (wn * C::FN + (i ? i - C::FM : 0)) * 32 * 128);
        else
            o.x[i - 1] =
                *reinterpret_cast<const v4i *>(p + (C::BN + (wm * C::FM + i - 1) * 32) * 128);
    };
    auto reads = [&](uint32_t stage, int ks, Operands &o) {
        return [&, stage, ks](int i) {
            if (i < OPERANDS)
                read(stage, ks, i, o);
        };
    };
    constexpr std::integral_constant<int, 0> K0{};
    constexpr std::integral_constant<int, 1> K1{};
    constexpr std::integral_constant<int, 2> K2{};
    constexpr std::integral_constant<int, 3> K3{};

    uint32_t st = 0;
    whole = W.whole(0);
#pragma unroll
    for (int i = 0; i < OPERANDS; ++i)
        ask_scales(i, 0);
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        aim_rows();
#pragma unroll
        for (int i = 0; i < C::LOADS; ++i)
            load((uint32_t)(n * C::STAGE), i);
        if (n == 0)
            advance();
    }
    pers::wait_vm_lgkm0<0>();
    pers::barrier();
#pragma unroll
    for (int i = 0; i < OPERANDS; ++i) {
        take_scales(i, false);
        now[i] = next[i];
        read(0, 0, i, f[0]);
    }
    bool stored = false;        // stores were issued since the last wait
    int m0, n0;
    place(u, m0, n0);
    int bias = (int)ask_bias(n0);
    for (; u < end; u += wgs) {
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
#pragma unroll
            for (int j = 0; j < C::FM; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    acc[i][j][v] = 0.0f;
        for (int t = 0; t < steps; ++t) {
            // (k: the next step, whose rows were asked for last; never the second of a
            // tile's, an odd one, where t is 0.)
            const bool even = t > 0 && k % 2 == 0;
            const int pair = k / 2;
            auto read1 = reads(st, 1, f[1]), read2 = reads(st, 2, f[0]), read3 = reads(st, 3, f[1]);
            multiply(K0, f[0], read1);
            multiply(K1, f[1], read2);
            if (even) {
                whole = W.whole(pair);
#pragma unroll
                for (int i = 0; i < OPERANDS; ++i)
                    ask_scales(i, pair);
            }
            multiply(K2, f[0], read3);
            advance();
            aim_rows();
            // The next step's rows and scales have landed, and this wave has read all
            // of this step's.
            if (stored)
                pers::wait_vm_lgkm0<Walk::STORES>();
            else
                pers::wait_vm_lgkm0<0>();
            stored = false;
            pers::barrier();
            const bool odd = t % 2 == 0 && t + 1 < steps;
            multiply(K3, f[1], [&](int i) {
                if (i < OPERANDS) {
                    read(st ^ C::STAGE, 0, i, f[0]);
                    take_scales(i, odd);
                }
                if (i < C::LOADS)
                    load(st, i);
            });
            static_assert(C::LOADS <= PRODUCTS && OPERANDS <= PRODUCTS, "all beside a product");
#pragma unroll
            for (int i = 0; i < OPERANDS; ++i)
                now[i] = next[i];
            st ^= C::STAGE;
        }
        const int m1 = m0, n1 = n0, bias1 = bias;
        if (u + wgs < end)
            place(u + wgs, m0, n0);
        bias = (int)ask_bias(n0);
        // Rows of whole lines through LDS, BLOCKS of 32 channels at a time.
        T *y = static_cast<T *>(a.y) + (size_t)m1 * a.N;
        const uint32_t rows = uniform(min(a.M - m1, C::BM));
        const rsrc_t ry = make_rsrc(y, rows * (uint32_t)a.N * (uint32_t)sizeof(T));
        char *out = sm + 2 * C::STAGE + wave * Walk::OUT;
        // (A lane number of its own, or the compiler forms all addresses before the
        // loop and has no registers left in it.)
        int l = lane;
        asm volatile("" : "+v"(l));
        const int lr = l & 31, lh = l >> 5;
        float add[C::FN][16];
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                add[i][v] = __int_as_float(__builtin_amdgcn_ds_bpermute(
                    4 * (32 * i + 8 * (v / 4) + 4 * lh + v % 4), bias1));
#pragma unroll
        for (int j = 0; j < C::FM; ++j)
#pragma unroll
            for (int i0 = 0; i0 < C::FN; i0 += Walk::BLOCKS) {
#pragma unroll
                for (int i = 0; i < Walk::BLOCKS; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        float v[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[e] = acc[i0 + i][j][4 * q + e] + add[i0 + i][4 * q + e];
                        const int byte = (32 * i + 8 * q + 4 * lh) * (int)sizeof(T);
                        store_vec<T, 4>(reinterpret_cast<T *>(out + lr * 128 +
                                                              ((byte / 16) ^ ((lr >> 1) & 7)) * 16 +
                                                              byte % 16),
                                        v);
                    }
                between_lanes();
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int r = 8 * e + l / 8, c = l % 8;
                    const u32x4 val = *reinterpret_cast<const u32x4 *>(
                        out + r * 128 + 16 * (c ^ ((r >> 1) & 7)));
                    const int n = n1 + (wn * C::FN + i0) * 32 + Walk::PER * c;
                    const uint32_t m = (uint32_t)((wm * C::FM + j) * 32 + r);
                    __builtin_amdgcn_raw_buffer_store_b128(
                        val, ry,
                        n < a.N ? (m * (uint32_t)a.N + (uint32_t)n) * (uint32_t)sizeof(T) : kOOB, 0,
                        Walk::STREAM);
                }
                between_lanes();
                __builtin_amdgcn_sched_barrier(0);
            }
        stored = true;
    }
    pers::wait_vm_lgkm0<0>();
}

// Few tokens: the weight is read once, by workgroups of 16 channels whose four waves
// have every fourth 128 elements each, straight from memory as matrix operands (lane
// l: channel l % 16, block l / 16 of the four), against the tokens' codes read alike;
// the waves' sums meet in LDS.
constexpr int kMx4Few = 32;

template <class T, int MB> __global__ void __launch_bounds__(256) k_mx4_few(Mx4Linear a)
{
    constexpr int UNROLL = 4;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = blockIdx.x * 16, r = lane & 15, kb = lane >> 4;
    Mx4Rows W, X;
    W.init(a.W, a.sw, a.N, n0, 16, a.K128);
    X.init(a.X, a.sx, a.M, 0, a.M, a.K128);
    v4f_t acc[MB] = {};
    const uint32_t ow = n0 + r < a.N ? (uint32_t)r : kOOB;
    for (int s = wave; s < a.K128; s += 4 * UNROLL) {
        v4i w[UNROLL], x[UNROLL][MB];
        uint32_t ws[UNROLL], xs[UNROLL][MB];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int step = s + 4 * u;
            const bool in = step < a.K128;
            const uint32_t k = (uint32_t)(4 * step + kb);           // block
            const bool wi = in && ow != kOOB;
            w[u] = ld16(W.codes, wi ? ow * W.pitch + 16 * k : kOOB);
            ws[u] = __builtin_amdgcn_raw_buffer_load_b8(W.scales,
                                                        wi ? ow * W.scale_pitch + k : kOOB, 0, 0);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                const uint32_t m = (uint32_t)(16 * mb + r);
                const bool xi = in && (int)m < a.M;
                x[u][mb] = ld16(X.codes, xi ? m * X.pitch + 16 * k : kOOB);
                xs[u][mb] = __builtin_amdgcn_raw_buffer_load_b8(
                    X.scales, xi ? m * X.scale_pitch + k : kOOB, 0, 0);
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u)
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                acc[mb] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(
                    operand(w[u]), operand(x[u][mb]), acc[mb], kFp4, kFp4, 0, (int)ws[u], 0,
                    (int)xs[u][mb]);
    }
    // Register v of lane l: channel 4 (l / 16) + v, token l % 16.
    __shared__ v4f_t part[4][MB][64];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
        part[wave][mb][lane] = acc[mb];
    __syncthreads();
    for (int mb = wave; mb < MB; mb += 4) {
        const int m = 16 * mb + r;
        if (m >= a.M)
            continue;
        const v4f_t s = (part[0][mb][lane] + part[1][mb][lane]) +
                        (part[2][mb][lane] + part[3][mb][lane]);
        T *y = static_cast<T *>(a.y) + (size_t)m * a.N;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int n = n0 + 4 * kb + v;
            if (n < a.N)
                y[n] = (T)(s[v] + (a.bias ? a.bias[n] : 0.0f));
        }
    }
}

// Tokens go out in as many launches as keep one below 2^22 tiles.
template <class C, class T> hipError_t launch_tiles(const Mx4Linear &all, hipStream_t stream)
{
    const long long tiles_n = (all.N + (long long)C::BN - 1) / C::BN;
    const long long tiles_m = (all.M + (long long)C::BM - 1) / C::BM;
    const long long most = (1LL << 22) / tiles_n, step = most > 1 ? most : 1;
    for (long long tm = 0; tm < tiles_m; tm += step) {
        const long long n = tiles_m - tm < step ? tiles_m - tm : step, m = tm * C::BM;
        Mx4Linear a = all;
        a.X += (size_t)m * a.K128 * 64;
        a.sx += (size_t)m * a.K128 * 4;
        a.y = static_cast<T *>(a.y) + (size_t)m * a.N;
        a.M = (int)(all.M - m < n * C::BM ? all.M - m : n * C::BM);
        k_mx4_gemm<C, T><<<(unsigned)(n * tiles_n), C::NT, 0, stream>>>(a);
        if (hipError_t e = hipGetLastError())
            return e;
    }
    return hipSuccess;
}

template <class C, class T> hipError_t launch_walk(const Mx4Linear &a, hipStream_t stream)
{
    k_mx4_walk<C, T><<<256, C::NT, 0, stream>>>(a, (a.M + C::BM - 1) / C::BM,
                                                (a.N + C::BN - 1) / C::BN);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_linear(const Mx4Linear &a, hipStream_t stream)
{
    return with_type(a.type, [&](auto zero) {
        using T = decltype(zero);
        // (Few / tiles of 64, us: 1152 -> 3456 of 16 tokens 3.1 / 4.0, 32 3.5 / 4.1, 64 4.2
        // / 4.1; 1152 -> 9000 of 1 3.8 / 3.9, 16 4.4 / 4.1, 32 5.7 / 4.2; 4608 -> 1152 of
        // 32 7.2 / 7.9, 64 10.2 / 8.0.)
        if (a.M <= kMx4Few && (long long)a.M * a.N <= 1 << 17) {
            const unsigned grid = (unsigned)((a.N + 15LL) / 16);
            if (a.M <= 16)
                k_mx4_few<T, 1><<<grid, 256, 0, stream>>>(a);
            else
                k_mx4_few<T, 2><<<grid, 256, 0, stream>>>(a);
            return hipGetLastError();
        }
        const long long t128 = ((a.M + 127LL) / 128) * ((a.N + 127LL) / 128);
        const long long t256 = ((a.M + 255LL) / 256) * ((a.N + 255LL) / 256);
        // Tiles as large as still come to half a round.  (64 / 128 / 256, us, 1152
        // channels in: 2304 x 4096 18.8 / 17.5 / 16.3, 1500 x 3000 11.0 / 10.6 / 14.1,
        // 512 x 2304 6.9 / 7.6 / 12.6.)
        if (t256 >= 140) {
            // The walk stores whole 16-byte chunks at 32-bit offsets within a tile, and
            // takes two steps of 256 elements or more.
            const int per = 16 / (int)sizeof(T);
            if (a.N % per == 0 && reinterpret_cast<uintptr_t>(a.y) % 16 == 0 && a.N < (1 << 21) &&
                t256 < (1 << 30) && a.K128 > 2)
                return launch_walk<Mx4Cfg<256, 256, 4, 2>, T>(a, stream);
            return launch_tiles<Mx4Cfg<256, 256, 4, 2>, T>(a, stream);
        }
        if (t128 >= 140)
            return launch_tiles<Mx4Cfg<128, 128, 2, 2>, T>(a, stream);
        return launch_tiles<Mx4Cfg<64, 64, 2, 2>, T>(a, stream);
    });
}

}  // namespace tasq
