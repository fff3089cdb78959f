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
#include "branch_internal.h"
#include "floats.h"
#include "gemm_core.h"
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
    // The four scales of row r, step t, that lane half h meets, one a byte: blocks
    // 2 i + h of the step's eight.
    __device__ __forceinline__ uint2 request(int r, int t) const
    {
        const uint32_t at = 8u * (uint32_t)t, o = (uint32_t)r * scale_pitch + at;
        uint2 u;
        u.x = __builtin_amdgcn_raw_buffer_load_b32(scales, at < scale_pitch ? o : kOOB, 0, 0);
        u.y = __builtin_amdgcn_raw_buffer_load_b32(scales, at + 4 < scale_pitch ? o + 4 : kOOB, 0,
                                                   0);
        return u;
    }
};

__device__ __forceinline__ uint32_t half_scales(uint2 u)
{
    const uint32_t h = (threadIdx.x & 63) >> 5;
    return __builtin_amdgcn_perm(u.y, u.x, 0x06040200u + h * 0x01010101u);
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
    uint2 sw[C::FN], sx[C::FM];
    auto scales = [&](int t) {
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
            sw[i] = W.request((wn * C::FN + i) * 32 + r32, t);
#pragma unroll
        for (int j = 0; j < C::FM; ++j)
            sx[j] = X.request((wm * C::FM + j) * 32 + r32, t);
    };
    const int steps = (a.K128 + 1) / 2;
    stage(0);
    scales(0);
    for (int t = 0; t < steps; ++t) {
        uint32_t cw[C::FN], cx[C::FM];
#pragma unroll
        for (int i = 0; i < C::FN; ++i)
            cw[i] = half_scales(sw[i]);
#pragma unroll
        for (int j = 0; j < C::FM; ++j)
            cx[j] = half_scales(sx[j]);
        __builtin_amdgcn_s_waitcnt(0x0f70);         // vmcnt(0): the stage has landed
        __syncthreads();
        if (t + 1 < steps) {
            stage(t + 1);
            scales(t + 1);
        }
        const char *at = sm + (t & 1) * C::STAGE;
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
                    acc[i][j] = mfma_mx4<ks>(w[i], x[j], acc[i][j], cw[i], cx[j]);
        };
        step(std::integral_constant<int, 0>{});
        step(std::integral_constant<int, 1>{});
        step(std::integral_constant<int, 2>{});
        step(std::integral_constant<int, 3>{});
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

// Few tokens: the weight is read once, by workgroups of 16 channels whose four waves
// have every fourth 128 elements each, straight from memory as matrix operands (lane
// l: channel l % 16, block l / 16 of the four), against the tokens' codes read alike;
// the waves' sums meet in LDS.
constexpr int kMx4Few = 64;

template <class T, int MB> __global__ void __launch_bounds__(256) k_mx4_few(Mx4Linear a)
{
    constexpr int UNROLL = MB <= 2 ? 4 : 2;
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

}  // namespace

hipError_t launch_mx4_linear(const Mx4Linear &a, hipStream_t stream)
{
    return with_type(a.type, [&](auto zero) {
        using T = decltype(zero);
        // (16 channels to a workgroup: from 2^28 on they are more than a launch takes.)
        if (a.M <= kMx4Few && a.N < (1 << 28)) {
            const unsigned grid = (unsigned)((a.N + 15LL) / 16);
            if (a.M <= 16)
                k_mx4_few<T, 1><<<grid, 256, 0, stream>>>(a);
            else if (a.M <= 32)
                k_mx4_few<T, 2><<<grid, 256, 0, stream>>>(a);
            else
                k_mx4_few<T, 4><<<grid, 256, 0, stream>>>(a);
            return hipGetLastError();
        }
        const long long t128 = ((a.M + 127LL) / 128) * ((a.N + 127LL) / 128);
        const long long t256 = ((a.M + 255LL) / 256) * ((a.N + 255LL) / 256);
        if (t256 >= 140)
            return launch_tiles<Mx4Cfg<256, 256, 4, 2>, T>(a, stream);
        if (t128 >= 140)
            return launch_tiles<Mx4Cfg<128, 128, 2, 2>, T>(a, stream);
        return launch_tiles<Mx4Cfg<64, 64, 2, 2>, T>(a, stream);
    });
}

}  // namespace tasq
