// Masked int8 linear with one activation scale per token and one weight scale
// per channel:
//
//   y[m][n] = (sum_k X[m][k] W_b[n][k]) * sx[m] * sw[n] (+ bias[n]),
//
// W_b = W & keep_mask(b), the sum exact in int32, y fp32, bfloat16 or half,
// rounded once.  The K loops are those of gemm_core.h and gemm_pers.h; the
// epilogue is their own: a factor per row, and 16-bit outputs that cross LDS so
// that a lane stores 16 bytes of a row.  8192x1152 -> 3456 to bfloat16 40 us, 1.62
// POP/s, 4096x2240 -> 6720 to fp32 76, 1.63: bound by the K loop and by the last
// round of tiles, whose stores nothing hides.
#include "block_internal.h"
#include "floats.h"
#include "gemm_pers.h"

namespace tasq {

namespace {

// Rows of the staged output are padded by 16 bytes, so that the 32 rows that
// an accumulator register spans do not meet in one bank.
template <class C> constexpr int kOutPitch = C::WTN * 2 + 16;

// Between the lanes of a wave that write LDS and those that read it: the hardware
// keeps the order, and with this the compiler does too.
__device__ __forceinline__ void wave_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Applies the factors and stores one wave's sub-tile.  Register v of a 32x32
// accumulator in lane l is row 8*(v/4) + 4*(l/32) + v%4, column l%32.
template <class C, class T>
__device__ __forceinline__ void token_epilogue(const TokenLinear &t, int m0, int n0,
                                               const v16i (&acc)[C::FM][C::FN], char *lds,
                                               const float *rows)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
    const int mw = m0 + wm * C::WTM, nw = n0 + wn * C::WTN;
    float scale[C::FN], bias[C::FN];
#pragma unroll
    for (int j = 0; j < C::FN; ++j) {
        const int n = nw + 32 * j + (lane & 31);
        scale[j] = n < t.N ? t.sw[n] : 0.0f;
        bias[j] = n < t.N && t.bias ? t.bias[n] : 0.0f;
    }
    T *y = static_cast<T *>(t.y);
    char *out = lds + wave * 32 * kOutPitch<C>;
#pragma unroll
    for (int i = 0; i < C::FM; ++i) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int r0 = 8 * q + 4 * (lane >> 5);
            const float4 f =
                *reinterpret_cast<const float4 *>(rows + wm * C::WTM + 32 * i + r0);
            const float rs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
            for (int j = 0; j < C::FN; ++j) {
                const int n = nw + 32 * j + (lane & 31);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float val =
                        (float)acc[i][j][4 * q + v] * (rs[v] * scale[j]) + bias[j];
                    if constexpr (sizeof(T) == 4) {
                        const int m = mw + 32 * i + r0 + v;
                        if (m < t.M && n < t.N)
                            y[(size_t)m * t.N + n] = val;
                    } else {
                        *reinterpret_cast<T *>(out + (r0 + v) * kOutPitch<C> +
                                               2 * (32 * j + (lane & 31))) = (T)val;
                    }
                }
            }
        }
        if constexpr (sizeof(T) == 2) {
            wave_fence();
            constexpr int CH = C::WTN / 8;          // 16-byte chunks per row
            const bool wide = t.N % 8 == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0;
            for (int e = lane; e < 32 * CH; e += 64) {
                const int r = e / CH, c = e % CH;
                const int m = mw + 32 * i + r, n = nw + 8 * c;
                const char *p = out + r * kOutPitch<C> + 16 * c;
                if (m >= t.M || n >= t.N)
                    continue;
                if (wide) {
                    *reinterpret_cast<u32x4 *>(y + (size_t)m * t.N + n) =
                        *reinterpret_cast<const u32x4 *>(p);
                } else {
                    for (int k = 0; k < 8 && n + k < t.N; ++k)
                        y[(size_t)m * t.N + n + k] = reinterpret_cast<const T *>(p)[k];
                }
            }
            wave_fence();
        }
    }
}

template <class C, bool ALIGNED, class T>
__global__ void __launch_bounds__(C::NT, C::OCC) k_token_gemm(TokenLinear t, int tiles_m,
                                                              int tiles_n)
{
    constexpr int OUT = C::WAVES_M * C::WAVES_N * 32 * kOutPitch<C> / 16;
    constexpr int SMA = C::NSTAGE * C::BM * C::CPR, SMB = C::NSTAGE * C::BN * C::CPR;
    __shared__ v4i sm[SMA + SMB > OUT ? SMA + SMB : OUT];
    __shared__ float rows[C::BM];
    LayerDesc d{};
    d.X = t.X;
    d.W = t.W;
    d.M = t.M;
    d.N = t.N;
    d.K = t.K;
    d.bits = t.bits;
    int tm, tn;
    tile_coords(xcd_remap(blockIdx.x, gridDim.x), tiles_m, tiles_n, tm, tn);
    const int m0 = tm * C::BM, n0 = tn * C::BN;
    for (int r = threadIdx.x; r < C::BM; r += C::NT)
        rows[r] = m0 + r < t.M ? t.sx[m0 + r] : 0.0f;
    v16i acc[C::FM][C::FN];
    mainloop<C, ALIGNED, KIND_LINEAR, false>(d, keep_mask_dword(t.bits), m0, n0, 0, t.K,
                                             (t.K + C::BK - 1) / C::BK, acc, sm, sm + SMA,
                                             [] {});
    __syncthreads();            // rows is there, and the K loop's LDS is free
    token_epilogue<C, T>(t, m0, n0, acc, reinterpret_cast<char *>(sm), rows);
}

// The persistent walk of gemm_pers.h with a token epilogue.
struct TokenLayer : LayerDesc {
    const float *rows;          // [M] token scales
    void *out;                  // [M][N] of T, below 2 GiB; 16-bit rows 16-byte aligned
};

template <class C, class T> struct TokenEpilogue {
    float scale[C::FN], bias[C::FN], row;

    __device__ __forceinline__ void request(const TokenLayer &d, int m0, int n0, int)
    {
        const int lane = threadIdx.x & 63, wn = (threadIdx.x >> 6) % C::WAVES_N;
        const rsrc_t rsw = make_rsrc(d.sw, (uint32_t)d.N * 4u);
        const rsrc_t rb = make_rsrc(d.bias, d.bias ? (uint32_t)d.N * 4u : 0u);
        const rsrc_t rr = make_rsrc(d.rows, (uint32_t)d.M * 4u);
#pragma unroll
        for (int j = 0; j < C::FN; ++j) {
            const uint32_t on = 4u * (uint32_t)(n0 + wn * C::WTN + j * 32 + (lane & 31));
            scale[j] =
                __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rsw, on, 0, 0));
            bias[j] =
                __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rb, on, 0, 0));
        }
        const uint32_t om = threadIdx.x < C::BM ? 4u * (uint32_t)(m0 + (int)threadIdx.x) : kOOB;
        row = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rr, om, 0, 0));
    }

    __device__ __forceinline__ void write(const TokenLayer &d, int m0, int n0,
                                          const v16i (&acc)[C::FM][C::FN], char *smB) const
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const int wm = wave / C::WAVES_N, wn = wave % C::WAVES_N;
        float *rows = reinterpret_cast<float *>(smB);
        char *out = smB + 4 * C::BM + wave * 32 * kOutPitch<C>;
        pers::wait_lgkm0();
        pers::barrier();
        if (threadIdx.x < C::BM)
            rows[threadIdx.x] = row;
        pers::wait_lgkm0();
        pers::barrier();
        constexpr uint32_t ES = sizeof(T);
        const rsrc_t ry = make_rsrc(d.out, (uint32_t)d.M * (uint32_t)d.N * ES);
        const int mw = m0 + wm * C::WTM, nw = n0 + wn * C::WTN;
#pragma unroll
        for (int i = 0; i < C::FM; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r0 = 8 * q + 4 * (lane >> 5);
                const float4 f =
                    *reinterpret_cast<const float4 *>(rows + wm * C::WTM + 32 * i + r0);
                const float rs[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
                for (int j = 0; j < C::FN; ++j) {
                    const int n = nw + 32 * j + (lane & 31);
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const float val =
                            (float)acc[i][j][4 * q + v] * (rs[v] * scale[j]) + bias[j];
                        if constexpr (ES == 4) {
                            // Rows past M fall past the buffer's end.
                            const int m = mw + 32 * i + r0 + v;
                            st32(ry,
                                 n < d.N ? ((uint32_t)m * (uint32_t)d.N + (uint32_t)n) * 4u : kOOB,
                                 __float_as_uint(val));
                        } else {
                            *reinterpret_cast<T *>(out + (r0 + v) * kOutPitch<C> +
                                                   2 * (32 * j + (lane & 31))) = (T)val;
                        }
                    }
                }
            }
            if constexpr (ES == 2) {
                constexpr int CH = C::WTN / 8;
                wave_fence();
#pragma unroll
                for (int e = 0; e < CH / 2; ++e) {
                    const int r = (64 * e + lane) / CH, c = lane % CH;
                    const int m = mw + 32 * i + r, n = nw + 8 * c;
                    const u32x4 u = *reinterpret_cast<const u32x4 *>(out + r * kOutPitch<C> + 16 * c);
                    __builtin_amdgcn_raw_buffer_store_b128(
                        u, ry, n < d.N ? ((uint32_t)m * (uint32_t)d.N + (uint32_t)n) * 2u : kOOB,
                        0, 0);
                }
                wave_fence();
            }
        }
        pers::wait_lgkm0();
        pers::barrier();
    }
};

template <class C, class T>
__global__ void __launch_bounds__(C::NT, C::OCC) k_token_gemm_walk(TokenLayer d, XcdRuns runs)
{
    __shared__ __attribute__((aligned(1024))) char sm[PersOperands<C>::LDS];
    persistent_ds<C, TokenEpilogue<C, T>>(OneLayerOf<TokenLayer>{d}, RunWalk(runs, 1), sm);
}

template <class C, class T> hipError_t launch_walk(const TokenLinear &t, hipStream_t stream)
{
    TokenLayer d{};
    d.X = t.X;
    d.W = t.W;
    d.sw = t.sw;
    d.bias = t.bias;
    d.rows = t.sx;
    d.out = t.y;
    d.M = t.M;
    d.N = t.N;
    d.K = t.K;
    d.bits = t.bits;
    fill_tiles<C>(d);
    const long long tiles = (long long)d.tiles_m * d.tiles_n;
    XcdRuns runs;
    for (int x = 0; x <= 8; ++x)
        runs.begin[x] = (int)(tiles * x / 8);
    k_token_gemm_walk<C, T><<<256, C::NT, 0, stream>>>(d, runs);
    return hipGetLastError();
}

template <class C, class T>
hipError_t launch_cfg(const TokenLinear &t, bool aligned, hipStream_t stream)
{
    const int tm = (t.M + C::BM - 1) / C::BM, tn = (t.N + C::BN - 1) / C::BN;
    const long long grid = (long long)tm * tn;
    if (grid > 0x7fffffffLL)
        return hipErrorInvalidValue;
    if (aligned)
        k_token_gemm<C, true, T><<<(unsigned)grid, C::NT, 0, stream>>>(t, tm, tn);
    else
        k_token_gemm<C, false, T><<<(unsigned)grid, C::NT, 0, stream>>>(t, tm, tn);
    return hipGetLastError();
}

// Few tokens: the weight is read once, by workgroups of 16 channels whose four
// waves have every fourth 64 bytes of K each, straight from memory as matrix
// operands (lane l: channel l%16, bytes 16 (l/16) .. of the 64), against the
// tokens' codes read alike; the waves' int32 sums meet in LDS.  Bound by the
// latency of one round of loads and the launch: 1x1152 -> 3456 (4 MB) 3.7 us,
// 16x4608 -> 1152 7.2 (13.7 with 64x64 tiles), 64x1152 -> 3456 6.2 (5.8).
// Off the alignment of 16 bytes (a row's length is enough for that) each load is
// several, and the tokens' are repeated by every workgroup: up to eight tokens,
// 1x5538 -> 4090 12.7 a call and 24.4 with 64x64 tiles, 8x2315 -> 4436 11.4 and 12.7,
// 16x1151 -> 3456 8.8 and 7.6.
constexpr int kFewTokens = 64, kFewTokensAnywhere = 8;

// Sixteen codes of a row of K >= 16 from byte k on, zeros past its end, at any
// alignment.
__device__ __forceinline__ v4i row_chunk(const int8_t *row, int k, int K, bool live)
{
    const int at = k + 16 <= K ? k : K - 16, s = 8 * (k - at);
    const Packed<int8_t, 16> c = *reinterpret_cast<const Packed<int8_t, 16> *>(row + at);
    uint64_t lo = c.w[0] | (uint64_t)c.w[1] << 32, hi = c.w[2] | (uint64_t)c.w[3] << 32;
    if (s) {
        lo = s >= 128 ? 0 : s >= 64 ? hi >> (s - 64) : lo >> s | hi << (64 - s);
        hi = s >= 64 ? 0 : hi >> s;
    }
    lo = live ? lo : 0;
    hi = live ? hi : 0;
    return {(int)lo, (int)(lo >> 32), (int)hi, (int)(hi >> 32)};
}

template <class T, int MB, bool ALIGNED>
__global__ void __launch_bounds__(256) k_token_few(TokenLinear t)
{
    constexpr int UNROLL = MB <= 2 ? 8 : 4;
    typedef int v4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int n0 = blockIdx.x * 16, r = lane & 15, kb = 16 * (lane >> 4);
    const int mask = (int)keep_mask_dword(t.bits);
    v4 acc[MB] = {};
    auto multiply = [&](v4i w, const v4i (&x)[MB]) {
        const v4i wm = {w.x & mask, w.y & mask, w.z & mask, w.w & mask};
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
            acc[mb] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wm, x[mb], acc[mb], 0, 0, 0);
    };
    if constexpr (ALIGNED) {
        const rsrc_t rw = make_rsrc(t.W, (uint32_t)t.N * (uint32_t)t.K);
        const rsrc_t rx = make_rsrc(t.X, (uint32_t)t.M * (uint32_t)t.K);
        const uint32_t ow = n0 + r < t.N ? (uint32_t)(n0 + r) * (uint32_t)t.K : kOOB;
        uint32_t ox[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
            ox[mb] = 16 * mb + r < t.M ? (uint32_t)(16 * mb + r) * (uint32_t)t.K : kOOB;
        for (int k0 = 64 * wave; k0 < t.K; k0 += 256 * UNROLL) {
            v4i w[UNROLL], x[UNROLL][MB];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int k = k0 + 256 * u + kb;
                const bool in = k < t.K;            // K % 16 == 0: whole chunks
                w[u] = ld16(rw, in ? ow + (uint32_t)k : kOOB);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    x[u][mb] = ld16(rx, in ? ox[mb] + (uint32_t)k : kOOB);
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
                multiply(w[u], x[u]);
        }
    } else {
        // Rows past the end are read as the last ones and not used.
        const int8_t *pw = t.W + (size_t)min(n0 + r, t.N - 1) * t.K;
        const int8_t *px[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
            px[mb] = t.X + (size_t)min(16 * mb + r, t.M - 1) * t.K;
        const int whole = t.K / 64;                 // steps of 64
        int step = wave;
        for (; step + 4 * (UNROLL - 1) < whole; step += 4 * UNROLL) {
            v4i w[UNROLL], x[UNROLL][MB];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const int k = 64 * (step + 4 * u) + kb;
                w[u] = row_chunk(pw, k, 0x7fffffff, true);
#pragma unroll
                for (int mb = 0; mb < MB; ++mb)
                    x[u][mb] = row_chunk(px[mb], k, 0x7fffffff, true);
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
                multiply(w[u], x[u]);
        }
        for (; 64 * step < t.K; step += 4) {
            const int k = 64 * step + kb;
            v4i x[MB];
            const v4i w = row_chunk(pw, k, t.K, k < t.K);
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
                x[mb] = row_chunk(px[mb], k, t.K, k < t.K);
            multiply(w, x);
        }
    }
    // Register v of lane l: channel 4 (l/16) + v, token l%16.
    __shared__ v4 part[4][MB][64];
#pragma unroll
    for (int mb = 0; mb < MB; ++mb)
        part[wave][mb][lane] = acc[mb];
    __syncthreads();
    for (int mb = wave; mb < MB; mb += 4) {
        const int m = 16 * mb + r;
        if (m >= t.M)
            continue;
        const v4 s = part[0][mb][lane] + part[1][mb][lane] + part[2][mb][lane] + part[3][mb][lane];
        const float sx = t.sx[m];
        T *y = static_cast<T *>(t.y) + (size_t)m * t.N;
#pragma unroll
        for (int v = 0; v < 4; ++v) {
            const int n = n0 + 4 * (lane >> 4) + v;
            if (n < t.N)
                y[n] = (T)((float)s[v] * (sx * t.sw[n]) + (t.bias ? t.bias[n] : 0.0f));
        }
    }
}

template <class T> hipError_t launch_few(const TokenLinear &t, bool aligned, hipStream_t stream)
{
    const unsigned grid = (unsigned)((t.N + 15) / 16);
    if (!aligned)
        k_token_few<T, 1, false><<<grid, 256, 0, stream>>>(t);
    else if (t.M <= 16)
        k_token_few<T, 1, true><<<grid, 256, 0, stream>>>(t);
    else if (t.M <= 32)
        k_token_few<T, 2, true><<<grid, 256, 0, stream>>>(t);
    else
        k_token_few<T, 4, true><<<grid, 256, 0, stream>>>(t);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_tokens(const TokenLinear &t, hipStream_t stream)
{
    const bool aligned = t.K % 16 == 0 && reinterpret_cast<uintptr_t>(t.X) % 16 == 0 &&
                         reinterpret_cast<uintptr_t>(t.W) % 16 == 0 &&
                         (long long)t.M * t.K < (1LL << 31) && (long long)t.N * t.K < (1LL << 31);
    return with_type(t.type, [&](auto zero) {
        using T = decltype(zero);
        // (16 channels to a workgroup: from 2^28 on they are more than a launch takes.)
        if (t.M <= (aligned ? kFewTokens : kFewTokensAnywhere) && (aligned || t.K >= 16) &&
            t.N < (1 << 28))
            return launch_few<T>(t, aligned, stream);
        // Tiles of 64x64 where larger ones would leave compute units idle, else
        // 128x128, and from about half a tile per compute unit on 256x256, as a
        // persistent walk where the operands allow it.  us, 64x64 / 128x128 /
        // walk, bfloat16 out: 300x1152 -> 3456 7.5 / 9.9 / 17.0, 1024x1280 -> 3840
        // 13.5 / 12.2 / 19.3, 8192x1152 -> 1152 (160 tiles of 256x256) 22.5 / 23.1 /
        // 20.9, 4096x640 -> 5120 (320) 30.5 / 25.9 / 26.6, 8192x1152 -> 3456 (448)
        // 61.5 / 49.0 / 39.7; 4096x2240 -> 6720 fp32 131 / 108 / 74.  (fp32 out leaves
        // 128x128 slowly: 1024x1152 -> 4608 17.9 / 21.6 / 16.9.)
        const long long t128 = ((t.M + 127LL) / 128) * ((t.N + 127LL) / 128);
        const long long t256 = ((t.M + 255LL) / 256) * ((t.N + 255LL) / 256);
        if (t256 >= 140) {
            const bool rows = sizeof(T) == 4 ||
                              (t.N % 8 == 0 && reinterpret_cast<uintptr_t>(t.y) % 16 == 0);
            // The walk's stores take 32-bit byte offsets: those of the last tile's
            // rows past M have to fall past the output's end as well and not come
            // round to its start, as those of 66 rows of 4,300,000 in fp32 would.
            const long long row = (long long)t.N * (int)sizeof(T);
            const bool fits = t.M * row < (1LL << 31) &&
                              (t.M + 255LL) / 256 * 256 * row <= (1LL << 32);
            if (aligned && rows && fits && t.K > 0)
                return launch_walk<Cfg<256, 256, 128, 2, 4, 1>, T>(t, stream);
            // (8192x1151 -> 3456 56 us, 69 with 128x128.)
            return launch_cfg<Cfg<256, 256, 128, 2, 4, 1>, T>(t, aligned, stream);
        }
        if (t128 >= 200)
            return launch_cfg<Cfg<128, 128, 128, 2, 2, 2>, T>(t, aligned, stream);
        return launch_cfg<Cfg<64, 64, 128, 2, 2, 2, 4>, T>(t, aligned, stream);
    });
}

}  // namespace tasq
