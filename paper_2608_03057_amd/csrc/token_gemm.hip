// Masked int8 linear with one activation scale per token and one weight scale
// per channel:
//
//   y[m][n] = (sum_k X[m][k] W_b[n][k]) * sx[m] * sw[n] (+ bias[n]),
//
// W_b = W & keep_mask(b), the sum exact in int32, y fp32, bfloat16 or half,
// rounded once.  The K loop is that of gemm_core.h; the epilogue is its own:
// a factor per row, and 16-bit outputs that cross LDS so that a lane stores 16
// bytes of a row.
#include "block_internal.h"
#include "floats.h"
#include "gemm_core.h"

namespace tasq {

namespace {

// Rows of the staged output are padded by 16 bytes, so that the 32 rows that
// an accumulator register spans do not meet in one bank.
template <class C> constexpr int kOutPitch = C::WTN * 2 + 16;

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
            __builtin_amdgcn_wave_barrier();
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
            __builtin_amdgcn_wave_barrier();
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

template <class C, class T> hipError_t launch_cfg(const TokenLinear &t, hipStream_t stream)
{
    const int tm = (t.M + C::BM - 1) / C::BM, tn = (t.N + C::BN - 1) / C::BN;
    const long long grid = (long long)tm * tn;
    if (grid > 0x7fffffffLL)
        return hipErrorInvalidValue;
    const bool aligned = t.K % 16 == 0 && reinterpret_cast<uintptr_t>(t.X) % 16 == 0 &&
                         reinterpret_cast<uintptr_t>(t.W) % 16 == 0 &&
                         (long long)t.M * t.K < (1LL << 31) && (long long)t.N * t.K < (1LL << 31);
    if (aligned)
        k_token_gemm<C, true, T><<<(unsigned)grid, C::NT, 0, stream>>>(t, tm, tn);
    else
        k_token_gemm<C, false, T><<<(unsigned)grid, C::NT, 0, stream>>>(t, tm, tn);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_linear_tokens(const TokenLinear &t, hipStream_t stream)
{
    return with_type(t.type, [&](auto zero) {
        using T = decltype(zero);
        const long long big = ((t.M + 127LL) / 128) * ((t.N + 127LL) / 128);
        if (big >= 256)
            return launch_cfg<Cfg<128, 128, 128, 2, 2, 2>, T>(t, stream);
        return launch_cfg<Cfg<64, 64, 128, 2, 2, 2>, T>(t, stream);
    });
}

}  // namespace tasq
