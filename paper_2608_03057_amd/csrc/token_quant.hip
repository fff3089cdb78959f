// Symmetric 8-bit activation codes with one scale per token:
//
//   s[m] = max_k |x[m][k]| * RN(1 / 127),   Q[m][k] = round(x[m][k] / s[m]),
//
// decided in IEEE single precision (one product; a correctly rounded division,
// then ties to even); a token of zeros has s = 0 and codes 0.  The maximum keeps
// NaN, so that a token that is not finite has a scale that is not.
//
// One read of x: a row stays in the registers of the threads that loaded it
// between its maximum and its codes, a wave to a row up to 2048 elements, which
// needs no barrier, and a workgroup above.  Bound by memory where there are several
// rounds of rows: 8192x4608 bfloat16 21.1 us a call, 5.4 TB/s of activations and codes.
// 8192 rows of 1152 are one wave for each place on the GPU, a chain of load, maximum,
// division and store with nothing behind it: bfloat16 9.5 us a call (10.4 to 11.6
// traced alone), 3.0 TB/s, fp32 9.8, 4.8 TB/s.
#include "block_internal.h"
#include "floats.h"
#include "quant.h"

namespace tasq {

namespace {

// Scale of a row and its codes' divisor.
struct TokenScale {
    float s;
    Divider div;
    __device__ __forceinline__ explicit TokenScale(float top)
        : s(__fmul_rn(top, 1.0f / 127.0f)), div(s)
    {
    }
    // The code as a whole number.  (EXACT: the common case of Divider, decided
    // once for a row.)
    template <bool EXACT> __device__ __forceinline__ float code(float x) const
    {
        const float q = EXACT ? div(x) : s == 0.0f ? 0.0f : __fdiv_rn(x, s);
        return __builtin_amdgcn_fmed3f(__builtin_rintf(q), -127.0f, 127.0f);
    }
    // Eight codes.
    __device__ __forceinline__ uint2 codes(const float (&v)[8]) const
    {
        float q[8];
        if (div.exact) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                q[e] = code<true>(v[e]) + 128.0f;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                q[e] = code<false>(v[e]) + 128.0f;
        }
        return make_uint2(pack_codes(q[0], q[1], q[2], q[3]), pack_codes(q[4], q[5], q[6], q[7]));
    }
};

// The larger, or NaN if either is (fmaxf would take the other).
__device__ __forceinline__ float larger(float a, float b)
{
    return __builtin_elementwise_maximum(a, b);
}

// Maximum over the TPR threads of a row (TPR 64: a wave; 256: a workgroup).
template <int TPR> __device__ __forceinline__ float row_max(float v)
{
    v = group_reduce<64>(v, larger);
    if constexpr (TPR > 64) {
        __shared__ float part[TPR / 64];
        if ((threadIdx.x & 63) == 0)
            part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < TPR / 64; ++w)
            v = larger(v, part[w]);
    }
    return v;
}

// Rows of up to 8 * NV * TPR elements at any alignment and stride; the last K % 8
// elements of a row are one thread's, one by one.  (8192x1151 bfloat16 11.0 us a
// call; 15.8 with a read for the maximum and one for the codes, element by element.)
template <class T, int TPR, int NV>
__global__ void __launch_bounds__(256) k_quantize_tokens(const T *__restrict__ x, int M, int K,
                                                         long long stride,
                                                         int8_t *__restrict__ q,
                                                         float *__restrict__ sx)
{
    const int m = blockIdx.x * (256 / TPR) + threadIdx.x / TPR;
    if (m >= M)
        return;                 // whole waves (TPR 64) or nobody (TPR 256)
    const int t = threadIdx.x % TPR;
    const T *row = x + (size_t)m * stride;
    int8_t *out = q + (size_t)m * K;
    float v[NV][8];
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int k = 8 * (t + i * TPR);
        if (k + 8 <= K) {
            reinterpret_cast<const Packed<T, 8> *>(row + k)->floats(v[i]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[i][e] = k + e < K ? (float)row[k + e] : 0.0f;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            top = larger(top, fabsf(v[i][e]));
    const TokenScale ts(row_max<TPR>(top));
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int k = 8 * (t + i * TPR);
        if (k >= K)
            continue;
        const uint2 c = ts.codes(v[i]);
        if (k + 8 <= K) {
            *reinterpret_cast<Packed<int8_t, 8> *>(out + k) = {c.x, c.y};
        } else {
            for (int e = 0; e < K - k; ++e)
                out[k + e] = (int8_t)((e < 4 ? c.x : c.y) >> (8 * (e & 3)));
        }
    }
    if (t == 0)
        sx[m] = ts.s;
}

// Longer rows, read twice (the second time from L2), element by element: 2048x20000
// bfloat16 67 us a call, 1.8 TB/s.
template <class T>
__global__ void __launch_bounds__(256) k_quantize_tokens_any(const T *__restrict__ x, int K,
                                                             long long stride,
                                                             int8_t *__restrict__ q,
                                                             float *__restrict__ sx)
{
    const int m = blockIdx.x;
    const T *row = x + (size_t)m * stride;
    float top = 0.0f;
    for (int k = threadIdx.x; k < K; k += 256)
        top = larger(top, fabsf((float)row[k]));
    const TokenScale ts(row_max<256>(top));
    for (int k = threadIdx.x; k < K; k += 256)
        q[(size_t)m * K + k] = (int8_t)(int)ts.code<false>((float)row[k]);
    if (threadIdx.x == 0)
        sx[m] = ts.s;
}

template <class T, int TPR, int NV>
hipError_t launch_rows(const T *x, int M, int K, long long stride, int8_t *q, float *sx,
                       hipStream_t stream)
{
    const int rows = 256 / TPR;
    k_quantize_tokens<T, TPR, NV><<<(M + rows - 1) / rows, 256, 0, stream>>>(x, M, K, stride, q,
                                                                           sx);
    return hipGetLastError();
}

template <class T>
hipError_t launch_typed(const T *x, int M, int K, long long stride, int8_t *q, float *sx,
                        hipStream_t stream)
{
    if (K > 256 * 8 * 8) {
        k_quantize_tokens_any<T><<<M, 256, 0, stream>>>(x, K, stride, q, sx);
        return hipGetLastError();
    }
    if (K <= 64 * 8)
        return launch_rows<T, 64, 1>(x, M, K, stride, q, sx, stream);
    if (K <= 64 * 8 * 2)
        return launch_rows<T, 64, 2>(x, M, K, stride, q, sx, stream);
    if (K <= 64 * 8 * 3)
        return launch_rows<T, 64, 3>(x, M, K, stride, q, sx, stream);
    if (K <= 64 * 8 * 4)
        return launch_rows<T, 64, 4>(x, M, K, stride, q, sx, stream);
    if (K <= 256 * 8 * 2)
        return launch_rows<T, 256, 2>(x, M, K, stride, q, sx, stream);
    if (K <= 256 * 8 * 4)
        return launch_rows<T, 256, 4>(x, M, K, stride, q, sx, stream);
    return launch_rows<T, 256, 8>(x, M, K, stride, q, sx, stream);
}

}  // namespace

hipError_t launch_quantize_tokens(const void *x, int type, int M, int K, long long stride,
                                  int8_t *q, float *sx, hipStream_t stream)
{
    // A launch has fewer than 2^32 threads: 2^22 rows of up to 256 threads each.
    constexpr int ROWS = 1 << 22;
    return with_type(type, [&](auto zero) {
        using T = decltype(zero);
        for (int m = 0; m < M; m += ROWS) {
            const hipError_t e =
                launch_typed<T>(static_cast<const T *>(x) + (size_t)m * stride,
                                M - m < ROWS ? M - m : ROWS, K, stride, q + (size_t)m * K, sx + m,
                                stream);
            if (e != hipSuccess)
                return e;
        }
        return hipSuccess;
    });
}

}  // namespace tasq
