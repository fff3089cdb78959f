// Microscaled 4-bit floating point (the e2m1 elements and e8m0 block scales of the
// OCP Microscaling Formats specification, v1.0, with its conversion):
//
//   e = floor(log2(max_32 |x|)) - 2, at least -127,   scale = 2^e as the byte e + 127,
//   code = e2m1(x 2^-e): 0, .5, 1, 1.5, 2, 3, 4, 6 and a sign, to the nearest, ties to
//   the even code, values beyond 6 to 6,
//
// for every 32 consecutive elements of a row.  A block with a NaN or an infinity has
// the scale NaN (byte 255).  The product with 2^-e is exact (a result that is not is
// below the least code's half), so a code is one decision.
//
// A lane has eight elements, four lanes a block; rows are filled up to a multiple of
// 128 elements with zeros, so that codes and scales of all rows are one run of whole
// dwords.  Bound by memory: x is read once, a quarter of its bytes (bfloat16) written:
// 8192 x 1152 in 6.9 us, 4096 x 2240 of fp32 in 8.5 (24 and 42 MB, short of a copy's
// rate by the first loads' latency).
#include "branch_internal.h"
#include "floats.h"

namespace tasq {

namespace {

__device__ __forceinline__ float larger(float a, float b)
{
    return __builtin_elementwise_maximum(a, b);     // NaN if either is
}

template <class T>
__global__ void __launch_bounds__(256) k_quantize_mx4(const T *__restrict__ x, long long first,
                                                      long long units, int K, int vectors,
                                                      long long stride,
                                                      uint32_t *__restrict__ codes,
                                                      uint8_t *__restrict__ scales)
{
    const long long u = first + (long long)blockIdx.x * 256 + threadIdx.x;
    if (u >= units)
        return;                 // whole blocks
    const long long m = u / vectors;
    const int k = 8 * (int)(u - m * vectors);
    const T *p = x + m * stride + k;
    float v[8];
    if (k + 8 <= K) {
        reinterpret_cast<const Packed<T, 8> *>(p)->floats(v);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            v[e] = k + e < K ? (float)p[e] : 0.0f;
    }
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        top = larger(top, fabsf(v[e]));
    top = group_reduce<4>(top, larger);
    const int exponent = (int)(__float_as_uint(top) >> 23) & 255;
    const bool bad = exponent == 255;
    const int byte = bad ? 255 : max(exponent - 2, 0);
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = bad ? 0.0f : ldexpf(v[e], 127 - byte);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], 1.0f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], 1.0f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], 1.0f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], 1.0f, 3);
    codes[u] = c;
    if (threadIdx.x % 4 == 0)
        scales[u / 4] = (uint8_t)byte;
}

}  // namespace

hipError_t launch_quantize_mx4(const void *x, int type, int M, int K, long long stride,
                               uint8_t *codes, uint8_t *scales, hipStream_t stream)
{
    const int vectors = (K + 127) / 128 * 16;
    const long long units = (long long)M * vectors;
    constexpr long long MOST = 1LL << 30;           // threads of a launch
    return with_type(type, [&](auto zero) {
        using T = decltype(zero);
        for (long long u = 0; u < units; u += MOST) {
            const long long n = units - u < MOST ? units - u : MOST;
            k_quantize_mx4<T><<<(unsigned)((n + 255) / 256), 256, 0, stream>>>(
                static_cast<const T *>(x), u, units, K, vectors, stride,
                reinterpret_cast<uint32_t *>(codes), scales);
            if (hipError_t e = hipGetLastError())
                return e;
        }
        return hipSuccess;
    });
}

}  // namespace tasq
