// The three floating types of activations and their conversions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tasq.h"

namespace tasq {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Pair;
template <> struct Pair<bf16_t> { typedef bf16_t type __attribute__((ext_vector_type(2))); };
template <> struct Pair<f16_t> { typedef f16_t type __attribute__((ext_vector_type(2))); };

// Two floats rounded to nearest even, the first in the low half.
template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b)
{
    const f32x2 v = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, typename Pair<T>::type));
}

template <class T> __device__ __forceinline__ f32x2 unpack2(uint32_t u)
{
    return __builtin_convertvector(__builtin_bit_cast(typename Pair<T>::type, u), f32x2);
}

// N consecutive elements as they lie in memory, at the alignment of one: a load
// or store takes the same instructions as an aligned one.
template <class T, int N> struct __attribute__((packed, aligned(sizeof(T)))) Packed {
    static constexpr int kWords = N * (int)sizeof(T) / 4;
    uint32_t w[kWords];

    __device__ __forceinline__ void floats(float (&v)[N]) const
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4) {
                v[i] = __uint_as_float(w[i]);
            } else {
                const f32x2 f = unpack2<T>(w[i]);
                v[2 * i] = f.x;
                v[2 * i + 1] = f.y;
            }
        }
    }
    __device__ __forceinline__ void set(const float (&v)[N])
    {
#pragma unroll
        for (int i = 0; i < kWords; ++i) {
            if constexpr (sizeof(T) == 4)
                w[i] = __float_as_uint(v[i]);
            else
                w[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
        }
    }
};

// N consecutive elements as floats: N * sizeof(T) bytes in loads of up to 16
// bytes, p aligned to the smaller of 16 and that size.
template <class T, int N> __device__ __forceinline__ void load_vec(const T *p, float (&v)[N])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i) {
                const float4 f = reinterpret_cast<const float4 *>(p)[i];
                v[4 * i] = f.x;
                v[4 * i + 1] = f.y;
                v[4 * i + 2] = f.z;
                v[4 * i + 3] = f.w;
            }
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                v[i] = p[i];
        }
    } else if constexpr (N == 8) {
        const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 f = unpack2<T>(u[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    } else if constexpr (N == 4) {
        const u32x2 u = *reinterpret_cast<const u32x2 *>(p);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const f32x2 f = unpack2<T>(u[i]);
            v[2 * i] = f.x;
            v[2 * i + 1] = f.y;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = (float)p[i];
    }
}

template <class T, int N> __device__ __forceinline__ void store_vec(T *p, const float (&v)[N])
{
    if constexpr (sizeof(T) == 4) {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N / 4; ++i)
                reinterpret_cast<float4 *>(p)[i] =
                    make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                p[i] = v[i];
        }
    } else if constexpr (N == 8) {
        u32x4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            u[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<u32x4 *>(p) = u;
    } else if constexpr (N == 4) {
        u32x2 u;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            u[i] = pack2<T>(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<u32x2 *>(p) = u;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            p[i] = (T)v[i];
    }
}

// v of all N lanes of a group (N a power of two, groups aligned) combined by f,
// in every lane: exchanges within the vector unit, which take a few
// instructions' time where one through LDS takes a hundred cycles.
template <int CTRL> __device__ __forceinline__ float dpp_move(float v)
{
    const int i = (int)__float_as_uint(v);
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(i, i, CTRL, 0xf, 0xf, false));
}

template <int N, class F> __device__ __forceinline__ float group_reduce(float v, F f)
{
    if constexpr (N >= 2)
        v = f(v, dpp_move<0xB1>(v));        // lane ^ 1
    if constexpr (N >= 4)
        v = f(v, dpp_move<0x4E>(v));        // lane ^ 2
    if constexpr (N >= 8)
        v = f(v, dpp_move<0x141>(v));       // mirrored within eight
    if constexpr (N >= 16)
        v = f(v, dpp_move<0x140>(v));       // mirrored within sixteen
    if constexpr (N >= 32) {
        const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v),
                                                        false, false);
        v = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    if constexpr (N >= 64) {
        const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v),
                                                        false, false);
        v = f(__uint_as_float(p[0]), __uint_as_float(p[1]));
    }
    return v;
}

inline int type_bytes(int type) { return type == TASQ_TYPE_F32 ? 4 : 2; }

// f with a value of the type that `type` names.
template <class F> inline hipError_t with_type(int type, F f)
{
    switch (type) {
    case TASQ_TYPE_F32: return f(0.0f);
    case TASQ_TYPE_BF16: return f(bf16_t{});
    default: return f(f16_t{});
    }
}

}  // namespace tasq
