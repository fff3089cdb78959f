// What the tiled products around a block's linears share: loads to LDS, and the way of
// 32x32 accumulators to rows of 16-byte stores.
#pragma once

#include "floats.h"
#include "rows.h"

namespace tasq {

typedef float v16f_t __attribute__((ext_vector_type(16)));

// A value that is the same in all lanes, in a scalar register.
__device__ __forceinline__ uint32_t uniform(int v)
{
    return (uint32_t)__builtin_amdgcn_readfirstlane(v);
}

// Lane l's 16 bytes at `off` of the buffer to lds + 16 l; zeros out of bounds.
__device__ __forceinline__ void load_chunk_to_lds(rsrc_t r, char *lds, uint32_t off)
{
#ifdef __HIP_DEVICE_COMPILE__       // the host pass knows no 16-byte form
    typedef __attribute__((address_space(3))) void lds_t;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t *)lds, 16, off, 0, 0, 0);
#endif
}

// The same, not known to the compiler as a write to LDS, for which it would wait
// before every transposing load: the caller waits (vmcnt) before the barrier that hands
// the bytes on.  lds, an offset in LDS, is the same in all lanes.  (m0 cannot be named
// as overwritten: a kernel uses this form or the one above, not both.)
__device__ __forceinline__ void load_chunk_unseen(rsrc_t r, uint32_t lds, uint32_t off)
{
#ifdef __HIP_DEVICE_COMPILE__
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(uniform((int)lds)), "v"(off), "s"(r)
                 : "memory");
#endif
}

// Where in LDS p is.
__device__ __forceinline__ uint32_t lds_offset(const char *p)
{
#ifdef __HIP_DEVICE_COMPILE__
    typedef __attribute__((address_space(3))) const char lds_t;
    return (uint32_t)(uintptr_t)(lds_t *)p;
#else
    return 0;
#endif
}

// Between the lanes of a wave that write LDS and those that read it: the hardware
// keeps the order, and with this the compiler does too.
__device__ __forceinline__ void between_lanes()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Bytes of LDS that a wave with FC blocks of 32 columns needs for store_tile.
template <class T, int FC> constexpr int kOutBytes = 32 * (FC * 32 * (int)sizeof(T) + 16);

// Stores a wave's FC x FR blocks as rows row0.. and columns col0.. of y [rows][cols]:
// register v of block [i][j] in lane l is column 32 i + 8 (v / 4) + 4 (l / 32) + v % 4 of
// row 32 j + l % 32, so that a lane has four neighbours of a row, which cross LDS
// together (rows padded by 16 bytes); then a lane stores 16 bytes of a row.  f(i, q, v)
// changes the four values of columns 32 i + 8 q + 4 (l / 32) on.
template <class T, int FC, int FR, class F>
__device__ __forceinline__ void store_tile(T *y, int rows, int cols, int row0, int col0, char *lds,
                                           const v16f_t (&acc)[FC][FR], F f)
{
    constexpr int PITCH = FC * 32 * (int)sizeof(T) + 16;
    constexpr int PER = 16 / (int)sizeof(T), CH = FC * 32 / PER;    // chunks of a row
    const int lane = threadIdx.x & 63;
    const bool wide = cols % PER == 0 && (reinterpret_cast<uintptr_t>(y) & 15) == 0;
#pragma unroll
    for (int j = 0; j < FR; ++j) {
#pragma unroll
        for (int i = 0; i < FC; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float v[4];
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = acc[i][j][4 * q + e];
                f(i, q, v);
                store_vec<T, 4>(reinterpret_cast<T *>(lds + (lane & 31) * PITCH) + 32 * i + 8 * q +
                                    4 * (lane >> 5),
                                v);
            }
        between_lanes();
#pragma unroll
        for (int e = 0; e < CH / 2; ++e) {
            const int r = (64 * e + lane) / CH, c = (64 * e + lane) % CH;
            const int m = row0 + 32 * j + r, n = col0 + PER * c;
            const u32x4 u = *reinterpret_cast<const u32x4 *>(lds + r * PITCH + 16 * c);
            if (m >= rows || n >= cols)
                continue;
            T *to = y + (size_t)m * cols + n;
            if (wide) {
                *reinterpret_cast<u32x4 *>(to) = u;
            } else if (n + PER <= cols) {       // at any address
                *reinterpret_cast<Packed<T, PER> *>(to) = __builtin_bit_cast(Packed<T, PER>, u);
            } else {
                T one[PER];
                __builtin_memcpy(one, &u, 16);
#pragma unroll
                for (int k = 0; k < PER; ++k)
                    if (n + k < cols)
                        to[k] = one[k];
            }
        }
        between_lanes();
    }
}

}  // namespace tasq
