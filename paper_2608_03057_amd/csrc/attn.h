// Softmax attention for gfx950: what the forward and the backward kernels
// share.
//
// A product of two tiles always has its streamed operand (rows staged in LDS)
// as the first matrix operand and its resident one (32 columns of a wave, in
// registers) as the second, both with the head dimension innermost:
//   S^T[key][query] = K Q^T.
// Register v of a 32x32 accumulator in lane l is row 8 (v/4) + 4 (l/32) + v%4,
// column l%32, so a lane holds 16 rows of one column: column maxima and sums
// are register work plus one exchange between lanes l and l + 32.  The next
// product, O^T[d][query] = V^T P^T, takes P^T as its second operand, whose
// lane l wants eight rows of column l%32: the four-row groups that the lane
// already has, provided the first operand's k order is permuted alike, so P
// never leaves its registers.  The first operand V^T is read from the
// row-major V tile by the transposing LDS load (four rows of 16 columns per
// 16 lanes).
#pragma once

#include "block_internal.h"
#include "floats.h"
#include "rows.h"

namespace tasq {

typedef float v16f_t __attribute__((ext_vector_type(16)));
typedef short v4s_t __attribute__((ext_vector_type(4)));
typedef bf16_t v8bf_t __attribute__((ext_vector_type(8)));
typedef f16_t v8h_t __attribute__((ext_vector_type(8)));

__device__ __forceinline__ v16f_t mfma(bf16_t, u32x4 a, u32x4 b, v16f_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf_t, a),
                                                   __builtin_bit_cast(v8bf_t, b), c, 0, 0, 0);
}

__device__ __forceinline__ v16f_t mfma(f16_t, u32x4 a, u32x4 b, v16f_t c)
{
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8h_t, a),
                                                  __builtin_bit_cast(v8h_t, b), c, 0, 0, 0);
}

constexpr int kAttnTile = 64;           // rows of a streamed tile
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A tile of KS * 16 columns (the head dimension rounded up) in LDS: rows of
// 2 KS 16-byte chunks without padding, as the loads to LDS write them, chunk c
// of row r at place c ^ key(r), so that the rows that an operand read spans
// fall in distinct banks.
template <int KS> struct Tile {
    static constexpr int kPitch = KS * 32;
    // The transposing load of an odd KS reads 32 bytes past a row's columns.
    static constexpr int kBytes = kAttnTile * kPitch + 32;
    static constexpr int DB = (KS + 1) / 2;     // 32-row blocks of the transposed tile

    static __device__ __forceinline__ int key(int r)
    {
        return KS % 4 == 0 ? r & 7 : KS % 4 == 2 ? (r >> 1) & 3 : (r >> 2) & 1;
    }

    // This lane's part of the addresses.
    static constexpr int NR = KS % 4 == 0 ? 4 : KS % 4 == 2 ? 2 : 1;
    static constexpr int NC = KS % 4 == 0 ? 2 : 1;
    uint32_t row[NR], col[NC];

    __device__ __forceinline__ Tile()
    {
        const int lane = threadIdx.x & 63, h = lane >> 5;
        const int r = lane & 31;
#pragma unroll
        for (int i = 0; i < NR; ++i)
            row[i] = (uint32_t)(r * kPitch + 16 * ((2 * i + h) ^ key(r)));
        const int c = 4 * h + ((lane & 15) >> 2), x = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
#pragma unroll
        for (int i = 0; i < NC; ++i)
            col[i] = (uint32_t)(c * kPitch + 16 * ((4 * i + x) ^ key(c)) + 8 * (lane & 1));
    }
    // Operand of rows 32 rb .. +31, columns 16 ks .. +15.
    __device__ __forceinline__ u32x4 rows(const char *lds, int rb, int ks) const
    {
        return *reinterpret_cast<const u32x4 *>(lds + row[ks % NR] + rb * 32 * kPitch +
                                                32 * (ks - ks % NR));
    }
    // Transposed operand: columns 32 db .. +31 as rows, rows r0 .. r0 + 15 (r0 a
    // multiple of 16) in the order in which an accumulator holds them as k.
    __device__ __forceinline__ u32x4 columns(const char *lds, int r0, int db) const
    {
        typedef __attribute__((address_space(3))) v4s_t lds_t;
        const char *p = lds + col[db % NC] + r0 * kPitch + 64 * (db - db % NC);
        const u32x2 lo =
            __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)p));
        const u32x2 hi = __builtin_bit_cast(
            u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t *)(p + 8 * kPitch)));
        return u32x4{lo.x, lo.y, hi.x, hi.y};
    }
};

// Lane l's 16 bytes at `off` of the buffer to lds + 16 l; zeros where the
// offset is out of bounds.
__device__ __forceinline__ void load_to_lds(rsrc_t r, char *lds, uint32_t off)
{
#ifdef __HIP_DEVICE_COMPILE__       // the host pass knows no 16-byte form
    typedef __attribute__((address_space(3))) void lds_t;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lds_t *)lds, 16, off, 0, 0, 0);
#endif
}

// One wave's share of staging two tiles: waves 0 and 1 load the halves of the
// first operand's, waves 2 and 3 of the second's, straight into LDS (1 KB an
// instruction, rows `stride` bytes apart, dim elements each).
template <int KS> struct Stager {
    uint32_t off[KS], bytes;
    int half, place;            // of the two tiles of a buffer

    __device__ __forceinline__ void init(int wave, uint32_t stride, int dim)
    {
        half = wave & 1;
        place = (wave >> 1) * Tile<KS>::kBytes + half * 32 * Tile<KS>::kPitch;
        bytes = (kAttnTile - 1) * stride + 2u * (uint32_t)dim;
#pragma unroll
        for (int i = 0; i < KS; ++i) {
            const int r = row(i), c = slot(i) ^ Tile<KS>::key(r);
            off[i] = 8 * c < dim ? (uint32_t)r * stride + 16u * (uint32_t)c : kOOB;
        }
    }
    __device__ __forceinline__ int row(int i) const
    {
        return 32 * half + (64 * i + (int)(threadIdx.x & 63)) / (2 * KS);
    }
    __device__ __forceinline__ int slot(int i) const
    {
        return (64 * i + (int)(threadIdx.x & 63)) % (2 * KS);
    }
    // Requests the rows from p on whose bit in `live` is set; all else is
    // written as zero and not read.  wait() before the barrier that hands the
    // buffer on.
    __device__ __forceinline__ void request(const void *p, uint64_t live, char *buffer) const
    {
        const rsrc_t r = make_rsrc(p, bytes);
        char *to = buffer + place;
        if (live == ~0ull) {
#pragma unroll
            for (int i = 0; i < KS; ++i)
                load_to_lds(r, to + 1024 * i, off[i]);
        } else {
#pragma unroll
            for (int i = 0; i < KS; ++i)
                load_to_lds(r, to + 1024 * i, (live >> row(i)) & 1 ? off[i] : kOOB);
        }
    }
    static __device__ __forceinline__ void wait()
    {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    }
};

// Resident operand: 32 columns of a wave, column l%32 at `p` of each lane
// (or none), KS steps of 16 of the head dimension.
template <int KS>
__device__ __forceinline__ void load_columns(const void *p, bool ok, int dim, u32x4 (&f)[KS])
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        f[ks] = u32x4{0, 0, 0, 0};
        if (ok && 16 * ks + 8 * h < dim)
            f[ks] = reinterpret_cast<const u32x4 *>(p)[2 * ks + h];
    }
}

// Values of lanes l and l + 32 exchanged: (this half's, the other half's)
// combined by f in both lanes.
template <class F> __device__ __forceinline__ float across_halves(float x, F f)
{
    const uint32_t u = __float_as_uint(x);
    const auto p = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    return f(__uint_as_float(p[0]), __uint_as_float(p[1]));
}

// Eight accumulator rows 16 s .. of a block as the second operand's k.
template <class T> __device__ __forceinline__ u32x4 pack_rows(const float (&x)[16], int s)
{
    u32x4 u;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        u[i] = pack2<T>(x[8 * s + 2 * i], x[8 * s + 2 * i + 1]);
    return u;
}

// Stores a transposed accumulator, rows d and columns l%32, as rows of T:
// column l%32 is the row at p of the lanes l and l + 32 (or none), values
// times f.  Two four-row groups change places between the halves, so that a
// lane has eight neighbouring values.
template <class T, int DB>
__device__ __forceinline__ void store_columns(T *p, bool ok, int dim, const v16f_t (&acc)[DB],
                                              float f)
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; j += 2) {
            u32x4 u;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const auto s = __builtin_amdgcn_permlane32_swap(
                    pack2<T>(acc[db][4 * j + 2 * i] * f, acc[db][4 * j + 2 * i + 1] * f),
                    pack2<T>(acc[db][4 * j + 4 + 2 * i] * f, acc[db][4 * j + 5 + 2 * i] * f),
                    false, false);
                u[i] = s[0];
                u[2 + i] = s[1];
            }
            const int d = 32 * db + 8 * (j + h);
            if (ok && d < dim)
                *reinterpret_cast<u32x4 *>(p + d) = u;
        }
}

// The same as rows of fp32.
template <int DB>
__device__ __forceinline__ void store_columns_f32(float *p, bool ok, int dim,
                                                  const v16f_t (&acc)[DB], float f)
{
    const int h = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = 32 * db + 8 * j + 4 * h;
            if (ok && d < dim)
                *reinterpret_cast<float4 *>(p + d) =
                    make_float4(acc[db][4 * j] * f, acc[db][4 * j + 1] * f,
                                acc[db][4 * j + 2] * f, acc[db][4 * j + 3] * f);
        }
}

// -inf where the row's bit in `live` is off, else 0, for the 16 rows of block
// rb that the lane holds.
__device__ __forceinline__ float dead_row(uint64_t live, int rb, int i)
{
    const uint32_t off = ~((uint32_t)(live >> (32 * rb)) >> (4 * ((threadIdx.x & 63) >> 5)));
    const int bit = 8 * (i / 4) + i % 4;
    uint32_t u = (uint32_t)((int)(off << (31 - bit)) >> 31) & 0xff800000u;
    asm("" : "+v"(u));      // or the compiler makes a branch of each row
    return __uint_as_float(u);
}

// Keys of a batch entry that count at all.
__device__ __forceinline__ int key_count(const AttnCall &a, int b)
{
    if (!a.kv_lengths)
        return a.kv_len;
    return min(max(a.kv_lengths[b], 0), a.kv_len);
}

// Key head and batch entry of a workgroup's u.  Entries with lengths take turns
// head by head, so that an XCD's run of workgroups has of the long and the short
// ones alike: 4096 tokens among themselves, batch 2, 100% and 30% of the keys, 16
// heads of 72 170 us and 459 backward, 180 and 600 with the entries one after the
// other.  (Over a few tiles of keys it is 2% slower.)
__device__ __forceinline__ void head_and_entry(const AttnCall &a, int u, int &hk, int &b)
{
    const bool turns = a.kv_lengths && a.kv_len > 8 * kAttnTile;
    const int inner = turns ? a.batch : a.kv_heads, i = u % inner, o = u / inner;
    hk = turns ? o : i;
    b = turns ? i : o;
}

// Tiles t0 .. t1 - 1 of range sp of the n keys that count in length: where the
// entries have lengths, as many ranges of the tiles that each has, so that short
// ones do not leave workgroups idle.
__device__ __forceinline__ void key_range(const AttnCall &a, int n, int sp, int &t0, int &t1)
{
    const int tiles = (n + kAttnTile - 1) / kAttnTile;
    const int each = a.kv_lengths ? (tiles + a.splits - 1) / a.splits : a.split_tiles;
    t0 = sp * each;
    t1 = min(tiles, t0 + each);
}

// Bits of the keys of tile t that count, the keys below n and with a nonzero
// byte in the mask (`byte`: that of key 64 t + lane).
__device__ __forceinline__ uint64_t live_keys(const AttnCall &a, int n, int t, int byte)
{
    const int left = n - kAttnTile * t;
    uint64_t live = left >= kAttnTile ? ~0ull : left <= 0 ? 0ull : (1ull << left) - 1;
    if (a.key_mask)
        live &= __ballot(byte != 0);
    return live;
}

__device__ __forceinline__ int mask_byte(const AttnCall &a, int b, int n, int t)
{
    const int key = kAttnTile * t + (int)(threadIdx.x & 63);
    return a.key_mask && key < n ? a.key_mask[(size_t)b * a.kv_len + key] : 0;
}

// Workgroups are dispatched round-robin over the 8 XCDs; this bijection gives
// each XCD one contiguous run of a launch's logical workgroups, so that those which
// read the same keys meet in one L2.
__device__ __forceinline__ int attn_unit(const AttnCall &a)
{
    const int pid = blockIdx.x, G = gridDim.x;
    const int per = G / 8, more = G % 8, x = pid % 8;
    return a.first_unit + x * per + min(x, more) + pid / 8;
}

}  // namespace tasq
