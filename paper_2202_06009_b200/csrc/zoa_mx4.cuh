// Storage of a 4-bit microscaled matrix [rows, cols], and the rounding to it.
//
// Values: E2M1 codes (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives) with one E8M0 scale byte b, standing for
// 2^(b - 127), per 32 neighbours of a row; b = 255 is NaN.
//
// The matrix is cut into tiles of 128 rows by 256 columns, row tile by row tile, 17408 bytes each:
//   bytes [0, 1024)      scales: two groups of 128 columns, 512 bytes each; row r, block c of the group
//                        (c = 0..3) at (r % 32) * 16 + (r / 32) * 4 + c
//   bytes [1024, 17408)  codes: 128 bytes per row; the 16 bytes of block c (c = 0..7) at c ^ (r % 8); the even
//                        column of a pair in the low nibble
// This is byte for byte what the tensor core reads: the scales as tcgen05.cp copies them to tensor memory, the
// codes as a K-major operand under the 128-byte swizzle.  A tile, or its first rows, is therefore one contiguous
// bulk copy with no tensor map, and the scales travel with their codes.  Columns past the end hold code 0 and
// scale byte 0, so they add nothing to a product; rows past the end are not written and reach only results that
// are not stored.
#pragma once

#include "zoa_ops.h"

#include <type_traits>

namespace zoa {

constexpr int kMxTileRows = 128, kMxTileCols = 256, kMxBlock = 32;
constexpr size_t kMxMaxSide = (size_t)1 << 30;   // keeps every index product below 2^63
constexpr int kMxScaleBytes = 1024, kMxCodeBytes = 16384, kMxTileBytes = kMxScaleBytes + kMxCodeBytes;

__host__ __device__ inline long long mx_tiles(long long n, int per) { return (n + per - 1) / per; }

__device__ __forceinline__ int mx_scale_at(int r, int block)   // within a tile; block = 0..7
{
    return (block >> 2) * 512 + (r & 31) * 16 + (r >> 5) * 4 + (block & 3);
}
__device__ __forceinline__ int mx_code_at(int r, int block) { return kMxScaleBytes + r * 128 + ((block ^ (r & 7)) << 4); }

// Scale byte of a block whose largest magnitude is `most`: floor(log2 most) - 2, the exponent that puts it in
// [4, 8); not below 2^-127; NaN if the block holds a NaN or an infinity (`most` must then be one of them).
__device__ __forceinline__ uint32_t mx_scale_byte(float most)
{
    const uint32_t e = (__float_as_uint(most) >> 23) & 0xFFu;
    return e == 255u ? 255u : e > 2u ? e - 2u : 0u;
}
// 1 / scale, exact (2^127 at most, 2^-125 at least); 0 for a NaN block, whose codes are stored as 0.
__device__ __forceinline__ float mx_inverse(uint32_t byte) { return byte == 255u ? 0.0f : __uint_as_float((254u - byte) << 23); }
__device__ __forceinline__ float mx_scale(uint32_t byte)
{
    return byte == 255u ? __uint_as_float(0x7FC00000u) : byte ? __uint_as_float(byte << 23) : __uint_as_float(0x00400000u);
}

// Eight values, already divided by their scale, in four pairs of binary32 (the first in the low half) to eight codes,
// round to nearest even, 6 at most; the first in the lowest nibble.
__device__ __forceinline__ uint32_t mx_codes8(const uint64_t *p)
{
    uint32_t out;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t.reg .f32 x, y;\n\t"
        "mov.b64 {x, y}, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 a, y, x;\n\t"
        "mov.b64 {x, y}, %2;\n\tcvt.rn.satfinite.e2m1x2.f32 b, y, x;\n\t"
        "mov.b64 {x, y}, %3;\n\tcvt.rn.satfinite.e2m1x2.f32 c, y, x;\n\t"
        "mov.b64 {x, y}, %4;\n\tcvt.rn.satfinite.e2m1x2.f32 d, y, x;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(out)
        : "l"(p[0]), "l"(p[1]), "l"(p[2]), "l"(p[3]));
    return out;
}

// Eight neighbours of a row as they lie in memory.
template <typename T>
struct Raw8 {
    static constexpr int kWords = 2 * (int)sizeof(T);
    uint32_t w[kWords];
};

// `have` of the eight exist (0 or less: none); the others are 0.
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const T *at, long long have, bool vec)
{
    Raw8<T> r;
    if (vec && have >= 8) {
#pragma unroll
        for (int k = 0; k < Raw8<T>::kWords; k += 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(at) + k / 4);
            r.w[k] = v.x;
            r.w[k + 1] = v.y;
            r.w[k + 2] = v.z;
            r.w[k + 3] = v.w;
        }
        return r;
    }
#pragma unroll
    for (int k = 0; k < Raw8<T>::kWords; ++k) {
        if constexpr (sizeof(T) == 4) {
            r.w[k] = k < have ? reinterpret_cast<const uint32_t *>(at)[k] : 0u;
        } else {
            const uint16_t *p = reinterpret_cast<const uint16_t *>(at) + 2 * k;
            r.w[k] = (2 * k < have ? p[0] : 0u) | (2 * k + 1 < have ? (uint32_t)p[1] << 16 : 0u);
        }
    }
    return r;
}

// The larger of two magnitudes (of each half, for the 16-bit types); a NaN wins.  binary32 compares its bits, which
// order finite < inf < NaN without their sign.
template <typename T>
__device__ __forceinline__ uint32_t larger(uint32_t magnitude, uint32_t w)
{
    if constexpr (sizeof(T) == 4) {
        return max(magnitude, w & 0x7FFFFFFFu);
    } else {
        using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
        const T2 r = __hmax2_nan(*reinterpret_cast<const T2 *>(&magnitude), __habs2(*reinterpret_cast<const T2 *>(&w)));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
}
// Of the two halves of a word of a 16-bit type: bits of magnitudes order like the magnitudes.
__device__ __forceinline__ uint32_t larger_half(uint32_t m) { return max(m & 0xFFFFu, m >> 16); }
// The magnitude of one element (the low half word of the 16-bit types) as binary32.
template <typename T>
__device__ __forceinline__ float magnitude_f32(uint32_t m)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(m);
    else {
        float lo, hi;
        unpack2<T>(m, lo, hi);
        return lo;
    }
}

__device__ __forceinline__ uint64_t times2(uint32_t lo, uint32_t hi, uint64_t by)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"((uint64_t)hi << 32 | lo), "l"(by));
    return r;
}
template <typename T>
__device__ __forceinline__ uint32_t codes8(const Raw8<T> &r, float inv)
{
    const uint64_t by = (uint64_t)__float_as_uint(inv) << 32 | __float_as_uint(inv);
    uint64_t p[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) {
            p[k] = times2(r.w[2 * k], r.w[2 * k + 1], by);
        } else {
            float lo, hi;
            unpack2<T>(r.w[k], lo, hi);
            p[k] = times2(__float_as_uint(lo), __float_as_uint(hi), by);
        }
    }
    return mx_codes8(p);
}

// A whole block of a row, 32 elements, as they lie in memory.
template <typename T>
struct Raw32 {
    static constexpr int kWords = 8 * (int)sizeof(T);
    uint32_t w[kWords];
    __device__ __forceinline__ Raw8<T> eight(int k) const
    {
        Raw8<T> r;
#pragma unroll
        for (int i = 0; i < Raw8<T>::kWords; ++i) r.w[i] = w[k * Raw8<T>::kWords + i];
        return r;
    }
};
template <typename T>
__device__ __forceinline__ Raw32<T> load32(const T *at, long long have, bool vec)
{
    Raw32<T> r;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Raw8<T> e = load8(at + 8 * k, have - 8 * k, vec);
#pragma unroll
        for (int i = 0; i < Raw8<T>::kWords; ++i) r.w[k * Raw8<T>::kWords + i] = e.w[i];
    }
    return r;
}
// Its scale byte, and its codes.
template <typename T>
__device__ __forceinline__ uint4 round32_block(const Raw32<T> &r, uint32_t &byte)
{
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < Raw32<T>::kWords; ++k) m = larger<T>(m, r.w[k]);
    if (sizeof(T) == 2) m = larger_half(m);
    byte = mx_scale_byte(magnitude_f32<T>(m));
    if (byte == 255u) return make_uint4(0, 0, 0, 0);
    const float inv = mx_inverse(byte);
    return make_uint4(codes8(r.eight(0), inv), codes8(r.eight(1), inv), codes8(r.eight(2), inv), codes8(r.eight(3), inv));
}
// The scale word of four neighbouring blocks, one to a lane, lane & 3 being the block: complete in all four.
__device__ __forceinline__ uint32_t scale_word(uint32_t byte, int lane)
{
    uint32_t w = byte << (8 * (lane & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 1);
    w |= __shfl_xor_sync(0xffffffffu, w, 2);
    return w;
}

// A matrix to be rounded both ways (out may be NULL), and the launch for one or two of them (b.rows = 0: one).
struct BothJob {
    const void *x;
    uint8_t *out, *out_t;
    long long rows, cols, ld;
    int vec;
};
zoa_status mx4_check_source(const char *me, const void *x, int dtype, size_t rows, size_t cols, size_t ld, const void *out, const void *out_t);
BothJob mx4_both_job(const void *x, int dtype, size_t rows, size_t cols, size_t ld, void *out, void *out_t);
zoa_status mx4_launch_both(const char *me, int dtype, const BothJob &a, const BothJob &b, cudaStream_t s);

// Scale byte of the block that this lane shares with its three neighbours.
template <typename T>
__device__ __forceinline__ uint32_t block_scale(const Raw8<T> &r)
{
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < Raw8<T>::kWords; ++k) m = larger<T>(m, r.w[k]);
    if (sizeof(T) == 2) m = larger_half(m);
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
    m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
    return mx_scale_byte(magnitude_f32<T>(m));
}

// Eight codes as eight binary16, the lowest nibble first.
__device__ __forceinline__ void mx_halves8(uint32_t codes, uint32_t *v)
{
    asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
        : "r"(codes));
}

}  // namespace zoa
