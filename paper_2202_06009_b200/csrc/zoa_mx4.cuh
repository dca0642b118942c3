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

}  // namespace zoa
