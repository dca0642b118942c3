// Rounding to 4-bit microscaled form (along the rows, along the columns, or both from one read) and reading back.
#include "zoa_mx4.cuh"

namespace zoa {
namespace {

constexpr int kRowWarps = 8;      // warps of a block of quantize_rows_kernel
constexpr int kRowsPerWarp = 4;   // rows whose loads a warp has in flight at once

// The 4-byte scale words of a row's two groups of 128 columns, from the scale byte that every lane of block
// lane / 4 holds: complete in lanes 0 and 16.
__device__ __forceinline__ uint32_t gather_scales(uint32_t byte, int lane)
{
    uint32_t w = byte << (8 * ((lane >> 2) & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 4);
    w |= __shfl_xor_sync(0xffffffffu, w, 8);
    return w;
}

// One warp takes 256 columns (a line of a tile) of kRowsPerWarp rows at a time, a lane 8 neighbours: a block is four
// lanes.  Warps walk over the matrix, the next rows' loads in flight beside this one's arithmetic.
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) quantize_rows_kernel(const T *__restrict__ x, long long rows, long long cols,
                                                                       long long ld, bool vec, uint8_t *__restrict__ out)
{
    const int lane = threadIdx.x & 31;
    const int tiles_c = (int)mx_tiles(cols, kMxTileCols);
    // A warp's place (rows from r0, tile tile_c) moves on by the number of warps, kept as whole rows of tiles and a rest.
    const unsigned warps = gridDim.x * kRowWarps, me = blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    const long long step_rows = (long long)(warps / tiles_c) * kRowsPerWarp;
    const int step_tiles = (int)(warps % tiles_c);
    long long next_r0 = (long long)(me / tiles_c) * kRowsPerWarp;
    int next_tile = (int)(me % tiles_c);
    Raw8<T> next[kRowsPerWarp];
    auto fetch = [&] {
        const long long c = (long long)next_tile * kMxTileCols + lane * 8;
        const T *at = x + next_r0 * ld + c;
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i, at += ld)
            if (next_r0 + i < rows) next[i] = load8(at, cols - c, vec);
    };
    fetch();
    while (next_r0 < rows) {
        Raw8<T> v[kRowsPerWarp];
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i) v[i] = next[i];
        const long long r0 = next_r0;
        const int tile_c = next_tile;
        next_r0 += step_rows;
        next_tile += step_tiles;
        if (next_tile >= tiles_c) {
            next_tile -= tiles_c;
            next_r0 += kRowsPerWarp;
        }
        fetch();
        const int there = (int)(rows - r0 < kRowsPerWarp ? rows - r0 : kRowsPerWarp), rr = (int)(r0 % kMxTileRows);
        uint8_t *tile = out + ((r0 / kMxTileRows) * tiles_c + tile_c) * kMxTileBytes;       // kRowsPerWarp divides its rows
        uint8_t *codes_at = tile + kMxScaleBytes + rr * 128 + (lane & 3) * 4, *scales_at = tile + mx_scale_at(rr, lane >> 2);
        const int line = ((lane >> 2) ^ (rr & 7)) << 4;
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i) {
            if (i >= there) break;
            const uint32_t byte = block_scale(v[i]);
            const uint32_t codes = byte == 255u ? 0u : codes8(v[i], mx_inverse(byte));
            const uint32_t scales = gather_scales(byte, lane);
            *reinterpret_cast<uint32_t *>(codes_at + i * 128 + (line ^ (i << 4))) = codes;
            if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(scales_at + i * 16) = scales;
        }
    }
}

// One block takes 128 x 128 elements: rounds them along the rows as it loads them, keeps them in shared memory and
// rounds them along the columns (the rows of the transposed matrix) from there, a thread 32 rows of one column (of a
// pair of columns for the 16-bit types).  Four neighbouring lanes take the four blocks of a column, so that they write
// 64 bytes of a line together; the columns' places in shared memory are shifted by 8 words for each block of rows, so
// that those lanes read different banks.
constexpr int kBothThreads = 256;
constexpr int kBothSide = 128;
template <typename T>
__global__ void __launch_bounds__(kBothThreads) quantize_both_kernel(const T *__restrict__ x, long long rows, long long cols,
                                                                     long long ld, bool vec, uint8_t *__restrict__ out,
                                                                     uint8_t *__restrict__ out_t)
{
    constexpr int kRowWords = kBothSide * (int)sizeof(T) / 4, kPasses = kBothSide / 16;
    extern __shared__ __align__(16) unsigned char both_smem[];
    uint32_t *tile_s = reinterpret_cast<uint32_t *>(both_smem);   // [128][kRowWords]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c0 = (long long)blockIdx.x * kBothSide, r0 = (long long)blockIdx.y * kBothSide;
    const long long tiles_c = mx_tiles(cols, kMxTileCols), tiles_ct = mx_tiles(rows, kMxTileCols);
    const int half = lane >> 4, l16 = lane & 15;
    const int group = (int)((c0 / kBothSide) & 1);                      // which half of a tile's columns
    uint8_t *tile = out ? out + ((r0 / kMxTileRows) * tiles_c + c0 / kMxTileCols) * kMxTileBytes : nullptr;
    const bool last_half = group == 0 && c0 + kBothSide >= cols;        // the tile's second half has no block of its own

    // A half warp holds 128 columns of a row; all loads first.  Rows that are not aligned go element by element to
    // shared memory, where they are.
    Raw8<T> v[kPasses];
    auto word_at = [&](int rr, int k) { return tile_s + rr * kRowWords + ((l16 * Raw8<T>::kWords + k) ^ ((rr >> 5) * 8)); };
    if (vec) {
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int rr = i * 16 + warp * 2 + half;
            v[i] = load8(x + (r0 + rr) * ld + c0 + l16 * 8, r0 + rr < rows ? cols - c0 - l16 * 8 : 0, true);
        }
    } else {
        using Bits = typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type;
        const int col = threadIdx.x % kBothSide;
#pragma unroll 8
        for (int i = 0; i < kBothSide / 2; ++i) {
            const int rr = i * 2 + threadIdx.x / kBothSide;
            Bits e = 0;
            if (r0 + rr < rows && c0 + col < cols) e = reinterpret_cast<const Bits *>(x)[(r0 + rr) * ld + c0 + col];
            const int word = sizeof(T) == 4 ? col : col >> 1;
            Bits *at = reinterpret_cast<Bits *>(tile_s + rr * kRowWords + (word ^ ((rr >> 5) * 8)));
            at[sizeof(T) == 4 ? 0 : col & 1] = e;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int rr = i * 16 + warp * 2 + half;
#pragma unroll
            for (int k = 0; k < Raw8<T>::kWords; k += 4) {
                const uint4 w = *reinterpret_cast<const uint4 *>(word_at(rr, k));
                v[i].w[k] = w.x;
                v[i].w[k + 1] = w.y;
                v[i].w[k + 2] = w.z;
                v[i].w[k + 3] = w.w;
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kPasses; ++i) {
        const int rr = i * 16 + warp * 2 + half;
        if (vec) {
#pragma unroll
            for (int k = 0; k < Raw8<T>::kWords; k += 4)
                *reinterpret_cast<uint4 *>(word_at(rr, k)) = make_uint4(v[i].w[k], v[i].w[k + 1], v[i].w[k + 2], v[i].w[k + 3]);
        }
        if (!tile) continue;
        const uint32_t byte = block_scale(v[i]);
        const uint32_t codes = byte == 255u ? 0u : codes8(v[i], mx_inverse(byte));
        const uint32_t scales = gather_scales(byte, lane);
        if (r0 + rr >= rows) continue;
        *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, group * 4 + (l16 >> 2)) + (l16 & 3) * 4) = codes;
        if (l16 == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, group * 4)) = scales;
        if (last_half) {
            *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, 4 + (l16 >> 2)) + (l16 & 3) * 4) = 0u;
            if (l16 == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, 4)) = 0u;
        }
    }
    __syncthreads();
    const int group_t = (int)((r0 / kBothSide) & 1);
    const bool last_half_t = group_t == 0 && r0 + kBothSide >= rows;
    uint8_t *tile_t = out_t + ((c0 / kMxTileRows) * tiles_ct + r0 / kMxTileCols) * kMxTileBytes;
    const int blk = lane & 3;
    // One column's codes and scale; the four lanes' scale bytes make a word.
    auto store_column = [&](int cc, uint32_t byte, uint4 codes) {
        uint32_t word = byte << (8 * blk);
        word |= __shfl_xor_sync(0xffffffffu, word, 1);
        word |= __shfl_xor_sync(0xffffffffu, word, 2);
        if (c0 + cc >= cols) return;
        if (byte == 255u) codes = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4 *>(tile_t + mx_code_at(cc, group_t * 4 + blk)) = codes;
        if (blk == 0) *reinterpret_cast<uint32_t *>(tile_t + mx_scale_at(cc, group_t * 4)) = word;
        if (last_half_t) {
            *reinterpret_cast<uint4 *>(tile_t + mx_code_at(cc, 4 + blk)) = make_uint4(0, 0, 0, 0);
            if (blk == 0) *reinterpret_cast<uint32_t *>(tile_t + mx_scale_at(cc, 4)) = 0u;
        }
    };
    for (int col = threadIdx.x >> 2; col < kRowWords; col += kBothThreads / 4) {     // a word: one column, or a pair
        uint32_t w[32];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            w[k] = tile_s[(blk * 32 + k) * kRowWords + (col ^ (blk * 8))];
            m = larger<T>(m, w[k]);
        }
        constexpr int kColumns = 4 / (int)sizeof(T);
        uint32_t byte[kColumns], codes[kColumns][4];
        uint64_t by[kColumns];
#pragma unroll
        for (int h = 0; h < kColumns; ++h) {
            byte[h] = mx_scale_byte(magnitude_f32<T>(kColumns == 1 ? m : h ? m >> 16 : m & 0xFFFFu));
            const float inv = mx_inverse(byte[h]);
            by[h] = (uint64_t)__float_as_uint(inv) << 32 | __float_as_uint(inv);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            uint64_t p[kColumns][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t a = w[8 * q + 2 * k], b = w[8 * q + 2 * k + 1];
                if constexpr (kColumns == 1) {
                    p[0][k] = times2(a, b, by[0]);
                } else {
                    float a0, a1, b0, b1;
                    unpack2<T>(a, a0, a1);
                    unpack2<T>(b, b0, b1);
                    p[0][k] = times2(__float_as_uint(a0), __float_as_uint(b0), by[0]);
                    p[1][k] = times2(__float_as_uint(a1), __float_as_uint(b1), by[1]);
                }
            }
#pragma unroll
            for (int h = 0; h < kColumns; ++h) codes[h][q] = mx_codes8(p[h]);
        }
#pragma unroll
        for (int h = 0; h < kColumns; ++h) store_column(kColumns * col + h, byte[h], make_uint4(codes[h][0], codes[h][1], codes[h][2], codes[h][3]));
    }
}

// Eight codes and their scale byte as bfloat16: the bytes of the eight magnitudes (0, 0.5, 1, 1.5, 2, 3, 4, 6 are
// 0000 3F00 3F80 3FC0 4000 4040 4080 40C0) looked up four at a time, the signs put in, and one exact product by the
// scale, which bfloat16 holds whatever its exponent.
__device__ __forceinline__ uint4 values8(uint32_t codes, uint32_t byte)
{
    const uint32_t sel = codes & 0x77777777u;
    uint32_t word[4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t low = __byte_perm(0xC0800000u, 0xC0804000u, sel >> (16 * h)), high = __byte_perm(0x3F3F3F00u, 0x40404040u, sel >> (16 * h));
        word[2 * h] = __byte_perm(low, high, 0x5140);
        word[2 * h + 1] = __byte_perm(low, high, 0x7362);
    }
    const uint32_t scale = byte == 255u ? 0x7FC0u : byte ? byte << 7 : 0x0040u;
    const uint32_t scale2 = scale << 16 | scale;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t pair = codes >> (8 * k);
        word[k] |= (pair << 12 & 0x8000u) | (pair << 24 & 0x80000000u);
        const __nv_bfloat162 v = __hmul2(*reinterpret_cast<const __nv_bfloat162 *>(&word[k]), *reinterpret_cast<const __nv_bfloat162 *>(&scale2));
        word[k] = *reinterpret_cast<const uint32_t *>(&v);
    }
    return make_uint4(word[0], word[1], word[2], word[3]);
}

// A warp reads 256 columns of kReadRows rows, a lane the 8 values of one 4-byte word of each.
constexpr int kReadRows = 8;
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) dequantize_kernel(const uint8_t *__restrict__ in, long long rows, long long cols,
                                                                    T *__restrict__ out, long long ld, bool vec)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long tile_c = blockIdx.x, tiles_c = gridDim.x;
    const long long c = tile_c * kMxTileCols + lane * 8;
    const long long r0 = ((long long)blockIdx.y * kRowWarps + warp) * kReadRows;
    if (c >= cols || r0 >= rows) return;
    const int there = (int)(rows - r0 < kReadRows ? rows - r0 : kReadRows), rr = (int)(r0 % kMxTileRows);       // kReadRows divides a tile's rows
    const uint8_t *tile = in + ((r0 / kMxTileRows) * tiles_c + tile_c) * kMxTileBytes;
    const uint8_t *codes_at = tile + kMxScaleBytes + rr * 128 + (lane & 3) * 4, *scales_at = tile + mx_scale_at(rr, lane >> 2);
    uint32_t codes[kReadRows], bytes[kReadRows];
#pragma unroll
    for (int i = 0; i < kReadRows; ++i) {
        if (i >= there) break;
        codes[i] = __ldg(reinterpret_cast<const uint32_t *>(codes_at + i * 128 + (((lane >> 2) ^ i) << 4)));
        bytes[i] = __ldg(scales_at + i * 16);
    }
    const bool whole = vec && c + 8 <= cols;
    T *dst = out + r0 * ld + c;
#pragma unroll
    for (int i = 0; i < kReadRows; ++i, dst += ld) {
        if (i >= there) break;
        if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            if (whole) {
                *reinterpret_cast<uint4 *>(dst) = values8(codes[i], bytes[i]);
                continue;
            }
        }
        const float s = mx_scale(bytes[i]);
        float v[8];
        uint32_t h[4];
        mx_halves8(codes[i], h);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float lo, hi;
            unpack2<__half>(h[k], lo, hi);
            v[2 * k] = lo * s;
            v[2 * k + 1] = hi * s;
        }
        if (whole) {
            *reinterpret_cast<uint4 *>(dst) = Vec<T>::pack(v);
            if constexpr (sizeof(T) == 4) *reinterpret_cast<uint4 *>(dst + 4) = Vec<T>::pack(v + 4);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) dst[k] = from_f32<T>(v[k]);
        }
    }
}

bool rows_vectorised(const void *p, int dtype, size_t ld) { return aligned16(p) && ld * dtype_bytes(dtype) % 16 == 0; }

}  // namespace
}  // namespace zoa

using namespace zoa;

extern "C" size_t zoa_mx4_size(size_t rows, size_t cols)
{
    if (rows < 1 || cols < 1 || rows > kMxMaxSide || cols > kMxMaxSide) return 0;
    return (size_t)(mx_tiles((long long)rows, kMxTileRows) * mx_tiles((long long)cols, kMxTileCols)) * kMxTileBytes;
}

extern "C" zoa_status zoa_mx4_quantize(const void *x, int dtype, size_t rows, size_t cols, size_t ld, void *out, void *out_t,
                                       void *stream)
{
    const char *me = "zoa_mx4_quantize";
    if (!dtype_ok(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, dtype);
    if (rows > kMxMaxSide || cols > kMxMaxSide) return ops_fail(ZOA_ERR_ARG, "%s: rows and cols must be at most 2^30", me);
    if (rows == 0 || cols == 0) return ZOA_OK;
    if (!x || (!out && !out_t)) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    if (ld < cols) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least cols", me);
    if (reinterpret_cast<uintptr_t>(x) % dtype_bytes(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: x is not aligned to its element type", me);
    if (!aligned16(out) || !aligned16(out_t)) return ops_fail(ZOA_ERR_ARG, "%s: out and out_t must be 16-byte aligned", me);
    const bool vec = rows_vectorised(x, dtype, ld);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    const long long R = (long long)rows, C = (long long)cols, L = (long long)ld;
    if (!out_t) {
        const long long blocks = mx_tiles(mx_tiles(R, kRowsPerWarp) * mx_tiles(C, kMxTileCols), kRowWarps), most = 4ll * ops_sm_count();
        with_type(dtype, [&](auto t) {
            using T = decltype(t);
            quantize_rows_kernel<T><<<(unsigned)(blocks < most ? blocks : most), kRowWarps * 32, 0, s>>>(static_cast<const T *>(x), R, C, L, vec,
                                                                                                       static_cast<uint8_t *>(out));
        });
        return ops_launched(me);
    }
    if (mx_tiles(R, kBothSide) > 65535) return ops_fail(ZOA_ERR_ARG, "%s: at most 8388480 rows when out_t is asked for", me);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const int smem = kBothSide * kBothSide * (int)sizeof(T);
        if (smem > 48 * 1024) {
            static SmemLimit limit;
            if (limit.ensure(quantize_both_kernel<T>, smem) != cudaSuccess) return;   // the launch below reports it
        }
        quantize_both_kernel<T><<<dim3((unsigned)mx_tiles(C, kBothSide), (unsigned)mx_tiles(R, kBothSide)), kBothThreads, smem, s>>>(
            static_cast<const T *>(x), R, C, L, vec, static_cast<uint8_t *>(out), static_cast<uint8_t *>(out_t));
    });
    return ops_launched(me);
}

extern "C" zoa_status zoa_mx4_dequantize(const void *q, size_t rows, size_t cols, void *out, int dtype, size_t ld, void *stream)
{
    const char *me = "zoa_mx4_dequantize";
    if (!dtype_ok(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, dtype);
    if (rows > kMxMaxSide || cols > kMxMaxSide) return ops_fail(ZOA_ERR_ARG, "%s: rows and cols must be at most 2^30", me);
    if (rows == 0 || cols == 0) return ZOA_OK;
    if (!q || !out) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    if (ld < cols) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least cols", me);
    if (!aligned16(q)) return ops_fail(ZOA_ERR_ARG, "%s: q must be 16-byte aligned", me);
    if (reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: out is not aligned to its element type", me);
    const bool vec = rows_vectorised(out, dtype, ld);
    const long long R = (long long)rows, C = (long long)cols, L = (long long)ld, per = kRowWarps * kReadRows, gy = mx_tiles(R, per);
    zoa_status st = ZOA_OK;
    // gridDim.y holds 65535 blocks: a larger matrix takes several launches, whole row tiles each.
    for (long long y = 0; y < gy && st == ZOA_OK; y += 65532) {
        const long long n = gy - y < 65532 ? gy - y : 65532, r = y * per;
        with_type(dtype, [&](auto t) {
            using T = decltype(t);
            dequantize_kernel<T><<<dim3((unsigned)mx_tiles(C, kMxTileCols), (unsigned)n), kRowWarps * 32, 0, static_cast<cudaStream_t>(stream)>>>(
                static_cast<const uint8_t *>(q) + r / kMxTileRows * mx_tiles(C, kMxTileCols) * kMxTileBytes, R - r, C,
                static_cast<T *>(out) + r * L, L, vec);
        });
        st = ops_launched(me);
    }
    return st;
}
