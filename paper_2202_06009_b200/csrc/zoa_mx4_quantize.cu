// Rounding to 4-bit microscaled form (along the rows, along the columns, or both from one read) and reading back.
#include "zoa_mx4.cuh"

namespace zoa {
namespace {

constexpr int kRowWarps = 8;      // warps of a block of quantize_rows_kernel
constexpr int kRowsPerWarp = 4;   // rows a warp takes at once

// The 4-byte scale words of a row's two groups of 128 columns, from the scale byte that every lane of block
// lane / 4 holds: complete in lanes 0 and 16.
__device__ __forceinline__ uint32_t gather_scales(uint32_t byte, int lane)
{
    uint32_t w = byte << (8 * ((lane >> 2) & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 4);
    w |= __shfl_xor_sync(0xffffffffu, w, 8);
    return w;
}

// A warp takes 256 columns (a line of a tile) of four rows at a time, a lane one block of 32 columns.  Warps walk over the
// matrix, the next rows' loads in flight beside this one's arithmetic.  What bounds it beside memory is instructions:
// a lane to a block needs no exchange for the block's maximum and one scale for 32 elements (with four lanes to a block
// 16384 x 4096 took 35 us; this way 26, 6.5 TB/s, the copy rate).
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) quantize_rows_kernel(const T *__restrict__ x, long long rows, long long cols,
                                                                       long long ld, bool vec, uint8_t *__restrict__ out)
{
    const int lane = threadIdx.x & 31, row = lane >> 3, block = lane & 7;
    const int tiles_c = (int)mx_tiles(cols, kMxTileCols);
    // A warp's place (rows from r0, tile tile_c) moves on by the number of warps, kept as whole rows of tiles and a rest.
    const unsigned warps = gridDim.x * kRowWarps, me = blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    const long long step_rows = (long long)(warps / tiles_c) * kRowsPerWarp;
    const int step_tiles = (int)(warps % tiles_c);
    long long next_r0 = (long long)(me / tiles_c) * kRowsPerWarp;
    int next_tile = (int)(me % tiles_c);
    Raw32<T> next;
    auto fetch = [&] {
        const long long c = (long long)next_tile * kMxTileCols + block * kMxBlock, r = next_r0 + row;
        if (r < rows) next = load32(x + r * ld + c, cols - c, vec);
    };
    fetch();
    while (next_r0 < rows) {
        const Raw32<T> v = next;
        const long long r0 = next_r0;
        const int tile_c = next_tile;
        next_r0 += step_rows;
        next_tile += step_tiles;
        if (next_tile >= tiles_c) {
            next_tile -= tiles_c;
            next_r0 += kRowsPerWarp;
        }
        fetch();
        uint32_t byte;
        const uint4 codes = round32_block(v, byte);
        const uint32_t scales = scale_word(byte, lane);
        if (r0 + row >= rows) continue;
        uint8_t *tile = out + ((r0 / kMxTileRows) * tiles_c + tile_c) * kMxTileBytes;       // kRowsPerWarp divides its rows
        const int rr = (int)(r0 % kMxTileRows) + row;
        *reinterpret_cast<uint4 *>(tile + mx_code_at(rr, block)) = codes;
        if ((lane & 3) == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, block)) = scales;
    }
}

// The same for binary32, where a lane's block would be a whole 128-byte line: four lanes to a block, so that a load takes
// neighbours (8192 x 4096: 34 us, a lane to a block 43).
__global__ void __launch_bounds__(kRowWarps * 32) quantize_rows_f32_kernel(const float *__restrict__ x, long long rows, long long cols, long long ld,
                                                                          bool vec, uint8_t *__restrict__ out)
{
    const int lane = threadIdx.x & 31;
    const int tiles_c = (int)mx_tiles(cols, kMxTileCols);
    const unsigned warps = gridDim.x * kRowWarps, me = blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    const long long step_rows = (long long)(warps / tiles_c) * kRowsPerWarp;
    const int step_tiles = (int)(warps % tiles_c);
    long long next_r0 = (long long)(me / tiles_c) * kRowsPerWarp;
    int next_tile = (int)(me % tiles_c);
    Raw8<float> next[kRowsPerWarp];
    auto fetch = [&] {
        const long long c = (long long)next_tile * kMxTileCols + lane * 8;
        const float *at = x + next_r0 * ld + c;
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i, at += ld)
            if (next_r0 + i < rows) next[i] = load8(at, cols - c, vec);
    };
    fetch();
    while (next_r0 < rows) {
        Raw8<float> v[kRowsPerWarp];
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
        uint8_t *tile = out + ((r0 / kMxTileRows) * tiles_c + tile_c) * kMxTileBytes;
#pragma unroll
        for (int i = 0; i < kRowsPerWarp; ++i) {
            if (i >= there) break;
            const uint32_t byte = block_scale(v[i]);
            const uint32_t codes = byte == 255u ? 0u : codes8(v[i], mx_inverse(byte));
            const uint32_t scales = gather_scales(byte, lane);
            *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr + i, lane >> 2) + (lane & 3) * 4) = codes;
            if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr + i, lane >> 2)) = scales;
        }
    }
}

// One block takes 128 x 128 elements: rounds them along the rows as it loads them, keeps them in shared memory and
// rounds them along the columns (the rows of the transposed matrix) from there.  Along the rows a thread takes one block
// of 32 columns at a time, along the columns 32 rows of one column (of a pair of columns for the 16-bit types).  Four
// neighbouring lanes take the four blocks of a row or column, so that they write 64 bytes of a line together; the
// columns' places in shared memory are shifted by 8 words for each block of rows, so that those lanes read different
// banks.  (binary32: as in quantize_rows_f32_kernel along the rows.)  16384 x 4096 bfloat16 in 47 us, 4.4 TB/s of the
// bytes it must move, binary32 in 77, 4.4.  No single limit is reached (issue slots 64 %, ALU 52 %, device memory 32 %): loads,
// rows and columns follow one another behind two barriers, and only other blocks' run beside them.
constexpr int kBothThreads = 256;
constexpr int kBothSide = 128;
template <typename T>
constexpr int kBothPitch = kBothSide * (int)sizeof(T) / 4 + (sizeof(T) == 4 ? 0 : 4);      // words a row
template <typename T>
__global__ void __launch_bounds__(kBothThreads, sizeof(T) == 4 ? 3 : 4) quantize_both_kernel(const BothJob first, const BothJob second, const unsigned first_blocks)
{
    constexpr int kRowWords = kBothSide * (int)sizeof(T) / 4, kPitch = kBothPitch<T>;
    extern __shared__ __align__(16) unsigned char both_smem[];
    uint32_t *tile_s = reinterpret_cast<uint32_t *>(both_smem);   // [128][kPitch]
    const bool is_second = blockIdx.x >= first_blocks;
    const BothJob &job = is_second ? second : first;
    const long long rows = job.rows, cols = job.cols, ld = job.ld;
    const T *x = static_cast<const T *>(job.x);
    const unsigned index = is_second ? blockIdx.x - first_blocks : blockIdx.x, across = (unsigned)mx_tiles(cols, kBothSide);
    const long long c0 = (long long)(index % across) * kBothSide, r0 = (long long)(index / across) * kBothSide;
    const int lane = threadIdx.x & 31, blk = lane & 3;
    const long long tiles_c = mx_tiles(cols, kMxTileCols), tiles_ct = mx_tiles(rows, kMxTileCols);
    const int group = (int)((c0 / kBothSide) & 1);                      // which half of a tile's columns
    uint8_t *tile = job.out ? job.out + ((r0 / kMxTileRows) * tiles_c + c0 / kMxTileCols) * kMxTileBytes : nullptr;
    const bool last_half = group == 0 && c0 + kBothSide >= cols;        // the tile's second half has no block of its own
    auto word_at = [&](int rr, int word) { return tile_s + rr * kPitch + (word ^ ((rr >> 5) * 8)); };
    // One row's (column's) codes and scale, to line r of `to`; the four lanes' scale bytes make a word.
    auto store_line = [&](uint8_t *to, int r, int half, bool exists, bool clear_next, uint32_t byte, const uint4 &codes) {
        const uint32_t scales = scale_word(byte, lane);
        if (!exists) return;
        *reinterpret_cast<uint4 *>(to + mx_code_at(r, half * 4 + blk)) = codes;
        if (blk == 0) *reinterpret_cast<uint32_t *>(to + mx_scale_at(r, half * 4)) = scales;
        if (clear_next) {
            *reinterpret_cast<uint4 *>(to + mx_code_at(r, 4 + blk)) = make_uint4(0, 0, 0, 0);
            if (blk == 0) *reinterpret_cast<uint32_t *>(to + mx_scale_at(r, 4)) = 0u;
        }
    };

    // Along the rows; all loads first.  Rows that are not aligned go element by element to shared memory, where they are.
    if (!job.vec) {
        using Bits = typename std::conditional<sizeof(T) == 4, uint32_t, uint16_t>::type;
        const int col = threadIdx.x % kBothSide;
#pragma unroll 8
        for (int i = 0; i < kBothSide / 2; ++i) {
            const int rr = i * 2 + threadIdx.x / kBothSide;
            Bits e = 0;
            if (r0 + rr < rows && c0 + col < cols) e = reinterpret_cast<const Bits *>(x)[(r0 + rr) * ld + c0 + col];
            reinterpret_cast<Bits *>(word_at(rr, sizeof(T) == 4 ? col : col >> 1))[sizeof(T) == 4 ? 0 : col & 1] = e;
        }
        __syncthreads();
    }
    // Between registers and shared memory, whichever has them.
    auto settle = [&](uint32_t *w, int words, int rr, int first) {
#pragma unroll
        for (int k = 0; k < words; k += 4) {
            uint4 *at = reinterpret_cast<uint4 *>(word_at(rr, first + k));
            if (job.vec) {
                *at = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
            } else {
                const uint4 v = *at;
                w[k] = v.x;
                w[k + 1] = v.y;
                w[k + 2] = v.z;
                w[k + 3] = v.w;
            }
        }
    };
    if constexpr (sizeof(T) == 4) {      // four lanes to a block, half a warp to a row, as in quantize_rows_f32_kernel
        constexpr int kPasses = kBothSide / 16;
        const int half = lane >> 4, l16 = lane & 15, warp = threadIdx.x >> 5;
        Raw8<T> v[kPasses];
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int rr = i * 16 + warp * 2 + half;
            if (job.vec) v[i] = load8(x + (r0 + rr) * ld + c0 + l16 * 8, r0 + rr < rows ? cols - c0 - l16 * 8 : 0, true);
        }
#pragma unroll
        for (int i = 0; i < kPasses; ++i) {
            const int rr = i * 16 + warp * 2 + half;
            settle(v[i].w, 8, rr, l16 * 8);
            if (!tile) continue;
            const uint32_t byte = block_scale(v[i]), codes = byte == 255u ? 0u : codes8(v[i], mx_inverse(byte));
            const uint32_t scales = gather_scales(byte, lane);
            if (r0 + rr >= rows) continue;
            *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, group * 4 + (l16 >> 2)) + (l16 & 3) * 4) = codes;
            if (l16 == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, group * 4)) = scales;
            if (last_half) {
                *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, 4 + (l16 >> 2)) + (l16 & 3) * 4) = 0u;
                if (l16 == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, 4)) = 0u;
            }
        }
    } else {
        Raw32<T> v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rr = i * 64 + (threadIdx.x >> 2);
            const long long c = c0 + blk * kMxBlock;
            if (job.vec) v[i] = load32(x + (r0 + rr) * ld + c, r0 + rr < rows ? cols - c : 0, true);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int rr = i * 64 + (threadIdx.x >> 2);
            settle(v[i].w, Raw32<T>::kWords, rr, blk * Raw32<T>::kWords);
            if (!tile) continue;
            uint32_t byte;
            const uint4 codes = round32_block(v[i], byte);
            store_line(tile, rr, group, r0 + rr < rows, last_half, byte, codes);
        }
    }
    __syncthreads();
    const int group_t = (int)((r0 / kBothSide) & 1);
    const bool last_half_t = group_t == 0 && r0 + kBothSide >= rows;
    uint8_t *tile_t = job.out_t + ((c0 / kMxTileRows) * tiles_ct + r0 / kMxTileCols) * kMxTileBytes;
    for (int col = threadIdx.x >> 2; col < kRowWords; col += kBothThreads / 4) {     // a word: one column, or a pair
        uint32_t w[32];
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            w[k] = *word_at(blk * 32 + k, col);
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
            for (int h = 0; h < kColumns; ++h) codes[h][q] = byte[h] == 255u ? 0u : mx_codes8(p[h]);
        }
#pragma unroll
        for (int h = 0; h < kColumns; ++h) {
            const int cc = kColumns * col + h;
            store_line(tile_t, cc, group_t, c0 + cc < cols, last_half_t, byte[h], make_uint4(codes[h][0], codes[h][1], codes[h][2], codes[h][3]));
        }
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

// A warp reads 256 columns of kReadRows rows, a lane the 8 values of one 4-byte word of each.  16384 x 4096 to bfloat16
// in 31 us (5.5 TB/s), binary16 31, binary32 75 (4.1).
constexpr int kReadRows = 8;
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) dequantize_kernel(const uint8_t *__restrict__ in, long long rows, long long cols,
                                                                    T *__restrict__ out, long long ld, bool vec)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long tile_c = blockIdx.x, tiles_c = gridDim.x;
    const long long c = tile_c * kMxTileCols + lane * 8;
    const long long r0 = ((long long)blockIdx.y * kRowWarps + warp) * kReadRows;
    __shared__ __align__(16) float turn[kRowWarps][kMxTileCols];       // a row, for stores of neighbours where rows are not aligned
    if (r0 >= rows || (vec && c >= cols)) return;
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
        } else if (vec) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c + k < cols) dst[k] = from_f32<T>(v[k]);
        } else {
            *reinterpret_cast<float4 *>(&turn[warp][lane * 8]) = make_float4(v[0], v[1], v[2], v[3]);
            *reinterpret_cast<float4 *>(&turn[warp][lane * 8 + 4]) = make_float4(v[4], v[5], v[6], v[7]);
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (c - lane * 8 + k * 32 + lane < cols) dst[k * 32 - lane * 7] = from_f32<T>(turn[warp][k * 32 + lane]);
            __syncwarp();
        }
    }
}

bool rows_vectorised(const void *p, int dtype, size_t ld) { return aligned16(p) && ld * dtype_bytes(dtype) % 16 == 0; }

}  // namespace

zoa_status mx4_check_source(const char *me, const void *x, int dtype, size_t rows, size_t cols, size_t ld, const void *out, const void *out_t)
{
    if (!dtype_ok(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, dtype);
    if (rows > kMxMaxSide || cols > kMxMaxSide) return ops_fail(ZOA_ERR_ARG, "%s: rows and cols must be at most 2^30", me);
    if (rows == 0 || cols == 0) return ZOA_OK;
    if (!x || (!out && !out_t)) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    if (ld < cols) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least cols", me);
    if (reinterpret_cast<uintptr_t>(x) % dtype_bytes(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: x is not aligned to its element type", me);
    if (!aligned16(out) || !aligned16(out_t)) return ops_fail(ZOA_ERR_ARG, "%s: out and out_t must be 16-byte aligned", me);
    if (out_t && mx_tiles((long long)rows, kBothSide) * mx_tiles((long long)cols, kBothSide) > (1ll << 30))
        return ops_fail(ZOA_ERR_ARG, "%s: at most 2^44 elements when out_t is asked for", me);
    return ZOA_OK;
}

BothJob mx4_both_job(const void *x, int dtype, size_t rows, size_t cols, size_t ld, void *out, void *out_t)
{
    return BothJob{x, static_cast<uint8_t *>(out), static_cast<uint8_t *>(out_t), (long long)rows, (long long)cols, (long long)ld,
                   (int)rows_vectorised(x, dtype, ld)};
}

zoa_status mx4_launch_both(const char *me, int dtype, const BothJob &a, const BothJob &b, cudaStream_t s)
{
    const long long of_a = mx_tiles(a.rows, kBothSide) * mx_tiles(a.cols, kBothSide), of_b = mx_tiles(b.rows, kBothSide) * mx_tiles(b.cols, kBothSide);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        constexpr int kSmem = kBothSide * kBothPitch<T> * 4;
        static SmemLimit limit;
        if (limit.ensure(quantize_both_kernel<T>, kSmem) != cudaSuccess) return;   // the launch below reports it
        quantize_both_kernel<T><<<(unsigned)(of_a + of_b), kBothThreads, kSmem, s>>>(a, b, (unsigned)of_a);
    });
    return ops_launched(me);
}

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
    if (ops_gave_up()) return ops_refuse(me);
    const zoa_status st = mx4_check_source(me, x, dtype, rows, cols, ld, out, out_t);
    if (st != ZOA_OK || rows == 0 || cols == 0) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (out_t) return mx4_launch_both(me, dtype, mx4_both_job(x, dtype, rows, cols, ld, out, out_t), BothJob{}, s);
    const bool vec = rows_vectorised(x, dtype, ld);
    const long long R = (long long)rows, C = (long long)cols;
    const long long blocks = mx_tiles(mx_tiles(R, kRowsPerWarp) * mx_tiles(C, kMxTileCols), kRowWarps), most = 4ll * ops_sm_count();
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        const unsigned grid = (unsigned)(blocks < most ? blocks : most);
        uint8_t *to = static_cast<uint8_t *>(out);
        if constexpr (sizeof(T) == 4) quantize_rows_f32_kernel<<<grid, kRowWarps * 32, 0, s>>>(static_cast<const T *>(x), R, C, (long long)ld, vec, to);
        else quantize_rows_kernel<T><<<grid, kRowWarps * 32, 0, s>>>(static_cast<const T *>(x), R, C, (long long)ld, vec, to);
    });
    return ops_launched(me);
}

extern "C" zoa_status zoa_mx4_dequantize(const void *q, size_t rows, size_t cols, void *out, int dtype, size_t ld, void *stream)
{
    const char *me = "zoa_mx4_dequantize";
    if (ops_gave_up()) return ops_refuse(me);
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
