// Rounding to 4-bit microscaled form (along the rows, along the columns, or both from one read) and reading back.
#include "zoa_mx4.cuh"

namespace zoa {
namespace {

constexpr int kRowWarps = 8;      // warps of a block of quantize_rows_kernel
constexpr int kRowsPerWarp = 4;   // rows whose loads a warp has in flight at once

// Eight neighbours of a row as binary32; columns past `cols` are 0.
template <typename T>
__device__ __forceinline__ void load8(const T *row, long long c, long long cols, bool vec, float *v)
{
    if (vec && c + 8 <= cols) {
        if constexpr (sizeof(T) == 4) {
            Vec<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(row + c)), v);
            Vec<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(row + c + 4)), v + 4);
        } else {
            Vec<T>::unpack(__ldg(reinterpret_cast<const uint4 *>(row + c)), v);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = c + k < cols ? to_f32(row[c + k]) : 0.0f;
}

// The 4-byte scale words of a row's two groups of 128 columns, from the scale byte that every lane of block
// lane / 4 holds: complete in lanes 0 and 16.
__device__ __forceinline__ uint32_t gather_scales(uint32_t byte, int lane)
{
    uint32_t w = byte << (8 * ((lane >> 2) & 3));
    w |= __shfl_xor_sync(0xffffffffu, w, 4);
    w |= __shfl_xor_sync(0xffffffffu, w, 8);
    return w;
}

// One warp takes 256 columns (a line of a tile) of kRowsPerWarp rows, a lane 8 neighbours: a block is four lanes.
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) quantize_rows_kernel(const T *__restrict__ x, long long rows, long long cols,
                                                                       long long ld, bool vec, uint8_t *__restrict__ out)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long tile_c = blockIdx.x, tiles_c = gridDim.x;
    const long long c = tile_c * kMxTileCols + lane * 8;
    const long long r0 = ((long long)blockIdx.y * kRowWarps + warp) * kRowsPerWarp;
    float v[kRowsPerWarp][8];
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i)
        if (r0 + i < rows) load8(x + (r0 + i) * ld, c, cols, vec, v[i]);
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
        const long long r = r0 + i;
        if (r >= rows) return;
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) most = max(most, mx_abs_bits(v[i][k]));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const uint32_t byte = mx_scale_byte(__uint_as_float(most));
        const uint32_t codes = byte == 255u ? 0u : mx_codes8(v[i], mx_inverse(byte));
        const uint32_t scales = gather_scales(byte, lane);
        uint8_t *tile = out + ((r / kMxTileRows) * tiles_c + tile_c) * kMxTileBytes;
        const int rr = (int)(r % kMxTileRows);
        *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, lane >> 2) + (lane & 3) * 4) = codes;
        if ((lane & 15) == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, lane >> 2)) = scales;
    }
}

// One block takes 128 x 128 elements: rounds them along the rows as it loads them, keeps them in shared memory
// and rounds them along the columns (the rows of the transposed matrix) from there.
constexpr int kBothThreads = 256;
constexpr int kBothSide = 128;
template <typename T>
__global__ void __launch_bounds__(kBothThreads) quantize_both_kernel(const T *__restrict__ x, long long rows, long long cols,
                                                                     long long ld, bool vec, uint8_t *__restrict__ out,
                                                                     uint8_t *__restrict__ out_t)
{
    extern __shared__ __align__(16) unsigned char both_smem[];
    T *tile_s = reinterpret_cast<T *>(both_smem);   // [128][128]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long c0 = (long long)blockIdx.x * kBothSide, r0 = (long long)blockIdx.y * kBothSide;
    const long long tiles_c = mx_tiles(cols, kMxTileCols), tiles_ct = mx_tiles(rows, kMxTileCols);
    const int half = lane >> 4, l16 = lane & 15;
    const int group = (int)((c0 / kBothSide) & 1);                      // which half of a tile's columns
    uint8_t *tile = out ? out + ((r0 / kMxTileRows) * tiles_c + c0 / kMxTileCols) * kMxTileBytes : nullptr;

    // A half warp holds 128 columns of a row.
#pragma unroll
    for (int i = 0; i < kBothSide / 16; ++i) {
        const int rr = (warp * (kBothSide / 16) + i) * 2 + half;
        float v[8];
        if (r0 + rr < rows) {
            load8(x + (r0 + rr) * ld, c0 + l16 * 8, cols, vec, v);
        } else {
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = 0.0f;
        }
        T *keep = tile_s + rr * kBothSide + l16 * 8;
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<uint4 *>(keep) = Vec<T>::pack(v);
            *reinterpret_cast<uint4 *>(keep + 4) = Vec<T>::pack(v + 4);
        } else {
            *reinterpret_cast<uint4 *>(keep) = Vec<T>::pack(v);
        }
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) most = max(most, mx_abs_bits(v[k]));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
        most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
        const uint32_t byte = mx_scale_byte(__uint_as_float(most));
        const uint32_t codes = byte == 255u ? 0u : mx_codes8(v, mx_inverse(byte));
        const uint32_t scales = gather_scales(byte, lane);
        if (tile && r0 + rr < rows) {
            const int block = group * 4 + (l16 >> 2);
            *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, block) + (l16 & 3) * 4) = codes;
            if (l16 == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, group * 4)) = scales;
        }
        // The last group of a row that ends in a tile's first half also clears the second half.
        if (tile && r0 + rr < rows && group == 0 && c0 + kBothSide >= cols) {
            *reinterpret_cast<uint32_t *>(tile + mx_code_at(rr, 4 + (l16 >> 2)) + (l16 & 3) * 4) = 0u;
            if (l16 == 0) *reinterpret_cast<uint32_t *>(tile + mx_scale_at(rr, 4)) = 0u;
        }
    }
    __syncthreads();
    // A thread takes the 32 rows of one block of one column.
    const int group_t = (int)((r0 / kBothSide) & 1);
    uint8_t *tile_t = out_t + ((c0 / kMxTileRows) * tiles_ct + r0 / kMxTileCols) * kMxTileBytes;
    for (int item = threadIdx.x; item < kBothSide * 4; item += kBothThreads) {
        const int cc = item & (kBothSide - 1), blk = item / kBothSide;
        if (c0 + cc >= cols) continue;
        float v[32];
        uint32_t most = 0;
#pragma unroll
        for (int k = 0; k < 32; ++k) {
            v[k] = to_f32(tile_s[(blk * 32 + k) * kBothSide + cc]);
            most = max(most, mx_abs_bits(v[k]));
        }
        const uint32_t byte = mx_scale_byte(__uint_as_float(most));
        const float inv = mx_inverse(byte);
        uint4 codes = make_uint4(0, 0, 0, 0);
        if (byte != 255u) codes = make_uint4(mx_codes8(v, inv), mx_codes8(v + 8, inv), mx_codes8(v + 16, inv), mx_codes8(v + 24, inv));
        *reinterpret_cast<uint4 *>(tile_t + mx_code_at(cc, group_t * 4 + blk)) = codes;
        tile_t[mx_scale_at(cc, group_t * 4 + blk)] = (uint8_t)byte;
        if (group_t == 0 && r0 + kBothSide >= rows) {
            *reinterpret_cast<uint4 *>(tile_t + mx_code_at(cc, 4 + blk)) = make_uint4(0, 0, 0, 0);
            tile_t[mx_scale_at(cc, 4 + blk)] = 0;
        }
    }
}

// A warp reads 256 columns of a row, a lane the 8 values of one 4-byte word.
template <typename T>
__global__ void __launch_bounds__(kRowWarps * 32) dequantize_kernel(const uint8_t *__restrict__ in, long long rows, long long cols,
                                                                    T *__restrict__ out, long long ld, bool vec)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long tile_c = blockIdx.x, tiles_c = gridDim.x;
    const long long c = tile_c * kMxTileCols + lane * 8;
    const long long r0 = ((long long)blockIdx.y * kRowWarps + warp) * kRowsPerWarp;
    if (c >= cols) return;
    uint32_t codes[kRowsPerWarp];
    uint32_t bytes[kRowsPerWarp];
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
        const long long r = r0 + i;
        if (r >= rows) break;
        const uint8_t *tile = in + ((r / kMxTileRows) * tiles_c + tile_c) * kMxTileBytes;
        const int rr = (int)(r % kMxTileRows);
        codes[i] = __ldg(reinterpret_cast<const uint32_t *>(tile + mx_code_at(rr, lane >> 2) + (lane & 3) * 4));
        bytes[i] = __ldg(tile + mx_scale_at(rr, lane >> 2));
    }
#pragma unroll
    for (int i = 0; i < kRowsPerWarp; ++i) {
        const long long r = r0 + i;
        if (r >= rows) break;
        const float s = mx_scale(bytes[i]);
        float v[8];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t h2;
            asm("{\n\t.reg .b8 lo, hi;\n\t.reg .b16 t;\n\tcvt.u16.u32 t, %1;\n\tmov.b16 {lo, hi}, t;\n\tcvt.rn.f16x2.e2m1x2 %0, lo;\n\t}"
                : "=r"(h2)
                : "r"(codes[i] >> (8 * k)));
            float lo, hi;
            unpack2<__half>(h2, lo, hi);
            v[2 * k] = lo * s;
            v[2 * k + 1] = hi * s;
        }
        T *dst = out + r * ld + c;
        if (vec && c + 8 <= cols) {
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
    zoa_status st = ZOA_OK;
    if (!out_t) {
        const long long per = kRowWarps * kRowsPerWarp, gy = mx_tiles(R, per);
        // gridDim.y holds 65535 blocks: a larger matrix takes several launches, whole row tiles each.
        for (long long y = 0; y < gy && st == ZOA_OK; y += 65532) {
            const long long n = gy - y < 65532 ? gy - y : 65532, r = y * per;
            with_type(dtype, [&](auto t) {
                using T = decltype(t);
                quantize_rows_kernel<T><<<dim3((unsigned)mx_tiles(C, kMxTileCols), (unsigned)n), kRowWarps * 32, 0, s>>>(
                    static_cast<const T *>(x) + r * L, R - r, C, L, vec,
                    static_cast<uint8_t *>(out) + r / kMxTileRows * mx_tiles(C, kMxTileCols) * kMxTileBytes);
            });
            st = ops_launched(me);
        }
        return st;
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
    const long long R = (long long)rows, C = (long long)cols, L = (long long)ld, per = kRowWarps * kRowsPerWarp, gy = mx_tiles(R, per);
    zoa_status st = ZOA_OK;
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
