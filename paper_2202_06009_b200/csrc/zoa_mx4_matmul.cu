// Products of 4-bit microscaled matrices on the tensor cores: C[i, j] = sum_k A[i, k] B[j, k], both operands in the
// tiles of zoa_mx4.cuh, sums in binary32.
#include "zoa_async.cuh"
#include "zoa_mx4.cuh"

namespace zoa {
namespace {

// ---- tensor core ------------------------------------------------------------------------------------------
// Shared-memory operand descriptors.  Codes: K-major, 128-byte swizzle, 8-row groups 1024 bytes apart.  Scales: no
// swizzle, groups of 8 rows x 16 bytes 128 bytes apart.
__device__ __forceinline__ uint64_t codes_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | (64ull << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ uint64_t scales_desc(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFF) >> 4) | (1ull << 16) | (8ull << 32) | (1ull << 46);
}
// Instruction descriptor: E2M1 operands, K-major both, E8M0 scales, M x N; `id` names the pair of scale bytes of a
// 32-bit scale word that this step of 64 columns uses (0: bytes 0 and 1, 2: bytes 2 and 3).
__host__ __device__ constexpr uint32_t mma_desc(int m, int n, uint32_t id)
{
    return (id << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) | (1u << 23) | ((uint32_t)(m >> 4) << 24) | (id << 29);
}
__device__ __forceinline__ void mma_mx4(uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t sfa, uint32_t sfb, bool accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.u32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate)
        : "memory");
}
// 32 rows x 16 bytes of scales to four columns of tensor memory, repeated for the four groups of 32 lanes.
__device__ __forceinline__ void copy_scales(uint32_t tmem, uint64_t desc)
{
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(tmem), "l"(desc) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void load_columns32(uint32_t tmem, uint32_t *v)
{
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]),
          "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]),
          "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]),
          "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(tmem));
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
}

struct MatmulArgs {
    const uint8_t *a, *b;     // tiles
    void *out;
    long long m, n, ld;
    int tiles_k;              // tiles of 256 columns
    int vec;                  // rows of `out` are 16-byte aligned
    int test_stop;            // > 0: the copies stop after this many tiles (error-path test)
    WaitLimit limit;
};

constexpr int kStages = 6;
constexpr int kStageBytes = 2 * kMxTileBytes;
constexpr int kTmemColumns = 256;                    // 128 of sums, then 16 of scales per stage
constexpr int kScaleColumns = 16;
struct MatmulShared {
    unsigned long long full[kStages], empty[kStages], done;
    uint32_t tmem;
    int gave_up;
};
constexpr int kMatmulSmem = kStages * kStageBytes + 1024 + (int)sizeof(MatmulShared);

template <typename T>
__device__ __forceinline__ void store32(T *row, long long j, long long n, bool vec, const uint32_t *w)
{
    float v[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) v[k] = __uint_as_float(w[k]);
    if (vec && j + 32 <= n) {
#pragma unroll
        for (int k = 0; k < 32; k += Vec<T>::kElems) *reinterpret_cast<uint4 *>(row + j + k) = Vec<T>::pack(v + k);
        return;
    }
#pragma unroll
    for (int k = 0; k < 32; ++k)
        if (j + k < n) row[j + k] = from_f32<T>(v[k]);
}

// One block computes 128 x 128 of C.  Warp 0 copies tiles into the ring, warp 1 issues the tensor core's work,
// warps 2 to 5 store the result.
template <typename T>
__global__ void __launch_bounds__(192) matmul_kernel(const MatmulArgs g)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    MatmulShared *sh = reinterpret_cast<MatmulShared *>(ring + kStages * kStageBytes);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int issued = 0;           // tiles whose copies thread 0 has started
    const long long i0 = (long long)blockIdx.x * 128, j0 = (long long)blockIdx.y * 128;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&sh->full[s]), 1);
            mbar_init(smem_addr(&sh->empty[s]), 1);
        }
        mbar_init(smem_addr(&sh->done), 1);
        sh->gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh->tmem)), "r"(kTmemColumns)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = sh->tmem;
    volatile int *gave_up = &sh->gave_up;

    if (warp == 0 && lane == 0) {
        const uint32_t bytes_a = kMxScaleBytes + 128 * (uint32_t)(g.m - i0 < 128 ? g.m - i0 : 128);
        const uint32_t bytes_b = kMxScaleBytes + 128 * (uint32_t)(g.n - j0 < 128 ? g.n - j0 : 128);
        const uint8_t *a = g.a + (long long)blockIdx.x * g.tiles_k * kMxTileBytes;
        const uint8_t *b = g.b + (long long)blockIdx.y * g.tiles_k * kMxTileBytes;
        for (int k = 0; k < g.tiles_k; ++k) {
            const int s = k % kStages;
            if (g.test_stop > 0 && k >= g.test_stop) break;
            if (!mbar_wait(smem_addr(&sh->empty[s]), (uint32_t)(k / kStages & 1) ^ 1u, gave_up, g.limit)) break;
            const uint32_t full = smem_addr(&sh->full[s]), dst = smem_addr(ring + s * kStageBytes);
            mbar_expect(full, bytes_a + bytes_b);
            bulk_load(dst, a + (long long)k * kMxTileBytes, bytes_a, full);
            bulk_load(dst + kMxTileBytes, b + (long long)k * kMxTileBytes, bytes_b, full);
            ++issued;
        }
    } else if (warp == 1 && lane == 0) {
        for (int k = 0; k < g.tiles_k; ++k) {
            const int s = k % kStages;
            if (!mbar_wait(smem_addr(&sh->full[s]), (uint32_t)(k / kStages & 1), gave_up, g.limit)) break;
            const uint32_t base_a = smem_addr(ring + s * kStageBytes), base_b = base_a + kMxTileBytes;
            const uint32_t sf = tmem + 128 + s * kScaleColumns;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                copy_scales(sf + h * 4, scales_desc(base_a + h * 512));
                copy_scales(sf + 8 + h * 4, scales_desc(base_b + h * 512));
            }
            const uint64_t da = codes_desc(base_a + kMxScaleBytes), db = codes_desc(base_b + kMxScaleBytes);
#pragma unroll
            for (int q = 0; q < 4; ++q)      // 64 columns a step: 32 bytes of a 128-byte line
                mma_mx4(tmem, da + 2 * q, db + 2 * q, q & 1 ? mma_desc(128, 128, 2) : mma_desc(128, 128, 0), sf + (q >> 1) * 4,
                        sf + 8 + (q >> 1) * 4, k > 0 || q > 0);
            commit(smem_addr(&sh->empty[s]));
        }
        commit(smem_addr(&sh->done));
    }
    __syncwarp();
    const bool finished = mbar_wait(smem_addr(&sh->done), 0, gave_up, g.limit);
    if (threadIdx.x == 0 && *gave_up) {      // copies in flight land before the block's shared memory is released
        for (int q = issued > kStages ? issued - kStages : 0; q < issued; ++q)
            mbar_drain(smem_addr(&sh->full[q % kStages]), (uint32_t)(q / kStages & 1), g.limit);
    }
    if (warp >= 2 && finished && !*gave_up) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int quarter = warp & 3;
        const long long i = i0 + quarter * 32 + lane;
        T *row = static_cast<T *>(g.out) + i * g.ld;
        for (int c = 0; c < 128; c += 32) {
            if (j0 + c >= g.n) break;
            uint32_t v[32];
            load_columns32(tmem + ((uint32_t)(quarter * 32) << 16) + c, v);
            if (i < g.m) store32(row, j0 + c, g.n, g.vec, v);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemColumns) : "memory");
    }
}

zoa_status check_matrix(const char *me, const char *name, const void *p)
{
    if (!p) return ops_fail(ZOA_ERR_ARG, "%s: %s is NULL", me, name);
    if (!aligned16(p)) return ops_fail(ZOA_ERR_ARG, "%s: %s must be 16-byte aligned", me, name);
    return ZOA_OK;
}

}  // namespace
}  // namespace zoa

using namespace zoa;

extern "C" zoa_status zoa_mx4_matmul(const void *a, const void *b, size_t m, size_t n, size_t k, void *out, int dtype, size_t ld,
                                     void *stream)
{
    const char *me = "zoa_mx4_matmul";
    if (!dtype_ok(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, dtype);
    if (m > kMxMaxSide || n > kMxMaxSide || k > kMxMaxSide) return ops_fail(ZOA_ERR_ARG, "%s: m, n and k must be at most 2^30", me);
    if (m == 0 || n == 0) return ZOA_OK;
    if (!out) return ops_fail(ZOA_ERR_ARG, "%s: out is NULL", me);
    if (ld < n) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least n", me);
    if (reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: out is not aligned to its element type", me);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (k == 0) {      // an empty sum
        if (cudaMemset2DAsync(out, ld * dtype_bytes(dtype), 0, n * dtype_bytes(dtype), m, s) != cudaSuccess) return ops_launched(me);
        return ZOA_OK;
    }
    zoa_status st = check_matrix(me, "a", a);
    if (st == ZOA_OK) st = check_matrix(me, "b", b);
    if (st != ZOA_OK) return st;
    MatmulArgs g{};
    g.a = static_cast<const uint8_t *>(a);
    g.b = static_cast<const uint8_t *>(b);
    g.out = out;
    g.m = (long long)m;
    g.n = (long long)n;
    g.ld = (long long)ld;
    g.tiles_k = (int)mx_tiles((long long)k, kMxTileCols);
    g.vec = aligned16(out) && ld * dtype_bytes(dtype) % 16 == 0;
    g.test_stop = ops_test_stop();
    g.limit.error_word = ops_error_word();
    g.limit.ns = ops_wait_limit_ns();
    if (!g.limit.error_word) return ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        static SmemLimit limit;
        if (limit.ensure(matmul_kernel<T>, kMatmulSmem) != cudaSuccess) return;
        matmul_kernel<T><<<dim3((unsigned)mx_tiles(g.m, 128), (unsigned)mx_tiles(g.n, 128)), 192, kMatmulSmem, s>>>(g);
    });
    return ops_launched(me);
}

extern "C" size_t zoa_mx4_linear_work(size_t m, size_t n, size_t k)
{
    (void)n;
    return zoa_mx4_size(m, k);
}

extern "C" zoa_status zoa_mx4_linear(const void *x, int dtype, size_t m, size_t k, size_t ldx, const void *b, size_t n, void *out,
                                     size_t ld, void *work, void *stream)
{
    if (m && n && k && zoa_mx4_linear_work(m, n, k) && !work) return ops_fail(ZOA_ERR_ARG, "zoa_mx4_linear: work is NULL");
    const zoa_status st = zoa_mx4_quantize(x, dtype, m, k, ldx, work, nullptr, stream);
    return st != ZOA_OK ? st : zoa_mx4_matmul(work, b, m, n, k, out, dtype, ld, stream);
}

extern "C" zoa_status zoa_mx4_linear_forward(const void *x, int x_type, size_t ldx, const void *w, int w_type, size_t ldw, size_t m,
                                             size_t n, size_t k, void *y, size_t ldy, void *xt, void *wt, void *work, void *stream)
{
    const char *me = "zoa_mx4_linear_forward";
    if (m && n && k && (!xt || !wt || !work)) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    void *wq = static_cast<unsigned char *>(work) + zoa_mx4_size(m, k);
    zoa_status st = zoa_mx4_quantize(x, x_type, m, k, ldx, work, xt, stream);
    if (st == ZOA_OK) st = zoa_mx4_quantize(w, w_type, n, k, ldw, wq, wt, stream);
    return st != ZOA_OK ? st : zoa_mx4_matmul(work, wq, m, n, k, y, x_type, ldy, stream);
}

extern "C" zoa_status zoa_mx4_linear_backward(const void *dy, int dy_type, size_t ld_dy, size_t m, size_t n, size_t k, const void *xt,
                                              const void *wt, void *dx, int dx_type, size_t ld_dx, void *dw, int dw_type, size_t ld_dw,
                                              void *work, void *stream)
{
    const char *me = "zoa_mx4_linear_backward";
    if (!dx && !dw) return ops_fail(ZOA_ERR_ARG, "%s: neither dx nor dw is asked for", me);
    if (m && n && !work) return ops_fail(ZOA_ERR_ARG, "%s: work is NULL", me);
    void *dyt = static_cast<unsigned char *>(work) + zoa_mx4_size(m, n);
    zoa_status st = zoa_mx4_quantize(dy, dy_type, m, n, ld_dy, dx ? work : nullptr, dw ? dyt : nullptr, stream);
    if (st == ZOA_OK && dx) st = zoa_mx4_matmul(work, wt, m, k, n, dx, dx_type, ld_dx, stream);
    if (st == ZOA_OK && dw) st = zoa_mx4_matmul(dyt, xt, n, k, m, dw, dw_type, ld_dw, stream);
    return st;
}
