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
// These are called by whole warps and issued by the thread whose `one` is set (elect_one): a branch around them would
// keep the compiler from holding their operands in uniform registers, which cost 60 to 90 cycles an instruction.
__device__ __forceinline__ uint32_t elect_one()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one;
}
#define ZOA_MMA_MX4(group)                                                                                                \
    asm volatile(                                                                                                         \
        "{\n\t.reg .pred p, q;\n\t"                                                                                       \
        "setp.ne.u32 p, %6, 0;\n\t"                                                                                       \
        "setp.ne.u32 q, %7, 0;\n\t"                                                                                       \
        "@q tcgen05.mma.cta_group::" #group ".kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" \
        ::"r"(d), "l"(a), "l"(b), "r"(desc), "r"(sfa), "r"(sfb), "r"((uint32_t)accumulate), "r"(one)                      \
        : "memory")
// kPair: the tensor cores of two SMs on one tile, issued by the first block of the cluster for both.
template <bool kPair = false>
__device__ __forceinline__ void mma_mx4(uint32_t one, uint32_t d, uint64_t a, uint64_t b, uint32_t desc, uint32_t sfa, uint32_t sfb,
                                        bool accumulate)
{
    if constexpr (kPair) ZOA_MMA_MX4(2);
    else ZOA_MMA_MX4(1);
}
// 32 rows x 16 bytes of scales to four columns of tensor memory, repeated for the four groups of 32 lanes.
#define ZOA_IF_ONE(instruction) "{\n\t.reg .pred q;\n\tsetp.ne.u32 q, %0, 0;\n\t@q " instruction "\n\t}"
template <bool kPair = false>
__device__ __forceinline__ void copy_scales(uint32_t one, uint32_t tmem, uint64_t desc)
{
    if constexpr (kPair) asm volatile(ZOA_IF_ONE("tcgen05.cp.cta_group::2.32x128b.warpx4 [%1], %2;") ::"r"(one), "r"(tmem), "l"(desc) : "memory");
    else asm volatile(ZOA_IF_ONE("tcgen05.cp.cta_group::1.32x128b.warpx4 [%1], %2;") ::"r"(one), "r"(tmem), "l"(desc) : "memory");
}
// The work issued so far arrives on the barrier when it is done; of a pair, at the same place in both blocks.
__device__ __forceinline__ void commit(uint32_t one, uint32_t bar)
{
    asm volatile(ZOA_IF_ONE("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%1];") ::"r"(one), "r"(bar) : "memory");
}
__device__ __forceinline__ void commit_pair(uint32_t one, uint32_t bar)
{
    asm volatile(ZOA_IF_ONE("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%1], %2;") ::"r"(one),
                 "r"(bar), "h"((uint16_t)3)
                 : "memory");
}
__device__ __forceinline__ void expect_one(uint32_t one, uint32_t bar, uint32_t bytes)
{
    asm volatile(ZOA_IF_ONE("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%1], %2;") ::"r"(one), "r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_load_one(uint32_t one, uint32_t dst, const void *src, uint32_t bytes, uint32_t bar)
{
    asm volatile(ZOA_IF_ONE("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%1], [%2], %3, [%4];") ::"r"(one), "r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
// A bounded wait of a whole warp.
template <bool kCluster = false>
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *gave_up, const WaitLimit &limit)
{
    return __all_sync(0xffffffffu, mbar_wait<kCluster>(bar, parity, gave_up, limit));
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
}
__device__ __forceinline__ void store_columns8(uint32_t tmem, const uint32_t *v)
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(tmem), "r"(v[0]), "r"(v[1]), "r"(v[2]),
                 "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ __forceinline__ void columns_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void columns_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

struct MatmulArgs {
    const uint8_t *a, *b;     // tiles
    void *out;
    long long m, n, ld;
    int tiles_k;              // tiles of 256 columns
    int k_steps;              // steps of 64 columns, the last one perhaps partly zeros
    int vec;                  // rows of `out` are 16-byte (1) or 32-byte (2) aligned
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
    const int warp = (int)__reduce_max_sync(0xffffffffu, threadIdx.x >> 5), lane = threadIdx.x & 31;
    int issued = 0;           // tiles whose copies warp 0 has started
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
    const uint32_t tmem = __reduce_or_sync(0xffffffffu, sh->tmem);       // a uniform register
    volatile int *gave_up = &sh->gave_up;

    if (warp == 0) {
        const uint32_t one = elect_one();
        const uint32_t bytes_a = kMxScaleBytes + 128 * (uint32_t)(g.m - i0 < 128 ? g.m - i0 : 128);
        const uint32_t bytes_b = kMxScaleBytes + 128 * (uint32_t)(g.n - j0 < 128 ? g.n - j0 : 128);
        const uint8_t *a = g.a + (long long)blockIdx.x * g.tiles_k * kMxTileBytes;
        const uint8_t *b = g.b + (long long)blockIdx.y * g.tiles_k * kMxTileBytes;
        for (int k = 0; k < g.tiles_k; ++k) {
            const int s = k % kStages;
            if (g.test_stop > 0 && k >= g.test_stop) break;
            if (!warp_wait(smem_addr(&sh->empty[s]), (uint32_t)(k / kStages & 1) ^ 1u, gave_up, g.limit)) break;
            const uint32_t full = smem_addr(&sh->full[s]), dst = smem_addr(ring + s * kStageBytes);
            expect_one(one, full, bytes_a + bytes_b);
            bulk_load_one(one, dst, a + (long long)k * kMxTileBytes, bytes_a, full);
            bulk_load_one(one, dst + kMxTileBytes, b + (long long)k * kMxTileBytes, bytes_b, full);
            ++issued;
        }
    } else if (warp == 1) {
        const uint32_t one = elect_one();
        for (int k = 0; k < g.tiles_k; ++k) {
            const int s = k % kStages;
            if (!warp_wait(smem_addr(&sh->full[s]), (uint32_t)(k / kStages & 1), gave_up, g.limit)) break;
            const uint32_t base_a = smem_addr(ring + s * kStageBytes), base_b = base_a + kMxTileBytes;
            const uint32_t sf = tmem + 128 + s * kScaleColumns;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                copy_scales(one, sf + h * 4, scales_desc(base_a + h * 512));
                copy_scales(one, sf + 8 + h * 4, scales_desc(base_b + h * 512));
            }
            const uint64_t da = codes_desc(base_a + kMxScaleBytes), db = codes_desc(base_b + kMxScaleBytes);
#pragma unroll
            for (int q = 0; q < 4; ++q)      // 64 columns a step: 32 bytes of a 128-byte line
                mma_mx4(one, tmem, da + 2 * q, db + 2 * q, q & 1 ? mma_desc(128, 128, 2) : mma_desc(128, 128, 0), sf + (q >> 1) * 4,
                        sf + 8 + (q >> 1) * 4, k > 0 || q > 0);
            commit(one, smem_addr(&sh->empty[s]));
        }
        commit(one, smem_addr(&sh->done));
    }
    __syncwarp();
    const bool finished = mbar_wait(smem_addr(&sh->done), 0, gave_up, g.limit);
    if (warp == 0 && *gave_up) {      // copies in flight land before the block's shared memory is released
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
            columns_loaded();
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

// ---- pairs of SMs, large products --------------------------------------------------------------------------
// A cluster of two blocks computes 256 x 256 of C at a time, each block the sums of 128 rows, and walks over the tiles
// with a stride.  Every byte of A goes to one SM and every byte of B's codes too (the tensor cores read the partner's
// half from its shared memory); only B's scales go to both.  The sums fill half of tensor memory; the scales of the
// stages in flight take the rest, so the next tile starts when the sums have been taken to registers, not when they
// have been stored.
constexpr int kPairStages = 6;
constexpr int kPairStageBytes = kMxTileBytes + 2 * kMxScaleBytes + kMxCodeBytes;    // A tile; B scales of both halves; B codes
constexpr int kPairScaleColumns = 24;                                              // 8 for A, 16 for B
constexpr int kPairThreads = 448;
struct PairShared {
    unsigned long long full[kPairStages], scaled[kPairStages], empty[kPairStages], sums_full, sums_empty, finished;
    uint32_t tmem;
    int gave_up;
};
constexpr int kPairSmem = kPairStages * kPairStageBytes + 1024 + (int)sizeof(PairShared);

struct PairTile {
    long long i0;        // this block's first row of A
    long long j0;        // the pair's first row of B
    int rows, cols;      // this block's rows that exist (0..128); the pair's columns, a multiple of 32
};
__device__ __forceinline__ PairTile pair_tile(const MatmulArgs &g, long long t, int rank)
{
    // Tiles go down strips 8 tiles wide, so that the tiles in flight share rows of both operands.
    const long long tiles_m = (g.m + 255) / 256, tiles_n = (g.n + 255) / 256;
    const long long strip = t / (tiles_m * 8), first = strip * 8, width = tiles_n - first < 8 ? tiles_n - first : 8;
    const long long in = t - strip * tiles_m * 8;
    PairTile p;
    p.i0 = in / width * 256 + rank * 128;
    p.j0 = (first + in % width) * 256;
    p.rows = (int)(g.m - p.i0 < 0 ? 0 : g.m - p.i0 < 128 ? g.m - p.i0 : 128);
    p.cols = (int)(g.n - p.j0 < 256 ? (g.n - p.j0 + 31) / 32 * 32 : 256);
    return p;
}

// 32 neighbours of a row of the result, already of type T; n is the row's length.
template <typename T>
__device__ __forceinline__ void store_row32(T *row, long long j, long long n, int vec, const uint32_t *w)
{
    constexpr int kWords = 32 * (int)sizeof(T) / 4;
    if (vec && j + 32 <= n) {
        uint32_t *dst = reinterpret_cast<uint32_t *>(row + j);
        if (vec == 2) {
#pragma unroll
            for (int k = 0; k < kWords; k += 8)
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + k), "r"(w[k]), "r"(w[k + 1]), "r"(w[k + 2]),
                             "r"(w[k + 3]), "r"(w[k + 4]), "r"(w[k + 5]), "r"(w[k + 6]), "r"(w[k + 7])
                             : "memory");
        } else {
#pragma unroll
            for (int k = 0; k < kWords; k += 4) *reinterpret_cast<uint4 *>(dst + k) = make_uint4(w[k], w[k + 1], w[k + 2], w[k + 3]);
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        if (j + k >= n) continue;
        if constexpr (sizeof(T) == 4) {
            reinterpret_cast<uint32_t *>(row)[j + k] = w[k];
        } else {
            reinterpret_cast<uint16_t *>(row)[j + k] = (uint16_t)(w[k >> 1] >> (16 * (k & 1)));
        }
    }
}
// Sums as loaded from tensor memory, rounded to T (two to a word for the 16-bit types).
template <typename T>
__device__ __forceinline__ void round32(const uint32_t *v, uint32_t *w)
{
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        if constexpr (sizeof(T) == 4) w[k] = v[k];
        else if (k % 2 == 0) w[k / 2] = pack2<T>(__uint_as_float(v[k]), __uint_as_float(v[k + 1]));
    }
}

// Warp 0 copies tiles, warps 2 to 5 bring their scales to tensor memory, warp 1 of the first block issues the products,
// warps 6 to 13 take the sums: four quarters of the rows, two halves of the columns.
template <typename T>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1) matmul_pair_kernel(const MatmulArgs g, const long long tiles)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    PairShared *sh = reinterpret_cast<PairShared *>(ring + kPairStages * kPairStageBytes);
    const int warp = (int)__reduce_max_sync(0xffffffffu, threadIdx.x >> 5), lane = threadIdx.x & 31, rank = (int)cluster_rank();
    const long long first = blockIdx.x / 2, stride = gridDim.x / 2;

    if (threadIdx.x == 0) {
        for (int s = 0; s < kPairStages; ++s) {
            mbar_init(smem_addr(&sh->full[s]), 1);
            mbar_init(smem_addr(&sh->scaled[s]), 8);       // four warps of both blocks
            mbar_init(smem_addr(&sh->empty[s]), 1);
        }
        mbar_init(smem_addr(&sh->sums_full), 1);
        mbar_init(smem_addr(&sh->sums_empty), 16);
        mbar_init(smem_addr(&sh->finished), 1);
        sh->gave_up = 0;
        mbar_init_done();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_addr(&sh->tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = __reduce_or_sync(0xffffffffu, sh->tmem);       // a uniform register
    volatile int *gave_up = &sh->gave_up;

    if (warp == 0) {
        const uint32_t one = elect_one();
        int s = 0, issued = 0;
        uint32_t parity = 0;
        bool ok = true;
        for (long long t = first; t < tiles && ok; t += stride) {
            const PairTile p = pair_tile(g, t, rank);
            // B: scales of the pair's up to two tiles to both blocks, codes by halves of the pair's columns; a half may
            // begin in one tile and end in the next.  Rows past the end are neither copied nor stored.
            const long long exist = g.n - p.j0 < p.cols ? g.n - p.j0 : p.cols;
            const int half = p.cols / 2, b0 = rank * half, b1 = (int)(exist < b0 + half ? (exist > b0 ? exist : b0) : b0 + half);
            const int two = exist > 128;
            const int cut = b0 < 128 ? (b1 < 128 ? b1 : 128) : b0;      // b0 .. cut lie in the first tile, cut .. b1 in the second
            const long long next_b = (long long)g.tiles_k * kMxTileBytes;
            const uint8_t *a = g.a + p.i0 / 128 * next_b, *b = g.b + p.j0 / 128 * next_b;
            const uint32_t bytes_a = p.rows ? kMxScaleBytes + 128 * (uint32_t)p.rows : 0;
            const uint32_t bytes_1 = 128 * (uint32_t)(cut - b0), bytes_2 = 128 * (uint32_t)(b1 - cut);
            const uint32_t bytes = bytes_a + kMxScaleBytes * (1 + two) + bytes_1 + bytes_2;
            const uint8_t *b_1 = b + kMxScaleBytes + b0 * 128, *b_2 = b + next_b + kMxScaleBytes + (cut - 128) * 128;
            for (int k = 0; k < g.tiles_k; ++k) {
                ok = !(g.test_stop > 0 && issued >= g.test_stop) && warp_wait(smem_addr(&sh->empty[s]), parity ^ 1u, gave_up, g.limit);
                if (!ok) break;
                const uint32_t full = smem_addr(&sh->full[s]), dst = smem_addr(ring + s * kPairStageBytes);
                const uint32_t dst_sf = dst + kMxTileBytes, dst_b = dst_sf + 2 * kMxScaleBytes;
                expect_one(one, full, bytes);
                if (bytes_a) bulk_load_one(one, dst, a, bytes_a, full);
                if (bytes_1) bulk_load_one(one, dst_b, b_1, bytes_1, full);
                if (bytes_2) bulk_load_one(one, dst_b + bytes_1, b_2, bytes_2, full);
                bulk_load_one(one, dst_sf, b, kMxScaleBytes, full);
                if (two) bulk_load_one(one, dst_sf + kMxScaleBytes, b + next_b, kMxScaleBytes, full);
                a += kMxTileBytes;
                b += kMxTileBytes;
                b_1 += kMxTileBytes;
                b_2 += kMxTileBytes;
                ++issued;
                if (++s == kPairStages) {
                    s = 0;
                    parity ^= 1u;
                }
            }
        }
        // Everything has been read when this completes; after giving up, copies in flight land first.
        const bool done = warp_wait(smem_addr(&sh->finished), 0, gave_up, g.limit);
        if (!done || *gave_up)
            for (int q = issued > kPairStages ? issued - kPairStages : 0; q < issued; ++q)
                mbar_drain(smem_addr(&sh->full[q % kPairStages]), (uint32_t)(q / kPairStages & 1), g.limit);
    } else if (warp == 1 && rank == 0) {
        const uint32_t one = elect_one();
        int s = 0;
        uint32_t parity = 0, round = 0;
        bool ok = true;
        for (long long t = first; t < tiles && ok; t += stride, ++round) {
            const PairTile p = pair_tile(g, t, 0);
            const uint32_t desc = mma_desc(256, p.cols, 0);
            if (round > 0 && !warp_wait(smem_addr(&sh->sums_empty), (round - 1) & 1u, gave_up, g.limit)) break;
            for (int k = 0; k < g.tiles_k; ++k) {
                // both blocks' copies have landed and their scales are in tensor memory
                if (!(ok = warp_wait(smem_addr(&sh->scaled[s]), parity, gave_up, g.limit))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t base_a = smem_addr(ring + s * kPairStageBytes), base_b = base_a + kMxTileBytes + 2 * kMxScaleBytes;
                const uint32_t sf = tmem + 256 + s * kPairScaleColumns;
                const uint64_t da = codes_desc(base_a + kMxScaleBytes), db = codes_desc(base_b);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (4 * k + q < g.k_steps)
                        mma_mx4<true>(one, tmem, da + 2 * q, db + 2 * q, desc | (q & 1 ? mma_desc(0, 0, 2) : 0), sf + (q >> 1) * 4,
                                      sf + 8 + (q >> 1) * 8, k > 0 || q > 0);
                commit_pair(one, smem_addr(&sh->empty[s]));
                if (++s == kPairStages) {
                    s = 0;
                    parity ^= 1u;
                }
            }
            if (ok) commit_pair(one, smem_addr(&sh->sums_full));
        }
        commit_pair(one, smem_addr(&sh->finished));
    } else if (warp >= 2 && warp < 6) {
        // Scales to tensor memory, a warp for each quarter of its lanes.  (The tensor core can copy them itself, but it
        // does so in line with its products: six copies a stage took as long as two of its four products.)
        const int quarter = warp & 3;
        int s = 0;
        uint32_t parity = 0;
        bool ok = true;
        for (long long t = first; t < tiles && ok; t += stride)
            for (int k = 0; k < g.tiles_k; ++k) {
                if (!(ok = warp_wait(smem_addr(&sh->full[s]), parity, gave_up, g.limit))) break;
                const unsigned char *stage = ring + s * kPairStageBytes;
                const uint4 *a = reinterpret_cast<const uint4 *>(stage) + lane, *b = reinterpret_cast<const uint4 *>(stage + kMxTileBytes) + lane;
                uint32_t v[24];
                // columns: A's two groups of 128, then of B for each group its two halves
                const uint4 w[6] = {a[0], a[32], b[0], b[64], b[32], b[96]};
#pragma unroll
                for (int i = 0; i < 6; ++i) {
                    v[4 * i] = w[i].x;
                    v[4 * i + 1] = w[i].y;
                    v[4 * i + 2] = w[i].z;
                    v[4 * i + 3] = w[i].w;
                }
                const uint32_t sf = tmem + ((uint32_t)(quarter * 32) << 16) + 256 + s * kPairScaleColumns;
                store_columns8(sf, v);
                store_columns8(sf + 8, v + 8);
                store_columns8(sf + 16, v + 16);
                columns_stored();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    // The stores have been waited for, so nothing is left for a release at cluster scope to order.
                    if (rank == 0) mbar_arrive(smem_addr(&sh->scaled[s]));
                    else mbar_tell(smem_addr(&sh->scaled[s]), 0);
                }
                if (++s == kPairStages) {
                    s = 0;
                    parity ^= 1u;
                }
            }
    } else if (warp >= 6) {
        const int quarter = warp & 3, half = (warp - 6) >> 2;
        uint32_t round = 0;
        for (long long t = first; t < tiles; t += stride, ++round) {
            const PairTile p = pair_tile(g, t, rank);
            if (!__all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->sums_full), round & 1u, gave_up, g.limit))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            // Batches of columns kept for after the release, as many as the registers hold; the others are stored at once.
            constexpr int kKept = sizeof(T) == 4 ? 2 : 3;
            const int r = quarter * 32 + lane;
            T *row = static_cast<T *>(g.out) + (p.i0 + r) * g.ld;
            uint32_t w[kKept][32 * sizeof(T) / 4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t v[32];
                load_columns32(tmem + ((uint32_t)(quarter * 32) << 16) + half * 128 + c * 32, v);
                columns_loaded();
                const int at = c < 4 - kKept ? 0 : c - (4 - kKept);
                round32<T>(v, w[at]);
                if (c < 4 - kKept && r < p.rows && half * 128 + c * 32 < p.cols) store_row32<T>(row, p.j0 + half * 128 + c * 32, g.n, g.vec, w[at]);
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
            __syncwarp();
            // Nothing written here is for the partner: a release would wait for the last tile's stores.
            if (lane == 0) mbar_tell(smem_addr(&sh->sums_empty), 0);
            if (r < p.rows) {
#pragma unroll
                for (int c = 4 - kKept; c < 4; ++c)
                    if (half * 128 + c * 32 < p.cols) store_row32<T>(row, p.j0 + half * 128 + c * 32, g.n, g.vec, w[c - (4 - kKept)]);
            }
        }
    }
    __syncwarp();
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    cluster_sync();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
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
    g.k_steps = (int)mx_tiles((long long)k, 64);
    const size_t row_bytes = ld * dtype_bytes(dtype), at = reinterpret_cast<uintptr_t>(out);
    g.vec = (at | row_bytes) % 32 == 0 ? 2 : (at | row_bytes) % 16 == 0 ? 1 : 0;
    g.test_stop = ops_test_stop();
    g.limit.error_word = ops_error_word();
    g.limit.ns = ops_wait_limit_ns();
    if (!g.limit.error_word) return ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me);
    const int sms = ops_sm_count();
    if (sms < 2) return ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me);
    const long long pair_tiles = mx_tiles(g.m, 256) * mx_tiles(g.n, 256);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (pair_tiles >= sms / 2) {
            static SmemLimit limit;
            if (limit.ensure(matmul_pair_kernel<T>, kPairSmem) != cudaSuccess) return;
            const long long pairs = pair_tiles < sms / 2 ? pair_tiles : sms / 2;
            matmul_pair_kernel<T><<<(unsigned)(2 * pairs), kPairThreads, kPairSmem, s>>>(g, pair_tiles);
            return;
        }
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
