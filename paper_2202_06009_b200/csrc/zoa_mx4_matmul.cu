// Products of 4-bit microscaled matrices on the tensor cores: C[i, j] = sum_k A[i, k] B[j, k], both operands in the
// tiles of zoa_mx4.cuh, sums in binary32.
#include "zoa_async.cuh"
#include "zoa_mx4.cuh"

#include <algorithm>

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
__device__ __forceinline__ void copy_scales(uint32_t one, uint32_t tmem, uint64_t desc)
{
    asm volatile(ZOA_IF_ONE("tcgen05.cp.cta_group::1.32x128b.warpx4 [%1], %2;") ::"r"(one), "r"(tmem), "l"(desc) : "memory");
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
    bool vec;                 // rows of `out` are 16-byte aligned
    int test_stop;            // > 0: the copies stop at this k tile (error-path test)
    WaitLimit limit;
};

// ---- one SM a tile, small products --------------------------------------------------------------------------
// A block computes 128 x kBN of C, or its share of the sum over k: the `splits` blocks of a cluster divide the k tiles
// and add their sums up through each other's shared memory, in the order of their ranks.  Narrow tiles and splits put a
// product of few rows on all SMs; what bounds it then is the chain of latencies of one block (set-up, first copies, sums,
// stores: about 5 us).  Three or four stages, so that two blocks share an SM and one's chain runs beside the other's:
// 4096 x 1024 x 512 in 8.1 us, with six stages and one block 12.5.
template <int kBN>
struct Small {
    static_assert(kBN == 64 || kBN == 128, "scales begin at even columns");
    static constexpr int kStages = kBN == 128 ? 3 : 4;
    static constexpr int kStageBytes = kMxTileBytes + kMxScaleBytes + kBN * 128;       // A tile; B scales; B codes
    static constexpr int kScaleColumns = 16;                                           // 8 for A, 8 for B
    static constexpr int kTmemColumns = kBN + 16 * kStages > 256 ? 512 : 256;
    static constexpr int kPitch = kBN + 4;          // floats; rows 4 banks apart
    struct Shared {
        unsigned long long full[kStages], empty[kStages], done;
        uint32_t tmem;
        int gave_up;
    };
    static constexpr int kSmem = kStages * kStageBytes + 1024 + (int)sizeof(Shared);
};

__device__ __forceinline__ float4 load_from_block(uint32_t addr, uint32_t rank)
{
    uint32_t remote;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(remote) : "memory");
    return v;
}

// Warp 0 copies tiles into the ring, warp 1 issues the tensor core's work, warps 2 to 5 take the sums; all store.
template <typename T, int kBN>
__global__ void __launch_bounds__(192) matmul_kernel(const MatmulArgs g, const int splits, const int tiles_n)
{
    using S = Small<kBN>;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    typename S::Shared *sh = reinterpret_cast<typename S::Shared *>(ring + S::kStages * S::kStageBytes);
    const int warp = (int)__reduce_max_sync(0xffffffffu, threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int split = splits > 1 ? (int)(blockIdx.x % (unsigned)splits) : 0;
    const unsigned tile = blockIdx.x / (unsigned)splits;
    const long long i0 = (long long)(tile / (unsigned)tiles_n) * 128, j0 = (long long)(tile % (unsigned)tiles_n) * kBN;
    const int k0 = (int)((long long)g.tiles_k * split / splits), k1 = (int)((long long)g.tiles_k * (split + 1) / splits);
    const int rows = (int)(g.m - i0 < 128 ? g.m - i0 : 128), cols = (int)(g.n - j0 < kBN ? g.n - j0 : kBN);
    int issued = 0;           // tiles whose copies warp 0 has started

    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(smem_addr(&sh->full[s]), 1);
            mbar_init(smem_addr(&sh->empty[s]), 1);
        }
        mbar_init(smem_addr(&sh->done), 1);
        sh->gave_up = 0;
        mbar_init_done();
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh->tmem)), "n"(S::kTmemColumns)
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
        const int row_b = (int)(j0 % kMxTileRows);      // this block's first row in its tile of B
        const uint32_t bytes_a = kMxScaleBytes + 128 * (uint32_t)rows, bytes_b = 128 * (uint32_t)cols;
        const uint8_t *a = g.a + (i0 / kMxTileRows * g.tiles_k + k0) * kMxTileBytes;
        const uint8_t *b = g.b + (j0 / kMxTileRows * g.tiles_k + k0) * kMxTileBytes;
        int s = 0;
        uint32_t parity = 1;
        for (int k = k0; k < k1; ++k) {
            if (g.test_stop > 0 && k >= g.test_stop) break;
            if (!warp_wait(smem_addr(&sh->empty[s]), parity, gave_up, g.limit)) break;
            const uint32_t full = smem_addr(&sh->full[s]), dst = smem_addr(ring + s * S::kStageBytes);
            expect_one(one, full, bytes_a + kMxScaleBytes + bytes_b);
            bulk_load_one(one, dst, a, bytes_a, full);
            bulk_load_one(one, dst + kMxTileBytes, b, kMxScaleBytes, full);
            bulk_load_one(one, dst + kMxTileBytes + kMxScaleBytes, b + kMxScaleBytes + row_b * 128, bytes_b, full);
            a += kMxTileBytes;
            b += kMxTileBytes;
            ++issued;
            if (++s == S::kStages) {
                s = 0;
                parity ^= 1u;
            }
        }
    } else if (warp == 1) {
        const uint32_t one = elect_one();
        // The column of the scales of this block's first row: 0 or 2.  (Scales begin at even columns; tiles of 32 columns
        // would begin at odd ones.)
        const uint32_t column_b = (uint32_t)(j0 % kMxTileRows) / 32;
        int s = 0;
        uint32_t parity = 0;
        for (int k = k0; k < k1; ++k) {
            if (!warp_wait(smem_addr(&sh->full[s]), parity, gave_up, g.limit)) break;
            const uint32_t base_a = smem_addr(ring + s * S::kStageBytes), base_b = base_a + kMxTileBytes;
            const uint32_t sf = tmem + kBN + s * S::kScaleColumns;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                copy_scales(one, sf + h * 4, scales_desc(base_a + h * 512));
                copy_scales(one, sf + 8 + h * 4, scales_desc(base_b + h * 512));
            }
            const uint64_t da = codes_desc(base_a + kMxScaleBytes), db = codes_desc(base_b + kMxScaleBytes);
#pragma unroll
            for (int q = 0; q < 4; ++q)      // 64 columns a step: 32 bytes of a 128-byte line
                if (4 * k + q < g.k_steps)
                    mma_mx4(one, tmem, da + 2 * q, db + 2 * q, q & 1 ? mma_desc(128, kBN, 2) : mma_desc(128, kBN, 0), sf + (q >> 1) * 4,
                            sf + 8 + (q >> 1) * 4 + column_b, k > k0 || q > 0);
            commit(one, smem_addr(&sh->empty[s]));
            if (++s == S::kStages) {
                s = 0;
                parity ^= 1u;
            }
        }
        commit(one, smem_addr(&sh->done));
    }
    const bool finished = warp_wait(smem_addr(&sh->done), 0, gave_up, g.limit);
    if (warp == 0 && *gave_up) {      // copies in flight land before the block's shared memory is used otherwise
        for (int q = issued > S::kStages ? issued - S::kStages : 0; q < issued; ++q)
            mbar_drain(smem_addr(&sh->full[q % S::kStages]), (uint32_t)(q / S::kStages & 1), g.limit);
    }
    __syncthreads();
    // The ring is free: the sums go there, so that rows can be stored by neighbouring threads whatever their alignment.
    float *sums = reinterpret_cast<float *>(ring);
    if (warp >= 2 && finished) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        const int quarter = warp & 3;
        float *mine = sums + (quarter * 32 + lane) * S::kPitch;
#pragma unroll
        for (int c = 0; c < kBN; c += 32) {
            uint32_t v[32];
            load_columns32(tmem + ((uint32_t)(quarter * 32) << 16) + c, v);
            columns_loaded();
#pragma unroll
            for (int k = 0; k < 32; k += 4) *reinterpret_cast<uint4 *>(mine + c + k) = make_uint4(v[k], v[k + 1], v[k + 2], v[k + 3]);
        }
        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    }
    __syncthreads();
    if (splits > 1) cluster_sync();
    // This block's rows of the result: all of them, or its share of the cluster's.
    const int r0 = rows * split / splits, r1 = rows * (split + 1) / splits;
    for (int x = threadIdx.x; x < (r1 - r0) * (kBN / 4); x += 192) {
        const int r = r0 + x / (kBN / 4), c = x % (kBN / 4) * 4;
        if (c >= cols) continue;
        float4 v;
        if (splits == 1) {
            v = *reinterpret_cast<const float4 *>(sums + r * S::kPitch + c);
        } else {
            const uint32_t at = smem_addr(sums + r * S::kPitch + c);
            v = load_from_block(at, 0);
            for (int o = 1; o < splits; ++o) {
                const float4 w = load_from_block(at, (uint32_t)o);
                v.x += w.x;
                v.y += w.y;
                v.z += w.z;
                v.w += w.w;
            }
        }
        T *dst = static_cast<T *>(g.out) + (i0 + r) * g.ld + j0 + c;
        if (g.vec && c + 4 <= cols) {
            if constexpr (sizeof(T) == 4) *reinterpret_cast<float4 *>(dst) = v;
            else *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<T>(v.x, v.y), pack2<T>(v.z, v.w));
        } else {
            dst[0] = from_f32<T>(v.x);
            if (c + 1 < cols) dst[1] = from_f32<T>(v.y);
            if (c + 2 < cols) dst[2] = from_f32<T>(v.z);
            if (c + 3 < cols) dst[3] = from_f32<T>(v.w);
        }
    }
    __syncthreads();
    if (splits > 1) cluster_sync();      // nobody leaves while others read its sums
    if (warp == 1) {
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::kTmemColumns) : "memory");
    }
}

// ---- pairs of SMs, large products --------------------------------------------------------------------------
// A cluster of two blocks computes 256 x 256 of C at a time, each block the sums of 128 rows, and walks over the tiles
// with a stride: 16384 x 8192 x 4096 in 205 us (5.4 PFLOP/s; 236 us back to back under the power limit),
// 8192 x 8192 x 16384 in 369 (6.0).  What bounds it is the copies that feed it: a product of 256 x 256 x 64 takes 203
// cycles with the copies of the next ones beside it, 43 bytes a cycle into every SM, and 169 on operands that are there
// already; results that leave in the same time add to that (short sums: 16384 x 6400 x 1600 81 us, nothing stored 68).
// Every byte of A goes to one SM and every byte of B's codes too (the tensor cores read the partner's half from its
// shared memory); only B's scales go to both.
constexpr int kPairStages = 5;
constexpr int kPairStageBytes = kMxTileBytes + 2 * kMxScaleBytes + kMxCodeBytes;    // A tile; B scales of both halves; B codes
constexpr int kPairScaleColumns = 24;                                              // 8 for A, 16 for B
constexpr int kPairThreads = 448;
// Where the sums of a pair's even and odd tiles lie: 256 columns from 0 and from 128.  They share 128 columns (the sums of
// two tiles and the scales do not fit side by side); the next tile begins when these have been taken, which also says
// that all of the tile before has been.
constexpr int kPairOverlap = 128;
static_assert(256 + kPairOverlap + kPairStages * kPairScaleColumns <= 512, "tensor memory has 512 columns");
__device__ __forceinline__ uint32_t pair_sums_at(uint32_t round) { return round & 1 ? kPairOverlap : 0; }
struct alignas(16) PairShared {
    unsigned long long full[kPairStages], scaled[kPairStages], empty[kPairStages], sums_full, sums_empty, finished;
    uint32_t tmem;
    int gave_up;
};
constexpr int kTurnPitch = 33;                       // floats; a warp's 32 x 32 sums, turned so that lanes hold neighbours
constexpr int kPairSmem = kPairStages * kPairStageBytes + 1024 + (int)sizeof(PairShared) + 8 * 32 * kTurnPitch * 4;

// Up to two products in one launch, the first with the longer sums: `tiles` in the first and in both.  The pairs take
// the first's tiles with a stride.  Where that leaves some pairs one short, these take `extra` of the second's each, about
// as long as the one; what remains goes round all, beginning with them.
struct PairArgs {
    MatmulArgs product[2];
    long long tiles[2];
    int extra;
};
// (Compiled apart for one product: the walk over two costs it 3 to 6 %.)
template <bool kTwo>
struct PairWalk {
    long long at, pairs, pair, phase_end, first, both;
    int phase, extra;
    __device__ __forceinline__ PairWalk(const PairArgs &p)
        : at(blockIdx.x / 2), pairs(gridDim.x / 2), pair(blockIdx.x / 2), phase_end(p.tiles[0]), first(p.tiles[0]), both(p.tiles[1]), phase(0),
          extra(p.extra)
    {
        settle();
    }
    __device__ __forceinline__ bool more() const { return at < both; }
    __device__ __forceinline__ bool second() const { return kTwo && at >= first; }
    __device__ __forceinline__ long long tile() const { return second() ? at - first : at; }
    __device__ __forceinline__ void next()
    {
        at += kTwo && phase == 1 ? pairs - first % pairs : pairs;
        settle();
    }
    __device__ __forceinline__ void settle()
    {
        if constexpr (!kTwo) return;
        if (phase == 0 && at >= phase_end && first < both) {      // every pair's own tiles of the first product are done
            const long long taken = first % pairs, free = pairs - taken;
            phase = 1;
            phase_end = first + extra * free;
            at = pair < taken ? phase_end : first + pair - taken;
        }
        if (phase == 1 && at >= phase_end) {
            const long long taken = first % pairs;
            phase = 2;
            at = phase_end + (pair < taken ? pair + pairs - taken : pair - taken);
        }
    }
};

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

// 128 bytes of each of a warp's 32 rows (lane = row, already of type T), turned through shared memory so that a store writes
// whole lines; rows are 16-byte aligned.  With a lane storing 32-byte pieces of its own row the stores held the copies up:
// 16384 x 6400 x 1600 to bfloat16 88 us, this way 84, and 81 where results leave the L2 before operands do; to binary32 123,
// 108 and 103.
template <typename T>
__device__ __forceinline__ void store_lines(T *first, long long ld, int rows, int cols, const uint32_t *w, float *turn)
{
    constexpr int kPiece = 16 / (int)sizeof(T);
    const int lane = threadIdx.x & 31;
    uint4 *pieces = reinterpret_cast<uint4 *>(turn);
    __syncwarp();
#pragma unroll
    for (int p = 0; p < 8; ++p) pieces[lane * 8 + (p ^ (lane & 7))] = make_uint4(w[4 * p], w[4 * p + 1], w[4 * p + 2], w[4 * p + 3]);
    __syncwarp();
    const int col = (lane & 7) * kPiece;
    T *at = first + (lane >> 3) * ld + col;
#pragma unroll
    for (int i = 0; i < 8; ++i, at += 4 * ld) {
        const int row = i * 4 + (lane >> 3);
        if (row >= rows) break;
        const uint4 v = pieces[row * 8 + ((lane & 7) ^ (row & 7))];
        if (col + kPiece <= cols) {
            __stcs(reinterpret_cast<uint4 *>(at), v);
        } else {
            const T *e = reinterpret_cast<const T *>(&v);
#pragma unroll
            for (int k = 0; k < kPiece; ++k)
                if (col + k < cols) at[k] = e[k];
        }
    }
}
// 32 columns of rows that are not aligned, element by element.
template <typename T>
__device__ __forceinline__ void store_turned(T *first, long long ld, int rows, int cols, const uint32_t *w, float *turn)
{
    const int lane = threadIdx.x & 31;
    __syncwarp();
#pragma unroll
    for (int k = 0; k < 32; ++k) {
        float v;
        if constexpr (sizeof(T) == 4) {
            v = __uint_as_float(w[k]);
        } else {
            float lo, hi;
            unpack2<T>(w[k >> 1], lo, hi);
            v = k & 1 ? hi : lo;
        }
        turn[lane * kTurnPitch + k] = v;
    }
    __syncwarp();
    if (lane < cols)
        for (int r = 0; r < rows; ++r) first[r * ld + lane] = from_f32<T>(turn[r * kTurnPitch + lane]);
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
template <typename T, bool kTwo>
__global__ void __launch_bounds__(kPairThreads, 1) __cluster_dims__(2, 1, 1) matmul_pair_kernel(const __grid_constant__ PairArgs args)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    unsigned char *ring = reinterpret_cast<unsigned char *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    PairShared *sh = reinterpret_cast<PairShared *>(ring + kPairStages * kPairStageBytes);
    const int warp = (int)__reduce_max_sync(0xffffffffu, threadIdx.x >> 5), lane = threadIdx.x & 31, rank = (int)cluster_rank();
    const WaitLimit limit = args.product[0].limit;

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
        for (PairWalk<kTwo> walk(args); walk.more() && ok; walk.next()) {
            const MatmulArgs &g = args.product[walk.second()];
            const PairTile p = pair_tile(g, walk.tile(), rank);
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
                ok = !(args.product[0].test_stop > 0 && issued >= args.product[0].test_stop) && warp_wait(smem_addr(&sh->empty[s]), parity ^ 1u, gave_up, limit);
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
        const bool done = warp_wait(smem_addr(&sh->finished), 0, gave_up, limit);
        if (!done || *gave_up)
            for (int q = issued > kPairStages ? issued - kPairStages : 0; q < issued; ++q)
                mbar_drain(smem_addr(&sh->full[q % kPairStages]), (uint32_t)(q / kPairStages & 1), limit);
    } else if (warp == 1 && rank == 0) {
        const uint32_t one = elect_one();
        int s = 0;
        uint32_t parity = 0, round = 0;
        bool ok = true;
        for (PairWalk<kTwo> walk(args); walk.more() && ok; walk.next(), ++round) {
            const MatmulArgs &g = args.product[walk.second()];
            const PairTile p = pair_tile(g, walk.tile(), 0);
            const uint32_t desc = mma_desc(256, p.cols, 0);
            const uint32_t sums = tmem + pair_sums_at(round);
            if (round > 0 && !warp_wait<true>(smem_addr(&sh->sums_empty), (round - 1) & 1u, gave_up, limit)) break;
            for (int k = 0; k < g.tiles_k; ++k) {
                // both blocks' copies have landed and their scales are in tensor memory
                if (!(ok = warp_wait<true>(smem_addr(&sh->scaled[s]), parity, gave_up, limit))) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                const uint32_t base_a = smem_addr(ring + s * kPairStageBytes), base_b = base_a + kMxTileBytes + 2 * kMxScaleBytes;
                const uint32_t sf = tmem + 256 + kPairOverlap + s * kPairScaleColumns;
                const uint64_t da = codes_desc(base_a + kMxScaleBytes), db = codes_desc(base_b);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (4 * k + q < g.k_steps)
                        mma_mx4<true>(one, sums, da + 2 * q, db + 2 * q, desc | (q & 1 ? mma_desc(0, 0, 2) : 0), sf + (q >> 1) * 4,
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
        for (PairWalk<kTwo> walk(args); walk.more() && ok; walk.next()) {
            const int tiles_k = args.product[walk.second()].tiles_k;
            for (int k = 0; k < tiles_k; ++k) {
                if (!(ok = warp_wait(smem_addr(&sh->full[s]), parity, gave_up, limit))) break;
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
                const uint32_t sf = tmem + ((uint32_t)(quarter * 32) << 16) + 256 + kPairOverlap + s * kPairScaleColumns;
                store_columns8(sf, v);
                store_columns8(sf + 8, v + 8);
                store_columns8(sf + 16, v + 16);
                columns_stored();
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) {
                    // To the first block goes the news that this one's copies have landed, which the fence puts ahead of the
                    // arrival, and that its scales are in tensor memory, which wait::st and the fences of tcgen05 do.
                    // (A release at cluster scope instead: 16384 x 8192 x 4096 in 415 us for 205.)
                    if (rank == 0) {
                        mbar_arrive(smem_addr(&sh->scaled[s]));
                    } else {
                        release_shared();
                        mbar_tell(smem_addr(&sh->scaled[s]), 0);
                    }
                }
                if (++s == kPairStages) {
                    s = 0;
                    parity ^= 1u;
                }
            }
        }
    } else if (warp >= 6) {
        const int quarter = warp & 3, half = (warp - 6) >> 2;
        float *turn = reinterpret_cast<float *>(sh + 1) + (warp - 6) * 32 * kTurnPitch;
        uint32_t round = 0;
        for (PairWalk<kTwo> walk(args); walk.more(); walk.next(), ++round) {
            const MatmulArgs &g = args.product[walk.second()];
            const PairTile p = pair_tile(g, walk.tile(), rank);
            if (!__all_sync(0xffffffffu, mbar_wait(smem_addr(&sh->sums_full), round & 1u, gave_up, limit))) break;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            const int here = p.rows - quarter * 32 < 32 ? p.rows - quarter * 32 : 32;       // of this warp's rows
            T *corner = static_cast<T *>(g.out) + (p.i0 + quarter * 32) * g.ld + p.j0;
            // First the half of the columns that the next tile's sums will lie in, then the other.
            const int shared = pair_sums_at(round + 1);
            const uint32_t sums = tmem + ((uint32_t)(quarter * 32) << 16) + pair_sums_at(round);
#pragma unroll
            for (int pass = 0; pass < 2; ++pass) {
                const int col = (pass == 0 ? shared : kPairOverlap - shared) + half * 64;
                constexpr int kWords = 32 * (int)sizeof(T) / 4;       // of 32 columns
                uint32_t v[64], w[2 * kWords];
                load_columns32(sums + col, v);
                load_columns32(sums + col + 32, v + 32);
                columns_loaded();
                round32<T>(v, w);
                round32<T>(v + 32, w + kWords);
                if (pass == 0) {
                    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                    __syncwarp();
                    // Only tensor memory is handed over: its loads have been waited for and fenced.
                    if (lane == 0) mbar_tell(smem_addr(&sh->sums_empty), 0);
                }
                constexpr int kAtOnce = 128 / (int)sizeof(T);
                const int have = (int)(g.n - p.j0 - col < 64 ? g.n - p.j0 - col : 64);
#pragma unroll
                for (int c = 0; c < 64; c += 32) {
                    if (c >= have) break;
                    if (!g.vec) store_turned<T>(corner + col + c, g.ld, here, have - c, w + c * (int)sizeof(T) / 4, turn);
                    else if (c % kAtOnce == 0) store_lines<T>(corner + col + c, g.ld, here, have - c, w + c * (int)sizeof(T) / 4, turn);
                }
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

// Which kernel, how wide a tile, how many splits: the least time by what the kernels measured on one B200 (launches
// back to back, in tenths of a microsecond): a pair tile 4.3 per k tile + 10, and 45 once; a tile of 128 (64) columns 4
// (3.2) per k tile + 45 (35), and 10 once; two blocks to an SM 1.4 times as long per k tile and 10 more; splits 18.
// E.g. 1024 x 4096 x 1024 by pairs 7.7 us, 128 columns 9.0, 64 columns 12.2; 77 x 1600 x 6400 by 64 columns and 4 splits
// 7.6, 1 split 11.9, 128 columns and 8 splits 8.2, 1 split 12.9.
struct ProductPlan {
    int columns, splits;       // columns 256: pairs of SMs
    double time;               // tenths of a microsecond
};
long long pair_tiles(const MatmulArgs &g) { return mx_tiles(g.m, 256) * mx_tiles(g.n, 256); }
double pair_tile_time(const MatmulArgs &g) { return 4.3 * g.tiles_k + 10.0; }
// Two products by pairs in one launch, and its time by the same figures.
PairArgs pair_both(const MatmulArgs &a, const MatmulArgs &b, int sms, double *time)
{
    const bool swap = a.tiles_k < b.tiles_k;
    PairArgs p{};
    p.product[0] = swap ? b : a;
    p.product[1] = swap ? a : b;
    const long long first = pair_tiles(p.product[0]), second = pair_tiles(p.product[1]);
    p.tiles[0] = first;
    p.tiles[1] = first + second;
    const long long pairs = first + second < sms / 2 ? first + second : sms / 2, free = pairs - first % pairs;
    const double of_first = pair_tile_time(p.product[0]), of_second = pair_tile_time(p.product[1]);
    p.extra = free < pairs ? (int)(of_first / of_second) : 0;
    const long long full = first / pairs, rest = second - p.extra * free;
    const double own = (double)full * of_first, most = own + (free < pairs ? of_first : 0.0);
    *time = 45.0 + (rest > 0 ? most + (double)((rest + pairs - 1) / pairs) * of_second : std::max(most, own + (double)((second + free - 1) / free) * of_second));
    return p;
}
ProductPlan product_plan(const MatmulArgs &g, int sms)
{
    ProductPlan best{256, 1, 0.0};
    double least = (double)((pair_tiles(g) + sms / 2 - 1) / (sms / 2)) * pair_tile_time(g) + 45.0;
    for (int columns = 128; columns >= 64; columns /= 2)
        for (int splits = 1; splits <= 8 && splits <= g.tiles_k; splits *= 2) {
            const double blocks = (double)mx_tiles(g.m, 128) * (double)mx_tiles(g.n, columns) * splits;
            if (blocks > 1e6) continue;
            const double rounds = (double)(long long)((blocks + 2 * sms - 1) / (2 * sms)), tiles = (double)((g.tiles_k + splits - 1) / splits);
            const bool shared = blocks > sms;
            const double time = rounds * (tiles * (columns == 128 ? 4.0 : 3.2) * (shared ? 1.4 : 1.0) + (columns == 128 ? 45.0 : 35.0)) + 10.0 +
                                (shared ? 10.0 : 0.0) + (splits > 1 ? 18.0 : 0.0);
            if (time < least) {
                least = time;
                best = ProductPlan{columns, splits, 0.0};
            }
        }
    best.time = least;
    return best;
}

template <typename T, int kBN>
void launch_small(const MatmulArgs &g, int splits, cudaStream_t s)
{
    static SmemLimit limit;
    auto kernel = matmul_kernel<T, kBN>;
    if (limit.ensure(kernel, Small<kBN>::kSmem) != cudaSuccess) return;       // the caller reports it
    const int tiles_n = (int)mx_tiles(g.n, kBN);
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(mx_tiles(g.m, 128) * tiles_n * splits));
    cfg.blockDim = dim3(192);
    cfg.dynamicSmemBytes = Small<kBN>::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {(unsigned)splits, 1, 1};
    cfg.attrs = &at;
    cfg.numAttrs = splits > 1;
    cudaLaunchKernelEx(&cfg, kernel, g, splits, tiles_n);
}

template <typename T, bool kTwo>
void launch_pairs(const PairArgs &p, int sms, cudaStream_t s)
{
    static SmemLimit limit;
    if (limit.ensure(matmul_pair_kernel<T, kTwo>, kPairSmem) != cudaSuccess) return;       // the caller reports it
    const long long pairs = p.tiles[1] < sms / 2 ? p.tiles[1] : sms / 2;
    matmul_pair_kernel<T, kTwo><<<(unsigned)(2 * pairs), kPairThreads, kPairSmem, s>>>(p);
}

// ---- few rows ------------------------------------------------------------------------------------------------
// out = Q(x) b^T for up to four rows of x, as when tokens are generated one at a time: every block rounds x for itself
// (a few thousand elements) into shared memory while its weights are on their way, and multiplies on the ordinary
// cores.  One row, 1600 -> 6400: 4.0 us (b's 5.4 MB at the copy rate 0.8, an empty launch about 2.2); 4096 -> 4096: 6.0,
// bounded by the instructions that turn codes into binary16 and add them up.  A lane takes a block of 32 columns of one row of b: its codes
// are 16 bytes and become pairs of binary16, x's elements lie as binary16; eight products of elements (multiples of
// 1/4, at most 36) add up to less than 2^11 quarters, so sums of eight are exact in binary16, those of a block in
// binary32.
constexpr int kFewRows = 4, kFewWarps = 8, kFewAhead = 4;
constexpr int kFewSmem = 200 * 1024;

// 2^(a + b - 254) by two factors, neither of which leaves binary32's range.
__device__ __forceinline__ float times_scales(float v, uint32_t a, uint32_t b)
{
    if (a == 255u || b == 255u) return __uint_as_float(0x7FC00000u);
    const int e = (int)(a + b) - 254, half = e >> 1;
    return v * __uint_as_float((uint32_t)(half + 127) << 23) * __uint_as_float((uint32_t)(e - half + 127) << 23);
}
__device__ __forceinline__ void halves8(uint32_t codes, __half2 *v) { mx_halves8(codes, reinterpret_cast<uint32_t *>(v)); }

template <typename T, int kRows>
__global__ void __launch_bounds__(kFewWarps * 32) few_rows_kernel(const T *__restrict__ x, long long ldx, bool vec, const MatmulArgs g,
                                                                  long long k_cols, int parts)
{
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ float part_s[kFewWarps][4][kRows];
    // x: [row][k tile][piece of 8 elements of a block][block] of 16 bytes, so that the eight blocks a warp reads lie in
    // different banks; then [row][k tile][block] scale bytes.
    uint4 *x_s = reinterpret_cast<uint4 *>(smem_raw);
    uint8_t *scale_s = smem_raw + (size_t)kRows * g.tiles_k * 512;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int group = warp / parts, part = warp % parts;              // which four rows of b; which of the k tiles
    const int rows_b = kFewWarps / parts * 4;                         // rows of b a block takes at a time
    // This lane's row of b and, kFewAhead at a time, the k tiles whose codes are on their way.
    long long n_next = (long long)blockIdx.x * rows_b + group * 4 + (lane >> 3);
    int t_next = part;
    uint4 codes[kFewAhead];
    uint32_t bytes[kFewAhead];
    auto fetch = [&] {
        const int r = (int)(n_next % kMxTileRows), block = (lane & 7) ^ (r & 7);
        const uint8_t *tile = g.b + (n_next / kMxTileRows * g.tiles_k + t_next) * kMxTileBytes;
        const uint8_t *codes_at = tile + kMxScaleBytes + r * 128 + (lane & 7) * 16, *scale_at = tile + mx_scale_at(r, block);
#pragma unroll
        for (int i = 0; i < kFewAhead; ++i) {
            codes[i] = make_uint4(0, 0, 0, 0);
            bytes[i] = 0;
            if (n_next < g.n && t_next + i * parts < g.tiles_k) {
                codes[i] = __ldg(reinterpret_cast<const uint4 *>(codes_at + (long long)(i * parts) * kMxTileBytes));
                bytes[i] = __ldg(scale_at + (long long)(i * parts) * kMxTileBytes);
            }
        }
        t_next += kFewAhead * parts;
        if (t_next - part >= (g.tiles_k - part + parts - 1) / parts * parts) {
            t_next = part;
            n_next += (long long)gridDim.x * rows_b;
        }
    };
    fetch();
    // x: a warp takes a line of 256 columns, a lane 8 of them.
    for (int line = warp; line < kRows * g.tiles_k; line += kFewWarps) {
        const int row = line / g.tiles_k, t = line % g.tiles_k;
        const long long c = (long long)t * kMxTileCols + lane * 8;
        const Raw8<T> v = load8(x + row * ldx + c, row < g.m ? k_cols - c : 0, vec);
        const uint32_t byte = block_scale(v), q = byte == 255u ? 0u : codes8(v, mx_inverse(byte));
        __half2 e[4];
        halves8(q, e);
        x_s[line * 32 + (lane & 3) * 8 + (lane >> 2)] = *reinterpret_cast<const uint4 *>(e);
        if ((lane & 3) == 0) scale_s[line * 8 + (lane >> 2)] = (uint8_t)byte;
    }
    __syncthreads();
    for (long long first = (long long)blockIdx.x * rows_b; first < g.n; first += (long long)gridDim.x * rows_b) {
        const int block = (lane & 7) ^ (int)((first + group * 4 + (lane >> 3)) & 7);
        float sum[kRows] = {};
        for (int t0 = part; t0 < g.tiles_k; t0 += kFewAhead * parts) {
            uint4 now[kFewAhead];
            uint32_t scale[kFewAhead];
#pragma unroll
            for (int i = 0; i < kFewAhead; ++i) {
                now[i] = codes[i];
                scale[i] = bytes[i];
            }
            fetch();
#pragma unroll
            for (int i = 0; i < kFewAhead; ++i) {
                const int t = t0 + i * parts;
                if (t >= g.tiles_k) break;
                __half2 w[16];
                halves8(now[i].x, w);
                halves8(now[i].y, w + 4);
                halves8(now[i].z, w + 8);
                halves8(now[i].w, w + 12);
#pragma unroll
                for (int m = 0; m < kRows; ++m) {
                    const uint4 *at = x_s + (m * g.tiles_k + t) * 32 + block;
                    float s = 0.0f;
#pragma unroll
                    for (int p = 0; p < 4; p += 2) {          // sixteen elements: eight products in either half
                        const uint4 a0 = at[p * 8], a1 = at[p * 8 + 8];
                        const __half2 *e0 = reinterpret_cast<const __half2 *>(&a0), *e1 = reinterpret_cast<const __half2 *>(&a1);
                        __half2 acc = __hmul2(w[4 * p], e0[0]);
#pragma unroll
                        for (int k = 1; k < 4; ++k) acc = __hfma2(w[4 * p + k], e0[k], acc);
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc = __hfma2(w[4 * p + 4 + k], e1[k], acc);
                        const float2 f = __half22float2(acc);
                        s += f.x + f.y;
                    }
                    sum[m] += times_scales(s, scale[i], scale_s[(m * g.tiles_k + t) * 8 + block]);
                }
            }
        }
        __syncthreads();          // the last round's part_s has been read
#pragma unroll
        for (int m = 0; m < kRows; ++m) {
            sum[m] += __shfl_xor_sync(0xffffffffu, sum[m], 1);
            sum[m] += __shfl_xor_sync(0xffffffffu, sum[m], 2);
            sum[m] += __shfl_xor_sync(0xffffffffu, sum[m], 4);
            if ((lane & 7) == 0) part_s[warp][lane >> 3][m] = sum[m];
        }
        __syncthreads();
        // One thread per row of b and row of x adds the parts, in order.
        for (int i = threadIdx.x; i < rows_b * kRows; i += kFewWarps * 32) {
            const int m = i / rows_b, rb = i % rows_b;
            const long long at = first + rb;
            if (m >= g.m || at >= g.n) continue;
            float v = part_s[rb / 4 * parts][rb % 4][m];
            for (int p = 1; p < parts; ++p) v += part_s[rb / 4 * parts + p][rb % 4][m];
            static_cast<T *>(g.out)[m * g.ld + at] = from_f32<T>(v);
        }
    }
}

// Rows that few_rows_kernel is compiled for, or 0 where the tensor cores are as fast in two launches (measured on one
// B200: 2 x 4096 x 4096 7.8 us here, 9.3 there; 1 x 8192 x 8192 13.2 and 11.2; 4 x 6400 x 1600 8.1 and 8.1) or x is too
// large for a block's shared memory.
int few_rows(size_t m, size_t n, size_t k)
{
    const int rows = m <= 1 ? 1 : m <= 2 ? 2 : kFewRows;
    const bool small = m <= (size_t)kFewRows && n <= kMxMaxSide && k <= kMxMaxSide && (double)m * (double)n * (double)k <= (double)(1 << 25);
    return small && (size_t)mx_tiles((long long)k, kMxTileCols) * rows * 520 <= (size_t)kFewSmem ? rows : 0;
}

template <typename T, int kRows>
void launch_few(const void *x, long long ldx, bool vec, const MatmulArgs &g, long long k, int sms, cudaStream_t s)
{
    static SmemLimit limit;
    auto kernel = few_rows_kernel<T, kRows>;
    if (limit.ensure(kernel, kFewSmem) != cudaSuccess) return;       // the caller reports it
    // Warps that share rows of b divide its k tiles between them: more of them while there are fewer than two blocks
    // an SM and every warp keeps two tiles.  No more blocks than the SMs hold: each rounds x once.
    int parts = 1;
    while (parts < kFewWarps && mx_tiles(g.n, 4 * kFewWarps / parts) < 2 * sms && g.tiles_k >= 4 * parts) parts *= 2;
    const long long blocks = mx_tiles(g.n, 4 * kFewWarps / parts), most = (kRows == 1 ? 3ll : 2ll) * sms;
    kernel<<<(unsigned)(blocks < most ? blocks : most), kFewWarps * 32, (size_t)kRows * g.tiles_k * 520, s>>>(static_cast<const T *>(x), ldx, vec, g,
                                                                                                            k, parts);
}

zoa_status check_matrix(const char *me, const char *name, const void *p)
{
    if (!p) return ops_fail(ZOA_ERR_ARG, "%s: %s is NULL", me, name);
    if (!aligned16(p)) return ops_fail(ZOA_ERR_ARG, "%s: %s must be 16-byte aligned", me, name);
    return ZOA_OK;
}

zoa_status check_product(const char *me, size_t m, size_t n, size_t k, const void *out, int dtype, size_t ld)
{
    if (!dtype_ok(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, dtype);
    if (m > kMxMaxSide || n > kMxMaxSide || k > kMxMaxSide) return ops_fail(ZOA_ERR_ARG, "%s: m, n and k must be at most 2^30", me);
    if (m == 0 || n == 0) return ZOA_OK;
    if (!out) return ops_fail(ZOA_ERR_ARG, "%s: out is NULL", me);
    if (ld < n) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least n", me);
    if (reinterpret_cast<uintptr_t>(out) % dtype_bytes(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: out is not aligned to its element type", me);
    return ZOA_OK;
}

// What the kernels take of a product that is not empty, checked; and how many SMs there are.
zoa_status product_args(const char *me, const void *a, const void *b, size_t m, size_t n, size_t k, void *out, int dtype, size_t ld,
                        MatmulArgs &g, int &sms)
{
    zoa_status st = check_matrix(me, "a", a);
    if (st == ZOA_OK) st = check_matrix(me, "b", b);
    if (st != ZOA_OK) return st;
    g.a = static_cast<const uint8_t *>(a);
    g.b = static_cast<const uint8_t *>(b);
    g.out = out;
    g.m = (long long)m;
    g.n = (long long)n;
    g.ld = (long long)ld;
    g.tiles_k = (int)mx_tiles((long long)k, kMxTileCols);
    g.k_steps = (int)mx_tiles((long long)k, 64);
    g.vec = (reinterpret_cast<uintptr_t>(out) | (ld * dtype_bytes(dtype))) % 16 == 0;
    g.test_stop = ops_test_stop();
    g.limit.error_word = ops_error_word();
    g.limit.ns = ops_wait_limit_ns();
    if (!g.limit.error_word) return ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me);
    sms = ops_sm_count();
    return sms < 2 ? ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me) : ZOA_OK;
}

}  // namespace
}  // namespace zoa

using namespace zoa;

extern "C" zoa_status zoa_mx4_matmul(const void *a, const void *b, size_t m, size_t n, size_t k, void *out, int dtype, size_t ld,
                                     void *stream)
{
    const char *me = "zoa_mx4_matmul";
    if (ops_gave_up()) return ops_refuse(me);
    zoa_status st = check_product(me, m, n, k, out, dtype, ld);
    if (st != ZOA_OK || m == 0 || n == 0) return st;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    if (k == 0) {      // an empty sum
        if (cudaMemset2DAsync(out, ld * dtype_bytes(dtype), 0, n * dtype_bytes(dtype), m, s) != cudaSuccess) return ops_launched(me);
        return ZOA_OK;
    }
    MatmulArgs g{};
    int sms = 0;
    st = product_args(me, a, b, m, n, k, out, dtype, ld, g, sms);
    if (st != ZOA_OK) return st;
    const ProductPlan plan = product_plan(g, sms);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (plan.columns == 256) {
            PairArgs p{};
            p.product[0] = g;
            p.tiles[0] = p.tiles[1] = pair_tiles(g);
            launch_pairs<T, false>(p, sms, s);
        } else if (plan.columns == 128) {
            launch_small<T, 128>(g, plan.splits, s);
        } else {
            launch_small<T, 64>(g, plan.splits, s);
        }
    });
    return ops_launched(me);
}

extern "C" size_t zoa_mx4_linear_work(size_t m, size_t n, size_t k)
{
    return few_rows(m, n, k) ? 0 : zoa_mx4_size(m, k);
}

extern "C" zoa_status zoa_mx4_linear(const void *x, int dtype, size_t m, size_t k, size_t ldx, const void *b, size_t n, void *out,
                                     size_t ld, void *work, void *stream)
{
    const char *me = "zoa_mx4_linear";
    if (ops_gave_up()) return ops_refuse(me);
    if (!m || !n) return check_product(me, m, n, k, out, dtype, ld);
    const int rows = few_rows(m, n, k);
    if (!rows || !k) {
        zoa_status st = mx4_check_source(me, x, dtype, m, k, ldx, work, nullptr);
        if (st == ZOA_OK) st = check_product(me, m, n, k, out, dtype, ld);
        if (st == ZOA_OK && k) st = check_matrix(me, "b", b);
        if (st == ZOA_OK) st = zoa_mx4_quantize(x, dtype, m, k, ldx, work, nullptr, stream);
        return st != ZOA_OK ? st : zoa_mx4_matmul(work, b, m, n, k, out, dtype, ld, stream);
    }
    if (!dtype_ok(dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, dtype);
    if (n > kMxMaxSide || k > kMxMaxSide) return ops_fail(ZOA_ERR_ARG, "%s: n and k must be at most 2^30", me);
    if (!x || !out) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    if (ldx < k || ld < n) return ops_fail(ZOA_ERR_ARG, "%s: ldx must be at least k and ld at least n", me);
    if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(out)) % dtype_bytes(dtype))
        return ops_fail(ZOA_ERR_ARG, "%s: x or out is not aligned to its element type", me);
    const zoa_status st = check_matrix(me, "b", b);
    if (st != ZOA_OK) return st;
    const int sms = ops_sm_count();
    if (sms < 2) return ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me);
    MatmulArgs g{};
    g.b = static_cast<const uint8_t *>(b);
    g.out = out;
    g.m = (long long)m;
    g.n = (long long)n;
    g.ld = (long long)ld;
    g.tiles_k = (int)mx_tiles((long long)k, kMxTileCols);
    const bool vec = aligned16(x) && ldx * dtype_bytes(dtype) % 16 == 0;
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    with_type(dtype, [&](auto t) {
        using T = decltype(t);
        if (rows == 1) launch_few<T, 1>(x, (long long)ldx, vec, g, (long long)k, sms, s);
        else if (rows == 2) launch_few<T, 2>(x, (long long)ldx, vec, g, (long long)k, sms, s);
        else launch_few<T, kFewRows>(x, (long long)ldx, vec, g, (long long)k, sms, s);
    });
    return ops_launched(me);
}

extern "C" zoa_status zoa_mx4_linear_forward(const void *x, int x_type, size_t ldx, const void *w, int w_type, size_t ldw, size_t m,
                                             size_t n, size_t k, void *y, size_t ldy, void *xt, void *wt, void *work, void *stream)
{
    const char *me = "zoa_mx4_linear_forward";
    if (ops_gave_up()) return ops_refuse(me);
    if (m && n && k && (!xt || !wt || !work)) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    void *wq = static_cast<unsigned char *>(work) + zoa_mx4_size(m, k);
    zoa_status st = mx4_check_source(me, x, x_type, m, k, ldx, work, xt);
    if (st == ZOA_OK) st = mx4_check_source(me, w, w_type, n, k, ldw, wq, wt);
    if (st == ZOA_OK) st = check_product(me, m, n, k, y, x_type, ldy);
    if (st != ZOA_OK) return st;
    if (x_type == w_type && m && n && k) {      // one launch for both
        st = mx4_launch_both(me, x_type, mx4_both_job(x, x_type, m, k, ldx, work, xt), mx4_both_job(w, w_type, n, k, ldw, wq, wt),
                             static_cast<cudaStream_t>(stream));
    } else {
        st = zoa_mx4_quantize(x, x_type, m, k, ldx, work, xt, stream);
        if (st == ZOA_OK) st = zoa_mx4_quantize(w, w_type, n, k, ldw, wq, wt, stream);
    }
    return st != ZOA_OK ? st : zoa_mx4_matmul(work, wq, m, n, k, y, x_type, ldy, stream);
}

extern "C" zoa_status zoa_mx4_linear_backward(const void *dy, int dy_type, size_t ld_dy, size_t m, size_t n, size_t k, const void *xt,
                                              const void *wt, void *dx, int dx_type, size_t ld_dx, void *dw, int dw_type, size_t ld_dw,
                                              void *work, void *stream)
{
    const char *me = "zoa_mx4_linear_backward";
    if (ops_gave_up()) return ops_refuse(me);
    if (!dx && !dw && m && n && k) return ops_fail(ZOA_ERR_ARG, "%s: neither dx nor dw is asked for", me);      // (an empty one may be NULL)
    if (m && n && k && !work) return ops_fail(ZOA_ERR_ARG, "%s: work is NULL", me);
    void *dyt = static_cast<unsigned char *>(work) + zoa_mx4_size(m, n);
    void *dy_rows = dx ? work : nullptr, *dy_columns = dw ? dyt : nullptr;
    zoa_status st = k ? mx4_check_source(me, dy, dy_type, m, n, ld_dy, dy_rows, dy_columns) : ZOA_OK;
    if (st == ZOA_OK && dx) st = check_product(me, m, k, n, dx, dx_type, ld_dx);
    if (st == ZOA_OK && dw) st = check_product(me, n, k, m, dw, dw_type, ld_dw);
    if (st == ZOA_OK && dx && m && n && k) st = check_matrix(me, "wt", wt);
    if (st == ZOA_OK && dw && m && n && k) st = check_matrix(me, "xt", xt);
    if (st == ZOA_OK && k) st = zoa_mx4_quantize(dy, dy_type, m, n, ld_dy, dy_rows, dy_columns, stream);
    if (st == ZOA_OK && dx && dw && dx_type == dw_type && m && n && k) {
        // Both in one launch where that is no slower: small ones fill the SMs together (rounding and both products, 512 x 1024
        // -> 4096: 25.0 -> 20.6 us, 1777 x 1001 -> 1333 31.8 -> 25.5), of large ones the last tiles of the longer sums run
        // beside the others' (16384 x 1600 -> 6400: 219 -> 203).
        MatmulArgs of_x{}, of_w{};
        int sms = 0;
        st = product_args(me, work, wt, m, k, n, dx, dx_type, ld_dx, of_x, sms);
        if (st == ZOA_OK) st = product_args(me, dyt, xt, n, k, m, dw, dw_type, ld_dw, of_w, sms);
        if (st != ZOA_OK) return st;
        double together = 0.0;
        const PairArgs p = pair_both(of_x, of_w, sms, &together);
        if (together <= product_plan(of_x, sms).time + product_plan(of_w, sms).time) {
            with_type(dx_type, [&](auto t) { launch_pairs<decltype(t), true>(p, sms, static_cast<cudaStream_t>(stream)); });
            return ops_launched(me);
        }
    }
    if (st == ZOA_OK && dx) st = zoa_mx4_matmul(work, wt, m, k, n, dx, dx_type, ld_dx, stream);
    if (st == ZOA_OK && dw) st = zoa_mx4_matmul(dyt, xt, n, k, m, dw, dw_type, ld_dw, stream);
    return st;
}
