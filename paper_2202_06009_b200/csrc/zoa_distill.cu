// Distillation from a teacher's top logits: loss, its gradient, or both (the mathematics stands at
// zoa_distill_topk in include/zoa.h).
//
// With m the row's largest logit, e_j = exp((z_j - m) / T) and f_j = exp(z_j - m), everything a row needs is
//   m,  s = sum e_j,  s1 = sum f_j,  r = sum of e_j over unlisted j
// and the gradient is, for coefficients that are the same for the whole row,
//   unlisted j: cu e_j + cb f_j        listed j: ca e_j - c0 p_j + cb f_j        label: - ch more.
#include "zoa_async.cuh"
#include "zoa_ops.h"

#include <cfloat>
#include <type_traits>

namespace zoa {
namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLeastRest = 1e-30f;   // unlisted tokens with less of the student's mass count as none: p_r / q_r stays finite
constexpr size_t kMaxTop = 2048, kMaxVocab = (size_t)1 << 20;

struct DistillArgs {
    const void *logits;
    const int32_t *index;
    const void *teacher;
    const float *lse;
    const int32_t *labels;
    const float *weight;
    const float *grad_loss;   // of the backward call, or NULL
    const float *stats_in;    // of the backward call, or NULL
    float *loss, *stats;
    void *grad;
    long long rows, ld_logits, ld_grad;
    int vocab, top;
    float temperature, inv_t, soft_weight, hard_weight;
};

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Running sums of part of a row relative to its largest logit.
struct alignas(16) Sums {
    float m, s, s1, r;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }
// exp((a - m) c) for a <= m; 1 where they are equal, infinities included.
__device__ __forceinline__ float shrink(float a, float m, float c) { return a == m ? 1.0f : ex2((a - m) * c); }
__device__ __forceinline__ Sums join(const Sums &a, const Sums &b, float c)
{
    Sums o;
    o.m = fmaxf(a.m, b.m);
    const float fa = shrink(a.m, o.m, c), fb = shrink(b.m, o.m, c);
    o.s = a.s * fa + b.s * fb;
    o.r = a.r * fa + b.r * fb;
    o.s1 = a.s1 * shrink(a.m, o.m, kLog2e) + b.s1 * shrink(b.m, o.m, kLog2e);
    return o;
}
__device__ __forceinline__ float warp_sum(float v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float warp_max(float v)      // passes over a NaN like fmaxf
{
    float m;
    asm("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(m) : "f"(v));
    return m;
}
// The sums of a warp's threads: one change of base each, then plain sums.
__device__ __forceinline__ Sums warp_join(const Sums &a, float c)
{
    Sums o;
    o.m = warp_max(a.m);
    const float f = shrink(a.m, o.m, c);
    o.s = warp_sum(a.s * f);
    o.r = warp_sum(a.r * f);
    o.s1 = warp_sum(a.s1 * shrink(a.m, o.m, kLog2e));
    return o;
}

__device__ __forceinline__ uint64_t pair(float lo, float hi)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float &lo, float &hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ __forceinline__ uint64_t ex2_2(uint64_t y)
{
    float lo, hi;
    unpair(y, lo, hi);
    return pair(ex2(lo), ex2(hi));
}

// A 16-byte vector as pairs of binary32, and its largest element.
template <typename T>
struct Pairs {
    static constexpr int kCount = 4;
    static __device__ __forceinline__ void unpack(const uint4 &w, uint64_t *x)
    {
        float lo, hi;
        unpack2<T>(w.x, lo, hi);
        x[0] = pair(lo, hi);
        unpack2<T>(w.y, lo, hi);
        x[1] = pair(lo, hi);
        unpack2<T>(w.z, lo, hi);
        x[2] = pair(lo, hi);
        unpack2<T>(w.w, lo, hi);
        x[3] = pair(lo, hi);
    }
    static __device__ __forceinline__ uint32_t pack_pair(uint64_t v)
    {
        float lo, hi;
        unpair(v, lo, hi);
        return pack2<T>(lo, hi);
    }
    static __device__ __forceinline__ uint4 pack(const uint64_t *x)
    {
        return make_uint4(pack_pair(x[0]), pack_pair(x[1]), pack_pair(x[2]), pack_pair(x[3]));
    }
    using T2 = typename std::conditional<std::is_same<T, __half>::value, __half2, __nv_bfloat162>::type;
    static __device__ __forceinline__ T2 as2(uint32_t w) { return *reinterpret_cast<const T2 *>(&w); }
    // The largest elements of several vectors, joined as they lie, and taken apart once.
    using Max = T2;
    static __device__ __forceinline__ Max largest(const uint4 &w) { return __hmax2(__hmax2(as2(w.x), as2(w.y)), __hmax2(as2(w.z), as2(w.w))); }
    static __device__ __forceinline__ Max larger(Max a, Max b) { return __hmax2(a, b); }
    static __device__ __forceinline__ float value(Max m)
    {
        float lo, hi;
        unpack2<T>(*reinterpret_cast<const uint32_t *>(&m), lo, hi);
        return fmaxf(lo, hi);
    }
};
template <>
struct Pairs<float> {
    static constexpr int kCount = 2;
    static __device__ __forceinline__ void unpack(const uint4 &w, uint64_t *x)
    {
        x[0] = (uint64_t)w.y << 32 | w.x;
        x[1] = (uint64_t)w.w << 32 | w.z;
    }
    static __device__ __forceinline__ uint4 pack(const uint64_t *x)
    {
        return make_uint4((uint32_t)x[0], (uint32_t)(x[0] >> 32), (uint32_t)x[1], (uint32_t)(x[1] >> 32));
    }
    using Max = float;
    static __device__ __forceinline__ Max largest(const uint4 &w)
    {
        return fmaxf(fmaxf(__uint_as_float(w.x), __uint_as_float(w.y)), fmaxf(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    static __device__ __forceinline__ Max larger(Max a, Max b) { return fmaxf(a, b); }
    static __device__ __forceinline__ float value(Max m) { return m; }
};

template <typename T> constexpr uint32_t kMinusInfBits = sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00u : 0xFF80u;

// A row's elements before the first 16-byte boundary (`head`), the vectors from there, the elements after the last.
// Bit j + shift of the bitmap stands for element j, so that a vector's bits lie in one byte.
template <typename T>
struct RowCut {
    int head, vecs, tail, shift;
    __device__ __forceinline__ RowCut(const T *row, int vocab)
    {
        constexpr int E = Vec<T>::kElems;
        head = (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T));
        head = head < vocab ? head : vocab;
        vecs = (vocab - head) / E;
        tail = vocab - head - vecs * E;
        shift = (E - head) & (E - 1);
    }
};

// One entry of a row's list.
struct Entry {
    int token;       // -1: skipped
    float z;         // the student's logit
    float p;         // the teacher's logit, then its probability
    int first;       // this block's token, and its first entry
};

constexpr int kMaxCluster = 8, kMaxWarps = 8;
constexpr int kBatch = 4;                 // vectors a thread has in flight
constexpr int kThreadsPerSm = 1024;       // what 64 registers a thread leave room for

struct DistillShared {
    unsigned long long exchange;
    Sums part[kMaxWarps];
    Sums theirs[2][kMaxCluster];
    float mass, soft;
    int any, twice, gave_up;
};

// A cluster of `blocks` blocks takes a row, each block a slice of it: one for many rows, up to eight for few.  Pass 1
// reads the row for its sums, pass 2 reads it again (from L2: the rows in flight fit there) and writes the gradient.
// Several blocks share an SM, so that one row's fixed costs - the list's dependent loads, the joins, the coefficients -
// run beside other rows' sums.  The sum over the unlisted tokens is the whole sum less the listed ones, where that is at
// least a 64th of the whole (its rounding error is then below 64 times that of a sum); other rows are summed again with
// the listed tokens left out by a bitmap.
//
// What bounds it, apart from device memory: exponentials, one per element and pass.  exp(z - m) is the square of
// exp((z - m) / 2), so at temperature 2 the hard part needs none of its own (kPower 2), at temperature 1 it is the
// soft part's (kPower 0, also where there is no hard part); other temperatures pay for both (kPower -1).  8192 x 50257
// bfloat16 with labels, loss alone and with the gradient: T = 1 138 and 312 us, T = 2 144 and 320, T = 1.5 or 4 218 and 440;
// binary32 rows are bound by memory at any of them (4096 x 30522: 85 to 88, 208).
//
// Threads a row: 128 for the loss alone, where more rows in flight hide more (8192 x 50257: 138 us, 256 threads 158;
// 8192 x 2000: 35 and 62); 256 with a gradient, where more rows in flight no longer fit L2 between the passes (8192 x 50257
// 312 us, 128 threads 391; 8192 x 30522 alike; on 8192 x 2000, all of whose rows fit, 128 would take 48 for 82).
// kAlone: one block a row.
template <typename T, int kPower, int kThreads, bool kAlone>
__global__ void __launch_bounds__(kThreads, kThreadsPerSm / kThreads) distill_kernel(const DistillArgs a, const int cluster_blocks,
                                                                                     const WaitLimit limit)
{
    const int blocks = kAlone ? 1 : cluster_blocks;
    constexpr int E = Vec<T>::kElems, P = Pairs<T>::kCount, kWarps = kThreads / 32;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ DistillShared sh;
    Entry *list = reinterpret_cast<Entry *>(smem_raw);                                   // [top]
    uint32_t *bits = reinterpret_cast<uint32_t *>(smem_raw + sizeof(Entry) * a.top);     // listed tokens
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const long long row = blockIdx.x / (unsigned)blocks;
    const int rank = (int)(blockIdx.x % (unsigned)blocks);
    const float inv_t = a.inv_t, c = kLog2e * inv_t;
    const T *z = static_cast<const T *>(a.logits) + row * a.ld_logits;
    T *grad = a.grad ? static_cast<T *>(a.grad) + row * a.ld_grad : nullptr;
    const RowCut<T> cut(z, a.vocab);
    // This block's vectors, and the single elements that its first threads take: the head's with the first block, the
    // tail's with the last.
    const int per = (cut.vecs + blocks - 1) / blocks, q0 = min(rank * per, cut.vecs), q1 = min(q0 + per, cut.vecs);
    const int heads = rank == 0 ? cut.head : 0, singles = heads + (rank == blocks - 1 ? cut.tail : 0);
    const int single = tid < heads ? tid : cut.head + cut.vecs * E + tid - heads;        // for tid < singles
    auto mine = [&](int j) {
        return j < cut.head ? rank == 0 : j >= cut.head + cut.vecs * E ? rank == blocks - 1 : (j - cut.head) / E >= q0 && (j - cut.head) / E < q1;
    };
    auto listed_bits = [&](int j) { return bits[(j + cut.shift) >> 5] >> ((j + cut.shift) & 31); };

    // Vectors go kBatch at a time, the next batch's loads in flight beside this one's arithmetic; the first batch of a
    // pass is asked for before the fixed costs that come ahead of it.
    const uint4 *vectors = reinterpret_cast<const uint4 *>(z + cut.head);
    constexpr uint32_t kNone = sizeof(T) == 4 ? kMinusInfBits<T> : kMinusInfBits<T> * 0x10001u;
    constexpr int kStep = kBatch * kThreads;
    const int whole = (q1 - q0) / kStep, batches = (q1 - q0 + kStep - 1) / kStep;       // batches that are whole for all threads; all
    const int last = (q1 - q0 - whole * kStep + kThreads - 1) / kThreads;               // vectors a thread has in a batch that is not, at most
    uint4 ahead[kBatch];          // the batch that is on its way
    auto fetch = [&](int i) {
        const int q = q0 + i * kStep + tid;
        if (i < whole) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) ahead[k] = vectors[q + k * kThreads];
        } else if (i < batches) {
#pragma unroll
            for (int k = 0; k < kBatch; ++k) ahead[k] = q + k * kThreads < q1 ? vectors[q + k * kThreads] : make_uint4(kNone, kNone, kNone, kNone);
        }
    };
    // f(batch, number) for every batch of the row, the next one on its way; the first has been fetched.  (Two batches by
    // turns would save the copies, but the longer loops miss the instruction cache: 334 -> 366 us for 8192 x 50257.)
    auto each_batch = [&](auto f) {
#pragma unroll 1
        for (int i = 0; i < batches; ++i) {
            uint4 word[kBatch];
#pragma unroll
            for (int k = 0; k < kBatch; ++k) word[k] = ahead[k];
            fetch(i + 1);
            f(word, i);
        }
    };

    float w = a.weight ? a.weight[row] : 1.0f;
    if (a.grad_loss) w *= a.grad_loss[row];
    fetch(0);
    if (w == 0.0f) {        // nothing of the row is looked at
        if (grad) {
            const RowCut<T> g(grad, a.vocab);
            const int gper = (g.vecs + blocks - 1) / blocks, g0 = min(rank * gper, g.vecs), g1 = min(g0 + gper, g.vecs);
            for (int q = g0 + tid; q < g1; q += kThreads) reinterpret_cast<uint4 *>(grad + g.head)[q] = make_uint4(0, 0, 0, 0);
            if (rank == 0 && tid < g.head + g.tail) grad[tid < g.head ? tid : g.vecs * E + tid] = from_f32<T>(0.0f);
        }
        if (tid == 0 && rank == 0) {
            if (a.loss) a.loss[row] = 0.0f;
            if (a.stats) reinterpret_cast<float4 *>(a.stats)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return;
    }
    if (tid == 0) {
        sh.twice = 0;
        sh.gave_up = 0;
        if (blocks > 1) {
            mbar_init(smem_addr(&sh.exchange), (uint32_t)blocks);
            mbar_init_done();
        }
    }

    // The list.
    for (int k = tid; k < (a.vocab + E + 31) / 32; k += kThreads) bits[k] = 0;
    for (int k = tid; k < a.top; k += kThreads) {
        const int i = a.index[row * a.top + k];
        const bool ok = i >= 0 && i < a.vocab;
        list[k] = Entry{ok ? i : -1, ok ? to_f32(z[i]) : 0.0f, to_f32(static_cast<const T *>(a.teacher)[row * a.top + k]), 0};
    }
    const int label = a.labels ? a.labels[row] : -1;
    const bool hard = label >= 0 && label < a.vocab;
    const float z_label = hard ? to_f32(z[label]) : 0.0f;
    __syncthreads();
    // From here on other blocks may replace their slices of the row by gradients, once they have waited for this.
    if (blocks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");

    for (int k = tid; k < a.top; k += kThreads) {
        const int i = list[k].token;
        if (i < 0) continue;
        const uint32_t bit = 1u << ((i + cut.shift) & 31);
        if (atomicOr(&bits[(i + cut.shift) >> 5], bit) & bit) sh.twice = 1;
        else list[k].first = mine(i);
    }
    __syncthreads();
    if (sh.twice)         // the earliest entry of a token counts as its first, whichever thread came first: equal calls add in equal order
        for (int k = tid; k < a.top; k += kThreads) {
            const int i = list[k].token;
            bool first = i >= 0 && mine(i);
            for (int o = 0; o < k && first; ++o) first = list[o].token != i;
            list[k].first = first;
        }
    if (warp == kWarps - 1) {          // the teacher's probabilities, by one warp beside the others' sums
        float high = -INFINITY;
        bool some = false;
        for (int k = lane; k < a.top; k += 32)
            if (list[k].token >= 0) {
                some = true;
                high = fmaxf(high, list[k].p);
            }
        int any = __any_sync(0xffffffffu, some);
        // log p = (logit - high) / T - log_norm: without the largest taken off first, logits far from zero would lose their digits
        float log_norm = a.lse ? a.lse[row] : 0.0f;
        high = a.lse ? 0.0f : base_of(warp_max(high));
        if (!a.lse) {
            float sum = 0.0f;
            for (int k = lane; k < a.top; k += 32)
                if (list[k].token >= 0) sum += ex2((list[k].p - high) * c);
            sum = warp_sum(sum);
            if (sum == 0.0f) any = 0;            // a list of -inf says nothing
            log_norm = any ? logf(sum) : 0.0f;
        }
        float mass = 0.0f, soft = 0.0f;
        for (int k = lane; k < a.top; k += 32) {
            const float log_p = (list[k].p - high) * inv_t - log_norm;
            const float p = list[k].token >= 0 && any ? ex2(log_p * kLog2e) : 0.0f;
            list[k].p = p;
            mass += p;
            if (p != 0.0f) soft += p * log_p;
        }
        mass = warp_sum(mass);
        soft = warp_sum(soft);
        if (lane == 0) {
            sh.mass = mass;
            sh.soft = soft;
            sh.any = any;
        }
    }

    // The student's sums.
    Sums t;
    if (a.stats_in) {
        const float4 s4 = reinterpret_cast<const float4 *>(a.stats_in)[row];
        t = Sums{s4.x, s4.y, s4.z, s4.w};
        __syncthreads();
    }
    for (int masked = 0; !a.stats_in; ++masked) {
        // The list's share: where its tokens are left out of the row's sums they are added here, else they are taken from
        // the sum over the rest; each token once.
        t = Sums{-INFINITY, 0.0f, 0.0f, 0.0f};
        if (masked || a.lse)
            for (int k = tid; k < a.top; k += kThreads) {
                if (!list[k].first) continue;
                const float x = list[k].z, one = x == -INFINITY ? 0.0f : 1.0f + 0.0f * x;      // NaN for +inf and NaN
                t = join(t, masked ? Sums{x, one, one, 0.0f} : Sums{x, 0.0f, 0.0f, -one}, c);
            }
        float m = t.m;
        uint64_t minus_m = pair(-base_of(m), -base_of(m)), s2 = pair(0.0f, 0.0f), f2 = s2;
        const uint64_t c2 = pair(c, c), l2 = pair(kLog2e, kLog2e);
        // The base need not be the maximum itself: powers up to 2^40 above it lose nothing in binary32, and the sums are
        // rebased for a logit further above alone (else nearly every vector would, for one lane or other).
        const float slack = 40.0f / fmaxf(c, kLog2e);
        auto rebase = [&](float vm) {
            if (vm > m + slack) {
                const float f = ex2((m - vm) * c), f1 = ex2((m - vm) * kLog2e);
                s2 = mul2(s2, pair(f, f));
                f2 = mul2(f2, pair(f1, f1));
                t.s *= f;
                t.r *= f;
                t.s1 *= f1;
                m = vm;
                minus_m = pair(-m, -m);
            }
        };
        auto take = [&](const uint4 &word) {
            uint64_t x[P];
            Pairs<T>::unpack(word, x);
#pragma unroll
            for (int k = 0; k < P; ++k) {
                const uint64_t d = add2(x[k], minus_m), e = ex2_2(mul2(d, c2));
                s2 = add2(s2, e);
                if (kPower == 2) f2 = fma2(e, e, f2);
                if (kPower == -1) f2 = add2(f2, ex2_2(mul2(d, l2)));
            }
        };
        const uint8_t *vector_bits = reinterpret_cast<const uint8_t *>(bits);
        const int first_bit = cut.head + cut.shift;          // a multiple of E
        auto without_listed = [&](uint4 &word, int q) {       // listed elements as -inf
            const uint32_t in = E == 8 ? vector_bits[(first_bit >> 3) + q] : vector_bits[(first_bit + q * E) >> 3] >> ((first_bit + q * E) & 7) & 15u;
            if (in) {
                uint32_t *x = &word.x;
#pragma unroll
                for (int k = 0; k < E; ++k)
                    if (in >> k & 1) {
                        if (E == 4) x[k] = kNone;
                        else x[k >> 1] = k & 1 ? (x[k >> 1] & 0xFFFFu) | (kNone & 0xFFFF0000u) : (x[k >> 1] & 0xFFFF0000u) | (kNone & 0xFFFFu);
                    }
            }
        };
        if (masked) {
#pragma unroll 1
            for (int q = q0 + tid; q < q1; q += kThreads) {
                uint4 word = vectors[q];
                without_listed(word, q);
                rebase(Pairs<T>::value(Pairs<T>::largest(word)));
                take(word);
            }
        } else {
            each_batch([&](const uint4 (&word)[kBatch], int i) {
                auto vm = Pairs<T>::largest(word[0]);
#pragma unroll
                for (int k = 1; k < kBatch; ++k) vm = Pairs<T>::larger(vm, Pairs<T>::largest(word[k]));
                rebase(Pairs<T>::value(vm));
                const int n = i < whole ? kBatch : last;
#pragma unroll
                for (int k = 0; k < kBatch; ++k)
                    if (k < n) take(word[k]);
            });
        }
        if (tid < singles && !(masked && listed_bits(single) & 1)) {
            const float x = to_f32(z[single]);
            rebase(x);
            const float d = x - base_of(m);
            s2 = add2(s2, pair(ex2(d * c), 0.0f));
            f2 = add2(f2, pair(ex2(d * kLog2e), 0.0f));
        }
        if (grad) fetch(0);
        float lo, hi;
        unpair(s2, lo, hi);
        t.m = m;
        t.r += lo + hi;
        t.s += lo + hi;
        unpair(f2, lo, hi);
        t.s1 = kPower == 0 ? t.s : t.s1 + (lo + hi);
        t = warp_join(t, c);
        if (lane == 0) sh.part[warp] = t;
        __syncthreads();
        t = warp_join(lane < kWarps ? sh.part[lane] : Sums{-INFINITY, 0.0f, 0.0f, 0.0f}, c);
        if (blocks > 1) {      // every block tells every block
            if (!masked) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
            const uint32_t bar = smem_addr(&sh.exchange);
            if (warp == 0 && lane < blocks) {
                uint32_t remote;
                asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(remote) : "r"(smem_addr(&sh.theirs[masked][rank])), "r"(lane));
                asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(remote), "f"(t.m), "f"(t.s), "f"(t.s1), "f"(t.r)
                             : "memory");
                mbar_arrive_at(bar, (uint32_t)lane);
            }
            mbar_wait<true>(bar, (uint32_t)masked, &sh.gave_up, limit);
            t = warp_join(lane < blocks ? sh.theirs[masked][lane] : Sums{-INFINITY, 0.0f, 0.0f, 0.0f}, c);
        }
        if (!masked && a.lse && t.r < t.s * 0.015625f) {
            __syncthreads();          // all have read the parts
            continue;
        }
        t.m = base_of(t.m);
        if (a.stats && tid == 0 && rank == 0) reinterpret_cast<float4 *>(a.stats)[row] = make_float4(t.m, t.s, t.s1, t.r);
        break;
    }
    if (blocks > 1) {          // nobody leaves before the others are done with its memory
        if (a.stats_in) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
        asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
    }

    const bool any = sh.any;
    const bool empty = t.s == 0.0f;      // every token masked out
    const float mass = sh.mass, p_rest = a.lse ? fmaxf(0.0f, 1.0f - mass) : 0.0f;
    const bool rest = p_rest > 0.0f && t.r > kLeastRest * t.s;
    if (a.loss && rank == 0 && warp == 0) {
        const float log_s = logf(t.s);
        float soft = 0.0f;
        for (int k = lane; k < a.top; k += 32)
            if (list[k].p != 0.0f) soft -= list[k].p * ((list[k].z - t.m) * inv_t - log_s);
        soft = warp_sum(soft) + sh.soft;
        if (rest) soft += p_rest * (logf(p_rest) - (logf(t.r) - log_s));
        float loss = any ? a.soft_weight * a.temperature * a.temperature * soft : 0.0f;
        if (hard) loss += a.hard_weight * (logf(t.s1) - (z_label - t.m));
        if (t.s != t.s) loss = t.s;
        if (lane == 0) a.loss[row] = empty ? 0.0f : w * loss;
    }
    if (grad) {
        const float c0 = any ? w * a.soft_weight * a.temperature : 0.0f;
        // (a row whose loss has no term of the rest has none in its gradient)
        const float ca = empty ? 0.0f : c0 * (a.lse || mass != mass ? mass + (rest ? p_rest : 0.0f) : 1.0f) / t.s;
        const float cu = rest && !empty ? ca - c0 * p_rest / t.r : ca;
        const float ch = hard ? w * a.hard_weight : 0.0f;
        const float cb = empty ? 0.0f : ch / t.s1;
        const uint64_t minus_m = pair(-t.m, -t.m), c2 = pair(c, c), l2 = pair(kLog2e, kLog2e);
        // temperature 1, or no hard part at all: the two exponentials are one
        const float cu_all = kPower == 0 ? cu + cb : cu;
        const uint64_t cu2 = pair(cu_all, cu_all), cb2 = pair(cb, cb);
        const bool same = ((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0;
        each_batch([&](const uint4 (&word)[kBatch], int i) {
            const int q = q0 + i * kStep + tid;
#pragma unroll
            for (int h = 0; h < kBatch; ++h) {
                if (i >= whole && q + h * kThreads >= q1) break;
                uint64_t x[P];
                Pairs<T>::unpack(word[h], x);
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    const uint64_t d = add2(x[k], minus_m), e = ex2_2(mul2(d, c2));
                    if (kPower == 0) x[k] = mul2(cu2, e);
                    if (kPower == 2) x[k] = mul2(e, fma2(cb2, e, cu2));
                    if (kPower == -1) x[k] = fma2(cb2, ex2_2(mul2(d, l2)), mul2(cu2, e));
                }
                if (same) {
                    __stcs(reinterpret_cast<uint4 *>(grad + cut.head) + q + h * kThreads, Pairs<T>::pack(x));
                } else {
                    T *g = grad + cut.head + (q + h * kThreads) * E;
#pragma unroll
                    for (int k = 0; k < P; ++k) {
                        float lo, hi;
                        unpair(x[k], lo, hi);
                        g[2 * k] = from_f32<T>(lo);
                        g[2 * k + 1] = from_f32<T>(hi);
                    }
                }
            }
        });
        if (tid < singles) {
            const float d = to_f32(z[single]) - t.m;
            grad[single] = from_f32<T>(cu * ex2(d * c) + cb * ex2(d * kLog2e));
        }
        __syncthreads();
        // Listed tokens and the label, in binary32 from their own logits, over what has been stored there.
        const bool twice = sh.twice;
        for (int k = tid; k < a.top; k += kThreads) {
            const int i = list[k].token;
            if (i < 0 || !mine(i)) continue;
            float p = list[k].p;
            if (twice) {       // all its entries together, in the same order for each of them
                p = 0.0f;
                for (int o = 0; o < a.top; ++o) p += list[o].token == i ? list[o].p : 0.0f;
            }
            const float d = list[k].z - t.m;
            float g = ca * ex2(d * c) - c0 * p + cb * ex2(d * kLog2e);
            if (i == label) g -= ch;
            grad[i] = from_f32<T>(empty ? 0.0f : g);
        }
        if (hard && tid == 0 && mine(label) && !(listed_bits(label) & 1)) {
            const float d = z_label - t.m;
            grad[label] = from_f32<T>(empty ? 0.0f : cu * ex2(d * c) + cb * ex2(d * kLog2e) - ch);
        }
    }
    if (blocks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

template <typename T, int kPower, int kThreads, bool kAlone>
void launch_kernel(const DistillArgs &a, int blocks, const WaitLimit &wait_limit, cudaStream_t s)
{
    static SmemLimit limit;
    auto kernel = distill_kernel<T, kPower, kThreads, kAlone>;
    if (limit.ensure(kernel, (int)(kMaxTop * sizeof(Entry) + kMaxVocab / 8 + 64)) != cudaSuccess) return;     // the caller reports it
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)(a.rows * blocks));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = sizeof(Entry) * (size_t)a.top + (size_t)(a.vocab + Vec<T>::kElems + 31) / 32 * 4;
    cfg.stream = s;
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {(unsigned)blocks, 1, 1};
    cfg.attrs = &at;
    cfg.numAttrs = blocks > 1;
    cudaLaunchKernelEx(&cfg, kernel, a, blocks, wait_limit);
}

zoa_status launch(const char *me, const zoa_distill_args *x, const float *stats_in, const float *grad_loss, float *loss, float *stats,
                  void *grad, size_t ld_grad, void *stream)
{
    if (ops_gave_up()) return ops_refuse(me);
    if (!x) return ops_fail(ZOA_ERR_ARG, "%s: args is NULL", me);
    if (!dtype_ok(x->dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, x->dtype);
    if (x->vocab < 1 || x->vocab > kMaxVocab) return ops_fail(ZOA_ERR_ARG, "%s: vocab must be in [1, 2^20]", me);
    if (x->top < 1 || x->top > kMaxTop) return ops_fail(ZOA_ERR_ARG, "%s: top must be in [1, 2048]", me);
    if (x->rows > ((size_t)1 << 31) - 1) return ops_fail(ZOA_ERR_ARG, "%s: at most 2^31 - 1 rows", me);
    if (x->ld_logits < x->vocab || (grad && ld_grad < x->vocab)) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least vocab", me);
    if (!(x->temperature >= FLT_MIN) || x->temperature * 0.0f != 0.0f)      // so that 1 / T and its product with log2 e are finite
        return ops_fail(ZOA_ERR_ARG, "%s: temperature must be positive, finite and not subnormal", me);
    if (!(x->soft_weight * 0.0f == 0.0f) || !(x->hard_weight * 0.0f == 0.0f))
        return ops_fail(ZOA_ERR_ARG, "%s: soft_weight and hard_weight must be finite", me);
    if (x->rows == 0) return ZOA_OK;
    if (!x->logits || !x->index || !x->teacher) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    const size_t e = dtype_bytes(x->dtype);
    if (reinterpret_cast<uintptr_t>(x->logits) % e || reinterpret_cast<uintptr_t>(x->teacher) % e || reinterpret_cast<uintptr_t>(grad) % e)
        return ops_fail(ZOA_ERR_ARG, "%s: a matrix is not aligned to its element type", me);
    const uintptr_t words = reinterpret_cast<uintptr_t>(x->index) | reinterpret_cast<uintptr_t>(x->teacher_lse) | reinterpret_cast<uintptr_t>(x->labels) |
                            reinterpret_cast<uintptr_t>(x->row_weight) | reinterpret_cast<uintptr_t>(loss) | reinterpret_cast<uintptr_t>(grad_loss);
    if (words % 4) return ops_fail(ZOA_ERR_ARG, "%s: a vector or the list is not 4-byte aligned", me);
    if (!aligned16(stats) || !aligned16(stats_in)) return ops_fail(ZOA_ERR_ARG, "%s: stats must be 16-byte aligned", me);
    if (grad == x->logits && ld_grad != x->ld_logits)
        return ops_fail(ZOA_ERR_ARG, "%s: a gradient that replaces the logits has their ld", me);
    cudaStream_t s = static_cast<cudaStream_t>(stream);
    DistillArgs a{};
    a.logits = x->logits;
    a.index = x->index;
    a.teacher = x->teacher;
    a.lse = x->teacher_lse;
    a.labels = x->labels;
    a.weight = x->row_weight;
    a.grad_loss = grad_loss;
    a.stats_in = stats_in;
    a.loss = loss;
    a.stats = stats;
    a.grad = grad;
    a.rows = (long long)x->rows;
    a.ld_logits = (long long)x->ld_logits;
    a.ld_grad = (long long)ld_grad;
    a.vocab = (int)x->vocab;
    a.top = (int)x->top;
    a.temperature = x->temperature;
    a.inv_t = 1.0f / x->temperature;
    a.soft_weight = x->soft_weight;
    a.hard_weight = x->hard_weight;
    const int sms = ops_sm_count();
    WaitLimit wait_limit{ops_error_word(), ops_wait_limit_ns()};
    if (sms < 1 || !wait_limit.error_word) return ops_fail(ZOA_ERR_CUDA, "%s: no usable current device", me);
    // Blocks for a row: more while all of them fit the device at once (four to an SM) and a slice stays above 4 KB.
    int blocks = 1;
    while (blocks < kMaxCluster && a.rows * blocks * 2 <= 4 * sms && (size_t)a.vocab * e / (blocks * 2) >= 4096) blocks *= 2;
    if (a.rows * blocks > 0x7FFFFFFFll) return ops_fail(ZOA_ERR_ARG, "%s: at most 2^31 - 1 rows", me);
    with_type(x->dtype, [&](auto t) {
        using T = decltype(t);
        const int power = a.temperature == 1.0f || !a.labels ? 0 : a.temperature == 2.0f ? 2 : -1;
        auto go = [&](auto p) {
            constexpr int kPower = decltype(p)::value;
            if (blocks > 1) launch_kernel<T, kPower, 256, false>(a, blocks, wait_limit, s);
            else if (a.grad) launch_kernel<T, kPower, 256, true>(a, 1, wait_limit, s);
            else launch_kernel<T, kPower, 128, true>(a, 1, wait_limit, s);
        };
        if (power == 0) go(std::integral_constant<int, 0>{});
        else if (power == 2) go(std::integral_constant<int, 2>{});
        else go(std::integral_constant<int, -1>{});
    });
    return ops_launched(me);
}

}  // namespace
}  // namespace zoa

using namespace zoa;

extern "C" zoa_status zoa_distill_topk(const zoa_distill_args *args, float *loss, float *stats, void *grad, size_t ld_grad, void *stream)
{
    if (args && args->rows && !loss && !stats && !grad) return ops_fail(ZOA_ERR_ARG, "zoa_distill_topk: no output asked for");
    return launch("zoa_distill_topk", args, nullptr, nullptr, loss, stats, grad, ld_grad, stream);
}

extern "C" zoa_status zoa_distill_topk_backward(const zoa_distill_args *args, const float *stats, const float *grad_loss, void *grad,
                                                size_t ld_grad, void *stream)
{
    if (args && args->rows && (!stats || !grad_loss || !grad)) return ops_fail(ZOA_ERR_ARG, "zoa_distill_topk_backward: a NULL pointer");
    return launch("zoa_distill_topk_backward", args, stats, grad_loss, nullptr, nullptr, grad, ld_grad, stream);
}
