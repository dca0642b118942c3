// Distillation from a teacher's top logits: loss, its gradient, or both (the mathematics stands at
// zoa_distill_topk in include/zoa.h).
//
// With m the row's largest logit, e_j = exp((z_j - m) / T) and f_j = exp(z_j - m), everything a row needs is
//   m,  s = sum e_j,  s1 = sum f_j,  r = sum of e_j over unlisted j
// and the gradient is, for coefficients that are the same for the whole row,
//   unlisted j: cu e_j + cb f_j        listed j: ca e_j - c0 p_j + cb f_j        label: - ch more.
#include "zoa_ops.h"

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
struct Sums {
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
__device__ __forceinline__ Sums shuffle_join(Sums a, float c)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        Sums b;
        b.m = __shfl_xor_sync(0xffffffffu, a.m, o);
        b.s = __shfl_xor_sync(0xffffffffu, a.s, o);
        b.s1 = __shfl_xor_sync(0xffffffffu, a.s1, o);
        b.r = __shfl_xor_sync(0xffffffffu, a.r, o);
        a = join(a, b, c);
    }
    return a;
}

template <int kWarps>
__device__ __forceinline__ float block_sum(float v, float *scratch)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) t += scratch[w];
    return t;
}
template <int kWarps>
__device__ __forceinline__ float block_max(float v, float *scratch)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    __syncthreads();
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    float t = scratch[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) t = fmaxf(t, scratch[w]);
    return t;
}

// A row cut into 16-byte vectors: `head` elements before the first aligned address, then `vecs` vectors, then
// `tail` elements.  Bit j + shift of the bitmap stands for element j, so that a vector's bits start at a multiple
// of its length.
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

constexpr int kStreamThreads = 512, kStreamWarps = kStreamThreads / 32;

// One block per row; the row is read once for the sums and once more, from L2, for the gradient.
template <typename T>
__global__ void __launch_bounds__(kStreamThreads) distill_stream_kernel(const DistillArgs a)
{
    constexpr int E = Vec<T>::kElems;
    extern __shared__ __align__(16) unsigned char smem_raw[];
    __shared__ float scratch[32];
    __shared__ Sums part[kStreamWarps];
    float *p_s = reinterpret_cast<float *>(smem_raw);                  // [top] teacher's probability, 0 for a skipped entry
    float *z_s = p_s + a.top;                                          // [top] student's logit there
    int *i_s = reinterpret_cast<int *>(z_s + a.top);                   // [top] token, -1 for a skipped entry
    uint32_t *bits = reinterpret_cast<uint32_t *>(i_s + a.top);        // listed tokens
    const long long row = blockIdx.x;
    const int tid = threadIdx.x;
    const float inv_t = a.inv_t, c = kLog2e * inv_t;
    const T *z = static_cast<const T *>(a.logits) + row * a.ld_logits;
    T *grad = a.grad ? static_cast<T *>(a.grad) + row * a.ld_grad : nullptr;
    float w = a.weight ? a.weight[row] : 1.0f;
    if (a.grad_loss) w *= a.grad_loss[row];
    const RowCut<T> cut(z, a.vocab);
    const bool same = grad && (((reinterpret_cast<uintptr_t>(grad) ^ reinterpret_cast<uintptr_t>(z)) & 15) == 0);

    if (w == 0.0f) {        // nothing of the row is looked at
        if (grad)
            for (int j = tid; j < a.vocab; j += kStreamThreads) grad[j] = from_f32<T>(0.0f);
        if (tid == 0) {
            if (a.loss) a.loss[row] = 0.0f;
            if (a.stats) reinterpret_cast<float4 *>(a.stats)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
        }
        return;
    }

    // The teacher's list.
    const int words = (a.vocab + E + 31) / 32;
    for (int k = tid; k < words; k += kStreamThreads) bits[k] = 0;
    float high = -INFINITY;
    int any = 0;
    for (int k = tid; k < a.top; k += kStreamThreads) {
        const int i = a.index[row * a.top + k];
        const bool ok = i >= 0 && i < a.vocab;
        const float t = to_f32(static_cast<const T *>(a.teacher)[row * a.top + k]);
        i_s[k] = ok ? i : -1;
        p_s[k] = t;
        z_s[k] = ok ? to_f32(z[i]) : 0.0f;
        if (ok) {
            high = fmaxf(high, t);
            any = 1;
        }
    }
    any = __syncthreads_or(any);
    int twice = 0;           // a token is listed more than once
    for (int k = tid; k < a.top; k += kStreamThreads)
        if (i_s[k] >= 0) {
            const uint32_t bit = 1u << ((i_s[k] + cut.shift) & 31);
            twice |= (atomicOr(&bits[(i_s[k] + cut.shift) >> 5], bit) & bit) != 0;
        }
    twice = __syncthreads_or(twice);
    float log_norm;          // log of the teacher's normaliser at temperature T
    if (a.lse) {
        log_norm = a.lse[row];
    } else {
        high = base_of(block_max<kStreamWarps>(high, scratch));
        float sum = 0.0f;
        for (int k = tid; k < a.top; k += kStreamThreads)
            if (i_s[k] >= 0) sum += ex2((p_s[k] - high) * c);
        sum = block_sum<kStreamWarps>(sum, scratch);
        if (sum == 0.0f) any = 0;            // a list of -inf says nothing
        log_norm = any ? logf(sum) + high * inv_t : 0.0f;
    }
    float mass = 0.0f, soft = 0.0f;      // sum p; sum p (log p - (z_k - m) / T) without the student's part yet
    for (int k = tid; k < a.top; k += kStreamThreads) {
        const float log_p = p_s[k] * inv_t - log_norm;
        const float p = i_s[k] >= 0 ? ex2(log_p * kLog2e) : 0.0f;
        p_s[k] = p;
        mass += p;
        if (p > 0.0f) soft += p * log_p;
        else if (p != p) soft += p;
    }
    mass = block_sum<kStreamWarps>(mass, scratch);
    const float p_rest = a.lse ? fmaxf(0.0f, 1.0f - mass) : 0.0f;

    // The student's sums.
    Sums t{-INFINITY, 0.0f, 0.0f, 0.0f};
    if (a.stats_in) {
        const float4 s4 = reinterpret_cast<const float4 *>(a.stats_in)[row];
        t = Sums{s4.x, s4.y, s4.z, s4.w};
    } else {
        auto take = [&](const float *v, uint32_t listed, int n) {
            float vm = v[0];
            for (int k = 1; k < n; ++k) vm = fmaxf(vm, v[k]);
            if (vm > t.m) {
                const float f = ex2((t.m - vm) * c);
                t.s *= f;
                t.r *= f;
                t.s1 *= ex2((t.m - vm) * kLog2e);
                t.m = vm;
            }
            const float b = base_of(t.m);
            for (int k = 0; k < n; ++k) {
                const float e = ex2((v[k] - b) * c);
                t.s += e;
                if (!(listed >> k & 1)) t.r += e;
                t.s1 += ex2((v[k] - b) * kLog2e);
            }
        };
        for (int q = tid; q < cut.vecs; q += kStreamThreads) {
            const int j = cut.head + q * E;
            float v[E];
            Vec<T>::unpack(*reinterpret_cast<const uint4 *>(z + j), v);
            take(v, bits[(j + cut.shift) >> 5] >> ((j + cut.shift) & 31), E);
        }
        for (int x = tid; x < cut.head + cut.tail; x += kStreamThreads) {
            const int j = x < cut.head ? x : cut.vecs * E + x;
            const float v = to_f32(z[j]);
            take(&v, bits[(j + cut.shift) >> 5] >> ((j + cut.shift) & 31), 1);
        }
        t = shuffle_join(t, c);
        if ((tid & 31) == 0) part[tid >> 5] = t;
        __syncthreads();
        t = part[0];
        for (int k = 1; k < kStreamWarps; ++k) t = join(t, part[k], c);
        t.m = base_of(t.m);
    }
    const int label = a.labels ? a.labels[row] : -1;
    const bool hard = label >= 0 && label < a.vocab;
    const bool empty = t.s == 0.0f;      // every token masked out
    const bool rest = p_rest > 0.0f && t.r > kLeastRest * t.s;
    const float log_s = logf(t.s);
    if (a.stats && tid == 0) reinterpret_cast<float4 *>(a.stats)[row] = make_float4(t.m, t.s, t.s1, t.r);
    if (a.loss) {
        for (int k = tid; k < a.top; k += kStreamThreads)
            if (p_s[k] > 0.0f) soft -= p_s[k] * ((z_s[k] - t.m) * inv_t - log_s);
        soft = block_sum<kStreamWarps>(soft, scratch);
        if (rest) soft += p_rest * (logf(p_rest) - (logf(t.r) - log_s));
        float loss = any ? a.soft_weight * a.temperature * a.temperature * soft : 0.0f;
        if (hard) loss += a.hard_weight * (logf(t.s1) - (to_f32(z[label]) - t.m));
        if (t.s != t.s) loss = t.s;
        if (tid == 0) a.loss[row] = empty ? 0.0f : w * loss;
    }
    if (!grad) return;
    __syncthreads();
    const float z_label = hard ? to_f32(z[label]) : 0.0f;
    const float c0 = any ? w * a.soft_weight * a.temperature : 0.0f;
    const float ca = empty ? 0.0f : c0 * (a.lse ? mass + p_rest : 1.0f) / t.s;
    const float cu = rest && !empty ? ca - c0 * p_rest / t.r : ca;
    const float ch = hard ? w * a.hard_weight : 0.0f;
    const float cb = empty ? 0.0f : ch / t.s1;
    const float nan = t.s != t.s ? t.s : 0.0f;     // a NaN row is NaN throughout
    __syncthreads();                               // z_label has been read before grad may replace it
    for (int q = tid; q < cut.vecs; q += kStreamThreads) {
        const int j = cut.head + q * E;
        float v[E];
        Vec<T>::unpack(*reinterpret_cast<const uint4 *>(z + j), v);
#pragma unroll
        for (int k = 0; k < E; ++k) {
            const float d = v[k] - t.m;
            v[k] = cu * ex2(d * c) + (hard ? cb * ex2(d * kLog2e) : 0.0f) + nan;
        }
        if (same) {
            *reinterpret_cast<uint4 *>(grad + j) = Vec<T>::pack(v);
        } else {
#pragma unroll
            for (int k = 0; k < E; ++k) grad[j + k] = from_f32<T>(v[k]);
        }
    }
    for (int x = tid; x < cut.head + cut.tail; x += kStreamThreads) {
        const int j = x < cut.head ? x : cut.vecs * E + x;
        const float d = to_f32(z[j]) - t.m;
        grad[j] = from_f32<T>(cu * ex2(d * c) + (hard ? cb * ex2(d * kLog2e) : 0.0f) + nan);
    }
    __syncthreads();
    // Listed tokens and the label, in binary32 from their own logits, over what the loops above stored there.
    for (int k = tid; k < a.top; k += kStreamThreads) {
        const int i = i_s[k];
        if (i < 0) continue;
        const float d = z_s[k] - t.m;
        float p = p_s[k];
        if (twice) {         // all its entries together, in the same order for each of them
            p = 0.0f;
            for (int o = 0; o < a.top; ++o) p += i_s[o] == i ? p_s[o] : 0.0f;
        }
        float v = ca * ex2(d * c) - c0 * p + (hard ? cb * ex2(d * kLog2e) : 0.0f) + nan;
        if (i == label) v -= ch;
        grad[i] = from_f32<T>(empty ? 0.0f : v);
    }
    if (hard && tid == 0 && !(bits[(label + cut.shift) >> 5] >> ((label + cut.shift) & 31) & 1)) {
        const float d = z_label - t.m;
        grad[label] = from_f32<T>(empty ? 0.0f : cu * ex2(d * c) + cb * ex2(d * kLog2e) - ch + nan);
    }
}

zoa_status launch(const char *me, const zoa_distill_args *x, const float *stats_in, const float *grad_loss, float *loss, float *stats,
                  void *grad, size_t ld_grad, void *stream)
{
    if (!x) return ops_fail(ZOA_ERR_ARG, "%s: args is NULL", me);
    if (!dtype_ok(x->dtype)) return ops_fail(ZOA_ERR_ARG, "%s: unknown element type %d", me, x->dtype);
    if (x->vocab < 1 || x->vocab > kMaxVocab) return ops_fail(ZOA_ERR_ARG, "%s: vocab must be in [1, 2^20]", me);
    if (x->top < 1 || x->top > kMaxTop) return ops_fail(ZOA_ERR_ARG, "%s: top must be in [1, 2048]", me);
    if (x->rows > ((size_t)1 << 31) - 1) return ops_fail(ZOA_ERR_ARG, "%s: at most 2^31 - 1 rows", me);
    if (x->ld_logits < x->vocab || (grad && ld_grad < x->vocab)) return ops_fail(ZOA_ERR_ARG, "%s: ld must be at least vocab", me);
    if (!(x->temperature > 0.0f) || x->temperature * 0.0f != 0.0f) return ops_fail(ZOA_ERR_ARG, "%s: temperature must be positive and finite", me);
    if (!(x->soft_weight * 0.0f == 0.0f) || !(x->hard_weight * 0.0f == 0.0f))
        return ops_fail(ZOA_ERR_ARG, "%s: soft_weight and hard_weight must be finite", me);
    if (x->rows == 0) return ZOA_OK;
    if (!x->logits || !x->index || !x->teacher) return ops_fail(ZOA_ERR_ARG, "%s: a NULL pointer", me);
    const size_t e = dtype_bytes(x->dtype);
    if (reinterpret_cast<uintptr_t>(x->logits) % e || reinterpret_cast<uintptr_t>(x->teacher) % e || reinterpret_cast<uintptr_t>(grad) % e)
        return ops_fail(ZOA_ERR_ARG, "%s: a matrix is not aligned to its element type", me);
    if (!aligned16(stats) || !aligned16(stats_in)) return ops_fail(ZOA_ERR_ARG, "%s: stats must be 16-byte aligned", me);
    if (grad == x->logits && ld_grad != x->ld_logits)
        return ops_fail(ZOA_ERR_ARG, "%s: a gradient that replaces the logits has their ld", me);
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
    with_type(x->dtype, [&](auto t) {
        using T = decltype(t);
        const int smem = a.top * 12 + (a.vocab + Vec<T>::kElems + 31) / 32 * 4;
        static SmemLimit limit;
        if (limit.ensure(distill_stream_kernel<T>, (int)(kMaxTop * 12 + kMaxVocab / 8 + 64)) != cudaSuccess) return;
        distill_stream_kernel<T><<<(unsigned)a.rows, kStreamThreads, smem, static_cast<cudaStream_t>(stream)>>>(a);
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
