// Shared by the operators that need no handle (4-bit microscaled tensors, distillation): the thread's
// error text, launch checks, element types, and the option words of zoa_ops_set_option.
#pragma once

#include <atomic>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/zoa.h"

namespace zoa {

// Sets the text of zoa_ops_last_error for this thread and returns `s` (a fixed buffer: nothing here can throw).
zoa_status ops_fail(zoa_status s, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
// cudaGetLastError after a launch of `what`.
zoa_status ops_launched(const char *what);
// SMs of the current device (cached); 0 if the device cannot be asked.
int ops_sm_count();
// The device's address of the current device's word that a kernel sets when a bounded wait ran out; NULL if it cannot be had.
int *ops_error_word();
// Whether a kernel has set it since zoa_ops_check_device last cleared it: every call that enqueues then returns ops_refuse.
bool ops_gave_up();
zoa_status ops_refuse(const char *what);
// ZOA_OPT_WAIT_LIMIT_MS in nanoseconds and ZOA_OPT_TEST_STOP_AFTER_TILES, as zoa_ops_set_option last left them.
unsigned long long ops_wait_limit_ns();
int ops_test_stop();

// Raises a kernel's dynamic shared-memory limit the first time it is needed on a device; one object per kernel.
struct SmemLimit {
    std::atomic<int> have[64] = {};
    template <typename Kernel>
    cudaError_t ensure(Kernel kern, int bytes)
    {
        int dev = 0;
        const cudaError_t e = cudaGetDevice(&dev);
        if (e != cudaSuccess) return e;
        if (dev >= 0 && dev < 64 && have[dev].load(std::memory_order_acquire) >= bytes) return cudaSuccess;
        const cudaError_t f = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (f == cudaSuccess && dev >= 0 && dev < 64) have[dev].store(bytes, std::memory_order_release);
        return f;
    }
};

inline bool dtype_ok(int t) { return t == ZOA_F32 || t == ZOA_F16 || t == ZOA_BF16; }
inline size_t dtype_bytes(int t) { return t == ZOA_F32 ? 4 : 2; }
inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Calls f with a value of the element type `t` (checked before with dtype_ok).
template <typename F>
inline void with_type(int t, F f)
{
    if (t == ZOA_F32) f(float{});
    else if (t == ZOA_F16) f(__half{});
    else f(__nv_bfloat16{});
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
// One rounding (to nearest even) on the way out; halves above 65504 become infinite as in any conversion.
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Two values as one 32-bit word of a 16-bit type, `lo` first in memory.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <typename T> __device__ __forceinline__ void unpack2(uint32_t w, float &lo, float &hi);
template <> __device__ __forceinline__ void unpack2<__half>(uint32_t w, float &lo, float &hi)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
    lo = f.x;
    hi = f.y;
}
template <> __device__ __forceinline__ void unpack2<__nv_bfloat16>(uint32_t w, float &lo, float &hi)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}

// A 16-byte vector of T (8 or 4 elements) from binary32.
template <typename T>
struct Vec {
    static constexpr int kElems = 16 / (int)sizeof(T);
    static __device__ __forceinline__ uint4 pack(const float *v)
    {
        return make_uint4(pack2<T>(v[0], v[1]), pack2<T>(v[2], v[3]), pack2<T>(v[4], v[5]), pack2<T>(v[6], v[7]));
    }
};
template <>
struct Vec<float> {
    static constexpr int kElems = 4;
    static __device__ __forceinline__ uint4 pack(const float *v)
    {
        return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
    }
};

}  // namespace zoa
