// State shared by the handle-free operators: error text, device facts, options, the device-side error word.
#include "zoa_ops.h"

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <mutex>

namespace zoa {

static thread_local char t_error[320] = "";
static std::atomic<int> g_wait_limit_ms{2000};
static std::atomic<int> g_test_stop{0};
static __device__ int g_ops_error = 0;

zoa_status ops_fail(zoa_status s, const char *fmt, ...)
{
    va_list args;
    va_start(args, fmt);
    vsnprintf(t_error, sizeof t_error, fmt, args);
    va_end(args);
    return s;
}

zoa_status ops_launched(const char *what)
{
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ZOA_OK : ops_fail(ZOA_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

int ops_sm_count()
{
    static std::atomic<int> count[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return 0;
    int n = count[dev].load(std::memory_order_relaxed);
    if (n == 0 && cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess)
        count[dev].store(n, std::memory_order_relaxed);
    return n;
}

int *ops_error_word()
{
    static std::atomic<int *> word[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return nullptr;
    int *p = word[dev].load(std::memory_order_acquire);
    if (!p) {
        void *q = nullptr;
        if (cudaGetSymbolAddress(&q, g_ops_error) != cudaSuccess) return nullptr;
        p = static_cast<int *>(q);
        word[dev].store(p, std::memory_order_release);
    }
    return p;
}

unsigned long long ops_wait_limit_ns() { return 1000000ull * (unsigned long long)g_wait_limit_ms.load(); }
int ops_test_stop() { return g_test_stop.load(); }

}  // namespace zoa

using namespace zoa;

extern "C" const char *zoa_ops_last_error(void) { return t_error; }

extern "C" zoa_status zoa_ops_set_option(int option, int value)
{
    if (option == ZOA_OPT_WAIT_LIMIT_MS && value >= 1) {
        g_wait_limit_ms = value;
        return ZOA_OK;
    }
    if (option == ZOA_OPT_TEST_STOP_AFTER_TILES && value >= 0) {
        g_test_stop = value;
        return ZOA_OK;
    }
    return ops_fail(ZOA_ERR_ARG, "zoa_ops_set_option: unknown option %d or bad value %d", option, value);
}

extern "C" zoa_status zoa_ops_check_device(void)
{
    int *word = ops_error_word();
    cudaError_t e = cudaDeviceSynchronize();
    int set = 0;
    if (e == cudaSuccess && word) e = cudaMemcpy(&set, word, sizeof set, cudaMemcpyDeviceToHost);
    if (e != cudaSuccess || !word) return ops_fail(ZOA_ERR_CUDA, "zoa_ops_check_device: %s", cudaGetErrorString(e));
    if (!set) return ZOA_OK;
    set = 0;
    e = cudaMemcpy(word, &set, sizeof set, cudaMemcpyHostToDevice);
    if (e != cudaSuccess) return ops_fail(ZOA_ERR_CUDA, "zoa_ops_check_device: %s", cudaGetErrorString(e));
    return ops_fail(ZOA_ERR_DEVICE, "a kernel gave up on a bounded wait; its result is undefined");
}
