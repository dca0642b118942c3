// State shared by the handle-free operators: error text, device facts, options, the device-side error word.
#include "zoa_ops.h"

#include <atomic>
#include <cstdarg>
#include <cstdio>
#include <new>

namespace zoa {

static thread_local char t_error[320] = "";
static std::atomic<int> g_wait_limit_ms{2000};
static std::atomic<int> g_test_stop{0};

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

// A word of pinned, mapped host memory for each device, made once and kept: kernels set it, the host reads it without
// synchronising.
struct ErrorWord {
    volatile int *host;
    int *device;
};
static std::atomic<ErrorWord *> g_words[64];
static std::atomic<ErrorWord *> *word_of_device()
{
    int dev = 0;
    return cudaGetDevice(&dev) == cudaSuccess && dev >= 0 && dev < 64 ? &g_words[dev] : nullptr;
}

int *ops_error_word()
{
    std::atomic<ErrorWord *> *at = word_of_device();
    if (!at) return nullptr;
    ErrorWord *word = at->load(std::memory_order_acquire);
    if (word) return word->device;
    void *host = nullptr, *device = nullptr;
    word = new (std::nothrow) ErrorWord;
    if (!word || cudaHostAlloc(&host, sizeof(int), cudaHostAllocMapped | cudaHostAllocPortable) != cudaSuccess ||
        cudaHostGetDevicePointer(&device, host, 0) != cudaSuccess) {
        if (host) cudaFreeHost(host);
        delete word;
        return nullptr;
    }
    *word = ErrorWord{static_cast<int *>(host), static_cast<int *>(device)};
    *word->host = 0;
    ErrorWord *other = nullptr;
    if (at->compare_exchange_strong(other, word, std::memory_order_acq_rel)) return word->device;
    cudaFreeHost(host);          // another thread was first
    delete word;
    return other->device;
}

bool ops_gave_up()
{
    const std::atomic<ErrorWord *> *at = word_of_device();
    const ErrorWord *word = at ? at->load(std::memory_order_acquire) : nullptr;
    return word && *word->host != 0;
}
zoa_status ops_refuse(const char *what)
{
    return ops_fail(ZOA_ERR_DEVICE, "%s: an earlier kernel gave up on a bounded wait; its result is undefined (zoa_ops_check_device clears this)", what);
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
    const cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return ops_fail(ZOA_ERR_CUDA, "zoa_ops_check_device: %s", cudaGetErrorString(e));
    if (!ops_gave_up()) return ZOA_OK;
    *word_of_device()->load(std::memory_order_acquire)->host = 0;
    return ops_fail(ZOA_ERR_DEVICE, "a kernel gave up on a bounded wait; its result is undefined");
}
