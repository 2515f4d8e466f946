// The handle of a kernel on the device of a stream, and a launch by it.
#ifndef ECSPMV_KERNEL_HANDLE_H
#define ECSPMV_KERNEL_HANDLE_H

#include <hip/hip_runtime.h>
#include <atomic>
#include <cstddef>
#include <cstdint>

namespace ecs {

// handle of a kernel on the device of `stream` (the null stream: the current one), which need not be the current device;
// asked for once per device and kept as long as the library is loaded
template <auto KERNEL>
static int kernel_handle(void *stream, hipFunction_t *f)
{
    constexpr int kMaxDev = 64;
    static std::atomic<hipFunction_t> cached[kMaxDev];
    int current = 0, dev = 0;
    hipError_t e = hipGetDevice(&current);
    if (e != hipSuccess) return (int)e;
    dev = current;
    if (stream) e = hipStreamGetDevice((hipStream_t)stream, &dev);
    if (e != hipSuccess) return (int)e;
    const bool keep = dev >= 0 && dev < kMaxDev;
    if (keep) *f = cached[dev].load(std::memory_order_acquire);
    if (*f) return 0;
    if (dev != current) e = hipSetDevice(dev);             // symbols are looked up on the current device
    if (e != hipSuccess) return (int)e;
    e = hipGetFuncBySymbol(f, reinterpret_cast<const void *>(KERNEL));
    if (dev != current) {
        const hipError_t back = hipSetDevice(current);
        if (e == hipSuccess) e = back;
    }
    if (e != hipSuccess) return (int)e;
    if (keep) cached[dev].store(*f, std::memory_order_release);
    return 0;
}

// one launch of a kernel whose only parameter is an Args, handed over as it lies in memory; LDS is the kernel's own
template <auto KERNEL, class Args>
static int launch_args(const Args &args, uint32_t gx, uint32_t gy, uint32_t gz, uint32_t threads, void *stream)
{
    hipFunction_t f = nullptr;
    const int e = kernel_handle<KERNEL>(stream, &f);
    if (e) {
        (void)hipGetLastError();                           // the caller has it; not left behind for others
        return e;
    }
    size_t bytes = sizeof(Args);
    void *extra[] = {HIP_LAUNCH_PARAM_BUFFER_POINTER, const_cast<Args *>(&args), HIP_LAUNCH_PARAM_BUFFER_SIZE, &bytes, HIP_LAUNCH_PARAM_END};
    const hipError_t s = hipModuleLaunchKernel(f, gx, gy, gz, threads, 1, 1, 0, (hipStream_t)stream, nullptr, extra);
    if (s != hipSuccess) (void)hipGetLastError();
    return (int)s;
}

}  // namespace ecs
#endif
