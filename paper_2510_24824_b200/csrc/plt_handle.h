// What the handles of the rotation, the draft verification and the shared prefixes have in common: the message of the last
// error, the device they live on and the status word their kernels set bits in.
#pragma once
#include <cuda_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "plt_host.h"

namespace plt {

struct HandleBase {
    int device = 0;
    uint32_t* status = nullptr;
    char err[512] = "";
};

// `none`: where a failure without a handle leaves its message (a thread's own).
inline plt_status handle_fail(HandleBase* h, char* none, plt_status code, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(h ? h->err : none, 512, fmt, ap);
    va_end(ap);
    return code;
}

// cudaSuccess and an sm_100 device, or why not (the device is made current by the caller).
inline plt_status check_device(int device, char* none, int* sms) {
    cudaDeviceProp prop;
    const cudaError_t e = cudaGetDeviceProperties(&prop, device);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();
        return handle_fail(nullptr, none, PLT_ERR_CUDA, "cudaGetDeviceProperties: %s", cudaGetErrorString(e));
    }
    if (prop.major != 10)
        return handle_fail(nullptr, none, PLT_ERR_UNSUPPORTED, "device %d is sm_%d%d; this library is built for sm_100a only",
                           device, prop.major, prop.minor);
    if (sms) *sms = prop.multiProcessorCount;
    return PLT_OK;
}

// Reads and clears the status word behind what `stream` holds.
inline plt_status handle_check(HandleBase* h, char* none, cudaStream_t stream, uint32_t* out_bits) {
    DeviceScope scope(h->device);
    if (scope.err != cudaSuccess) return handle_fail(h, none, PLT_ERR_CUDA, "cudaSetDevice: %s", cudaGetErrorString(scope.err));
    uint32_t bits = 0;
    cudaError_t e = cudaMemcpyAsync(&bits, h->status, 4, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaMemsetAsync(h->status, 0, 4, stream);
    if (e == cudaSuccess) e = cudaStreamSynchronize(stream);
    if (e != cudaSuccess) return handle_fail(h, none, PLT_ERR_CUDA, "reading the device status word: %s", cudaGetErrorString(e));
    if (out_bits) *out_bits = bits;
    if (bits == 0) return PLT_OK;
    return handle_fail(h, none, PLT_ERR_DEVICE_CHECK, "device status 0x%x:%s%s%s%s%s%s%s", bits,
                       (bits & kDevSeqLenClamped) ? " a length out of range (clamped)" : "",
                       (bits & kDevPageIdClamped) ? " page id out of range" : "",
                       (bits & kDevWaitTimeout) ? " a bounded wait ran out (output invalid)" : "",
                       (bits & kDevWinLenClamped) ? " win_lens entry out of range (clamped)" : "",
                       (bits & kDevTokenRange) ? " drafted token out of range (refused)" : "",
                       (bits & kDevNoProbability) ? " a row without probabilities" : "",
                       (bits & kDevGroupClamped) ? " a group's bounds, a prefix length or a start out of range (clamped)" : "");
}

inline bool misaligned(const void* p, uintptr_t unit) { return ((uintptr_t)p & (unit - 1)) != 0; }

}  // namespace plt
