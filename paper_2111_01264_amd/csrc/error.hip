// Thread-local error message behind dqn_last_error(), and the argument checks that calls without a handle share.
#include "common.h"

#include <mutex>

namespace dqn {

char* error_buffer()
{
    static thread_local char buf[512] = {0};
    return buf;
}

int fail(int code, const char* fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(error_buffer(), 512, fmt, ap);
    va_end(ap);
    return code;
}

hipError_t raise_dynamic_lds(const void* kernel, int bytes)
{
    constexpr int kKernels = 64, kDevices = 64;   // (beyond these nothing is remembered, and the runtime is asked every time)
    static std::mutex mu;
    static struct { const void* kernel; int bytes[kDevices]; } allowed[kKernels];
    int device = 0;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return e;
    std::lock_guard<std::mutex> lock(mu);
    int i = 0;
    while (i < kKernels && allowed[i].kernel && allowed[i].kernel != kernel) ++i;
    const bool known = i < kKernels && device >= 0 && device < kDevices;
    if (known && allowed[i].kernel == kernel && allowed[i].bytes[device] >= bytes) return hipSuccess;
    const hipError_t r = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (r == hipSuccess && known) { allowed[i].kernel = kernel; allowed[i].bytes[device] = bytes; }
    return r;
}

int check_type(const char* who, int32_t type)
{
    if (type != DQN_TYPE_FP32 && type != DQN_TYPE_BF16 && type != DQN_TYPE_FP16) return fail(DQN_EINVAL, "%s: type %d", who, type);
    return DQN_OK;
}

int check_stream(const char* who, void* stream, hipStream_t* out)
{
    *out = static_cast<hipStream_t>(stream);
    if (*out == hipStreamLegacy) *out = nullptr;   // its other name, which not every runtime's calls know: hipStreamGetDevice follows it as a pointer
    if (!*out) return DQN_OK;   // the null stream is the current device's
    int current = -1;
    hipDevice_t owner = -1;
    DQN_HIP(hipGetDevice(&current));
    DQN_HIP(hipStreamGetDevice(*out, &owner));
    if (owner != current) return fail(DQN_EINVAL, "%s: the stream belongs to device %d, the current device is %d", who, owner, current);
    return DQN_OK;
}

}  // namespace dqn

extern "C" const char* dqn_last_error(void) { return dqn::error_buffer(); }
