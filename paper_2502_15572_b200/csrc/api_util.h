// What the C entry points share: messages of failing calls and checks of addresses.
#pragma once

#include <cstdarg>
#include <cstdio>

#include "../../include/dresd.h"
#include "internal.h"

namespace dresd {

inline dresd_status fail(dresd_status st, const char *fmt, ...)
{
    char msg[512];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(msg, sizeof msg, fmt, ap);
    va_end(ap);
    set_last_error(msg);
    return st;
}
inline dresd_status fail_cuda(cudaError_t e, const char *what)
{
    return fail(DRESD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

// Memory of `device` (a kernel must not be given another GPU's), or managed memory.
inline bool is_device_ptr(const void *p, int device)
{
    if (!p) return false;
    cudaPointerAttributes at;
    if (cudaPointerGetAttributes(&at, p) != cudaSuccess) {
        cudaGetLastError();
        return false;
    }
    return (at.type == cudaMemoryTypeDevice && at.device == device) || at.type == cudaMemoryTypeManaged;
}

inline bool aligned(const void *p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

}  // namespace dresd
