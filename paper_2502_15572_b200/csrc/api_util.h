// What the C entry points share: messages of failing calls, checks of addresses, tensor maps.
#pragma once

#include <atomic>
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
// The same for int32 and fp32 arrays.
inline bool is_word_ptr(const void *p, int device) { return aligned(p, 4) && is_device_ptr(p, device); }

typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                  const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

inline EncodeTiledFn encode_tiled_fn()
{
    static std::atomic<EncodeTiledFn> known{nullptr};      // several host threads may come here first
    EncodeTiledFn fn = known.load();
    if (!fn) {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            known.store(fn = reinterpret_cast<EncodeTiledFn>(p));
    }
    return fn;
}

// Zeros beyond the ends.
inline bool encode(CUtensorMap *map, const void *base, int dtype, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
            const cuuint32_t *box, CUtensorMapSwizzle swizzle = CU_TENSOR_MAP_SWIZZLE_128B)
{
    const cuuint32_t ones[3] = {1, 1, 1};
    EncodeTiledFn fn = encode_tiled_fn();
    return fn && fn(map,
                    dtype == kE4M3  ? CU_TENSOR_MAP_DATA_TYPE_UINT8
                    : dtype == kF16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                    : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                    rank, const_cast<void *>(base), dims, strides, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace dresd
