// Host-side helpers that the planners (api.cu, paged_api.cu) share.
#pragma once
#include <cudaTypedefs.h>

#include "internal.h"

namespace lookm {

extern thread_local int g_launches;      // kernels that the last call on this host thread enqueued

struct DeviceInfo { int sms = 0; int cc_major = 0; bool ok = false; };
int device_info(DeviceInfo& out);        // of the current device; LOOKM_OK or why it can't be used

PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder();      // nullptr: the driver has none

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

template <class T>
T* at(void* ws, size_t off) { return reinterpret_cast<T*>(static_cast<char*>(ws) + off); }

}  // namespace lookm

#define LOOKM_CUDA(expr)                                  \
    do {                                                  \
        if ((expr) != cudaSuccess) return LOOKM_ERR_CUDA; \
    } while (0)
#define LOOKM_TRY(expr)                   \
    do {                                  \
        int st_ = (expr);                 \
        if (st_ != LOOKM_OK) return st_;  \
    } while (0)
