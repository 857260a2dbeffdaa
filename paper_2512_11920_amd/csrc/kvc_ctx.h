// The host side of a context, shared by the sources that hold entry points.
#pragma once
#include <atomic>

#include "kvc_common.h"

struct kvc_ctx {
    int prefetch_policy = 0;
    int window_capacity = 0;      // window engines this device holds at once (0: unknown); an upper bound on useful omega
    int wide_capacity = 0;        // ... and wide engines (0: unknown)
    void* static_work = nullptr;  // device address of `scratch` on this context's device
    kvc_config cfg;
    kvc::Geometry g;
    int device;
    kvc::DevState* st;  // device
    uint8_t* pool;
    uint64_t pool_bytes;
    bool pool_in_hbm, desc_in_hbm;  // plain memory of this device
    kvc_desc* desc;
    uint64_t n_desc;
    std::atomic<uint64_t> waiting{0};  // its part of g_waiting
};

namespace kvc {

// Notes a failure for kvc_strerror(KVC_ERR_HIP).
bool hip_ok(hipError_t e);

// The address by which the device sees memory that it can reach: its own, or pinned and mapped host memory.  False: other memory, which a kernel would fault on.
bool seen_by_device(void** p, hipPointerAttribute_t* attr);

// Every call must be made with the context's device current: buffers and streams belong to it.
bool on_ctx_device(const kvc_ctx* ctx);

}  // namespace kvc
