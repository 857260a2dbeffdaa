// tests/launch_recorder.cpp with memory told apart by its address, and the buffers that compaction's kernels get, for tests/cache_calls.py.
// Addresses from 2^46 on are memory that the device cannot reach; from 2^45 on pinned host memory, which the device sees 2^44 lower; others are on the device.
#include "kvc_cache.h"

#define hipPointerGetAttributes every_address_alike
#define hipLaunchKernel noted_launch
#include "launch_recorder.cpp"
#undef hipPointerGetAttributes
#undef hipLaunchKernel

static const void *pool_out, *desc_out;

extern "C" {
const void* rec_pool_out() { return pool_out; }
const void* rec_desc_out() { return desc_out; }

hipError_t hipLaunchKernel(const void* f, dim3 grid, dim3 block, void** args, size_t lds, hipStream_t s) {
    const std::string& name = names().at(f);
    if (name.find("k_moveE") != std::string::npos || name.find("k_compact_smallE") != std::string::npos) {
        const kvc::CompactArgs* a = static_cast<const kvc::CompactArgs*>(args[0]);
        pool_out = a->pool_out, desc_out = a->desc_out;
    }
    return noted_launch(f, grid, block, args, lds, s);
}
hipError_t hipPointerGetAttributes(hipPointerAttribute_t* a, const void* p) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    memset(a, 0, sizeof *a);
    a->type = at >> 46 ? hipMemoryTypeUnregistered : at >> 45 ? hipMemoryTypeHost : hipMemoryTypeDevice;
    a->devicePointer = reinterpret_cast<void*>(at >> 46 ? 0 : at >> 45 ? at - (1ull << 44) : at);
    return hipSuccess;
}
}
