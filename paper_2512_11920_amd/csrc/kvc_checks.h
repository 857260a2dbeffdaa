// What the entry points of the decode-step operators check of their arguments.
#pragma once
#include "kvc_cache.h"
#include "kvc_ctx.h"

namespace kvc {

constexpr int64_t kMaxGroups = (1ll << 24) - 1;  // workgroups of 256 threads a launch holds
constexpr int32_t kMaxLayers = 65535;             // of a call; the layer is a grid dimension of its own

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
inline bool strides_ok(const int64_t* s) {
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || (s[i] & 7)) return false;
    return true;
}
// where values begin: `v`, or behind the key pages of `k`
inline const uint16_t* values_of(const kvc_ctx* ctx, const void* k, const void* v, int32_t n_kv) {
    return v ? static_cast<const uint16_t*>(v) : static_cast<const uint16_t*>(k) + n_kv * ctx->g.page_stride;
}
inline bool heads_ok(const kvc_ctx* ctx, const void* v, int32_t n_kv) { return n_kv >= 1 && (int64_t)n_kv * (v ? 1 : 2) == ctx->g.ppb; }
// Query rows are counted in 31 bits, and joined by one launch, d / 8 threads a row.
inline bool rows_ok(int64_t n_seq, int64_t n_q, int64_t n_heads, int d) {
    return n_seq * n_heads <= INT32_MAX / n_q && n_seq * n_heads * n_q <= kMaxGroups * (2048 / d);
}
inline int launched(hipError_t e) { return hip_ok(e) ? KVC_OK : KVC_ERR_HIP; }

struct Buffer {
    const void* at;
    uint64_t n;
};
inline bool apart(const Buffer& a, const Buffer& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return x <= y ? y - x >= a.n : x - y >= b.n;
}

}  // namespace kvc
