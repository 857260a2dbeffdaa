// Attention over the paged cache, compiled once per head dimension (-DKVC_HEAD_DIM=d).
#include "kvc_attend.h"

#ifndef KVC_HEAD_DIM
#error "KVC_HEAD_DIM: the head dimension to compile"
#endif

namespace kvc {

__device__ inline uint32_t length_of(const AttendArgs& a, int32_t len, int32_t blocks) {
    const int64_t most = (int64_t)blocks * a.g.N;
    if (len > most) {
        if (threadIdx.x == 0) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
        return (uint32_t)most;
    }
    return len < 0 ? 0 : (uint32_t)len;
}

// Group of sequence s: the prefix whose range of sequences holds it, or -1.
__device__ inline int prefix_of(const AttendArgs& a, int s) {
    for (int g = 0; g < a.n_prefix; ++g)
        if (s >= a.prefix_first[g] && s < a.prefix_first[g + 1]) return g;
    return -1;
}

// A wave per sequence, KV head and 16 query rows: the prefix's tokens, then the sequence's.
template <int D>
__global__ __launch_bounds__(64, 1) void k_attend(AttendArgs a) {
    const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    const int s = blockIdx.x, h = blockIdx.y, row = blockIdx.z * 16 + n;
    const bool have = row < a.rows;
    const int head = h * a.group + (have ? row / a.n_q : 0), i = have ? row % a.n_q : 0;
    Rows<D> r;
    const uint16_t* q = a.q + s * a.q_strides[0] + i * a.q_strides[1] + head * a.q_strides[2];
#pragma unroll
    for (int c = 0; c < D / 32; ++c) r.q[c] = *reinterpret_cast<const uint4v*>(q + 32 * c + 8 * g);
#pragma unroll
    for (int c = 0; c < D / 16; ++c) r.o[c] = float4v{0.f, 0.f, 0.f, 0.f};
    r.m = -INFINITY;
    r.l = 0.f;
    const int prefix = prefix_of(a, s);
    for (int part = prefix < 0 ? 1 : 0; part < 2; ++part) {
        Source src;
        src.k = a.k_cache + h * a.g.page_stride;
        src.v = a.v_cache + h * a.g.page_stride;
        uint32_t limit;
        if (part == 0) {
            src.table = a.prefix_table + (int64_t)prefix * a.max_prefix_blocks;
            src.len = limit = length_of(a, a.prefix_lens[prefix], a.max_prefix_blocks);
        } else {
            src.table = a.table + (int64_t)s * a.max_blocks;
            src.len = length_of(a, a.lens[s], a.max_blocks);
            const int64_t sees = (int64_t)a.lens[s] - (a.n_q - 1 - i);
            limit = sees < 0 ? 0 : sees < src.len ? (uint32_t)sees : src.len;
        }
        for (uint32_t t = 0; t < src.len; t += kTile) {
            Tokens<D> x;
            load_tokens<D>(x, a, src, t);
            add_tokens<D>(r, x, a.scale_log2, t, limit);
        }
    }
    const float l = row_sum(r.l);
    if (!have) return;
    store_pieces<D, 0>(r, a.out + s * a.out_strides[0] + i * a.out_strides[1] + head * a.out_strides[2], l == 0.f ? 0.f : 1.f / l, g);
    if (a.lse && g == 0) a.lse[((int64_t)s * a.n_q + i) * a.n_heads + head] = lse_of(r.m, l);
}

template <>
hipError_t launch_attend<KVC_HEAD_DIM>(const AttendArgs& a, hipStream_t s) {
    return launch_kernel(k_attend<KVC_HEAD_DIM>, dim3((unsigned)a.n_seq, (unsigned)a.n_kv, (unsigned)((a.rows + 15) / 16)), dim3(64), s, a);
}

}  // namespace kvc
