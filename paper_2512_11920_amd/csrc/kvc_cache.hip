// Kernels that move blocks, tokens and payloads: append, copy, fork, free, compaction.
#include <algorithm>

#include "kvc_cache.h"

namespace kvc {

__device__ inline void bad_index(DevState* st) { atomicOr(&st->status, KVC_ST_BAD_INDEX); }

// ---- append: a workgroup per new token, a lane per 16 bytes of its K and V rows, so that one lookup serves a token's heads.  Bound by memory, or by the launch where
// there are few tokens: 16 sequences of 512 new tokens, 8 x 128 (67 MB moved), 12.0 us, 5.6 TB/s; one token of 4 x 64, 1.8 us.
__global__ __launch_bounds__(256) void k_append(AppendArgs a) {
    const uint32_t s = fast_div(blockIdx.x, a.by_n_new), i = blockIdx.x - s * (uint32_t)a.n_new;
    const int64_t t = (int64_t)a.lens[s] - a.n_new + i;
    if (t < 0) return;
    const uint32_t at = fast_div((uint32_t)t, a.by_N), row = (uint32_t)t - at * (uint32_t)a.g.N;
    if (at >= (uint32_t)a.max_blocks) {
        if (threadIdx.x == 0) bad_index(a.st);
        return;
    }
    const int32_t block = a.table[(int64_t)s * a.max_blocks + at];
    if (block < 0) return;
    if (block >= a.n_cache_blocks) {
        if (threadIdx.x == 0) bad_index(a.st);
        return;
    }
    const int64_t to = block * a.g.block_stride + row * a.g.row_stride;
    const uint32_t each = (uint32_t)(a.n_kv * a.g.lpr);
    for (uint32_t c = threadIdx.x; c < 2 * each; c += blockDim.x) {
        const bool v = c >= each;
        const uint32_t e = v ? c - each : c, h = fast_div(e, a.by_lpr), k = e - h * (uint32_t)a.g.lpr;
        const uint16_t* from = v ? a.v_new + s * a.v_strides[0] + i * a.v_strides[1] + h * a.v_strides[2]
                                 : a.k_new + s * a.k_strides[0] + i * a.k_strides[1] + h * a.k_strides[2];
        uint16_t* into = (v ? a.v_cache : a.k_cache) + to + h * a.g.page_stride;
        reinterpret_cast<uint4*>(into)[k] = reinterpret_cast<const uint4*>(from)[k];
    }
}

// ---- copy: a workgroup per 16 KB of a block, four loads of 16 bytes a lane on their way before the first store, and stores past the caches, as nobody reads the copies soon.
// Bound by memory: 64 blocks of 64 KB in each of 80 layers, from 4 sources (356 MB), 67 us, 5.3 TB/s; 2.2 us where there is one.
__global__ __launch_bounds__(256) void k_copy_blocks(CopyArgs a) {
    const int64_t layer = blockIdx.y;
    const uint32_t pair = fast_div(blockIdx.x, a.by_pieces), piece = blockIdx.x - pair * (uint32_t)a.pieces;
    const int32_t src = a.src[pair], dst = a.dst[pair];
    if (src < 0 || dst < 0) return;
    const int64_t from = layer * a.per_layer + src, to = layer * a.per_layer + dst;
    if (src >= a.per_layer || dst >= a.per_layer || from >= a.n_cache_blocks || to >= a.n_cache_blocks) {
        if (threadIdx.x == 0) bad_index(a.st);
        return;
    }
    const uint16_t* x = a.cache + from * a.g.block_stride;
    uint16_t* y = a.cache + to * a.g.block_stride;
    uint4v r[kCopyChunks / 256];
    int64_t at[kCopyChunks / 256];
#pragma unroll
    for (int k = 0; k < kCopyChunks / 256; ++k) {
        const uint32_t c = piece * kCopyChunks + k * 256 + threadIdx.x;
        at[k] = -1;
        r[k] = uint4v{0, 0, 0, 0};
        if (c < (uint32_t)a.chunks) {
            if (a.dense) {
                at[k] = 8ll * c;
            } else {
                const uint32_t line = fast_div(c, a.by_lpr), page = fast_div(line, a.by_N);
                at[k] = page * a.g.page_stride + (line - page * (uint32_t)a.g.N) * a.g.row_stride + 8 * (c - line * (uint32_t)a.g.lpr);
            }
            r[k] = *reinterpret_cast<const uint4v*>(x + at[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < kCopyChunks / 256; ++k)
        if (at[k] >= 0) __builtin_nontemporal_store(r[k], reinterpret_cast<uint4v*>(y + at[k]));
}

// ---- fork and free: a lane per descriptor.  Bound by memory: 8,192 blocks of 16 pages in each of 80 layers (335 MB), 52 us, 6.4 TB/s.
__device__ inline uint4 no_page() { return make_uint4(0, 0, 0, (uint32_t)KVC_MODE_INVALID << 16); }

template <bool FORK>
__global__ __launch_bounds__(256) void k_ids(IdsArgs a) {
    const int64_t p = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (p >= a.n_pages) return;
    const uint32_t i = fast_div((uint32_t)p, a.by_ppb), page = (uint32_t)p - i * (uint32_t)a.ppb;
    const int32_t dst = a.dst[i], src = FORK ? a.src[i] : 0;
    if (dst < 0 || src < 0) return;
    if (dst >= a.per_layer || src >= a.per_layer) {
        if (page == 0) bad_index(a.st);
        return;
    }
    uint4* desc = reinterpret_cast<uint4*>(a.desc) + (int64_t)blockIdx.y * a.per_layer * a.ppb + page;
    uint4v* to = reinterpret_cast<uint4v*>(desc + (int64_t)dst * a.ppb);
    if (FORK) __builtin_nontemporal_store(reinterpret_cast<const uint4v*>(desc)[(int64_t)src * a.ppb], to);
    else *reinterpret_cast<uint4*>(to) = no_page();
}

// ---- compaction.  A unit's new place is its rank among the units that are held, so payloads keep their order and shared ones are moved once: one bit a unit
// is marked (k_mark), counted (k_count, k_base) and ranked again where units are moved and pages renamed (k_move).  A pool of 1.09 GB, 589,824 pages of 16 x 128 in random order of which
// half are live: 268 us, 185 of them for the bytes that have to move.
__global__ __launch_bounds__(256) void k_bits_zero(CompactArgs a) {
    const uint64_t n = a.groups * kGroupWords / 2;
    for (uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (uint64_t)gridDim.x * 256) reinterpret_cast<uint4*>(a.bits)[i] = make_uint4(0, 0, 0, 0);
}

// A page's span in units, and whether it is held at all; one that leaves the pool is not.
struct Span {
    uint64_t from;
    uint32_t n, kind;  // kind: 0 none, 1 live, 2 corrupt
};
__device__ inline Span span_of(const uint4& d, uint64_t units) {
    const uint64_t off = d.x | (uint64_t)d.y << 32;
    const uint32_t mode = d.w >> 16 & 0xFF;
    Span s{off / 16, d.w & 0xFFFF, 1};
    if (mode == KVC_MODE_INVALID) s.kind = 0;
    else if (mode > KVC_MODE_CHAN || (off & 15) || s.from > units || s.n > units - s.from) s.kind = 2;
    return s;
}

// Marks the units of a page's payload: the first and the last word are or-ed, whole words between them are stored (a store of all ones takes nothing
// from a shared or neighbouring payload).
template <class Or, class Ones>
__device__ inline void mark(const Span& s, Or or_word, Ones ones) {
    if (s.kind != 1 || s.n == 0) return;
    const uint64_t end = s.from + s.n, first = s.from / 64, last = (end - 1) / 64;
    const uint32_t lo = s.from & 63, hi = (uint32_t)(end - 1) & 63;
    // all ones from bit lo up, and up to bit hi, by 32-bit halves
    const uint32_t l0 = lo < 32 ? ~0u << lo : 0, l1 = lo < 32 ? ~0u : ~0u << (lo - 32);
    const uint32_t h0 = hi < 32 ? ~0u >> (31 - hi) : ~0u, h1 = hi < 32 ? 0 : ~0u >> (63 - hi);
    const unsigned long long low = l0 | (unsigned long long)l1 << 32, high = h0 | (unsigned long long)h1 << 32;
    if (first == last) {
        or_word(first, low & high);
        return;
    }
    or_word(first, low);
    for (uint64_t w = first + 1; w < last; ++w) ones(w);
    or_word(last, high);
}

// Bound by the atomics, which go past the caches of the XCDs: 590,000 in 44 us where the table is in no order, 17 us where it is in the pool's.  (Neighbours' words joined
// in a wave first: 45 and 13 us.)
__global__ __launch_bounds__(256) void k_mark(CompactArgs a) {
    const uint64_t i = (uint64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= a.n_desc) return;
    const Span s = span_of(reinterpret_cast<const uint4*>(a.desc)[i], a.units);
    if (s.kind == 2) atomicOr(&a.st->status, KVC_ST_CORRUPT);
    mark(s, [&](uint64_t w, unsigned long long v) { atomicOr(a.bits + w, v); }, [&](uint64_t w) { a.bits[w] = ~0ull; });
}

__device__ inline uint32_t scan_wave(uint32_t v) {  // inclusive
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t o = __shfl_up(v, k);
        if (lane >= k) v += o;
    }
    return v;
}

// Inclusive sums over a workgroup of 1,024, and their total.
__device__ inline uint32_t scan_group(uint32_t v, uint32_t (&part)[16], uint32_t& all) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x / 64, upto = scan_wave(v);
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    uint32_t before = 0;
    all = 0;
#pragma unroll
    for (uint32_t w = 0; w < 16; ++w) {
        before += w < wave ? part[w] : 0;
        all += part[w];
    }
    __syncthreads();
    return before + upto;
}

// a workgroup per group, a lane per word; 6 us for 1,036 groups
__global__ __launch_bounds__(1024) void k_count(CompactArgs a) {
    __shared__ uint32_t part[16];
    const uint64_t w = (uint64_t)blockIdx.x * kGroupWords + threadIdx.x;
    const uint32_t n = __popcll(a.bits[w]);
    uint32_t all;
    const uint32_t upto = scan_group(n, part, all);
    a.before[w] = (uint16_t)(upto - n);  // (at most 65,536 - 64)
    if (threadIdx.x == 0) a.base[blockIdx.x] = all;
}

// one workgroup: sums of all groups before each; 5 us for 1,036
__global__ __launch_bounds__(1024) void k_base(CompactArgs a) {
    __shared__ uint32_t part[16];
    unsigned long long sum = 0;
    for (uint64_t g0 = 0; g0 < a.groups; g0 += 1024) {
        const uint64_t g = g0 + threadIdx.x;
        const uint32_t n = g < a.groups ? (uint32_t)a.base[g] : 0;
        uint32_t all;
        const uint32_t upto = scan_group(n, part, all);
        if (g < a.groups) a.base[g] = sum + upto - n;
        sum += all;
    }
    if (threadIdx.x == 0) *a.used = 16 * (sum < a.out_units ? sum : a.out_units);
}

// set bits of a word below bit b
__device__ inline uint32_t bits_below(unsigned long long bits, uint32_t b) {
    const uint32_t lo = (uint32_t)bits, hi = (uint32_t)(bits >> 32);
    return b < 32 ? __popc(lo & ~(~0u << b)) : __popc(lo) + __popc(hi & ~(~0u << (b - 32)));
}

// The descriptor of a page whose payload's first unit has the rank that `rank_of` gives.
template <class F>
__device__ inline uint4 rename(uint4 d, const CompactArgs& a, F rank_of) {
    const Span s = span_of(d, a.units);
    if (s.kind != 1) return no_page();
    const uint64_t at = s.n ? rank_of(s.from) : 0;
    if (at + s.n > a.out_units) {
        atomicOr(&a.st->status, KVC_ST_POOL_FULL);
        return no_page();
    }
    d.x = (uint32_t)(at * 16);
    d.y = (uint32_t)(at >> 28);
    return d;
}

// A wave moves what is held of kMoveWords words, 4 KB of pool: lane i has unit i of each word, loads it if it is held and stores it to its rank.
// The workgroups of a megabyte are dealt to the XCDs so that each has a run of them, as neighbours write to the same lines.  1.09 GB, 16 x 128 pages, half of them
// live and in random order, 1.16 GB of traffic: 64 words a wave 241 us, 16 words 224, 4 words 212, and 204 us with runs (5.7 TB/s).
constexpr uint32_t kMoveWords = 4, kMoveGroups = (uint32_t)kGroupWords / (4 * kMoveWords);  // words of a wave; workgroups of 1,024 words

__device__ inline void move_words(const CompactArgs& a, uint64_t first) {
    const uint32_t lane = threadIdx.x & 63;
    const uint64_t word = first + lane % kMoveWords, base = a.base[first / kGroupWords];
    const unsigned long long bits = a.bits[word];
    const uint32_t lo = (uint32_t)bits, hi = (uint32_t)(bits >> 32), before = a.before[word];
    const uint4v* from = reinterpret_cast<const uint4v*>(a.pool) + first * 64 + lane;
    uint4v* to = reinterpret_cast<uint4v*>(a.pool_out) + base;
    const uint64_t room = a.out_units > base ? a.out_units - base : 0;
    const auto held = [&](uint32_t w) {  // whether the lane's unit of word w is
        const uint32_t half = lane < 32 ? __builtin_amdgcn_readlane(lo, w) : __builtin_amdgcn_readlane(hi, w);
        return (half >> (lane & 31) & 1) != 0;
    };
    uint4v x[kMoveWords];
#pragma unroll
    for (uint32_t w = 0; w < kMoveWords; ++w)
        if (held(w)) x[w] = from[w * 64];
#pragma unroll
    for (uint32_t w = 0; w < kMoveWords; ++w) {
        const uint32_t wl = __builtin_amdgcn_readlane(lo, w), wh = __builtin_amdgcn_readlane(hi, w);
        const uint32_t at = __builtin_amdgcn_readlane(before, w) + __builtin_amdgcn_mbcnt_hi(wh, __builtin_amdgcn_mbcnt_lo(wl, 0));
        if (held(w) && at < room) to[at] = x[w];
    }
}

// the first `movers` workgroups move payloads, the others rename pages
__global__ __launch_bounds__(256) void k_move(CompactArgs a, uint32_t movers) {
    if (blockIdx.x < movers) {
        const uint32_t i = blockIdx.x % kMoveGroups, run = i % 8 * (kMoveGroups / 8) + i / 8;
        move_words(a, blockIdx.x / kMoveGroups * kGroupWords + (run * 4 + threadIdx.x / 64) * kMoveWords);
        return;
    }
    const uint64_t i = (uint64_t)(blockIdx.x - movers) * 256 + threadIdx.x;
    if (i >= a.n_desc) return;
    reinterpret_cast<uint4*>(a.desc_out)[i] = rename(reinterpret_cast<const uint4*>(a.desc)[i], a, [&](uint64_t unit) {
        const uint64_t w = unit / 64;
        return a.base[w / kGroupWords] + a.before[w] + bits_below(a.bits[w], unit & 63);
    });
}

// A pool that one workgroup compacts: everything but payloads and descriptors is in LDS, and there is one launch.  Half of a pool of 16 KB: 3.3 us, 14.2 by the kernels above;
// of 256 KB, as much as goes this way, 5.7 and 15.4.
__global__ __launch_bounds__(1024) void k_compact_small(CompactArgs a) {
    __shared__ unsigned long long bits[kSmallWords];
    __shared__ uint32_t before[kSmallWords];
    __shared__ uint32_t part[16];
    const uint32_t t = threadIdx.x;
    if (t < kSmallWords) bits[t] = 0;
    __syncthreads();
    for (uint64_t i = t; i < a.n_desc; i += 1024) {
        const Span s = span_of(reinterpret_cast<const uint4*>(a.desc)[i], a.units);
        if (s.kind == 2) atomicOr(&a.st->status, KVC_ST_CORRUPT);
        mark(s, [&](uint64_t w, unsigned long long v) { atomicOr(&bits[w], v); }, [&](uint64_t w) { atomicOr(&bits[w], ~0ull); });
    }
    __syncthreads();
    const uint32_t n = t < kSmallWords ? __popcll(bits[t]) : 0;
    uint32_t all;
    const uint32_t upto = scan_group(n, part, all);
    if (t < kSmallWords) before[t] = upto - n;
    if (t == 0) *a.used = 16 * (all < a.out_units ? all : a.out_units);
    __syncthreads();
    for (uint32_t u = t; u < a.units; u += 1024) {
        const uint32_t w = u / 64, b = u & 63;
        const uint64_t at = before[w] + bits_below(bits[w], b);
        const uint32_t half = b < 32 ? (uint32_t)bits[w] : (uint32_t)(bits[w] >> 32);
        if ((half >> (b & 31) & 1) && at < a.out_units) reinterpret_cast<uint4*>(a.pool_out)[at] = reinterpret_cast<const uint4*>(a.pool)[u];
    }
    for (uint64_t i = t; i < a.n_desc; i += 1024)
        reinterpret_cast<uint4*>(a.desc_out)[i] =
            rename(reinterpret_cast<const uint4*>(a.desc)[i], a, [&](uint64_t unit) { return (uint64_t)before[unit / 64] + bits_below(bits[unit / 64], unit & 63); });
}

__global__ void k_adopt(DevState* st, const unsigned long long* used) {
    if (threadIdx.x == 0) st->cursor16 = *used / 16;
}

// ---- launches.
static unsigned groups(uint64_t n, uint64_t each) { return (unsigned)((n + each - 1) / each); }

hipError_t launch_append(const AppendArgs& a, hipStream_t s) {
    const int lanes = 2 * a.n_kv * a.g.lpr;
    return launch_kernel(k_append, dim3((unsigned)(a.n_seq * a.n_new)), dim3(lanes <= 64 ? 64 : lanes <= 128 ? 128 : 256), s, a);
}

hipError_t launch_copy_blocks(const CopyArgs& a, hipStream_t s) {
    return launch_kernel(k_copy_blocks, dim3((unsigned)(a.n * a.pieces), (unsigned)a.n_layers), dim3(256), s, a);
}

hipError_t launch_fork(const IdsArgs& a, hipStream_t s) { return launch_kernel(k_ids<true>, dim3(groups(a.n_pages, 256), (unsigned)a.n_layers), dim3(256), s, a); }
hipError_t launch_free(const IdsArgs& a, hipStream_t s) { return launch_kernel(k_ids<false>, dim3(groups(a.n_pages, 256), (unsigned)a.n_layers), dim3(256), s, a); }

hipError_t launch_compact(const CompactArgs& a, hipStream_t s) {
    if (a.units <= 64 * kSmallWords && a.n_desc <= kSmallPages) return launch_kernel(k_compact_small, dim3(1), dim3(1024), s, a);
    hipError_t e = launch_kernel(k_bits_zero, dim3((unsigned)std::min<uint64_t>(groups(a.groups * kGroupWords / 2, 256), 2048)), dim3(256), s, a);
    if (e == hipSuccess) e = launch_kernel(k_mark, dim3(groups(a.n_desc, 256)), dim3(256), s, a);
    if (e == hipSuccess) e = launch_kernel(k_count, dim3((unsigned)a.groups), dim3(1024), s, a);
    if (e == hipSuccess) e = launch_kernel(k_base, dim3(1), dim3(1024), s, a);
    const uint32_t movers = (uint32_t)a.groups * kMoveGroups;
    if (e == hipSuccess) e = launch_kernel(k_move, dim3(movers + groups(a.n_desc, 256)), dim3(256), s, a, movers);
    return e;
}

hipError_t launch_adopt(DevState* st, const unsigned long long* used, hipStream_t s) { return launch_kernel(k_adopt, dim3(1), dim3(64), s, st, used); }

}  // namespace kvc
