// How attention and its like divide their work: the items of a list (a sequence's tiles of tokens) are added up by every workgroup for itself, as lengths are on the
// device, and each worker takes an equal share of all of them.
#pragma once
#include "kvc_attend.h"

namespace kvc {

__device__ inline uint32_t length_of(const AttendArgs& a, int32_t len, int32_t blocks) {
    const int64_t most = (int64_t)blocks * a.g.N;
    if (len > most) {
        atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
        return (uint32_t)most;
    }
    return len < 0 ? 0 : (uint32_t)len;
}
__device__ inline uint32_t own_length(const AttendArgs& a, int s) { return length_of(a, a.lens[s], a.max_blocks); }

// How the tiles of prefixes are divided: `each` to a worker, or, if `apart`, so many of one unit to a worker, as if units were multiples of it.
struct Division {
    uint32_t each, apart;
    __device__ uint32_t room(uint32_t tiles) const { return apart ? (tiles + each - 1) / each * each : tiles; }
};

// ---- dividing the work: sums of f(0..n-1), with the items dealt to the 256 threads of a workgroup in runs of `each`.
struct Sums {
    uint32_t before[256], wave[4], all, each;
    uint32_t workers[8];
    Division division;
};
template <class F>
__device__ inline void add_up(Sums& s, uint32_t n, F f) {
    const uint32_t t = threadIdx.x, lane = t & 63, each = (n + 255) / 256;
    uint32_t sum = 0;
    if (t < 256)
        for (uint32_t i = t * each; i < n && i < (t + 1) * each; ++i) sum += f(i);
    uint32_t upto = sum;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t o = __shfl_up(upto, k);
        if (lane >= (uint32_t)k) upto += o;
    }
    if (lane == 63 && t < 256) s.wave[t / 64] = upto;
    __syncthreads();
    if (t < 256) {
        uint32_t base = 0;
        for (uint32_t w = 0; w < t / 64; ++w) base += s.wave[w];
        s.before[t] = base + upto - sum;
        if (t == 255) s.all = base + upto, s.each = each;
    }
    __syncthreads();
}
// The sum before every item, and of all, for k_join.
template <class F>
__device__ inline void write_starts(const Sums& s, uint32_t* start, uint32_t n, F f) {
    const uint32_t t = threadIdx.x;
    if (t >= 256) return;
    uint32_t at = s.before[t];
    for (uint32_t i = t * s.each; i < n && i < (t + 1) * s.each; ++i) {
        start[i] = at;
        at += f(i);
    }
    if (t == 0) start[n] = s.all;
}
// The item that holds position p < s.all, and the sum before it.
struct Item {
    uint32_t i, start;
};
template <class F>
__device__ inline Item find_item(const Sums& s, uint32_t n, uint32_t p, F f) {
    uint32_t lo = 0;  // the last run that begins at or before p (runs of no work begin where the next does)
#pragma unroll
    for (uint32_t k = 128; k; k /= 2)
        if (s.before[lo + k] <= p) lo += k;
    Item r{lo * s.each, s.before[lo]};
    while (r.i + 1 < n) {
        const uint32_t v = f(r.i);
        if (p - r.start < v) break;
        r.start += v;
        ++r.i;
    }
    return r;
}
__device__ inline uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// tiles a worker takes
__device__ inline uint32_t share(uint32_t tiles, uint32_t workers) { return max(1u, (tiles + workers - 1) / workers); }

// Eight channels of the output, from their sums and the weights'.
__device__ inline uint4v finished(const float4v (&o)[2], float l) {
    const float f = l == 0.f ? 0.f : 1.f / l;
    uint4v v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        half2 x;
        x[0] = (_Float16)(o[e / 2][e % 2 * 2] * f);
        x[1] = (_Float16)(o[e / 2][e % 2 * 2 + 1] * f);
        v[e] = __builtin_bit_cast(uint32_t, x);
    }
    return v;
}

// What joins pieces: the weight that a piece with reference m has relative to `top`, the largest of the row's.  A piece may have the reference -infinity, which is
// smaller than any other and equal to itself, and yet hold NaN in its sums (all its scores are NaN, or -infinity and a value infinite), so that none is passed over:
// one in which the row saw no token adds zeros.
__device__ inline float join_weight(float m, float top) { return m == top ? 1.f : power2(m - top); }

// Where a worker is in its share.
struct Place {
    uint32_t s, u, t, tiles, len;  // sequence; unit u of it (head and row tile); tile t of `tiles`
};

}  // namespace kvc
