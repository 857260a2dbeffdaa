// Eviction: of every sequence and KV head, `keep` tokens stay, the last `recent` positions and the heaviest of the others.  Tokens of a head may lie in any order, as attention does not
// look at it, so what stays is not moved together from the beginning on: tokens at slots from `keep` on that stay go to the slots below it whose tokens leave, of which there are as many.
// Sources and destinations are then apart, and no more is moved than has to be.
#include "kvc_divide.h"
#include "kvc_fp4.h"

namespace kvc {

constexpr uint32_t kSelectThreads = 512, kSelectWaves = kSelectThreads / 64;
constexpr uint32_t kKeysKept = 16384;  // in LDS, 64 KB, so that two workgroups are on a compute unit

// Weights in the order of whole numbers: -infinity..., zeros of either sign alike, ...infinity, NaN, and tokens that are safe.
__device__ inline uint32_t order_of(float w) {
    if (w != w) return 0xFFFFFFFEu;
    const uint32_t b = __float_as_uint(w == 0.f ? 0.f : w);
    return b >> 31 ? ~b : b | 0x80000000u;
}

template <int N>
struct Number {
    static constexpr int value = N;
};

// set bits of lanes before this one
__device__ inline uint32_t before_lane(uint64_t lanes) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0)); }

constexpr uint32_t kSafe = 0xFFFFFFFFu;
__device__ inline uint32_t key_of(float w, int32_t position, int64_t safe_from) { return position >= safe_from ? kSafe : order_of(w); }

// The sum over a wave's lanes up to this one.  (Within rows of 16 lanes, then rows 0 and 2 into 1 and 3, then the first half into the second; without LDS.)
template <int CONTROL, int ROWS>
__device__ inline uint32_t plus_lane(uint32_t v) { return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CONTROL, ROWS, 0xF, false); }
__device__ inline uint32_t sum_upto(uint32_t v) {
    v = plus_lane<0x111, 0xF>(v);  // one lane back, two, four, eight
    v = plus_lane<0x112, 0xF>(v);
    v = plus_lane<0x114, 0xF>(v);
    v = plus_lane<0x118, 0xF>(v);
    v = plus_lane<0x142, 0xA>(v);  // lane 15 of the row before
    return plus_lane<0x143, 0xC>(v);  // lane 31
}
// Sums of what the waves left in LDS: before this one's, and of all.
struct Before {
    uint32_t here, all;
    __device__ Before(const uint32_t (&of_wave)[kSelectWaves], uint32_t wave) {
        const int v = (int)of_wave[threadIdx.x % kSelectWaves];
        here = all = 0;
#pragma unroll
        for (uint32_t k = 0; k < kSelectWaves; ++k) {
            const uint32_t n = (uint32_t)__builtin_amdgcn_readlane(v, k);
            here += k < wave ? n : 0;
            all += n;
        }
    }
};

// What a workgroup of the selection has: a sequence and head.
struct Unit {
    uint32_t s, len, keep;  // len: 0 where it is below zero
    int32_t given;
    int64_t safe_from;
    const float* weights;
    const int32_t* positions;
    float* weights_out;
    int32_t* positions_out;

    __device__ explicit Unit(const EvictArgs& a) {
        s = fast_div(blockIdx.x, a.by_n_kv);
        given = a.lens[s];
        len = (uint32_t)max(given, 0);
        keep = (uint32_t)max(a.keep[s], 0);
        safe_from = (int64_t)a.seen[s] - min((uint32_t)a.recent, keep);
        const int64_t at = (int64_t)blockIdx.x * a.width;
        weights = a.weights + at;
        positions = a.positions + at;
        weights_out = a.weights_out + at;
        positions_out = a.positions_out + at;
    }
    // Whether nothing leaves: there are no more tokens than stay, or one has no block or no weight; what is kept for them is then copied as it is.  Called by all threads.
    __device__ bool settled(const EvictArgs& a) const {
        bool bad = given > a.width || (int64_t)given > (int64_t)a.max_blocks * a.g.N;
        if (!bad)
            for (uint32_t i = threadIdx.x; (int64_t)i * a.g.N < len; i += kSelectThreads) {
                const int32_t block = a.table[(int64_t)s * a.max_blocks + i];
                bad = bad || block < 0 || block >= a.n_cache_blocks;
            }
        bad = __syncthreads_or(bad);
        const bool all = bad || len <= keep;
        if (threadIdx.x == 0) {
            if (bad) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
            if (all) a.counts[blockIdx.x] = 0;
            if (blockIdx.x == s * a.n_kv) a.left[s] = bad ? given : (int32_t)min(len, keep);
        }
        if (all) {
            const uint32_t n = min(len, (uint32_t)a.width);
            if (weights_out != weights)
                for (uint32_t t = threadIdx.x; t < n; t += kSelectThreads) weights_out[t] = weights[t];
            if (positions_out != positions)
                for (uint32_t t = threadIdx.x; t < n; t += kSelectThreads) positions_out[t] = positions[t];
        }
        return all;
    }
};

// ---- which tokens leave: a workgroup per sequence and head, whose waves have slots in a row each, up to I * 64 of them in registers.  The key of the heaviest that leaves is found 11 bits at a time, by
// counting; of equal keys the lowest slots leave.  Slots that leave below `keep`, and those from there on that stay, are numbered in order, and meet in LDS.
// Bound by barriers, of which each of up to three counts has three, and by how late the weights arrive: 512 heads of 4,097 slots 15.9 us, of 8,192 27.0.  (512 threads: one token of 4,097 left in 21.2 us with the moves on an earlier
// step, with 256 in 23.5, with 1,024 in 25.6.)
template <int I>
__global__ __launch_bounds__(kSelectThreads, I <= 17 ? 4 : 2) void k_select(EvictArgs a) {
    constexpr uint32_t kBins = 2048, kEach = kBins / kSelectThreads;
    __shared__ uint32_t bins[kBins], sums[kSelectWaves], fillers_of[kSelectWaves], digit, next_rank, whole;
    __shared__ uint16_t hole_of[I * kSelectThreads / 2];
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid / 64);
    const Unit u(a);
    const uint32_t part = (u.len + kSelectThreads - 1) / kSelectThreads * 64, from = wave * part + lane;
    float w[I];
    int32_t position[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {  // (all at once, before anything is known of the sequence; behind the last slot the last one again)
        const int64_t at = min(from + 64 * i, (uint32_t)a.width - 1);
        w[i] = a.width ? u.weights[at] : 0.f;
        position[i] = a.width ? u.positions[at] : 0;
    }
#pragma unroll
    for (uint32_t k = 0; k < kEach; ++k) bins[tid + k * kSelectThreads] = 0;
    if (u.settled(a)) return;  // (past a barrier)
    const uint32_t len = u.len, keep = u.keep;
    uint32_t key[I];
    bool mine[I];
#pragma unroll
    for (int i = 0; i < I; ++i) {
        mine[i] = 64u * i < part && from + 64 * i < len;
        key[i] = key_of(w[i], position[i], u.safe_from);
    }
    uint32_t prefix = 0, rank = len - keep;  // the rank-th smallest (from 1) of the keys that begin as prefix does
    const auto pass = [&](auto shift_, auto bits_) {  // -> whether all keys that begin with the digits found leave: no more of them are needed, prefix is the key behind those
        constexpr int shift = decltype(shift_)::value, bits = decltype(bits_)::value;
#pragma unroll
        for (int i = 0; i < I; ++i)
            if (mine[i] && key[i] != kSafe && (shift + bits == 32 || (key[i] ^ prefix) >> (shift + bits & 31) == 0)) atomicAdd(&bins[key[i] >> shift & (1u << bits) - 1], 1u);
        __syncthreads();
        uint32_t n[kEach], here = 0;
#pragma unroll
        for (uint32_t k = 0; k < kEach; ++k) {
            here += n[k] = bins[kEach * tid + k];
            bins[kEach * tid + k] = 0;  // (for the next one, two barriers from here)
        }
        uint32_t upto = sum_upto(here);
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        const Before others(sums, wave);
        if (rank > others.all) {  // tokens that are safe leave too (and are not counted: they are in a row, and would wait for each other)
            prefix = kSafe;
            rank -= others.all;
            __syncthreads();  // (the sums are used again)
            return true;
        }
        upto += others.here;
        uint32_t before = upto - here;
        if (before < rank && rank <= upto) {  // (one thread)
            uint32_t k = 0, count = n[0];
#pragma unroll
            for (uint32_t j = 0; j + 1 < kEach; ++j)
                if (k == j && before + n[j] < rank) before += n[j], k = j + 1, count = n[j + 1];
            digit = kEach * tid + k;
            next_rank = rank - before;
            whole = count == rank - before;
        }
        __syncthreads();
        prefix |= digit << shift;
        rank = next_rank;
        if (!whole) return false;
        prefix += (1u << shift) - (prefix >> shift == kSafe >> shift ? 1 : 0);  // (the last such keys end below kSafe)
        rank = 0;
        return true;
    };
    if (!pass(Number<21>(), Number<11>()) && !pass(Number<10>(), Number<11>())) pass(Number<0>(), Number<10>());
    // keys below `prefix` leave, and the first `rank` that equal it
    uint32_t equal = 0;
#pragma unroll
    for (int i = 0; i < I; ++i) equal += __popcll(__ballot(mine[i] && key[i] == prefix));
    if (lane == 0) sums[wave] = equal;
    __syncthreads();
    uint32_t seen = Before(sums, wave).here;
    bool hole[I], filler[I];
    uint32_t holes = 0, fillers = 0;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const uint64_t same = __ballot(mine[i] && key[i] == prefix);
        const bool leaves = mine[i] && (key[i] < prefix || (key[i] == prefix && seen + before_lane(same) < rank));
        seen += __popcll(same);
        hole[i] = leaves && from + 64 * i < keep;
        filler[i] = mine[i] && !leaves && from + 64 * i >= keep;
        holes += __popcll(__ballot(hole[i]));
        fillers += __popcll(__ballot(filler[i]));
    }
    __syncthreads();  // (the sums are used again)
    if (lane == 0) sums[wave] = holes, fillers_of[wave] = fillers;
    __syncthreads();
    const Before holes_before(sums, wave);
    uint32_t hole_at = holes_before.here, filler_at = Before(fillers_of, wave).here;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const uint32_t t = from + 64 * i;
        const uint64_t all = __ballot(hole[i]);
        if (hole[i]) hole_of[hole_at + before_lane(all)] = (uint16_t)t;
        hole_at += __popcll(all);
        if (!hole[i] && mine[i] && t < keep) {
            if (u.weights_out != u.weights) u.weights_out[t] = w[i];
            if (u.positions_out != u.positions) u.positions_out[t] = position[i];
        }
    }
    if (tid == 0) a.counts[blockIdx.x] = (int32_t)holes_before.all;
    __syncthreads();
    int32_t* hole_list = a.holes + (int64_t)blockIdx.x * a.most;
    int32_t* filler_list = a.fillers + (int64_t)blockIdx.x * a.most;
#pragma unroll
    for (int i = 0; i < I; ++i) {
        const uint64_t all = __ballot(filler[i]);
        if (filler[i]) {
            const uint32_t j = filler_at + before_lane(all), to = hole_of[j];
            hole_list[j] = (int32_t)to;
            filler_list[j] = (int32_t)(from + 64 * i);
            u.weights_out[to] = w[i];
            u.positions_out[to] = position[i];
        }
        filler_at += __popcll(all);
    }
}

struct LongLds {
    uint32_t keys[kKeysKept];
    uint32_t bins[256];
    uint32_t ties[kSelectWaves], holes[kSelectWaves], fillers[kSelectWaves];
    uint32_t digit, rank;
};

// ---- more than 16,384 slots: the same, with keys that are made again each time they are needed, 8 bits at a time.  128 heads of 16,385 slots, of which one leaves: 109 us, where 16,368 take 28 in
// registers.
__global__ __launch_bounds__(kSelectThreads) void k_select_long(EvictArgs a) {
    __shared__ LongLds lds;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid / 64);
    const Unit u(a);
    if (u.settled(a)) return;
    const uint32_t len = u.len, keep = u.keep;
    const float* weights = u.weights;
    const int32_t* positions = u.positions;
    float* weights_out = u.weights_out;
    int32_t* positions_out = u.positions_out;
    const int64_t unit = blockIdx.x;
    const auto make_key = [&](uint32_t t) { return key_of(weights[t], positions[t], u.safe_from); };
    const bool kept = len <= kKeysKept;
    const auto key = [&](uint32_t t) { return kept ? lds.keys[t] : make_key(t); };
    if (kept)
        for (uint32_t t = tid; t < len; t += kSelectThreads) lds.keys[t] = make_key(t);
    uint32_t prefix = 0, rank = len - keep;  // the rank-th smallest (from 1) of the keys that begin as prefix does
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) lds.bins[tid] = 0;
        __syncthreads();
        for (uint32_t t = tid; t < len; t += kSelectThreads) {
            const uint32_t k = key(t);
            if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&lds.bins[k >> shift & 255], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            uint32_t n[4], mine = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += n[j] = lds.bins[4 * lane + j];
            uint32_t upto = mine;
#pragma unroll
            for (int k = 1; k < 64; k *= 2) {
                const uint32_t o = __shfl_up(upto, k);
                if (lane >= (uint32_t)k) upto += o;
            }
            uint32_t before = upto - mine;
            if (before < rank && rank <= upto) {  // (one lane)
                uint32_t j = 0;
                while (before + n[j] < rank) before += n[j++];
                lds.digit = 4 * lane + j;
                lds.rank = rank - before;
            }
        }
        __syncthreads();
        prefix |= lds.digit << shift;
        rank = lds.rank;
    }
    // keys below `prefix` leave, and the first `rank` that equal it.  Each wave goes through slots in a row, 64 at a time.
    const uint32_t part = (len + kSelectThreads - 1) / kSelectThreads * 64, from = min(wave * part, len), to = min(from + part, len);
    uint32_t ties = 0;
    for (uint32_t t = from + lane; t - lane < to; t += 64) ties += __popcll(__ballot(t < to && key(t) == prefix));
    if (lane == 0) lds.ties[wave] = ties;
    __syncthreads();
    uint32_t ties_before = 0;
    for (uint32_t w = 0; w < wave; ++w) ties_before += lds.ties[w];
    const auto walk = [&](auto each) {  // each(t, hole, filler, which lanes have holes, which have fillers)
        uint32_t seen = ties_before;
        for (uint32_t t = from + lane; t - lane < to; t += 64) {
            const uint32_t k = t < to ? key(t) : 0xFFFFFFFFu;
            const uint64_t equal = __ballot(t < to && k == prefix);
            const bool leaves = t < to && (k < prefix || (k == prefix && seen + before_lane(equal) < rank));
            seen += __popcll(equal);
            const bool hole = leaves && t < keep, filler = t < to && !leaves && t >= keep;
            each(t, hole, filler, __ballot(hole), __ballot(filler));
        }
    };
    uint32_t holes = 0, fillers = 0;
    walk([&](uint32_t, bool, bool, uint64_t h, uint64_t f) { holes += __popcll(h), fillers += __popcll(f); });
    if (lane == 0) lds.holes[wave] = holes, lds.fillers[wave] = fillers;
    __syncthreads();
    uint32_t hole_at = 0, filler_at = 0, count = 0;
    for (uint32_t w = 0; w < kSelectWaves; ++w) {
        if (w < wave) hole_at += lds.holes[w], filler_at += lds.fillers[w];
        count += lds.holes[w];
    }
    int32_t* hole_list = a.holes + unit * a.most;
    int32_t* filler_list = a.fillers + unit * a.most;
    walk([&](uint32_t t, bool hole, bool filler, uint64_t h, uint64_t f) {
        if (hole) hole_list[hole_at + before_lane(h)] = (int32_t)t;
        if (filler) filler_list[filler_at + before_lane(f)] = (int32_t)t;
        hole_at += __popcll(h);
        filler_at += __popcll(f);
        if (!hole && t < to && t < keep) {
            if (weights_out != weights) weights_out[t] = weights[t];
            if (positions_out != positions) positions_out[t] = positions[t];
        }
    });
    if (tid == 0) a.counts[unit] = (int32_t)count;
    __syncthreads();
    for (uint32_t j = tid; j < count; j += kSelectThreads) {
        const int32_t hole = hole_list[j], filler = filler_list[j];
        weights_out[hole] = weights[filler];
        positions_out[hole] = positions[filler];
    }
}

// ---- the rows move: the moves of all sequences and heads, in equal shares to the workgroups, 64 at a time: a thread each finds where they go from and to, then the workgroup moves them, a lane per 16 bytes
// of keys or values (and the exponent that belongs to them).  Bound by memory: half of 8,192 tokens of 64 sequences, 8 KV heads of 128 channels, 0.54 GB that are read and written in rows of 256
// bytes, 226 us, 4.7 TB/s (0.3 GB in 4 bits, rows of 64 bytes and exponents one by one: 93 us, 3.3 TB/s); one token of each head 4.2 us.
constexpr uint32_t kMoveGroups = 2048, kMoves = 64;

template <bool FP4>
__global__ __launch_bounds__(256) void k_move_rows(EvictArgs a) {
    __shared__ Sums sums;
    struct Move {
        int64_t from, to;        // bytes from the beginning of a cache to a row's page, and FP16: to the row
        uint32_t row_from, row_to;
    };
    __shared__ Move moves[kMoves];
    const uint32_t units = (uint32_t)a.n_seq * a.n_kv, tid = threadIdx.x;
    if (blockIdx.x == 0)
        for (uint32_t s = tid; s < (uint32_t)a.n_seq; s += 256) a.new_lens[s] = a.left[s];
    const auto count_of = [&](uint32_t u) { return (uint32_t)a.counts[u]; };
    add_up(sums, units, count_of);
    const uint32_t all = sums.all, each = share(all, gridDim.x);
    uint32_t begin = blockIdx.x * each;
    if (begin >= all) return;
    const uint32_t end = min(begin + each, all), lanes = (uint32_t)(FP4 ? a.g.d / 32 : a.g.lpr);  // of a row
    for (; begin < end; begin += kMoves) {
        const uint32_t n = min(kMoves, end - begin);
        __syncthreads();
        if (tid < n) {
            const Item it = find_item(sums, units, begin + tid, count_of);
            const int64_t at = (int64_t)it.i * a.most + (begin + tid - it.start);
            const uint32_t s = fast_div(it.i, a.by_n_kv), h = it.i - s * a.n_kv, from = (uint32_t)a.fillers[at], to = (uint32_t)a.holes[at];
            const uint32_t in_from = fast_div(from, a.by_N), in_to = fast_div(to, a.by_N);
            const int64_t b_from = a.table[(int64_t)s * a.max_blocks + in_from], b_to = a.table[(int64_t)s * a.max_blocks + in_to];
            Move m;
            m.row_from = from - in_from * (uint32_t)a.g.N;
            m.row_to = to - in_to * (uint32_t)a.g.N;
            if (FP4) {
                m.from = b_from * a.f.block + (int64_t)h * a.f.page;
                m.to = b_to * a.f.block + (int64_t)h * a.f.page;
            } else {
                m.from = 2 * (b_from * a.g.block_stride + h * a.g.page_stride + m.row_from * a.g.row_stride);
                m.to = 2 * (b_to * a.g.block_stride + h * a.g.page_stride + m.row_to * a.g.row_stride);
            }
            moves[tid] = m;
        }
        __syncthreads();
        const uint32_t items = n * 2 * lanes;
        constexpr uint32_t kAtOnce = 4;
        for (uint32_t i0 = tid; i0 < items; i0 += 256 * kAtOnce) {
            uint4v r[kAtOnce];
            uint8_t e[kAtOnce];
            uint8_t* to[kAtOnce];
            uint8_t* exp_to[kAtOnce];
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j) {
                const uint32_t i = i0 + 256 * j;
                to[j] = nullptr;
                if (i < items) {
                    const uint32_t row = fast_div(i, a.by_lanes), c = i - row * lanes;
                    const Move& m = moves[row >> 1];
                    uint8_t* base = row & 1 ? a.v : a.k;
                    if (FP4) {
                        const uint8_t* from = base + m.from;
                        r[j] = *reinterpret_cast<const uint4v*>(from + m.row_from * (uint32_t)(a.g.d / 2) + 16 * c);
                        e[j] = from[a.f.exps + c * (uint32_t)a.g.N + m.row_from];
                        to[j] = base + m.to + m.row_to * (uint32_t)(a.g.d / 2) + 16 * c;
                        exp_to[j] = base + m.to + a.f.exps + c * (uint32_t)a.g.N + m.row_to;
                    } else {
                        r[j] = *reinterpret_cast<const uint4v*>(base + m.from + 16 * c);
                        to[j] = base + m.to + 16 * c;
                    }
                }
            }
#pragma unroll
            for (uint32_t j = 0; j < kAtOnce; ++j)
                if (to[j]) {
                    __builtin_nontemporal_store(r[j], reinterpret_cast<uint4v*>(to[j]));
                    if (FP4) *exp_to[j] = e[j];
                }
        }
    }
}

hipError_t launch_evict(const EvictArgs& a, hipStream_t s) {
    constexpr int per = (int)kSelectThreads;
    const auto select = a.width <= 2 * per ? k_select<2> : a.width <= 5 * per ? k_select<5> : a.width <= 9 * per ? k_select<9> : a.width <= 17 * per ? k_select<17> : a.width <= 32 * per ? k_select<32> : k_select_long;
    const hipError_t e = launch_kernel(select, dim3((unsigned)a.n_seq * (unsigned)a.n_kv), dim3(kSelectThreads), s, a);
    return e != hipSuccess ? e : launch_kernel(a.fp4 ? k_move_rows<true> : k_move_rows<false>, dim3(kMoveGroups), dim3(256), s, a);
}

}  // namespace kvc
