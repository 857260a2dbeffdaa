// The attention weight that tokens get, compiled once per head dimension (-DKVC_HEAD_DIM=d): W[s][h][t] += sum over the queries of head h's group that see t of e^(scale <q, k_t> - lse).
//
// Scores are made with queries as rows and tokens as columns, S = Q K^T, so that a lane of group g = lane / 16 has four queries' scores of one token: they are added in the lane, then over the four
// groups.  A token's weight is written by one lane in one order: the same call gives the same bits.
#include "kvc_attend_fp4.h"

#ifndef KVC_HEAD_DIM
#error "KVC_HEAD_DIM: the head dimension to compile"
#endif

namespace kvc {

// tokens of sequence s that weights are kept for
__device__ inline uint32_t weighed_length(const WeighArgs& x, int s) {
    const uint32_t len = own_length(x.a, s);
    if (len <= (uint32_t)x.width) return len;
    atomicOr(&x.a.st->status, KVC_ST_BAD_INDEX);
    return (uint32_t)x.width;
}
__device__ inline SourceFp4 keys_of(const WeighArgs& x, uint32_t s, uint32_t h, uint32_t len) {
    return SourceFp4{x.a.table + (int64_t)s * x.a.max_blocks, len, x.k ? x.k + (int64_t)h * x.f.page : reinterpret_cast<const uint8_t*>(x.a.k_cache + h * x.a.g.page_stride), nullptr};
}

// Keys of 32 tokens on their way: token 8 * (n / 4) + 4u + n % 4 of them is column n of score tile u.
template <int D, bool FP4, bool EIGHT>
struct KeyTile {
    KeysFp4<D> packed;
    uint4v keys[2][D / 32];
    uint32_t there;  // bit u

    __device__ void load(const WeighArgs& x, const SourceFp4& s, const Spots<EIGHT>& spots, uint32_t t, bool live, bool& bad) {
        const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, first = t + 8 * (n >> 2) + (n & 3);
        there = 0;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const Spot at = key_spot<EIGHT>(spots, u);
            const bool have = is_there(x.a, at.block, live && first + 4 * u < s.len, bad);
            there |= have ? 1u << u : 0u;
            if constexpr (!FP4) {
                // (strides are multiples of 8 elements, and counted in these)
                const uint64_t chunk = (uint64_t)(uint32_t)at.block * (uint32_t)(x.a.g.block_stride / 8) + (uint64_t)at.row * (uint32_t)(x.a.g.row_stride / 8);
                const bytes_at row = have ? (bytes_at)s.k + 16 * chunk : (bytes_at)kZeroRow;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) keys[u][c] = load_from<uint4v>(row + 64 * c + 16 * g);
            }
        }
        if constexpr (FP4) load_keys<D, EIGHT>(packed, x.a, x.f, s, spots, t, live, bad);
    }
    __device__ void expand(uint4v (&to)[2][D / 32]) const {
        if constexpr (FP4) {
            Tokens<D> tokens;
            expand_keys<D, EIGHT>(tokens, packed);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int c = 0; c < D / 32; ++c) to[u][c] = tokens.k[u][c];
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int c = 0; c < D / 32; ++c) to[u][c] = keys[u][c];
        }
    }
};

// Query row `row` of a sequence and KV head: its token, and where it and its sum are.
struct Row {
    uint32_t i, head;
    __device__ Row(const AttendArgs& a, uint32_t h, uint32_t row) {
        const uint32_t in = fast_div(row, a.by_n_q);
        i = row - in * a.n_q;
        head = h * a.group + in;
    }
    __device__ const uint16_t* query(const AttendArgs& a, uint32_t s) const { return a.q + s * a.q_strides[0] + i * a.q_strides[1] + head * a.q_strides[2]; }
    __device__ float lse(const AttendArgs& a, uint32_t s) const { return a.lse[((int64_t)s * a.n_q + i) * a.n_heads + head]; }
    // -lse in powers of two; a query that sees nothing gives weights of zero
    __device__ static float low(float lse) { return lse == -INFINITY ? -INFINITY : -lse * 1.44269504088896341f; }
    // tokens it sees
    __device__ uint32_t limit(const AttendArgs& a, uint32_t full, uint32_t len) const {
        const uint32_t later = a.n_q - 1 - i;
        return min(full > later ? full - later : 0, len);
    }
};

// 16 queries, and of the lane's four (4g..4g+3): -lse, and the tokens they see.
template <int D>
struct Queries {
    uint4v q[D / 32];
    float low[4];
    uint32_t limit[4];

    template <bool FP4>
    __device__ void load(const WeighArgs& x, uint32_t s, uint32_t h, uint32_t full, uint32_t len, uint32_t rt) {
        const AttendArgs& a = x.a;
        const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, last = (uint32_t)a.rows - 1;
        {
            const uint16_t* from = Row(a, h, min(rt * 16 + n, last)).query(a, s);
            if constexpr (FP4) {
                load_query<D>(q, from, g);
            } else {
#pragma unroll
                for (int k = 0; k < D / 32; ++k) q[k] = *reinterpret_cast<const uint4v*>(from + 32 * k + 8 * g);
            }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t row = rt * 16 + 4 * g + r;
            const Row of(a, h, min(row, last));
            low[r] = Row::low(of.lse(a, s));
            limit[r] = row <= last ? of.limit(a, full, len) : 0;
        }
    }
};

template <int D>
__device__ inline void score(float4v (&s)[2], const uint4v (&q)[D / 32], const uint4v (&k)[2][D / 32]) {
    s[0] = s[1] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, q[c]), __builtin_bit_cast(half8, k[u][c]), s[u], 0, 0, 0);
}
// ALL: every query sees every token.
template <bool ALL>
__device__ inline void add_weights(float (&sum)[2], const float4v (&s)[2], float scale_log2, const float (&low)[4], const uint32_t (&limit)[4], uint32_t token) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float w = power2(fmaf(s[u][r], scale_log2, low[r]));
            sum[u] += ALL || token + 4 * u < limit[r] ? w : 0.f;
        }
}

template <bool B>
struct Flag {
    static constexpr bool value = B;
};

// What a lane's tokens got, added to what they had, and positions of those that are new.
struct Result {
    float* after;
    int32_t* positions;

    // lanes 0 to 31 write a token each, this one
    __device__ static uint32_t token(uint32_t t) {
        const uint32_t lane = threadIdx.x & 63;
        return t + 8 * ((lane & 15) >> 2) + 4 * (lane >> 4 & 1) + (lane & 3);
    }
    __device__ void store(float (&sum)[2], uint32_t there, float had, const WeighArgs& x, uint32_t t, uint32_t full, uint32_t len, int32_t seen) const {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sum[u] = row_sum(sum[u]);
            if (!(there >> u & 1)) sum[u] = 0.f;
        }
        const uint32_t lane = threadIdx.x & 63, at = token(t), from_end = full - at;
        if (lane >= 32 || at >= len) return;
        const bool is_new = from_end <= (uint32_t)x.a.n_q;
        after[at] = (is_new ? 0.f : had) + (lane < 16 ? sum[0] : sum[1]);
        if (is_new) positions[at] = (int32_t)((uint32_t)seen - from_end);
    }
};
__device__ inline Result result_of(const WeighArgs& x, uint32_t s, uint32_t h) {
    const int64_t at = ((int64_t)s * x.a.n_kv + h) * x.width;
    return Result{x.after + at, x.positions + at};
}

// ---- few queries: bound by memory.  Work is divided as attention divides it, a unit being a sequence and a KV head, and tiles are on their way as in k_own_fp4.  ONE: a head has 16 queries
// or fewer, which stay in registers.  64 sequences of 512 to 8,192 tokens, 8 KV heads of 128 channels, 8 query heads each, FP16: 117 us, 589 MB at 5.0 TB/s, where a copy reaches 5.7.
template <int D, bool FP4, bool EIGHT, bool ONE>
__global__ __launch_bounds__(256, D <= 128 ? 2 : 1) void k_weigh(WeighArgs x) {
    __shared__ Sums sums;
    const AttendArgs& a = x.a;
    const uint32_t worker = uniform(blockIdx.x * 4 + threadIdx.x / 64);
    const auto tiles_of = [&](uint32_t s) { return (weighed_length(x, s) + kTile - 1) / kTile; };
    add_up(sums, a.n_seq, tiles_of);
    const uint32_t units = a.n_kv, all = uniform(sums.all) * units, each = share(all, x.workers);
    const uint32_t begin = worker * each, end = min(begin + each, all);
    if (begin >= end) return;

    Place c;
    {
        const Item it = find_item(sums, a.n_seq, begin / units, tiles_of);
        c.s = uniform(it.i);
        c.len = uniform(weighed_length(x, c.s));
        c.tiles = (c.len + kTile - 1) / kTile;
        const uint32_t rel = begin - uniform(it.start) * units;
        c.u = rel / c.tiles;
        c.t = rel - c.u * c.tiles;
    }
    uint32_t left = end - begin;
    const auto next = [&](const Place& p, uint32_t ahead) {
        Place n = p;
        if (left <= ahead || ++n.t < n.tiles) return n;
        n.t = 0;
        if (++n.u < units) return n;
        n.u = 0;
        do {
            ++n.s;
            n.len = uniform(weighed_length(x, n.s));
        } while (n.len == 0);
        n.tiles = (n.len + kTile - 1) / kTile;
        return n;
    };
    struct Ahead {
        KeyTile<D, FP4, EIGHT> keys;
        float had;
    };
    bool bad = false;
    Finder<EIGHT> finder;
    const auto find = [&](const Place& p, bool first) { return finder.find(a, a.table + (int64_t)p.s * a.max_blocks, p.len, p.t, first); };
    const auto load = [&](Ahead& to, const Place& p, const Spots<EIGHT>& spots, bool live) {
        to.keys.load(x, keys_of(x, p.s, p.u, p.len), spots, p.t * kTile, live, bad);
        to.had = load_from<float>((bytes_at)(x.before + ((int64_t)p.s * a.n_kv + p.u) * x.width + min(Result::token(p.t * kTile), p.len - 1)));
    };

    const uint32_t lane = threadIdx.x & 63, row_tiles = (a.rows + 15) / 16;
    Queries<D> q;
    uint32_t full;
    int32_t seen;
    const auto open = [&](const Place& p) {
        full = uniform((uint32_t)a.lens[p.s]);
        seen = x.seen[p.s];
        if (ONE) q.template load<FP4>(x, p.s, p.u, full, p.len, 0);
        asm volatile("" : "+v"(seen));  // (waited for here, not in every step)
#pragma unroll
        for (int k = 0; k < D / 32; ++k) asm volatile("" : "+v"(q.q[k]));
    };
    // c: the tile computed; c1 and c2: those on their way; c3: the one whose blocks are looked up
    Ahead tiles[3];
    Place c1 = next(c, 1), c2 = next(c1, 2);
    const Spots<EIGHT> at = find(c, true), at1 = find(c1, c1.t == 0);
    Spots<EIGHT> at2 = find(c2, c2.t == 0);
    open(c);
    load(tiles[0], c, at, true);
    load(tiles[1], c1, at1, left > 1);
    const auto step = [&](Ahead& now, Ahead& then) {  // -> whether it was the last one
        const Place c3 = next(c2, 3);
        const Spots<EIGHT> at3 = find(c3, c3.t == 0);
        __builtin_amdgcn_sched_barrier(0);
        load(then, c2, at2, left > 2);
        __builtin_amdgcn_sched_barrier(0);
        const uint32_t t = c.t * kTile, token = t + 8 * ((lane & 15) >> 2) + (lane & 3);
        uint4v keys[2][D / 32];
        now.keys.expand(keys);
        float sum[2] = {0.f, 0.f};
        float4v s[2];
        if (ONE) {
            score<D>(s, q.q, keys);
            add_weights<false>(sum, s, a.scale_log2, q.low, q.limit, token);
        } else {
            for (uint32_t rt = 0; rt < row_tiles; ++rt) {
                q.template load<FP4>(x, c.s, c.u, full, c.len, rt);
                score<D>(s, q.q, keys);
                add_weights<false>(sum, s, a.scale_log2, q.low, q.limit, token);
            }
        }
        result_of(x, c.s, c.u).store(sum, now.keys.there, now.had, x, t, full, c.len, seen);
        if (left == 1) return true;
        if (c1.t == 0) open(c1);
        c = c1;
        c1 = c2;
        c2 = c3;
        at2 = at3;
        --left;
        return false;
    };
    while (!step(tiles[0], tiles[2]) && !step(tiles[1], tiles[0]) && !step(tiles[2], tiles[1])) {
    }
    if (bad) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
}

// ---- many queries: bound by the products, the powers and reading LDS.  A workgroup takes 64 tokens of a sequence and head, whose keys stay in the registers of every wave; 64 queries at a time come to LDS, the next
// ones on their way meanwhile, with their -lse and the tokens they see, and each wave takes 16 of them.
// 256 queries of 64 heads, 4 prompts of 1,024 to 2,048 tokens, 8 KV heads of 128 channels in 4 bits: 42 us among other calls, 610 TFLOP/s with one power for every
// 256 FLOP; 44 to 48 where such calls follow each other with nothing between them, as the clock falls then.
constexpr uint32_t kChunk = 2 * kTile;
template <int D, bool FP4, bool EIGHT>
__global__ __launch_bounds__(256, D <= 128 && (EIGHT || !FP4 || D <= 96) ? 3 : 2) void k_weigh_many(WeighArgs x) {
    constexpr uint32_t kStride = 2 * D + 16;  // bytes of a query in LDS: 16 lanes that read the same channels of 16 queries meet in no bank
    constexpr uint32_t kRows = 64;
    constexpr uint32_t kLanes = 256 / kRows, kPieces = (D / 8 + kLanes - 1) / kLanes;  // threads that load a query, and pieces of 16 bytes of each
    __shared__ Sums sums;
    __shared__ __align__(16) uint8_t queries[2][kRows * kStride];
    __shared__ __align__(16) float lows[2][kRows];
    __shared__ __align__(16) uint32_t limits[2][kRows];
    __shared__ float of_waves[4][4][64];  // [wave][score tile][lane]: sums
    const AttendArgs& a = x.a;
    const uint32_t tid = threadIdx.x, lane = tid & 63, wave = uniform(tid / 64), n = lane & 15, g = lane >> 4, stages = (a.rows + kRows - 1) / kRows;
    const auto chunks_of = [&](uint32_t s) { return (weighed_length(x, s) + kChunk - 1) / kChunk; };
    add_up(sums, a.n_seq, chunks_of);
    const uint32_t all = uniform(sums.all) * a.n_kv;
    bool bad = false;
    // (workgroups go to the XCDs in turn: an XCD's take neighbouring chunks, whose queries are the same)
    const uint32_t of_xcd = (all + 7) / 8, first = blockIdx.x % 8 * of_xcd, last = min(first + of_xcd, all);
    for (uint32_t chunk = first + blockIdx.x / 8; chunk < last; chunk += gridDim.x / 8) {
        const Item it = find_item(sums, a.n_seq, chunk / a.n_kv, chunks_of);
        const uint32_t s = uniform(it.i), len = uniform(weighed_length(x, s)), chunks = (len + kChunk - 1) / kChunk, rel = chunk - uniform(it.start) * a.n_kv, h = rel / chunks;
        const uint32_t t = (rel - h * chunks) * kChunk, full = uniform((uint32_t)a.lens[s]);
        uint4v ahead[kPieces];
        float lse_ahead = 0.f;
        uint32_t limit_ahead = 0;
        const auto ask = [&](uint32_t stage) {
            const bytes_at from = (bytes_at)Row(a, h, min(stage * kRows + tid / kLanes, (uint32_t)a.rows - 1)).query(a, s);
#pragma unroll
            for (uint32_t k = 0; k < kPieces; ++k) ahead[k] = load_from<uint4v>(from + 16 * min(kLanes * k + tid % kLanes, D / 8 - 1u));
            if (tid < kRows) {
                const uint32_t row = stage * kRows + tid;
                const Row of(a, h, min(row, (uint32_t)a.rows - 1));
                lse_ahead = of.lse(a, s);  // (and no more, which would be to wait for it here)
                limit_ahead = row < (uint32_t)a.rows ? of.limit(a, full, len) : 0;
            }
        };
        const auto put = [&](uint32_t buffer) {
#pragma unroll
            for (uint32_t k = 0; k < kPieces; ++k) {
                const uint32_t c = kLanes * k + tid % kLanes;
                if (c < D / 8) *reinterpret_cast<uint4v*>(&queries[buffer][tid / kLanes * kStride + c * 16]) = ahead[k];
            }
            if (tid < kRows) lows[buffer][tid] = Row::low(lse_ahead), limits[buffer][tid] = limit_ahead;
        };
        const SourceFp4 src = keys_of(x, s, h, len);
        Finder<EIGHT> finder;
        KeyTile<D, FP4, EIGHT> tile[2];
        const Spots<EIGHT> at = finder.find(a, src.table, len, t / kTile, true), at1 = finder.find(a, src.table, len, t / kTile + 1, false);
        tile[0].load(x, src, at, t, true, bad);
        tile[1].load(x, src, at1, t + kTile, t + kTile < len, bad);
        ask(0);
        uint4v keys[2][2][D / 32];
        float had[2], sum[2][2] = {};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            tile[j].expand(keys[j]);
            had[j] = load_from<float>((bytes_at)(x.before + ((int64_t)s * a.n_kv + h) * x.width + min(Result::token(t + j * kTile), len - 1)));
        }
        const uint32_t token = t + 8 * (n >> 2) + (n & 3);
        // (queries that see all of the chunk, and exist, need no comparison)
        const bool all_seen = t + kChunk + a.n_q <= full + 1 && t + kChunk <= len;
        for (uint32_t stage = 0; stage < stages; ++stage) {
            const uint32_t buffer = stage & 1;
            put(buffer);  // (the waves that read this buffer are past the last barrier)
            __syncthreads();
            if (stage + 1 < stages) ask(stage + 1);
            const auto add = [&](auto all_) {
                const uint32_t r = 16 * wave;
                const uint16_t* row = reinterpret_cast<const uint16_t*>(&queries[buffer][(r + n) * kStride]);
                const float4v l = *reinterpret_cast<const float4v*>(&lows[buffer][r + 4 * g]);
                const float low[4] = {l[0], l[1], l[2], l[3]};
                const uint4v m = *reinterpret_cast<const uint4v*>(&limits[buffer][r + 4 * g]);
                const uint32_t limit[4] = {m[0], m[1], m[2], m[3]};
                float4v sc[2][2];
#pragma unroll
                for (int k = 0; k < 4; ++k) sc[k / 2][k % 2] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    const half8 q = __builtin_bit_cast(half8, *reinterpret_cast<const uint4v*>(row + (FP4 ? query_channel<D>(c, g) : 32 * c + 8 * g)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) sc[k / 2][k % 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(q, __builtin_bit_cast(half8, keys[k / 2][k % 2][c]), sc[k / 2][k % 2], 0, 0, 0);
                    if (D > 192 && c % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (there are no registers for all of a query)
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) add_weights<decltype(all_)::value>(sum[j], sc[j], a.scale_log2, low, limit, token + j * kTile);
            };
            if (all_seen && (stage + 1) * kRows <= (uint32_t)a.rows) add(Flag<true>());
            else add(Flag<false>());
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) of_waves[wave][k][lane] = sum[k / 2][k % 2];
        __syncthreads();  // (and the buffers are used again)
        if (wave < 2) {  // a wave for each half of the tokens
            float all_waves[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const uint32_t k = 2 * wave + u;
                all_waves[u] = (of_waves[0][k][lane] + of_waves[1][k][lane]) + (of_waves[2][k][lane] + of_waves[3][k][lane]);
            }
            if (wave == 0) result_of(x, s, h).store(all_waves, tile[0].there, had[0], x, t, full, len, x.seen[s]);
            else result_of(x, s, h).store(all_waves, tile[1].there, had[1], x, t + kTile, full, len, x.seen[s]);
        }
        __syncthreads();
    }
    if (bad) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
}

template <int D, bool FP4, bool EIGHT>
static hipError_t launch_weigh_of(const WeighArgs& x, hipStream_t s) {
    if (x.many) return launch_kernel(k_weigh_many<D, FP4, EIGHT>, dim3(x.workers), dim3(256), s, x);
    return launch_kernel(x.a.rows <= 16 ? k_weigh<D, FP4, EIGHT, true> : k_weigh<D, FP4, EIGHT, false>, dim3(x.workers / 4), dim3(256), s, x);
}

template <>
hipError_t launch_weigh<KVC_HEAD_DIM>(const WeighArgs& x, hipStream_t s) {
    constexpr int D = KVC_HEAD_DIM;
    const bool eight = x.a.g.N % 8 == 0;
    if (x.k) return eight ? launch_weigh_of<D, true, true>(x, s) : launch_weigh_of<D, true, false>(x, s);
    return eight ? launch_weigh_of<D, false, true>(x, s) : launch_weigh_of<D, false, false>(x, s);
}

}  // namespace kvc
