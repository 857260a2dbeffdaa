// The attention weight that tokens get, compiled once per head dimension (-DKVC_HEAD_DIM=d): W[s][h][t] += sum over the queries of head h's group that see t of e^(scale <q, k_t> - lse).
//
// Scores are made with queries as rows and tokens as columns, S = Q K^T, so that a lane of group g has four queries' scores of one token: they are added in the lane, then over the four
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

// Keys of 32 tokens on their way, and what their tokens had.
template <int D, bool FP4, bool EIGHT>
struct KeyTile {
    KeysFp4<D> packed;
    Tokens<D> keys;
    float had;
    bool there[2];  // the lane's tokens

    __device__ void load(const WeighArgs& x, const SourceFp4& s, const Blocks<EIGHT>& b, const Place& p) {
        const uint32_t t = p.t * kTile;
        if constexpr (FP4) load_keys<D, EIGHT>(packed, x.a, x.f, s, b, t);
        else load_keys<D, EIGHT>(keys, x.a, s.at, b, t);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int32_t block = b.key(u);
            there[u] = block >= 0 && block < x.a.n_cache_blocks;
        }
        const uint32_t lane = threadIdx.x & 63, token = token_of(t);
        had = 0.f;
        if (lane < 32 && token < p.len && (int64_t)token < (int64_t)x.a.lens[p.s] - x.a.n_q) had = x.before[((int64_t)p.s * x.a.n_kv + p.u) * x.width + token];
    }
    __device__ const Tokens<D>& expand() {
        if constexpr (FP4) expand_keys<D, EIGHT>(keys, packed);
        return keys;
    }
    // token whose weight lanes 0 to 31 write
    __device__ static uint32_t token_of(uint32_t t) {
        const uint32_t lane = threadIdx.x & 63;
        return t + 8 * ((lane & 15) >> 2) + 4 * (lane >> 4 & 1) + (lane & 3);
    }
};

// 16 queries, and of the lane's four (4g..4g+3): -lse in powers of two, and the tokens they see.
template <int D>
struct Queries {
    uint4v q[D / 32];
    float low[4];
    uint32_t limit[4];

    template <bool FP4>
    __device__ void load(const WeighArgs& x, const Place& p, uint32_t rt) {
        const AttendArgs& a = x.a;
        const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, len = (uint32_t)a.lens[p.s];
        {
            const uint32_t row = min(rt * 16 + n, (uint32_t)a.rows - 1), in = fast_div(row, a.by_n_q), i = row - in * a.n_q;
            const uint16_t* from = a.q + p.s * a.q_strides[0] + i * a.q_strides[1] + (p.u * a.group + in) * a.q_strides[2];
            if constexpr (FP4) load_query<D>(q, from, g);
            else
#pragma unroll
                for (int k = 0; k < D / 32; ++k) q[k] = *reinterpret_cast<const uint4v*>(from + 32 * k + 8 * g);
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const uint32_t row = rt * 16 + 4 * g + r, in = fast_div(min(row, (uint32_t)a.rows - 1), a.by_n_q), i = min(row, (uint32_t)a.rows - 1) - in * a.n_q, later = a.n_q - 1 - i;
            const float lse = a.lse[((int64_t)p.s * a.n_q + i) * a.n_heads + p.u * a.group + in];
            low[r] = lse == -INFINITY ? -INFINITY : -lse * 1.44269504088896341f;  // (a query that sees nothing: weights of zero)
            limit[r] = row < (uint32_t)a.rows ? min(len > later ? len - later : 0, p.len) : 0;
        }
    }
};

template <int D>
__device__ inline void add_weights(float (&sum)[2], const WeighArgs& x, const Queries<D>& q, const Tokens<D>& k, uint32_t t) {
    float4v s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int c = 0; c < D / 32; ++c)
#pragma unroll
        for (int u = 0; u < 2; ++u)
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, q.q[c]), __builtin_bit_cast(half8, k.k[u][c]), s[u], 0, 0, 0);
    const uint32_t lane = threadIdx.x & 63, token = t + 8 * ((lane & 15) >> 2) + (lane & 3);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float w = power2(fmaf(s[u][r], x.a.scale_log2, q.low[r]));
            sum[u] += token + 4 * u < q.limit[r] ? w : 0.f;
        }
}

// Work is divided as attention divides it, a unit being a sequence and a KV head.  FEW: a head has 16 queries or fewer, which stay in registers.
template <int D, bool FP4, bool EIGHT, bool FEW>
__global__ __launch_bounds__(256, 2) void k_weigh(WeighArgs x) {
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
    const auto advance = [&](Place& p) {  // (there is a next tile)
        if (++p.t < p.tiles) return;
        p.t = 0;
        if (++p.u < units) return;
        p.u = 0;
        do {
            ++p.s;
            p.len = uniform(weighed_length(x, p.s));
        } while (p.len == 0);
        p.tiles = (p.len + kTile - 1) / kTile;
    };
    const auto source = [&](const Place& p) {
        return SourceFp4{Source{a.table + (int64_t)p.s * a.max_blocks, FP4 ? nullptr : a.k_cache + p.u * a.g.page_stride, nullptr, p.len}, FP4 ? x.k + (int64_t)p.u * x.f.page : nullptr, nullptr};
    };

    const uint32_t lane = threadIdx.x & 63, row_tiles = (a.rows + 15) / 16;
    Queries<D> q;
    // c: the tile computed; c1: the one loaded; c2: the one whose blocks are looked up
    Place c1 = c, c2 = c;
    uint32_t left = end - begin;
    KeyTile<D, FP4, EIGHT> here, next;
    Blocks<EIGHT> b = find_blocks<EIGHT>(a, source(c).at, c.t * kTile);
    if (FEW) q.template load<FP4>(x, c, 0);
    here.load(x, source(c), b, c);
    if (left > 1) {
        advance(c1);
        b = find_blocks<EIGHT>(a, source(c1).at, c1.t * kTile);
        c2 = c1;
    }
    const auto step = [&](KeyTile<D, FP4, EIGHT>& now, KeyTile<D, FP4, EIGHT>& then) {  // -> whether it was the last one
        if (left > 1) {
            then.load(x, source(c1), b, c1);
            if (left > 2) {
                advance(c2);
                b = find_blocks<EIGHT>(a, source(c2).at, c2.t * kTile);
            }
        }
        const uint32_t t = c.t * kTile;
        const Tokens<D>& keys = now.expand();
        float sum[2] = {0.f, 0.f};
        if (FEW) {
            add_weights(sum, x, q, keys, t);
        } else {
            for (uint32_t rt = 0; rt < row_tiles; ++rt) {
                q.template load<FP4>(x, c, rt);
                add_weights(sum, x, q, keys, t);
            }
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            sum[u] = row_sum(sum[u]);
            if (!now.there[u]) sum[u] = 0.f;
        }
        const uint32_t token = now.token_of(t);
        if (lane < 32 && token < c.len) {
            const int64_t at = ((int64_t)c.s * a.n_kv + c.u) * x.width + token;
            const int64_t from_end = (int64_t)a.lens[c.s] - token;
            x.after[at] = now.had + (lane < 16 ? sum[0] : sum[1]);
            if (from_end <= a.n_q) x.positions[at] = (int32_t)(x.seen[c.s] - from_end);
        }
        if (left == 1) return true;
        if (FEW && c1.t == 0) q.template load<FP4>(x, c1, 0);
        c = c1;
        c1 = c2;
        --left;
        return false;
    };
    while (!step(here, next) && !step(next, here)) {
    }
}

template <int D, bool FP4>
static hipError_t launch_weigh_of(const WeighArgs& x, hipStream_t s) {
    const bool eight = x.a.g.N % 8 == 0, few = x.a.rows <= 16;
    return launch_kernel(eight ? (few ? k_weigh<D, FP4, true, true> : k_weigh<D, FP4, true, false>) : (few ? k_weigh<D, FP4, false, true> : k_weigh<D, FP4, false, false>), dim3(x.workers / 4), dim3(256), s, x);
}

template <>
hipError_t launch_weigh<KVC_HEAD_DIM>(const WeighArgs& x, hipStream_t s) {
    return x.k ? launch_weigh_of<KVC_HEAD_DIM, true>(x, s) : launch_weigh_of<KVC_HEAD_DIM, false>(x, s);
}

}  // namespace kvc
