// Attention over a paged cache in 4 bits, compiled once per head dimension (-DKVC_HEAD_DIM=d).  The work is divided as attention over FP16 divides a call without prefixes
// (kvc_attend.hip), pieces are joined by its k_join, and a tile becomes FP16 in registers (kvc_attend_fp4.h).
#include "kvc_attend_fp4.h"

#ifndef KVC_HEAD_DIM
#error "KVC_HEAD_DIM: the head dimension to compile"
#endif

namespace kvc {

template <int D, bool EIGHT>
struct TileFp4 {
    KeysFp4<D> k;
    ValuesFp4<D, EIGHT> v;
    uint32_t there;

    __device__ void load(const AttendFp4Args& x, const SourceFp4& s, const Spots<EIGHT>& spots, uint32_t t, bool live, bool& bad) {
        load_keys<D, EIGHT>(k, x.a, x.f, s, spots, t, live, bad);
        there = load_values<D, EIGHT>(v, x.a, x.f, s, spots, t, live, bad);
    }
};

// Whether a value of the tile may not be finite: exponents from 141 on, of which append writes NaN's.  (Tokens that are not there have zeros.)
template <int D, bool EIGHT>
__device__ inline bool may_be_infinite(const ValuesFp4<D, EIGHT>& x) {
    uint32_t any = 0;
#pragma unroll
    for (int p = 0; p < piece_count(D); ++p)
#pragma unroll
        for (int i = 0; i < (EIGHT ? 2 : 8); ++i) any |= ((x.e[p][i] & 0x7F7F7F7Fu) + 0x73737373u) & x.e[p][i] & 0x80808080u;
    return __any(any != 0);
}

// Values of 8 tokens, times the rows' weights, two channels at a time (there are few registers); `mine`: rows for which the result is taken.
template <int D, int R, bool EIGHT, int P = 0>
__device__ inline void add_values_of(Rows<D> (&r)[R], const ValuesFp4<D, EIGHT>& x, const half8 (&p)[R], const bool (&mine)[R]) {
    if constexpr (P < piece_count(D)) {
        using Q = Piece<D, P>;
#pragma unroll
        for (int c = 0; c < Q::w / 2; ++c) {
            Tokens<32> two;  // (a piece of two channels a lane)
#pragma unroll
            for (int j = 0; j < 8; ++j) two.v[j][0] = __builtin_bit_cast(uint32_t, two_channels(x.c[j][P], exponent<EIGHT>(x.e[P], j), c));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const half8 v = __builtin_bit_cast(half8, value_column<32, 0>(two, j));
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    float4v& o = r[i].o[Q::before / 16 + 2 * c + j];
                    const float4v n = __builtin_amdgcn_mfma_f32_16x16x32_f16(v, p[i], o, 0, 0, 0);
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = mine[i] ? n[e] : o[e];
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        add_values_of<D, R, EIGHT, P + 1>(r, x, p, mine);
    }
}

template <int D, int R, bool EIGHT>
__device__ inline void make_scores(float4v (&s)[R][2], const Rows<D> (&r)[R], const KeysFp4<D>& k) {
    Tokens<D> tokens;
    expand_keys<D, EIGHT>(tokens, k);
#pragma unroll
    for (int j = 0; j < R; ++j) scores(s[j], r[j], tokens);
}

// Scores of tokens t + 8g.. become weights, as `weights` has it (kvc_attend.h); all: every row sees every token.  Whether a row's reference has to follow is asked lane by lane: its maximum over the four
// lanes is needed only then.  (A score is scaled first and made relative then, each rounded: in one step, against a reference that was rounded, the largest of scores beyond 2^27 would not be its own reference.)
template <int D>
__device__ inline half8 weights_of(Rows<D>& r, const float4v (&s)[2], float scale_log2, bool all, uint32_t there, uint32_t t, uint32_t limit) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = s[j / 4][j % 4] * scale_log2;
    if (!all) {
        const uint32_t first = t + 8 * ((threadIdx.x & 63) >> 4), n = limit > first ? limit - first : 0, seen = there & (n >= 8 ? 0xFFu : ~(~0u << n));
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = seen >> j & 1 ? v[j] : -INFINITY;
    }
    float top = fmaxf(v[0], v[1]);
#pragma unroll
    for (int j = 2; j < 8; ++j) top = fmaxf(top, v[j]);
    if (__any(top > r.m + kLag)) {  // (a row's first token too: its reference is -infinity)
        const float m = fmaxf(r.m, row_max(top)), f = r.m == -INFINITY ? 0.f : power2(r.m - m);
        r.m = m;
        r.l *= f;
#pragma unroll
        for (int i = 0; i < D / 16; ++i) r.o[i] *= f;
    }
    const float low = (r.m == -INFINITY ? 0.f : r.m) - kLift;
    float w[8];
    half8 p;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        w[j] = power2(v[j] - low);
        p[j] = (_Float16)w[j];
    }
    r.l += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
    return p;
}

// What a wave does with a tile's scores and values.  Among the last n_q tokens some rows see values that others do not, and weight zero times one that is not finite is NaN: there, rows that see
// so many of the tile's tokens are done by themselves, the other tokens' values being zero.  seen_by_all: tokens that every row sees.
template <int D, int R, bool EIGHT>
__device__ inline void add_tile_fp4(Rows<D> (&r)[R], const AttendFp4Args& x, TileFp4<D, EIGHT>& tile, const float4v (&s)[R][2], uint32_t t, uint32_t seen_by_all, const uint32_t (&limit)[R]) {
    const bool all = t + kTile <= seen_by_all && __all(tile.there == 0xFF);
    half8 p[R];
#pragma unroll
    for (int j = 0; j < R; ++j) p[j] = weights_of(r[j], s[j], x.a.scale_log2, all, tile.there, t, limit[j]);
    if (!all) {
        keep_values<D, EIGHT>(tile.v, tile.there);
        if (x.a.n_q > 1 && t + kTile > seen_by_all && may_be_infinite<D, EIGHT>(tile.v)) {
            const uint32_t first = t + 8 * ((threadIdx.x & 63) >> 4);
#pragma nounroll
            for (uint32_t cut = 1; cut <= kTile; ++cut) {  // rows that see the tile's first `cut` tokens, and no more
                bool mine[R], any = false;
#pragma unroll
                for (int j = 0; j < R; ++j) {
                    mine[j] = min(limit[j] > t ? limit[j] - t : 0, (uint32_t)kTile) == cut;
                    any = any || mine[j];
                }
                if (!__any(any)) continue;
                const uint32_t n = t + cut > first ? t + cut - first : 0;
                ValuesFp4<D, EIGHT> v = tile.v;
                keep_values<D, EIGHT>(v, n >= 8 ? 0xFFu : ~(~0u << n));
                add_values_of<D, R, EIGHT>(r, v, p, mine);
            }
            return;
        }
    }
    Tokens<D> tokens;
    expand_values<D, EIGHT>(tokens, tile.v);
    add_values<D, R>(r, tokens, p);
}

// ---- any lengths: a worker is a wave that takes tiles of one unit (a KV head and its rows), as many as any other, from sequence to sequence; two tiles are on their way while one is computed, the block numbers
// of a third are looked up.  For each tile of 32 tokens 34 d bytes are read and become FP16, and for each 16 rows there are d / 8 MFMAs: of up to 16 rows memory and instructions cost about the same, and
// neither hides the other fully.  64 sequences of 512 to 8,192 tokens, 8 KV heads of 128 channels, 8 query heads each: 65 us (and 6 to join), 305 MB at 4.7 TB/s, some 5 of them a chain of reads before the first tile (lengths, table, rows); on an earlier step that took 70, 66 with the products left out, 52 with all blocks in the caches.  2,048
// waves are what registers allow; 4,096 in two turns take 83.  With 24 and 32 rows it takes 104 and 106 at
// best, 110 and 114 on average in a row of calls: the registers leave one wave on a SIMD, whose conversions and products follow each other with nothing beside them; the products alone would take 28, the bytes 55.
template <int D, int R, bool EIGHT>
__device__ inline void own_part_fp4(const AttendFp4Args& x, Sums& sums, uint32_t worker) {
    const AttendArgs& a = x.a;
    const auto tiles_of = [&](uint32_t s) { return (own_length(a, s) + kTile - 1) / kTile; };
    add_up(sums, a.n_seq, tiles_of);
    if (worker < 4) write_starts(sums, a.own_start, a.n_seq, tiles_of);
    const uint32_t units = a.n_kv * a.own_tiles, all = uniform(sums.all), each = share(all, a.own_workers / units), range = worker / units;
    const uint32_t begin = range * each, end = min(begin + each, all);
    if (worker >= a.own_workers || begin >= end) return;

    Place c;
    {
        const Item it = find_item(sums, a.n_seq, begin, tiles_of);
        c.s = uniform(it.i);
        c.len = uniform(own_length(a, c.s));
        c.tiles = (c.len + kTile - 1) / kTile;
        c.u = worker - range * units;
        c.t = begin - uniform(it.start);
    }
    const auto advance = [&](Place& p) {  // (there is a next tile)
        if (++p.t < p.tiles) return;
        p.t = 0;
        do {
            ++p.s;
            p.len = uniform(own_length(a, p.s));
        } while (p.len == 0);
        p.tiles = (p.len + kTile - 1) / kTile;
    };
    const auto source = [&](const Place& p) {
        const uint32_t h = p.u / a.own_tiles;
        return SourceFp4{a.table + (int64_t)p.s * a.max_blocks, p.len, x.k + (int64_t)h * x.f.page, x.v + (int64_t)h * x.f.page};
    };

    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    Rows<D> r[R];
    uint32_t limit[R], seen_by_all = 0;
    // (where registers are short, what only a sequence's begin and end need is made there, and not kept over the tiles)
    const auto column = [&] {
        uint32_t here = n;
        if (!EIGHT && D * R <= 128) asm volatile("" : "+v"(here));
        return here;
    };
    const auto open = [&](const Place& p) {
        const uint32_t n = column();
        const uint32_t len = uniform((uint32_t)a.lens[p.s]), later = (uint32_t)a.n_q - 1;
        seen_by_all = min(len > later ? len - later : 0, p.len);
        const uint32_t h = p.u / a.own_tiles, rt = p.u - h * a.own_tiles;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            clear(r[j]);
            const uint32_t row = min((rt * R + j) * 16 + n, (uint32_t)a.rows - 1);  // (rows beyond the last are computed with it, and not stored)
            const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q;
            load_query<D>(r[j].q, a.q + p.s * a.q_strides[0] + i * a.q_strides[1] + (h * a.group + in) * a.q_strides[2], g);
            const uint32_t after = later - i;
            limit[j] = min(len > after ? len - after : 0, p.len);
#pragma unroll
            for (int k = 0; k < D / 32; ++k) asm volatile("" : "+v"(r[j].q[k]));  // (waited for here, not in every step)
        }
    };
    const auto close = [&](const Place& p, uint32_t first_tile) {
        const uint32_t n = column();
        const uint32_t h = p.u / a.own_tiles, rt = p.u - h * a.own_tiles;
        const bool whole = first_tile == 0 && p.t + 1 == p.tiles;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const float l = row_sum(r[j].l);
            const uint32_t row = (rt * R + j) * 16 + n;
            if (row >= (uint32_t)a.rows) continue;
            const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q, head = h * a.group + in;
            if (whole) {
                store_pieces<D, 0>(r[j], a.out + p.s * a.out_strides[0] + i * a.out_strides[1] + head * a.out_strides[2], l == 0.f ? 0.f : 1.f / l, g);
                if (a.lse && g == 0) a.lse[((int64_t)p.s * a.n_q + i) * a.n_heads + head] = lse_of(r[j].m - kLift, l);
            } else {
                const int64_t slot = a.own_slots + (int64_t)(2 * worker + (first_tile == 0 ? 1 : 0)) * (16 * R) + 16 * j + n;
                store_sums<D>(r[j], a.sums + slot * D, g);
                if (g == 0) a.stats[slot] = float2v{r[j].m - kLift, l};
            }
        }
    };

    // places[0]: the tile computed; the ones behind it are on their way, kAhead of them; the last, which is asked for in this step, has been looked up, and the tile behind it is looked up before, so that
    // waiting for block numbers is not waiting for tiles.  All loads are made in any case (behind the last tile, of zeros): the compiler then knows how many come after those that it waits for.
    constexpr uint32_t kAhead = EIGHT ? 2 : 1;  // (exponents that are not loaded eight at once take more registers)
    uint32_t left = end - begin, first_tile = c.t;
    const auto next = [&](const Place& p, uint32_t ahead) {
        Place n = p;
        if (left > ahead) advance(n);
        return n;
    };
    Finder<EIGHT> finder;
    const auto find = [&](const Place& p, bool first) { return finder.find(a, a.table + (int64_t)p.s * a.max_blocks, p.len, p.t, first); };
    bool bad = false;
    TileFp4<D, EIGHT> tiles[kAhead + 1];
    Place places[kAhead + 1];
    Spots<EIGHT> spots[kAhead + 1];
#pragma unroll
    for (uint32_t i = 0; i <= kAhead; ++i) {
        places[i] = i ? next(places[i - 1], i) : c;
        spots[i] = find(places[i], i == 0 || places[i].t == 0);
    }
    open(c);
#pragma unroll
    for (uint32_t i = 0; i < kAhead; ++i) tiles[i].load(x, source(places[i]), spots[i], places[i].t * kTile, left > i, bad);
    Spots<EIGHT> found = spots[kAhead];
    const auto step = [&](TileFp4<D, EIGHT>& now, TileFp4<D, EIGHT>& then) {  // -> whether it was the last one
        const Place behind = next(places[kAhead], kAhead + 1);
        const Spots<EIGHT> at = find(behind, behind.t == 0);
        __builtin_amdgcn_sched_barrier(0);
        then.load(x, source(places[kAhead]), found, places[kAhead].t * kTile, left > kAhead, bad);
        __builtin_amdgcn_sched_barrier(0);
        float4v s[R][2];
        make_scores<D, R, EIGHT>(s, r, now.k);
        add_tile_fp4<D, R, EIGHT>(r, x, now, s, places[0].t * kTile, seen_by_all, limit);
        if (left == 1 || places[1].t == 0) {
            close(places[0], first_tile);
            if (left == 1) return true;
            open(places[1]);
            first_tile = 0;
        }
#pragma unroll
        for (uint32_t i = 0; i < kAhead; ++i) places[i] = places[i + 1];
        places[kAhead] = behind;
        found = at;
        --left;
        return false;
    };
    if constexpr (kAhead == 2) {
        while (!step(tiles[0], tiles[2]) && !step(tiles[1], tiles[0]) && !step(tiles[2], tiles[1])) {
        }
    } else {
        while (!step(tiles[0], tiles[1]) && !step(tiles[1], tiles[0])) {
        }
    }
    if (bad) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
}

template <int D, int R, bool EIGHT>
__global__ __launch_bounds__(256, D * R <= 128 ? 2 : 1) void k_own_fp4(AttendFp4Args x) {
    __shared__ Sums sums;
    own_part_fp4<D, R, EIGHT>(x, sums, uniform(blockIdx.x * 4 + threadIdx.x / 64));
}

// ---- short sequences: a workgroup of kDirectWaves takes a unit, its waves the tiles in turn, and they join their sums in LDS: one launch.  Bound by the chain of reads of a wave's tiles and by the launch: one sequence of 256 tokens,
// 4 heads of 64, 5.3 us; 8 sequences of 1,024 to 2,048 tokens, 32 heads of 128, 15.2 us (54 MB).
template <int D, int R, bool EIGHT>
__global__ __launch_bounds__(64 * kDirectWaves, D * R <= 128 ? 2 : 1) void k_direct_fp4(AttendFp4Args x) {
    const AttendArgs& a = x.a;
    __shared__ float2v stats[kDirectWaves][16 * R];
    __shared__ __align__(16) float sums[kDirectWaves][16 * R][D];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x / 64);
    const uint32_t units = a.n_kv * a.own_tiles, s = blockIdx.x / units, u = blockIdx.x - s * units, h = u / a.own_tiles, rt = u - h * a.own_tiles;
    SourceFp4 src{a.table + (int64_t)s * a.max_blocks, (uint32_t)a.max_blocks * (uint32_t)a.g.N, x.k + (int64_t)h * x.f.page, x.v + (int64_t)h * x.f.page};
    Finder<EIGHT> finder;
    Spots<EIGHT> spots = {};
    if (a.max_blocks) spots = finder.find(a, src.table, src.len, wave, true);  // (as far as the table's row goes)
    Rows<D> r[R];
    uint32_t later[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        clear(r[j]);
        const uint32_t row = min((rt * R + j) * 16 + n, (uint32_t)a.rows - 1);
        const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q;
        load_query<D>(r[j].q, a.q + s * a.q_strides[0] + i * a.q_strides[1] + (h * a.group + in) * a.q_strides[2], g);
        later[j] = a.n_q - 1 - i;
    }
    const uint32_t len = uniform((uint32_t)max(a.lens[s], 0));
    src.len = uniform(own_length(a, s));
    const uint32_t tiles = (src.len + kTile - 1) / kTile;
    bool bad = false;
    if (wave < tiles) {
        uint32_t limit[R];
#pragma unroll
        for (int j = 0; j < R; ++j) limit[j] = min(len > later[j] ? len - later[j] : 0, src.len);
        const uint32_t later_most = (uint32_t)a.n_q - 1, seen_by_all = min(len > later_most ? len - later_most : 0, src.len);
        uint32_t t = wave;
        if constexpr (D * R <= pipelined_fp4(EIGHT)) {
            // the next tile is on its way while this one is computed, its place in the table looked up before
            TileFp4<D, EIGHT> here, next;
            here.load(x, src, spots, t * kTile, true, bad);
            spots = finder.find(a, src.table, src.len, t + kDirectWaves, true);
            const auto step = [&](TileFp4<D, EIGHT>& now, TileFp4<D, EIGHT>& then) {  // -> whether it was the last one
                const Spots<EIGHT> at = finder.find(a, src.table, src.len, t + 2 * kDirectWaves, true);
                __builtin_amdgcn_sched_barrier(0);
                then.load(x, src, spots, (t + kDirectWaves) * kTile, t + kDirectWaves < tiles, bad);
                __builtin_amdgcn_sched_barrier(0);
                float4v sc[R][2];
                make_scores<D, R, EIGHT>(sc, r, now.k);
                add_tile_fp4<D, R, EIGHT>(r, x, now, sc, t * kTile, seen_by_all, limit);
                spots = at;
                t += kDirectWaves;
                return t >= tiles;
            };
            while (!step(here, next) && !step(next, here)) {
            }
        } else {  // (there are no registers for two)
            for (;;) {
                TileFp4<D, EIGHT> tile;
                tile.load(x, src, spots, t * kTile, true, bad);
                float4v sc[R][2];
                make_scores<D, R, EIGHT>(sc, r, tile.k);
                add_tile_fp4<D, R, EIGHT>(r, x, tile, sc, t * kTile, seen_by_all, limit);
                t += kDirectWaves;
                if (t >= tiles) break;
                spots = finder.find(a, src.table, src.len, t, true);
            }
        }
    }
    if (bad) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
    const uint32_t workers = min(tiles, kDirectWaves);
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const float l = row_sum(r[j].l);
        if (wave < workers) {
            store_sums<D>(r[j], sums[wave][16 * j + n], g);
            if (g == 0) stats[wave][16 * j + n] = float2v{r[j].m - kLift, l};
        }
    }
    __syncthreads();
    for (uint32_t k = threadIdx.x; k < 16 * R * (D / 8); k += 64 * kDirectWaves) {
        const uint32_t in_tile = k / (D / 8), c = k % (D / 8), row = rt * R * 16 + in_tile;
        if (row >= (uint32_t)a.rows) continue;
        float m = -INFINITY, l = 0.f;
        for (uint32_t w = 0; w < workers; ++w) m = fmaxf(m, stats[w][in_tile][0]);
        float4v o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        for (uint32_t w = 0; w < workers; ++w) {
            const float2v st = stats[w][in_tile];
            const float f = join_weight(st[0], m);
            const float4v* v = reinterpret_cast<const float4v*>(&sums[w][in_tile][8 * c]);
            l += st[1] * f;
            o[0] += v[0] * f;
            o[1] += v[1] * f;
        }
        const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q, head = h * a.group + in;
        *reinterpret_cast<uint4v*>(a.out + s * a.out_strides[0] + i * a.out_strides[1] + head * a.out_strides[2] + 8 * c) = finished(o, l);
        if (a.lse && c == 0) a.lse[((int64_t)s * a.n_q + i) * a.n_heads + head] = lse_of(m, l);
    }
}

template <int D, int R>
static hipError_t launch_parts_fp4(const AttendFp4Args& x, hipStream_t s) {
    const bool eight = x.a.g.N % 8 == 0;
    if (x.a.direct) {  // (only where it fits: direct_fp4)
        const dim3 grid((unsigned)x.a.n_seq * x.a.n_kv * x.a.own_tiles), block(64 * kDirectWaves);
        if constexpr (direct_fits_fp4(D, R, true))
            if (eight) return launch_kernel(k_direct_fp4<D, R, true>, grid, block, s, x);
        if constexpr (direct_fits_fp4(D, R, false))
            if (!eight) return launch_kernel(k_direct_fp4<D, R, false>, grid, block, s, x);
        return hipErrorInvalidValue;
    }
    return launch_kernel(eight ? k_own_fp4<D, R, true> : k_own_fp4<D, R, false>, dim3((x.a.own_workers + 3) / 4), dim3(256), s, x);
}

template <>
hipError_t launch_attend_fp4<KVC_HEAD_DIM>(const AttendFp4Args& x, hipStream_t s) {
    constexpr int D = KVC_HEAD_DIM;
    hipError_t e;
    if constexpr (D <= 192) e = x.a.own_rows == 32 ? launch_parts_fp4<D, 2>(x, s) : launch_parts_fp4<D, 1>(x, s);
    else e = launch_parts_fp4<D, 1>(x, s);
    return e != hipSuccess || x.a.direct ? e : launch_join<D>(x.a, true, s);
}

}  // namespace kvc
