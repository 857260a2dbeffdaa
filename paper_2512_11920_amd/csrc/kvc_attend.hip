// Attention over the paged cache, compiled once per head dimension (-DKVC_HEAD_DIM=d).
//
// Work is divided evenly, whatever the lengths are: what a call has to do is a list of units (a sequence, a KV head and some of
// its query rows; or a prefix, a KV head and some rows of its group), each of so many tiles of tokens, and worker w of W takes the tiles from w * T / W to
// (w + 1) * T / W of all T.  A unit that one worker has alone is finished there; the pieces of others are left as sums and joined
// by k_join.  Lengths are on the device, so each workgroup adds them up for itself.
#include "kvc_divide.h"

#ifndef KVC_HEAD_DIM
#error "KVC_HEAD_DIM: the head dimension to compile"
#endif

namespace kvc {

__device__ inline uint32_t prefix_length(const AttendArgs& a, int g) { return length_of(a, a.prefix_lens[g], a.max_prefix_blocks); }

// Sequences of prefix g.
struct Range {
    int begin, end;
};
__device__ inline Range group_of_prefix(const AttendArgs& a, int g) {
    Range r;
    r.begin = min(max(a.prefix_first[g], 0), a.n_seq);
    r.end = min(max(a.prefix_first[g + 1], r.begin), a.n_seq);
    return r;
}
// The prefix that sequence s has, or -1: the last one that begins at or before it, if the next one does not.
__device__ inline int prefix_of(const AttendArgs& a, int s) {
    int lo = 0, hi = a.n_prefix;  // first[lo..hi) may be at or before s
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (a.prefix_first[mid] <= s) lo = mid + 1;
        else hi = mid;
    }
    return lo > 0 && s < a.prefix_first[lo] ? lo - 1 : -1;
}

constexpr uint32_t kPieceCost = 7;

// ---- the sequences' own tokens: bound by memory, as a token's keys and values serve only the few rows of one head's group.  A worker is a wave: tiles of 32 tokens go from memory to its registers, keys of the next tile while this
// one's scores become weights, values while the next scores are made, so that a tile is always on its way; the block table is read one
// tile further ahead.  R: tiles of 16 rows that share the tokens.
// 64 sequences of 512 to 8,192 tokens, 8 x 128, 8 rows (1.14 GB): 207 us, 5.5 TB/s, a copy's rate; 8 of 1,024 to 2,048, 32 x 128, a row each (201 MB): 33 us, 6.0 TB/s.  Short calls are bound
// by reads of memory that wait for each other (lengths, table, keys, and the join's): one sequence of 8,192 tokens, 8 x 128, 16.5 us.
// The part of wave `worker`; called by all waves of a workgroup.
template <int D, int R, bool EIGHT>
__device__ inline void own_part(const AttendArgs& a, Sums& sums, uint32_t worker) {
    const auto tiles_of = [&](uint32_t s) { return (own_length(a, s) + kTile - 1) / kTile; };
    add_up(sums, a.n_seq, tiles_of);
    if (worker < 4) write_starts(sums, a.own_start, a.n_seq, tiles_of);
    const uint32_t units = a.n_kv * a.own_tiles, all = uniform(sums.all) * units, each = share(all, a.own_workers);
    const uint32_t begin = worker * each, end = min(begin + each, all);
    if (begin >= end) return;

    Place c;
    {
        const Item it = find_item(sums, a.n_seq, begin / units, tiles_of);
        c.s = uniform(it.i);
        c.len = uniform(own_length(a, c.s));
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
            p.len = uniform(own_length(a, p.s));
        } while (p.len == 0);
        p.tiles = (p.len + kTile - 1) / kTile;
    };
    const auto source = [&](const Place& p) {
        const uint32_t h = p.u / a.own_tiles;
        return Source{a.table + (int64_t)p.s * a.max_blocks, a.k_cache + h * a.g.page_stride, a.v_cache + h * a.g.page_stride, p.len};
    };

    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
    Rows<D> r[R];
    uint32_t limit[R];
    const auto open = [&](const Place& p) {
        const uint32_t h = p.u / a.own_tiles, rt = p.u - h * a.own_tiles;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            clear(r[j]);
            const uint32_t row = min((rt * R + j) * 16 + n, (uint32_t)a.rows - 1);  // (rows beyond the last are computed with it, and not stored)
            const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q;
            const uint16_t* q = a.q + p.s * a.q_strides[0] + i * a.q_strides[1] + (h * a.group + in) * a.q_strides[2];
#pragma unroll
            for (int k = 0; k < D / 32; ++k) r[j].q[k] = *reinterpret_cast<const uint4v*>(q + 32 * k + 8 * g);
            const uint32_t later = a.n_q - 1 - i, len = (uint32_t)a.lens[p.s];
            limit[j] = min(len > later ? len - later : 0, p.len);
        }
    };
    const auto close = [&](const Place& p, uint32_t first_tile) {
        const uint32_t h = p.u / a.own_tiles, rt = p.u - h * a.own_tiles;
        const bool whole = first_tile == 0 && p.t + 1 == p.tiles, alone = whole && prefix_of(a, p.s) < 0;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const float l = row_sum(r[j].l);
            const uint32_t row = (rt * R + j) * 16 + n;
            if (row >= (uint32_t)a.rows) continue;
            const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q, head = h * a.group + in;
            if (alone) {
                store_pieces<D, 0>(r[j], a.out + p.s * a.out_strides[0] + i * a.out_strides[1] + head * a.out_strides[2], l == 0.f ? 0.f : 1.f / l, g);
                if (a.lse && g == 0) a.lse[((int64_t)p.s * a.n_q + i) * a.n_heads + head] = lse_of(r[j].m - kLift, l);
            } else {
                const int64_t slot = whole ? ((int64_t)p.s * a.n_kv + h) * a.rows + row
                                           : a.own_slots + (int64_t)(2 * worker + (first_tile == 0 ? 1 : 0)) * (16 * R) + 16 * j + n;
                store_sums<D>(r[j], a.sums + slot * D, g);
                if (g == 0) a.stats[slot] = float2v{r[j].m - kLift, l};
            }
        }
    };

    // c: the tile computed; c1: the one loaded; c2: the one whose blocks are looked up
    Place c1 = c, c2 = c;
    uint32_t left = end - begin, first_tile = c.t;
    Tokens<D> x;
    Blocks<EIGHT> b = find_blocks<EIGHT>(a, source(c), c.t * kTile);
    open(c);
    load_keys<D, EIGHT>(x, a, source(c), b, c.t * kTile);
    uint32_t there = load_values<D, EIGHT>(x, a, source(c), b, c.t * kTile);
    if (left > 1) {
        advance(c1);
        b = find_blocks<EIGHT>(a, source(c1), c1.t * kTile);
        c2 = c1;
    }
    for (;;) {
        float4v s[R][2];
#pragma unroll
        for (int j = 0; j < R; ++j) scores(s[j], r[j], x);
        Blocks<EIGHT> ahead = b;
        if (left > 1) {
            load_keys<D, EIGHT>(x, a, source(c1), b, c1.t * kTile);
            if (left > 2) {
                advance(c2);
                ahead = find_blocks<EIGHT>(a, source(c2), c2.t * kTile);
            }
        }
        half8 p[R];
#pragma unroll
        for (int j = 0; j < R; ++j) p[j] = weights(r[j], s[j], a.scale_log2, there, c.t * kTile, limit[j]);
        add_tile<D, R>(r, x, p, c.t * kTile, c.len, a.n_q, limit);
        if (left > 1) there = load_values<D, EIGHT>(x, a, source(c1), b, c1.t * kTile);
        if (left == 1 || c1.t == 0) {
            close(c, first_tile);
            if (left == 1) break;
            open(c1);
            first_tile = 0;
        }
        c = c1;
        c1 = c2;
        b = ahead;
        --left;
    }
}

// ---- prefixes: many rows share the tokens, and the products count.  A worker is a workgroup: 32 rows of a group to a wave, and the waves share tiles of 32 tokens in LDS,
// which go there straight from memory, a quarter of each by every wave.  There is room for four: one is used, the next is there, two are on their way.  A step has one barrier: behind
// it the next tile's scores are made beside the present one's weights, then the present one's values are added.  32 rows a wave, as 64 leave room in the registers for one
// wave on a SIMD only (600 us instead of 418 where it was tried: with results in accumulation registers, from which each score was moved first, and weights that waited for their scores;
// the present step was not measured with 64), and two workgroups of 4 waves rather than one of 8, so that one computes while the other waits (418 and 448).
// 32,768 tokens, 16,384 rows, 128 channels (275 GFLOP): 336 to 343 us on two cards, 800 to 820 TFLOP/s, where a large product of matrices reaches 1,280.  (In calls that follow each other the clock
// falls for the first milliseconds: 334 to 430 us.)  A wave's step takes 1,360 cycles of its SIMD: 512 of products, and what
// of the rest does not fit beside them: reading LDS (512 for a workgroup), loads to LDS (317), 125 vector instructions, 17 of them powers.
constexpr uint32_t kStages = 4, kAhead = 8;
typedef float float16v __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
#define KVC_LDS(p) (__attribute__((address_space(3))) void*)(p)

// How keys and values of 32 tokens lie in LDS, in chunks of 16 bytes, C to a row.  Two kinds of read shall meet in no bank (16 chunks wide): one chunk
// of 16 consecutive tokens (keys), and four chunks of four consecutive tokens (values).  So the low bits of a chunk's number are turned by its
// token: as many tokens as begin in one bank differ in them, the nearest ones by fours.
template <int D>
struct Layout {
    static constexpr uint32_t C = D / 8, kMask = C % 16 == 0 ? 15 : C % 8 == 0 ? 7 : 3;
    __host__ __device__ static constexpr uint32_t turn(uint32_t t) { return C % 16 == 0 ? (t & 3) << 2 | (t >> 2 & 3) : C % 8 == 0 ? (t >> 1 & 1) << 2 | (t >> 2 & 3) : t >> 2 & 3; }
};

// A load from memory to LDS, BYTES for each lane: to `to`, the same in all lanes, + BYTES * lane.  (The compiler's own form of it makes reads of any tile wait for
// the loads of all of them.  The caller waits: wait_for_loads, then a barrier.  The sequence sets m0, of which the
// compiler cannot be told, as it reserves that register: nothing else in these kernels uses it, and a test of the generated code looks at that.)
template <int BYTES>
__device__ inline void load_to_lds(uint64_t from, void* to) {
    const uint32_t at = uniform((uint32_t)reinterpret_cast<uintptr_t>(KVC_LDS(to)));
    if constexpr (BYTES == 16) asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(from), "s"(at) : "memory");
    else asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" ::"v"(from), "s"(at) : "memory");
}

// Waits until at most N of the wave's loads are on their way.
template <uint32_t N>
__device__ inline void wait_for_loads() {
    __builtin_amdgcn_s_waitcnt((N & 15) | N >> 4 << 14 | 7 << 4 | 15 << 8);
}

template <uint32_t N>
struct Constant {
    static constexpr uint32_t value = N;
};

// What prefix_part has in LDS.
template <int D>
struct PrefixTiles {
    uint4v tile[kStages][2][32 * Layout<D>::C];   // [stage][keys, values]
    uint32_t ids[kPrefixWaves][kAhead][64];       // [wave][tile]: block of token n
    uint64_t rows[kPrefixWaves][32];              // [wave]: where the next tile's rows are
};

// The part of workgroup `worker`.
template <int D>
__device__ inline void prefix_part(const AttendArgs& a, Sums& sums, PrefixTiles<D>& lds, uint32_t worker) {
    using L = Layout<D>;
    auto& tile = lds.tile;
    auto& ids = lds.ids;
    auto& rows_at = lds.rows;
    constexpr uint32_t C = L::C, kLoads = C / kPrefixWaves, kRows = 32 * kPrefixWaves, kKeys = (L::kMask + 1) / 2, kValues = (L::kMask + 1) / 4;
    const auto row_tiles = [&](uint32_t g) {
        const Range r = group_of_prefix(a, g);
        return ((uint32_t)(r.end - r.begin) * a.rows + kRows - 1) / kRows;
    };
    const auto tiles_of = [&](uint32_t g) { return (prefix_length(a, g) + kTile - 1) / kTile; };
    Division div{1, 0};
    const auto work_of = [&](uint32_t g) { return row_tiles(g) * div.room(tiles_of(g)); };
    // groups out of order could hold a sequence twice, and more rows than there are: none is taken then
    bool disorder = false;
    for (uint32_t i = threadIdx.x; i < (uint32_t)a.n_prefix; i += 256) disorder = disorder || a.prefix_first[i] > a.prefix_first[i + 1];
    const bool ordered = !__syncthreads_or(disorder);
    if (disorder) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
    // A piece takes as long to begin and to end as kPieceCost tiles, so a worker rather has up to so many tiles more than two pieces.  Lanes 32c + g find out how many
    // workers it would take if each had c tiles more than an even share, but of one unit.  45 sequences in 5 groups, 6 x 96, N = 24, prefixes of a few hundred: 30 us, 33 by even shares;
    // 151 sequences in 6 groups, 8 x 160: 58 and 73; a prefix of 4,096 for 64 sequences, whose even shares are parts of one unit each, 38.2 and 37.6.
    if (a.n_prefix <= 32 && (uint32_t)(a.n_prefix * a.n_kv) <= a.prefix_workers) {
        const uint32_t g = threadIdx.x % 32, c = threadIdx.x / 32;
        const bool have = ordered && g < (uint32_t)a.n_prefix;
        const uint32_t rts = have ? row_tiles(g) : 0, tiles = have ? tiles_of(g) : 0;
        uint32_t total = rts * tiles;
        for (int k = 1; k < a.n_prefix; k *= 2) total += __shfl_xor(total, k);
        div.each = share(uniform(total) * a.n_kv, a.prefix_workers);
        uint32_t n = min(rts * ((tiles + div.each + c - 1) / (div.each + c)), a.prefix_workers + 1);
        for (int k = 1; k < a.n_prefix; k *= 2) n += __shfl_xor(n, k);
        if (g == 0) sums.workers[c] = n * a.n_kv;
        __syncthreads();
        uint32_t more = kPieceCost + 1;
#pragma unroll
        for (uint32_t k = kPieceCost + 1; k-- > 0;) more = uniform(sums.workers[k]) <= a.prefix_workers ? k : more;
        div.apart = more <= kPieceCost;
        div.each += div.apart ? more : 0;
        add_up(sums, ordered ? a.n_prefix : 0, work_of);
    } else {
        add_up(sums, ordered ? a.n_prefix : 0, work_of);
        div.each = share(uniform(sums.all) * a.n_kv, a.prefix_workers);
    }
    if (worker == 0) {
        write_starts(sums, a.prefix_start, a.n_prefix, work_of);
        if (threadIdx.x == 0) a.prefix_start[a.n_prefix + 1] = div.each << 1 | (div.apart ? 1 : 0);
    }
    if (threadIdx.x == 0) sums.division = div;  // (kept here: there are few registers)
    __syncthreads();
    const uint32_t all = uniform(sums.all) * a.n_kv, each = div.each;
    const uint32_t begin = worker * each;
    if (begin >= all) return;
    uint32_t left = min(each, all - begin);

    const uint32_t lane = threadIdx.x & 63, wave = uniform(threadIdx.x / 64), n = lane & 31, h2 = lane >> 5;
    // Waves 0 and 1 load keys, 2 and 3 values, half of a tile each: load j brings 64 chunks, of which this lane's is at byte `from` of the row of `token`.
    const uint32_t kind = wave / 2, half = wave & 1;
    // (Where 64 chunks are whole rows, and where a row's length is a power of two, a lane's numbers differ by constants only.)
    constexpr bool kRegular = 64 % C == 0, kSquare = C % 16 == 0;
    uint32_t token_of[kRegular ? 1 : kLoads], from_of[kRegular ? 1 : kLoads];
#pragma unroll
    for (uint32_t j = 0; j < (kRegular ? 1 : kLoads); ++j) {
        const uint32_t i = (half * kLoads + j) * 64 + lane;
        token_of[j] = i / C;
        from_of[j] = 16 * (i % C ^ L::turn(token_of[j]));
    }
    const auto token = [&](uint32_t j) { return kRegular ? token_of[0] + j * (64 / C) : token_of[j]; };
    const auto from = [&](uint32_t j) { return kRegular ? from_of[0] ^ 16 * L::turn(j * (64 / C)) : from_of[j]; };
    // What this lane reads of a tile of keys: row n, chunk 2c + h2; of values: a group of 16 lanes reads 16 channels of 4 tokens and gets
    // a channel's 4 tokens each, so rows 4 * h2 + l16 / 4 (+ 8, 16, 24), 8 bytes of chunk 4c + vc.
    const uint32_t l16 = lane & 15, vrow = 4 * h2 + l16 / 4, vc = (lane >> 4 & 1) * 2 + (l16 & 3) / 2;
    uint32_t keys_at[kSquare ? 1 : kKeys], values_at[2][kSquare ? 1 : kValues];
#pragma unroll
    for (uint32_t v = 0; v < (kSquare ? 1 : kKeys); ++v) keys_at[v] = 16 * (n * C + ((2 * v + h2) ^ L::turn(n)));
    const auto key_at = [&](uint32_t c) { return (kSquare ? keys_at[0] ^ 32 * (c % kKeys) : keys_at[c % kKeys]) + 32 * (c - c % kKeys); };
#pragma unroll
    for (uint32_t e = 0; e < 2; ++e)
#pragma unroll
        for (uint32_t v = 0; v < (kSquare ? 1 : kValues); ++v) values_at[e][v] = 16 * ((8 * e + vrow) * C + ((4 * v + vc) ^ L::turn(8 * e + vrow))) + 8 * (l16 & 1);

    const auto value_at = [&](uint32_t e, uint32_t v) { return kSquare ? values_at[e][0] ^ 64 * v : values_at[e][v]; };

    const float scale = fmaxf(fabsf(a.scale_log2), 1e-38f);  // (of zero too, so that times the -infinity of a token that does not exist it is no NaN)
    const uint32_t flip = a.scale_log2 < 0.f ? 0x80008000u : 0u;  // a negative scale is the queries' sign
    const uint32_t blocks = (uint32_t)min(a.n_cache_blocks, (int64_t)INT32_MAX);
    // From tile to tile a token's place moves on by 32 tokens: so many blocks and so many rows, and another block where that leaves the block.
    // (Strides are multiples of 8 elements, and counted in these.)
    const uint32_t row_stride = (uint32_t)(a.g.row_stride / 8), block_stride = (uint32_t)(a.g.block_stride / 8);
    const uint32_t step_blocks = fast_div(kTile, a.by_N), row_step = (kTile - step_blocks * (uint32_t)a.g.N) * row_stride, row_end = (uint32_t)a.g.N * row_stride;
    bool bad = false;
    uint32_t g, u, t, tiles, rts;
    {
        const Item it = find_item(sums, a.n_prefix, begin / a.n_kv, work_of);
        g = uniform(it.i);
        tiles = uniform(tiles_of(g));
        rts = uniform(row_tiles(g));
        const uint32_t rel = begin - uniform(it.start) * a.n_kv, room = uniform(div.room(tiles));
        u = rel / room;
        t = rel - u * room;
    }
    for (;;) {
        const uint32_t h = u / rts, rt = u - h * rts, first_tile = t, n_tiles = min(tiles - t, left);
        // tokens that the piece may see, from its first on
        const uint32_t len = min(uniform(prefix_length(a, g)) - t * kTile, n_tiles * kTile);
        const Range seqs = group_of_prefix(a, g);
        const uint32_t rows = (uint32_t)(seqs.end - seqs.begin) * a.rows;
        const int32_t* table = a.prefix_table + (int64_t)g * a.max_prefix_blocks;
        const uint16_t* pages = (kind ? a.v_cache : a.k_cache) + h * a.g.page_stride;
        const uint32_t in_tile = wave * 32 + n, rr = rt * kRows + in_tile;  // the lane's row, of the tile and of the group

        uint4v q[D / 16];
        float16v o[D / 32];
        float m = -INFINITY, l = 0.f;
        {
            const uint32_t r = min(rr, rows - 1), sq = fast_div(r, a.by_rows), row = r - sq * a.rows, in = fast_div(row, a.by_n_q), i = row - in * a.n_q;
            const uint16_t* p = a.q + (seqs.begin + sq) * a.q_strides[0] + i * a.q_strides[1] + (h * a.group + in) * a.q_strides[2];
#pragma unroll
            for (int c = 0; c < D / 16; ++c) q[c] = *reinterpret_cast<const uint4v*>(p + 16 * c + 8 * h2) ^ flip;
            if (a.scale_log2 == 0.f) {  // (zero times each product: zero queries where they are finite, NaN where they are not, as zero times infinity)
#pragma unroll
                for (int c = 0; c < D / 16; ++c)
#pragma unroll
                    for (int e = 0; e < 4; ++e) q[c][e] = (((q[c][e] & 0x7C007C00u) + 0x04000400u) >> 15 & 0x00010001u) * 0x7E00u;
            }
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[c][e] = 0.f;
        }
        // token n of a tile: its entry of the table, and its row's place in the block; both for tiles in order
        uint32_t entry = fast_div(t * kTile + n, a.by_N), row = (t * kTile + n - entry * (uint32_t)a.g.N) * row_stride, row_now = row;
        const auto next_row = [&](uint32_t& r) {
            r += row_step;
            const bool next = r >= row_end;
            r -= next ? row_end : 0;
            return next;
        };
        const auto look_up = [&](uint32_t i) {
            load_to_lds<4>(reinterpret_cast<uint64_t>(table) + 4ull * (i * kTile + n < len ? entry : 0), &ids[wave][i % kAhead][0]);
            entry += step_blocks + (next_row(row) ? 1 : 0);
        };
        // finds the rows of tile i (tiles in order), for `load`; -> which of its tokens exist
        const auto locate = [&](uint32_t i) {
            const uint32_t block = ids[wave][i % kAhead][lane];
            const bool seen = i * kTile + n < len, there = seen && block < blocks;
            bad = bad || (seen && (int32_t)block >= 0 && !there);
            const uint64_t at = ((uint64_t)block * block_stride + row_now) * 16 + reinterpret_cast<uint64_t>(pages);
            next_row(row_now);
            rows_at[wave][n] = there ? at : reinterpret_cast<uint64_t>(kZeroRow);
            return (uint32_t)__ballot(there);
        };
        // loads the tile that was located last (a wave's accesses to LDS are in order, so its lanes need not wait for each other)
        const auto load = [&](uint32_t stage) {
            uint64_t at[kLoads];
#pragma unroll
            for (uint32_t j = 0; j < kLoads; ++j) at[j] = rows_at[wave][token(j)];
#pragma unroll
            for (uint32_t j = 0; j < kLoads; ++j) load_to_lds<16>(at[j] + from(j), &tile[stage][kind][(half * kLoads + j) * 64]);
        };
        // scores of a tile, in powers of two but for `scale`
        const auto make_scores = [&](float16v& x, uint32_t stage) {
            const char* p = reinterpret_cast<const char*>(&tile[stage][0][0]);
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = 0.f;
#pragma unroll
            for (uint32_t c = 0; c < D / 16; ++c) {
                const uint4v k = *reinterpret_cast<const uint4v*>(p + key_at(c));
                x = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, k), __builtin_bit_cast(half8, q[c]), x, 0, 0, 0);
            }
        };
        const auto hide = [&](float16v& x, uint32_t there) {  // scores of tokens that do not exist
            const uint32_t here = there >> (4 * h2);
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] = here >> (8 * (e / 4) + e % 4) & 1 ? x[e] : -INFINITY;
        };
        const auto largest = [&](const float16v& x) {
            float top = fmaxf(x[0], x[1]);
#pragma unroll
            for (int e = 2; e < 16; ++e) top = fmaxf(top, x[e]);
            return both32(top, false) * scale;
        };
        const auto follow = [&](float top) {
            if (!__any(top > m + kLag)) return;
            const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : power2(m - to);
            m = to;
            l *= f;
#pragma unroll
            for (int c = 0; c < D / 32; ++c) o[c] *= f;
        };

        // Tiles 0..2 on their way, the rows of tile 3 located, and the blocks of tiles 4 and 5 asked for; mask[k]: the tokens of tile i + 1 + k that exist.  What comes back
        // comes in order: the next tile and the blocks of the one to be located next are there when only what the last step asked for is missing.
        uint32_t mask[3];
#pragma unroll
        for (uint32_t i = 0; i < 5; ++i) look_up(i);
        wait_for_loads<0>();
        __syncthreads();  // (and the tiles of the last piece have been read)
        float16v s;
        {
            const uint32_t there = locate(0);
            load(0);
            mask[0] = locate(1);
            load(1);
            mask[1] = locate(2);
            load(2);
            mask[2] = locate(3);
            look_up(5);
            wait_for_loads<2 * kLoads + 1>();
            __syncthreads();
            make_scores(s, 0);
            if (there != ~0u) hide(s, there);
            follow(largest(s));
        }
        const auto step = [&](auto stage_, uint32_t i) {
            constexpr uint32_t stage = decltype(stage_)::value;
            // tile i + 1 is there, and every wave is done with tile i - 1, whose place tile i + 3 takes
            wait_for_loads<kLoads + 1>();
            __syncthreads();
            load((stage + 3) % kStages);  // (first of all: a prefix of 32,768 tokens and 256 sequences, 8 x 128, 482 us, 488 in the midst of the products, 495 behind them)
            // the next tile's scores, while this one's become weights
            float16v next;
            make_scores(next, (stage + 1) % kStages);  // (behind the last tile, of what lies there; it is not used)
            half8 v[2][D / 32];
            const auto read_values = [&](uint32_t j) {
                const char* values = reinterpret_cast<const char*>(&tile[stage][1][0]);
#pragma unroll
                for (uint32_t c = 0; c < D / 32; ++c) {
                    short4v part[2];
#pragma unroll
                    for (uint32_t e = 0; e < 2; ++e)
                        part[e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                            (__attribute__((address_space(3))) short4v*)KVC_LDS(values + value_at(e, c % kValues) + 16 * (16 * j * C) + 64 * (c - c % kValues)));
                    v[j][c] = __builtin_bit_cast(half8, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
                }
            };
            read_values(0);
            half8 p[2];
            const float low = kLift - (m == -INFINITY ? 0.f : m);
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const float w = power2(fmaf(s[e], scale, low));
                l += w;
                p[e / 8][e % 8] = (_Float16)w;
            }
            asm volatile("" : "+v"(p[0]), "+v"(p[1]), "+v"(l));  // (here, not behind the branches below, where the compiler would put them)
            // products with reads a few ahead of them and vector instructions between them (reads further ahead would not leave 256 registers enough)
            constexpr int kProduct = 0x8, kRead = 0x100, kTrans = 0x400, kVector = 0x2;
            __builtin_amdgcn_sched_group_barrier(kRead, 3, 0);
#pragma unroll
            for (uint32_t c = 0; c < D / 16; ++c) {
                __builtin_amdgcn_sched_group_barrier(kProduct, 1, 0);
                __builtin_amdgcn_sched_group_barrier(kRead, 2, 0);
                __builtin_amdgcn_sched_group_barrier(kTrans, 256 / D, 0);
                __builtin_amdgcn_sched_group_barrier(kVector, 640 / D, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            if (mask[0] != ~0u) hide(next, mask[0]);
            mask[0] = mask[1];
            mask[1] = mask[2];
            read_values(1);
#pragma unroll
            for (uint32_t j = 0; j < 2; ++j)
#pragma unroll
                for (uint32_t c = 0; c < D / 32; ++c) o[c] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[j][c], p[j], o[c], 0, 0, 0);
            const float top = largest(next);
            mask[2] = locate(i + 4);
            look_up(i + 6);
            if (i + 1 < n_tiles) follow(top);
            s = next;
        };
        for (uint32_t i = 0; i < n_tiles; i += 4) {
            step(Constant<0>(), i);
            if (i + 1 < n_tiles) step(Constant<1>(), i + 1);
            if (i + 2 < n_tiles) step(Constant<2>(), i + 2);
            if (i + 3 < n_tiles) step(Constant<3>(), i + 3);
        }
        wait_for_loads<0>();  // (nothing may be on its way to this LDS when another workgroup has it)
        const bool whole = first_tile == 0 && n_tiles == tiles;
        const float sum = both32(l, true);
        if (rr < rows) {
            const uint32_t sq = fast_div(rr, a.by_rows);
            const int64_t slot = whole ? a.prefix_whole + ((int64_t)(seqs.begin + sq) * a.n_kv + h) * a.rows + (rr - sq * a.rows)
                                       : a.prefix_slots + (int64_t)(2 * worker + (first_tile == 0 ? 1 : 0)) * kRows + in_tile;
            float* out = a.sums + slot * D + 4 * h2;
#pragma unroll
            for (int c = 0; c < D / 32; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    *reinterpret_cast<float4v*>(out + 32 * c + 8 * e) = float4v{o[c][4 * e], o[c][4 * e + 1], o[c][4 * e + 2], o[c][4 * e + 3]};
            if (h2 == 0) a.stats[slot] = float2v{m - kLift, sum};
        }
        left -= min(left, uniform(sums.division.room(tiles)) - first_tile);
        if (left == 0) break;
        t = 0;
        if (++u == rts * a.n_kv) {
            u = 0;
            do ++g;
            while (uniform(row_tiles(g) * tiles_of(g)) == 0);
            tiles = uniform(tiles_of(g));
            rts = uniform(row_tiles(g));
        }
    }
    if (bad) atomicOr(&a.st->status, KVC_ST_BAD_INDEX);
}

template <int D, int R, bool EIGHT>
__global__ __launch_bounds__(256, D * R <= 128 ? 2 : 1) void k_own(AttendArgs a) {
    __shared__ Sums sums;
    own_part<D, R, EIGHT>(a, sums, uniform(blockIdx.x * 4 + threadIdx.x / 64));
}

// Workgroups go to the XCDs in turn: an XCD's take neighbouring parts of a prefix's work, which read the same tokens.
__device__ inline uint32_t neighbour(uint32_t i, uint32_t n) { return i % 8 * (n / 8) + i / 8; }

template <int D>
__global__ __launch_bounds__(64 * kPrefixWaves, D <= 128 ? 2 : 1) void k_prefix(AttendArgs a) {
    __shared__ Sums sums;
    __shared__ PrefixTiles<D> lds;
    prefix_part<D>(a, sums, lds, neighbour(blockIdx.x, a.prefix_workers));
}

// Both in one launch, two workgroups on each compute unit: the first half of them begins with prefixes, which keep the matrix units busy, the other with
// the sequences' own tokens, which keep the memory busy; then they change: a prefix of 32,768 tokens and 256 sequences of 1 to 2,048, 8 x 128, 8 rows, 465 to 474 us (calls in a row 460 to 635), and 336 to 343 + 205 by themselves.  Where there is little to do for prefixes (a.apart) each half does its own alone.
template <int D, int R, bool EIGHT>
__global__ __launch_bounds__(256, 2) void k_both(AttendArgs a) {
    __shared__ Sums sums;
    __shared__ PrefixTiles<D> lds;
    const uint32_t half = gridDim.x / 2, i = blockIdx.x;
#pragma nounroll
    for (uint32_t turn = 0; turn < 2; ++turn) {
        if (turn == (i < half ? 0 : 1)) {
            if (!a.apart || i < half) prefix_part<D>(a, sums, lds, i < half ? neighbour(i, half) : half + neighbour(i - half, half));
        } else if (!a.apart || i >= half) {
            own_part<D, R, EIGHT>(a, sums, uniform((a.apart ? i - half : i) * 4 + threadIdx.x / 64));
        }
        __syncthreads();  // (the sums are used again)
    }
}

// ---- short sequences without a prefix.  A workgroup of kDirectWaves takes a unit, its waves the tiles in turn, and they join their sums in LDS: one launch, and the
// lengths, the block table and the queries are asked for at once.  Bound by two reads that follow from each other and the launch: 256 tokens, 4 heads x 64, 6 us.
template <int D, int R, bool EIGHT>
__global__ __launch_bounds__(64 * kDirectWaves, D * R <= 128 ? 2 : 1) void k_direct(AttendArgs a) {
    __shared__ float2v stats[kDirectWaves][16 * R];
    __shared__ __align__(16) float sums[kDirectWaves][16 * R][D];
    const uint32_t lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4, wave = uniform(threadIdx.x / 64);
    const uint32_t units = a.n_kv * a.own_tiles, s = blockIdx.x / units, u = blockIdx.x - s * units, h = u / a.own_tiles, rt = u - h * a.own_tiles;
    Source src{a.table + (int64_t)s * a.max_blocks, a.k_cache + h * a.g.page_stride, a.v_cache + h * a.g.page_stride, (uint32_t)a.max_blocks * (uint32_t)a.g.N};
    Blocks<EIGHT> b = find_blocks<EIGHT>(a, src, wave * kTile);  // (as far as the table's row goes)
    Rows<D> r[R];
    uint32_t later[R];
#pragma unroll
    for (int j = 0; j < R; ++j) {
        clear(r[j]);
        const uint32_t row = min((rt * R + j) * 16 + n, (uint32_t)a.rows - 1);
        const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q;
        const uint16_t* q = a.q + s * a.q_strides[0] + i * a.q_strides[1] + (h * a.group + in) * a.q_strides[2];
#pragma unroll
        for (int k = 0; k < D / 32; ++k) r[j].q[k] = *reinterpret_cast<const uint4v*>(q + 32 * k + 8 * g);
        later[j] = a.n_q - 1 - i;
    }
    const uint32_t len = uniform((uint32_t)max(a.lens[s], 0));
    src.len = uniform(own_length(a, s));
    const uint32_t tiles = (src.len + kTile - 1) / kTile;
    for (uint32_t t = wave; t < tiles; t += kDirectWaves) {
        if (t != wave) b = find_blocks<EIGHT>(a, src, t * kTile);
        b.end_at(t * kTile, src.len);  // (entries behind the last token are not block numbers)
        Tokens<D> x;
        load_keys<D, EIGHT>(x, a, src, b, t * kTile);
        const uint32_t there = load_values<D, EIGHT>(x, a, src, b, t * kTile);
        half8 p[R];
        uint32_t limit[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            float4v sc[2];
            scores(sc, r[j], x);
            limit[j] = min(len > later[j] ? len - later[j] : 0, src.len);
            p[j] = weights(r[j], sc, a.scale_log2, there, t * kTile, limit[j]);
        }
        add_tile<D, R>(r, x, p, t * kTile, src.len, a.n_q, limit);
    }
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
            const float4v* x = reinterpret_cast<const float4v*>(&sums[w][in_tile][8 * c]);
            l += st[1] * f;
            o[0] += x[0] * f;
            o[1] += x[1] * f;
        }
        const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q, head = h * a.group + in;
        *reinterpret_cast<uint4v*>(a.out + s * a.out_strides[0] + i * a.out_strides[1] + head * a.out_strides[2] + 8 * c) = finished(o, l);
        if (a.lse && c == 0) a.lse[((int64_t)s * a.n_q + i) * a.n_heads + head] = lse_of(m, l);
    }
}

// ---- joining pieces: D / 8 threads for 8 channels each, of a row and every a.join_lanes-th of its pieces.  A thread reads kAtOnce pieces at a time, as each read goes to memory
// and takes as long as all of them together; where there are few rows, whose pieces are many, threads share them out and join their sums in LDS.  4,096 rows of about 10 pieces of 128 channels (21 MB):
// 7.9 us; one or two pieces: 5 us, the time of the four reads that follow from each other.
constexpr uint32_t kAtOnce = 8;

// Where the pieces of a unit are, for one of its rows: `n` workers from w0 on have one each, or one has it whole.
struct Pieces {
    int64_t whole, slots;
    uint32_t n = 0, w0 = 0, rows = 0, stride = 1;  // stride: from a piece's worker to the next one's

    __device__ void find(uint32_t start, uint32_t tiles, uint32_t each) {
        w0 = start / each;
        n = (start + tiles - 1) / each - w0 + 1;
    }
    __device__ int64_t slot(uint32_t k) const { return n == 1 ? whole : slots + (int64_t)(2 * (w0 + k) * stride + (k == 0 ? 1 : 0)) * rows; }
};

// BY_UNIT: workers are dealt ranges of the sequences' tiles, the units of each range in turn (kvc_attend_fp4.hip); else ranges of the tiles of all units.
template <int D, bool BY_UNIT>
__global__ __launch_bounds__(256) void k_join(AttendArgs a) {
    constexpr uint32_t kEach = D / 8, kSlots = 256 / kEach;
    __shared__ __align__(16) float4v sums[kSlots][kEach][2];
    __shared__ float2v stats[kSlots];
    const uint32_t place = threadIdx.x / kEach, c = threadIdx.x % kEach, lanes = a.join_lanes, in_group = place / lanes, first = place % lanes;
    const uint32_t rows_here = kSlots / lanes;
    const int64_t id = (int64_t)blockIdx.x * rows_here + in_group;
    const bool have = in_group < rows_here && id < (int64_t)a.n_seq * a.n_kv * a.rows;
    const uint32_t row_id = have ? (uint32_t)id : 0, unit = fast_div(row_id, a.by_rows), row = row_id - unit * a.rows, s = unit / a.n_kv, h = unit - s * a.n_kv;
    Pieces own, shared;
    const uint32_t before = a.own_start[s], tiles = a.own_start[s + 1] - before, all = a.own_start[a.n_seq];
    const int g = a.n_prefix ? prefix_of(a, s) : -1;
    if (tiles) {
        const uint32_t units = a.n_kv * a.own_tiles, rt = row / a.own_rows, u = h * a.own_tiles + rt;
        if (BY_UNIT) own.find(before, tiles, share(all, a.own_workers / units));
        else own.find(before * units + u * tiles, tiles, share(all * units, a.own_workers));
        own.whole = row_id;
        own.rows = a.own_rows;
        own.slots = a.own_slots + (row - rt * a.own_rows) + (BY_UNIT ? (int64_t)2 * u * a.own_rows : 0);
        if (BY_UNIT) own.stride = units;
    }
    const bool finished_already = g < 0 && own.n == 1;  // by its worker
    if (g >= 0) {
        const Range seqs = group_of_prefix(a, g);
        const uint32_t ptiles = (prefix_length(a, g) + kTile - 1) / kTile;
        if (ptiles && a.prefix_start[a.n_prefix]) {
            const uint32_t rts = ((uint32_t)(seqs.end - seqs.begin) * a.rows + a.prefix_rows - 1) / a.prefix_rows;
            const uint32_t rr = (s - seqs.begin) * a.rows + row, rt = rr / a.prefix_rows;
            const uint32_t code = a.prefix_start[a.n_prefix + 1];
            const Division div{code >> 1, code & 1};
            shared.find(a.prefix_start[g] * a.n_kv + (h * rts + rt) * div.room(ptiles), ptiles, div.each);
            shared.whole = a.prefix_whole + row_id;
            shared.rows = a.prefix_rows;
            shared.slots = a.prefix_slots + (rr - rt * a.prefix_rows);
        }
    }
    float m = -INFINITY, l = 0.f;
    float4v o[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    const auto join = [&](float2v st, const float4v& x, const float4v& y, float top) {
        const float w = join_weight(st[0], top);
        l += st[1] * w;
        o[0] += x * w;
        o[1] += y * w;
    };
    const uint32_t n = have && !finished_already ? own.n + shared.n : 0;
    for (uint32_t k0 = first; k0 < n; k0 += kAtOnce * lanes) {
        float2v st[kAtOnce];
        float4v x[kAtOnce][2];
        float top = m;
#pragma unroll
        for (uint32_t j = 0; j < kAtOnce; ++j) {
            const uint32_t k = k0 + j * lanes;
            st[j] = float2v{-INFINITY, 0.f};
            x[j][0] = x[j][1] = float4v{0.f, 0.f, 0.f, 0.f};
            if (k < n) {
                const int64_t slot = k < own.n ? own.slot(k) : shared.slot(k - own.n);
                st[j] = a.stats[slot];
                const float4v* p = reinterpret_cast<const float4v*>(a.sums + slot * D + 8 * c);
                x[j][0] = p[0];
                x[j][1] = p[1];
            }
        }
#pragma unroll
        for (uint32_t j = 0; j < kAtOnce; ++j) top = fmaxf(top, st[j][0]);
        const float f = join_weight(m, top);
        m = top;
        l *= f;
        o[0] *= f;
        o[1] *= f;
#pragma unroll
        for (uint32_t j = 0; j < kAtOnce; ++j) join(st[j], x[j][0], x[j][1], top);
    }
    if (lanes > 1) {
        if (place < kSlots) {
            sums[place][c][0] = o[0];
            sums[place][c][1] = o[1];
            if (c == 0) stats[place] = float2v{m, l};
        }
        __syncthreads();
        if (first == 0 && have) {
            float top = m;
            for (uint32_t j = 1; j < lanes; ++j) top = fmaxf(top, stats[place + j][0]);
            const float f = join_weight(m, top);
            m = top;
            l *= f;
            o[0] *= f;
            o[1] *= f;
            for (uint32_t j = 1; j < lanes; ++j) join(stats[place + j], sums[place + j][c][0], sums[place + j][c][1], top);
        }
    }
    if (!have || first != 0 || finished_already) return;
    const uint32_t in = fast_div(row, a.by_n_q), i = row - in * a.n_q, head = h * a.group + in;
    *reinterpret_cast<uint4v*>(a.out + s * a.out_strides[0] + i * a.out_strides[1] + head * a.out_strides[2] + 8 * c) = finished(o, l);
    if (a.lse && c == 0) a.lse[((int64_t)s * a.n_q + i) * a.n_heads + head] = lse_of(m, l);
}

template <int D, int R>
static hipError_t launch_parts(const AttendArgs& a, hipStream_t s) {
    // 32 sequences of 1,000 to 8,000 tokens, N = 16, 8 x 128, 32 rows: 130 us with blocks found by eights, 139 without; 64 of 512 to 8,192, 8 rows, 210 either way
    const bool eight = a.g.N % 8 == 0;
    if constexpr (direct_fits(D, R))
        if (a.direct) return launch_kernel(eight ? k_direct<D, R, true> : k_direct<D, R, false>, dim3((unsigned)a.n_seq * a.n_kv * a.own_tiles), dim3(64 * kDirectWaves), s, a);
    if constexpr (both_fit(D, R))
        if (a.n_prefix) return launch_kernel(eight ? k_both<D, R, true> : k_both<D, R, false>, dim3(2 * kPrefixWorkers), dim3(256), s, a);
    const hipError_t e = launch_kernel(eight ? k_own<D, R, true> : k_own<D, R, false>, dim3(a.own_workers / 4), dim3(256), s, a);
    return e == hipSuccess && a.n_prefix ? launch_kernel(k_prefix<D>, dim3(a.prefix_workers), dim3(64 * kPrefixWaves), s, a) : e;
}

template <>
hipError_t launch_join<KVC_HEAD_DIM>(const AttendArgs& a, bool by_unit, hipStream_t s) {
    const uint32_t rows = 256 / (KVC_HEAD_DIM / 8) / a.join_lanes;
    return launch_kernel(by_unit ? k_join<KVC_HEAD_DIM, true> : k_join<KVC_HEAD_DIM, false>, dim3((unsigned)(((int64_t)a.n_seq * a.n_kv * a.rows + rows - 1) / rows)), dim3(256), s, a);
}

template <>
hipError_t launch_attend<KVC_HEAD_DIM>(const AttendArgs& a, hipStream_t s) {
    constexpr int D = KVC_HEAD_DIM;
    hipError_t e;
    if constexpr (D <= 192) e = a.own_rows == 32 ? launch_parts<D, 2>(a, s) : launch_parts<D, 1>(a, s);
    else e = launch_parts<D, 1>(a, s);
    return e != hipSuccess || a.direct ? e : launch_join<D>(a, false, s);
}

}  // namespace kvc
