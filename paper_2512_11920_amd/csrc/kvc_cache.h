// Shared declarations of the decode-step operators: their entry points (kvc_cache_api.hip), the kernels that move
// blocks, tokens and payloads (kvc_cache.hip) and attention (kvc_attend.hip).
#pragma once
#include <algorithm>

#include "kvc_common.h"

namespace kvc {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));  // (arrays of the runtime's uint4 end up in memory)

typedef float float2v __attribute__((ext_vector_type(2)));

struct AppendArgs {
    uint16_t* k_cache;
    uint16_t* v_cache;  // already at the first value page
    int64_t n_cache_blocks;
    const int32_t* table;
    const int32_t* lens;
    const uint16_t* k_new;
    const uint16_t* v_new;
    int64_t k_strides[3], v_strides[3];
    int32_t max_blocks, n_seq, n_new, n_kv;
    Geometry g;
    FastDiv by_N, by_n_new, by_lpr;
    DevState* st;
};

constexpr int kCopyChunks = 1024;  // that a workgroup copies

struct CopyArgs {
    uint16_t* cache;
    int64_t n_cache_blocks;
    const int32_t* src;
    const int32_t* dst;
    int32_t n, n_layers;
    int64_t per_layer;
    Geometry g;
    int32_t chunks;  // 16 bytes each, of a block
    int32_t pieces;  // kCopyChunks each, of a block
    bool dense;      // the block is one run of memory
    FastDiv by_lpr, by_N, by_pieces;
    DevState* st;
};

struct IdsArgs {  // fork and free
    kvc_desc* desc;
    const int32_t* src;
    const int32_t* dst;
    int64_t n_pages;  // n blocks * ppb, per layer
    int32_t ppb, n_layers;
    int64_t per_layer;
    FastDiv by_ppb;
    DevState* st;
};

// Compaction works on a bitmap of the pool's 16-byte units: a set bit is a unit that a live payload holds.  A unit's new place is its
// rank, the number of set bits before it.  A group is 1,024 words of the bitmap, 65,536 units, 1 MB of pool.
constexpr uint64_t kGroupWords = 1024;
constexpr uint32_t kSmallWords = 256, kSmallPages = 4096;  // a pool that one workgroup compacts: 256 KB

struct CompactArgs {
    const uint8_t* pool;
    uint64_t units, out_units;  // 16-byte units of the two pools
    uint8_t* pool_out;
    const kvc_desc* desc;
    kvc_desc* desc_out;
    uint64_t n_desc, groups;
    unsigned long long* bits;  // [groups * kGroupWords]
    uint16_t* before;          // [groups * kGroupWords]: set bits of the group before the word
    unsigned long long* base;  // [groups]: set bits of a group, then of all groups before it
    unsigned long long* used;  // out: bytes
    DevState* st;
};

inline uint64_t compact_groups(uint64_t pool_bytes) { return (pool_bytes / 16 + 64 * kGroupWords - 1) / (64 * kGroupWords); }
inline uint64_t round_256(uint64_t n) { return (n + 255) / 256 * 256; }

struct AttendArgs {
    const uint16_t* q;
    uint16_t* out;
    float* lse;
    int64_t q_strides[3], out_strides[3];
    const uint16_t* k_cache;
    const uint16_t* v_cache;  // already at the first value page
    int64_t n_cache_blocks;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* prefix_table;
    const int32_t* prefix_lens;
    const int32_t* prefix_first;
    int32_t max_blocks, max_prefix_blocks, n_prefix, n_seq, n_q, n_heads, n_kv, group;
    int32_t rows;   // query rows of one sequence and KV head: group * n_q
    float scale_log2;  // scale * log2(e)
    Geometry g;
    FastDiv by_N, by_rows, by_n_q;
    DevState* st;
    // the workspace, see AttendPlan
    uint32_t join_lanes;  // threads that share the pieces of a row's eight channels
    uint32_t own_tiles;  // row tiles of one sequence and KV head
    uint32_t own_workers, prefix_workers, own_rows, prefix_rows;
    bool direct;  // a workgroup for every unit, and nothing else
    bool apart;   // both parts in one launch, by workgroups of their own
    uint32_t* own_start;     // [n_seq + 1]
    uint32_t* prefix_start;  // [n_prefix + 2]: and how they are divided
    float* sums;             // [slots][d]
    float2v* stats;          // [slots]: reference and sum of the weights
    int64_t own_slots, prefix_whole, prefix_slots;   // first slots of what the own part shares, and of the prefix part's
};

// Workers of a call and what they need of the workspace.  Each worker may share a unit at either end of its part, so it has two slots for sums
// of so many rows; rows whose own and prefix parts each have one worker still have to be joined, so there is a slot for each row of either.
struct AttendPlan {
    uint32_t own_rows, prefix_rows;  // of a worker
    uint32_t own_workers, prefix_workers;
    uint64_t rows, slots, starts;    // query rows; slots; bytes of the sums of tiles
    uint64_t bytes;
};
// The sequences' own tokens: a wave on each SIMD.  (8 KB of keys and 8 KB of values on their way for each are enough; of 2,048 waves each has half as much, and as much to begin
// with: 64 sequences of 512 to 8,192 tokens, 8 x 128, 217 us with 2,048, 211 with 1,024; 8 of 1,024 to 2,048, 32 x 128, 37.3 and 36.8; 4 of 1,000 to
// 4,000 26.4 and 20.6.  Narrower heads have less in a tile, and more waves: 64 of 4,096 to 16,384, 8 x 32, 227 us with 1,024, 135 with 4,096; 1,024 to 16,384, 8 x 64, 226 and, with
// 2,048, 207.)  Prefixes: as many workgroups as the GPU holds at once, or half of them.
constexpr uint32_t kOwnWorkers = 1024, kPrefixWorkers = 256;
constexpr uint32_t kPrefixWaves = 4;                          // of a workgroup

// Up to so many tiles of prefixes (of 32 tokens, 128 rows and a KV head; as the tables are wide, which may be more than there are), half of the workgroups have the prefixes and
// half the sequences' own tokens; beyond it every one has a part of both, which divides better but begins twice.  8 KV heads x 128, 8 query heads each, both parts by all / apart, us; own tokens few (1 to
// 512) and many (512 to 2,048; for 128 sequences 512 to 4,096): prefix of 4,096 for 64 sequences (4,096 tiles) 51.4 / 39.4; 16,384 and 64 (16,384 tiles) 79 / 78; 8,192 and 256
// (32,768 tiles) 159 / 152 and 333 / 296; 32,768 and 64 (32,768 tiles, 41,000 as they are counted here) 119 / 121 and 156 / 144; 12,288 and 256 (49,152 tiles) 186 / 188 and 342 / 305; 32,768 and 128
// (65,536 tiles) 202 / 217 and 330 / 289; 16,384 and 256 (65,536 tiles) 226 / 235 and 359 / 319; 32,768 and 192 (98,304 tiles) 296 / 336; 24,576 and 256 with 1 to 2,048 (98,304 tiles) 399 / 394; 32,768 and
// 256 with 1 to 2,048 (131,072 tiles) 481 / 483.  So calls of many own tokens would rather be apart beyond it too, but these are counted on the device.
constexpr int64_t kApartTiles = 40960;
// A call without prefixes whose tables hold at most so many tiles of 32 tokens is done by a workgroup of 8 waves for each unit, in one launch: one sequence of
// 256 tokens, 4 heads x 64, 6.4 us instead of 9.7.  (Wider tables take the other way, however short the sequences are.)
constexpr uint32_t kDirectWaves = 8, kDirectTiles = 16;
constexpr bool direct_fits(int d, int row_tiles) { return d <= 224 && d * row_tiles <= 256; }  // into LDS and 256 registers

// Whether the kernel that does both parts keeps two workgroups of its own on a compute unit (256 registers).
constexpr bool both_fit(int d, int row_tiles) { return d * row_tiles <= 128; }

inline AttendPlan plan_attend(int64_t n_seq, int64_t n_q, int64_t n_heads, int64_t n_kv, int d, int64_t n_prefix) {
    AttendPlan p;
    // rows that share a tile's tokens, in steps of 16.  32 sequences of 1,000 to 8,000 tokens, 8 x 128, 32 rows: 130 us with 32, 187 with 16; one of 8,000 24 and 22.5.
    // (32 rows of heads beyond 192 do not fit into the registers.)
    p.own_rows = n_heads / n_kv * n_q <= 16 || d > 192 ? 16 : 32;
    p.prefix_rows = 32 * kPrefixWaves;
    p.own_workers = n_prefix ? (both_fit(d, (int)p.own_rows / 16) ? 2 : 1) * kOwnWorkers : std::max(1u, 128u / (d * p.own_rows / 16)) * kOwnWorkers;
    p.prefix_workers = n_prefix ? (d <= 128 ? 2 : 1) * kPrefixWorkers : 0;
    p.rows = (uint64_t)(n_seq * n_heads * n_q);
    p.slots = p.rows + 2ull * p.own_workers * p.own_rows + (n_prefix ? p.rows + 2ull * p.prefix_workers * p.prefix_rows : 0);
    p.starts = round_256((uint64_t)(n_seq + 1) * 4) + round_256((uint64_t)(n_prefix + 2) * 4);
    p.bytes = p.starts + round_256(p.slots * 8) + p.slots * (uint64_t)d * 4;
    return p;
}

hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_copy_blocks(const CopyArgs& a, hipStream_t s);
hipError_t launch_fork(const IdsArgs& a, hipStream_t s);
hipError_t launch_free(const IdsArgs& a, hipStream_t s);
hipError_t launch_compact(const CompactArgs& a, hipStream_t s);
hipError_t launch_adopt(DevState* st, const unsigned long long* used, hipStream_t s);

// attention, one source per head dimension
template <int D>
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);
// its second launch, which joins the pieces that the first left in the workspace
template <int D>
hipError_t launch_join(const AttendArgs& a, bool by_unit, hipStream_t s);

}  // namespace kvc
