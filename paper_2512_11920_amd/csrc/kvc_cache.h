// Shared declarations of the decode-step operators: their entry points (kvc_cache_api.hip), the kernels that move
// blocks, tokens and payloads (kvc_cache.hip) and attention (kvc_attend.hip).
#pragma once
#include "kvc_common.h"

namespace kvc {

typedef uint32_t uint4v __attribute__((ext_vector_type(4)));  // (arrays of the runtime's uint4 end up in memory)

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
// rank, the number of set bits before it.  A tile is 64 words of the bitmap, 4,096 units, 64 KB of pool.
constexpr uint64_t kTileWords = 64, kTileUnits = kTileWords * 64;

struct CompactArgs {
    const uint8_t* pool;
    uint64_t units, out_units;  // 16-byte units of the two pools
    uint8_t* pool_out;
    const kvc_desc* desc;
    kvc_desc* desc_out;
    uint64_t n_desc, tiles;
    unsigned long long* bits;  // [tiles * kTileWords]
    uint16_t* before;          // [tiles * kTileWords]: set bits of the tile before the word
    unsigned long long* base;  // [tiles]: set bits of a tile, then of all tiles before it
    unsigned long long* used;  // out: bytes
    DevState* st;
};

inline uint64_t compact_tiles(uint64_t pool_bytes) { return (pool_bytes / 16 + kTileUnits - 1) / kTileUnits; }
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
    FastDiv by_N, by_rows;
    DevState* st;
};

hipError_t launch_append(const AppendArgs& a, hipStream_t s);
hipError_t launch_copy_blocks(const CopyArgs& a, hipStream_t s);
hipError_t launch_fork(const IdsArgs& a, hipStream_t s);
hipError_t launch_free(const IdsArgs& a, hipStream_t s);
hipError_t launch_compact(const CompactArgs& a, hipStream_t s);
hipError_t launch_adopt(DevState* st, const unsigned long long* used, hipStream_t s);

// attention, one source per head dimension
template <int D>
hipError_t launch_attend(const AttendArgs& a, hipStream_t s);

}  // namespace kvc
