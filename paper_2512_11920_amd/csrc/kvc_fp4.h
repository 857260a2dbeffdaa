// Shared declarations of the operators that keep the paged cache small: a cache held in 4 bits (kvc_fp4.hip, kvc_attend_fp4.hip), the attention weight that
// tokens get (kvc_weigh.hip), eviction (kvc_evict.hip), and their entry points (kvc_fp4_api.hip).
#pragma once
#include "kvc_cache.h"

namespace kvc {

// A page in 4 bits: N rows of d/2 bytes of codes, then for every 32 channels the N tokens' exponent bytes, then what makes it a multiple of 16 bytes.  The
// exponents of 8 tokens are 8 bytes in a row, as one lane needs them of a group of channels.
struct Fp4Pages {
    uint32_t page, exps;  // bytes of a page; where its exponents begin
    int64_t block;        // bytes of a block
};
inline Fp4Pages fp4_pages(int N, int d, int64_t ppb) {
    Fp4Pages f;
    f.exps = (uint32_t)(N * d / 2);
    f.page = (uint32_t)((N * 17 * d / 32 + 15) / 16 * 16);
    f.block = ppb * f.page;
    return f;
}

constexpr uint32_t kTurn = 4;

struct AppendFp4Args {
    uint8_t* k_cache;
    uint8_t* v_cache;  // already at the first value page
    Fp4Pages f;
    AppendArgs a;      // (its caches are not looked at)
    bool wide;         // kTurn new tokens to a workgroup, else one
    uint32_t turns;    // workgroups of a sequence
    FastDiv by_turns;
};

struct UnpackFp4Args {
    const uint8_t* cache;
    uint16_t* out;
    int64_t n_cache_blocks, n_out_blocks;
    const int32_t* src;  // NULL: block i
    const int32_t* dst;
    Fp4Pages f;
    Geometry g;
    int32_t n, chunks, pieces;  // as in CopyArgs
    FastDiv by_lpr, by_N, by_pieces;
    DevState* st;
};

struct AttendFp4Args {
    AttendArgs a;  // (its caches are not looked at)
    const uint8_t* k;
    const uint8_t* v;  // already at the first value page
    Fp4Pages f;
};

struct WeighArgs {
    AttendArgs a;           // out, v_cache and the workspace are not looked at; lse is read
    const uint8_t* k;       // a cache in 4 bits, or NULL
    Fp4Pages f;
    const float* before;    // [n_seq][n_kv][width]
    float* after;
    int32_t* positions;     // [n_seq][n_kv][width]
    const int32_t* seen;    // [n_seq]
    int32_t width;
    bool many;              // queries
    uint32_t workers;       // waves, or workgroups of many queries
};

struct EvictArgs {
    uint8_t* k;
    uint8_t* v;  // already at the first value page
    bool fp4;
    Fp4Pages f;
    Geometry g;
    int64_t n_cache_blocks;
    const int32_t* table;
    const int32_t* lens;
    const int32_t* keep;
    const float* weights;
    float* weights_out;
    const int32_t* positions;
    int32_t* positions_out;
    const int32_t* seen;
    int32_t* new_lens;
    int32_t recent, width, max_blocks, n_seq, n_kv;
    int32_t most;  // moves of a sequence and head, at most
    FastDiv by_N, by_n_kv, by_lanes;  // (lanes that move a row)
    DevState* st;
    // the workspace
    int32_t* counts;   // [n_seq * n_kv]: moves
    int32_t* left;     // [n_seq]: tokens that stay
    int32_t* holes;    // [n_seq * n_kv][most]
    int32_t* fillers;  // [n_seq * n_kv][most]
};

// Workers of attention over a cache in 4 bits: a tile is a quarter of FP16's bytes, so more waves are needed for as many bytes on their way, and they fit.  A whole number of them for each
// unit (a KV head and its row tiles), which takes one range of the sequences' tiles; one at least.
inline AttendPlan plan_attend_fp4(int64_t n_seq, int64_t n_q, int64_t n_heads, int64_t n_kv, int d) {
    AttendPlan p = plan_attend(n_seq, n_q, n_heads, n_kv, d, 0);
    // (waves on a SIMD, as registers are enough for: 64 sequences of 4,096 to 16,384 tokens, 8 x 32, 88.0 us with two, 80.2 with three; 8 x 64 100.7 and 110.8)
    const int64_t workers = (d * p.own_rows / 16 <= 32 ? 3 : d * p.own_rows / 16 <= 128 ? 2 : 1) * kOwnWorkers, units = n_kv * ((n_heads / n_kv * n_q + p.own_rows - 1) / p.own_rows), ranges = std::max<int64_t>(1, workers / units);
    p.own_workers = (uint32_t)(ranges * units);
    p.slots = p.rows + (ranges > 1 ? 2ull * p.own_workers * p.own_rows : 0);  // (of one range nothing is shared)
    p.bytes = p.starts + round_256(p.slots * 8) + p.slots * (uint64_t)d * 4;
    return p;
}
// Into LDS and 256 registers (eight: pages of a multiple of 8 tokens, whose exponents are read eight at once); and channels times row tiles with which a workgroup's next tile fits too.
constexpr bool direct_fits_fp4(int d, int row_tiles, bool eight) { return direct_fits(d, row_tiles) && (eight || d * row_tiles <= 160); }
constexpr int pipelined_fp4(bool eight) { return eight ? 128 : 64; }
// Whether a call is done by a workgroup for every unit, in one launch, by the units and by the tokens that a row of the table has room for.  Its waves are as busy as the sequence is long, where divided work is even,
// but takes a second launch and a chain of reads to be divided.  8 KV heads x 128, 8 query heads each, sequences of one length, us, divided / so: 8 units of 1,024 tokens 12.1 / 9.8, of 2,048 12.8 / 14.3, of 4,096 13.7 /
// 23.3; 32 units 13.6 / 9.8, 16.0 / 14.6, 17.5 / 23.6; 128 units 17.0 / 10.6, 20.0 / 15.1, 25.4 / 24.2, of 8,192 41.2 / 43.1; 256 units 19.6 / 11.4, 25.0 / 16.5, 40.7 / 30.8, 65.2 / 55.9; 512 units 24.9 / 20.9, 41.2 / 34.8;
// 1,024 units of 128 16.2 / 18.6, of 448 23.4 / 27.7; 2,048 units 17.6 / 34.8, 34.7 / 56.3.  Sequences of a sixteenth of that length and more: 256 units of up to 8,192 tokens 46.0 / 43.8, 512 units of up to 2,048 28.5 / 26.4,
// of up to 8,192 75.1 / 76.5 (heads of 96 70.5 / 82.1).  32 rows of 128 channels, or 8 of 192, for which there are no registers for a tile on its way: 128 units of 448 19.2 / 11.9, 14.9 / 9.1; 512 units 28.0 / 22.6, 21.0 / 17.6; 1,024
// units 31.3 / 44.4, 28.5 / 34.2.  Lengths are on the device, and the rule goes by the table alone: where one sequence is long among short ones its workgroup is what the call waits for.  32 sequences, 256 units: one of 8,192 tokens
// and 31 of 256 19.8 / 40.2, one of 4,096 16.3 / 23.2 (a table one block wider than 8,192 tokens has them divided); 64 sequences, 512 units, one of 2,048 and 63 of 128 15.6 / 14.4.
inline bool direct_fp4(int d, bool eight, int row_tiles, int64_t units, int64_t tokens) {
    if (!direct_fits_fp4(d, row_tiles, eight) || units > 512) return false;
    if (tokens <= (int64_t)kDirectTiles * 32) return true;
    return d * row_tiles <= pipelined_fp4(eight) && (tokens <= 1024 || (tokens <= 2048 && units >= 32) || (tokens <= 8192 && units > 128 && units <= 256));
}
// Waves that weigh a few queries' tokens.  64 sequences of 1,024 to 8,192 tokens, 8 KV heads, 8 query heads each, us with two, three and four waves on a SIMD: 128 channels in 4 bits 47.2, 44.1, 53.4, in FP16 126.0, 124.1, 124.6; 64 in 4 bits 36.7,
// 32.9, 31.5, in FP16 69.0, 70.8, 70.7; 32 34.6, 30.9, 29.8 and 43.6, 40.8, 41.7.  Workgroups that weigh many: three to a compute unit, which is what LDS has room for of 128 channels.
constexpr uint32_t kWeighWorkers = 3 * 1024, kWeighGroups = 3 * 256;
// Queries of a sequence and KV head beyond which they share a workgroup's keys.  64 sequences of 512 to 4,096 tokens, the same heads, inputs that change from call to call, us, few / many: 24 rows, 128 channels 141 / 178, in 4 bits
// 52 / 97; 64 rows 230 / 178, 92 / 96 (64 channels 80 / 118, 66 / 75; 32 sequences of 256 channels 212 / 233, 108 / 121); 128 rows 398 / 198, 169 / 121 (128 / 132, 115 / 94; 360 / 254, 191 / 157).  So FP16 keys of 128
// channels would rather share from fewer rows on than the others.  (Few: the rows' queries are read again for every tile.)
constexpr uint32_t kManyRows = 64;

hipError_t launch_append_fp4(const AppendFp4Args& a, hipStream_t s);
hipError_t launch_unpack_fp4(const UnpackFp4Args& a, hipStream_t s);
hipError_t launch_evict(const EvictArgs& a, hipStream_t s);

// one source per head dimension
template <int D>
hipError_t launch_attend_fp4(const AttendFp4Args& a, hipStream_t s);
template <int D>
hipError_t launch_weigh(const WeighArgs& a, hipStream_t s);

}  // namespace kvc
