// Entry points of the operators that keep the paged cache small (see include/kvc.h): argument checks and kernel launches only.
#include <cmath>

#include "kvc_checks.h"
#include "kvc_fp4.h"

using namespace kvc;

static Fp4Pages pages_of(const kvc_ctx* ctx) { return fp4_pages(ctx->g.N, ctx->g.d, ctx->g.ppb); }
// A block's bytes, and strides of FP16 in steps of 8, are counted in 32 bits.
static bool blocks_ok(const kvc_ctx* ctx, bool fp4) {
    return fp4 ? pages_of(ctx).block <= UINT32_MAX : ctx->g.block_stride / 8 <= UINT32_MAX && ctx->g.row_stride / 8 <= UINT32_MAX;
}
// where values begin: `v`, or behind the key pages of `k`
static const uint8_t* values_fp4(const Fp4Pages& f, const void* k, const void* v, int32_t n_kv) {
    return v ? static_cast<const uint8_t*>(v) : static_cast<const uint8_t*>(k) + (int64_t)n_kv * f.page;
}
// Tokens of a table's row are counted in 31 bits.
static bool tokens_ok(const kvc_ctx* ctx, int32_t max_blocks) { return (int64_t)max_blocks * ctx->g.N <= INT32_MAX - 256; }
// New tokens of a call from which on several of a sequence share a workgroup.
constexpr int64_t kManyNew = 2048;
static bool product_ok(int64_t a, int64_t b, int64_t c) { return (__int128)a * b * c <= INT32_MAX; }

// What attention and the weighing of tokens have in common.
static AttendArgs attend_args(const kvc_ctx* ctx, const void* q, const int64_t* q_strides, int64_t n_cache_blocks, const int32_t* table, const int32_t* lens, int32_t max_blocks, int32_t n_seq,
                              int32_t n_q, int32_t n_heads, int32_t n_kv, float scale) {
    AttendArgs a = {};
    a.q = static_cast<const uint16_t*>(q);
    for (int i = 0; i < 3; ++i) a.q_strides[i] = q_strides[i];
    a.n_cache_blocks = n_cache_blocks;
    a.table = table;
    a.lens = lens;
    a.max_blocks = max_blocks;
    a.n_seq = n_seq;
    a.n_q = n_q;
    a.n_heads = n_heads;
    a.n_kv = n_kv;
    a.group = n_heads / n_kv;
    a.rows = a.group * n_q;
    a.scale_log2 = scale * 1.44269504088896341f;
    a.g = ctx->g;
    a.by_N = make_fast_div((uint32_t)ctx->g.N);
    a.by_rows = make_fast_div((uint32_t)a.rows);
    a.by_n_q = make_fast_div((uint32_t)n_q);
    a.st = ctx->st;
    a.join_lanes = 1;
    return a;
}

extern "C" {

uint64_t kvc_fp4_block_bytes(int32_t tokens_per_block, int32_t head_dim, int32_t pages_per_block) {
    if (tokens_per_block < 1 || head_dim < 32 || head_dim > 256 || head_dim % 32 || (int64_t)tokens_per_block * head_dim > 4096 || pages_per_block < 1) return 0;
    return (uint64_t)fp4_pages(tokens_per_block, head_dim, pages_per_block).block;
}

int kvc_append_fp4(kvc_ctx* ctx, const kvc_append_t* p, void* stream) {
    if (!ctx || !p || p->n_seq < 0 || p->n_new < 0 || p->max_blocks < 0 || p->n_cache_blocks < 0) return KVC_ERR_ARG;
    if (!heads_ok(ctx, p->d_v_cache, p->n_kv_heads)) return KVC_ERR_ARG;
    if (p->n_seq == 0 || p->n_new == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!p->d_k_cache || (!p->d_block_table && p->max_blocks) || !p->d_lens || !p->d_k_new || !p->d_v_new) return KVC_ERR_ARG;
    if (!aligned(p->d_k_cache, 16) || !aligned(p->d_v_cache, 16) || !aligned(p->d_k_new, 16) || !aligned(p->d_v_new, 16)) return KVC_ERR_ARG;
    if (!strides_ok(p->k_strides) || !strides_ok(p->v_strides)) return KVC_ERR_ARG;
    if ((int64_t)p->n_seq * p->n_new > kMaxGroups || !product_ok(2, p->n_kv_heads, ctx->g.lpr)) return KVC_ERR_ARG;
    AppendFp4Args x = {};
    x.f = pages_of(ctx);
    x.k_cache = static_cast<uint8_t*>(p->d_k_cache);
    x.v_cache = const_cast<uint8_t*>(values_fp4(x.f, p->d_k_cache, p->d_v_cache, p->n_kv_heads));
    AppendArgs& a = x.a;
    a.n_cache_blocks = p->n_cache_blocks;
    a.table = p->d_block_table;
    a.lens = p->d_lens;
    a.k_new = static_cast<const uint16_t*>(p->d_k_new);
    a.v_new = static_cast<const uint16_t*>(p->d_v_new);
    for (int i = 0; i < 3; ++i) a.k_strides[i] = p->k_strides[i], a.v_strides[i] = p->v_strides[i];
    a.max_blocks = p->max_blocks;
    a.n_seq = p->n_seq;
    a.n_new = p->n_new;
    a.n_kv = p->n_kv_heads;
    a.g = ctx->g;
    a.by_N = make_fast_div((uint32_t)ctx->g.N);
    a.by_n_new = make_fast_div((uint32_t)p->n_new);
    a.by_lpr = make_fast_div((uint32_t)ctx->g.lpr);
    a.st = ctx->st;
    x.wide = (int64_t)p->n_seq * p->n_new >= kManyNew && p->n_new > 1;
    x.turns = x.wide ? ((uint32_t)p->n_new + kTurn - 1) / kTurn : (uint32_t)p->n_new;
    x.by_turns = make_fast_div(x.turns);
    return launched(launch_append_fp4(x, static_cast<hipStream_t>(stream)));
}

int kvc_unpack_fp4(kvc_ctx* ctx, void* d_out, int64_t n_out_blocks, const void* d_cache, int64_t n_cache_blocks, const int32_t* d_src_ids, const int32_t* d_dst_ids, int32_t n, void* stream) {
    if (!ctx || n_out_blocks < 0 || n_cache_blocks < 0 || n < 0) return KVC_ERR_ARG;
    if (n == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!d_out || !d_cache || !aligned(d_out, 16) || !aligned(d_cache, 16)) return KVC_ERR_ARG;
    if ((!d_src_ids && n > n_cache_blocks) || (!d_dst_ids && n > n_out_blocks)) return KVC_ERR_ARG;
    UnpackFp4Args a;
    a.cache = static_cast<const uint8_t*>(d_cache);
    a.out = static_cast<uint16_t*>(d_out);
    a.n_cache_blocks = n_cache_blocks;
    a.n_out_blocks = n_out_blocks;
    a.src = d_src_ids;
    a.dst = d_dst_ids;
    a.f = pages_of(ctx);
    a.g = ctx->g;
    a.n = n;
    const int64_t chunks = (int64_t)ctx->g.ppb * ctx->g.N * ctx->g.lpr;
    if (chunks > (1ll << 30)) return KVC_ERR_ARG;
    a.chunks = (int32_t)chunks;
    a.pieces = (a.chunks + kCopyChunks - 1) / kCopyChunks;
    if (a.pieces > kMaxGroups / n) return KVC_ERR_ARG;
    a.by_lpr = make_fast_div((uint32_t)ctx->g.lpr);
    a.by_N = make_fast_div((uint32_t)ctx->g.N);
    a.by_pieces = make_fast_div((uint32_t)a.pieces);
    a.st = ctx->st;
    return launched(launch_unpack_fp4(a, static_cast<hipStream_t>(stream)));
}

uint64_t kvc_attend_fp4_workspace(int32_t n_seq, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim) {
    if (n_seq < 0 || n_q < 1 || n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads || head_dim < 32 || head_dim > 256 || head_dim % 32) return 0;
    if (!rows_ok(n_seq, n_q, n_heads, head_dim)) return 0;
    return plan_attend_fp4(n_seq, n_q, n_heads, n_kv_heads, head_dim).bytes;
}

int kvc_attend_fp4(kvc_ctx* ctx, const kvc_attend_t* p, void* stream) {
    if (!ctx || !p || p->n_seq < 0 || p->n_q < 1 || p->max_blocks < 0 || p->n_prefix != 0 || p->n_cache_blocks < 0) return KVC_ERR_ARG;
    if (!heads_ok(ctx, p->d_v_cache, p->n_kv_heads) || p->n_heads < p->n_kv_heads || p->n_heads % p->n_kv_heads) return KVC_ERR_ARG;
    if (p->n_seq == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!p->d_q || !p->d_out || !p->d_k_cache || (!p->d_block_table && p->max_blocks) || !p->d_lens) return KVC_ERR_ARG;
    if (!aligned(p->d_q, 16) || !aligned(p->d_out, 16) || !aligned(p->d_k_cache, 16) || !aligned(p->d_v_cache, 16)) return KVC_ERR_ARG;
    if (!strides_ok(p->q_strides) || !strides_ok(p->out_strides)) return KVC_ERR_ARG;
    if (!rows_ok(p->n_seq, p->n_q, p->n_heads, ctx->g.d) || !tokens_ok(ctx, p->max_blocks) || !blocks_ok(ctx, true)) return KVC_ERR_ARG;
    const AttendPlan plan = plan_attend_fp4(p->n_seq, p->n_q, p->n_heads, p->n_kv_heads, ctx->g.d);
    const int64_t own_tokens = (int64_t)p->max_blocks * ctx->g.N, rows = (int64_t)(p->n_heads / p->n_kv_heads) * p->n_q, own_tiles = (rows + plan.own_rows - 1) / plan.own_rows;
    if (!product_ok(own_tiles * p->n_kv_heads, p->n_seq, own_tokens / 32 + 1)) return KVC_ERR_ARG;
    if (!p->d_work || !aligned(p->d_work, 256) || p->work_bytes < plan.bytes) return KVC_ERR_ARG;
    if (!std::isfinite(p->scale * 1.44269504088896341f)) return KVC_ERR_ARG;
    AttendFp4Args x;
    x.f = pages_of(ctx);
    x.k = static_cast<const uint8_t*>(p->d_k_cache);
    x.v = values_fp4(x.f, p->d_k_cache, p->d_v_cache, p->n_kv_heads);
    x.a = attend_args(ctx, p->d_q, p->q_strides, p->n_cache_blocks, p->d_block_table, p->d_lens, p->max_blocks, p->n_seq, p->n_q, p->n_heads, p->n_kv_heads, p->scale);
    AttendArgs& a = x.a;
    a.out = static_cast<uint16_t*>(p->d_out);
    a.lse = p->d_lse;
    for (int i = 0; i < 3; ++i) a.out_strides[i] = p->out_strides[i];
    a.own_tiles = (uint32_t)own_tiles;
    a.own_workers = plan.own_workers;
    a.direct = direct_fp4(ctx->g.d, ctx->g.N % 8 == 0, plan.own_rows / 16, own_tiles * p->n_kv_heads * p->n_seq, own_tokens);
    // (as attention over FP16 has it)
    const int64_t threads = (int64_t)plan.rows * (ctx->g.d / 8);
    while (a.join_lanes < 16 && a.join_lanes * 2 * (ctx->g.d / 8) <= 256 && threads * a.join_lanes * 2 <= 1 << 17) a.join_lanes *= 2;
    uint8_t* w = static_cast<uint8_t*>(p->d_work);
    a.own_start = reinterpret_cast<uint32_t*>(w);
    a.stats = reinterpret_cast<float2v*>(w + plan.starts);
    a.sums = reinterpret_cast<float*>(w + plan.starts + round_256(plan.slots * 8));
    a.own_rows = plan.own_rows;
    a.own_slots = (int64_t)plan.rows;
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (ctx->g.d) {
        case 32: return launched(launch_attend_fp4<32>(x, s));
        case 64: return launched(launch_attend_fp4<64>(x, s));
        case 96: return launched(launch_attend_fp4<96>(x, s));
        case 128: return launched(launch_attend_fp4<128>(x, s));
        case 160: return launched(launch_attend_fp4<160>(x, s));
        case 192: return launched(launch_attend_fp4<192>(x, s));
        case 224: return launched(launch_attend_fp4<224>(x, s));
        case 256: return launched(launch_attend_fp4<256>(x, s));
    }
    return KVC_ERR_UNSUPPORTED;
}

int kvc_weigh(kvc_ctx* ctx, const kvc_weigh_t* p, void* stream) {
    if (!ctx || !p || p->n_seq < 0 || p->n_q < 1 || p->max_blocks < 0 || p->n_cache_blocks < 0 || p->width < 0) return KVC_ERR_ARG;
    if (p->n_kv_heads < 1 || (p->n_kv_heads != ctx->g.ppb && 2ll * p->n_kv_heads != ctx->g.ppb) || p->n_heads < p->n_kv_heads || p->n_heads % p->n_kv_heads) return KVC_ERR_ARG;
    if (p->n_seq == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!p->d_q || !p->d_k_cache || (!p->d_block_table && p->max_blocks) || !p->d_lens || !p->d_lse || !p->d_seen) return KVC_ERR_ARG;
    if (p->width && (!p->d_weights || !p->d_weights_out || !p->d_positions)) return KVC_ERR_ARG;
    if (!aligned(p->d_q, 16) || !aligned(p->d_k_cache, 16) || !strides_ok(p->q_strides)) return KVC_ERR_ARG;
    if (!rows_ok(p->n_seq, p->n_q, p->n_heads, ctx->g.d) || !tokens_ok(ctx, p->max_blocks) || !blocks_ok(ctx, p->fp4) || p->width > INT32_MAX - 256) return KVC_ERR_ARG;
    if (!product_ok(p->n_kv_heads, p->n_seq, (int64_t)p->max_blocks * ctx->g.N / 32 + 1)) return KVC_ERR_ARG;
    if (!std::isfinite(p->scale * 1.44269504088896341f)) return KVC_ERR_ARG;
    const uint64_t bytes = (uint64_t)p->n_seq * p->n_kv_heads * p->width * 4;
    if (p->d_weights != p->d_weights_out && !apart({p->d_weights, bytes}, {p->d_weights_out, bytes})) return KVC_ERR_ARG;
    if (!apart({p->d_positions, bytes}, {p->d_weights, bytes}) || !apart({p->d_positions, bytes}, {p->d_weights_out, bytes})) return KVC_ERR_ARG;
    WeighArgs x;
    x.a = attend_args(ctx, p->d_q, p->q_strides, p->n_cache_blocks, p->d_block_table, p->d_lens, p->max_blocks, p->n_seq, p->n_q, p->n_heads, p->n_kv_heads, p->scale);
    x.a.lse = const_cast<float*>(p->d_lse);
    x.a.k_cache = p->fp4 ? nullptr : static_cast<const uint16_t*>(p->d_k_cache);
    x.k = p->fp4 ? static_cast<const uint8_t*>(p->d_k_cache) : nullptr;
    x.f = pages_of(ctx);
    x.before = p->d_weights;
    x.after = p->d_weights_out;
    x.positions = p->d_positions;
    x.seen = p->d_seen;
    x.width = p->width;
    x.many = x.a.rows > (int32_t)kManyRows;
    x.workers = x.many ? kWeighGroups : kWeighWorkers;
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (ctx->g.d) {
        case 32: return launched(launch_weigh<32>(x, s));
        case 64: return launched(launch_weigh<64>(x, s));
        case 96: return launched(launch_weigh<96>(x, s));
        case 128: return launched(launch_weigh<128>(x, s));
        case 160: return launched(launch_weigh<160>(x, s));
        case 192: return launched(launch_weigh<192>(x, s));
        case 224: return launched(launch_weigh<224>(x, s));
        case 256: return launched(launch_weigh<256>(x, s));
    }
    return KVC_ERR_UNSUPPORTED;
}

// Workspace: moves of every sequence and head and how many they are, and tokens that stay.  (Slots are counted in 31 bits, moves too; a workgroup of 512 threads has a sequence and head.)
uint64_t kvc_evict_workspace(int32_t n_seq, int32_t n_kv_heads, int32_t width) {
    if (n_seq < 0 || n_kv_heads < 1 || width < 0 || width > INT32_MAX - 256 || !product_ok(n_seq, n_kv_heads, width / 2 + 1)) return 0;
    if ((int64_t)n_seq * n_kv_heads > kMaxGroups / 4) return 0;
    const uint64_t units = (uint64_t)n_seq * n_kv_heads;
    return round_256(units * 4) + round_256((uint64_t)n_seq * 4) + 2 * round_256(units * (uint64_t)(width / 2) * 4) + 256;
}

int kvc_evict(kvc_ctx* ctx, const kvc_evict_t* p, void* stream) {
    if (!ctx || !p || p->n_seq < 0 || p->max_blocks < 0 || p->n_cache_blocks < 0 || p->width < 0 || p->recent < 0) return KVC_ERR_ARG;
    if (!heads_ok(ctx, p->d_v_cache, p->n_kv_heads)) return KVC_ERR_ARG;
    const uint64_t need = kvc_evict_workspace(p->n_seq, p->n_kv_heads, p->width);
    if (!need) return KVC_ERR_ARG;
    if (p->n_seq == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!p->d_k_cache || (!p->d_block_table && p->max_blocks) || !p->d_lens || !p->d_keep || !p->d_seen || !p->d_new_lens) return KVC_ERR_ARG;
    if (p->width && (!p->d_weights || !p->d_weights_out || !p->d_positions || !p->d_positions_out)) return KVC_ERR_ARG;
    if (!aligned(p->d_k_cache, 16) || !aligned(p->d_v_cache, 16)) return KVC_ERR_ARG;
    if (!tokens_ok(ctx, p->max_blocks)) return KVC_ERR_ARG;
    if (!p->d_work || !aligned(p->d_work, 256) || p->work_bytes < need) return KVC_ERR_ARG;
    const uint64_t bytes = (uint64_t)p->n_seq * p->n_kv_heads * p->width * 4;
    const Buffer w = {p->d_weights, bytes}, wo = {p->d_weights_out, bytes}, o = {p->d_positions, bytes}, oo = {p->d_positions_out, bytes};
    if ((w.at != wo.at && !apart(w, wo)) || (o.at != oo.at && !apart(o, oo)) || !apart(w, o) || !apart(w, oo) || !apart(wo, o) || !apart(wo, oo)) return KVC_ERR_ARG;
    EvictArgs a;
    a.fp4 = p->fp4 != 0;
    a.f = pages_of(ctx);
    a.k = static_cast<uint8_t*>(p->d_k_cache);
    a.v = a.fp4 ? const_cast<uint8_t*>(values_fp4(a.f, p->d_k_cache, p->d_v_cache, p->n_kv_heads))
                : reinterpret_cast<uint8_t*>(const_cast<uint16_t*>(values_of(ctx, p->d_k_cache, p->d_v_cache, p->n_kv_heads)));
    a.g = ctx->g;
    a.n_cache_blocks = p->n_cache_blocks;
    a.table = p->d_block_table;
    a.lens = p->d_lens;
    a.keep = p->d_keep;
    a.weights = p->d_weights;
    a.weights_out = p->d_weights_out;
    a.positions = p->d_positions;
    a.positions_out = p->d_positions_out;
    a.seen = p->d_seen;
    a.new_lens = p->d_new_lens;
    a.recent = p->recent;
    a.width = p->width;
    a.max_blocks = p->max_blocks;
    a.n_seq = p->n_seq;
    a.n_kv = p->n_kv_heads;
    a.most = p->width / 2;
    a.by_N = make_fast_div((uint32_t)ctx->g.N);
    a.by_n_kv = make_fast_div((uint32_t)p->n_kv_heads);
    a.by_lanes = make_fast_div((uint32_t)(a.fp4 ? ctx->g.d / 32 : ctx->g.lpr));
    a.st = ctx->st;
    uint8_t* at = static_cast<uint8_t*>(p->d_work);
    const uint64_t units = (uint64_t)p->n_seq * p->n_kv_heads, list = round_256(units * (uint64_t)a.most * 4);
    a.counts = reinterpret_cast<int32_t*>(at);
    a.left = reinterpret_cast<int32_t*>(at + round_256(units * 4));
    a.holes = reinterpret_cast<int32_t*>(at + round_256(units * 4) + round_256((uint64_t)p->n_seq * 4));
    a.fillers = reinterpret_cast<int32_t*>(reinterpret_cast<uint8_t*>(a.holes) + list);
    return launched(launch_evict(a, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
