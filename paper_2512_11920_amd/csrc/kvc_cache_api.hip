// Entry points of the decode-step operators (see include/kvc.h): argument checks and kernel launches only.
#include <cmath>

#include "kvc_cache.h"
#include "kvc_ctx.h"

using namespace kvc;

static constexpr int64_t kMaxGroups = (1ll << 24) - 1;  // workgroups of 256 threads a launch holds
static constexpr int32_t kMaxLayers = 65535;             // of a call; the layer is a grid dimension of its own

static bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static bool strides_ok(const int64_t* s) {
    for (int i = 0; i < 3; ++i)
        if (s[i] < 0 || (s[i] & 7)) return false;
    return true;
}
// where values begin: `v`, or behind the key pages of `k`
static const uint16_t* values_of(const kvc_ctx* ctx, const void* k, const void* v, int32_t n_kv) {
    return v ? static_cast<const uint16_t*>(v) : static_cast<const uint16_t*>(k) + n_kv * ctx->g.page_stride;
}
static bool heads_ok(const kvc_ctx* ctx, const void* v, int32_t n_kv) { return n_kv >= 1 && (int64_t)n_kv * (v ? 1 : 2) == ctx->g.ppb; }
// Query rows are counted in 31 bits, and joined by one launch, d / 8 threads a row.
static bool rows_ok(int64_t n_seq, int64_t n_q, int64_t n_heads, int d) {
    return n_seq * n_heads <= INT32_MAX / n_q && n_seq * n_heads * n_q <= kMaxGroups * (2048 / d);
}
static int launched(hipError_t e) { return hip_ok(e) ? KVC_OK : KVC_ERR_HIP; }

extern "C" {

int kvc_append(kvc_ctx* ctx, const kvc_append_t* p, void* stream) {
    if (!ctx || !p || p->n_seq < 0 || p->n_new < 0 || p->max_blocks < 0 || p->n_cache_blocks < 0) return KVC_ERR_ARG;
    if (!heads_ok(ctx, p->d_v_cache, p->n_kv_heads)) return KVC_ERR_ARG;
    if (p->n_seq == 0 || p->n_new == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!p->d_k_cache || (!p->d_block_table && p->max_blocks) || !p->d_lens || !p->d_k_new || !p->d_v_new) return KVC_ERR_ARG;
    if (!aligned(p->d_k_cache, 16) || !aligned(p->d_v_cache, 16) || !aligned(p->d_k_new, 16) || !aligned(p->d_v_new, 16)) return KVC_ERR_ARG;
    if (!strides_ok(p->k_strides) || !strides_ok(p->v_strides)) return KVC_ERR_ARG;
    if ((int64_t)p->n_seq * p->n_new > kMaxGroups) return KVC_ERR_ARG;
    AppendArgs a;
    a.k_cache = static_cast<uint16_t*>(p->d_k_cache);
    a.v_cache = const_cast<uint16_t*>(values_of(ctx, p->d_k_cache, p->d_v_cache, p->n_kv_heads));
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
    return launched(launch_append(a, static_cast<hipStream_t>(stream)));
}

uint64_t kvc_attend_workspace(int32_t n_seq, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_prefix) {
    if (n_seq < 0 || n_q < 1 || n_kv_heads < 1 || n_heads < n_kv_heads || n_heads % n_kv_heads || head_dim < 32 || head_dim > 256 || head_dim % 32 || n_prefix < 0) return 0;
    if (!rows_ok(n_seq, n_q, n_heads, head_dim)) return 0;
    return plan_attend(n_seq, n_q, n_heads, n_kv_heads, head_dim, n_prefix).bytes;
}

int kvc_attend(kvc_ctx* ctx, const kvc_attend_t* p, void* stream) {
    if (!ctx || !p || p->n_seq < 0 || p->n_q < 1 || p->max_blocks < 0 || p->n_prefix < 0 || p->max_prefix_blocks < 0 || p->n_cache_blocks < 0) return KVC_ERR_ARG;
    if (!heads_ok(ctx, p->d_v_cache, p->n_kv_heads) || p->n_heads < p->n_kv_heads || p->n_heads % p->n_kv_heads) return KVC_ERR_ARG;
    if (p->n_seq == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!p->d_q || !p->d_out || !p->d_k_cache || (!p->d_block_table && p->max_blocks) || !p->d_lens) return KVC_ERR_ARG;
    if (!aligned(p->d_q, 16) || !aligned(p->d_out, 16) || !aligned(p->d_k_cache, 16) || !aligned(p->d_v_cache, 16)) return KVC_ERR_ARG;
    if (!strides_ok(p->q_strides) || !strides_ok(p->out_strides)) return KVC_ERR_ARG;
    if (p->n_prefix > 0 && ((!p->d_prefix_table && p->max_prefix_blocks) || !p->d_prefix_lens || !p->d_prefix_first)) return KVC_ERR_ARG;
    if (!rows_ok(p->n_seq, p->n_q, p->n_heads, ctx->g.d)) return KVC_ERR_ARG;
    // a row's tokens are counted in 31 bits, and so are the tiles of all units
    const int64_t own_tokens = (int64_t)p->max_blocks * ctx->g.N, prefix_tokens = (int64_t)p->max_prefix_blocks * ctx->g.N;
    if (own_tokens > INT32_MAX - 256 || prefix_tokens > INT32_MAX - 256 || ctx->g.block_stride / 8 > UINT32_MAX) return KVC_ERR_ARG;
    const AttendPlan plan = plan_attend(p->n_seq, p->n_q, p->n_heads, p->n_kv_heads, ctx->g.d, p->n_prefix);
    const int64_t rows = (int64_t)(p->n_heads / p->n_kv_heads) * p->n_q, own_tiles = (rows + plan.own_rows - 1) / plan.own_rows;
    const int64_t prefix_tiles = (rows * p->n_seq + plan.prefix_rows - 1) / plan.prefix_rows + p->n_prefix;
    const auto product = [](int64_t a, int64_t b, int64_t c) { return (__int128)a * b * c; };
    if (product(own_tiles * p->n_kv_heads, p->n_seq, own_tokens / 32 + 1) > INT32_MAX) return KVC_ERR_ARG;
    if (p->n_prefix && product(prefix_tiles, p->n_kv_heads, prefix_tokens / 32 + 1) > INT32_MAX) return KVC_ERR_ARG;
    if (!p->d_work || !aligned(p->d_work, 256) || p->work_bytes < plan.bytes) return KVC_ERR_ARG;
    if (!std::isfinite(p->scale * 1.44269504088896341f)) return KVC_ERR_ARG;
    AttendArgs a;
    a.q = static_cast<const uint16_t*>(p->d_q);
    a.out = static_cast<uint16_t*>(p->d_out);
    a.lse = p->d_lse;
    for (int i = 0; i < 3; ++i) a.q_strides[i] = p->q_strides[i], a.out_strides[i] = p->out_strides[i];
    a.k_cache = static_cast<const uint16_t*>(p->d_k_cache);
    a.v_cache = values_of(ctx, p->d_k_cache, p->d_v_cache, p->n_kv_heads);
    a.n_cache_blocks = p->n_cache_blocks;
    a.table = p->d_block_table;
    a.lens = p->d_lens;
    a.prefix_table = p->d_prefix_table;
    a.prefix_lens = p->d_prefix_lens;
    a.prefix_first = p->d_prefix_first;
    a.max_blocks = p->max_blocks;
    a.max_prefix_blocks = p->max_prefix_blocks;
    a.n_prefix = p->n_prefix;
    a.n_seq = p->n_seq;
    a.n_q = p->n_q;
    a.n_heads = p->n_heads;
    a.n_kv = p->n_kv_heads;
    a.group = p->n_heads / p->n_kv_heads;
    a.rows = a.group * a.n_q;
    a.scale_log2 = p->scale * 1.44269504088896341f;
    a.g = ctx->g;
    a.by_N = make_fast_div((uint32_t)ctx->g.N);
    a.by_rows = make_fast_div((uint32_t)a.rows);
    a.by_n_q = make_fast_div((uint32_t)a.n_q);
    a.st = ctx->st;
    a.own_tiles = (uint32_t)own_tiles;
    a.own_workers = plan.own_workers;
    a.prefix_workers = plan.prefix_workers;
    a.direct = p->n_prefix == 0 && direct_fits(ctx->g.d, plan.own_rows / 16) && own_tokens <= (int64_t)kDirectTiles * 32 && product(own_tiles, p->n_kv_heads, p->n_seq) <= kMaxGroups / 2;
    // (tables may be longer than the prefixes in them)
    a.apart = p->n_prefix && both_fit(ctx->g.d, plan.own_rows / 16) && product(prefix_tiles, p->n_kv_heads, prefix_tokens / 32 + 1) <= kApartTiles;
    // Few rows have many pieces: about 2^17 threads join them, at most 16 to a row's channels.  One sequence of 8,192 tokens, 8 x 128, the whole call: 35 us with one to a
    // row's channels, 16 with 16.  (4,096 rows of 9 or 10 pieces: 6.8 us with two, 7.4 with one, 9.5 with four.)
    const int64_t threads = (int64_t)plan.rows * (ctx->g.d / 8);
    a.join_lanes = 1;
    while (a.join_lanes < 16 && a.join_lanes * 2 * (ctx->g.d / 8) <= 256 && threads * a.join_lanes * 2 <= 1 << 17) a.join_lanes *= 2;
    if (a.apart) {
        a.own_workers = kOwnWorkers;
        a.prefix_workers = kPrefixWorkers;
    }
    uint8_t* w = static_cast<uint8_t*>(p->d_work);
    a.own_start = reinterpret_cast<uint32_t*>(w);
    a.prefix_start = reinterpret_cast<uint32_t*>(w + round_256((uint64_t)(p->n_seq + 1) * 4));
    a.stats = reinterpret_cast<float2v*>(w + plan.starts);
    a.sums = reinterpret_cast<float*>(w + plan.starts + round_256(plan.slots * 8));
    a.own_rows = plan.own_rows;
    a.prefix_rows = plan.prefix_rows;
    a.own_slots = (int64_t)plan.rows;
    a.prefix_whole = a.own_slots + 2ll * plan.own_workers * plan.own_rows;
    a.prefix_slots = a.prefix_whole + (int64_t)plan.rows;
    hipStream_t s = static_cast<hipStream_t>(stream);
    switch (ctx->g.d) {
        case 32: return launched(launch_attend<32>(a, s));
        case 64: return launched(launch_attend<64>(a, s));
        case 96: return launched(launch_attend<96>(a, s));
        case 128: return launched(launch_attend<128>(a, s));
        case 160: return launched(launch_attend<160>(a, s));
        case 192: return launched(launch_attend<192>(a, s));
        case 224: return launched(launch_attend<224>(a, s));
        case 256: return launched(launch_attend<256>(a, s));
    }
    return KVC_ERR_UNSUPPORTED;
}

int kvc_copy_blocks(kvc_ctx* ctx, void* d_cache, int64_t n_cache_blocks, const int32_t* d_src_ids, const int32_t* d_dst_ids, int32_t n, int32_t n_layers,
                    int64_t blocks_per_layer, void* stream) {
    if (!ctx || n_cache_blocks < 0 || n < 0 || n_layers < 0 || blocks_per_layer < 0) return KVC_ERR_ARG;
    if (n == 0 || n_layers == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!d_cache || !aligned(d_cache, 16) || !d_src_ids || !d_dst_ids) return KVC_ERR_ARG;
    if (n_layers > kMaxLayers || blocks_per_layer > n_cache_blocks / n_layers) return KVC_ERR_ARG;
    CopyArgs a;
    a.cache = static_cast<uint16_t*>(d_cache);
    a.n_cache_blocks = n_cache_blocks;
    a.src = d_src_ids;
    a.dst = d_dst_ids;
    a.n = n;
    a.n_layers = n_layers;
    a.per_layer = blocks_per_layer;
    a.g = ctx->g;
    const int64_t chunks = (int64_t)ctx->g.ppb * ctx->g.N * ctx->g.lpr;
    if (chunks > (1ll << 30)) return KVC_ERR_ARG;
    a.chunks = (int32_t)chunks;
    a.pieces = (a.chunks + kCopyChunks - 1) / kCopyChunks;
    if (a.pieces > kMaxGroups / n) return KVC_ERR_ARG;
    a.dense = (ctx->g.row_stride == ctx->g.d && ctx->g.page_stride == ctx->g.E) || (ctx->g.page_stride == ctx->g.d && ctx->g.row_stride == (int64_t)ctx->g.ppb * ctx->g.d);
    a.by_lpr = make_fast_div((uint32_t)ctx->g.lpr);
    a.by_N = make_fast_div((uint32_t)ctx->g.N);
    a.by_pieces = make_fast_div((uint32_t)a.pieces);
    a.st = ctx->st;
    return launched(launch_copy_blocks(a, static_cast<hipStream_t>(stream)));
}

static int ids_call(kvc_ctx* ctx, bool fork, const int32_t* src, const int32_t* dst, int32_t n, int32_t n_layers, int64_t per_layer, void* stream) {
    if (!ctx || n < 0 || n_layers < 0 || per_layer < 0) return KVC_ERR_ARG;
    if (!ctx->pool) return KVC_ERR_NOT_BOUND;
    if (n == 0 || n_layers == 0) return KVC_OK;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!dst || (fork && !src)) return KVC_ERR_ARG;
    if (n_layers > kMaxLayers || (uint64_t)per_layer > ctx->n_desc / (uint64_t)ctx->g.ppb / (uint64_t)n_layers) return KVC_ERR_ARG;
    IdsArgs a;
    a.desc = ctx->desc;
    a.src = src;
    a.dst = dst;
    a.n_pages = (int64_t)n * ctx->g.ppb;
    if (a.n_pages > INT32_MAX) return KVC_ERR_ARG;
    a.ppb = ctx->g.ppb;
    a.n_layers = n_layers;
    a.per_layer = per_layer;
    a.by_ppb = make_fast_div((uint32_t)ctx->g.ppb);
    a.st = ctx->st;
    hipStream_t s = static_cast<hipStream_t>(stream);
    return launched(fork ? launch_fork(a, s) : launch_free(a, s));
}

int kvc_fork_blocks(kvc_ctx* ctx, const int32_t* d_src_ids, const int32_t* d_dst_ids, int32_t n, int32_t n_layers, int64_t pool_blocks_per_layer, void* stream) {
    return ids_call(ctx, true, d_src_ids, d_dst_ids, n, n_layers, pool_blocks_per_layer, stream);
}

int kvc_free_blocks(kvc_ctx* ctx, const int32_t* d_ids, int32_t n, int32_t n_layers, int64_t pool_blocks_per_layer, void* stream) {
    return ids_call(ctx, false, nullptr, d_ids, n, n_layers, pool_blocks_per_layer, stream);
}

// Workspace: the bitmap, the counts within groups, the groups' sums.
uint64_t kvc_compact_workspace(uint64_t pool_bytes) {
    const uint64_t groups = compact_groups(pool_bytes);
    return groups * kGroupWords * 10 + round_256(groups * 8);
}

struct Buffer {
    const void* at;
    uint64_t n;
};
static bool apart(const Buffer& a, const Buffer& b) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
    return x <= y ? y - x >= a.n : x - y >= b.n;
}

int kvc_compact_pool(kvc_ctx* ctx, void* d_pool_out, uint64_t pool_out_bytes, kvc_desc* d_desc_out, uint64_t* d_used_out, void* d_work, uint64_t work_bytes, void* stream) {
    if (!ctx) return KVC_ERR_ARG;
    if (!ctx->pool) return KVC_ERR_NOT_BOUND;
    if (!on_ctx_device(ctx)) return KVC_ERR_ARG;
    if (!d_pool_out || !d_desc_out || !d_used_out || !d_work || pool_out_bytes == 0 || (pool_out_bytes & 15)) return KVC_ERR_ARG;
    if (!aligned(d_pool_out, 16) || !aligned(d_desc_out, 16) || !aligned(d_used_out, 8) || !aligned(d_work, 256)) return KVC_ERR_ARG;
    if (work_bytes < kvc_compact_workspace(ctx->pool_bytes)) return KVC_ERR_ARG;
    // (where the bound ones may be, these may be: see kvc_bind_pool)
    hipPointerAttribute_t attr;
    void* desc_at = d_desc_out;
    if (!seen_by_device(&d_pool_out, &attr) || !seen_by_device(&desc_at, &attr)) return KVC_ERR_ARG;
    d_desc_out = static_cast<kvc_desc*>(desc_at);
    const Buffer written[] = {{d_pool_out, pool_out_bytes}, {d_desc_out, ctx->n_desc * 16}, {d_used_out, 8}, {d_work, kvc_compact_workspace(ctx->pool_bytes)}};
    for (const Buffer& w : written) {
        if (!apart(w, {ctx->pool, ctx->pool_bytes}) || !apart(w, {ctx->desc, ctx->n_desc * 16})) return KVC_ERR_ARG;
        for (const Buffer* o = written; o != &w; ++o)
            if (!apart(w, *o)) return KVC_ERR_ARG;
    }
    CompactArgs a;
    a.pool = ctx->pool;
    a.units = ctx->pool_bytes / 16;
    a.out_units = pool_out_bytes / 16;
    a.pool_out = static_cast<uint8_t*>(d_pool_out);
    a.desc = ctx->desc;
    a.desc_out = d_desc_out;
    a.n_desc = ctx->n_desc;
    a.groups = compact_groups(ctx->pool_bytes);
    if (a.groups * 64 + a.n_desc / 256 > (uint64_t)kMaxGroups - 1) return KVC_ERR_ARG;
    uint8_t* w = static_cast<uint8_t*>(d_work);
    a.bits = reinterpret_cast<unsigned long long*>(w);
    w += a.groups * kGroupWords * 8;
    a.before = reinterpret_cast<uint16_t*>(w);
    w += a.groups * kGroupWords * 2;
    a.base = reinterpret_cast<unsigned long long*>(w);
    a.used = reinterpret_cast<unsigned long long*>(d_used_out);
    a.st = ctx->st;
    return launched(launch_compact(a, static_cast<hipStream_t>(stream)));
}

int kvc_adopt_pool(kvc_ctx* ctx, void* d_pool, uint64_t pool_bytes, kvc_desc* d_desc, uint64_t n_desc_pages, const uint64_t* d_used, void* stream) {
    if (!ctx || !d_used || !aligned(d_used, 8) || !on_ctx_device(ctx)) return KVC_ERR_ARG;
    const int rc = kvc_bind_pool(ctx, d_pool, pool_bytes, d_desc, n_desc_pages);
    if (rc != KVC_OK) return rc;
    return launched(launch_adopt(ctx->st, reinterpret_cast<const unsigned long long*>(d_used), static_cast<hipStream_t>(stream)));
}

}  // extern "C"
