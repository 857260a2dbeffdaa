/*
 * kvc.h -- C ABI of libkvc: the KV-cache page codec of CXL-SpecKV for one AMD MI355X (gfx950).
 *
 * The library encodes paged FP16 K/V blocks into a compressed pool when they are offloaded
 * (the paper's Compression Engine, Section 3.5.2, Algorithm 2) and decodes pool blocks back into
 * a paged FP16 buffer when they are prefetched (Decompression Engine, Section 3.5.3; the
 * scatter-gather fetch through a translation table of Section 3.4.2, Algorithm 1).  The remote
 * (CXL) tier of the paper is a second buffer in the same GPU's HBM.
 *
 * Geometry.  A PAGE is N tokens x d channels of one KV head, FP16, row-major (N*d*2 bytes; 16 x 128
 * gives the paper's 4 KB page).  Any N >= 1 and any d that is a multiple of 32 up to 256 with N*d <= 4096 is
 * accepted.  The kernels are compiled per channel count and page length; pages that are a whole number of
 * 512-element passes with N in {8, 16, 32} (every d at N = 16) have instantiations of their own, other token
 * counts run on ones that read N at run time (a little slower).  A BLOCK is `pages_per_block` pages (all KV
 * heads, or K and V of all heads, of one 16-token block).  A cache buffer is FP16 [n_blocks][ppb][N][d] unless
 * kvc_set_cache_layout gives other strides.
 *
 * Compressed form of a page = one 16-byte descriptor (kvc_desc) + a payload of n16*16 bytes in
 * the pool.  Payload by mode:
 *   0 RAW    the N*d*2 input bytes unchanged (requested, or the page holds a NaN/Inf);
 *   1 INT8   q[j][i] = round_half_even(x * (1/s)), s = max|X|/127 (binary32), N*d bytes;
 *   2 DELTA  q differenced along i (first column verbatim), wrapped to 8 bits, zig-zag mapped to
 *            u, cut into groups of 32; header of one 4-bit code per group (group g in byte g/2,
 *            even g in the low nibble) followed by the group bodies; code w in 1..8 = literal
 *            packet, 4*w bytes, u_k in bits [k*w,(k+1)*w) of the little-endian bit string;
 *   3 RLE    as 2, plus code 0 = 32 zeros (no body) and code 9 = 32 copies of one byte (1 byte);
 *   4 PACK   as 3 with u = zig-zag of q itself, no differencing (for data without correlation
 *            along the channel index; not part of the paper's algorithm);
 *   5 CHAN   as 4 with the values regrouped so that a group holds one pair of neighbouring channels
 *            over the 16 tokens of the page (see KVC_MODE_CHAN below; N = 16, d = 64, 128 or 256 only; not part
 *            of the paper's algorithm);
 *   payloads are zero-padded to 16 bytes; a mode-2/3/4/5 page whose payload would not be smaller
 *   than its INT8 payload is stored as mode 1.
 * Decoding yields fp16(fp32(q) * s), one binary32 multiply and one round-to-nearest-even.
 *
 * Memory.  Every data pointer below is DEVICE memory allocated and owned by the caller; the
 * library owns only the host-side context and a small device state block (pool cursor, sticky
 * status).  `stream` is a hipStream_t passed as void* (NULL = the default stream).
 *
 * Asynchrony and errors.  compress / decompress / gather only enqueue kernels.  They return 0 or a
 * negative KVC_ERR_* for faults the host can see (nothing is enqueued then).  Faults only the
 * device can see set sticky KVC_ST_* bits: the page gets mode 0xFF (compress) or is zero-filled
 * (decompress); kvc_stats() reports them.  Block ids < 0 mean "skip this block".
 * Calls on one context that overlap on different streams race on the pool cursor; serialise them.
 * A context belongs to the device that was current in kvc_create; calls made with another device
 * current return KVC_ERR_ARG.  A context is not thread-safe: one host thread at a time.
 * The data calls (compress, decompress, gather, prefetch, reset) launch kernels only: no allocation, no
 * memset, no synchronisation, so a stream that is being captured into a HIP graph may record them.
 * One data call handles at most 2^26 - 4 pages (blocks * pages_per_block; 256 GiB of 4 KB pages: the
 * largest launch of 256-thread workgroups, one wave per page, that stays below 2^32 threads); more is
 * KVC_ERR_ARG.
 */
#ifndef KVC_H
#define KVC_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define KVC_OK 0
#define KVC_ERR_ARG (-1)          /* bad argument (null pointer, size out of range) */
#define KVC_ERR_NOT_BOUND (-2)    /* kvc_bind_pool has not been called */
#define KVC_ERR_HIP (-3)          /* a HIP runtime call failed */
#define KVC_ERR_POOL_FULL (-4)    /* reported by kvc_stats: at least one page did not fit */
#define KVC_ERR_CORRUPT (-5)      /* reported by kvc_stats: bad descriptor, payload or index */
#define KVC_ERR_UNSUPPORTED (-6)  /* geometry the kernels are not built for */
#define KVC_ERR_TOO_LARGE (-7)    /* the call exceeds the library's static workspace */

#define KVC_MODE_RAW 0
#define KVC_MODE_INT8 1
#define KVC_MODE_DELTA 2
#define KVC_MODE_RLE 3
#define KVC_MODE_PACK 4 /* extension beyond Algorithm 2: as 3 without the delta step (u = zigzag(q)) */
/* Extension beyond Algorithm 2, for 16-token pages: the packets of mode 4 over groups that hold one
 * pair of neighbouring channels across the 16 tokens, so that each pair packs at its own width.
 * With o = c / 8 the channel's octet, j = (c / 2) mod 4 its pair inside the octet and W = min(16, d / 8),
 * element (t, c) goes to group ((o div W) * 4 + j) * W + o mod W, position
 * (t mod 4) * 8 + (t div 4) * 2 + c mod 2.  Compress produces it, and decompress reads it, for
 * tokens_per_block = 16 and head_dim 64, 128 or 256 only. */
#define KVC_MODE_CHAN 5
#define KVC_MODE_INVALID 0xFF

#define KVC_ST_POOL_FULL 1u  /* a page did not fit into the pool */
#define KVC_ST_CORRUPT 2u    /* descriptor/payload failed validation on decode */
#define KVC_ST_BAD_INDEX 4u  /* a block id or table entry pointed outside its buffer */

typedef struct kvc_ctx kvc_ctx; /* opaque host object */

/* Page descriptor, 16 bytes, little-endian.  The paper's output <s, D_RLE> (Algorithm 2) is
 * {scale, payload at off}. */
typedef struct {
    uint64_t off;  /* byte offset of the payload in the pool, multiple of 16 */
    float scale;   /* s; 0 for RAW and all-zero pages */
    uint16_t n16;  /* payload bytes / 16, padding included */
    uint8_t mode;  /* KVC_MODE_* */
    uint8_t rsvd;  /* 0 */
} kvc_desc;

typedef struct {
    int32_t tokens_per_block; /* N >= 1 */
    int32_t head_dim;         /* d: a multiple of 32, 32..256;  N*d <= 4096 */
    int32_t pages_per_block;  /* ppb >= 1 */
    int32_t scheme;           /* mode requested from compress: 0..5 (5: N = 16, d = 64, 128 or 256 only, else KVC_ERR_UNSUPPORTED) */
} kvc_config;

typedef struct {
    uint64_t pool_bytes_used; /* bytes handed out by the pool cursor (capped at the pool size) */
    uint64_t pages[6];        /* bound descriptors per mode 0..5 */
    uint64_t pages_invalid;   /* bound descriptors with mode 0xFF (never written, or did not fit) */
    uint64_t payload_bytes;   /* sum of n16*16 over descriptors of mode 0..5 */
    uint32_t status;          /* OR of KVC_ST_* since the last kvc_reset_pool */
    uint32_t rsvd;
} kvc_stats_t;

/* Create / destroy a context.  kvc_create allocates the device state block on the current device. */
int kvc_create(kvc_ctx** out, const kvc_config* cfg);
void kvc_destroy(kvc_ctx* ctx);

/* Change the mode compress requests (0..5, with the geometry limit of mode 5); takes effect for later calls. */
int kvc_set_scheme(kvc_ctx* ctx, int32_t scheme);

/* Layout of the FP16 cache buffers read by compress and written by decompress / gather / prefetch,
 * in FP16 elements: element (token j, channel i) of page p of block b is at
 * b*block_stride + p*page_stride + j*row_stride + i.  Default (and all three = 0): contiguous pages,
 * row_stride = d, page_stride = N*d, block_stride = ppb*N*d.  Example: a [block][token][head][d] cache has
 * row_stride = H*d, page_stride = d, block_stride = N*H*d.  Strides are multiples of 8 (128-bit
 * accesses), row_stride >= d.  n_cache_blocks / n_out_blocks then count blocks of block_stride
 * elements; the caller guarantees the buffer covers the last block's last row. */
int kvc_set_cache_layout(kvc_ctx* ctx, int64_t block_stride, int64_t page_stride, int64_t row_stride);

/* Attach the compressed pool (pool_bytes, 16-byte aligned, any multiple of 16) and the descriptor
 * table (n_desc_pages entries; page p of pool block b is entry b*ppb + p).  Both caller-owned.
 * Either may also be pinned, device-mapped host memory (hipHostMalloc): the pool then sits behind
 * the host link, the closest single-GPU analogue of the paper's remote tier.  Pageable host
 * pointers are refused with KVC_ERR_ARG. */
int kvc_bind_pool(kvc_ctx* ctx, void* d_pool, uint64_t pool_bytes, kvc_desc* d_desc, uint64_t n_desc_pages);

/* Cursor = 0, status = 0, every descriptor = INVALID.  Enqueues fill kernels only. */
int kvc_reset_pool(kvc_ctx* ctx, void* stream);

/* Resume on a pool that was filled earlier: the cursor continues at used_bytes (a multiple of 16, at most
 * the pool size; the value kvc_stats reported as pool_bytes_used when the pool was saved), the status is
 * cleared, the descriptors are left as they are.  A pool, its descriptor table and that one number are a
 * complete checkpoint of the compressed tier: copy them back into buffers of the same sizes, bind them to
 * a context of the same geometry, call this, and compress, decompress and gather go on as before.
 * Enqueues one small kernel. */
int kvc_restore_pool(kvc_ctx* ctx, uint64_t used_bytes, void* stream);

/* Algorithm 2 over n blocks.  Block i is read from cache block src[i] (NULL: i) and stored as pool
 * block pool[i] (NULL: i).  d_cache: FP16 [n_cache_blocks][ppb][N][d].  Space comes from a bump
 * cursor; placement order inside the pool is unspecified, descriptors say where each page is.
 * Re-compressing into an occupied pool block leaks its old span until kvc_reset_pool. */
int kvc_compress_blocks(kvc_ctx* ctx, const void* d_cache, int64_t n_cache_blocks, const int32_t* d_src_block_ids,
                        const int32_t* d_pool_block_ids, int32_t n, void* stream);

/* As kvc_compress_blocks, with the requested mode given per block: d_block_scheme[i] in 0..5 where the
 * geometry has mode 5 (N = 16, d = 64, 128 or 256), else 0..4; higher values are read as the highest.
 * It applies to block i of the call.  This is the mechanism behind the paper's
 * layer-wise algorithm selection (Sections 3.1 (vi) and 3.6.3); the selection policy is the caller's. */
int kvc_compress_blocks_mixed(kvc_ctx* ctx, const void* d_cache, int64_t n_cache_blocks, const int32_t* d_src_block_ids,
                              const int32_t* d_pool_block_ids, const uint8_t* d_block_scheme, int32_t n, void* stream);

/* Inverse (Section 3.5.3) over n blocks: pool block pool[i] (NULL: i) is decoded into output block
 * dst[i] (NULL: i) of d_cache_out, FP16 [n_out_blocks][ppb][N][d]. */
int kvc_decompress_blocks(kvc_ctx* ctx, void* d_cache_out, int64_t n_out_blocks, const int32_t* d_pool_block_ids,
                          const int32_t* d_dst_block_ids, int32_t n, void* stream);

/* Prefetch fetch of Algorithm 1: for every layer l, sequence s and j < k, logical block
 * pred[s][j] is translated through block_table[s][.] to a pool block of that layer
 * (l*pool_blocks_per_layer + entry) and decoded into output block (l*n_seq + s)*k + j of d_out,
 * FP16 [n_layers*n_seq*k][ppb][N][d].  d_block_table: int32 [n_seq][max_blocks]; d_pred: int32
 * [n_seq][k].  pred < 0 or a table entry < 0 skips the block; values beyond their range set
 * KVC_ST_BAD_INDEX and zero-fill the block. */
int kvc_gather_decompress(kvc_ctx* ctx, void* d_out, const int32_t* d_block_table, int32_t max_blocks,
                          const int32_t* d_pred, int32_t n_seq, int32_t k, int32_t n_layers,
                          int64_t pool_blocks_per_layer, void* stream);

/* Speculative prefetch of Algorithm 1 into a double-buffered L2 prefetch buffer (Section 3.3.1), for
 * layers [layer_begin, layer_end) of one decode step; the token predictor is outside (d_pred is given).
 *   d_l2    FP16 [2][n_layers*n_seq*k][ppb][N][d]: two halves; this call fills half `fill_half`, the
 *           other half is what the previous step filled (and what attention may be reading).  Under
 *           kvc_set_cache_layout a slot is a block of that layout: slot i of half h starts at element
 *           (h*n_layers*n_seq*k + i) * block_stride.
 *   d_tags  int32 [2][n_layers*n_seq*k]: pool block held by every slot, -1 = empty (kvc_prefetch_reset).
 *   d_fetch int32 [n_layers*n_seq*k], out: pool block decoded into slot (l,s,j) by this call, or -1.
 *   d_loc   int32 [n_layers*n_seq*k], out: where the consumer finds predicted block (l,s,j):
 *           half*n_slots + slot (>= 0), -2 = resident in the GPU-local cache (logical block >=
 *           d_l1_first_block[s]; pass NULL for no L1), -1 = no block (pred < 0, table entry < 0, or an
 *           index out of range, which also sets KVC_ST_BAD_INDEX).
 * For every (layer, sequence) the k predictions are taken in order: translate through the block
 * table; if the pool block is in L1, in any slot of the other half, in a slot of this half already
 * settled in this step, or already in its own slot j, nothing is fetched (the residency test
 * "A_phys not in L1 u L2"); otherwise slot j of this half is claimed and the block decoded into it.
 * Stale slots are never cleared, only overwritten (lazy invalidation, Section 3.4.3).
 * k <= 32.  Calls for disjoint layer ranges may run on different streams (layer l+1, l+2 prefetch while layer l
 * computes, Section 3.4.4); calls for the same layers must be ordered. */
/* Slot policy of kvc_prefetch_layers.  0 (default): as described above, prediction j uses slot j
 * (Algorithm 1's L2[i]).  1: slot reuse -- a block wanted by this step that already sits in ANY slot of
 * either half stays there, and a block in neither half is decoded into the lowest slot of the half being
 * filled whose content this step does not want; d_fetch is then indexed by destination slot.  A window
 * sliding over consecutive blocks then transfers one block per new block instead of k. */
int kvc_set_prefetch_policy(kvc_ctx* ctx, int32_t policy);
int kvc_prefetch_reset(kvc_ctx* ctx, int32_t* d_tags, int32_t n_seq, int32_t k, int32_t n_layers, void* stream);
int kvc_prefetch_layers(kvc_ctx* ctx, void* d_l2, int32_t* d_tags, int32_t* d_fetch, int32_t* d_loc,
                        const int32_t* d_block_table, int32_t max_blocks, const int32_t* d_pred,
                        const int32_t* d_l1_first_block, int32_t n_seq, int32_t k, int32_t n_layers, int32_t layer_begin,
                        int32_t layer_end, int64_t pool_blocks_per_layer, int32_t fill_half, void* stream);

/* kvc_prefetch_layers with Algorithm 1's outstanding-request window (WaitCompletion over at most
 * Omega_max concurrent transfers; Section 3.4.2 gives the paper's controller a window of 16): the
 * transfers the planner issues are queued in issue order (layer, sequence, slot) and carried out by at
 * most `omega` transfer engines (workgroups), each holding one block in flight: an engine asks for no
 * payload of a block before the block it carried out before that is complete in memory.  An engine carries
 * out its entries in queue order.  Which ones it takes is unspecified: the first few of every engine are
 * dealt in advance (in a row, or one to each engine in turn), the others are taken as they come, up to
 * eight in a row.  omega >= 1; a small omega leaves most of the GPU to the computation
 * the prefetch hides behind, a large one approaches kvc_prefetch_layers.  Plan arrays (tags, fetch, loc)
 * and buffer contents are those of kvc_prefetch_layers.
 *   d_notify  int64 [n_layers + 4], device, out.  Entry l (layers of the call only): 0 while transfers
 *             of layer l are outstanding, then the device's wall clock (hipDeviceAttributeWallClockRate
 *             ticks, never 0) at which its last transfer was reported complete -- the ready notification
 *             a consumer may poll or wait for; a layer that needed no transfer is stamped when the window
 *             opens.  Engines report up to eight blocks at a time: at the end of the entries they took in a
 *             row, or, looking ahead, when the next block is one of another layer and has been asked for.
 *             A layer may thus be complete up to seven blocks of one engine before its stamp.
 *             [n_layers] = clock when the window opened, [n_layers+1] = transfers issued by the call,
 *             [n_layers+2] = transfer engines the call put to work: at most omega, at most one per transfer
 *             issued, at most what the GPU holds at once (1,024 to 1,792 on MI355X, by page shape), and
 *             beyond 256 only while each engine has at least eight transfers; no more blocks than that are
 *             ever in flight,
 *             [n_layers+3] = 0 until every transfer of the call has completed, then that clock value; who
 *             sees it finds all layers stamped.
 *   d_work    device workspace of at least kvc_prefetch_window_workspace(n_blocks, n_layers_call) bytes,
 *             256-byte aligned, n_blocks = (layer_end - layer_begin) * n_seq * k, n_layers_call =
 *             layer_end - layer_begin; caller-owned, contents meaningless between calls.  Calls that
 *             overlap in time need workspaces and notify arrays of their own.
 * A call over no slots (layer_begin = layer_end, n_seq = 0 or k = 0) does nothing. */
uint64_t kvc_prefetch_window_workspace(int64_t n_blocks, int32_t n_layers_call);
/* Rate of the clock the d_notify stamps count, in kHz, on the current device (KVC_ERR_HIP if the query fails). */
int kvc_wall_clock_khz(int32_t* khz);
int kvc_prefetch_layers_window(kvc_ctx* ctx, void* d_l2, int32_t* d_tags, int32_t* d_fetch, int32_t* d_loc,
                               const int32_t* d_block_table, int32_t max_blocks, const int32_t* d_pred,
                               const int32_t* d_l1_first_block, int32_t n_seq, int32_t k, int32_t n_layers,
                               int32_t layer_begin, int32_t layer_end, int64_t pool_blocks_per_layer, int32_t fill_half,
                               int32_t omega, int64_t* d_notify, void* d_work, uint64_t work_bytes, void* stream);

/* kvc_prefetch_layers_window for callers that cannot allocate and have no workspace to pass: code under
 * HIP graph capture, tight serving loops, harnesses that forbid allocation.  The window's queue lives in
 * a static device array inside the library (about 260 KB per GPU, held from library load until the
 * process ends), so one call covers at most 65,536 slots ((layer_end - layer_begin) * n_seq * k) and at
 * most 1,024 layers; more returns KVC_ERR_TOO_LARGE and enqueues nothing.  The call itself allocates and
 * frees nothing and only launches kernels (the array is cleared by them, not by a memset).  Results are
 * those of kvc_prefetch_layers_window.  Every call on one GPU, from any context, shares the one array:
 * calls that overlap in time on a GPU (different streams, or different contexts) race on it; order them. */
int kvc_prefetch_layers_window_static(kvc_ctx* ctx, void* d_l2, int32_t* d_tags, int32_t* d_fetch, int32_t* d_loc,
                                      const int32_t* d_block_table, int32_t max_blocks, const int32_t* d_pred,
                                      const int32_t* d_l1_first_block, int32_t n_seq, int32_t k, int32_t n_layers,
                                      int32_t layer_begin, int32_t layer_end, int64_t pool_blocks_per_layer,
                                      int32_t fill_half, int32_t omega, int64_t* d_notify, void* stream);

/* ---- Decode steps over the paged cache ---------------------------------------------------------
 * What a serving program does with the FP16 cache and the compressed pool between offload and fetch: it
 * writes new tokens' keys and values into the cache, computes attention over it, forks sequences, and gives
 * up the blocks of those that ended.  The calls follow the rules above: they only enqueue kernels (and may
 * be recorded into a HIP graph), block ids < 0 mean "no block", an id or table entry beyond its buffer sets
 * KVC_ST_BAD_INDEX and counts as no block.
 *
 * The cache has the context's geometry and layout (kvc_set_cache_layout).  Keys of KV head h are page h of a
 * block.  Their values are page n_kv_heads + h of the same block where d_v_cache is NULL (pages_per_block =
 * 2 * n_kv_heads), else page h of the same block of d_v_cache (pages_per_block = n_kv_heads).  Token t of a
 * sequence is row t mod N of the block that entry t div N of its row of the block table names. */

/* New tokens of a batch: token i (of n_new) of sequence s has its K and V rows written to position
 * lens[s] - n_new + i of the sequence, so that lens counts the new tokens already, as kvc_attend takes it.
 * Positions below 0 and positions without a block are skipped. */
typedef struct {
    void* d_k_cache;
    void* d_v_cache;        /* NULL: values are in d_k_cache */
    int64_t n_cache_blocks; /* of either */
    const int32_t* d_block_table; /* [n_seq][max_blocks] */
    const int32_t* d_lens;        /* [n_seq] */
    const void* d_k_new;    /* FP16: element (s, i, h, c) at s*k_strides[0] + i*k_strides[1] + h*k_strides[2] + c */
    const void* d_v_new;
    int64_t k_strides[3], v_strides[3]; /* FP16 elements, multiples of 8; both pointers 16-byte aligned */
    int32_t max_blocks, n_seq, n_new, n_kv_heads;
} kvc_append_t;
int kvc_append(kvc_ctx* ctx, const kvc_append_t* a, void* stream);

/* Attention of the last n_q tokens of every sequence over the sequence's tokens, and over a prefix that a
 * group of consecutive sequences shares.  n_heads query heads, n_heads / n_kv_heads of them to a KV head.
 * Query i of sequence s sees the tokens t < lens[s] - (n_q - 1 - i) of its own row of d_block_table, and all
 * prefix_lens[g] tokens of row g of d_prefix_table where prefix_first[g] <= s < prefix_first[g+1].  With
 * x_t = scale * <q, k_t> and m = max x_t:  out = sum e^(x_t - m) v_t / sum e^(x_t - m), and, where asked for,
 * lse = m + ln sum e^(x_t - m).  Tokens without a block do not exist: what memory holds in their place, and
 * behind the last token, is never read into a sum, and an infinite or NaN value of one of the last tokens only into
 * those of the queries that see it.  A query that sees no token gets out = 0, lse = -inf, and so does one all of whose scores are -infinity (its weights
 * are taken as zero, which 0 / 0 leaves open).  A NaN score that a query sees makes its out and lse NaN.  An infinite value that it sees with a weight of zero (the score is
 * -infinity, or the weight was rounded, below 2^-34 of the largest) makes its channel of out NaN, or infinite where it is of one of the last tokens.
 * Each prefix is read once for its group, not once for every sequence.  Lengths beyond their table's row set
 * KVC_ST_BAD_INDEX and are cut to it.  Sums, maxima and products are held in 32 bits; the weights e^(x_t - m)
 * are rounded to FP16 (11 bits, far from its smallest numbers) for the product with the values.
 * Groups out of order set KVC_ST_BAD_INDEX, and no prefix is seen then.  d_out must not overlap what is read.
 * Lengths are on the device, so the width of a table stands for the longest: a call is refused if n_seq * n_kv_heads * (a KV head's rows of a sequence, by 16 or 32) *
 * (max_blocks * N / 32 + 1) passes 2^31 - 1, or the like of the prefixes (rows of all groups by 128); and which kernels it takes goes by the widths.
 * d_work: device memory of at least kvc_attend_workspace(...) bytes, 256-byte aligned, contents meaningless
 * between calls; calls that overlap in time need workspaces of their own. */
typedef struct {
    const void* d_q;        /* FP16: element (s, i, head, c) at s*q_strides[0] + i*q_strides[1] + head*q_strides[2] + c */
    void* d_out;            /* FP16, with out_strides likewise */
    float* d_lse;           /* NULL, or [n_seq][n_q][n_heads] */
    int64_t q_strides[3], out_strides[3]; /* FP16 elements, multiples of 8; both pointers 16-byte aligned */
    const void* d_k_cache;
    const void* d_v_cache;  /* NULL: values are in d_k_cache */
    int64_t n_cache_blocks; /* of either */
    const int32_t* d_block_table;  /* [n_seq][max_blocks] */
    const int32_t* d_lens;         /* [n_seq], the last n_q tokens included */
    const int32_t* d_prefix_table; /* [n_prefix][max_prefix_blocks]; the three may be NULL where n_prefix = 0 */
    const int32_t* d_prefix_lens;  /* [n_prefix] */
    const int32_t* d_prefix_first; /* [n_prefix + 1], non-decreasing, 0..n_seq; sequences outside all groups have no prefix */
    int32_t max_blocks, max_prefix_blocks, n_prefix, n_seq, n_q, n_heads, n_kv_heads;
    float scale;                   /* finite */
    void* d_work;
    uint64_t work_bytes;
} kvc_attend_t;
int kvc_attend(kvc_ctx* ctx, const kvc_attend_t* a, void* stream);
/* Workspace of a call of these sizes, in bytes (0: sizes that kvc_attend refuses, with whatever tables). */
uint64_t kvc_attend_workspace(int32_t n_seq, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_prefix);

/* A cache in 4 bits: the values of the same pages, in about a quarter of the memory.  32 neighbouring channels of a token share a power of two 2^e, and each is one of
 * 0, 0.5, 1, 1.5, 2, 3, 4, 6 of it, with a sign.  e is the smallest whole number with max |x| <= 7 * 2^e, and at most 13; a magnitude becomes the nearest of the eight,
 * halfway the one of even number, beyond 6 * 2^e that.  (So nothing is off by more than 2^e, but for magnitudes beyond 57,344 = 7 * 2^13, which become 49,152.)  32
 * channels of which one is infinite or NaN are all NaN.  What is written so stands for FP16 numbers; of other codes and exponents (half of 2^-26, 6 * 2^14) the nearest FP16 value, or infinity.
 * A page is N * d/2 bytes of codes (token by token, channel 2i in the low half of byte i; the sign is the code's highest bit, the rest the
 * number of the magnitude), N bytes of e + 127 for every 32 channels in turn (0 where all are zero, 255 for NaN), and 0 to 15 bytes that make a multiple of 16.  A block is
 * pages_per_block pages in a row, a cache blocks in a row, whatever kvc_set_cache_layout says; 16-byte aligned. */
uint64_t kvc_fp4_block_bytes(int32_t tokens_per_block, int32_t head_dim, int32_t pages_per_block); /* 0: a shape that kvc_create refuses */

/* kvc_append into a cache in 4 bits: the caches of *a are in 4 bits, the new rows are FP16.  Refused: heads whose rows of one token, K and V, are 2^31 pieces of 16 bytes or more. */
int kvc_append_fp4(kvc_ctx* ctx, const kvc_append_t* a, void* stream);

/* Blocks of a cache in 4 bits, in FP16: block src[i] of d_cache goes to block dst[i] of d_out (NULL: i), i < n.  d_out has the context's geometry and layout; no block
 * may be destination twice, and the two may not overlap.  A pair with an id < 0 is skipped, one with an id beyond its buffer too, and sets KVC_ST_BAD_INDEX. */
int kvc_unpack_fp4(kvc_ctx* ctx, void* d_out, int64_t n_out_blocks, const void* d_cache, int64_t n_cache_blocks, const int32_t* d_src_ids, const int32_t* d_dst_ids, int32_t n, void* stream);

/* kvc_attend over a cache in 4 bits, as if its values were in FP16: the same numbers, rounded the same way.  There are no prefixes (n_prefix = 0; d_prefix_* are not looked at):
 * parts can be joined by their lse. */
int kvc_attend_fp4(kvc_ctx* ctx, const kvc_attend_t* a, void* stream);
/* Workspace of a call of these sizes, in bytes (0: sizes that it refuses, with whatever tables). */
uint64_t kvc_attend_fp4_workspace(int32_t n_seq, int32_t n_q, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);

/* The attention weight that tokens get.  For every sequence s, KV head h and token t < lens[s]
 *     weights_out[s][h][t] = w + sum over queries i and heads of h's group of e^(scale * <q, k_t> - lse),
 * over the queries that see t, which are those of kvc_attend (query i sees the tokens t < lens[s] - (n_q - 1 - i)), with w = weights[s][h][t], or 0 for the last n_q tokens,
 * which are new; those also get their position, positions[s][h][t] = seen[s] - (lens[s] - t).  lse is what attention over the same tokens gave (of all tokens that the weights shall
 * sum to one over: with a prefix, of both parts); a query with lse = -infinity gives nothing.  Where a NaN score or lse is seen, the weight is NaN.  Tokens without a block get
 * nothing, and what lies behind lens[s] in the arrays is not touched.  Scores, weights and sums are held in 32 bits, added in a fixed order.  weights_out may be weights.
 * Lengths beyond the table's row or `width` set KVC_ST_BAD_INDEX and are cut. */
typedef struct {
    const void* d_q;         /* FP16, with q_strides as in kvc_attend_t */
    int64_t q_strides[3];
    const void* d_k_cache;   /* pages h < n_kv_heads of a block are keys; pages_per_block is n_kv_heads or twice that */
    int64_t n_cache_blocks;
    const int32_t* d_block_table; /* [n_seq][max_blocks] */
    const int32_t* d_lens;        /* [n_seq] */
    const float* d_lse;           /* [n_seq][n_q][n_heads] */
    const float* d_weights;       /* [n_seq][n_kv_heads][width] */
    float* d_weights_out;
    int32_t* d_positions;         /* [n_seq][n_kv_heads][width] */
    const int32_t* d_seen;        /* [n_seq]: tokens that the sequence has had, evicted and new ones included */
    int32_t max_blocks, n_seq, n_q, n_heads, n_kv_heads, width;
    int32_t fp4;                  /* the cache is in 4 bits */
    float scale;                  /* finite */
} kvc_weigh_t;
int kvc_weigh(kvc_ctx* ctx, const kvc_weigh_t* a, void* stream);

/* Eviction.  Of every sequence and KV head keep[s] of the lens[s] tokens stay (all, if there are no more): those at positions >= seen[s] - min(recent, keep[s]), and of the
 * others the ones with the largest weights; of equal weights the lowest slots leave first, and NaN is larger than all.  (If more than keep[s] are at such positions, the highest slots of them stay.)  The slots t < keep[s] hold what stays: a token that stays below
 * keep[s] keeps its slot, and those from there on go, in order, to the slots that were left, in order.  Keys, values, weights and positions go with the token, each head for itself; new_lens[s]
 * is what stays.  Attention does not look at the order, and positions say which token is where.  What lies from new_lens[s] on is not touched.
 * Blocks are written in place: those that hold slots below keep[s] must be the sequence's alone (copies of FP16 blocks: kvc_copy_blocks; blocks in 4 bits are kvc_fp4_block_bytes bytes in a row, and copied as
 * such).  A sequence with a token that has no block, or lies beyond its table's row or `width`,
 * stays as it is, and sets KVC_ST_BAD_INDEX.  weights_out may be weights, positions_out positions, new_lens lens. */
typedef struct {
    void* d_k_cache;
    void* d_v_cache;        /* NULL: values are in d_k_cache */
    int64_t n_cache_blocks; /* of either */
    const int32_t* d_block_table; /* [n_seq][max_blocks] */
    const int32_t* d_lens;        /* [n_seq] */
    const int32_t* d_keep;        /* [n_seq]; below 0: 0 */
    const int32_t* d_seen;        /* [n_seq] */
    int32_t* d_new_lens;          /* [n_seq] */
    const float* d_weights;       /* [n_seq][n_kv_heads][width] */
    float* d_weights_out;
    const int32_t* d_positions;   /* [n_seq][n_kv_heads][width] */
    int32_t* d_positions_out;
    int32_t max_blocks, n_seq, n_kv_heads, width;
    int32_t recent;               /* >= 0 */
    int32_t fp4;                  /* the caches are in 4 bits */
    void* d_work;                 /* kvc_evict_workspace bytes, 256-byte aligned, contents meaningless between calls; calls that overlap in time need their own */
    uint64_t work_bytes;
} kvc_evict_t;
int kvc_evict(kvc_ctx* ctx, const kvc_evict_t* a, void* stream);
/* (0: sizes that kvc_evict refuses) */
uint64_t kvc_evict_workspace(int32_t n_seq, int32_t n_kv_heads, int32_t width);

/* Copy of blocks of an FP16 cache: in every layer l < n_layers, block l*blocks_per_layer + src[i] is copied to block
 * l*blocks_per_layer + dst[i] of the same cache, i < n.  One block may be copied to several; no block may be
 * both source and destination, nor destination twice. */
int kvc_copy_blocks(kvc_ctx* ctx, void* d_cache, int64_t n_cache_blocks, const int32_t* d_src_ids, const int32_t* d_dst_ids, int32_t n,
                    int32_t n_layers, int64_t blocks_per_layer, void* stream);

/* Fork of pool blocks, ids as in kvc_copy_blocks (l*pool_blocks_per_layer + id): block dst[i] becomes a second name of what
 * block src[i] holds.  Payloads are never written in place, so both share them: only descriptors are copied.
 * What dst[i] held before is given up (its span stays in use until kvc_compact_pool or kvc_reset_pool). */
int kvc_fork_blocks(kvc_ctx* ctx, const int32_t* d_src_ids, const int32_t* d_dst_ids, int32_t n, int32_t n_layers, int64_t pool_blocks_per_layer,
                    void* stream);

/* Pool blocks l*pool_blocks_per_layer + ids[i] are given up: their descriptors become INVALID.  A payload that another
 * block shares stays that block's. */
int kvc_free_blocks(kvc_ctx* ctx, const int32_t* d_ids, int32_t n, int32_t n_layers, int64_t pool_blocks_per_layer, void* stream);

/* The payloads that the bound descriptor table still names, moved together: to the beginning of d_pool_out, in the
 * order of their offsets, shared payloads once, with d_desc_out (as many entries as the bound table) naming
 * their new places and *d_used_out the bytes they take.  The bound pool and table are only read: decodes may go on,
 * until kvc_adopt_pool puts the context on the new ones.  A descriptor whose payload leaves the bound pool
 * becomes INVALID and sets KVC_ST_CORRUPT; one whose payload does not fit into pool_out_bytes becomes INVALID and sets
 * KVC_ST_POOL_FULL.  d_pool_out and d_desc_out may be in pinned, device-mapped host memory, as the bound ones may.  Pointers 16-byte aligned (d_used_out 8, d_work 256); none of the new
 * buffers may overlap another, or a bound one. */
int kvc_compact_pool(kvc_ctx* ctx, void* d_pool_out, uint64_t pool_out_bytes, kvc_desc* d_desc_out, uint64_t* d_used_out, void* d_work,
                     uint64_t work_bytes, void* stream);
/* Workspace of kvc_compact_pool on a bound pool of pool_bytes, in bytes: about a hundredth of it, and 10 KB. */
uint64_t kvc_compact_workspace(uint64_t pool_bytes);

/* kvc_bind_pool on buffers that kvc_compact_pool has filled: the cursor goes to *d_used (device memory, read on the
 * stream), the status stays.  The old buffers may be released when the compaction, and whatever else was enqueued on them, has run.
 * Graphs that were captured before go on with the old ones. */
int kvc_adopt_pool(kvc_ctx* ctx, void* d_pool, uint64_t pool_bytes, kvc_desc* d_desc, uint64_t n_desc_pages, const uint64_t* d_used, void* stream);

/* Reduce the descriptor table and read the device state.  The only call that synchronises
 * (on `stream`).  Returns KVC_ERR_POOL_FULL / KVC_ERR_CORRUPT if the matching status bit is set
 * (out is filled either way), else 0. */
int kvc_stats(kvc_ctx* ctx, kvc_stats_t* out, void* stream);

const char* kvc_strerror(int code);

/* ---- Verification and measurement hooks -------------------------------------------------------
 * The calls below are not steps of the codec path and no codec call depends on them.  They exist so
 * that a test can check the encoder's scale arithmetic exhaustively, so that a benchmark can time a
 * plain copy with the codec's access shape on the same device, through the same library, and so that it
 * can record the clocks the runtime reports beside the bandwidth it measures. */

/* Shader clock, memory clock (both kHz) and memory bus width (bits) of the current device, as
 * hipDeviceGetAttribute reports them; any pointer may be NULL.  KVC_ERR_HIP if a query fails. */
int kvc_device_clocks(int32_t* shader_khz, int32_t* memory_khz, int32_t* memory_bus_bits);

/* The scaling step of Algorithm 2 on its own: for n page maxima given as FP16 bit patterns (sign
 * ignored) write s = amax / 127 and s_inv = 1 / s as the encoder computes them (binary32); 0, Inf
 * and NaN give 0 for both.  All three arrays are device memory.  The encoder does not use IEEE
 * division instructions for these quotients; this call lets a test compare its arithmetic with
 * plain division for every possible maximum. */
int kvc_page_scales(const uint16_t* d_amax, float* d_scale, float* d_scale_inv, uint64_t n, void* stream);

/* dst[0..nbytes) = src[0..nbytes), a wavefront per contiguous 4 KB with 128-bit loads and stores;
 * nbytes a multiple of 16 and at most 2^38 - 4096 (else KVC_ERR_ARG); both pointers device memory, 16-byte
 * aligned, not overlapping.  The bandwidth yardstick the codec kernels are compared with. */
int kvc_copy_bytes(void* d_dst, const void* d_src, uint64_t nbytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* KVC_H */
