/*
 * libtidal — decode-step attention of TidalDecode's Position Persistent Sparse
 * Attention (arxiv 2410.05076) for NVIDIA B200 (sm_100a).
 *
 * The library covers the attention branch of the paper's Algorithm 1 for one
 * decode step: full attention over the whole KV cache (full-attention layers),
 * full attention that also ranks every cached token by its query-key inner
 * product and keeps the top k (token selection layers), and sparse attention
 * over only the positions kept by the last selection layer (all other
 * layers), and the cache update (the new token's key and value rows written
 * into the cache). Beside it stand a coarser selection of whole blocks of 16
 * tokens with its attention, and the filling of paged caches (page tables and
 * slot maps from request lengths, many tokens' rows), and what a prompt needs
 * on its way there: norms and rotary positions of queries and keys, attention
 * of chunks of new tokens, the attention weight every cached position receives
 * and the eviction of those that receive least. Projections and FFN are the
 * caller's; the decode step takes queries and keys that are position-encoded.
 *
 * Conventions shared by every call
 *   - All tensor pointers are DEVICE pointers unless a parameter says "host".
 *     The caller owns every buffer; the library owns only its context and the
 *     workspace inside it and keeps no reference to caller memory after the
 *     work it enqueued has run.
 *   - Calls enqueue work on the CUDA stream passed as `stream` (a cudaStream_t
 *     cast to void*, NULL = the legacy default stream) and return without
 *     waiting for it, except where stated.
 *   - Return value: TIDAL_OK or a negative tidal_status_t. Argument errors are
 *     detected on the host before anything is enqueued. Nothing throws or
 *     aborts across this boundary. Problems only the device can see (a token
 *     index outside the cache, a page id outside the pool) make the kernel skip
 *     that element and set a sticky status word read by tidal_device_status().
 *   - q is bf16 [batch, num_q_heads, head_dim] contiguous; outputs are fp32
 *     [batch, num_q_heads, head_dim] contiguous. Arithmetic: bf16 inputs,
 *     fp32 accumulation.
 *   - A context holds scratch memory and counters that its calls share: use it
 *     from one host thread and on one stream at a time (work of consecutive
 *     calls may overlap on that stream; calls on two streams need two contexts).
 *   - There is no CPU path: on a machine without a usable GPU tidal_create()
 *     fails with TIDAL_ERR_CUDA.
 */
#ifndef TIDAL_H
#define TIDAL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct tidal_ctx tidal_ctx_t;     /* opaque: device, workspace, kernel attributes */
typedef int32_t tidal_status_t;

enum {
    TIDAL_OK = 0,
    TIDAL_ERR_INVALID = -1,       /* bad argument (NULL pointer, k <= 0, misaligned stride, ...) */
    TIDAL_ERR_UNSUPPORTED = -2,   /* valid request outside what is built (head_dim != 128, ...) */
    TIDAL_ERR_NOMEM = -3,         /* workspace allocation failed */
    TIDAL_ERR_CUDA = -4,          /* a CUDA runtime call failed */
    TIDAL_ERR_TIMEOUT = -5,       /* a bounded wait of a kernel on its own copies or products expired: a bug, results invalid */
    TIDAL_ERR_INDEX = -6,         /* device saw a token index or page id out of range */
    TIDAL_ERR_TOO_LARGE = -7,     /* tidal_sparse_attn_noalloc only: problem exceeds its fixed scratch */
    TIDAL_ERR_PAGES = -9,         /* tidal_page_map: the request does not fit its arrays or the pool (nothing was changed) */
    TIDAL_ERR_INTERNAL = -8       /* a kernel found the host's launch plan inconsistent: a bug, results invalid */
};

enum { TIDAL_KV_CONTIG = 0, TIDAL_KV_PAGED = 1 };

/* Granularity of the selected token set (number of index heads Hi).
 * PER_QHEAD is the paper's definition (Eq. 1 and Section 3.1 are per attention
 * head): Hi = num_q_heads. The other two rank by the sum of the member heads'
 * scaled logits: PER_KVHEAD has Hi = num_kv_heads, SHARED has Hi = 1. */
enum { TIDAL_SEL_PER_QHEAD = 0, TIDAL_SEL_PER_KVHEAD = 1, TIDAL_SEL_SHARED = 2 };

/* Layer types of Algorithm 1 / Figure 2. */
enum { TIDAL_LAYER_FULL = 0, TIDAL_LAYER_SELECT = 1, TIDAL_LAYER_SPARSE = 2 };

/* KV cache of one layer. Strides count bf16 ELEMENTS and must be multiples of
 * 8 (16 bytes); k and v must be 16-byte aligned; a row (head_dim elements of
 * one position and KV head) is contiguous.
 *   contiguous: K[b, pos, g, c] at k + b*stride_b + pos*stride_pos + g*stride_head + c
 *   paged:      page = page_table[b*max_pages_per_seq + pos/page_size], slot = pos%page_size,
 *               K[b, pos, g, c] at k + page*stride_page + slot*stride_pos + g*stride_head + c
 * V uses the same strides from `v`. The cache already contains the token being
 * decoded (Algorithm 1 appends before attention), so ctx_lens[b] >= 1 counts it. */
typedef struct {
    int32_t batch, num_q_heads, num_kv_heads, head_dim;   /* head_dim == 128; Hq % Hkv == 0; Hq/Hkv <= 8 */
    int32_t kv_layout;                                    /* TIDAL_KV_CONTIG or TIDAL_KV_PAGED */
    const void *k, *v;                                    /* device, bf16 */
    int64_t stride_b, stride_pos, stride_head, stride_page;
    const int32_t *page_table;      /* device int32 [batch, max_pages_per_seq]; paged only */
    int32_t page_size;              /* 16 (paged only) */
    int32_t max_pages_per_seq;
    int32_t num_pages;              /* physical pages in the pool; page ids are checked against it */
    const int32_t *ctx_lens;        /* device int32 [batch] */
    int32_t max_ctx_len;            /* host upper bound of ctx_lens; 1 .. 262144 */
    float sm_scale;                 /* 0 => 1/sqrt(head_dim), the scale of Eq. 1 */
    int32_t kv_dtype;               /* TIDAL_KV_BF16 (0) or TIDAL_KV_FP8_E4M3 */
    const float *k_scale, *v_scale; /* FP8 only: device float [num_kv_heads] each, NULL = 1 */
} tidal_kv_t;

/* Element type of the cache. The paper assumes half precision; TIDAL_KV_FP8_E4M3 is this library's
 * 8-bit variant: k and v hold OCP FP8 E4M3 codes (no infinities, largest value 448) and element
 * (b, pos, g, c) stands for decode(code) * k_scale[g] (v_scale[g] for V); attention is Eq. 1 on those
 * values. Strides still count elements, i.e. bytes, and must be multiples of 16; a row is 128
 * contiguous bytes. The query stays bf16 (it is converted to fp16 inside the kernels, exactly for
 * magnitudes between 6.1e-5 and 65504). Not available: tidal_set_attend_newest,
 * tidal_sparse_attn_noalloc, tidal_set_select_margin (ignored). */
enum { TIDAL_KV_BF16 = 0, TIDAL_KV_FP8_E4M3 = 1 };

/* Create a context on CUDA device `device`. workspace_bytes preallocates that much scratch
 * (0 = none). Whatever a later call needs beyond what the context holds is allocated inside that
 * call (which then also synchronises the device): use tidal_reserve() to do all of it up front. */
tidal_status_t tidal_create(tidal_ctx_t **ctx, int device, size_t workspace_bytes);
tidal_status_t tidal_destroy(tidal_ctx_t *ctx);

/* Allocates, now, everything later calls with this cache shape (batch, heads, max_ctx_len) and a
 * budget up to k will need: the scratch workspace and the small block of counters and histograms
 * that scale with batch * num_q_heads. num_layers_host is the layer count of later
 * tidal_decode_step_host calls (0 if that call is not used). After it, calls with shapes no larger
 * allocate nothing and do not synchronise, so they can be captured into a CUDA graph from the first
 * one on. May allocate and synchronise itself; call it outside any capture. For max_ctx_len > 16384 it
 * also allocates the scratch of tidal_block_select (a fiftieth of the rest); if only that does not fit,
 * it succeeds without, and tidal_block_select returns TIDAL_ERR_NOMEM when it finds no memory either. */
tidal_status_t tidal_reserve(tidal_ctx_t *ctx, const tidal_kv_t *kv, int32_t k, int32_t num_layers_host);

/* Workspace a call with this cache shape and budget k needs (split-context
 * partial results, the score buffer of a selection layer, top-k histograms). */
size_t tidal_workspace_bytes(const tidal_kv_t *kv, int32_t k);

/* C.append(k, v) of Algorithm 1 for one layer: writes the new token's key and value rows
 * (k_new, v_new: device bf16 [batch, num_kv_heads, head_dim], contiguous, 16-byte aligned; for an
 * FP8 cache the rows are E4M3 codes already, quantised by the caller with the cache's scales) into
 * the cache at position ctx_lens[b] - 1, the slot that the lengths already count, through the
 * layout described by `kv` (contiguous or paged). The cache memory behind kv->k / kv->v is
 * WRITTEN by this call although the descriptor declares it const. Sequences with
 * ctx_lens[b] < 1 or > max_ctx_len and page ids outside the pool are skipped (the latter is
 * reported by tidal_device_status). q and k are expected position-encoded already: rotary or
 * other position encodings are the caller's. */
tidal_status_t tidal_kv_append(tidal_ctx_t *ctx, const tidal_kv_t *kv, const void *k_new,
                               const void *v_new, void *stream);

/* FullAttention(q, C[:]) of Algorithm 1, Eq. 1 per head:
 *   out[b,h,:] = softmax_j(q[b,h,:] . K[b,j,g,:] * sm_scale) V[b,j,g,:],  j < ctx_lens[b], g = h / (Hq/Hkv).
 * The single decode query sees every cached token (no mask). */
tidal_status_t tidal_full_attn(tidal_ctx_t *ctx, const tidal_kv_t *kv, const void *q,
                               float *out, void *stream);

/* Token selection layer of Algorithm 1 (Section 3: the inner products are
 * stored during full attention, then the k tokens with the highest values are
 * kept): out as tidal_full_attn, and for every (sequence, index head) the
 * k' = min(k, ctx_lens[b]) positions with the largest scaled logit, equal
 * logits resolved toward the lower position.
 *   idx       int32 [batch, Hi, k]: the positions in ascending order, padded with -1.
 *   idx_count int32 [batch] or NULL: receives k'.
 *   scores_opt float [batch, Hq, max_ctx_len] or NULL: receives the scaled
 *             logits q.k*sm_scale (entries at and beyond ctx_lens[b] are unspecified);
 *             with NULL they live in the workspace (with fewer index heads than
 *             query heads the workspace then holds only the per-KV-head sums). */
tidal_status_t tidal_select_attn(tidal_ctx_t *ctx, const tidal_kv_t *kv, const void *q,
                                 int32_t k, int32_t granularity, float *out, int32_t *idx,
                                 int32_t *idx_count, float *scores_opt, void *stream);

/* SparseAttention(q, C[rho]) of Algorithm 1: Eq. 1 restricted to the positions
 * listed for the query head's index head hi = h * Hi / Hq, softmax renormalised
 * over them. -1 is padding and skipped; any other entry outside
 * [0, ctx_lens[b]) is skipped too and reported as TIDAL_ERR_INDEX by
 * tidal_device_status(); a repeated
 * entry counts once per occurrence. Only the first idx_count[b] entries are
 * read when idx_count is given, else k. A head with no valid entry gets zeros.
 * num_index_heads must be Hq, Hkv or 1. */
tidal_status_t tidal_sparse_attn(tidal_ctx_t *ctx, const tidal_kv_t *kv, const void *q,
                                 const int32_t *idx, const int32_t *idx_count, int32_t k,
                                 int32_t num_index_heads, float *out, void *stream);

/* One decode step's attention for all layers (the loop of Algorithm 1):
 * schedule[i] (host, TIDAL_LAYER_*) picks the call for layer i; the token set
 * rho lives in idx/idx_count, is written by every selection layer and read by
 * the sparse layers after it. kv_per_layer (host array of descriptors),
 * q_per_layer and out_per_layer (host arrays of device pointers) have
 * num_layers entries. A sparse layer before the first selection layer is
 * TIDAL_ERR_INVALID. Everything is enqueued without host waits and is complete, in
 * stream order, when the work enqueued on `stream` is: a selection layer may run part
 * of its work (its value pass) on a second stream that the context owns, forked from
 * and joined back into `stream` with events, also inside a stream capture. */
tidal_status_t tidal_decode_step(tidal_ctx_t *ctx, int32_t num_layers, const uint8_t *schedule,
                                 const tidal_kv_t *kv_per_layer, const void *const *q_per_layer,
                                 float *const *out_per_layer, int32_t k, int32_t granularity,
                                 int32_t *idx, int32_t *idx_count, void *stream);

/* Optional deviation from Algorithm 1 (off by default): with enabled != 0 every later sparse layer on
 * this context also attends the newest token, position ctx_lens[b] - 1, whether or not it was
 * selected. A list that already ends with that position (lists from tidal_select_attn are ascending) is
 * left as it is, so the token never counts twice. tidal_sparse_attn then needs idx_count. */
tidal_status_t tidal_set_attend_newest(tidal_ctx_t *ctx, int32_t enabled);

/* Output type of every later call on this context: TIDAL_OUT_F32 (default; `out` arguments are
 * float*) or TIDAL_OUT_BF16 (the same `out` arguments then point to bf16 [batch, Hq, head_dim],
 * each value the fp32 result rounded to nearest even; out_host of tidal_decode_step_host likewise).
 * tidal_sparse_attn_noalloc always writes fp32. */
enum { TIDAL_OUT_F32 = 0, TIDAL_OUT_BF16 = 1 };
tidal_status_t tidal_set_output_dtype(tidal_ctx_t *ctx, int32_t dtype);

/* Step graphs. When `stream` is an ordinary stream (not the legacy or per-thread default, and not
 * being captured by the caller), tidal_decode_step and tidal_decode_step_host record their launches
 * once as a CUDA graph and replay it for as long as every argument (schedule, descriptors, pointers,
 * k, granularity) stays byte-for-byte the same: lengths and page tables live in device memory and
 * may change freely. Up to 16 recordings are kept per context. On by default; enabled = 0 turns it
 * off and frees the recordings. */
tidal_status_t tidal_set_graphs(tidal_ctx_t *ctx, int32_t enabled);

/* Optional candidate compaction inside a selection layer's attention kernel (off by default: on B200
 * it measured slower than ranking all scores from the fused histogram, about 122 against 104
 * microseconds per selection layer at 128K context; it is kept as a tested alternative). Applies to one sequence, one token set per query head, groups of at
 * most four and k <= max_ctx_len / 6; other cases always rank all scores. With margin > 0, every CTA
 * of the attention kernel estimates, from the first few hundred scores it sees, a provisional
 * threshold that about margin * k / N of a head's scores should reach, and lists the scores at or
 * above it; the top-k then runs on that list alone. The result is exact whatever the margin: the list
 * is used only if it provably contains the k best (its k-th best score is not below the largest
 * threshold any CTA used); otherwise all scores are ranked by the same kernel, which is slower.
 * margin: 0 = off (default); 3 is a sensible value; values below 1 make the shortcut fail on purpose
 * (that is how the tests reach the exact fallback). */
tidal_status_t tidal_set_select_margin(tidal_ctx_t *ctx, float margin);

/* Overlap between the layers of a step (on by default). tidal_decode_step receives every layer's
 * query, lengths, page table and cache up front, so all of them are complete, in stream order, before
 * the call. With enabled != 0 a full-attention or sparse layer therefore streams its whole input while
 * the layer before it is still finishing and waits for that layer only before it writes scratch memory
 * and its output (a sparse layer right after a selection layer always waits first: the top-k writes its
 * index list). With enabled = 0 a layer only prefetches cache rows ahead of the previous layer's end and
 * reads its query afterwards, as a caller would need whose queries are produced between the layers.
 * With the overlap on, a selection layer with per-head sets and fp32 outputs (one sequence, or a batch over a
 * 16-bit cache)
 * also runs as two passes: keys first (logits, their histogram, the largest logit per head), then the
 * top-k on `stream` while the values are streamed on the context's second stream beside it and beside
 * the sparse layers that follow.
 * The single-layer calls always wait for all earlier work in the stream before reading anything. */
tidal_status_t tidal_set_layer_overlap(tidal_ctx_t *ctx, int32_t enabled);

/* The step of Algorithm 1 including its cache update: layer i's new key and value rows
 * (k_new_per_layer[i], v_new_per_layer[i]: device bf16 [batch, Hkv, head_dim], as for
 * tidal_kv_append) are written at position ctx_lens[b] - 1 of layer i's cache, then the layers
 * run as in tidal_decode_step. All layers' rows are written by one launch ahead of the first
 * layer, which is equivalent because every layer's inputs are given up front. The caches are
 * WRITTEN although the descriptors declare them const. */
tidal_status_t tidal_decode_step_append(tidal_ctx_t *ctx, int32_t num_layers, const uint8_t *schedule,
                                        const tidal_kv_t *kv_per_layer, const void *const *q_per_layer,
                                        const void *const *k_new_per_layer,
                                        const void *const *v_new_per_layer, float *const *out_per_layer,
                                        int32_t k, int32_t granularity, int32_t *idx,
                                        int32_t *idx_count, void *stream);

/* The same step for a caller whose queries and outputs live in HOST memory
 * (pinned for full speed): q_host is bf16 [num_layers, batch, Hq, head_dim],
 * out_host fp32 of the same shape. Runs tidal_decode_step with idx/idx_count in
 * the workspace and WAITS for the stream. Page-locked buffers are read and written
 * by the kernels directly over the bus (q_host 16-byte aligned); pageable ones are
 * copied to and from a staging area on the device. The KV cache stays resident on
 * the device. */
tidal_status_t tidal_decode_step_host(tidal_ctx_t *ctx, int32_t num_layers, const uint8_t *schedule,
                                      const tidal_kv_t *kv_per_layer, const void *q_host,
                                      float *out_host, int32_t k, int32_t granularity, void *stream);

/* tidal_sparse_attn for callers that are not allowed to allocate device memory. (The paper has
 * no counterpart to this call; it exists for integration, not for the method.) Such callers are,
 * for example, a serving process that handed all device memory to its own pool at start-up, so
 * that a later cudaMalloc fails or is forbidden by policy; code running inside a latency-critical
 * loop where the implicit synchronisation of cudaMalloc/cudaFree is unacceptable; or a plug-in
 * that is called with the device already in a state where allocation is not permitted. The other
 * entry points need a context whose workspace is allocated (and may grow) behind the caller's back.
 *
 * This one takes no context and never calls cudaMalloc, cudaFree or any allocating routine: its
 * scratch (split partial results, arrival counters, pool cursors) is one static device array of
 * about 2.06 MiB (4096 partial rows) that every GPU loading the library holds until the process
 * exits. It runs on the CURRENT device. Arguments and results are those of tidal_sparse_attn,
 * with these differences:
 *   - batch * num_q_heads must not exceed 4096, otherwise TIDAL_ERR_TOO_LARGE (nothing enqueued);
 *   - an index entry >= ctx_lens[b] or a page id outside the pool is skipped but cannot be
 *     reported (there is no context to hold the status word);
 *   - all calls on a device share the one scratch array: two calls whose kernels can overlap on
 *     the GPU (different streams, no dependency) race; keep them on one stream or order them;
 *   - the first call on each device also does the one-time set-up (it resolves the array's device
 *     address and prepares the kernel, still without allocating): that first call should come
 *     before any stream capture. */
tidal_status_t tidal_sparse_attn_noalloc(const tidal_kv_t *kv, const void *q, const int32_t *idx,
                                         const int32_t *idx_count, int32_t k, int32_t num_index_heads,
                                         float *out, void *stream);

/* ---- Paged caches filled on the device ------------------------------------------------------------ */

/* Page tables and slot maps from request lengths, for a pool of pages of 16 positions. Every sequence goes from old_lens[b]
 * to new_lens[b] cached tokens (device int32 [batch], batch <= 4096, each in 0 .. 16 * max_pages_per_seq <= 262144): one
 * that grows takes pages, one that shrinks (new_lens[b] = 0: it has ended) gives its last ones back.
 *   free_pages     device int32 [num_pages], a stack of free page ids whose first *num_free entries count. The pages given
 *                  back are pushed in the order (sequence, logical page), then the growing sequences pop theirs in
 *                  the same order, so a page given back can be taken again in the same call. A page must not be
 *                  shared by two sequences when one of them gives it back.
 *   num_free       device int32, read; num_free_out, device int32, receives the new count (may be the same word).
 *   page_table     device int32 [batch, max_pages_per_seq]: entries P(old) .. P(new) - 1 of growing sequences are written
 *                  (P(x) = ceil(x / 16)), no others.
 *   slots          device int64 [max_tokens]: the new tokens of all sequences one after the other (sequence b's positions
 *                  old_lens[b] .. new_lens[b] - 1), token at position p of sequence b at slot page * 16 + p % 16;
 *                  entries behind the last token are -1, so that a write of max_tokens rows skips them.
 *   positions      device int32 [max_tokens] or NULL: p of every token, -1 behind the last.
 *   token_offsets  device int32 [batch + 1] or NULL: where each sequence's tokens start in slots; the total last.
 * A request that cannot be met as a whole (a length out of range, more than max_tokens tokens, more pages than are free,
 * *num_free outside 0 .. num_pages, a page id given back that is outside the pool, a stack that would pass num_pages)
 * changes neither page_table nor free_pages: num_free_out receives *num_free, every slot and position is -1, every offset
 * 0, and tidal_device_status reports TIDAL_ERR_PAGES. A page id outside the pool in a table or on the stack
 * gives its tokens slot -1 and reports TIDAL_ERR_INDEX. No arrays may overlap (but the two counts). */
tidal_status_t tidal_page_map(tidal_ctx_t *ctx, int32_t batch, const int32_t *old_lens, const int32_t *new_lens,
                              int32_t *page_table, int32_t max_pages_per_seq, int32_t num_pages, int32_t *free_pages,
                              const int32_t *num_free, int32_t *num_free_out, int32_t max_tokens, int64_t *slots,
                              int32_t *positions, int32_t *token_offsets, void *stream);

/* The rows of num_tokens tokens into one layer's cache, through a slot map: k_new, v_new device bf16, token t's rows
 * [num_kv_heads, head_dim] contiguous at t * k_stride / t * v_stride elements (multiples of 8; the bases 16-byte aligned),
 * so they may be slices of a fused projection's output. slots: device int64 [num_tokens]; paged caches: page * 16 + place
 * (tidal_page_map), contiguous ones: sequence * max_ctx_len + position. -1 is skipped; any other slot outside
 * the cache is skipped and reported as TIDAL_ERR_INDEX. If a slot is named twice, what it then holds is
 * not specified: pieces of both tokens' rows are possible. An FP8 cache receives E4M3 codes: x / k_scale[g] (fp32 quotient; v_scale for values) rounded to
 * the nearest code, ties to even, saturated at +-448, NaN kept. The cache is WRITTEN although the descriptor declares it
 * const; ctx_lens and page_table are not read. */
tidal_status_t tidal_kv_write(tidal_ctx_t *ctx, const tidal_kv_t *kv, int32_t num_tokens, const void *k_new, const void *v_new,
                              int64_t k_stride, int64_t v_stride, const int64_t *slots, void *stream);

/* ---- Block-sparse attention --------------------------------------------------------------------------
 * A coarser and cheaper selection than tidal_select_attn: blocks of 16 consecutive positions (one page) are
 * ranked by an upper bound of their logits, computed from 512 bytes per block and KV head instead of the
 * block's keys, and attention reads the chosen blocks whole. Sequences of length 0 are allowed here: they choose no
 * block and their output is zero. */

/* Key bounds of blocks: for block i of sequence b and KV head g the channelwise least and greatest key over the cached
 * positions of the block (positions at and beyond ctx_lens[b] do not count), as bf16 (exact; for an FP8 cache
 * of the codes' values without the scale), NaN where a key is NaN. A page that several sequences share must be full in
 * all of them.
 *   bounds  device bf16, 16-byte aligned; contiguous caches [batch, num_kv_heads, bound_blocks, 2, head_dim] with
 *           bound_blocks >= ceil(max_ctx_len / 16), paged ones one entry per physical page,
 *           [bound_blocks, num_kv_heads, 2, head_dim] with bound_blocks >= num_pages; least keys first.
 *   start_lens  device int32 [batch] or NULL: only blocks from start_lens[b] / 16 on are computed (the tokens before
 *           start_lens[b] were there at the last call), for a sequence that has become shorter from ctx_lens[b] / 16 on; NULL: all
 *           of them. Other blocks keep their bounds.
 *   max_new host upper bound of ctx_lens[b] - start_lens[b], which sizes the launch (tokens beyond it may be left out);
 *           0: not known. */
tidal_status_t tidal_block_bounds(tidal_ctx_t *ctx, const tidal_kv_t *kv, const int32_t *start_lens, int32_t max_new,
                                  void *bounds, int32_t bound_blocks, void *stream);

/* The blocks to attend: per query head the score of a block is sum_c max(q_c lo_c, q_c hi_c), no less than q.k for
 * any key k of the block; an index head's score is the sum over its member heads (with SHARED over an FP8 cache
 * each KV head's part is multiplied by its k_scale, which must be positive). Chosen are the m' = min(m, ceil(ctx_lens[b] / 16))
 * best, equal scores resolved toward the lower block, after the first keep_first and the last keep_last blocks, which count as better than
 * any score (lower ones first if they are more than m). The set is the one that the scores in 64 bits give. Blocks
 * with bounds, and index heads with queries, that are not finite have an unspecified order.
 *   idx       int32 [batch, Hi, m]: block numbers in ascending order, padded with -1.
 *   idx_count int32 [batch] or NULL: receives m'.
 * m <= 16384. With max_ctx_len <= 16384 no scratch memory is used; beyond that it is the context's and may grow inside the
 * call unless `stream` is being captured (TIDAL_ERR_NOMEM then; tidal_reserve provides it). Graphs captured earlier stay
 * valid when it grows. */
tidal_status_t tidal_block_select(tidal_ctx_t *ctx, const tidal_kv_t *kv, const void *q, const void *bounds, int32_t bound_blocks,
                                  int32_t m, int32_t granularity, int32_t keep_first, int32_t keep_last, int32_t *idx,
                                  int32_t *idx_count, void *stream);

/* Attention over the listed blocks: Eq. 1 restricted to the cached positions of the blocks listed for the query head's
 * index head h * Hi / Hq, renormalised over them. -1 is padding; any other entry outside the sequence's blocks is skipped and
 * reported as TIDAL_ERR_INDEX; a repeated block counts once per occurrence; any order. Only the first idx_count[b]
 * entries count when idx_count is given, else m (at most 2^30). A head without a valid entry gets zeros. num_index_heads
 * must be Hq, Hkv or 1. Output type as set by tidal_set_output_dtype; softmax weights enter the product with V
 * with 22 bits or more, statistics and sums are fp32. tidal_set_attend_newest has no effect here (keep_last does that).
 * Uses no scratch memory. */
tidal_status_t tidal_block_attn(tidal_ctx_t *ctx, const tidal_kv_t *kv, const void *q, const int32_t *idx,
                                const int32_t *idx_count, int32_t m, int32_t num_index_heads, float *out, void *stream);

/* ---- Queries and keys of new tokens: norms and rotary positions ------------------------------------------------- */

/* How positions rotate the channels of a head, filled by tidal_rope_init and passed to the calls below by its address (read on the
 * host, inside the call). */
enum { TIDAL_ROPE_HALF = 0, TIDAL_ROPE_INTERLEAVED = 1 };   /* channel i turns with channel i + rotary_dim / 2, or 2 i with 2 i + 1 */
typedef struct {
    int32_t rotary_dim;      /* channels 0 .. rotary_dim - 1 turn, the others stay: 16, 32, .. 128 */
    int32_t layout;          /* TIDAL_ROPE_HALF or TIDAL_ROPE_INTERLEAVED */
    float scale;             /* factor on cosines and sines */
    int32_t reserved;
    uint64_t step[64];       /* turns per position of every pair of channels, in 2^-64 of a turn */
} tidal_rope_t;

/* Frequencies, on the host: inv_freq[i], i < rotary_dim / 2, in radians per position, and the factor on cosines and sines (1 but for
 * RAMP). With f_i = base^(-2 i / rotary_dim):
 *   PLAIN   f_i.   LINEAR  f_i / factor.   BASE  f_i of the base  base * factor^(rotary_dim / (rotary_dim - 2))
 *   BANDS   f_i / factor where a pair turns fewer than `low` times over trained_len positions, f_i where it turns more than
 *           `high` times, linear in the number of turns between: (1 - s) f_i / factor + s f_i, s = (turns - low) / (high - low)
 *   RAMP    r f_i / factor + (1 - r) f_i, r rising linearly from 0 to 1 over the channel numbers from floor(c(high)) to ceil(c(low)), with
 *           c(n) = rotary_dim ln(trained_len / (2 pi n)) / (2 ln base) the one that turns n times; factor on cosines and
 *           sines 0.1 ln(factor) + 1
 * factor >= 1; 0 < low < high and trained_len > 0 where they are used. */
enum { TIDAL_ROPE_PLAIN = 0, TIDAL_ROPE_LINEAR = 1, TIDAL_ROPE_BASE = 2, TIDAL_ROPE_BANDS = 3, TIDAL_ROPE_RAMP = 4 };
tidal_status_t tidal_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double low, double high,
                                      double trained_len, double *inv_freq, double *cos_scale);

/* Fills `rope` from frequencies (host double [rotary_dim / 2], tidal_rope_frequencies' or any others, finite). */
tidal_status_t tidal_rope_init(tidal_rope_t *rope, int32_t rotary_dim, int32_t layout, const double *inv_freq, double cos_scale);

/* Queries and keys of num_tokens tokens normed (optional) and rotated to their positions.
 *   q, k       device bf16, token t's rows [num_q_heads, 128] / [num_kv_heads, 128] contiguous at t * q_stride / t * k_stride elements
 *              (multiples of 8; bases 16-byte aligned); one of the two may be NULL with 0 heads.
 *   positions  device int32 [num_tokens]; a negative one (tidal_page_map's padding) leaves the token's rows unwritten.
 *   q_weight, k_weight  device bf16 [128], 16-byte aligned, or NULL: with a weight w a row x becomes
 *              x w / sqrt(mean(x^2) + eps) first, the mean over the head's 128 channels; with NULL it is not normed.
 *   q_out, k_out  like q and k with their own strides; may be q and k themselves (same stride), no other overlap.
 * Pair (a, b) at position p becomes (a c - b s, b c + a s), c, s = scale * cos, sin(p f). Angles are exact to 2^-32 of a turn at any
 * position; arithmetic is fp32, rounded once. */
tidal_status_t tidal_rope(tidal_ctx_t *ctx, const tidal_rope_t *rope, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                          const void *q, int64_t q_stride, const void *k, int64_t k_stride, const int32_t *positions,
                          const void *q_weight, const void *k_weight, float eps, void *q_out, int64_t q_out_stride, void *k_out,
                          int64_t k_out_stride, void *stream);

/* The same with the keys, and the tokens' values, written into a layer's cache through a slot map (as tidal_kv_write: -1 is skipped, any other slot
 * outside the cache skipped and reported as TIDAL_ERR_INDEX, a slot named twice unspecified; a token with a negative position is
 * skipped altogether). Heads are the descriptor's. An FP8 cache receives the codes nearest to key / k_scale[g], the key in fp32 and
 * rounded only there; values as tidal_kv_write quantises them. q may be NULL (then q_out too). The cache is WRITTEN although
 * the descriptor declares it const; ctx_lens and page_table are not read. */
tidal_status_t tidal_rope_write(tidal_ctx_t *ctx, const tidal_rope_t *rope, const tidal_kv_t *kv, int32_t num_tokens, const void *q,
                                int64_t q_stride, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride,
                                const int32_t *positions, const int64_t *slots, const void *q_weight, const void *k_weight, float eps,
                                void *q_out, int64_t q_out_stride, void *stream);

/* ---- Chunks of new tokens --------------------------------------------------------------------------------------- */

/* Attention of the last tokens of every sequence: sequence b's queries are rows q_offsets[b] .. q_offsets[b + 1] - 1 of q, its n newest
 * tokens in order, whose keys and values the cache holds already (ctx_lens counts them): row i is the token at position
 * p = ctx_lens[b] - n + i. It sees position j where j < ctx_lens[b], j <= p if causal != 0, and j > p - window if window > 0.
 *   q          device bf16, token t's rows [num_q_heads, 128] contiguous at t * q_stride elements (a multiple of 8; base 16-byte aligned)
 *   q_offsets  device int32 [batch + 1], ascending from 0 (or more: rows before the first are left as they were) to at most num_tokens (tidal_page_map's
 *              token_offsets); others are cut to that and reported as TIDAL_ERR_INDEX. Sequences may bring no token, one, or all they have.
 *   max_new    host upper bound of the new tokens of a sequence (tokens beyond it may be left out); 0: not known
 *   out        [num_tokens, num_q_heads, 128] contiguous, type as set by tidal_set_output_dtype; lse: float [num_tokens, num_q_heads] or NULL,
 *              ln of the sum of exp(scaled logit) over what the row sees. Rows behind q_offsets[batch] are left as they were.
 * A row that sees nothing (or nothing but pages that are skipped) gets zeros and -infinity. What lies behind a sequence in its last page or row block may be anything. Pages whose
 * id is outside the pool are skipped and reported (not those that lie before the first new token's window whole, which may be gone); a value that is not finite reaches the rows that see it and no other. k_scale must be positive. Softmax weights enter the product with V as
 * bf16 (FP8 caches: fp16, and the query as fp16 too); maxima, sums and outputs are fp32. Scratch memory is of one size and
 * allocated with the context. */
tidal_status_t tidal_chunk_attn(tidal_ctx_t *ctx, const tidal_kv_t *kv, int32_t num_tokens, const void *q, int64_t q_stride,
                                const int32_t *q_offsets, int32_t max_new, int32_t causal, int32_t window, float *out, float *lse,
                                void *stream);

/* The attention weight that every cached position receives from those queries:
 *   weights[b, h, j] = decay * weights[b, h, j] + sum over the queries that see j and the query heads of h of exp(logit - lse)
 * with lse as tidal_chunk_attn wrote it for the same arguments. num_weight_heads: num_kv_heads (a sum per KV head), or 1 (over all heads).
 *   weights  device float [batch, num_weight_heads, stride], stride >= max_ctx_len; entries j < ctx_lens[b] are written, the chunk's own
 *            positions as if their weight before had been 0 (so nothing need be cleared when a sequence has become shorter and
 *            grows again), and with decay 0 all of them.
 *   last     > 0: only the last so many queries of each chunk count
 * Offsets and pages as there. With num_tokens 0 nothing is done. The sum's order does not change from call to call. No scratch memory. */
tidal_status_t tidal_chunk_weights(tidal_ctx_t *ctx, const tidal_kv_t *kv, int32_t num_tokens, const void *q, int64_t q_stride,
                                   const int32_t *q_offsets, int32_t max_new, int32_t causal, int32_t window, int32_t last,
                                   const float *lse, float decay, float *weights, int64_t stride, int32_t num_weight_heads, void *stream);

/* ---- Eviction ----------------------------------------------------------------------------------------------------- */

/* The positions that stay: per sequence and weight head the m' = min(m, ctx_lens[b]) with the largest weights, equal ones (0 and -0 are equal)
 * resolved toward the lower position, not-a-numbers last, after the first keep_first and the last keep_last positions, which count as better than
 * any weight (lower ones first if they are more than m).
 *   kept      int32 [batch, num_weight_heads, m]: positions in ascending order, padded with -1
 *   new_lens  int32 [batch]: m'; not kv->ctx_lens
 * weights as above. Only the descriptor's lengths and shape are read. No scratch memory. */
tidal_status_t tidal_evict_select(tidal_ctx_t *ctx, const tidal_kv_t *kv, const float *weights, int64_t stride, int32_t num_weight_heads,
                                  int32_t m, int32_t keep_first, int32_t keep_last, int32_t *kept, int32_t *new_lens, void *stream);

/* Key and value rows of listed positions moved to the front, in the lists' order: row j of sequence b and KV head g becomes row
 * kept[b, h, j], j < counts[b] (at most m), h = g or 0. num_list_heads: num_kv_heads, or 1 for one list for all heads. Lists of
 * tidal_evict_select, or tidal_select_attn's idx of granularity PER_KVHEAD or SHARED.
 *   into      NULL: within the cache; lists are ascending then, and no page belongs to two sequences. Otherwise the descriptor of the cache
 *             that receives the rows (same heads and element type; its ctx_lens is not read), of which no row is one that the lists name.
 *   weights   NULL, or float [batch, num_list_heads, stride] moved along to weights_out [.., stride_out], stride >= kv->max_ctx_len and
 *             stride_out >= min(m, the receiving max_ctx_len); within the cache weights_out may be weights, otherwise not.
 * -1 is skipped, another position outside [0, ctx_lens[b]) skipped and reported as TIDAL_ERR_INDEX, a page id outside the pool likewise, and so are entries
 * of a list from the receiving max_ctx_len on (within the cache: from ctx_lens[b] on).
 * ctx_lens holds the lengths before; the caller then takes new_lens (tidal_page_map gives the pages back), and key
 * bounds are computed anew. The cache is WRITTEN although the descriptor declares it const. */
tidal_status_t tidal_kv_gather(tidal_ctx_t *ctx, const tidal_kv_t *kv, const tidal_kv_t *into, const int32_t *kept, const int32_t *counts,
                               int32_t m, int32_t num_list_heads, const float *weights, int64_t stride, float *weights_out,
                               int64_t stride_out, void *stream);

/* Waits for `stream`, then reports and clears one kind of what the device has noted since: TIDAL_ERR_INTERNAL before
 * TIDAL_ERR_TIMEOUT before TIDAL_ERR_PAGES before TIDAL_ERR_INDEX. What else was noted stays for the next call, so that TIDAL_OK says that nothing
 * is left. TIDAL_ERR_CUDA if the stream reports an error. */
tidal_status_t tidal_device_status(tidal_ctx_t *ctx, void *stream);

/* Kernels launched through this context since it was created. */
int64_t tidal_launch_count(const tidal_ctx_t *ctx);

const char *tidal_strerror(tidal_status_t status);

#ifdef __cplusplus
}
#endif
#endif
