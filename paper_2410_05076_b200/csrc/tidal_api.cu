// C-ABI of libtidal: argument checking, workspace, launch planning.
// Every step of the attention path runs in the kernels of attn_kernels.cuh and
// topk_kernels.cuh, the block-sparse and page calls in those of block_*.cuh and page_kernels.cuh;
// nothing here computes on the host and there is no CPU path.
#include "../../include/tidal.h"

#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <mutex>
#include <type_traits>
#include <vector>
#include <new>

#include "attn_kernels.cuh"
#include "block_attn_kernels.cuh"
#include "block_kernels.cuh"
#include "block_select_kernels.cuh"
#include "chunk_kernels.cuh"
#include "evict_kernels.cuh"
#include "page_kernels.cuh"
#include "rope_kernels.cuh"
#include "split_select_kernels.cuh"
#include "topk_kernels.cuh"
#include "weight_kernels.cuh"

using namespace tidal;

namespace {

constexpr int MAX_CTX = 262144;
constexpr int GRID_MAX = 320;            // persistent CTAs per launch never exceed this (2 per SM on 148 SMs)
constexpr int MIN_TILES_PER_CTA = 8;     // do not cut work finer than 128 positions per CTA
constexpr int MAX_GROUP = 8;            // query heads per KV head that fit the 8 MMA columns

// Streaming (full / selection) and gather (sparse) launch shapes.
constexpr int DENSE_NW = 8, DENSE_STAGES = 3;
constexpr int SPARSE_NW = 4, SPARSE_STAGES = 3;
// 8-bit caches: ring slots are half as large, so twice as many keep the same bytes in flight.
constexpr int DENSE_STAGES8 = 4, SPARSE_STAGES8 = 4;
constexpr int SPARSE_NW8 = 6;
constexpr int DENSE_NW8 = 12;
constexpr size_t HIST_SMEM = HIST_SMEM_WORDS * sizeof(uint32_t);

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }


}  // namespace

struct tidal_ctx {
    int device = 0;
    int sm_count = 0;
    int dense_slots = 0, sparse_slots = 0;     // resident CTAs on the whole GPU
    void* ws = nullptr;                         // scratch: contents are garbage between calls
    size_t ws_bytes = 0;
    // Words that must read zero when a kernel starts (split counters, top-k cursors, arrival
    // counters and histograms). The kernels restore the zeros themselves, so this lives apart
    // from the scratch workspace, whose layout changes with the problem shape.
    void* state = nullptr;
    int state_rows = 0;                         // capacity in (sequence, head) rows
    int* status = nullptr;                      // device word, sticky
    // Scores of the block selection over long contexts. It grows by doubling; what it outgrows is kept until the context
    // goes if a call was captured with it, since the caller's graph then still names it, and given back otherwise.
    void* blk_ws = nullptr;
    size_t blk_ws_bytes = 0;
    bool blk_named = false;                     // a captured call uses blk_ws
    void* blk_old[64] = {};
    int blk_old_count = 0;
    int out_bf16 = 0;                           // outputs are written as bf16 instead of fp32
    int attend_newest = 0;                      // sparse layers also attend the newest token (not in the paper)
    int cursor_set = 0;                         // which of the sets of pool cursors the last attention launch used
    float select_margin = 0.f;                  // > 0: selection layers compact candidates above a provisional threshold aimed at this multiple of k'/N
    // Split selection layers run their value pass on a stream of the context's own, beside the top-k and
    // the sparse layers that follow on the caller's stream; two events fork and join the streams.
    cudaStream_t side = nullptr;
    cudaEvent_t ev_fork = nullptr, ev_join = nullptr;
    int split_select = 1;
    int layer_overlap = 1;                      // layers of a step may stream their inputs while the layer before them finishes
    int select_clusters[17] = {};               // clusters of 1 .. 16 CTAs that are resident together: block selection
    int attn_clusters[17] = {};                 // the same for four-warp CTAs of the block attention
    void* tok_ws = nullptr;                     // chunk attention of single tokens: partial results, counters and cursors (zero between launches)
    int chunk_clusters[2][17] = {};             // and for the chunk attention (16-bit, 8-bit caches)
    int evict_clusters[17] = {};                // and for the eviction's choice
    int64_t launches = 0;
    // Whole steps are recorded once as CUDA graphs (programmatic dependent launches included) and
    // replayed while every host-visible argument stays the same: one launch per step instead of one
    // per kernel. Keyed by the bytes of all arguments plus the workspace addresses they bake in.
    struct StepGraph {
        std::vector<unsigned char> key;
        cudaGraphExec_t exec = nullptr;
        int launches = 0;
        uint64_t last_use = 0;
    };
    std::vector<StepGraph> graphs;
    uint64_t graph_clock = 0;
    bool graphs_enabled = true;
    // The call before this one, byte for byte (arguments, the arrays they point to, the settings and the
    // workspace addresses): a step loop repeats it, and then validation, layout and key building are skipped.
    struct LastCall {
        std::vector<unsigned char> raw;
        cudaGraphExec_t exec = nullptr;
        int launches = 0;
    } last;
    std::vector<unsigned char> raw_scratch;
    cudaGraphExec_t ran_exec = nullptr;         // set by run_graphed: the graph it launched, if any
    int ran_launches = 0;
};

namespace {

struct WsLayout {
    size_t part_ml, part_o, scores, cand, bitmap, idx, idx_count, q_stage, out_stage, total;
    long long cand_stride, bitmap_stride;
    long long score_stride;
    int max_splits;
};

// Partial-result slots a (sequence, head) row can need: the CTAs of one launch are at most
// GRID_MAX, and an item of `tiles_max` tiles is cut into at most tiles/per_cta + 2 pieces where
// per_cta >= (one tile per item) * items / GRID_MAX.
int max_splits_for(const tidal_kv_t* kv) {
    const long long items = (long long)kv->batch * kv->num_kv_heads;
    const long long tiles_max = (kv->max_ctx_len + TILE - 1) / TILE;
    const long long bound = tiles_max * GRID_MAX / std::max(items, 1LL) + 2;
    return (int)std::max(1LL, std::min<long long>(GRID_MAX, bound));
}

// Persistent grid: every resident slot gets an equal share of the tiles, but no CTA is
// launched for fewer than MIN_TILES_PER_CTA tiles.
int grid_for(long long tiles_upper_bound, int slots) {
    const long long by_work = std::max(1LL, tiles_upper_bound / MIN_TILES_PER_CTA);
    return (int)std::max(1LL, std::min<long long>(std::min(slots, GRID_MAX), by_work));
}

// 2048 histogram bins per head while the group's columns fit the shared histogram, else 1024.
int hist_shift_for(const tidal_kv_t* kv) { return (kv->num_q_heads / kv->num_kv_heads) <= 4 ? 21 : 22; }

// One sequence: all items have the same length, so whole groups of CTAs can share an item's tiles.
int pooled_splits(const tidal_kv_t* kv, int items, int grid) {
    if (kv->batch != 1) return 0;
    const int S = grid / std::max(items, 1);
    return S >= 2 ? S : 0;
}

int hi_of(const tidal_kv_t* kv, int granularity) {
    switch (granularity) {
        case TIDAL_SEL_PER_QHEAD: return kv->num_q_heads;
        case TIDAL_SEL_PER_KVHEAD: return kv->num_kv_heads;
        case TIDAL_SEL_SHARED: return 1;
        default: return -1;
    }
}

tidal_status_t check_kv(const tidal_kv_t* kv) {
    if (!kv || !kv->k || !kv->v || !kv->ctx_lens) return TIDAL_ERR_INVALID;
    if (kv->batch <= 0 || kv->num_q_heads <= 0 || kv->num_kv_heads <= 0) return TIDAL_ERR_INVALID;
    if (kv->num_q_heads % kv->num_kv_heads != 0) return TIDAL_ERR_INVALID;
    if (kv->head_dim != HEAD_DIM) return TIDAL_ERR_UNSUPPORTED;
    if (kv->num_q_heads / kv->num_kv_heads > MAX_GROUP) return TIDAL_ERR_UNSUPPORTED;
    if (kv->max_ctx_len < 1 || kv->max_ctx_len > MAX_CTX) return TIDAL_ERR_INVALID;
    if (kv->batch > 65535 || kv->num_q_heads > 65535) return TIDAL_ERR_UNSUPPORTED;
    if ((long long)kv->batch * kv->num_q_heads > 262144) return TIDAL_ERR_UNSUPPORTED;   // split counters fit the zeroed head of the workspace
    if (((uintptr_t)kv->k | (uintptr_t)kv->v) & 15) return TIDAL_ERR_INVALID;
    if (kv->kv_dtype != TIDAL_KV_BF16 && kv->kv_dtype != TIDAL_KV_FP8_E4M3) return TIDAL_ERR_INVALID;
    // rows must start on 16-byte boundaries: 8 elements of 16 bits, 16 of 8 bits
    const int64_t align_mask = kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? 15 : 7;
    if ((kv->stride_pos | kv->stride_head | kv->stride_b | kv->stride_page) & align_mask) return TIDAL_ERR_INVALID;
    if (kv->kv_dtype == TIDAL_KV_FP8_E4M3 && ((((uintptr_t)kv->k_scale | (uintptr_t)kv->v_scale) & 3) != 0)) return TIDAL_ERR_INVALID;
    if ((kv->stride_pos | kv->stride_head) & 7) return TIDAL_ERR_INVALID;
    if (kv->stride_pos < 0 || kv->stride_head < 0 || kv->stride_b < 0 || kv->stride_page < 0) return TIDAL_ERR_INVALID;
    if (!(kv->sm_scale >= 0.f) || std::isinf(kv->sm_scale)) return TIDAL_ERR_INVALID;
    if (kv->kv_layout == TIDAL_KV_CONTIG) {
        if (kv->stride_b & 7) return TIDAL_ERR_INVALID;
        if (kv->stride_pos < HEAD_DIM && kv->max_ctx_len > 1) return TIDAL_ERR_INVALID;
    } else if (kv->kv_layout == TIDAL_KV_PAGED) {
        if (!kv->page_table) return TIDAL_ERR_INVALID;
        if (kv->page_size != TILE) return TIDAL_ERR_UNSUPPORTED;
        if (kv->stride_page & 7) return TIDAL_ERR_INVALID;
        if (kv->num_pages <= 0 || kv->max_pages_per_seq <= 0) return TIDAL_ERR_INVALID;
        if ((long long)kv->max_pages_per_seq * kv->page_size < kv->max_ctx_len) return TIDAL_ERR_INVALID;
    } else {
        return TIDAL_ERR_INVALID;
    }
    return TIDAL_OK;
}

// Workspace layout for a cache shape, budget k and (for the host-buffer step) layer count.
WsLayout layout_ws(const tidal_kv_t* kv, int k, int num_layers_host) {
    WsLayout w;
    const size_t rows = (size_t)kv->batch * kv->num_q_heads;
    size_t at = 0;
    w.max_splits = max_splits_for(kv);
    w.part_ml = at;   at += align_up(rows * w.max_splits * sizeof(float2), 256);
    w.part_o = at;    at += align_up(rows * w.max_splits * HEAD_DIM * sizeof(float), 256);
    w.score_stride = (long long)align_up((size_t)kv->max_ctx_len, 16);
    w.scores = at;    at += align_up(rows * (size_t)w.score_stride * sizeof(float), 256);
    w.cand_stride = w.score_stride;
    w.cand = at;      at += align_up(rows * (size_t)w.cand_stride * sizeof(uint2), 256);
    w.bitmap_stride = (long long)align_up((size_t)kv->max_ctx_len, TK_SPAN) / 32;
    w.bitmap = at;    at += align_up(rows * (size_t)w.bitmap_stride * sizeof(unsigned), 256);
    w.idx = at;       at += align_up(rows * (size_t)std::max(k, 1) * sizeof(int), 256);
    w.idx_count = at; at += align_up((size_t)kv->batch * sizeof(int), 256);
    w.q_stage = at;   at += align_up((size_t)num_layers_host * rows * HEAD_DIM * 2, 256);
    w.out_stage = at; at += align_up((size_t)num_layers_host * rows * HEAD_DIM * 4, 256);
    w.total = at;
    return w;
}

size_t ws_bytes_for(const tidal_kv_t* kv, int k, int num_layers_host) {
    return layout_ws(kv, k, num_layers_host).total;
}

void drop_graphs(tidal_ctx* ctx) {
    ctx->last.exec = nullptr;
    if (ctx->graphs.empty()) return;
    cudaDeviceSynchronize();
    for (auto& g : ctx->graphs) if (g.exec) cudaGraphExecDestroy(g.exec);
    ctx->graphs.clear();
}

tidal_status_t ensure_ws(tidal_ctx* ctx, size_t bytes) {
    if (ctx->ws_bytes >= bytes) return TIDAL_OK;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    drop_graphs(ctx);                           // they carry addresses inside the old workspace
    if (ctx->ws) { cudaDeviceSynchronize(); cudaFree(ctx->ws); ctx->ws = nullptr; ctx->ws_bytes = 0; }
    void* p = nullptr;
    if (cudaMalloc(&p, bytes) != cudaSuccess) { cudaGetLastError(); return TIDAL_ERR_NOMEM; }
    ctx->ws = p;
    ctx->ws_bytes = bytes;
    return TIDAL_OK;
}

// State layout for a capacity of R rows: counters | cursor | done | thr_max | side counters | side cursors |
// split max | split sum | tile_ctr sets, each
// [R][CTR_STRIDE], then hist[R][TK_BINS]. Consecutive attention launches rotate through the sets of
// pool cursors, so that a launch may use its set before its predecessor has finished with another.
// Every counter has a 128-byte line of its own: hundreds of warps hit them at once, and atomics to one
// line are served one after the other.
constexpr int CTR_STRIDE = 32;
constexpr int CURSOR_SETS = 6;
inline int* state_counters(const tidal_ctx* c) { return (int*)c->state; }
inline int* state_cursor(const tidal_ctx* c) { return (int*)c->state + (size_t)CTR_STRIDE * c->state_rows; }
inline int* state_done(const tidal_ctx* c) { return (int*)c->state + 2 * (size_t)CTR_STRIDE * c->state_rows; }
inline unsigned* state_thr_max(const tidal_ctx* c) { return (unsigned*)c->state + 3 * (size_t)CTR_STRIDE * c->state_rows; }
inline int* state_side_counters(const tidal_ctx* c) { return (int*)c->state + 4 * (size_t)CTR_STRIDE * c->state_rows; }
inline int* state_side_cursors(const tidal_ctx* c) { return (int*)c->state + 5 * (size_t)CTR_STRIDE * c->state_rows; }
inline unsigned* state_split_max(const tidal_ctx* c) { return (unsigned*)c->state + 6 * (size_t)CTR_STRIDE * c->state_rows; }
inline float* state_split_sum(const tidal_ctx* c) { return (float*)c->state + 7 * (size_t)CTR_STRIDE * c->state_rows; }
inline int* state_tile_ctr(const tidal_ctx* c) { return (int*)c->state + 8 * (size_t)CTR_STRIDE * c->state_rows; }
inline unsigned* state_hist(const tidal_ctx* c) { return (unsigned*)c->state + (8 + CURSOR_SETS) * (size_t)CTR_STRIDE * c->state_rows; }

tidal_status_t ensure_state(tidal_ctx* ctx, int rows) {
    if (ctx->state_rows >= rows) return TIDAL_OK;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    drop_graphs(ctx);
    if (ctx->state) { cudaDeviceSynchronize(); cudaFree(ctx->state); ctx->state = nullptr; ctx->state_rows = 0; }
    const int cap = (int)align_up((size_t)rows, 64);
    const size_t bytes = (size_t)cap * ((8 + CURSOR_SETS) * CTR_STRIDE + TK_BINS) * sizeof(int);
    void* p = nullptr;
    if (cudaMalloc(&p, bytes) != cudaSuccess) { cudaGetLastError(); return TIDAL_ERR_NOMEM; }
    // on a stream of its own, so that nothing here is the legacy stream's business, and waited for
    cudaStream_t zs = nullptr;
    bool zeroed = cudaStreamCreateWithFlags(&zs, cudaStreamNonBlocking) == cudaSuccess &&
                  cudaMemsetAsync(p, 0, bytes, zs) == cudaSuccess && cudaStreamSynchronize(zs) == cudaSuccess;
    if (zs) cudaStreamDestroy(zs);
    if (!zeroed) { cudaGetLastError(); cudaFree(p); return TIDAL_ERR_CUDA; }
    ctx->state = p;
    ctx->state_rows = cap;
    return TIDAL_OK;
}

tidal_status_t ensure_all(tidal_ctx* ctx, const tidal_kv_t* kv, size_t ws_bytes) {
    const tidal_status_t rc = ensure_state(ctx, kv->batch * kv->num_q_heads);
    return rc != TIDAL_OK ? rc : ensure_ws(ctx, ws_bytes);
}

void fill_common(AttnParams& a, const tidal_ctx* ctx, const tidal_kv_t* kv, const void* q, float* out,
                 const WsLayout& w) {
    std::memset(&a, 0, sizeof a);
    a.q = (const __nv_bfloat16*)q;
    a.k = (const __nv_bfloat16*)kv->k;
    a.v = (const __nv_bfloat16*)kv->v;
    a.out = out;
    a.out_bf16 = ctx->out_bf16;
    a.stride_b = kv->stride_b; a.stride_pos = kv->stride_pos; a.stride_head = kv->stride_head;
    a.stride_page = kv->stride_page;
    a.page_table = kv->page_table; a.max_pages = kv->max_pages_per_seq; a.num_pages = kv->num_pages;
    a.paged = kv->kv_layout == TIDAL_KV_PAGED;
    a.ctx_lens = kv->ctx_lens;
    a.max_ctx = kv->max_ctx_len;
    a.Hq = kv->num_q_heads; a.Hkv = kv->num_kv_heads; a.G = a.Hq / a.Hkv;
    a.scale = kv->sm_scale > 0.f ? kv->sm_scale : 1.0f / std::sqrt((float)kv->head_dim);
    a.scale_log2 = a.scale * 1.4426950408889634f;
    if (kv->kv_dtype == TIDAL_KV_FP8_E4M3) { a.k_scale = kv->k_scale; a.v_scale = kv->v_scale; }
    char* ws = (char*)ctx->ws;
    a.counters = state_counters(ctx);
    a.part_ml = (float2*)(ws + w.part_ml);
    a.part_o = (float*)(ws + w.part_o);
    a.max_splits = w.max_splits;
    a.batch = kv->batch;
    a.tile_ctr = state_tile_ctr(ctx);
    a.ctr_stride = CTR_STRIDE;
    a.hist_shift = hist_shift_for(kv);
    a.status = ctx->status;
}

template <int MODE, int NW, int STAGES, bool KV8 = false>
constexpr size_t attn_smem() {
    return (size_t)NW * STAGES * (KV8 ? STAGE_BYTES8 : STAGE_BYTES) +
           (MODE == MODE_SELECT ? HIST_SMEM : 0) + 1024;   // + alignment slack
}

template <int MODE, int NW, int STAGES, bool NEWEST = false, bool COMPACT = false, bool KV8 = false>
tidal_status_t launch_attn(tidal_ctx* ctx, AttnParams& a, int grid, int full_grid, cudaStream_t st) {
    // Programmatic dependent launch: the kernel may begin while its predecessor in the stream
    // drains; it waits (griddepcontrol.wait) before touching anything that predecessor wrote.
    a.pdl = 1;
    ctx->cursor_set = (ctx->cursor_set + 1) % CURSOR_SETS;
    a.tile_ctr = state_tile_ctr(ctx) + (size_t)ctx->cursor_set * CTR_STRIDE * ctx->state_rows;
    // A kernel that waits late triggers its successor at once, before it has itself waited for its
    // predecessor, so several consecutive launches can be resident together. The one thing a kernel
    // touches before its own wait is its set of pool cursors, last used CURSOR_SETS launches ago by a
    // kernel that must have finished with it. It has: the launches in between either waited before they
    // triggered (then stream order guarantees it), or each of them holds all its CTAs until its own
    // predecessor is complete and (CURSOR_SETS - 1) of them fill every resident slot of the GPU, so this
    // launch cannot have started while a CTA of that old kernel was still resident. Hence the rule:
    // early trigger only for pooled launches (every CTA stays until the wait) whose grid is at least
    // 1 / (CURSOR_SETS - 1) of the resident slots for this kernel's CTA size.
    a.trigger_early = a.wait_late && (long long)(CURSOR_SETS - 1) * grid >= full_grid;
    if (!a.trigger_early) a.wait_late = 0;      // without the early trigger the late wait only delays the successor
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(NW * 32, 1, 1);
    cfg.dynamicSmemBytes = attn_smem<MODE, NW, STAGES, KV8>();
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ctx->launches++;
    return cudaLaunchKernelEx(&cfg, attn_kernel<MODE, NW, STAGES, NEWEST, COMPACT, KV8>, a) == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}

// How a selection layer produces its ranking scores. Per query head: one row per head, histogram
// fused. Fewer index heads than query heads: the ranking score is the sum of the member heads'
// scaled logits; unless the caller wants the per-head scores, the attention kernel stores the
// group sums directly (one row per KV head; histogram fused when a set belongs to one KV head).
// With one sequence, one set per query head and enough scores per set, the attention kernel compacts
// candidates instead (no histogram) and a single CTA per head finishes the selection on them.
struct SelectPlan { bool agg, fuse, compact, split; int rows; };
constexpr int SCORE_NW = 16, SCORE_STAGES = 3;     // key rows only, 4 KB per tile: sixteen warps keep enough tiles in flight
constexpr int VALUE_NW = 8, VALUE_STAGES = 3;      // value rows + logits, 4.5 KB per tile: two CTAs per SM, also beside a sparse layer's CTA
constexpr size_t SCORE_SMEM = (size_t)SCORE_NW * SCORE_STAGES * TILE_BYTES + HIST_SMEM + 1024;
constexpr size_t VALUE_SMEM = (size_t)VALUE_NW * VALUE_STAGES * (TILE_BYTES + 512) + 1024;
constexpr int VALUE_NW8 = 7;                        // 8-bit caches: 32 positions (4 KB of codes + 1 KB of logits) per slot
constexpr size_t VALUE_SMEM8 = (size_t)VALUE_NW8 * VALUE_STAGES * (UNIT8_BYTES + 1024) + 1024;
constexpr int COMPACT_LIST_SMEM = 12288;      // candidates the compacting top-k keeps in shared memory

int dense_grid(const tidal_ctx* ctx, const tidal_kv_t* kv) {
    const long long tiles = (long long)kv->batch * kv->num_kv_heads * ((kv->max_ctx_len + TILE - 1) / TILE);
    return grid_for(tiles, ctx->dense_slots);
}

SelectPlan select_plan(const tidal_ctx* ctx, const tidal_kv_t* kv, int Hi, int k, bool caller_scores) {
    SelectPlan s;
    s.agg = Hi != kv->num_q_heads && !caller_scores;
    s.rows = s.agg ? kv->num_kv_heads : kv->num_q_heads;
    s.fuse = Hi == s.rows;
    s.compact = ctx->select_margin > 0.f && kv->kv_dtype == TIDAL_KV_BF16 && Hi == kv->num_q_heads && kv->batch == 1 &&
                kv->num_q_heads / kv->num_kv_heads <= CAND_COLS && 6LL * k <= kv->max_ctx_len &&
                pooled_splits(kv, kv->num_kv_heads, dense_grid(ctx, kv)) > 0;
    if (s.compact) s.fuse = false;
    s.split = false;
    return s;
}

// Inside a step a selection layer can run as two passes (split_select_kernels.cuh) when it has one
// sequence (or a batch over a 16-bit cache), per-head scores with the fused histogram and fp32 outputs.
bool can_split(const tidal_ctx* ctx, const tidal_kv_t* kv, const SelectPlan& sp) {
    if (!(ctx->split_select && ctx->layer_overlap && !ctx->out_bf16 && !sp.agg && sp.fuse && !sp.compact)) return false;
    if (kv->batch == 1) return pooled_splits(kv, kv->num_kv_heads, dense_grid(ctx, kv)) > 0;
    return kv->kv_dtype == TIDAL_KV_BF16;       // batches: the flat-split passes (16-bit caches)
}

// hist != nullptr: the kernel also accumulates the per-head histogram the top-k needs.
// How a layer's kernel treats the kernel before it in the stream (see AttnParams::wait_first / wait_late).
enum Dep { DEP_FIRST, DEP_PREFETCH, DEP_LATE };
// Where a sparse layer sits in a run of consecutive sparse layers of a step (see run_sparse).
enum Chain { CHAIN_NONE, CHAIN_FIRST, CHAIN_MIDDLE, CHAIN_LAST };

tidal_status_t run_dense(tidal_ctx* ctx, const tidal_kv_t* kv, const void* q, float* out, float* scores,
                         long long score_stride, bool fuse_hist, Dep dep, const WsLayout& w, cudaStream_t st,
                         bool agg = false, int compact_k = 0, bool private_scores = false) {
    AttnParams a;
    fill_common(a, ctx, kv, q, out, w);
    a.wait_first = dep == DEP_FIRST;
    // A selection layer writes scores while it streams: it may do so ahead of its wait only when no earlier
    // kernel can still be reading the score buffer (the step driver knows), and not with candidate lists.
    a.wait_late = dep == DEP_LATE && (scores == nullptr || (private_scores && compact_k == 0));
    int grid = dense_grid(ctx, kv);
    if (compact_k > 0) {
        a.compact = 1;
        a.cand = (uint2*)((char*)ctx->ws + w.cand);
        a.cand_stride = w.cand_stride;
        a.cand_cursor = state_cursor(ctx);
        a.thr_max = state_thr_max(ctx);
        a.margin = ctx->select_margin;
        a.budget = compact_k;
    }
    if (const int S = pooled_splits(kv, kv->batch * kv->num_kv_heads, grid)) {
        a.splits_per_item = S;        // the grid keeps its size: some items get one CTA more than others
    }
    a.scores = scores;
    a.score_stride = score_stride;
    a.agg = agg ? 1 : 0;
    a.hist = fuse_hist ? state_hist(ctx) : nullptr;
    if (kv->kv_dtype == TIDAL_KV_FP8_E4M3) {
        const int full8 = std::min(ctx->dense_slots, GRID_MAX);
        if (scores) return launch_attn<MODE_SELECT, DENSE_NW8, DENSE_STAGES8, false, false, true>(ctx, a, grid, full8, st);
        return launch_attn<MODE_FULL, DENSE_NW8, DENSE_STAGES8, false, false, true>(ctx, a, grid, full8, st);
    }
    if (scores && a.compact) {
        if (a.splits_per_item <= 0) return TIDAL_ERR_INTERNAL;      // select_plan admits pooled grids only
        return launch_attn<MODE_SELECT, DENSE_NW, DENSE_STAGES, false, true>(ctx, a, grid, std::min(ctx->dense_slots, GRID_MAX), st);
    }
    if (scores) return launch_attn<MODE_SELECT, DENSE_NW, DENSE_STAGES>(ctx, a, grid, std::min(ctx->dense_slots, GRID_MAX), st);
    return launch_attn<MODE_FULL, DENSE_NW, DENSE_STAGES>(ctx, a, grid, std::min(ctx->dense_slots, GRID_MAX), st);
}

// The context's second stream and the two events that fork and join it (created on first use).
tidal_status_t ensure_side_stream(tidal_ctx* ctx) {
    if (ctx->side) return TIDAL_OK;
    if (cudaStreamCreateWithFlags(&ctx->side, cudaStreamNonBlocking) != cudaSuccess ||
        cudaEventCreateWithFlags(&ctx->ev_fork, cudaEventDisableTiming) != cudaSuccess ||
        cudaEventCreateWithFlags(&ctx->ev_join, cudaEventDisableTiming) != cudaSuccess) {
        cudaGetLastError();
        return TIDAL_ERR_CUDA;
    }
    return TIDAL_OK;
}

// Pass 1 of a split selection layer on the caller's stream: logits, histogram, softmax statistics.
tidal_status_t run_score_pass(tidal_ctx* ctx, const tidal_kv_t* kv, const void* q, float* out, float* scores,
                              long long score_stride, Dep dep, bool scores_free, const WsLayout& w, cudaStream_t st) {
    AttnParams a;
    fill_common(a, ctx, kv, q, out, w);
    const int grid = dense_grid(ctx, kv);
    a.splits_per_item = kv->batch == 1 ? pooled_splits(kv, kv->num_kv_heads, grid) : 0;
    a.scores = scores;
    a.score_stride = score_stride;
    a.hist = state_hist(ctx);
    a.split_max = state_split_max(ctx);
    // the kernel writes scores while it streams: ahead of its wait only if nobody can still be reading them
    a.wait_first = !(dep == DEP_LATE && scores_free);
    a.wait_late = !a.wait_first;
    a.pdl = 1;
    ctx->cursor_set = (ctx->cursor_set + 1) % CURSOR_SETS;
    a.tile_ctr = state_tile_ctr(ctx) + (size_t)ctx->cursor_set * CTR_STRIDE * ctx->state_rows;
    a.trigger_early = a.wait_late && (long long)(CURSOR_SETS - 1) * grid >= std::min(ctx->dense_slots, GRID_MAX);
    if (a.wait_late && !a.trigger_early) { a.wait_late = 0; a.wait_first = 1; }
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(SCORE_NW * 32, 1, 1);
    cfg.dynamicSmemBytes = SCORE_SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    ctx->launches++;
    const bool rowc = kv->stride_pos == 2 * HEAD_DIM;     // K and V rows interleaved: constant offsets between the rows of a tile
    cudaError_t e;
    if (kv->batch > 1)
        e = rowc ? cudaLaunchKernelEx(&cfg, score_pass_flat_kernel<SCORE_NW, SCORE_STAGES, true>, a)
                 : cudaLaunchKernelEx(&cfg, score_pass_flat_kernel<SCORE_NW, SCORE_STAGES, false>, a);
    else if (kv->kv_dtype == TIDAL_KV_FP8_E4M3)
        e = rowc ? cudaLaunchKernelEx(&cfg, score_pass8_kernel<SCORE_NW, SCORE_STAGES, true>, a)
                 : cudaLaunchKernelEx(&cfg, score_pass8_kernel<SCORE_NW, SCORE_STAGES, false>, a);
    else
        e = rowc ? cudaLaunchKernelEx(&cfg, score_pass_kernel<SCORE_NW, SCORE_STAGES, true>, a)
                 : cudaLaunchKernelEx(&cfg, score_pass_kernel<SCORE_NW, SCORE_STAGES, false>, a);
    return e == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}

// Pass 2 on the context's second stream: it starts when pass 1 is complete and runs beside whatever
// the caller's stream does next. It owns a cursor and a counter array of its own and no other scratch.
tidal_status_t run_value_pass(tidal_ctx* ctx, const tidal_kv_t* kv, float* out, float* out_final, const float* scores,
                              long long score_stride, const WsLayout& w, cudaStream_t st) {
    AttnParams a;
    fill_common(a, ctx, kv, nullptr, out, w);
    a.out_final = out_final;
    a.scores = const_cast<float*>(scores);
    a.score_stride = score_stride;
    a.split_max = state_split_max(ctx);
    a.split_sum = state_split_sum(ctx);
    a.counters = state_side_counters(ctx);
    a.tile_ctr = state_side_cursors(ctx);
    a.pdl = 0;
    // most of the slots (its CTAs are the size of the sparse layers'): it shares the GPU with the top-k and the
    // first sparse layers; between 25 % and 100 % of the slots the step time moved by less than 2 %
    const int per_item = std::max(2, 85 * std::min(ctx->sparse_slots, GRID_MAX) / (100 * kv->num_kv_heads));
    const int grid = kv->batch == 1 ? per_item * kv->num_kv_heads : std::min(ctx->sparse_slots, GRID_MAX);
    a.splits_per_item = kv->batch == 1 ? per_item : 0;
    if (cudaEventRecord(ctx->ev_fork, st) != cudaSuccess || cudaStreamWaitEvent(ctx->side, ctx->ev_fork, 0) != cudaSuccess)
        return TIDAL_ERR_CUDA;
    const bool rowc = kv->stride_pos == 2 * HEAD_DIM;
    if (kv->batch > 1) {
        if (rowc) value_pass_flat_kernel<VALUE_NW, VALUE_STAGES, true><<<grid, VALUE_NW * 32, VALUE_SMEM, ctx->side>>>(a);
        else value_pass_flat_kernel<VALUE_NW, VALUE_STAGES, false><<<grid, VALUE_NW * 32, VALUE_SMEM, ctx->side>>>(a);
    } else if (kv->kv_dtype == TIDAL_KV_FP8_E4M3) {
        if (rowc) value_pass8_kernel<VALUE_NW8, VALUE_STAGES, true><<<grid, VALUE_NW8 * 32, VALUE_SMEM8, ctx->side>>>(a);
        else value_pass8_kernel<VALUE_NW8, VALUE_STAGES, false><<<grid, VALUE_NW8 * 32, VALUE_SMEM8, ctx->side>>>(a);
    } else if (rowc) value_pass_kernel<VALUE_NW, VALUE_STAGES, true><<<grid, VALUE_NW * 32, VALUE_SMEM, ctx->side>>>(a);
    else value_pass_kernel<VALUE_NW, VALUE_STAGES, false><<<grid, VALUE_NW * 32, VALUE_SMEM, ctx->side>>>(a);
    ctx->launches++;
    if (cudaGetLastError() != cudaSuccess) return TIDAL_ERR_CUDA;
    return cudaEventRecord(ctx->ev_join, ctx->side) == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}

// `rows`: score rows per sequence (query heads, or KV heads when the attention kernel stored group sums).
tidal_status_t run_topk(tidal_ctx* ctx, const tidal_kv_t* kv, const float* scores, long long score_stride,
                        int k, int rows, int Hi, bool hist_done, int* idx, int* idx_count, const WsLayout& w,
                        cudaStream_t st, bool compact = false) {
    TopkParams t;
    std::memset(&t, 0, sizeof t);
    t.scores = scores; t.score_stride = score_stride;
    t.ctx_lens = kv->ctx_lens; t.max_ctx = kv->max_ctx_len;
    t.Hq = rows; t.Hi = Hi; t.k = k;
    t.idx = idx; t.idx_count = idx_count;
    char* ws = (char*)ctx->ws;
    t.hist = state_hist(ctx);
    t.cursor = state_cursor(ctx);
    t.ctr_stride = CTR_STRIDE;
    t.done = state_done(ctx);
    t.cand = (uint2*)(ws + w.cand);
    t.cand_stride = w.cand_stride;
    t.bitmap = (unsigned*)(ws + w.bitmap);
    t.bitmap_stride = w.bitmap_stride;
    const int items = kv->batch * Hi;
    if (items > 65535) return TIDAL_ERR_UNSUPPORTED;
    const int parts = (kv->max_ctx_len + TK_SLICE - 1) / TK_SLICE;        // histogram kernel
    const int sel_parts = (kv->max_ctx_len + TK_SPAN - 1) / TK_SPAN;     // select kernel
    t.shift = hist_shift_for(kv);
    t.vec_ok = (((uintptr_t)scores & 15) == 0 && (score_stride & 3) == 0) ? 1 : 0;
    // Candidates the last CTA of a head can hold in shared memory (a threshold bin's population is about
    // 2000 of 131072 scores; larger lists are read from global memory). With more CTAs than fit the GPU at
    // once (batches), the buffer is cut to what fits beside the bitmaps in the 64 KB the score staging needs
    // anyway, so that three CTAs share an SM instead of two.
    const size_t words = (size_t)(kv->max_ctx_len + 31) / 32;
    t.cand_smem = 8192;
    {
        const long long ctas = (long long)((kv->max_ctx_len + TK_SPAN - 1) / TK_SPAN) * kv->batch * Hi;
        const size_t staging = (size_t)TK_SPAN * sizeof(float), bitmaps = 2 * words * sizeof(unsigned);
        if (ctas > 2LL * ctx->sm_count && bitmaps + 2048 * sizeof(uint2) <= staging)
            t.cand_smem = (int)((staging - bitmaps) / sizeof(uint2));
    }
    // the last CTA's bitmaps and candidate buffer, or every CTA's score staging area, whichever is larger
    size_t smem = std::max(2 * words * sizeof(unsigned) + (size_t)t.cand_smem * sizeof(uint2),
                           (size_t)TK_SPAN * sizeof(float));
    if (kv->max_ctx_len <= TK_SPAN) {
        // every row fits one CTA: staged scores, two bitmaps and 4096 candidates in shared memory
        t.solo_cand = 4096;
        smem = (size_t)TK_SPAN * sizeof(float) + 2 * (TK_SPAN / 32) * sizeof(unsigned) + (size_t)t.solo_cand * sizeof(uint2);
    }
    // Both kernels may become resident while the kernel before them drains (they wait for it first).
    t.pdl = 1;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.blockDim = dim3(TK_THREADS, 1, 1);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (compact) {
        t.thr_max = state_thr_max(ctx);
        t.list_smem = COMPACT_LIST_SMEM;
        const size_t bm_words = (size_t)(kv->max_ctx_len + 31) / 32;
        cfg.gridDim = dim3(items, 1, 1);
        cfg.dynamicSmemBytes = 2 * (bm_words + 1) * sizeof(unsigned) + (size_t)COMPACT_LIST_SMEM * sizeof(uint2);
        ctx->launches++;
        return cudaLaunchKernelEx(&cfg, topk_compact_kernel, t) == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
    }
    if (!hist_done) {
        cfg.gridDim = dim3(parts, items, 1);
        cfg.dynamicSmemBytes = 0;
        ctx->launches++;
        if (cudaLaunchKernelEx(&cfg, topk_hist_kernel, t) != cudaSuccess) return TIDAL_ERR_CUDA;
    }
    cfg.gridDim = dim3(sel_parts, items, 1);
    cfg.dynamicSmemBytes = smem;
    ctx->launches++;
    if (cudaLaunchKernelEx(&cfg, topk_select_kernel, t) != cudaSuccess) return TIDAL_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}

tidal_status_t run_sparse(tidal_ctx* ctx, const tidal_kv_t* kv, const void* q, const int* idx,
                          const int* idx_count, int k, int Hi, float* out, Dep dep, Chain chain, const WsLayout& w,
                          cudaStream_t st) {
    AttnParams a;
    fill_common(a, ctx, kv, q, out, w);
    a.wait_first = dep == DEP_FIRST;
    a.wait_late = dep == DEP_LATE;
    const int per_batch = (Hi == kv->num_q_heads) ? kv->num_q_heads : kv->num_kv_heads;
    const long long tiles = (long long)kv->batch * per_batch * ((k + TILE - 1) / TILE);
    const int full = std::min(ctx->sparse_slots, GRID_MAX);
    int grid = grid_for(tiles, ctx->sparse_slots);
    a.idx = idx; a.idx_count = idx_count; a.budget = k; a.Hi = Hi;
    // In a chain of sparse layers that overlap (late wait, early trigger) a launch takes about a third
    // of the resident slots, so that about three layers are in flight at any time, one behind the
    // other: while the CTAs of one layer start up (lengths, index entries, first rows: a chain of
    // dependent loads) or merge their results, the others keep the memory system busy. Every item gets
    // the same number of CTAs.
    // The first layer of a chain runs alone until its successors have joined it and gets about half
    // the slots; the last one, which nothing follows into the slots it frees, gets one CTA per item
    // more than a third (measured at cfg3: step 658 -> 645 us against a third everywhere).
    const int items = kv->batch * per_batch;
    if (chain != CHAIN_NONE) {
        // (a layer that gathers fewer bytes, an 8-bit cache or a small budget, still has the same start-up and
        // merge phases: four layers in flight below 48 MB per layer)
        const long long row_bytes = kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? 2 * ROW_BYTES8 : 4 * HEAD_DIM;
        const int depth = (long long)items * k * row_bytes < (48ll << 20) ? 4 : 3;
        const int third = std::max(1, (full + depth * items / 2) / (depth * items));
        const int S = chain == CHAIN_FIRST ? std::max(third, (full + items) / (2 * items))
                      : chain == CHAIN_LAST ? third + 1 : third;
        grid = std::min(grid, S * items);
    }
    if (const int S = pooled_splits(kv, items, grid)) {
        a.splits_per_item = S;
    }
    if (kv->kv_dtype == TIDAL_KV_FP8_E4M3) {
        if (ctx->attend_newest) return TIDAL_ERR_UNSUPPORTED;
        return launch_attn<MODE_SPARSE, SPARSE_NW8, SPARSE_STAGES8, false, false, true>(ctx, a, grid, std::min(ctx->sparse_slots, GRID_MAX), st);
    }
    if (ctx->attend_newest) return launch_attn<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES, true>(ctx, a, grid, std::min(ctx->sparse_slots, GRID_MAX), st);
    return launch_attn<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>(ctx, a, grid, std::min(ctx->sparse_slots, GRID_MAX), st);
}

template <typename K>
int resident_ctas(K kernel, int threads, size_t smem, int sm_count) {
    int per_sm = 0;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return -1;
    if (cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, kernel, threads, smem) != cudaSuccess) return -1;
    return per_sm * sm_count;
}

// ---- step graphs ------------------------------------------------------------------------------------
struct KeyBuilder {
    std::vector<unsigned char> bytes;
    template <typename T> void add(const T& v) {
        const unsigned char* p = reinterpret_cast<const unsigned char*>(&v);
        bytes.insert(bytes.end(), p, p + sizeof(T));
    }
    void add_raw(const void* p, size_t n) {
        const unsigned char* c = static_cast<const unsigned char*>(p);
        bytes.insert(bytes.end(), c, c + n);
    }
};

void step_key(KeyBuilder& kb, const tidal_ctx* ctx, int tag, int32_t num_layers, const uint8_t* schedule,
                     const tidal_kv_t* kvs, int32_t k, int32_t granularity, int host_layers) {
    kb.add(tag); kb.add(num_layers); kb.add(k); kb.add(granularity); kb.add(host_layers);
    kb.add(ctx->ws); kb.add(ctx->state); kb.add(ctx->out_bf16); kb.add(ctx->attend_newest); kb.add(ctx->layer_overlap); kb.add(ctx->select_margin); kb.add(ctx->split_select);
    kb.add_raw(schedule, (size_t)num_layers);
    for (int i = 0; i < num_layers; ++i) {
        // field by field: the struct has padding whose bytes are not the caller's to define
        const tidal_kv_t& v = kvs[i];
        kb.add(v.batch); kb.add(v.num_q_heads); kb.add(v.num_kv_heads); kb.add(v.head_dim); kb.add(v.kv_layout);
        kb.add(v.k); kb.add(v.v); kb.add(v.stride_b); kb.add(v.stride_pos); kb.add(v.stride_head); kb.add(v.stride_page);
        kb.add(v.page_table); kb.add(v.page_size); kb.add(v.max_pages_per_seq); kb.add(v.num_pages);
        kb.add(v.ctx_lens); kb.add(v.max_ctx_len); kb.add(v.sm_scale); kb.add(v.kv_dtype); kb.add(v.k_scale); kb.add(v.v_scale);
    }
}

// A stream can record a graph if it is a real stream (not the legacy or per-thread default) that is
// not already being captured by the caller.
bool graphable(const tidal_ctx* ctx, cudaStream_t st) {
    if (!ctx->graphs_enabled || st == nullptr || st == cudaStreamLegacy || st == cudaStreamPerThread) return false;
    cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &cs) != cudaSuccess) { cudaGetLastError(); return false; }
    return cs == cudaStreamCaptureStatusNone;
}

// Replays the recorded graph of `key`, or records one from `enqueue` (which must only launch work on
// `st`). Falls back to plain enqueueing when recording is not possible.
template <typename F>
tidal_status_t run_graphed(tidal_ctx* ctx, KeyBuilder& kb, cudaStream_t st, F&& enqueue) {
    constexpr size_t MAX_GRAPHS = 16;
    ctx->ran_exec = nullptr;
    if (!graphable(ctx, st)) return enqueue();
    ++ctx->graph_clock;
    for (auto& g : ctx->graphs) {
        if (g.key == kb.bytes) {
            g.last_use = ctx->graph_clock;
            if (cudaGraphLaunch(g.exec, st) != cudaSuccess) return TIDAL_ERR_CUDA;
            ctx->launches += g.launches;
            ctx->ran_exec = g.exec; ctx->ran_launches = g.launches;
            return TIDAL_OK;
        }
    }
    if (cudaStreamBeginCapture(st, cudaStreamCaptureModeThreadLocal) != cudaSuccess) { cudaGetLastError(); return enqueue(); }
    const int64_t before = ctx->launches;
    const tidal_status_t rc = enqueue();
    cudaGraph_t graph = nullptr;
    const cudaError_t end = cudaStreamEndCapture(st, &graph);
    const int recorded = (int)(ctx->launches - before);
    ctx->launches = before;                     // nothing has run yet
    if (rc != TIDAL_OK || end != cudaSuccess || !graph) {
        if (graph) cudaGraphDestroy(graph);
        cudaGetLastError();
        return rc != TIDAL_OK ? rc : enqueue();
    }
    cudaGraphExec_t exec = nullptr;
    const cudaError_t inst = cudaGraphInstantiate(&exec, graph, 0);
    cudaGraphDestroy(graph);
    if (inst != cudaSuccess || !exec) { cudaGetLastError(); return enqueue(); }
    if (ctx->graphs.size() >= MAX_GRAPHS) {     // forget the entry that has gone unused the longest
        size_t victim = 0;
        for (size_t i = 1; i < ctx->graphs.size(); ++i)
            if (ctx->graphs[i].last_use < ctx->graphs[victim].last_use) victim = i;
        if (ctx->last.exec == ctx->graphs[victim].exec) ctx->last.exec = nullptr;
        cudaGraphExecDestroy(ctx->graphs[victim].exec);   // deferred by the runtime while a launch is in flight
        ctx->graphs.erase(ctx->graphs.begin() + victim);
    }
    tidal_ctx::StepGraph g;
    g.key = std::move(kb.bytes);
    g.exec = exec;
    g.launches = recorded;
    g.last_use = ctx->graph_clock;
    ctx->graphs.push_back(std::move(g));
    if (cudaGraphLaunch(exec, st) != cudaSuccess) return TIDAL_ERR_CUDA;
    ctx->launches += recorded;
    ctx->ran_exec = exec; ctx->ran_launches = recorded;
    return TIDAL_OK;
}

// The bytes that decide what a step call does: compared with the previous call's before anything else.
void raw_call_key(std::vector<unsigned char>& r, const tidal_ctx* ctx, int tag, int32_t num_layers, const uint8_t* schedule,
                  const tidal_kv_t* kvs, const void* const* qs, float* const* outs, const void* p0, const void* p1,
                  int32_t k, int32_t granularity, cudaStream_t st) {
    struct Head {
        int tag; int32_t num_layers, k, granularity; cudaStream_t st; const void *p0, *p1, *ws, *state;
        int out_bf16, attend_newest, layer_overlap, split_select; float select_margin;
    } h;
    std::memset(&h, 0, sizeof h);
    h.tag = tag; h.num_layers = num_layers; h.k = k; h.granularity = granularity; h.st = st; h.p0 = p0; h.p1 = p1;
    h.ws = ctx->ws; h.state = ctx->state; h.out_bf16 = ctx->out_bf16; h.attend_newest = ctx->attend_newest;
    h.layer_overlap = ctx->layer_overlap; h.split_select = ctx->split_select; h.select_margin = ctx->select_margin;
    const size_t L = (size_t)num_layers;
    const size_t n_q = qs ? L * sizeof(void*) : 0, n_o = outs ? L * sizeof(void*) : 0;
    r.resize(sizeof h + L + L * sizeof(tidal_kv_t) + n_q + n_o);
    unsigned char* d = r.data();
    std::memcpy(d, &h, sizeof h); d += sizeof h;
    std::memcpy(d, schedule, L); d += L;
    std::memcpy(d, kvs, L * sizeof(tidal_kv_t)); d += L * sizeof(tidal_kv_t);
    if (n_q) { std::memcpy(d, qs, n_q); d += n_q; }
    if (n_o) std::memcpy(d, outs, n_o);
}

// Same call as the last one, which ran as a graph: launch that graph again.
bool replay_last(tidal_ctx* ctx, cudaStream_t st, tidal_status_t& rc) {
    if (!ctx->last.exec || ctx->raw_scratch != ctx->last.raw || !graphable(ctx, st)) return false;
    rc = cudaGraphLaunch(ctx->last.exec, st) == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
    if (rc == TIDAL_OK) ctx->launches += ctx->last.launches;
    return true;
}

void remember_last(tidal_ctx* ctx) {
    if (!ctx->ran_exec) { ctx->last.exec = nullptr; return; }
    ctx->last.raw = ctx->raw_scratch;
    ctx->last.exec = ctx->ran_exec;
    ctx->last.launches = ctx->ran_launches;
}

// ---- block-sparse operators --------------------------------------------------------------------------
// Scratch of a block selection over long contexts: score rows and their error bounds per chunk.
struct BlockWs {
    size_t scores, err, total;
    int npad, chunks;
};

BlockWs block_ws_layout(const tidal_kv_t* kv, int rows) {
    BlockWs w;
    const int blocks = (kv->max_ctx_len + TILE - 1) / TILE;
    w.npad = (int)align_up((size_t)blocks, 32);
    w.chunks = (blocks + SS_BLOCKS - 1) / SS_BLOCKS;
    w.scores = 0;
    w.err = align_up((size_t)kv->batch * rows * w.npad * sizeof(float), 256);
    w.total = w.err + align_up((size_t)kv->batch * rows * w.chunks * sizeof(float), 256);
    return w;
}

tidal_status_t ensure_block_ws(tidal_ctx* ctx, size_t bytes, const cudaStream_t* st) {
    if (st) {                                   // nothing may be allocated into a capture
        cudaStreamCaptureStatus cs = cudaStreamCaptureStatusNone;
        const bool known = cudaStreamIsCapturing(*st, &cs) == cudaSuccess;
        if (!known) cudaGetLastError();
        if (!known || cs != cudaStreamCaptureStatusNone) {
            if (ctx->blk_ws_bytes < bytes) return TIDAL_ERR_NOMEM;
            ctx->blk_named = true;
        }
    }
    if (ctx->blk_ws_bytes >= bytes) return TIDAL_OK;
    if (ctx->blk_named && ctx->blk_old_count == (int)(sizeof ctx->blk_old / sizeof ctx->blk_old[0])) return TIDAL_ERR_NOMEM;
    size_t want = std::max(bytes, 2 * ctx->blk_ws_bytes);
    void* p = nullptr;
    if (cudaMalloc(&p, want) != cudaSuccess) {
        cudaGetLastError();
        want = bytes;                           // twice as much is for the sake of later calls: this one can do without
        if (cudaMalloc(&p, want) != cudaSuccess) { cudaGetLastError(); return TIDAL_ERR_NOMEM; }
    }
    if (ctx->blk_named) {
        ctx->blk_old[ctx->blk_old_count++] = ctx->blk_ws;
    } else if (ctx->blk_ws) {
        cudaDeviceSynchronize();
        cudaFree(ctx->blk_ws);
    }
    ctx->blk_ws = p;
    ctx->blk_ws_bytes = want;
    ctx->blk_named = false;
    return TIDAL_OK;
}

// The context's device for the length of a call; the caller's own is current again afterwards.
struct DeviceScope {
    int before = -1;
    bool ok = false;
    explicit DeviceScope(int device) {
        if (cudaGetDevice(&before) != cudaSuccess) { before = -1; cudaGetLastError(); return; }
        ok = before == device || cudaSetDevice(device) == cudaSuccess;
        if (before == device) before = -1;
    }
    ~DeviceScope() { if (before >= 0) cudaSetDevice(before); }
};

constexpr int BA_SMEM_MAX = (int)ba_smem_most(8);

// How many clusters of 1 .. 16 CTAs of a kernel the GPU holds at once (the SMs of a processing cluster differ from chip to chip).
template <typename K>
void count_clusters(K kernel, int threads, size_t smem, int (&out)[17]) {
    for (int s = 1; s <= 16; ++s) {
        cudaLaunchConfig_t cfg;
        std::memset(&cfg, 0, sizeof cfg);
        cfg.gridDim = dim3(s, 1, 1);
        cfg.blockDim = dim3(threads, 1, 1);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = s; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&out[s], kernel, &cfg) != cudaSuccess) { cudaGetLastError(); out[s] = 0; }
    }
}

bool prepare_block_kernels() {
    auto wide = [](const void* k) {
        return cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess;
    };
    auto room = [](auto kernel, size_t bytes) {
        return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess;
    };
    auto select = [&](auto kernel, int blocks) {
        return wide((const void*)kernel) && room(kernel, sc_smem(blocks, MAX_GROUP, SB_MAX_CLUSTER * SC_WARPS));
    };
    auto attn = [&](auto kernel) { return wide((const void*)kernel) && room(kernel, BA_SMEM_MAX); };
    return select(block_select_kernel<2, false>, 64) && select(block_select_kernel<8, false>, 256) && select(block_select_kernel<0, false>, SC_MAX_BLOCKS) &&
           select(block_select_kernel<0, true>, SC_MAX_BLOCKS) && select(block_select_kernel<16, false>, 512) &&
           room(block_score_kernel, SS_SMEM) && room(block_rank_kernel<256, 4>, 4096 * 8) && room(block_rank_kernel<512, 4>, 8192 * 8) &&
           room(block_rank_kernel<1024, 4>, 16384 * 8) &&
           attn(block_attn_kernel<false, 8>) && attn(block_attn_kernel<true, 8>) && attn(block_attn_kernel<false, 4>) && attn(block_attn_kernel<true, 4>) &&
           attn(block_attn_kernel<false, 2>) && attn(block_attn_kernel<true, 2>) && attn(block_attn_kernel<false, 1>) && attn(block_attn_kernel<true, 1>) &&
           cudaFuncSetAttribute(page_map_kernel<PM_THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * (PM_MAX_BATCH + 1) * (int)sizeof(int)) == cudaSuccess;
}

void fill_block_cache(BlockCache& c, const tidal_ctx* ctx, const tidal_kv_t* kv, int bound_blocks) {
    std::memset(&c, 0, sizeof c);
    c.k = (const uint8_t*)kv->k; c.v = (const uint8_t*)kv->v;
    c.stride_b = kv->stride_b; c.stride_pos = kv->stride_pos; c.stride_head = kv->stride_head; c.stride_page = kv->stride_page;
    c.page_table = kv->page_table; c.max_pages = kv->max_pages_per_seq; c.num_pages = kv->num_pages;
    c.paged = kv->kv_layout == TIDAL_KV_PAGED;
    c.ctx_lens = kv->ctx_lens; c.max_ctx = kv->max_ctx_len;
    c.max_blocks = (kv->max_ctx_len + TILE - 1) / TILE;
    c.bound_blocks = bound_blocks;
    c.batch = kv->batch; c.Hq = kv->num_q_heads; c.Hkv = kv->num_kv_heads; c.G = c.Hq / c.Hkv;
    c.status = ctx->status;
}

// The bounds buffer must hold every block that the cache can name.
tidal_status_t check_bounds(const tidal_kv_t* kv, const void* bounds, int32_t bound_blocks) {
    if (!bounds || ((uintptr_t)bounds & 15)) return TIDAL_ERR_INVALID;
    const int need = kv->kv_layout == TIDAL_KV_PAGED ? kv->num_pages : (kv->max_ctx_len + TILE - 1) / TILE;
    return bound_blocks >= need ? TIDAL_OK : TIDAL_ERR_INVALID;
}

// Launch with programmatic stream serialization (the kernel waits first thing for the one before it) and, for cluster > 0,
// with thread-block clusters of that size.
template <typename P>
tidal_status_t launch_block(tidal_ctx* ctx, void (*kernel)(P), const P& p, int grid, int threads, size_t smem, int cluster,
                            cudaStream_t st) {
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    ctx->launches++;
    if (cudaLaunchKernelEx(&cfg, kernel, p) == cudaSuccess) return TIDAL_OK;
    cudaGetLastError();
    return TIDAL_ERR_CUDA;
}

// ---- chunks of new tokens ------------------------------------------------------------------------------
using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// The driver's encoder of tensor maps, found once (the library is not linked against the driver).
EncodeTiled encode_tiled() {
    static EncodeTiled found = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult how;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &how) != cudaSuccess ||
            how != cudaDriverEntryPointSuccess) { cudaGetLastError(); f = nullptr; }
        return (EncodeTiled)f;
    }();
    return found;
}

constexpr int64_t TMA_STRIDE_LIMIT = 1LL << 40;
static_assert(MAX_CTX <= CH_MAX_TILES * CH_TILE, "a bit per tile");

// A tensor map of `rank` dimensions, element strides from the second on; the innermost box is 128 bytes, swizzled.
bool tensor_map(CUtensorMap* map, bool bytes, const void* base, int rank, const uint64_t* dims, const int64_t* strides, const uint32_t* box) {
    EncodeTiled encode = encode_tiled();
    if (!encode) return false;
    cuuint64_t size[5], pitch[4];
    cuuint32_t block[5], one[5];
    for (int i = 0; i < rank; ++i) { size[i] = dims[i]; block[i] = box[i]; one[i] = 1; }
    for (int i = 1; i < rank; ++i) pitch[i - 1] = (cuuint64_t)strides[i - 1] * (bytes ? 1 : 2);
    return encode(map, bytes ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, rank, const_cast<void*>(base), size, pitch, block,
                  one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Maps of a cache's keys (or values): [page or sequence][head][position][channel], boxes of 64 channels (128 codes) by a page's or
// a tile's positions. A dimension without a stride has one element, whose coordinate is 0 (the multipliers).
template <typename P>
bool cache_maps(P& p, const tidal_kv_t* kv, CUtensorMap* k, CUtensorMap* v) {
    const bool fp8 = kv->kv_dtype == TIDAL_KV_FP8_E4M3, paged = kv->kv_layout == TIDAL_KV_PAGED;
    const int64_t outer = paged ? kv->stride_page : kv->stride_b;
    const int outer_mul = outer > 0, head_mul = kv->stride_head > 0;
    p.page_mul = p.batch_mul = outer_mul;
    p.head_mul = head_mul;
    const uint64_t dims[4] = {HEAD_DIM, (uint64_t)(paged ? TILE : kv->max_ctx_len), head_mul ? (uint64_t)kv->num_kv_heads : 1,
                              outer_mul ? (uint64_t)(paged ? kv->num_pages : kv->batch) : 1};
    const int64_t strides[3] = {kv->stride_pos > 0 ? kv->stride_pos : HEAD_DIM, head_mul ? kv->stride_head : HEAD_DIM, outer_mul ? outer : HEAD_DIM};
    const uint32_t box[4] = {fp8 ? 128u : 64u, (uint32_t)(paged ? TILE : CH_TILE), 1, 1};
    return tensor_map(k, fp8, kv->k, 4, dims, strides, box) && (!v || tensor_map(v, fp8, kv->v, 4, dims, strides, box));
}

bool query_map(CUtensorMap* map, const void* q, int num_tokens, int heads, int64_t stride, int group, int tokens) {
    const uint64_t dims[3] = {HEAD_DIM, (uint64_t)heads, (uint64_t)num_tokens};
    const int64_t strides[2] = {HEAD_DIM, num_tokens > 1 ? stride : (int64_t)heads * HEAD_DIM};
    const uint32_t box[3] = {64, (uint32_t)group, (uint32_t)tokens};
    return tensor_map(map, false, q, 3, dims, strides, box);
}

tidal_status_t check_chunk(const tidal_kv_t* kv, int32_t num_tokens, const void* q, int64_t q_stride, const int32_t* q_offsets, int32_t max_new,
                           int32_t window) {
    const tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (num_tokens < 0 || max_new < 0 || window < 0) return TIDAL_ERR_INVALID;
    if (num_tokens == 0) return TIDAL_OK;
    if (!q || !q_offsets || ((uintptr_t)q & 15) || (q_stride & 7)) return TIDAL_ERR_INVALID;
    if (num_tokens > 1 && q_stride < (int64_t)kv->num_q_heads * HEAD_DIM) return TIDAL_ERR_INVALID;
    if (kv->kv_layout == TIDAL_KV_PAGED && kv->stride_pos < HEAD_DIM) return TIDAL_ERR_INVALID;
    const int64_t esz = kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? 1 : 2;
    for (int64_t stride : {kv->stride_b, kv->stride_pos, kv->stride_head, kv->stride_page})
        if (stride >= TMA_STRIDE_LIMIT / esz) return TIDAL_ERR_UNSUPPORTED;
    return q_stride < TMA_STRIDE_LIMIT / 2 ? TIDAL_OK : TIDAL_ERR_UNSUPPORTED;
}

// Launch as launch_block does, with tensor maps as further arguments.
template <typename... Args>
tidal_status_t launch_maps(tidal_ctx* ctx, void (*kernel)(Args...), int grid, int threads, size_t smem, int cluster, cudaStream_t st, const Args&... args) {
    cudaLaunchConfig_t cfg;
    std::memset(&cfg, 0, sizeof cfg);
    cfg.gridDim = dim3(grid, 1, 1);
    cfg.blockDim = dim3(threads, 1, 1);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster; attr[1].val.clusterDim.y = 1; attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    ctx->launches++;
    if (cudaLaunchKernelEx(&cfg, kernel, args...) == cudaSuccess) return TIDAL_OK;
    cudaGetLastError();
    return TIDAL_ERR_CUDA;
}

// Scratch of the streaming kernel for single new tokens, two partial results of eight heads per CTA (see MODE_TOKENS): of one size for every shape,
// so that it is allocated with the context.
constexpr size_t TOK_ROWS = (size_t)GRID_MAX * 2 * 8;
constexpr size_t TOK_ML = TOK_ROWS * HEAD_DIM * sizeof(float), TOK_COUNTERS = TOK_ML + TOK_ROWS * sizeof(float2),
                 TOK_CURSORS = TOK_COUNTERS + (size_t)GRID_MAX * CTR_STRIDE * sizeof(int), TOK_TOTAL = TOK_CURSORS + (size_t)GRID_MAX * CTR_STRIDE * sizeof(int);

template <int NW, int STAGES, bool KV8>
tidal_status_t launch_tokens(tidal_ctx* ctx, const AttnParams& a, int grid, cudaStream_t st) {
    return launch_block(ctx, attn_kernel<MODE_TOKENS, NW, STAGES, false, false, KV8>, a, grid, NW * 32, attn_smem<MODE_TOKENS, NW, STAGES, KV8>(), 0, st);
}

tidal_status_t run_tokens(tidal_ctx* ctx, const tidal_kv_t* kv, int32_t num_tokens, const void* q, int64_t q_stride, const int32_t* q_offsets,
                          int causal, float* out, float* lse, cudaStream_t st) {
    AttnParams a;
    WsLayout none;
    std::memset(&none, 0, sizeof none);
    fill_common(a, ctx, kv, q, out, none);
    char* ws = (char*)ctx->tok_ws;
    a.part_o = (float*)ws; a.part_ml = (float2*)(ws + TOK_ML);
    a.counters = (int*)(ws + TOK_COUNTERS); a.tile_ctr = (int*)(ws + TOK_CURSORS);
    a.max_splits = GRID_MAX;
    a.q_offsets = q_offsets; a.num_tokens = num_tokens; a.causal = causal; a.q_stride = q_stride; a.lse = lse;
    a.pdl = 1; a.wait_first = 1;
    const int grid = dense_grid(ctx, kv);
    a.splits_per_item = pooled_splits(kv, kv->batch * kv->num_kv_heads, grid);
    return kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? launch_tokens<DENSE_NW8, DENSE_STAGES8, true>(ctx, a, grid, st) : launch_tokens<DENSE_NW, DENSE_STAGES, false>(ctx, a, grid, st);
}

bool prepare_prompt_kernels(tidal_ctx* ctx) {
    auto wide = [](const void* k) { return cudaFuncSetAttribute(k, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) == cudaSuccess; };
    auto room = [](auto kernel, size_t bytes) { return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes) == cudaSuccess; };
    if (!(wide((const void*)chunk_attn_kernel<false>) && wide((const void*)chunk_attn_kernel<true>) && wide((const void*)evict_select_kernel) &&
          room(chunk_attn_kernel<false>, ch_smem<false>()) && room(chunk_attn_kernel<true>, ch_smem<true>()) &&
          room(chunk_weights_kernel<false>, cw_smem(false)) && room(chunk_weights_kernel<true>, cw_smem(true)) &&
          room(attn_kernel<MODE_TOKENS, DENSE_NW, DENSE_STAGES>, attn_smem<MODE_TOKENS, DENSE_NW, DENSE_STAGES>()) &&
          room(attn_kernel<MODE_TOKENS, DENSE_NW8, DENSE_STAGES8, false, false, true>, attn_smem<MODE_TOKENS, DENSE_NW8, DENSE_STAGES8, true>()) &&
          room(evict_select_kernel, EV_SMEM_MAX)))
        return false;
    // the softmax warpgroups raise their registers within what the launch holds
    cudaFuncAttributes a;
    if (cudaFuncGetAttributes(&a, chunk_attn_kernel<false>) != cudaSuccess || a.numRegs * CH_THREADS < 256 * 216 + 128 * 72) return false;
    if (cudaFuncGetAttributes(&a, chunk_attn_kernel<true>) != cudaSuccess || a.numRegs * CH_THREADS8 < 256 * 208 + 256 * 48) return false;
    count_clusters(chunk_attn_kernel<false>, CH_THREADS, ch_smem<false>(), ctx->chunk_clusters[0]);
    count_clusters(chunk_attn_kernel<true>, CH_THREADS8, ch_smem<true>(), ctx->chunk_clusters[1]);
    count_clusters(evict_select_kernel, EV_THREADS, EV_SMEM_MAX / 2, ctx->evict_clusters);
    return true;
}

}  // namespace

extern "C" {

tidal_status_t tidal_create(tidal_ctx_t** out, int device, size_t workspace_bytes) {
    if (!out) return TIDAL_ERR_INVALID;
    *out = nullptr;
    int count = 0;
    if (cudaGetDeviceCount(&count) != cudaSuccess || device < 0 || device >= count) { cudaGetLastError(); return TIDAL_ERR_CUDA; }
    if (cudaSetDevice(device) != cudaSuccess) return TIDAL_ERR_CUDA;
    cudaDeviceProp prop;
    if (cudaGetDeviceProperties(&prop, device) != cudaSuccess) return TIDAL_ERR_CUDA;
    if (prop.major < 10) return TIDAL_ERR_UNSUPPORTED;
    tidal_ctx* ctx = new (std::nothrow) tidal_ctx();
    if (!ctx) return TIDAL_ERR_NOMEM;
    ctx->device = device;
    ctx->sm_count = prop.multiProcessorCount;
    const int d0 = resident_ctas(attn_kernel<MODE_FULL, DENSE_NW, DENSE_STAGES>, DENSE_NW * 32, attn_smem<MODE_FULL, DENSE_NW, DENSE_STAGES>(), ctx->sm_count);
    const int d1 = resident_ctas(attn_kernel<MODE_SELECT, DENSE_NW, DENSE_STAGES>, DENSE_NW * 32, attn_smem<MODE_SELECT, DENSE_NW, DENSE_STAGES>(), ctx->sm_count);
    const int d2 = resident_ctas(attn_kernel<MODE_SELECT, DENSE_NW, DENSE_STAGES, false, true>, DENSE_NW * 32, attn_smem<MODE_SELECT, DENSE_NW, DENSE_STAGES>(), ctx->sm_count);
    const int s0 = resident_ctas(attn_kernel<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>, SPARSE_NW * 32, attn_smem<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>(), ctx->sm_count);
    const int s1 = resident_ctas(attn_kernel<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES, true>, SPARSE_NW * 32, attn_smem<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>(), ctx->sm_count);
    const int e0 = resident_ctas(attn_kernel<MODE_FULL, DENSE_NW8, DENSE_STAGES8, false, false, true>, DENSE_NW8 * 32, attn_smem<MODE_FULL, DENSE_NW8, DENSE_STAGES8, true>(), ctx->sm_count);
    const int e1 = resident_ctas(attn_kernel<MODE_SELECT, DENSE_NW8, DENSE_STAGES8, false, false, true>, DENSE_NW8 * 32, attn_smem<MODE_SELECT, DENSE_NW8, DENSE_STAGES8, true>(), ctx->sm_count);
    const int e2 = resident_ctas(attn_kernel<MODE_SPARSE, SPARSE_NW8, SPARSE_STAGES8, false, false, true>, SPARSE_NW8 * 32, attn_smem<MODE_SPARSE, SPARSE_NW8, SPARSE_STAGES8, true>(), ctx->sm_count);
    const bool split_ok =
        cudaFuncSetAttribute(score_pass_kernel<SCORE_NW, SCORE_STAGES, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCORE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(score_pass_kernel<SCORE_NW, SCORE_STAGES, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCORE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(score_pass_flat_kernel<SCORE_NW, SCORE_STAGES, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCORE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(score_pass_flat_kernel<SCORE_NW, SCORE_STAGES, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCORE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(value_pass_flat_kernel<VALUE_NW, VALUE_STAGES, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VALUE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(value_pass_flat_kernel<VALUE_NW, VALUE_STAGES, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VALUE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(score_pass8_kernel<SCORE_NW, SCORE_STAGES, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCORE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(score_pass8_kernel<SCORE_NW, SCORE_STAGES, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)SCORE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(value_pass8_kernel<VALUE_NW8, VALUE_STAGES, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VALUE_SMEM8) == cudaSuccess &&
        cudaFuncSetAttribute(value_pass8_kernel<VALUE_NW8, VALUE_STAGES, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VALUE_SMEM8) == cudaSuccess &&
        cudaFuncSetAttribute(value_pass_kernel<VALUE_NW, VALUE_STAGES, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VALUE_SMEM) == cudaSuccess &&
        cudaFuncSetAttribute(value_pass_kernel<VALUE_NW, VALUE_STAGES, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)VALUE_SMEM) == cudaSuccess;
    const size_t topk_smem = 2 * (size_t)(MAX_CTX / 32) * sizeof(unsigned) + 8192 * sizeof(uint2);
    const bool topk_ok = cudaFuncSetAttribute(topk_select_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)topk_smem) == cudaSuccess;
    const size_t compact_smem = 2 * ((size_t)(MAX_CTX / 32) + 1) * sizeof(unsigned) + (size_t)COMPACT_LIST_SMEM * sizeof(uint2);
    const bool compact_ok = cudaFuncSetAttribute(topk_compact_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)compact_smem) == cudaSuccess;
    if (!prepare_block_kernels()) { cudaGetLastError(); delete ctx; return TIDAL_ERR_CUDA; }
    if (d0 <= 0 || d1 <= 0 || d2 < d1 || s0 <= 0 || s1 < s0 || e0 < d0 || e1 < d1 || e2 < s0 || !topk_ok || !compact_ok || !split_ok) { cudaGetLastError(); delete ctx; return TIDAL_ERR_CUDA; }
    if (!prepare_prompt_kernels(ctx)) { cudaGetLastError(); delete ctx; return TIDAL_ERR_CUDA; }
    count_clusters(block_select_kernel<0, false>, SC_THREADS, sc_smem(SC_MAX_BLOCKS, 1, 0), ctx->select_clusters);
    count_clusters(block_attn_kernel<false, 4>, 128, ba_smem<false>(MAX_GROUP, BA_MAX_CLUSTER, 4), ctx->attn_clusters);
    ctx->dense_slots = std::min(d0, d1);
    ctx->sparse_slots = s0;
    if (cudaMalloc((void**)&ctx->status, 256) != cudaSuccess || cudaMemset(ctx->status, 0, 256) != cudaSuccess) {
        cudaGetLastError(); delete ctx; return TIDAL_ERR_NOMEM;
    }
    if (cudaMalloc(&ctx->tok_ws, TOK_TOTAL) != cudaSuccess || cudaMemset(ctx->tok_ws, 0, TOK_TOTAL) != cudaSuccess) {
        cudaGetLastError(); cudaFree(ctx->tok_ws); cudaFree(ctx->status); delete ctx; return TIDAL_ERR_NOMEM;
    }
    if (workspace_bytes) {
        const tidal_status_t rc = ensure_ws(ctx, workspace_bytes);
        if (rc != TIDAL_OK) { cudaFree(ctx->tok_ws); cudaFree(ctx->status); delete ctx; return rc; }
    }
    *out = ctx;
    return TIDAL_OK;
}

tidal_status_t tidal_destroy(tidal_ctx_t* ctx) {
    if (!ctx) return TIDAL_ERR_INVALID;
    cudaSetDevice(ctx->device);
    cudaDeviceSynchronize();
    drop_graphs(ctx);
    if (ctx->side) cudaStreamDestroy(ctx->side);
    if (ctx->ev_fork) cudaEventDestroy(ctx->ev_fork);
    if (ctx->ev_join) cudaEventDestroy(ctx->ev_join);
    if (ctx->ws) cudaFree(ctx->ws);
    if (ctx->blk_ws) cudaFree(ctx->blk_ws);
    for (int i = 0; i < ctx->blk_old_count; ++i) cudaFree(ctx->blk_old[i]);
    if (ctx->state) cudaFree(ctx->state);
    if (ctx->tok_ws) cudaFree(ctx->tok_ws);
    if (ctx->status) cudaFree(ctx->status);
    delete ctx;
    return TIDAL_OK;
}

size_t tidal_workspace_bytes(const tidal_kv_t* kv, int32_t k) {
    if (check_kv(kv) != TIDAL_OK || k <= 0) return 0;
    return ws_bytes_for(kv, k, 0);
}

tidal_status_t tidal_reserve(tidal_ctx_t* ctx, const tidal_kv_t* kv, int32_t k, int32_t num_layers_host) {
    if (!ctx || k <= 0 || num_layers_host < 0 || num_layers_host > 1024) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    const tidal_status_t rs = ensure_side_stream(ctx);       // a later step's selection layers may use it
    if (rs != TIDAL_OK) return rs;
    const tidal_status_t ra = ensure_all(ctx, kv, ws_bytes_for(kv, k, num_layers_host));
    // Scratch of block selections over contexts that need some: the last, and no reason to fail, for callers that select no blocks
    // can do without it and tidal_block_select says itself when it is missing.
    if (ra == TIDAL_OK && (kv->max_ctx_len + TILE - 1) / TILE > SC_MAX_BLOCKS)
        ensure_block_ws(ctx, block_ws_layout(kv, kv->num_q_heads).total, nullptr);
    return ra;
}

static void fill_append(AppendParams& a, const tidal_ctx* ctx, const tidal_kv_t* kv, const void* k_new,
                        const void* v_new);

tidal_status_t tidal_kv_append(tidal_ctx_t* ctx, const tidal_kv_t* kv, const void* k_new, const void* v_new,
                               void* stream) {
    if (!ctx || !k_new || !v_new || (((uintptr_t)k_new | (uintptr_t)v_new) & 15)) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    AppendParams a;
    fill_append(a, ctx, kv, k_new, v_new);
    const int pairs = kv->batch * kv->num_kv_heads;
    kv_append_kernel<<<(pairs + 3) / 4, 128, 0, (cudaStream_t)stream>>>(a);
    ctx->launches++;
    return cudaGetLastError() == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}

static void fill_append(AppendParams& a, const tidal_ctx* ctx, const tidal_kv_t* kv, const void* k_new,
                        const void* v_new) {
    std::memset(&a, 0, sizeof a);
    a.k = (__nv_bfloat16*)const_cast<void*>(kv->k);
    a.v = (__nv_bfloat16*)const_cast<void*>(kv->v);
    a.k_new = (const __nv_bfloat16*)k_new;
    a.v_new = (const __nv_bfloat16*)v_new;
    a.stride_b = kv->stride_b; a.stride_pos = kv->stride_pos; a.stride_head = kv->stride_head;
    a.stride_page = kv->stride_page;
    a.page_table = kv->page_table; a.max_pages = kv->max_pages_per_seq; a.num_pages = kv->num_pages;
    a.paged = kv->kv_layout == TIDAL_KV_PAGED;
    a.ctx_lens = kv->ctx_lens; a.max_ctx = kv->max_ctx_len;
    a.batch = kv->batch; a.Hkv = kv->num_kv_heads;
    a.elem_bytes = kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? 1 : 2;
    a.status = ctx->status;
}

tidal_status_t tidal_full_attn(tidal_ctx_t* ctx, const tidal_kv_t* kv, const void* q, float* out, void* stream) {
    if (!ctx || !q || !out || ((uintptr_t)q & 15)) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    const WsLayout w = layout_ws(kv, 1, 0);
    if ((rc = ensure_all(ctx, kv, w.total)) != TIDAL_OK) return rc;
    return run_dense(ctx, kv, q, out, nullptr, 0, false, DEP_FIRST, w, (cudaStream_t)stream);
}

tidal_status_t tidal_select_attn(tidal_ctx_t* ctx, const tidal_kv_t* kv, const void* q, int32_t k,
                                 int32_t granularity, float* out, int32_t* idx, int32_t* idx_count,
                                 float* scores_opt, void* stream) {
    if (!ctx || !q || !out || !idx || ((uintptr_t)q & 15)) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (k <= 0 || k > kv->max_ctx_len) return TIDAL_ERR_INVALID;
    const int Hi = hi_of(kv, granularity);
    if (Hi <= 0) return TIDAL_ERR_INVALID;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    const WsLayout w = layout_ws(kv, k, 0);
    if ((rc = ensure_all(ctx, kv, w.total)) != TIDAL_OK) return rc;
    float* scores = scores_opt ? scores_opt : (float*)((char*)ctx->ws + w.scores);
    const long long stride = scores_opt ? (long long)kv->max_ctx_len : w.score_stride;
    cudaStream_t st = (cudaStream_t)stream;
    const SelectPlan sp = select_plan(ctx, kv, Hi, k, scores_opt != nullptr);
    if ((rc = run_dense(ctx, kv, q, out, scores, stride, sp.fuse, DEP_FIRST, w, st, sp.agg, sp.compact ? k : 0)) != TIDAL_OK) return rc;
    return run_topk(ctx, kv, scores, stride, k, sp.rows, Hi, sp.fuse, idx, idx_count, w, st, sp.compact);
}

tidal_status_t tidal_sparse_attn(tidal_ctx_t* ctx, const tidal_kv_t* kv, const void* q, const int32_t* idx,
                                 const int32_t* idx_count, int32_t k, int32_t num_index_heads, float* out,
                                 void* stream) {
    if (!ctx || !q || !out || !idx || ((uintptr_t)q & 15)) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (k <= 0) return TIDAL_ERR_INVALID;
    const int Hi = num_index_heads;
    if (Hi != kv->num_q_heads && Hi != kv->num_kv_heads && Hi != 1) return TIDAL_ERR_INVALID;
    if (ctx->attend_newest && !idx_count) return TIDAL_ERR_INVALID;   // the end of each list must be known
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    const WsLayout w = layout_ws(kv, k, 0);
    if ((rc = ensure_all(ctx, kv, w.total)) != TIDAL_OK) return rc;
    return run_sparse(ctx, kv, q, idx, idx_count, k, Hi, out, DEP_FIRST, CHAIN_NONE, w, (cudaStream_t)stream);
}

// Validates a step and sizes the workspace for it (may allocate and synchronise).
static tidal_status_t decode_step_prepare(tidal_ctx_t* ctx, int32_t num_layers, const uint8_t* schedule,
                                          const tidal_kv_t* kvs, const void* const* qs, float* const* outs,
                                          int32_t k, int32_t granularity, int host_layers) {
    // Validate everything before enqueuing anything.
    bool have_rho = false;
    size_t need = 0;
    for (int i = 0; i < num_layers; ++i) {
        tidal_status_t rc = check_kv(&kvs[i]);
        if (rc != TIDAL_OK) return rc;
        if (!qs[i] || !outs[i] || ((uintptr_t)qs[i] & 15)) return TIDAL_ERR_INVALID;
        if (kvs[i].batch != kvs[0].batch || kvs[i].num_q_heads != kvs[0].num_q_heads ||
            kvs[i].num_kv_heads != kvs[0].num_kv_heads) return TIDAL_ERR_INVALID;
        if (schedule[i] == TIDAL_LAYER_SELECT) {
            if (k > kvs[i].max_ctx_len) return TIDAL_ERR_INVALID;
            have_rho = true;
        } else if (schedule[i] == TIDAL_LAYER_SPARSE) {
            if (!have_rho) return TIDAL_ERR_INVALID;
        } else if (schedule[i] != TIDAL_LAYER_FULL) {
            return TIDAL_ERR_INVALID;
        }
        need = std::max(need, ws_bytes_for(&kvs[i], k, host_layers));
    }
    if (hi_of(&kvs[0], granularity) <= 0) return TIDAL_ERR_INVALID;
    return ensure_all(ctx, &kvs[0], need);
}

// Enqueues the layers of a prepared step: launches only, nothing that a stream capture forbids.
static tidal_status_t decode_step_enqueue(tidal_ctx_t* ctx, int32_t num_layers, const uint8_t* schedule,
                                          const tidal_kv_t* kvs, const void* const* qs, float* const* outs,
                                          int32_t k, int32_t granularity, int32_t* idx, int32_t* idx_count,
                                          int host_layers, cudaStream_t st, float* const* acc = nullptr) {
    const int Hi = hi_of(&kvs[0], granularity);
    tidal_status_t rc = TIDAL_OK;
    bool side_pending = false;                  // a value pass is in flight on the second stream
    for (int i = 0; i < num_layers; ++i) {
        const tidal_kv_t* kv = &kvs[i];
        const WsLayout w = layout_ws(kv, k, host_layers);
        // Every query, length, page table and cache row of the step was complete before the call, so a
        // layer may read all of them while the layer before it is still running and needs that layer to
        // have finished only before it writes scratch memory (DEP_LATE). The exceptions: the first
        // kernel of the step (whatever ran before it in the stream may have produced its inputs), and a
        // sparse layer right after a selection layer, whose index list is written by the top-k.
        const Dep dep = i == 0 ? DEP_FIRST : (ctx->layer_overlap ? DEP_LATE : DEP_PREFETCH);
        if (schedule[i] == TIDAL_LAYER_FULL) {
            rc = run_dense(ctx, kv, qs[i], outs[i], nullptr, 0, false, dep, w, st);
        } else if (schedule[i] == TIDAL_LAYER_SELECT) {
            float* scores = (float*)((char*)ctx->ws + w.scores);
            const SelectPlan sp = select_plan(ctx, kv, Hi, k, false);
            // The score buffer's last reader is the top-k of the selection layer before this one. If a
            // sparse layer ran in between, its first kernel waited for that top-k before it let anything
            // else start, so nobody reads the buffer any more; right after another selection layer, wait.
            const bool scores_free = i > 0 && schedule[i - 1] != TIDAL_LAYER_SELECT;
            // The value pass adds to the output rows, four floats at a time: in place, or in the device rows the
            // caller of this function set aside (outputs in host memory), from where its last CTAs write outs[i].
            float* const sums = (acc && acc[i]) ? acc[i] : outs[i];
            if (can_split(ctx, kv, sp) && ((uintptr_t)sums & 15) == 0 && ensure_side_stream(ctx) == TIDAL_OK) {
                // key pass -> (value pass on the second stream) | top-k -> the layers that follow. A value
                // pass still in flight reads the score buffer and the statistics this key pass overwrites.
                if (side_pending) { if (cudaStreamWaitEvent(st, ctx->ev_join, 0) != cudaSuccess) return TIDAL_ERR_CUDA; side_pending = false; }
                rc = run_score_pass(ctx, kv, qs[i], sums, scores, w.score_stride, dep, scores_free, w, st);
                if (rc == TIDAL_OK) rc = run_value_pass(ctx, kv, sums, sums == outs[i] ? nullptr : outs[i], scores, w.score_stride, w, st);
                side_pending = rc == TIDAL_OK;
            } else {
                rc = run_dense(ctx, kv, qs[i], outs[i], scores, w.score_stride, sp.fuse, dep, w, st, sp.agg, sp.compact ? k : 0, scores_free);
            }
            if (rc == TIDAL_OK) rc = run_topk(ctx, kv, scores, w.score_stride, k, sp.rows, Hi, sp.fuse, idx, idx_count, w, st, sp.compact);
        } else {
            const bool fresh_idx = i == 0 || schedule[i - 1] == TIDAL_LAYER_SELECT;
            const bool has_prev = i > 0 && schedule[i - 1] == TIDAL_LAYER_SPARSE;
            const bool has_next = i + 1 < num_layers && schedule[i + 1] == TIDAL_LAYER_SPARSE;
            const Chain chain = !ctx->layer_overlap || (!has_prev && !has_next) ? CHAIN_NONE
                                : !has_prev ? CHAIN_FIRST : !has_next ? CHAIN_LAST : CHAIN_MIDDLE;
            rc = run_sparse(ctx, kv, qs[i], idx, idx_count, k, Hi, outs[i], fresh_idx ? DEP_FIRST : dep, chain, w, st);
        }
        if (rc != TIDAL_OK) return rc;
    }
    // the step is complete on the caller's stream only when the second stream's work is
    if (side_pending && cudaStreamWaitEvent(st, ctx->ev_join, 0) != cudaSuccess) return TIDAL_ERR_CUDA;
    return TIDAL_OK;
}

tidal_status_t tidal_decode_step_append(tidal_ctx_t* ctx, int32_t num_layers, const uint8_t* schedule,
                                        const tidal_kv_t* kv_per_layer, const void* const* q_per_layer,
                                        const void* const* k_new_per_layer, const void* const* v_new_per_layer,
                                        float* const* out_per_layer, int32_t k, int32_t granularity, int32_t* idx,
                                        int32_t* idx_count, void* stream) {
    if (!ctx || num_layers <= 0 || !schedule || !kv_per_layer || !q_per_layer || !out_per_layer || !idx || !idx_count ||
        !k_new_per_layer || !v_new_per_layer || k <= 0)
        return TIDAL_ERR_INVALID;
    for (int i = 0; i < num_layers; ++i) {
        const tidal_status_t rc = check_kv(&kv_per_layer[i]);
        if (rc != TIDAL_OK) return rc;
        if (!k_new_per_layer[i] || !v_new_per_layer[i] ||
            (((uintptr_t)k_new_per_layer[i] | (uintptr_t)v_new_per_layer[i]) & 15)) return TIDAL_ERR_INVALID;
        if (kv_per_layer[i].batch != kv_per_layer[0].batch || kv_per_layer[i].num_kv_heads != kv_per_layer[0].num_kv_heads)
            return TIDAL_ERR_INVALID;
    }
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    // The whole step is validated (and its workspace sized) before the first row is written: an
    // argument error must leave the caches as they were.
    const tidal_status_t ok = decode_step_prepare(ctx, num_layers, schedule, kv_per_layer, q_per_layer, out_per_layer,
                                                  k, granularity, 0);
    if (ok != TIDAL_OK) return ok;
    const int pairs = kv_per_layer[0].batch * kv_per_layer[0].num_kv_heads;
    for (int l0 = 0; l0 < num_layers; l0 += APPEND_MAX_LAYERS) {
        const int n = std::min(APPEND_MAX_LAYERS, num_layers - l0);
        AppendBatchParams bp;
        std::memset(&bp, 0, sizeof bp);
        for (int j = 0; j < n; ++j) fill_append(bp.layer[j], ctx, &kv_per_layer[l0 + j], k_new_per_layer[l0 + j], v_new_per_layer[l0 + j]);
        kv_append_layers_kernel<<<dim3((pairs + 3) / 4, n, 1), 128, 0, (cudaStream_t)stream>>>(bp);
        ctx->launches++;
        if (cudaGetLastError() != cudaSuccess) return TIDAL_ERR_CUDA;
    }
    return tidal_decode_step(ctx, num_layers, schedule, kv_per_layer, q_per_layer, out_per_layer, k, granularity, idx,
                             idx_count, stream);
}

tidal_status_t tidal_decode_step(tidal_ctx_t* ctx, int32_t num_layers, const uint8_t* schedule,
                                 const tidal_kv_t* kv_per_layer, const void* const* q_per_layer,
                                 float* const* out_per_layer, int32_t k, int32_t granularity, int32_t* idx,
                                 int32_t* idx_count, void* stream) {
    if (!ctx || num_layers <= 0 || !schedule || !kv_per_layer || !q_per_layer || !out_per_layer || !idx || k <= 0)
        return TIDAL_ERR_INVALID;
    if (num_layers > 1024) return TIDAL_ERR_INVALID;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    tidal_status_t rc;
    raw_call_key(ctx->raw_scratch, ctx, 0, num_layers, schedule, kv_per_layer, q_per_layer, out_per_layer, idx, idx_count, k, granularity, st);
    if (replay_last(ctx, st, rc)) return rc;
    rc = decode_step_prepare(ctx, num_layers, schedule, kv_per_layer, q_per_layer, out_per_layer, k, granularity, 0);
    if (rc != TIDAL_OK) return rc;
    // (the workspace may just have moved: the remembered bytes must name the addresses the graph was built with)
    raw_call_key(ctx->raw_scratch, ctx, 0, num_layers, schedule, kv_per_layer, q_per_layer, out_per_layer, idx, idx_count, k, granularity, st);
    KeyBuilder kb;
    step_key(kb, ctx, 0, num_layers, schedule, kv_per_layer, k, granularity, 0);
    kb.add_raw(q_per_layer, sizeof(void*) * (size_t)num_layers);
    kb.add_raw(out_per_layer, sizeof(void*) * (size_t)num_layers);
    kb.add(idx); kb.add(idx_count);
    rc = run_graphed(ctx, kb, st, [&]() {
        return decode_step_enqueue(ctx, num_layers, schedule, kv_per_layer, q_per_layer, out_per_layer, k, granularity,
                                   idx, idx_count, 0, st);
    });
    if (rc == TIDAL_OK) remember_last(ctx); else ctx->last.exec = nullptr;
    return rc;
}

tidal_status_t tidal_set_attend_newest(tidal_ctx_t* ctx, int32_t enabled) {
    if (!ctx) return TIDAL_ERR_INVALID;
    ctx->attend_newest = enabled != 0;
    return TIDAL_OK;
}

tidal_status_t tidal_set_select_margin(tidal_ctx_t* ctx, float margin) {
    if (!ctx || !(margin >= 0.f) || margin > 64.f) return TIDAL_ERR_INVALID;
    ctx->select_margin = margin;
    return TIDAL_OK;
}

tidal_status_t tidal_set_layer_overlap(tidal_ctx_t* ctx, int32_t enabled) {
    if (!ctx) return TIDAL_ERR_INVALID;
    ctx->layer_overlap = enabled != 0;
    return TIDAL_OK;
}

tidal_status_t tidal_set_output_dtype(tidal_ctx_t* ctx, int32_t dtype) {
    if (!ctx || (dtype != TIDAL_OUT_F32 && dtype != TIDAL_OUT_BF16)) return TIDAL_ERR_INVALID;
    ctx->out_bf16 = dtype == TIDAL_OUT_BF16;
    return TIDAL_OK;
}

tidal_status_t tidal_set_graphs(tidal_ctx_t* ctx, int32_t enabled) {
    if (!ctx) return TIDAL_ERR_INVALID;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    ctx->graphs_enabled = enabled != 0;
    if (!ctx->graphs_enabled) drop_graphs(ctx);
    return TIDAL_OK;
}

tidal_status_t tidal_decode_step_host(tidal_ctx_t* ctx, int32_t num_layers, const uint8_t* schedule,
                                      const tidal_kv_t* kv_per_layer, const void* q_host, float* out_host,
                                      int32_t k, int32_t granularity, void* stream) {
    if (!ctx || num_layers <= 0 || num_layers > 1024 || !schedule || !kv_per_layer || !q_host || !out_host || k <= 0)
        return TIDAL_ERR_INVALID;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    tidal_status_t rc;
    raw_call_key(ctx->raw_scratch, ctx, 1, num_layers, schedule, kv_per_layer, nullptr, nullptr, q_host, out_host, k, granularity, st);
    if (replay_last(ctx, st, rc)) {
        if (rc != TIDAL_OK) return rc;
        return cudaStreamSynchronize(st) == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
    }
    rc = check_kv(&kv_per_layer[0]);
    if (rc != TIDAL_OK) return rc;
    // Size the workspace for every layer first so that the staging pointers stay put.
    size_t need = 0;
    for (int i = 0; i < num_layers; ++i) {
        if ((rc = check_kv(&kv_per_layer[i])) != TIDAL_OK) return rc;
        need = std::max(need, ws_bytes_for(&kv_per_layer[i], k, num_layers));
    }
    if ((rc = ensure_all(ctx, &kv_per_layer[0], need)) != TIDAL_OK) return rc;
    // All layers must share batch and head counts (checked again below); the staging
    // offsets depend only on those and on max_ctx_len of the layer used for the layout.
    const tidal_kv_t* kv0 = &kv_per_layer[0];
    for (int i = 1; i < num_layers; ++i)
        if (kv_per_layer[i].max_ctx_len != kv0->max_ctx_len) return TIDAL_ERR_UNSUPPORTED;
    const WsLayout w = layout_ws(kv0, k, num_layers);
    const size_t rows = (size_t)kv0->batch * kv0->num_q_heads;
    char* ws = (char*)ctx->ws;
    char* qd = ws + w.q_stage;
    float* od = (float*)(ws + w.out_stage);
    const size_t out_elem = ctx->out_bf16 ? 2 : 4;            // bytes per output element, device and host side
    // Page-locked host memory is addressable from the device: the kernels then read the queries from the
    // caller's buffer and write their outputs straight into it (each output element once, as posted
    // writes over the bus), and the two copies, which would otherwise run before the first and after
    // the last layer, disappear (cfg3: 699 -> 679 us per step). Pageable buffers go through the staging
    // area and copies.
    auto device_alias = [](const void* p) -> void* {
        cudaPointerAttributes at;
        if (cudaPointerGetAttributes(&at, p) != cudaSuccess) { cudaGetLastError(); return nullptr; }
        if (at.type != cudaMemoryTypeHost || at.devicePointer == nullptr) return nullptr;
        return at.devicePointer;
    };
    char* out_alias = (char*)device_alias(out_host);
    char* q_alias = (char*)device_alias(q_host);
    if (q_alias && ((uintptr_t)q_alias & 15)) q_alias = nullptr;      // query rows are read as 16-byte pieces
    const void* qs[1024];
    float* outs[1024];
    // (a selection layer may run as two passes whose second adds to the output rows with reductions: those
    // sums stay in the staging area and the pass's last CTAs write the finished rows to the caller's buffer)
    float* acc[1024];
    for (int i = 0; i < num_layers; ++i) {
        qs[i] = (q_alias ? q_alias : qd) + (size_t)i * rows * HEAD_DIM * 2;
        outs[i] = (float*)((out_alias ? out_alias : (char*)od) + (size_t)i * rows * HEAD_DIM * out_elem);
        acc[i] = (out_alias && schedule[i] == TIDAL_LAYER_SELECT) ? (float*)((char*)od + (size_t)i * rows * HEAD_DIM * out_elem) : nullptr;
    }
    if ((rc = decode_step_prepare(ctx, num_layers, schedule, kv_per_layer, qs, outs, k, granularity, num_layers)) != TIDAL_OK)
        return rc;
    auto enqueue = [&]() -> tidal_status_t {
        if (!q_alias && cudaMemcpyAsync(qd, q_host, (size_t)num_layers * rows * HEAD_DIM * 2, cudaMemcpyHostToDevice, st) != cudaSuccess)
            return TIDAL_ERR_CUDA;
        const tidal_status_t r = decode_step_enqueue(ctx, num_layers, schedule, kv_per_layer, qs, outs, k, granularity,
                                                     (int*)(ws + w.idx), (int*)(ws + w.idx_count), num_layers, st, acc);
        if (r != TIDAL_OK) return r;
        if (!out_alias && cudaMemcpyAsync(out_host, od, (size_t)num_layers * rows * HEAD_DIM * out_elem, cudaMemcpyDeviceToHost, st) != cudaSuccess)
            return TIDAL_ERR_CUDA;
        return TIDAL_OK;
    };
    // The copies can be recorded with the layers only when both host buffers are page-locked.
    auto pinned = [](const void* p) {
        cudaPointerAttributes at;
        if (cudaPointerGetAttributes(&at, p) != cudaSuccess) { cudaGetLastError(); return false; }
        return at.type == cudaMemoryTypeHost;
    };
    if (pinned(q_host) && pinned(out_host)) {
        KeyBuilder kb;
        step_key(kb, ctx, 1, num_layers, schedule, kv_per_layer, k, granularity, num_layers);
        kb.add(q_host); kb.add(out_host);
        rc = run_graphed(ctx, kb, st, enqueue);
        if (rc == TIDAL_OK) {
            raw_call_key(ctx->raw_scratch, ctx, 1, num_layers, schedule, kv_per_layer, nullptr, nullptr, q_host, out_host, k, granularity, st);
            remember_last(ctx);
        } else {
            ctx->last.exec = nullptr;
        }
    } else {
        ctx->last.exec = nullptr;
        rc = enqueue();
    }
    if (rc != TIDAL_OK) return rc;
    return cudaStreamSynchronize(st) == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}

tidal_status_t tidal_device_status(tidal_ctx_t* ctx, void* stream) {
    if (!ctx) return TIDAL_ERR_INVALID;
    if (cudaSetDevice(ctx->device) != cudaSuccess) return TIDAL_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)stream;
    if (cudaStreamSynchronize(st) != cudaSuccess) return TIDAL_ERR_CUDA;
    int word = 0;
    if (cudaMemcpy(&word, ctx->status, sizeof word, cudaMemcpyDeviceToHost) != cudaSuccess) return TIDAL_ERR_CUDA;
    if (word == 0) return TIDAL_OK;
    // one kind of trouble per call; the others wait for the next
    const int told = word & STATUS_SPLIT_OVERFLOW ? STATUS_SPLIT_OVERFLOW : word & STATUS_WAITED_OUT ? STATUS_WAITED_OUT :
                     word & STATUS_NO_PAGES ? STATUS_NO_PAGES : word;
    const int rest = word & ~told;
    if (cudaMemcpyAsync(ctx->status, &rest, sizeof rest, cudaMemcpyHostToDevice, st) != cudaSuccess ||
        cudaStreamSynchronize(st) != cudaSuccess) return TIDAL_ERR_CUDA;
    return told == STATUS_SPLIT_OVERFLOW ? TIDAL_ERR_INTERNAL : told == STATUS_WAITED_OUT ? TIDAL_ERR_TIMEOUT : told == STATUS_NO_PAGES ? TIDAL_ERR_PAGES : TIDAL_ERR_INDEX;
}


// ---- paged caches filled on the device, block-sparse attention -------------------------------------------
tidal_status_t tidal_page_map(tidal_ctx_t* ctx, int32_t batch, const int32_t* old_lens, const int32_t* new_lens,
                              int32_t* page_table, int32_t max_pages_per_seq, int32_t num_pages, int32_t* free_pages,
                              const int32_t* num_free, int32_t* num_free_out, int32_t max_tokens, int64_t* slots,
                              int32_t* positions, int32_t* token_offsets, void* stream) {
    if (!ctx || !old_lens || !new_lens || !page_table || !free_pages || !num_free || !num_free_out) return TIDAL_ERR_INVALID;
    if (batch <= 0 || max_pages_per_seq <= 0 || num_pages <= 0 || max_tokens < 0 || (max_tokens > 0 && !slots)) return TIDAL_ERR_INVALID;
    if (batch > PM_MAX_BATCH || (long long)max_pages_per_seq * TILE > MAX_CTX) return TIDAL_ERR_UNSUPPORTED;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    PageMapParams p;
    std::memset(&p, 0, sizeof p);
    p.batch = batch; p.max_pages = max_pages_per_seq; p.num_pages = num_pages; p.max_tokens = max_tokens;
    p.old_lens = old_lens; p.new_lens = new_lens; p.page_table = page_table; p.free_pages = free_pages;
    p.num_free = num_free; p.num_free_out = num_free_out;
    p.slots = (long long*)slots; p.positions = positions; p.token_offsets = token_offsets; p.status = ctx->status;
    p.arrivals = ctx->status + 32;                           // (a line of its own behind the status word, zeroed with it at creation)
    const size_t smem = 3 * ((size_t)batch + 1) * sizeof(int);
    // CTAs of 256 threads, whose barriers and scans are the shorter chain, for as many sequences as their scan holds, one for every
    // 512 tokens (64 requests' decode step: 3.1 us, 3.8 with 1024 threads; 295 K tokens of 8 prompts: 4.9 us, 5.1 with 1024 threads
    // for every 2048).
    if (batch <= PM_THREADS_SMALL * PM_PER) {
        const int grid = std::max(1, std::min(4 * ctx->sm_count, (int)(((long long)max_tokens + 511) / 512)));
        return launch_block(ctx, page_map_kernel<PM_THREADS_SMALL>, p, grid, PM_THREADS_SMALL, smem, 0, (cudaStream_t)stream);
    }
    const int grid = std::max(1, std::min(ctx->sm_count, (int)(((long long)max_tokens + 2047) / 2048)));
    return launch_block(ctx, page_map_kernel<PM_THREADS>, p, grid, PM_THREADS, smem, 0, (cudaStream_t)stream);
}

tidal_status_t tidal_kv_write(tidal_ctx_t* ctx, const tidal_kv_t* kv, int32_t num_tokens, const void* k_new, const void* v_new,
                              int64_t k_stride, int64_t v_stride, const int64_t* slots, void* stream) {
    if (!ctx || num_tokens < 0) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (num_tokens == 0) return TIDAL_OK;
    if (!k_new || !v_new || !slots || (((uintptr_t)k_new | (uintptr_t)v_new) & 15)) return TIDAL_ERR_INVALID;
    if (k_stride < 0 || v_stride < 0 || ((k_stride | v_stride) & 7)) return TIDAL_ERR_INVALID;
    const long long runs = ((long long)num_tokens + KW_TOKENS - 1) / KW_TOKENS;
    const long long grid = (runs * kv->num_kv_heads + KW_WARPS - 1) / KW_WARPS;
    if (grid * KW_WARPS > 0xffffffffLL) return TIDAL_ERR_UNSUPPORTED;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    KvWriteParams p;
    std::memset(&p, 0, sizeof p);
    p.k = (uint8_t*)const_cast<void*>(kv->k); p.v = (uint8_t*)const_cast<void*>(kv->v);
    p.k_new = (const __nv_bfloat16*)k_new; p.v_new = (const __nv_bfloat16*)v_new;
    p.k_stride = k_stride; p.v_stride = v_stride; p.slots = (const long long*)slots;
    p.num_tokens = num_tokens; p.Hkv = kv->num_kv_heads; p.paged = kv->kv_layout == TIDAL_KV_PAGED; p.max_ctx = kv->max_ctx_len;
    p.num_slots = p.paged ? (long long)kv->num_pages * TILE : (long long)kv->batch * kv->max_ctx_len;
    p.stride_b = kv->stride_b; p.stride_pos = kv->stride_pos; p.stride_head = kv->stride_head; p.stride_page = kv->stride_page;
    const long long esz = kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? 1 : 2;
    if (p.stride_page * esz <= 0xffffffffLL && p.stride_pos * esz <= 0xffffffffLL) {
        p.page_bytes = (unsigned)(p.stride_page * esz); p.pos_bytes = (unsigned)(p.stride_pos * esz);
    }
    p.k_scale = kv->k_scale; p.v_scale = kv->v_scale; p.status = ctx->status;
    return launch_block(ctx, kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? kv_write_kernel<true> : kv_write_kernel<false>, p, (int)grid,
                        KW_WARPS * 32, 0, 0, (cudaStream_t)stream);
}

tidal_status_t tidal_block_bounds(tidal_ctx_t* ctx, const tidal_kv_t* kv, const int32_t* start_lens, int32_t max_new, void* bounds,
                                  int32_t bound_blocks, void* stream) {
    if (!ctx || max_new < 0) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK || (rc = check_bounds(kv, bounds, bound_blocks)) != TIDAL_OK) return rc;
    BoundsParams p;
    fill_block_cache(p.c, ctx, kv, bound_blocks);
    p.start_lens = start_lens;
    p.bounds = (__nv_bfloat16*)bounds;
    // max_new tokens from `start` on lie in at most ceil((max_new - 1) / 16) + 1 blocks
    p.blocks = p.c.max_blocks;
    if (start_lens && max_new > 0) p.blocks = (int)std::min<long long>(p.blocks, ((long long)max_new - 1 + TILE - 1) / TILE + 1);
    const long long grid = ((long long)kv->batch * kv->num_kv_heads * p.blocks + BB_WARPS - 1) / BB_WARPS;
    if (grid > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    return launch_block(ctx, kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? block_bounds_kernel<true> : block_bounds_kernel<false>, p, (int)grid,
                        BB_WARPS * 32, 0, 0, (cudaStream_t)stream);
}

tidal_status_t tidal_block_select(tidal_ctx_t* ctx, const tidal_kv_t* kv, const void* q, const void* bounds, int32_t bound_blocks,
                                  int32_t m, int32_t granularity, int32_t keep_first, int32_t keep_last, int32_t* idx,
                                  int32_t* idx_count, void* stream) {
    if (!ctx || !q || !idx || ((uintptr_t)q & 15) || m <= 0 || keep_first < 0 || keep_last < 0) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK || (rc = check_bounds(kv, bounds, bound_blocks)) != TIDAL_OK) return rc;
    const int Hi = hi_of(kv, granularity);
    if (Hi <= 0 || m > MAX_CTX / TILE) return TIDAL_ERR_INVALID;
    const bool per_qhead = granularity == TIDAL_SEL_PER_QHEAD;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    SelectBlocksParams p;
    fill_block_cache(p.c, ctx, kv, bound_blocks);
    p.q = (const __nv_bfloat16*)q;
    p.bounds = (const __nv_bfloat16*)bounds;
    // one KV head's factor changes no order: it matters only where several KV heads are added up
    p.k_scale = kv->kv_dtype == TIDAL_KV_FP8_E4M3 && granularity == TIDAL_SEL_SHARED ? kv->k_scale : nullptr;
    p.mode = granularity; p.m = m; p.keep_first = keep_first; p.keep_last = keep_last;
    p.idx = idx; p.idx_count = idx_count;
    p.npad = (int)align_up((size_t)p.c.max_blocks, 32);
    p.scores = nullptr; p.err = nullptr; p.chunks = 0;
    const bool shared_set = granularity == TIDAL_SEL_SHARED;
    const int items = shared_set ? kv->batch : kv->batch * kv->num_kv_heads;
    const int rows = per_qhead ? p.c.G : 1;
    cudaStream_t st = (cudaStream_t)stream;
    // Up to 16384 positions one launch scores and ranks: 1024 positions 4.2 us against 8.4 of two launches, 16384 positions 7.0
    // against 9.5, eight ragged sequences of them 10.3 against 14.3 (a set per query head; only 256 items of one CTA each are
    // slower, 26.0 against 25.3). Beyond, a cluster is too few SMs for an item: 131072 positions 19.5 us against 12.4.
    if (p.c.max_blocks <= SC_MAX_BLOCKS) {
        // A cluster with a tile per warp and a CTA per row, or the largest one with which all items are resident together; a shared set
        // has a tile per KV head (6 sequences of 573 positions, 32 KV heads: 6.8 us; head after head in one CTA 53). Rows are ranked
        // by a warp each where there are more of them than CTAs, which would rank them one after the other (43 sequences of 2048
        // positions, 8 KV heads of 8 query heads: 15.2 us against 48.1; 24 of 6000: 17.7 against 29.4), and always up to 1024
        // positions, with a single CTA (1024 positions, four heads: 4.4 us against 6.0 of a CTA per row; 1376 items of 85
        // positions: 6.4 against 20.9). Else the CTA is faster (4096 positions, four heads: 7.1 us against 8.3).
        const int tiles = (p.c.max_blocks + 15) / 16, tasks = shared_set ? tiles * p.c.Hkv : tiles;
        const int want = shared_set ? tasks : (tasks + SC_WARPS - 1) / SC_WARPS;
        int cluster = std::min(SB_MAX_CLUSTER, p.c.max_blocks <= 64 ? want : std::max(want, rows));
        while (cluster > 1 && ctx->select_clusters[cluster] < items) --cluster;
        const bool by_warp = !shared_set && (p.c.max_blocks <= 64 || (p.c.max_blocks <= 512 && cluster < rows));
        const int warps = by_warp ? std::max(std::min((tasks + cluster - 1) / cluster, SC_WARPS), (rows + cluster - 1) / cluster) : SC_WARPS;
        const size_t smem = sc_smem(p.npad, (rows + cluster - 1) / cluster, shared_set ? cluster * warps : 0);
        auto launch = [&](auto kernel) { return launch_block(ctx, kernel, p, items * cluster, warps * 32, smem, cluster, st); };
        if (shared_set) return launch(block_select_kernel<0, true>);
        if (!by_warp) return launch(block_select_kernel<0, false>);
        if (p.c.max_blocks <= 64) return launch(block_select_kernel<2, false>);
        return p.c.max_blocks <= 256 ? launch(block_select_kernel<8, false>) : launch(block_select_kernel<16, false>);
    }
    const BlockWs w = block_ws_layout(kv, per_qhead ? kv->num_q_heads : kv->num_kv_heads);
    const long long grid = (long long)kv->batch * kv->num_kv_heads * w.chunks;
    if (grid > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
    if ((rc = ensure_block_ws(ctx, w.total, &st)) != TIDAL_OK) return rc;
    p.scores = (float*)((char*)ctx->blk_ws + w.scores); p.err = (float*)((char*)ctx->blk_ws + w.err);
    p.chunks = w.chunks;
    if ((rc = launch_block(ctx, block_score_kernel, p, (int)grid, 32, SS_SMEM, 0, st)) != TIDAL_OK) return rc;
    // Sixteen scores per thread, with as few threads as that takes: their barriers and scans are the shorter chain (131072
    // positions, 8 rows: 512 threads take 0.8 us less than 1024; ragged batch of 8 x 65536, 256 rows: 256 threads 3.1 us less than
    // 1024, and 3.3 us less than 128 with 32 scores each).
    const int rank_rows = kv->batch * Hi;
    const size_t keys = (size_t)p.npad * 8;
    if (p.c.max_blocks > 8192) return launch_block(ctx, block_rank_kernel<1024, 4>, p, rank_rows, 1024, keys, 0, st);
    if (p.c.max_blocks > 4096) return launch_block(ctx, block_rank_kernel<512, 4>, p, rank_rows, 512, keys, 0, st);
    return launch_block(ctx, block_rank_kernel<256, 4>, p, rank_rows, 256, keys, 0, st);
}

tidal_status_t tidal_block_attn(tidal_ctx_t* ctx, const tidal_kv_t* kv, const void* q, const int32_t* idx, const int32_t* idx_count,
                                int32_t m, int32_t num_index_heads, float* out, void* stream) {
    if (!ctx || !q || !out || !idx || ((uintptr_t)q & 15) || m <= 0) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    const int Hi = num_index_heads;
    if (Hi != kv->num_q_heads && Hi != kv->num_kv_heads && Hi != 1) return TIDAL_ERR_INVALID;
    if (m > BA_MAX_LIST) return TIDAL_ERR_UNSUPPORTED;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    BlockAttnParams p;
    fill_block_cache(p.c, ctx, kv, 0);
    p.q = (const __nv_bfloat16*)q;
    p.out = out; p.out_bf16 = ctx->out_bf16;
    p.idx = idx; p.idx_count = idx_count; p.m = m; p.Hi = Hi;
    const float scale = kv->sm_scale > 0.f ? kv->sm_scale : 1.0f / std::sqrt((float)kv->head_dim);
    p.scale_log2 = scale * 1.4426950408889634f;
    const bool fp8 = kv->kv_dtype == TIDAL_KV_FP8_E4M3;
    p.k_scale = fp8 ? kv->k_scale : nullptr;
    p.v_scale = fp8 ? kv->v_scale : nullptr;
    const int items = kv->batch * (Hi == kv->num_q_heads ? kv->num_q_heads : kv->num_kv_heads);
    const int ncols = Hi == kv->num_q_heads ? 1 : p.c.G;
    cudaStream_t st = (cudaStream_t)stream;
    // An item's warps: as many as its list has blocks, or as the GPU has room for, eight per SM. Four to a CTA, in clusters of up to 16 with
    // an SM per CTA (8 items of 256 blocks: 8.9 us in clusters of 16, 9.9 of 8). Eight to a CTA where the items leave no room for
    // more CTAs (32 items of 256 blocks over an 8-bit cache: 10.3 us against 13.6 with four) and the list is long enough to pay for
    // the larger merge, which grows with the heads (64 items of 16 blocks of 8 heads: 9.7 us, 6.5 with four). Single warps, in
    // clusters of four to six that fill seven of an SM's eight places (not all clusters would find eight), for more items than SMs with
    // lists that pay for the merge: warps spread more evenly than CTAs of four (160 items of 128 blocks, 8 bits: 19.3 us
    // against 25.4; 256 items: 25.2 against 26.1; 160 items of 24 blocks, 4 heads: 9.4 against 9.0; 256 of 64, 8 heads: 21.8 against
    // 18.5). Two or one to a CTA where there are more items than CTAs of four that the GPU holds (384 items of 10 blocks:
    // 7.0 us against 9.7; 704 of 2: 5.1 against 10.5).
    auto launch = [&](auto kernel8, auto kernel4, auto kernel2, auto kernel1, auto smem_of, auto over_ring) -> tidal_status_t {
        const int sms = ctx->sm_count, list = std::min(m, p.c.max_blocks);
        int cluster = 1, warps = 4;
        if (items > 4 * sms) {
            warps = 1;
        } else if (items > 2 * sms) {
            warps = 2;
        } else if (items > sms) {
            const int share = std::min(7 * sms / items, 6);
            if (share >= 4 && ncols <= 4 && list >= 16 * ncols && ctx->attn_clusters[share] > 0) warps = 1, cluster = share;
        } else {
            while (cluster < BA_MAX_CLUSTER && items * cluster * 2 <= sms && cluster * 5 < list && ctx->attn_clusters[cluster * 2] >= items) cluster *= 2;
            if (cluster <= 4 && cluster * 4 < list && items * cluster * 2 > sms && (cluster == 1 || list >= cluster * (8 + 4 * ncols))) warps = 8;
        }
        p.over_ring = over_ring(ncols, cluster, warps);
        return launch_block(ctx, warps == 8 ? kernel8 : warps == 4 ? kernel4 : warps == 2 ? kernel2 : kernel1, p, items * cluster, warps * 32,
                            smem_of(ncols, cluster, warps), cluster, st);
    };
    if (fp8)
        return launch(block_attn_kernel<true, 8>, block_attn_kernel<true, 4>, block_attn_kernel<true, 2>, block_attn_kernel<true, 1>, ba_smem<true>,
                      ba_over_ring<true>);
    return launch(block_attn_kernel<false, 8>, block_attn_kernel<false, 4>, block_attn_kernel<false, 2>, block_attn_kernel<false, 1>, ba_smem<false>,
                  ba_over_ring<false>);
}

// ---- a prompt's way into the cache: norms and rotary positions, chunk attention, eviction ----------------
tidal_status_t tidal_rope_frequencies(int32_t rotary_dim, double base, int32_t scaling, double factor, double low, double high,
                                      double trained_len, double* inv_freq, double* cos_scale) {
    if (!inv_freq || !cos_scale || rotary_dim <= 0 || !(base > 1.0) || std::isinf(base)) return TIDAL_ERR_INVALID;
    if (rotary_dim > HEAD_DIM || rotary_dim % 16) return TIDAL_ERR_UNSUPPORTED;
    if (scaling < TIDAL_ROPE_PLAIN || scaling > TIDAL_ROPE_RAMP) return TIDAL_ERR_INVALID;
    if (scaling != TIDAL_ROPE_PLAIN && (!(factor >= 1.0) || std::isinf(factor))) return TIDAL_ERR_INVALID;
    if (scaling >= TIDAL_ROPE_BANDS && (!(low > 0.0) || !(high > low) || std::isinf(high) || !(trained_len > 0.0) || std::isinf(trained_len))) return TIDAL_ERR_INVALID;
    const double n = rotary_dim, turn = 6.283185307179586476925;
    if (scaling == TIDAL_ROPE_BASE) base *= std::pow(factor, n / (n - 2.0));
    const double lo = std::max(std::floor(n * std::log(trained_len / (turn * high)) / (2.0 * std::log(base))), 0.0);
    const double hi = std::min(std::ceil(n * std::log(trained_len / (turn * low)) / (2.0 * std::log(base))), n - 1.0);
    for (int i = 0; i < rotary_dim / 2; ++i) {
        double f = std::pow(base, -2.0 * i / n);
        if (scaling == TIDAL_ROPE_LINEAR) f /= factor;
        if (scaling == TIDAL_ROPE_BANDS) {
            const double s = std::min(std::max((trained_len * f / turn - low) / (high - low), 0.0), 1.0);
            f = (1.0 - s) * f / factor + s * f;
        }
        if (scaling == TIDAL_ROPE_RAMP) {
            const double r = std::min(std::max((i - lo) / std::max(hi - lo, 0.001), 0.0), 1.0);
            f = r * f / factor + (1.0 - r) * f;
        }
        inv_freq[i] = f;
    }
    *cos_scale = scaling == TIDAL_ROPE_RAMP ? 0.1 * std::log(factor) + 1.0 : 1.0;
    return TIDAL_OK;
}

tidal_status_t tidal_rope_init(tidal_rope_t* rope, int32_t rotary_dim, int32_t layout, const double* inv_freq, double cos_scale) {
    if (!rope || !inv_freq || rotary_dim <= 0 || !std::isfinite(cos_scale)) return TIDAL_ERR_INVALID;
    if (layout != TIDAL_ROPE_HALF && layout != TIDAL_ROPE_INTERLEAVED) return TIDAL_ERR_INVALID;
    if (rotary_dim > HEAD_DIM || rotary_dim % 16) return TIDAL_ERR_UNSUPPORTED;
    for (int i = 0; i < rotary_dim / 2; ++i)
        if (!std::isfinite(inv_freq[i])) return TIDAL_ERR_INVALID;
    std::memset(rope, 0, sizeof *rope);
    rope->rotary_dim = rotary_dim; rope->layout = layout; rope->scale = (float)cos_scale;
    for (int i = 0; i < rotary_dim / 2; ++i) {
        // the fraction of a turn in 64 bits, in long double: a double's 53 would be off by 2^-22 of a turn at position 2^31
        const long double t = (long double)inv_freq[i] / 6.283185307179586476925286766559L;
        long double part = t - std::floor(t);
        part = std::floor(part * 18446744073709551616.0L + 0.5L);
        rope->step[i] = part >= 18446744073709551616.0L ? 0 : (uint64_t)part;
    }
    return TIDAL_OK;
}

static tidal_status_t check_rope(const tidal_rope_t* rope, int32_t num_tokens, float eps, const void* q_weight, const void* k_weight) {
    if (!rope || num_tokens < 0 || !(eps >= 0.f) || std::isinf(eps)) return TIDAL_ERR_INVALID;
    if (rope->rotary_dim <= 0 || rope->rotary_dim > HEAD_DIM || rope->rotary_dim % 16) return TIDAL_ERR_INVALID;
    if (rope->layout != TIDAL_ROPE_HALF && rope->layout != TIDAL_ROPE_INTERLEAVED) return TIDAL_ERR_INVALID;
    return (((uintptr_t)q_weight | (uintptr_t)k_weight) & 15) ? TIDAL_ERR_INVALID : TIDAL_OK;
}
// Rows of `heads` heads per token: in place, or apart from each other.
static bool rope_rows_ok(const void* x, int64_t stride, int heads, int32_t num_tokens) {
    if (!x || ((uintptr_t)x & 15) || (stride & 7)) return false;
    return num_tokens <= 1 || stride >= (int64_t)heads * HEAD_DIM;
}

static tidal_status_t run_rope(tidal_ctx_t* ctx, RopeParams& p, int mode, cudaStream_t st) {
    const int pairs = (p.Hq + 1) / 2 + (mode == ROPE_BACK ? 1 : 2) * ((p.Hkv + 1) / 2);
    // A warp per token where there are tokens enough to fill the GPU; for fewer, several warps with a share of the rows each (32/8 heads, normed; 64 tokens: a
    // warp each 6.5 us, as many as there are pairs 3.0; 256: 6.6, 5.4, and 4.3 as here; 4096: 16 and 40).
    const long long fill = 16LL * ctx->sm_count;
    p.parts = (int)std::max(1LL, std::min<long long>((pairs + 1) / 2, fill / std::max(p.num_tokens, 1)));
    const long long grid = ((long long)p.num_tokens * p.parts + RO_WARPS - 1) / RO_WARPS;
    if (grid > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    const bool half = p.rope.layout == TIDAL_ROPE_HALF, norm = p.q_weight || p.k_weight;
    auto launch = [&](auto h, auto n) {
        constexpr bool H = decltype(h)::value, N = decltype(n)::value;
        return launch_block(ctx, mode == ROPE_BACK ? rope_kernel<H, N, ROPE_BACK> : mode == ROPE_CACHE ? rope_kernel<H, N, ROPE_CACHE> : rope_kernel<H, N, ROPE_CACHE8>,
                            p, (int)grid, RO_WARPS * 32, 0, 0, st);
    };
    using T = std::integral_constant<bool, true>;
    using F = std::integral_constant<bool, false>;
    return half ? (norm ? launch(T(), T()) : launch(T(), F())) : (norm ? launch(F(), T()) : launch(F(), F()));
}

tidal_status_t tidal_rope(tidal_ctx_t* ctx, const tidal_rope_t* rope, int32_t num_tokens, int32_t num_q_heads, int32_t num_kv_heads,
                          const void* q, int64_t q_stride, const void* k, int64_t k_stride, const int32_t* positions,
                          const void* q_weight, const void* k_weight, float eps, void* q_out, int64_t q_out_stride, void* k_out,
                          int64_t k_out_stride, void* stream) {
    if (!ctx || num_q_heads < 0 || num_kv_heads < 0 || num_q_heads + (int64_t)num_kv_heads == 0) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_rope(rope, num_tokens, eps, q_weight, k_weight);
    if (rc != TIDAL_OK) return rc;
    if (num_q_heads > 65535 || num_kv_heads > 65535) return TIDAL_ERR_UNSUPPORTED;
    if (num_tokens == 0) return TIDAL_OK;
    if (!positions) return TIDAL_ERR_INVALID;
    if (num_q_heads ? !rope_rows_ok(q, q_stride, num_q_heads, num_tokens) || !rope_rows_ok(q_out, q_out_stride, num_q_heads, num_tokens) : q || q_out) return TIDAL_ERR_INVALID;
    if (num_kv_heads ? !rope_rows_ok(k, k_stride, num_kv_heads, num_tokens) || !rope_rows_ok(k_out, k_out_stride, num_kv_heads, num_tokens) : k || k_out) return TIDAL_ERR_INVALID;
    if (num_tokens > 1 && ((q && q == q_out && q_stride != q_out_stride) || (k && k == k_out && k_stride != k_out_stride))) return TIDAL_ERR_INVALID;
    RopeParams p;
    std::memset(&p, 0, sizeof p);
    p.rope = *rope;
    p.q = (const __nv_bfloat16*)q; p.k = (const __nv_bfloat16*)k; p.q_stride = q_stride; p.k_stride = k_stride;
    p.q_out = (__nv_bfloat16*)q_out; p.k_out = (__nv_bfloat16*)k_out; p.qo_stride = q_out_stride; p.ko_stride = k_out_stride;
    p.positions = positions; p.q_weight = (const __nv_bfloat16*)q_weight; p.k_weight = (const __nv_bfloat16*)k_weight; p.eps = eps;
    p.num_tokens = num_tokens; p.Hq = num_q_heads; p.Hkv = num_kv_heads; p.status = ctx->status;
    return run_rope(ctx, p, ROPE_BACK, (cudaStream_t)stream);
}

tidal_status_t tidal_rope_write(tidal_ctx_t* ctx, const tidal_rope_t* rope, const tidal_kv_t* kv, int32_t num_tokens, const void* q,
                                int64_t q_stride, const void* k_new, int64_t k_stride, const void* v_new, int64_t v_stride,
                                const int32_t* positions, const int64_t* slots, const void* q_weight, const void* k_weight, float eps,
                                void* q_out, int64_t q_out_stride, void* stream) {
    if (!ctx) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK || (rc = check_rope(rope, num_tokens, eps, q_weight, k_weight)) != TIDAL_OK) return rc;
    if (num_tokens == 0) return TIDAL_OK;
    if (!positions || !slots || !q != !q_out) return TIDAL_ERR_INVALID;
    if (!rope_rows_ok(k_new, k_stride, kv->num_kv_heads, num_tokens) || !rope_rows_ok(v_new, v_stride, kv->num_kv_heads, num_tokens)) return TIDAL_ERR_INVALID;
    if (q && (!rope_rows_ok(q, q_stride, kv->num_q_heads, num_tokens) || !rope_rows_ok(q_out, q_out_stride, kv->num_q_heads, num_tokens))) return TIDAL_ERR_INVALID;
    if (num_tokens > 1 && q && q == q_out && q_stride != q_out_stride) return TIDAL_ERR_INVALID;
    RopeParams p;
    std::memset(&p, 0, sizeof p);
    p.rope = *rope;
    p.q = (const __nv_bfloat16*)q; p.k = (const __nv_bfloat16*)k_new; p.v = (const __nv_bfloat16*)v_new;
    p.q_stride = q_stride; p.k_stride = k_stride; p.v_stride = v_stride;
    p.q_out = (__nv_bfloat16*)q_out; p.qo_stride = q_out_stride;
    p.positions = positions; p.q_weight = (const __nv_bfloat16*)q_weight; p.k_weight = (const __nv_bfloat16*)k_weight; p.eps = eps;
    p.num_tokens = num_tokens; p.Hq = q ? kv->num_q_heads : 0; p.Hkv = kv->num_kv_heads;
    p.ck = (uint8_t*)const_cast<void*>(kv->k); p.cv = (uint8_t*)const_cast<void*>(kv->v);
    p.slots = (const long long*)slots; p.paged = kv->kv_layout == TIDAL_KV_PAGED; p.max_ctx = kv->max_ctx_len;
    p.num_slots = p.paged ? (long long)kv->num_pages * TILE : (long long)kv->batch * kv->max_ctx_len;
    p.stride_b = kv->stride_b; p.stride_pos = kv->stride_pos; p.stride_head = kv->stride_head; p.stride_page = kv->stride_page;
    p.k_scale = kv->k_scale; p.v_scale = kv->v_scale; p.status = ctx->status;
    return run_rope(ctx, p, kv->kv_dtype == TIDAL_KV_FP8_E4M3 ? ROPE_CACHE8 : ROPE_CACHE, (cudaStream_t)stream);
}

tidal_status_t tidal_chunk_attn(tidal_ctx_t* ctx, const tidal_kv_t* kv, int32_t num_tokens, const void* q, int64_t q_stride,
                                const int32_t* q_offsets, int32_t max_new, int32_t causal, int32_t window, float* out, float* lse,
                                void* stream) {
    if (!ctx) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_chunk(kv, num_tokens, q, q_stride, q_offsets, max_new, window);
    if (rc != TIDAL_OK) return rc;
    if (num_tokens == 0) return TIDAL_OK;
    if (!out || ((uintptr_t)out & 15) || ((uintptr_t)lse & 3)) return TIDAL_ERR_INVALID;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    // One token each: products of 128 rows would be empty but for one group of heads, and the cache streams at memory speed through
    // the decode kernels (64 sequences of up to 16384: 346 us, 600 as a chunk; one of 33 positions: 7.6 and 8.7).
    if (max_new == 1 && (window == 0 || window >= MAX_CTX)) return run_tokens(ctx, kv, num_tokens, q, q_stride, q_offsets, causal != 0, out, lse, (cudaStream_t)stream);
    ChunkParams p;
    std::memset(&p, 0, sizeof p);
    fill_block_cache(p.c, ctx, kv, 0);
    p.q = (const __nv_bfloat16*)q; p.q_stride = num_tokens > 1 ? q_stride : 0;
    p.q_offsets = q_offsets; p.num_tokens = num_tokens; p.tile_tokens = CH_TILE / p.c.G;
    p.causal = causal != 0; p.window = window < MAX_CTX ? window : 0;        // (a window of the longest context hides nothing)
    p.scale_log2 = (kv->sm_scale > 0.f ? kv->sm_scale : 1.0f / std::sqrt((float)kv->head_dim)) * 1.4426950408889634f;
    const bool fp8 = kv->kv_dtype == TIDAL_KV_FP8_E4M3;
    if (fp8) { p.k_scale = kv->k_scale; p.v_scale = kv->v_scale; }
    p.out = out; p.out_bf16 = ctx->out_bf16; p.lse = lse;
    CUtensorMap qm, km, vm;
    if (!cache_maps(p, kv, &km, &vm) || !query_map(&qm, q, num_tokens, kv->num_q_heads, q_stride, p.c.G, p.tile_tokens)) return TIDAL_ERR_CUDA;
    // CTA tiles of all sequences: a sequence's last one may be partly filled
    const long long per = 2 * p.tile_tokens;
    long long tiles = num_tokens / per + std::min(kv->batch, num_tokens);
    if (max_new > 0) tiles = std::min(tiles, kv->batch * ((max_new + per - 1) / per));
    const long long units = tiles * kv->num_kv_heads;
    // Few rows: the cache is cut over the CTAs of a cluster, as long as all of them run at once and there is a tile of positions for each (8 tokens after
    // 992: 11.9 us, 16.8 with two tiles each, 23.2 uncut; 3 after 127 10.2 and 11.0 uncut; 8 of 16384 40 and 236; 32/8 heads).
    const int seen = window > 0 ? (int)std::min<long long>(kv->max_ctx_len, (long long)window + per) : kv->max_ctx_len;
    int ranks = 1;
    while (ranks < 16 && units * ranks * 2 <= ctx->sm_count && seen > ranks * CH_TILE && ctx->chunk_clusters[fp8][ranks * 2] >= units) ranks *= 2;
    if (units * ranks > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
    return fp8 ? launch_maps(ctx, chunk_attn_kernel<true>, (int)(units * ranks), CH_THREADS8, ch_smem<true>(), ranks, (cudaStream_t)stream, p, qm, km, vm)
               : launch_maps(ctx, chunk_attn_kernel<false>, (int)(units * ranks), CH_THREADS, ch_smem<false>(), ranks, (cudaStream_t)stream, p, qm, km, vm);
}

tidal_status_t tidal_chunk_weights(tidal_ctx_t* ctx, const tidal_kv_t* kv, int32_t num_tokens, const void* q, int64_t q_stride,
                                   const int32_t* q_offsets, int32_t max_new, int32_t causal, int32_t window, int32_t last,
                                   const float* lse, float decay, float* weights, int64_t stride, int32_t num_weight_heads, void* stream) {
    if (!ctx) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_chunk(kv, num_tokens, q, q_stride, q_offsets, max_new, window);
    if (rc != TIDAL_OK) return rc;
    if (last < 0 || !weights || ((uintptr_t)weights & 3) || stride < kv->max_ctx_len || !std::isfinite(decay)) return TIDAL_ERR_INVALID;
    if (num_weight_heads != kv->num_kv_heads && num_weight_heads != 1) return TIDAL_ERR_INVALID;
    if (num_tokens == 0) return TIDAL_OK;
    if (!lse || ((uintptr_t)lse & 3)) return TIDAL_ERR_INVALID;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    WeightParams p;
    std::memset(&p, 0, sizeof p);
    fill_block_cache(p.c, ctx, kv, 0);
    p.q_offsets = q_offsets; p.num_tokens = num_tokens;
    int most = max_new > 0 ? std::min(max_new, num_tokens) : num_tokens;
    if (last > 0) most = std::min(most, last);
    p.tile_tokens = std::min(CH_TILE / p.c.G, most);
    p.causal = causal != 0; p.window = window < MAX_CTX ? window : 0; p.last = last;     // (a window of the longest context hides nothing)
    p.scale_log2 = (kv->sm_scale > 0.f ? kv->sm_scale : 1.0f / std::sqrt((float)kv->head_dim)) * 1.4426950408889634f;
    const bool fp8 = kv->kv_dtype == TIDAL_KV_FP8_E4M3;
    if (fp8) p.k_scale = kv->k_scale;
    // New tokens that are a good part of the context see some tiles and not others: every gridDim.x-th tile evens that out (8192 tokens from the first on 731 us,
    // as runs 973; 4096 of 16384 842 and 889; 8300 of 65536 6763 and 7120). Below that runs, which meet fewer sequences and
    // queries, are as fast or faster (1024 of 16384 226 us, strided 228; 64 each of four of 16384 54 and 72).
    p.strided = most > p.tile_tokens && 8LL * most > kv->max_ctx_len;
    p.lse = lse; p.decay = decay; p.weights = weights; p.stride = stride; p.heads = num_weight_heads;
    CUtensorMap qm, km;
    if (!cache_maps(p, kv, &km, nullptr) || !query_map(&qm, q, num_tokens, kv->num_q_heads, q_stride, p.c.G, p.tile_tokens)) return TIDAL_ERR_CUDA;
    const long long tiles = (long long)kv->batch * num_weight_heads * ((kv->max_ctx_len + CH_TILE - 1) / CH_TILE);
    const int grid = (int)std::min<long long>(ctx->sm_count, tiles);
    return fp8 ? launch_maps(ctx, chunk_weights_kernel<true>, grid, CW_THREADS8, cw_smem(true), 1, (cudaStream_t)stream, p, qm, km)
               : launch_maps(ctx, chunk_weights_kernel<false>, grid, CW_THREADS, cw_smem(false), 1, (cudaStream_t)stream, p, qm, km);
}

tidal_status_t tidal_evict_select(tidal_ctx_t* ctx, const tidal_kv_t* kv, const float* weights, int64_t stride, int32_t num_weight_heads,
                                  int32_t m, int32_t keep_first, int32_t keep_last, int32_t* kept, int32_t* new_lens, void* stream) {
    if (!ctx) return TIDAL_ERR_INVALID;
    const tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (!weights || ((uintptr_t)weights & 3) || !kept || !new_lens || new_lens == kv->ctx_lens) return TIDAL_ERR_INVALID;
    if (m <= 0 || m > MAX_CTX || keep_first < 0 || keep_last < 0 || stride < kv->max_ctx_len) return TIDAL_ERR_INVALID;
    if (num_weight_heads != kv->num_kv_heads && num_weight_heads != 1) return TIDAL_ERR_INVALID;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    EvictParams p;
    std::memset(&p, 0, sizeof p);
    p.weights = weights; p.stride = stride; p.ctx_lens = kv->ctx_lens; p.max_ctx = kv->max_ctx_len; p.heads = num_weight_heads;
    p.m = m; p.keep_first = keep_first; p.keep_last = keep_last; p.kept = kept; p.new_lens = new_lens;
    const int rows = kv->batch * num_weight_heads;
    // A cluster holds a row; more CTAs than that needs from 12288 positions on, as long as all run at once and have 4096 keys each: two more barriers of a cluster
    // in every round cost 2 us (8 rows of 8192: one CTA 8.8 us, two 10.4; 13000: 11.7 and, of four, 10.7; 32768: 18.2 and, of eight, 12.5).
    int cluster = 1;
    while ((size_t)((kv->max_ctx_len + cluster - 1) / cluster) * 4 > EV_SMEM_MAX) cluster *= 2;
    while (cluster < EV_MAX_CLUSTER && kv->max_ctx_len > std::max(cluster * 4096, 12288) && rows * cluster * 2 <= ctx->sm_count && ctx->evict_clusters[cluster * 2] >= rows) cluster *= 2;
    const int slice = ((kv->max_ctx_len + cluster - 1) / cluster + 3) / 4 * 4;
    if ((long long)rows * cluster > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
    return launch_block(ctx, evict_select_kernel, p, rows * cluster, EV_THREADS, (size_t)slice * 4, cluster, (cudaStream_t)stream);
}

tidal_status_t tidal_kv_gather(tidal_ctx_t* ctx, const tidal_kv_t* kv, const tidal_kv_t* into, const int32_t* kept, const int32_t* counts,
                               int32_t m, int32_t num_list_heads, const float* weights, int64_t stride, float* weights_out,
                               int64_t stride_out, void* stream) {
    if (!ctx) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK || (into && (rc = check_kv(into)) != TIDAL_OK)) return rc;
    if (!kept || !counts || m <= 0 || m > MAX_CTX) return TIDAL_ERR_INVALID;
    if (num_list_heads != kv->num_kv_heads && num_list_heads != 1) return TIDAL_ERR_INVALID;
    const tidal_kv_t* to = into ? into : kv;
    if (to->batch != kv->batch || to->num_kv_heads != kv->num_kv_heads || to->kv_dtype != kv->kv_dtype) return TIDAL_ERR_INVALID;
    if (!weights != !weights_out) return TIDAL_ERR_INVALID;
    if (weights && ((((uintptr_t)weights | (uintptr_t)weights_out) & 3) || stride < kv->max_ctx_len || stride_out < std::min(m, to->max_ctx_len))) return TIDAL_ERR_INVALID;
    if (weights && weights == weights_out && (into || stride != stride_out)) return TIDAL_ERR_INVALID;
    DeviceScope dev(ctx->device);
    if (!dev.ok) return TIDAL_ERR_CUDA;
    GatherParams p;
    std::memset(&p, 0, sizeof p);
    fill_block_cache(p.from, ctx, kv, 0);
    p.k = (uint8_t*)const_cast<void*>(to->k); p.v = (uint8_t*)const_cast<void*>(to->v);
    p.stride_b = to->stride_b; p.stride_pos = to->stride_pos; p.stride_head = to->stride_head; p.stride_page = to->stride_page;
    p.page_table = to->page_table; p.max_pages = to->max_pages_per_seq; p.num_pages = to->num_pages;
    p.paged = to->kv_layout == TIDAL_KV_PAGED; p.max_ctx = to->max_ctx_len;
    p.kept = kept; p.counts = counts; p.heads = num_list_heads; p.m = m;
    const bool fp8 = kv->kv_dtype == TIDAL_KV_FP8_E4M3;
    p.row_bytes = HEAD_DIM * (fp8 ? 1 : 2);
    p.weights = weights; p.weights_out = weights_out; p.w_stride = stride; p.wo_stride = stride_out;
    if (into) {
        const long long per = GA_ROWS;
        const long long grid = ((long long)kv->batch * kv->num_kv_heads * ((m + per - 1) / per) + GA_WARPS - 1) / GA_WARPS;
        if (grid > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
        return launch_block(ctx, fp8 ? gather_copy_kernel<true> : gather_copy_kernel<false>, p, (int)grid, GA_WARPS * 32, 0, 0, (cudaStream_t)stream);
    }
    const long long grid = (long long)kv->batch * kv->num_kv_heads * (2 * p.row_bytes / GI_COLUMN) + (weights ? (long long)kv->batch * num_list_heads : 0);
    if (grid > 0x7fffffffLL) return TIDAL_ERR_UNSUPPORTED;
    return launch_block(ctx, gather_inplace_kernel, p, (int)grid, GI_THREADS, 0, 0, (cudaStream_t)stream);
}

int64_t tidal_launch_count(const tidal_ctx_t* ctx) { return ctx ? ctx->launches : 0; }

const char* tidal_strerror(tidal_status_t s) {
    switch (s) {
        case TIDAL_OK: return "ok";
        case TIDAL_ERR_INVALID: return "invalid argument";
        case TIDAL_ERR_UNSUPPORTED: return "unsupported configuration";
        case TIDAL_ERR_NOMEM: return "out of device memory";
        case TIDAL_ERR_CUDA: return "CUDA runtime error";
        case TIDAL_ERR_TIMEOUT: return "device-side wait timed out";
        case TIDAL_ERR_INDEX: return "token index or page id out of range";
        case TIDAL_ERR_TOO_LARGE: return "problem exceeds the fixed scratch of the allocation-free entry point";
        case TIDAL_ERR_PAGES: return "page map not built: lengths, tokens or pages beyond what the arrays and the pool hold";
        case TIDAL_ERR_INTERNAL: return "launch plan inconsistency detected on the device (results are invalid)";
        default: return "unknown status";
    }
}

}  // extern "C"

// =====================================================================================================
// Sparse attention for callers that must not allocate.
//
// Everything the kernel needs beyond the caller's inputs and outputs (the split partial results,
// the arrival counters, the pool cursors and a status word) lives in one file-scope device array
// of fixed size, so this entry point never calls cudaMalloc, cudaFree or anything that allocates.
// =====================================================================================================
namespace {

constexpr int NOALLOC_MAX_ROWS = 4096;      // (sequence, query head) rows; also the number of partial slots
constexpr size_t NOALLOC_PART_O = (size_t)NOALLOC_MAX_ROWS * HEAD_DIM * sizeof(float);   // 2 MiB
constexpr size_t NOALLOC_PART_ML = (size_t)NOALLOC_MAX_ROWS * sizeof(float2);           // 32 KiB
constexpr size_t NOALLOC_WORDS = 2 * (size_t)NOALLOC_MAX_ROWS * sizeof(int) + 256;      // counters, cursors, status
constexpr size_t NOALLOC_BYTES = NOALLOC_PART_O + NOALLOC_PART_ML + NOALLOC_WORDS;      // 2 MiB + 64 KiB + 256 B, about 2.06 MiB

// Held by every GPU that loads the library until the process exits. In host code this name is
// only a handle for cudaGetSymbolAddress, never a device address.
static __device__ __align__(256) unsigned char g_noalloc_scratch[NOALLOC_BYTES];

constexpr int NOALLOC_MAX_DEVICES = 64;
struct NoallocDevice {
    bool ready = false;
    unsigned char* scratch = nullptr;       // device address of g_noalloc_scratch on this GPU
    int slots = 0;                          // resident CTAs of the sparse kernel on this GPU
};
NoallocDevice g_noalloc_dev[NOALLOC_MAX_DEVICES];
std::mutex g_noalloc_mutex;

// Once per device, with that device current: resolve the scratch array's device address and
// prepare the kernel (shared-memory opt-in, occupancy). Allocates nothing.
tidal_status_t noalloc_setup(int device, const NoallocDevice** out) {
    std::lock_guard<std::mutex> lock(g_noalloc_mutex);
    NoallocDevice& d = g_noalloc_dev[device];
    if (!d.ready) {
        void* ptr = nullptr;
        if (cudaGetSymbolAddress(&ptr, g_noalloc_scratch) != cudaSuccess || ptr == nullptr) {
            cudaGetLastError();
            return TIDAL_ERR_CUDA;
        }
        int sms = 0;
        if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return TIDAL_ERR_CUDA;
        const int slots = resident_ctas(attn_kernel<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>, SPARSE_NW * 32,
                                        attn_smem<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>(), sms);
        if (slots <= 0) { cudaGetLastError(); return TIDAL_ERR_CUDA; }
        d.scratch = static_cast<unsigned char*>(ptr);
        d.slots = slots;
        d.ready = true;
    }
    *out = &d;
    return TIDAL_OK;
}

}  // namespace

extern "C" tidal_status_t tidal_sparse_attn_noalloc(const tidal_kv_t* kv, const void* q, const int32_t* idx,
                                                    const int32_t* idx_count, int32_t k,
                                                    int32_t num_index_heads, float* out, void* stream) {
    if (!q || !out || !idx || ((uintptr_t)q & 15)) return TIDAL_ERR_INVALID;
    tidal_status_t rc = check_kv(kv);
    if (rc != TIDAL_OK) return rc;
    if (k <= 0) return TIDAL_ERR_INVALID;
    const int Hi = num_index_heads;
    if (Hi != kv->num_q_heads && Hi != kv->num_kv_heads && Hi != 1) return TIDAL_ERR_INVALID;
    if (kv->kv_dtype != TIDAL_KV_BF16) return TIDAL_ERR_UNSUPPORTED;
    const long long rows = (long long)kv->batch * kv->num_q_heads;
    if (rows > NOALLOC_MAX_ROWS) return TIDAL_ERR_TOO_LARGE;
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) { cudaGetLastError(); return TIDAL_ERR_CUDA; }
    if (device < 0 || device >= NOALLOC_MAX_DEVICES) return TIDAL_ERR_UNSUPPORTED;
    const NoallocDevice* dev = nullptr;
    if ((rc = noalloc_setup(device, &dev)) != TIDAL_OK) return rc;

    // Every item (one query head, or one KV head's group) is shared by S CTAs through its pool
    // cursor; a row then needs S partial slots and the scratch holds NOALLOC_MAX_ROWS of them.
    const int per_batch = (Hi == kv->num_q_heads) ? kv->num_q_heads : kv->num_kv_heads;
    const int items = kv->batch * per_batch;
    const int tiles_item = (k + TILE - 1) / TILE;
    int S = std::max(1, std::min(dev->slots, GRID_MAX) / items);
    S = std::min(S, std::max(1, tiles_item / MIN_TILES_PER_CTA));
    while (S > 1 && rows * S > NOALLOC_MAX_ROWS) --S;

    unsigned char* base = dev->scratch;
    int* words = reinterpret_cast<int*>(base + NOALLOC_PART_O + NOALLOC_PART_ML);
    AttnParams a;
    std::memset(&a, 0, sizeof a);
    a.q = (const __nv_bfloat16*)q;
    a.k = (const __nv_bfloat16*)kv->k;
    a.v = (const __nv_bfloat16*)kv->v;
    a.out = out;
    a.stride_b = kv->stride_b; a.stride_pos = kv->stride_pos; a.stride_head = kv->stride_head;
    a.stride_page = kv->stride_page;
    a.page_table = kv->page_table; a.max_pages = kv->max_pages_per_seq; a.num_pages = kv->num_pages;
    a.paged = kv->kv_layout == TIDAL_KV_PAGED;
    a.ctx_lens = kv->ctx_lens;
    a.max_ctx = kv->max_ctx_len;
    a.Hq = kv->num_q_heads; a.Hkv = kv->num_kv_heads; a.G = a.Hq / a.Hkv;
    a.scale = kv->sm_scale > 0.f ? kv->sm_scale : 1.0f / std::sqrt((float)kv->head_dim);
    a.scale_log2 = a.scale * 1.4426950408889634f;
    a.batch = kv->batch;
    a.splits_per_item = S;
    a.idx = idx; a.idx_count = idx_count; a.budget = k; a.Hi = Hi;
    a.part_o = reinterpret_cast<float*>(base);
    a.part_ml = reinterpret_cast<float2*>(base + NOALLOC_PART_O);
    a.counters = words;
    a.tile_ctr = words + NOALLOC_MAX_ROWS;
    a.ctr_stride = 1;
    a.status = words + 2 * NOALLOC_MAX_ROWS;
    a.max_splits = S;
    a.hist_shift = 21;
    a.pdl = 0;
    a.wait_first = 1;

    cudaStream_t st = (cudaStream_t)stream;
    // The array keeps whatever the previous call left behind: the counters and cursors must read
    // zero when the kernel starts (the partial results are always written before they are read).
    if (cudaMemsetAsync(words, 0, NOALLOC_WORDS, st) != cudaSuccess) { cudaGetLastError(); return TIDAL_ERR_CUDA; }
    attn_kernel<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>
        <<<S * items, SPARSE_NW * 32, attn_smem<MODE_SPARSE, SPARSE_NW, SPARSE_STAGES>(), st>>>(a);
    return cudaGetLastError() == cudaSuccess ? TIDAL_OK : TIDAL_ERR_CUDA;
}
