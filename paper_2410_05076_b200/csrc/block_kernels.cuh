// Block-sparse decode attention: blocks of 16 positions (one page) ranked by an upper bound of their logits.
//
//   block_bounds_kernel  per block and KV head the channelwise least and greatest key (lo, hi), in bf16 (exact)
//   block_select_kernel  s = sum_c max(q_c lo_c, q_c hi_c) >= q . k for every key k of a block, and per index head the m
//                        blocks with the largest s, exactly, ties toward the lower block
//   block_attn_kernel    softmax attention over the cached positions of the listed blocks
#pragma once

#include "attn_kernels.cuh"

namespace tidal {

constexpr int BOUND_ELEMS = 2 * HEAD_DIM;                   // lo[128], hi[128] of one (block, KV head): 512 bytes

// What the block kernels share of the cache's description.
struct BlockCache {
    const uint8_t* k;
    const uint8_t* v;
    long long stride_b, stride_pos, stride_head, stride_page;
    const int* page_table;
    int max_pages, num_pages, paged;
    const int* ctx_lens;
    int max_ctx, max_blocks;                                // max_blocks = ceil(max_ctx / 16)
    int bound_blocks;                                       // contiguous caches: blocks per sequence that the bounds buffer holds
    int batch, Hq, Hkv, G;
    int* status;
};

__device__ __forceinline__ int cached_len(const BlockCache& c, int b) { return max(min(c.ctx_lens[b], c.max_ctx), 0); }

// Row of the bounds of (sequence b, block blk, KV head g): per physical page where the cache is paged.
__device__ __forceinline__ long long bounds_row(const BlockCache& c, int b, int blk, int page, int g) {
    return c.paged ? (long long)page * c.Hkv + g : ((long long)b * c.Hkv + g) * c.bound_blocks + blk;
}

// ---- key bounds ----------------------------------------------------------------------------------------------
// One warp per (sequence, KV head, block): it loads the block's key rows (16 x 256 bytes, or 16 x 128 of codes) with
// 16-byte loads that are all in flight together, takes packed minima and maxima and merges its row groups
// by shuffles. Bound by memory: the keys are read once, 512 bytes are written per 16 rows.
struct BoundsParams {
    BlockCache c;
    const int* start_lens;                                  // null: from the first block on
    int blocks;                                             // blocks per sequence to look at, from start / 16 on
    __nv_bfloat16* bounds;
};

__device__ __forceinline__ uint32_t bmin2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("min.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t bmax2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
// Two fp16 numbers that are E4M3 values -> bf16 (exact).
__device__ __forceinline__ uint32_t f16x2_to_bf16x2(uint32_t w) {
    float lo, hi;
    asm("{\n.reg .f16 l, h;\nmov.b32 {l, h}, %2;\ncvt.f32.f16 %0, l;\ncvt.f32.f16 %1, h;\n}\n" : "=f"(lo), "=f"(hi) : "r"(w));
    return pack_bf16(lo, hi);
}

constexpr int BB_WARPS = 8;

template <bool KV8>
__global__ void __launch_bounds__(BB_WARPS * 32) block_bounds_kernel(const BoundsParams p) {
    const BlockCache& c = p.c;
    const int lane = threadIdx.x & 31;
    const long long w = (long long)blockIdx.x * BB_WARPS + (threadIdx.x >> 5);
    const long long pair = w / p.blocks;
    pdl_wait();
    pdl_trigger();
    if (pair >= (long long)c.batch * c.Hkv) return;
    const int b = (int)(pair / c.Hkv), g = (int)(pair - (long long)b * c.Hkv);
    const int n = cached_len(c, b);
    const int start = p.start_lens ? max(p.start_lens[b], 0) : 0;
    const long long blk_l = (long long)(start / TILE) + (w - pair * p.blocks);
    if (blk_l * TILE >= n) return;
    const int blk = (int)blk_l, rows = min(TILE, n - blk * TILE);
    int page = 0;
    long long off = (long long)g * c.stride_head;
    if (c.paged) {
        page = __ldg(c.page_table + (long long)b * c.max_pages + blk);
        if ((unsigned)page >= (unsigned)c.num_pages) { if (lane == 0) atomicOr(c.status, STATUS_BAD_PAGE); return; }
        off += (long long)page * c.stride_page;
    } else {
        off += (long long)b * c.stride_b + (long long)blk * TILE * c.stride_pos;
    }
    constexpr uint32_t BPINF = 0x7f807f80u, BNINF = 0xff80ff80u;
    uint4* const out = reinterpret_cast<uint4*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS);
    if constexpr (!KV8) {
        const int piece = lane & 15, r0 = lane >> 4;        // rows r0 + 2 i
        uint4 x[8];
        const __nv_bfloat16* src = reinterpret_cast<const __nv_bfloat16*>(c.k) + off + r0 * c.stride_pos + piece * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (r0 + 2 * i < rows) x[i] = __ldg(reinterpret_cast<const uint4*>(src + 2 * i * c.stride_pos));
        uint32_t lo[4] = {BPINF, BPINF, BPINF, BPINF}, hi[4] = {BNINF, BNINF, BNINF, BNINF};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (r0 + 2 * i < rows) {
                const uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) { lo[j] = bmin2(lo[j], y[j]); hi[j] = bmax2(hi[j], y[j]); }
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            lo[j] = bmin2(lo[j], __shfl_xor_sync(0xffffffffu, lo[j], 16));
            hi[j] = bmax2(hi[j], __shfl_xor_sync(0xffffffffu, hi[j], 16));
        }
        out[lane] = r0 ? make_uint4(hi[0], hi[1], hi[2], hi[3]) : make_uint4(lo[0], lo[1], lo[2], lo[3]);
    } else {
        const int piece = lane & 7, r0 = lane >> 3;         // rows r0 + 4 i, sixteen codes each
        uint4 x[4];
        const uint8_t* src = c.k + off + r0 * c.stride_pos + piece * 16;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r0 + 4 * i < rows) x[i] = __ldg(reinterpret_cast<const uint4*>(src + 4 * i * c.stride_pos));
        uint32_t lo[8], hi[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) { lo[j] = BPINF; hi[j] = BNINF; }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (r0 + 4 * i < rows) {
                const uint32_t y[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t a, d;
                    e4m3x4_to_f16x2x2(y[j], a, d);
                    a = f16x2_to_bf16x2(a);
                    d = f16x2_to_bf16x2(d);
                    lo[2 * j] = bmin2(lo[2 * j], a); hi[2 * j] = bmax2(hi[2 * j], a);
                    lo[2 * j + 1] = bmin2(lo[2 * j + 1], d); hi[2 * j + 1] = bmax2(hi[2 * j + 1], d);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
#pragma unroll
            for (int sh = 8; sh <= 16; sh <<= 1) {
                lo[j] = bmin2(lo[j], __shfl_xor_sync(0xffffffffu, lo[j], sh));
                hi[j] = bmax2(hi[j], __shfl_xor_sync(0xffffffffu, hi[j], sh));
            }
        }
        // row group 0 writes the first half of its sixteen lo's, 1 the second; 2 and 3 the hi's
        uint32_t z[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = (r0 & 2) ? hi[j] : lo[j];
        const int h = r0 & 1;
        out[(r0 >> 1) * 16 + piece * 2 + h] = h ? make_uint4(z[4], z[5], z[6], z[7]) : make_uint4(z[0], z[1], z[2], z[3]);
    }
}

// ---- the m best blocks -----------------------------------------------------------------------------------------
// One launch, no scratch memory. A thread-block cluster serves an item: a (sequence, KV head), or a sequence where all
// heads share a set. Its CTAs score the item's blocks and push each score row (one per query head, or one
// sum) into the shared memory of the CTA that owns the row; after one cluster barrier the owners rank their rows, one
// per CTA, and the others leave.
//
// Scores. sum_c max(q_c lo_c, q_c hi_c) = q+ . hi + q- . lo with q+ = max(q, 0), q- = min(q, 0): two products, so 16 matrix
// instructions serve 16 blocks and the whole group of query heads. A warp takes 16 blocks x 512 bytes straight into the
// registers that are its A fragments (the contraction index may be relabelled: lane (gid, tig) holds the 16-byte
// pieces tig + 4 j of rows gid and gid + 8). Bound by memory: 512 bytes per block and KV head.
//
// The set is the one that the scores in 64 bits give. Every instruction starts from zero and its results are added in fp32:
// aligned to its largest product and cut at 2^-23 of that, 16 products lose at most 2^-19 of it, 16 instructions 2^-15;
// the additions (16 per score, three over a group, one per KV head) lose 2^-24 of sum_c |q_c| max|bound| each. Call that e.
// One histogram over the row's range gives the bin t of the need-th largest fp32 score x; a block with
// bin(x - 2e) > t is in for certain (x - 2e exceeds the need-th largest x, so its true value exceeds all but
// need - 1 others'), one with bin(x + 2e) < t is out; bin() is monotone, so rounding in it does no harm. What is left, a
// few blocks, is ranked by x; if the gap at the border is not more than 2e, those within 2e of it are evaluated in 64 bits
// and ranked by (score, lower block first). Rows that have no finite range or error bound, or too many blocks at
// the border, are evaluated in 64 bits wherever undecided.
struct SelectBlocksParams {
    BlockCache c;
    const __nv_bfloat16* q;
    const __nv_bfloat16* bounds;
    const float* k_scale;                                   // factors of the KV heads where several are added up (or null)
    int mode;                                               // TIDAL_SEL_*: rows of an item are its query heads, or their sum
    int m, keep_first, keep_last;
    int npad;                                               // blocks a score row has room for (a multiple of 32)
    int* idx;
    int* idx_count;
};

constexpr int SB_BINS = 2048;
constexpr int SB_CAND = 256;                                // border blocks ranked directly
constexpr int SB_MAX_CLUSTER = 16;
constexpr int SB_MAX_BLOCKS = 16384;
constexpr int SB_QROW = HEAD_DIM + 8;                       // padded query row in shared memory (elements)
constexpr int SB_RANGES = (SB_MAX_CLUSTER + 7) * 16;        // (rows of a CTA) x (CTAs) x (warps) at most
// Dynamic shared memory: 8 bytes per block (the row being ranked, then its keys in 64 bits), 4 for every further row.
__host__ __device__ constexpr size_t sb_smem(int npad, int rows_per_cta) { return (size_t)npad * (4 + 4 * (size_t)rows_per_cta); }

// Larger double <=> larger key; not-a-number above everything, -0 as +0.
__device__ __forceinline__ unsigned long long wide_key(double s) {
    s += 0.0;
    if (s != s) return ~0ull;
    const unsigned long long u = (unsigned long long)__double_as_longlong(s);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, int rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(cluster_addr(addr, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(cluster_addr(addr, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory"); }

// Exclusive prefix sum over the CTA. s_part must not be in use; it is free again after the next barrier.
template <int NT>
__device__ __forceinline__ int cta_scan(int v, int* s_part) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, sh);
        if (lane >= sh) x += y;
    }
    if (lane == 31) s_part[warp] = x;
    __syncthreads();
    const int w = lane < warp && lane < NT / 32 ? s_part[lane] : 0;
    return x - v + __reduce_add_sync(0xffffffffu, w);
}

// One block's score in 64 bits for query heads h0 .. h1 - 1, by a warp: four channels per lane and head.
__device__ __forceinline__ double wide_score(const SelectBlocksParams& p, int b, int h0, int h1, int blk, int lane) {
    const BlockCache& c = p.c;
    int page = 0;
    if (c.paged) {
        page = __ldg(c.page_table + (long long)b * c.max_pages + blk);
        if ((unsigned)page >= (unsigned)c.num_pages) return 0.0;
    }
    double acc = 0.0;
    int h = h0;
    for (int g = h0 / c.G; h < h1; ++g) {
        const uint2* bp = reinterpret_cast<const uint2*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS) + lane;
        const uint2 lo = __ldg(bp), hi = __ldg(bp + 32);
        double part = 0.0;
        for (; h < h1 && h < (g + 1) * c.G; ++h) {
            const uint2 q = __ldg(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h) * HEAD_DIM) + lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t qw = i & 2 ? q.y : q.x, lw = i & 2 ? lo.y : lo.x, hw = i & 2 ? hi.y : hi.x;
                const uint32_t bw = (i & 1 ? qw : qw << 16) >> 31 ? lw : hw;      // a negative q takes the least key
                const float qf = __uint_as_float(i & 1 ? qw & 0xffff0000u : qw << 16);
                const float bf = __uint_as_float(i & 1 ? bw & 0xffff0000u : bw << 16);
                part = fma((double)qf, (double)bf, part);
            }
        }
        acc += p.k_scale ? part * (double)__ldg(p.k_scale + g) : part;
    }
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, sh);
    return acc;
}

// NT threads per CTA: 512 with an SM to themselves, for few items, whose streaming wants every SM and whose ranking is the
// critical path; 256 twice on an SM, for batches, where one item's ranking hides behind another's stream.
template <int NT>
__global__ void __launch_bounds__(NT, NT == 512 ? 1 : 2) block_select_kernel(const SelectBlocksParams p) {
    constexpr int NW = NT / 32;
    constexpr int VECS = 8;                                 // groups of four scores per thread: rows of up to 32 NT blocks
    const BlockCache& c = p.c;
    extern __shared__ __align__(16) uint8_t sb_rows[];
    __shared__ __align__(16) __nv_bfloat16 s_q[2][8][SB_QROW];        // q-, q+ of a group
    __shared__ __align__(16) unsigned s_hist[SB_BINS];
    __shared__ float s_min[SB_RANGES], s_max[SB_RANGES], s_amax[SB_MAX_CLUSTER * NW];
    __shared__ float s_qpart[8];
    __shared__ int s_part[2][NW];
    __shared__ unsigned s_take[SB_MAX_BLOCKS / 32], s_cand[SB_MAX_BLOCKS / 32];      // one bit per block: in, undecided
    __shared__ unsigned long long s_key[SB_CAND];
    __shared__ float s_x[SB_CAND];
    __shared__ int s_blk[SB_CAND];
    __shared__ unsigned s_digit[256];
    __shared__ unsigned long long s_prefix;
    __shared__ int s_ncand, s_winners, s_bin, s_left;
    __shared__ float s_edge[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    int rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    cluster_arrive();                                       // waited for before the first write to another CTA
    const bool shared_set = p.mode == 2, per_qhead = p.mode == 0;
    const int item = blockIdx.x / size;
    const int b = shared_set ? item : item / c.Hkv, g0 = shared_set ? 0 : item - b * c.Hkv, g1 = shared_set ? c.Hkv : g0 + 1;
    const int rows = per_qhead ? c.G : 1;
    const int owners = min(rows, size);
    for (int i = tid; i < SB_BINS; i += NT) s_hist[i] = 0;
    if (tid == 0) { s_ncand = 0; s_winners = 0; }
    pdl_wait();
    pdl_trigger();
    const int len = c.ctx_lens[b];
    const uint32_t a_rows = smem_u32(sb_rows);
    // row slot s of a CTA: the first one lies where its keys go later
    auto row_at = [&](int slot) -> uint32_t { return slot == 0 ? 0u : (uint32_t)p.npad * (4u + 4u * slot); };
    const int n = (max(min(len, c.max_ctx), 0) + TILE - 1) / TILE;
    // blocks that are kept whatever they score
    auto forced = [&](int blk) { return blk < p.keep_first || blk >= n - p.keep_last; };

    float amax = 0.f, mn[2] = {INFINITY, INFINITY}, mx[2] = {-INFINITY, -INFINITY};
    bool first_write = true;
    for (int g = g0; g < g1; ++g) {
        if (g > g0) __syncthreads();
        for (int i = tid; i < 8 * HEAD_DIM / 2; i += NT) {
            const int h = i / (HEAD_DIM / 2), w = i % (HEAD_DIM / 2);
            const uint32_t x = h < c.G ? __ldg(reinterpret_cast<const uint32_t*>(p.q + ((long long)b * c.Hq + g * c.G + h) * HEAD_DIM) + w) : 0u;
            *reinterpret_cast<uint32_t*>(&s_q[0][h][2 * w]) = bmin2(x, 0u);
            *reinterpret_cast<uint32_t*>(&s_q[1][h][2 * w]) = bmax2(x, 0u);
        }
        const float factor = p.k_scale ? __ldg(p.k_scale + g) : 1.f;
        float gmax = 0.f;
        bool staged = false;
        for (int first = (rank * NW + warp) * 16; first < n; first += size * NW * 16) {
            const int r0 = first + gid, r1 = r0 + 8;
            bool on0 = r0 < n, on1 = r1 < n;
            int pg0 = 0, pg1 = 0;
            if (c.paged) {
                const int* row = c.page_table + (long long)b * c.max_pages;
                if (on0) pg0 = __ldg(row + r0);
                if (on1) pg1 = __ldg(row + r1);
                if ((unsigned)pg0 >= (unsigned)c.num_pages) { on0 = false; pg0 = 0; atomicOr(c.status, STATUS_BAD_PAGE); }
                if ((unsigned)pg1 >= (unsigned)c.num_pages) { on1 = false; pg1 = 0; atomicOr(c.status, STATUS_BAD_PAGE); }
            }
            const uint4* src0 = reinterpret_cast<const uint4*>(p.bounds + bounds_row(c, b, on0 ? r0 : 0, pg0, g) * BOUND_ELEMS) + tig;
            const uint4* src1 = reinterpret_cast<const uint4*>(p.bounds + bounds_row(c, b, on1 ? r1 : 0, pg1, g) * BOUND_ELEMS) + tig;
            const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
            uint4 x0[8], x1[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x0[j] = on0 ? __ldg(src0 + 4 * j) : zero;
                x1[j] = on1 ? __ldg(src1 + 4 * j) : zero;
            }
            if (!staged) { asm volatile("bar.sync 1, %0;\n" ::"n"(NT) : "memory"); staged = true; }      // s_q is there
            float s[4] = {0.f, 0.f, 0.f, 0.f};
            uint32_t top = 0u;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint4 q4 = *reinterpret_cast<const uint4*>(&s_q[j >> 2][gid][8 * (tig + 4 * (j & 3))]);
                float d[4] = {0.f, 0.f, 0.f, 0.f}, e[4] = {0.f, 0.f, 0.f, 0.f};
                mma_bf16_16816(d, x0[j].x, x1[j].x, x0[j].y, x1[j].y, q4.x, q4.y);
                mma_bf16_16816(e, x0[j].z, x1[j].z, x0[j].w, x1[j].w, q4.z, q4.w);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += d[i] + e[i];
                const uint32_t all[8] = {x0[j].x, x0[j].y, x0[j].z, x0[j].w, x1[j].x, x1[j].y, x1[j].z, x1[j].w};
#pragma unroll
                for (int i = 0; i < 8; ++i) top = bmax2(top, all[i] & 0x7fff7fffu);
            }
            gmax = fmaxf(gmax, fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xffff0000u)));
            if ((top & 0x7fffu) >= 0x7f80u || (top >> 16) >= 0x7f80u) gmax = INFINITY;    // no bound on the error
            if (first_write) { cluster_wait(); first_write = false; }
            const bool f0 = r0 < n && !forced(r0), f1 = r1 < n && !forced(r1);
            auto range = [&](int i, float v, bool on) {
                if (on) { mn[i] = fminf(mn[i], v); mx[i] = fmaxf(mx[i], fabsf(v) <= 3.4e38f ? v : INFINITY); }
            };
            if (per_qhead) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int col = 2 * tig + i;
                    if (col < c.G) {
                        const int owner = col % size;
                        const uint32_t at = a_rows + row_at(col / size);
                        if (r0 < n) st_cluster(at + 4 * r0, owner, s[i]);
                        if (r1 < n) st_cluster(at + 4 * r1, owner, s[2 + i]);
                        range(i, s[i], f0);
                        range(i, s[2 + i], f1);
                    }
                }
            } else {
                float x = s[0] + s[1], y = s[2] + s[3];
                x += __shfl_xor_sync(0xffffffffu, x, 1); y += __shfl_xor_sync(0xffffffffu, y, 1);
                x += __shfl_xor_sync(0xffffffffu, x, 2); y += __shfl_xor_sync(0xffffffffu, y, 2);
                if (tig == 0) {                             // (the same lane adds the next KV head's part)
                    x *= factor; y *= factor;
                    if (g > g0) {
                        if (r0 < n) x += ld_cluster(a_rows + 4 * r0, 0);
                        if (r1 < n) y += ld_cluster(a_rows + 4 * r1, 0);
                    }
                    if (r0 < n) st_cluster(a_rows + 4 * r0, 0, x);
                    if (r1 < n) st_cluster(a_rows + 4 * r1, 0, y);
                    if (g == g1 - 1) { range(0, x, f0); range(0, y, f1); }
                }
            }
        }
        if (!staged) asm volatile("bar.sync 1, %0;\n" ::"n"(NT) : "memory");
        amax = fmaxf(amax, gmax * fabsf(factor));
        // what e needs of the query: 2^-15 max|q| + (24 + Hkv) 2^-24 sum|q| per head (added up over the KV heads of a shared set)
        if (rank < owners && warp < c.G) {
            float sum = 0.f, big = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float v = __bfloat162float(s_q[1][warp][lane + 32 * i]) - __bfloat162float(s_q[0][warp][lane + 32 * i]);
                sum += v;
                big = fmaxf(big, v);
            }
#pragma unroll
            for (int sh = 16; sh >= 1; sh >>= 1) {
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, sh));
                sum += __shfl_xor_sync(0xffffffffu, sum, sh);
            }
            const float part = big * (1.f / 32768.f) + sum * (float)(24 + c.Hkv) * (1.f / 16777216.f);
            if (lane == 0) s_qpart[warp] = g > g0 ? s_qpart[warp] + part : part;
        }
    }
    if (first_write) cluster_wait();
#pragma unroll
    for (int sh = 16; sh >= 4; sh >>= 1) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            mn[i] = fminf(mn[i], __shfl_xor_sync(0xffffffffu, mn[i], sh));
            mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], sh));
        }
    }
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, sh));
    if (gid == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int col = 2 * tig + i;
            if (col < rows) {
                const uint32_t at = 4 * (((col / size) * size + rank) * NW + warp);
                st_cluster(smem_u32(s_min) + at, col % size, mn[i]);
                st_cluster(smem_u32(s_max) + at, col % size, mx[i]);
            }
        }
    }
    if (lane < owners) st_cluster(smem_u32(s_amax) + 4 * (rank * NW + warp), lane, amax);
    cluster_arrive();                                       // every score of the item is where it belongs ...
    const int kk = min(p.m, n), words = (n + 31) / 32;
    if (g0 == 0 && rank == 0 && tid == 0 && p.idx_count) p.idx_count[b] = kk;
    const int nforced = (int)min((long long)n, (long long)p.keep_first + p.keep_last), need = kk - nforced;
    const bool plain = need <= 0 || kk == n;               // every block, or the first kk of the kept ones
    auto clear_bits = [&]() {
        for (int w = tid; w < words; w += NT) {
            auto span = [&](int from, int to) -> unsigned {        // bits of this word for blocks from .. to - 1
                const int f = max(from - 32 * w, 0), t = min(to - 32 * w, 32);
                return f < t ? (0xffffffffu >> (32 - (t - f))) << f : 0u;
            };
            s_take[w] = kk == n ? span(0, n) : span(0, min(p.keep_first, n)) | span(max(n - p.keep_last, 0), n);
            s_cand[w] = 0;
        }
    };
    clear_bits();
    cluster_wait();                                         // ... and nobody touches another CTA's memory from here on
    if (rank >= owners) return;
    __syncthreads();

    for (int row = rank, slot = 0; row < rows; row += size, ++slot) {
        const int h0 = per_qhead ? g0 * c.G + row : g0 * c.G, h1 = per_qhead ? h0 + 1 : g1 * c.G;
        const int hi = per_qhead ? h0 : (shared_set ? 0 : g0), Hi = per_qhead ? c.Hq : (shared_set ? 1 : c.Hkv);
        int* const out = p.idx + ((long long)b * Hi + hi) * p.m;
        const float* const x = reinterpret_cast<const float*>(sb_rows + row_at(slot));
        unsigned long long* const keys = reinterpret_cast<unsigned long long*>(sb_rows);
        if (slot > 0) {
            for (int i = tid; i < SB_BINS; i += NT) s_hist[i] = 0;
            if (tid == 0) { s_ncand = 0; s_winners = 0; }
            clear_bits();
            __syncthreads();
        }
        for (int i = kk + tid; i < p.m; i += NT) out[i] = -1;
        if (!plain) {
            // ---- this thread's scores; range of the row and error bound, by every warp for itself ------------------
            float v[VECS][4];
            unsigned open = 0;                              // bit 4 j + u: v[j][u] is a block that may be chosen
#pragma unroll
            for (int j = 0; j < VECS; ++j) {
                const int at = (j * NT + tid) * 4;
                if (at < n) {                               // rows have room for a multiple of 32 blocks
                    const float4 t = *reinterpret_cast<const float4*>(x + at);
                    v[j][0] = t.x; v[j][1] = t.y; v[j][2] = t.z; v[j][3] = t.w;
#pragma unroll
                    for (int u = 0; u < 4; ++u) if (at + u < n && !forced(at + u)) open |= 1u << (4 * j + u);
                }
            }
            float lo = INFINITY, hi_s = -INFINITY, big = 0.f, qsum = 0.f;
            for (int i = lane; i < size * NW; i += 32) {
                lo = fminf(lo, s_min[slot * size * NW + i]);
                hi_s = fmaxf(hi_s, s_max[slot * size * NW + i]);
                big = fmaxf(big, s_amax[i]);
            }
#pragma unroll
            for (int sh = 16; sh >= 1; sh >>= 1) {
                lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, sh));
                hi_s = fmaxf(hi_s, __shfl_xor_sync(0xffffffffu, hi_s, sh));
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, sh));
            }
            if (per_qhead) qsum = s_qpart[row];
            else for (int h = 0; h < c.G; ++h) qsum += s_qpart[h];
            const float two_e = 2.01f * big * qsum, width = (hi_s - lo) / (float)(SB_BINS - 1);
            const float inv = 1.f / width;
            const bool all = !(hi_s <= 3.4e38f) || !(lo >= -3.4e38f) || !(two_e <= 3.4e38f) || !(width > 0.f) || !(inv <= 3.4e38f) || !(width <= 3.4e38f);
            float sure = INFINITY, least = -INFINITY;       // above the first: in; below the second: out
            if (!all) {
#pragma unroll
                for (int j = 0; j < VECS; ++j)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        if ((open >> (4 * j + u)) & 1u)
                            atomicAdd(&s_hist[max(0, min(SB_BINS - 1, __float2int_rd((v[j][u] - lo) * inv)))], 1u);
                __syncthreads();
                // the bin t of the need-th largest: counts from the top
                constexpr int PER = SB_BINS / NT;
                int h[PER], cnt = 0;
#pragma unroll
                for (int u = 0; u < PER; u += 4) {
                    const uint4 w = *reinterpret_cast<const uint4*>(&s_hist[SB_BINS - 4 - (tid * PER + u)]);
                    h[u] = w.w; h[u + 1] = w.z; h[u + 2] = w.y; h[u + 3] = w.x;
                    cnt += w.x + w.y + w.z + w.w;
                }
                int above = cta_scan<NT>(cnt, s_part[0]);
#pragma unroll
                for (int u = 0; u < PER; ++u) {
                    if (above < need && above + h[u] >= need) s_bin = SB_BINS - 1 - (tid * PER + u);
                    above += h[u];
                }
                __syncthreads();
                // Edges of the bin, moved outwards by 2 e and by more than what the binning rounds: (v - lo) inv and lo + t width
                // are each within a few 2^-24 of |lo| + |hi| in terms of v.
                const int t = s_bin;
                const float slack = two_e + (fabsf(lo) + fabsf(hi_s)) * (1.f / 1048576.f);
                if (t < SB_BINS - 1) sure = lo + (float)(t + 1) * width + slack;
                if (t > 0) least = lo + (float)t * width - slack;
            }
            // ---- in, out or undecided --------------------------------------------------------------------------------
            int winners = 0;
#pragma unroll
            for (int j = 0; j < VECS; ++j) {
                const int at = (j * NT + tid) * 4;
                if (at < n) {
                    unsigned in = 0, und = 0;
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        if ((open >> (4 * j + u)) & 1u) {
                            if (!all && v[j][u] > sure) in |= 1u << u;
                            else if (all || v[j][u] >= least) und |= 1u << u;
                        }
                    }
                    if (in) { atomicOr(&s_take[at >> 5], in << (at & 31)); winners += __popc(in); }
                    if (und) {
                        atomicOr(&s_cand[at >> 5], und << (at & 31));
                        int place = atomicAdd(&s_ncand, __popc(und));
#pragma unroll
                        for (int u = 0; u < 4; ++u)
                            if ((und >> u) & 1u) {
                                if (place < SB_CAND) { s_x[place] = v[j][u]; s_blk[place] = at + u; }
                                ++place;
                            }
                    }
                }
            }
            winners = __reduce_add_sync(0xffffffffu, winners);
            if (lane == 0 && winners) atomicAdd(&s_winners, winners);
            __syncthreads();
            const int ncand = s_ncand, want = need - s_winners;        // 1 <= want <= ncand
            auto take = [&](int blk) { atomicOr(&s_take[blk >> 5], 1u << (blk & 31)); };
            if (want == ncand) {
                for (int w = tid; w < words; w += NT) s_take[w] |= s_cand[w];
            } else if (!all && ncand <= SB_CAND) {
                // ranks by x; the want-th and the next
                int place = 0;
                if (tid < ncand) {
                    const float mine = s_x[tid];
                    const int blk = s_blk[tid];
                    for (int j = 0; j < ncand; ++j) place += s_x[j] > mine || (s_x[j] == mine && s_blk[j] < blk);
                    if (place == want - 1) s_edge[0] = mine;
                    if (place == want) s_edge[1] = mine;
                }
                __syncthreads();
                const float edge = s_edge[0];
                if (edge - s_edge[1] > two_e) {
                    if (tid < ncand && place < want) take(s_blk[tid]);
                } else {
                    // 64 bits for those within 2e of the border; the others are certain
                    for (int i = warp; i < ncand; i += NW) {
                        const float d = s_x[i] - edge;
                        unsigned long long k = d > 0.f ? ~0ull : 0ull;
                        if (fabsf(d) <= two_e) k = wide_key(wide_score(p, b, h0, h1, s_blk[i], lane));
                        if (lane == 0) s_key[i] = k;
                    }
                    __syncthreads();
                    if (tid < ncand) {
                        const unsigned long long k = s_key[tid];
                        const int blk = s_blk[tid];
                        int before = 0;
                        for (int j = 0; j < ncand; ++j) before += s_key[j] > k || (s_key[j] == k && s_blk[j] < blk);
                        if (before < want) take(blk);
                    }
                }
            } else {
                // ---- all undecided blocks in 64 bits; the want-th largest key eight bits at a time from the top --------
                // (the keys lie over the row, whose fp32 scores are not read any more)
                for (int w = warp; w < words; w += NW)
                    for (unsigned m = s_cand[w]; m; m &= m - 1) {
                        const int blk = w * 32 + __ffs(m) - 1;
                        const unsigned long long k = wide_key(wide_score(p, b, h0, h1, blk, lane));
                        if (lane == 0) keys[blk] = k;
                    }
                if (tid == 0) { s_prefix = 0ull; s_left = want; }
                for (int shift = 56; shift >= 0; shift -= 8) {
                    if (tid < 256) s_digit[tid] = 0;
                    __syncthreads();
                    const unsigned long long prefix = s_prefix;
                    for (int i = tid; i < n; i += NT) {
                        if (!((s_cand[i >> 5] >> (i & 31)) & 1u)) continue;
                        const unsigned long long k = keys[i];
                        if (shift == 56 || (k >> (shift + 8)) == prefix) atomicAdd(&s_digit[(unsigned)(k >> shift) & 255u], 1u);
                    }
                    __syncthreads();
                    if (tid == 0) {
                        int left = s_left, d = 255;
                        while (d > 0 && (int)s_digit[d] < left) left -= s_digit[d--];
                        s_prefix = (prefix << 8) | (unsigned)d;
                        s_left = left;
                    }
                    __syncthreads();
                }
                // larger ones are in, and as many of the equal ones as are wanted, the lower first
                const unsigned long long border = s_prefix;
                const int ties = s_left;
                constexpr int WPT = SB_MAX_BLOCKS / 32 / NT;
                unsigned in[WPT], equal[WPT];
                int mine = 0;
#pragma unroll
                for (int u = 0; u < WPT; ++u) {
                    const int w = tid * WPT + u;
                    in[u] = equal[u] = 0;
                    if (w < words)
                        for (unsigned m = s_cand[w]; m; m &= m - 1) {
                            const unsigned long long k = keys[w * 32 + __ffs(m) - 1];
                            if (k > border) in[u] |= m & (~m + 1u);
                            else if (k == border) equal[u] |= m & (~m + 1u);
                        }
                    mine += __popc(equal[u]);
                }
                int before = cta_scan<NT>(mine, s_part[0]);
#pragma unroll
                for (int u = 0; u < WPT; ++u) {
                    for (unsigned m = equal[u]; m; m &= m - 1) if (before++ < ties) in[u] |= m & (~m + 1u);
                    if (tid * WPT + u < words) s_take[tid * WPT + u] |= in[u];
                }
            }
            __syncthreads();
        }
        // ---- the chosen blocks in ascending order --------------------------------------------------------------------
        constexpr int WPT = SB_MAX_BLOCKS / 32 / NT;
        unsigned bits[WPT];
        int mine = 0;
#pragma unroll
        for (int u = 0; u < WPT; ++u) {
            bits[u] = tid * WPT + u < words ? s_take[tid * WPT + u] : 0u;
            mine += __popc(bits[u]);
        }
        int pos = cta_scan<NT>(mine, s_part[1]);
#pragma unroll
        for (int u = 0; u < WPT; ++u)
            for (unsigned m = bits[u]; m && pos < kk; m &= m - 1) out[pos++] = (tid * WPT + u) * 32 + __ffs(m) - 1;
        __syncthreads();                                    // the next row uses the same arrays
    }
}

// ---- attention over listed blocks ------------------------------------------------------------------------------
// Item = (sequence, KV head), or (sequence, query head) where every query head has its own list. A thread-block cluster
// serves an item: its warps take the listed blocks in turn, each with a private cp.async ring (no CTA barrier on the
// streaming path), the CTAs merge their (max, sum, O) through distributed shared memory. So the kernel
// needs no scratch memory, no counters and no second launch. The matrix instructions have positions as rows and the group's
// heads as columns: S^T = K Q^T, O^T += V^T P^T, so K and V are read once per KV head. The softmax weights enter the second product as the sum
// of two 16-bit numbers (bf16 over a bf16 cache, fp16 over an 8-bit one): 2^-16 relative instead of 2^-8 for
// one, for eight more matrix instructions per block on a path that waits for memory.
struct BlockAttnParams {
    BlockCache c;
    const __nv_bfloat16* q;
    void* out;
    int out_bf16;
    const int* idx;
    const int* idx_count;
    int m, Hi;
    float scale_log2;
    const float* k_scale;
    const float* v_scale;
};

struct BlockAcc {
    float m[2], l[2];
    float o[8][4];
};

// Raises the running maxima to cover this block's scaled logits; all lanes that share a tig agree afterwards.
__device__ __forceinline__ void raise_max(BlockAcc& acc, float mx0, float mx1) {
    if (__any_sync(0xffffffffu, (mx0 > acc.m[0]) || (mx1 > acc.m[1]))) {
#pragma unroll
        for (int sh = 4; sh <= 16; sh <<= 1) {
            mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, sh));
            mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, sh));
        }
        const float g0 = fmaxf(acc.m[0], mx0), g1 = fmaxf(acc.m[1], mx1);
        const float a0 = (g0 == -INFINITY) ? 1.f : fast_exp2(acc.m[0] - g0);
        const float a1 = (g1 == -INFINITY) ? 1.f : fast_exp2(acc.m[1] - g1);
        acc.l[0] *= a0;
        acc.l[1] *= a1;
#pragma unroll
        for (int t = 0; t < 8; ++t) { acc.o[t][0] *= a0; acc.o[t][1] *= a1; acc.o[t][2] *= a0; acc.o[t][3] *= a1; }
        acc.m[0] = g0;
        acc.m[1] = g1;
    }
}

// Softmax weights of one block from its scaled logits t (rows gid, gid + 8; this lane's two heads).
__device__ __forceinline__ void block_weights(BlockAcc& acc, const float (&s)[4], float scale_log2, int nvalid, int gid, float (&w)[4]) {
    const bool v0 = gid < nvalid, v1 = gid + 8 < nvalid;
    const float t0 = v0 ? s[0] * scale_log2 : -INFINITY, t1 = v0 ? s[1] * scale_log2 : -INFINITY;
    const float t2 = v1 ? s[2] * scale_log2 : -INFINITY, t3 = v1 ? s[3] * scale_log2 : -INFINITY;
    raise_max(acc, fmaxf(t0, t2), fmaxf(t1, t3));
    const float m0 = (acc.m[0] == -INFINITY) ? 0.f : acc.m[0], m1 = (acc.m[1] == -INFINITY) ? 0.f : acc.m[1];
    w[0] = fast_exp2(t0 - m0); w[1] = fast_exp2(t1 - m1);
    w[2] = fast_exp2(t2 - m0); w[3] = fast_exp2(t3 - m1);
    acc.l[0] += w[0] + w[2];
    acc.l[1] += w[1] + w[3];
}

// One block of a bf16 cache: 16 key rows at ks, 16 value rows at vs, 256 bytes each, piece c of row r at c ^ (r & 7).
__device__ __forceinline__ void consume_block(uint32_t ks, uint32_t vs, const uint32_t (&qf)[8][2], BlockAcc& acc, float scale_log2,
                                              int nvalid, int lane) {
    const int gid = lane >> 2;
    float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};
    const uint32_t kl = ks + ((lane & 7) + ((lane >> 3) & 1) * 8) * 256 + ((((lane >> 4) & 1) ^ (lane & 7)) << 4);
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
        uint32_t a[4], b[4];
        ldmatrix_x4(kl ^ (j << 5), a);
        ldmatrix_x4(kl ^ ((j + 1) << 5), b);
        mma_bf16_16816(s, a[0], a[1], a[2], a[3], qf[j][0], qf[j][1]);
        mma_bf16_16816(s2, b[0], b[1], b[2], b[3], qf[j + 1][0], qf[j + 1][1]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += s2[i];
    float w[4];
    block_weights(acc, s, scale_log2, nvalid, gid, w);
    const uint32_t h0 = pack_bf16(w[0], w[1]), h1 = pack_bf16(w[2], w[3]);
    const uint32_t l0 = pack_bf16(w[0] - __uint_as_float(h0 << 16), w[1] - __uint_as_float(h0 & 0xffff0000u));
    const uint32_t l1 = pack_bf16(w[2] - __uint_as_float(h1 << 16), w[3] - __uint_as_float(h1 & 0xffff0000u));
    const uint32_t ph0 = movmatrix_trans(h0), ph1 = movmatrix_trans(h1), pl0 = movmatrix_trans(l0), pl1 = movmatrix_trans(l1);
    const int rr = lane & 7, mb = (lane >> 3) & 1;
    const uint32_t vl = vs + (rr + ((lane >> 4) << 3)) * 256 + ((rr ^ mb) << 4);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        uint32_t a[4];
        ldmatrix_x4_trans(vl ^ (t << 5), a);
        mma_bf16_16816(acc.o[t], a[0], a[1], a[2], a[3], ph0, ph1);
        mma_bf16_16816(acc.o[t], a[0], a[1], a[2], a[3], pl0, pl1);
    }
}

__device__ __forceinline__ float f16_lo(uint32_t w) {
    float f;
    asm("{\n.reg .f16 l, h;\nmov.b32 {l, h}, %1;\ncvt.f32.f16 %0, l;\n}\n" : "=f"(f) : "r"(w));
    return f;
}
__device__ __forceinline__ float f16_hi(uint32_t w) { return f16_lo(w >> 16); }

// One block of an 8-bit cache (rows of 128 bytes of codes; layouts and fragment orders as in consume_tile8).
__device__ __forceinline__ void consume_block8(uint32_t ks, uint32_t vs, const uint32_t (&qf)[2][8], BlockAcc& acc, float scale_log2,
                                               int nvalid, int lane) {
    const int gid = lane >> 2, tig = lane & 3;
    float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};
    const uint32_t krow = ks + gid * ROW_BYTES8;
    const uint32_t kswz = (gid & 1) << 2;
#pragma unroll
    for (int sl = 0; sl < 2; ++sl) {
        uint32_t ka[4], kb[4];
        const uint32_t off = ((uint32_t)((tig + 4 * sl) ^ kswz)) << 4;
        lds128(krow + off, ka);
        lds128(krow + 8 * ROW_BYTES8 + off, kb);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a0, a2, a1, a3;
            e4m3x4_to_f16x2x2(ka[i], a0, a2);
            e4m3x4_to_f16x2x2(kb[i], a1, a3);
            if (i & 1) mma_f16_16816(s2, a0, a1, a2, a3, qf[sl][2 * i], qf[sl][2 * i + 1]);
            else mma_f16_16816(s, a0, a1, a2, a3, qf[sl][2 * i], qf[sl][2 * i + 1]);
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] += s2[i];
    float w[4];
    block_weights(acc, s, scale_log2, nvalid, gid, w);
    const uint32_t h0 = pack_f16(w[0], w[1]), h1 = pack_f16(w[2], w[3]);
    const uint32_t l0 = pack_f16(w[0] - f16_lo(h0), w[1] - f16_hi(h0)), l1 = pack_f16(w[2] - f16_lo(h1), w[3] - f16_hi(h1));
    const uint32_t ph0 = movmatrix_trans(h0), ph1 = movmatrix_trans(h1), pl0 = movmatrix_trans(l0), pl1 = movmatrix_trans(l1);
    const int rr = lane & 7, mi = lane >> 3;
    const uint32_t vbase = vs + (rr + ((mi >> 1) << 3)) * ROW_BYTES8;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint32_t m[4];
        ldmatrix_x4_trans(vbase + ((uint32_t)((2 * u + (mi & 1)) ^ rr) << 4), m);
        uint32_t x0, y0, x2, y2, x1, y1, x3, y3;
        e4m3x4_to_f16x2x2(__byte_perm(m[0], 0, 0x3120), x0, y0);
        e4m3x4_to_f16x2x2(__byte_perm(m[2], 0, 0x3120), x2, y2);
        mma_f16_16816(acc.o[2 * u], x0, y0, x2, y2, ph0, ph1);
        mma_f16_16816(acc.o[2 * u], x0, y0, x2, y2, pl0, pl1);
        e4m3x4_to_f16x2x2(__byte_perm(m[1], 0, 0x3120), x1, y1);
        e4m3x4_to_f16x2x2(__byte_perm(m[3], 0, 0x3120), x3, y3);
        mma_f16_16816(acc.o[2 * u + 1], x1, y1, x3, y3, ph0, ph1);
        mma_f16_16816(acc.o[2 * u + 1], x1, y1, x3, y3, pl0, pl1);
    }
}

constexpr int BA_WARPS = 4;
constexpr int BA_STAGES = 3, BA_STAGES8 = 6;                // the same bytes in flight

template <bool KV8>
constexpr size_t ba_smem() { return (size_t)BA_WARPS * (KV8 ? BA_STAGES8 * STAGE_BYTES8 : BA_STAGES * STAGE_BYTES) + 1024; }

template <bool KV8>
__global__ void __launch_bounds__(BA_WARPS * 32, 2) block_attn_kernel(const BlockAttnParams p) {
    constexpr int NW = BA_WARPS, STAGES = KV8 ? BA_STAGES8 : BA_STAGES, SLOT = KV8 ? STAGE_BYTES8 : STAGE_BYTES;
    const BlockCache& c = p.c;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
    __shared__ float s_mo[8][HEAD_DIM];                     // this CTA's un-normalised output rows
    __shared__ float s_m[8], s_l[8];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    int rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    const bool per_qhead = p.Hi == c.Hq;
    const int IY = per_qhead ? c.Hq : c.Hkv;
    const int item = blockIdx.x / size, b = item / IY, y = item - b * IY;
    const int g = per_qhead ? y / c.G : y;
    const int head0 = per_qhead ? y : g * c.G, ncols = per_qhead ? 1 : c.G;
    const int* row = p.idx + ((long long)b * p.Hi + (per_qhead ? y : (p.Hi == c.Hkv ? g : 0))) * p.m;
    pdl_wait();
    pdl_trigger();

    const int n = cached_len(c, b);
    const int cnt = p.idx_count ? min(p.idx_count[b], p.m) : p.m;
    const int stride = size * NW, me = rank * NW + warp;
    // blocks of this warp: list entries me + i * stride; lane l keeps what entry l of a run of 32 needs
    long long my_off = 0;
    int my_rows = 0;
    auto look_up = [&](int run) {
        const long long e = (long long)me + (long long)(run * 32 + lane) * stride;
        const int blk = e < cnt ? __ldg(row + e) : -1;
        my_rows = 0;
        my_off = 0;
        if (blk < -1 || (blk >= 0 && (long long)blk * TILE >= n)) atomicOr(c.status, STATUS_BAD_INDEX);
        else if (blk >= 0) {
            my_rows = min(TILE, n - blk * TILE);
            my_off = (long long)g * c.stride_head;
            if (c.paged) {
                const int page = __ldg(c.page_table + (long long)b * c.max_pages + blk);
                if ((unsigned)page < (unsigned)c.num_pages) my_off += (long long)page * c.stride_page;
                else { my_rows = 0; my_off = 0; atomicOr(c.status, STATUS_BAD_PAGE); }
            } else {
                my_off += (long long)b * c.stride_b + (long long)blk * TILE * c.stride_pos;
            }
        }
    };
    const int count = cnt > me ? (cnt - me + stride - 1) / stride : 0;
    look_up(0);
    const uint32_t ring = smem_u32(smem) + warp * STAGES * SLOT;
    const uint64_t policy = l2_evict_first_policy();
    const int c16 = lane & 15, rhalf = lane >> 4;           // bf16: piece c16 of rows rhalf + 2 i
    const int p8 = lane & 7, r8 = lane >> 3;                // codes: piece p8 of rows r8 + 4 i
    int issued = 0;
    int rows_of[STAGES];                                    // valid rows of the block in each slot
#pragma unroll
    for (int s = 0; s < STAGES; ++s) rows_of[s] = 0;
    auto issue = [&](uint32_t slot) -> int {
        int rows = 0;
        if (issued < count) {
            if (issued > 0 && (issued & 31) == 0) look_up(issued >> 5);
            rows = __shfl_sync(0xffffffffu, my_rows, issued & 31);
            const long long off = __shfl_sync(0xffffffffu, my_off, issued & 31);
            if (rows > 0) {
                if constexpr (KV8) {
                    const long long src = off + r8 * c.stride_pos + p8 * 16;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = r8 + 4 * i;
                        const bool on = r < rows;
                        const long long o = on ? src + 4 * i * c.stride_pos : 0;
                        cp_async16_hint(slot + r * ROW_BYTES8 + ((p8 ^ ((r & 1) << 2)) << 4), c.k + o, on ? 16 : 0, policy);
                        cp_async16_hint(slot + TILE_BYTES8 + r * ROW_BYTES8 + ((p8 ^ (r & 7)) << 4), c.v + o, on ? 16 : 0, policy);
                    }
                } else {
                    const long long src = 2 * (off + rhalf * c.stride_pos + c16 * 8);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int r = rhalf + 2 * i;
                        const bool on = r < rows;
                        const long long o = on ? src + 4 * i * c.stride_pos : 0;
                        const uint32_t d = slot + r * 256 + ((c16 ^ (r & 7)) << 4);
                        cp_async16_hint(d, c.k + o, on ? 16 : 0, policy);
                        cp_async16_hint(d + TILE_BYTES, c.v + o, on ? 16 : 0, policy);
                    }
                }
            }
            ++issued;
        }
        cp_async_commit();
        return rows;
    };
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) rows_of[s] = issue(ring + s * SLOT);

    uint32_t qf[8][2];
    uint32_t qf8[2][8];
    {
        const __nv_bfloat16* qrow = p.q + ((long long)b * c.Hq + head0 + min(gid, ncols - 1)) * HEAD_DIM;
        const bool on = gid < ncols;
        if constexpr (KV8) {
            const uint4* qp = reinterpret_cast<const uint4*>(qrow);
#pragma unroll
            for (int sl = 0; sl < 2; ++sl) {
                const int pc = tig + 4 * sl;
                const uint4 t0 = __ldg(qp + 2 * pc), t1 = __ldg(qp + 2 * pc + 1);
                const uint32_t w[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) qf8[sl][i] = on ? bf16x2_to_f16x2(w[i]) : 0u;
            }
        } else {
            const uint32_t* qw = reinterpret_cast<const uint32_t*>(qrow);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t w0 = __ldg(qw + 8 * j + tig), w1 = __ldg(qw + 8 * j + 4 + tig);
                qf[j][0] = on ? w0 : 0u;
                qf[j][1] = on ? w1 : 0u;
            }
        }
    }
    const float scale_log2 = p.scale_log2 * ((KV8 && p.k_scale) ? __ldg(p.k_scale + g) : 1.f);
    const float vscale = (KV8 && p.v_scale) ? __ldg(p.v_scale + g) : 1.f;
    BlockAcc acc;
    acc.m[0] = acc.m[1] = -INFINITY;
    acc.l[0] = acc.l[1] = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) { acc.o[t][0] = acc.o[t][1] = acc.o[t][2] = acc.o[t][3] = 0.f; }

    for (int it = 0; it < count;) {
#pragma unroll
        for (int s = 0; s < STAGES; ++s) {
            if (it < count) {
                cp_async_wait<STAGES - 2>();
                __syncwarp();                               // ... for every lane; the slot refilled next is done with
                constexpr int back = STAGES - 1;
                rows_of[(s + back) % STAGES] = issue(ring + ((s + back) % STAGES) * SLOT);
                const uint32_t ks = ring + s * SLOT;
                if (rows_of[s] > 0) {
                    if constexpr (KV8) consume_block8(ks, ks + TILE_BYTES8, qf8, acc, scale_log2, rows_of[s], lane);
                    else consume_block(ks, ks + TILE_BYTES, qf, acc, scale_log2, rows_of[s], lane);
                }
                ++it;
            }
        }
    }
    cp_async_wait<0>();

    // ---- merge: the warps of the CTA through its shared memory, then the CTAs of the cluster ------------------------
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
        acc.l[0] += __shfl_xor_sync(0xffffffffu, acc.l[0], sh);
        acc.l[1] += __shfl_xor_sync(0xffffffffu, acc.l[1], sh);
    }
    __syncthreads();                                        // all rings drained; their memory is used again
    float* mo = reinterpret_cast<float*>(smem);             // [NW][8][128]
    float2* mml = reinterpret_cast<float2*>(smem + NW * 8 * HEAD_DIM * 4);
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        float* w0 = mo + (warp * 8 + 2 * tig) * HEAD_DIM;
        float* w1 = w0 + HEAD_DIM;
        // fragment rows: d = 16 t + gid and + 8; over an 8-bit cache d = 16 t + 2 gid and + 1
        const int d0 = KV8 ? 16 * t + 2 * gid : 16 * t + gid, d1 = KV8 ? d0 + 1 : d0 + 8;
        w0[d0] = acc.o[t][0] * vscale; w1[d0] = acc.o[t][1] * vscale;
        w0[d1] = acc.o[t][2] * vscale; w1[d1] = acc.o[t][3] * vscale;
    }
    if (gid == 0) {
        mml[warp * 8 + 2 * tig] = make_float2(acc.m[0], acc.l[0]);
        mml[warp * 8 + 2 * tig + 1] = make_float2(acc.m[1], acc.l[1]);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < ncols * HEAD_DIM; e += NW * 32) {
        const int col = e >> 7, d = e & 127;
        float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, mml[w * 8 + col].x);
        // (a warp whose logits are all NaN has no maximum but a sum that is NaN: it goes in with factor 0)
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float2 ml = mml[w * 8 + col];
            const float f = (ml.x == -INFINITY) ? 0.f : fast_exp2(ml.x - M);
            L += ml.y * f;
            O += mo[(w * 8 + col) * HEAD_DIM + d] * f;
        }
        if (size == 1) {
            const float r = (L != 0.f) ? O / L : 0.f;
            const long long at = ((long long)b * c.Hq + head0 + col) * HEAD_DIM + d;
            if (p.out_bf16) reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(r);
            else reinterpret_cast<float*>(p.out)[at] = r;
        } else {
            s_mo[col][d] = O;
            if (d == 0) { s_m[col] = M; s_l[col] = L; }
        }
    }
    if (size == 1) return;
    cluster_arrive();
    cluster_wait();
    const uint32_t amo = smem_u32(&s_mo[0][0]), am = smem_u32(s_m), al = smem_u32(s_l);
    for (int e = rank * NW * 32 + threadIdx.x; e < ncols * HEAD_DIM; e += size * NW * 32) {
        const int col = e >> 7, d = e & 127;
        float M = -INFINITY, L = 0.f, O = 0.f;
        for (int r = 0; r < size; ++r) M = fmaxf(M, ld_cluster(am + 4 * col, r));
        for (int r = 0; r < size; ++r) {
            const float mr = ld_cluster(am + 4 * col, r), lr = ld_cluster(al + 4 * col, r);
            const float o = ld_cluster(amo + 4 * e, r);
            const float f = (mr == -INFINITY) ? 0.f : fast_exp2(mr - M);
            L += lr * f;
            O += o * f;
        }
        const float r = (L != 0.f) ? O / L : 0.f;
        const long long at = ((long long)b * c.Hq + head0 + col) * HEAD_DIM + d;
        if (p.out_bf16) reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(r);
        else reinterpret_cast<float*>(p.out)[at] = r;
    }
    cluster_arrive();
    cluster_wait();                                         // nobody leaves while its shared memory is read
}

}  // namespace tidal
