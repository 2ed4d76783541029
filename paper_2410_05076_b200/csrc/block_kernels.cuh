// Block-sparse decode attention: blocks of 16 positions (one page) ranked by an upper bound of their logits.
//
//   block_bounds_kernel  per block and KV head the channelwise least and greatest key (lo, hi), in bf16 (exact)
//   block_score_kernel   s = sum_c max(q_c lo_c, q_c hi_c) >= q . k for every key k of the block
//   block_topk_kernel    the m blocks with the largest s per index head, exactly, ties toward the lower block
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

// ---- block scores ----------------------------------------------------------------------------------------------
// sum_c max(q_c lo_c, q_c hi_c) = q+ . hi + q- . lo with q+ = max(q, 0), q- = min(q, 0): two products, so one pair of
// matrix instructions serves 16 blocks and the whole group of query heads. A warp takes 16 blocks x 512 bytes straight
// into the registers that are its A fragments (the contraction index may be relabelled: lane (gid, tig) holds the
// 16-byte pieces tig + 4 j of rows gid and gid + 8). Bound by memory; the result is an approximation in fp32 whose
// error the ranking kernel bounds (see there) from the largest |bound| that each CTA finds on the way.
struct ScoreParams {
    BlockCache c;
    const __nv_bfloat16* q;
    const __nv_bfloat16* bounds;
    const float* k_scale;                                   // factors of the KV heads where several of them are added up (or null)
    int group_sum;                                          // one row per KV head: the sum of its query heads' scores
    float* scores;                                          // [batch, Hq or Hkv, stride]
    long long stride;
    float* amax;                                            // [batch, Hkv, chunks] largest |bound| of the chunk
    int chunks;
};

constexpr int BS_WARPS = 4;
constexpr int BS_BLOCKS = BS_WARPS * 16;                    // blocks per CTA

__global__ void __launch_bounds__(BS_WARPS * 32) block_score_kernel(const ScoreParams p) {
    const BlockCache& c = p.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    pdl_wait();
    pdl_trigger();
    const int pair = blockIdx.x / p.chunks, chunk = blockIdx.x - pair * p.chunks;
    const int b = pair / c.Hkv, g = pair - b * c.Hkv;
    const int nblk = (cached_len(c, b) + TILE - 1) / TILE;
    const int first = chunk * BS_BLOCKS + warp * 16;
    __shared__ float s_amax[BS_WARPS];
    float amax = 0.f;
    if (first < nblk) {
        uint4 a[2][8];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int blk = first + gid + 8 * r;
            bool on = blk < nblk;
            int page = 0;
            if (on && c.paged) {
                page = __ldg(c.page_table + (long long)b * c.max_pages + blk);
                if ((unsigned)page >= (unsigned)c.num_pages) { on = false; atomicOr(c.status, STATUS_BAD_PAGE); }
            }
            const uint4* src = reinterpret_cast<const uint4*>(p.bounds + bounds_row(c, b, on ? blk : 0, page, g) * BOUND_ELEMS) + tig;
#pragma unroll
            for (int j = 0; j < 8; ++j) a[r][j] = on ? __ldg(src + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
        }
        float s[4] = {0.f, 0.f, 0.f, 0.f}, s2[4] = {0.f, 0.f, 0.f, 0.f};
        const uint4* qp = reinterpret_cast<const uint4*>(p.q + ((long long)b * c.Hq + g * c.G + min(gid, c.G - 1)) * HEAD_DIM) + tig;
        uint32_t mx = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint4 q4 = __ldg(qp + 4 * j);
            const uint32_t qw[4] = {q4.x, q4.y, q4.z, q4.w};
            uint32_t neg[4], pos[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                neg[i] = gid < c.G ? bmin2(qw[i], 0u) : 0u;
                pos[i] = gid < c.G ? bmax2(qw[i], 0u) : 0u;
            }
            const uint4 l0 = a[0][j], l1 = a[1][j], h0 = a[0][j + 4], h1 = a[1][j + 4];
            mma_bf16_16816(s, l0.x, l1.x, l0.y, l1.y, neg[0], neg[1]);
            mma_bf16_16816(s2, h0.x, h1.x, h0.y, h1.y, pos[0], pos[1]);
            mma_bf16_16816(s, l0.z, l1.z, l0.w, l1.w, neg[2], neg[3]);
            mma_bf16_16816(s2, h0.z, h1.z, h0.w, h1.w, pos[2], pos[3]);
            const uint32_t all[16] = {l0.x, l0.y, l0.z, l0.w, l1.x, l1.y, l1.z, l1.w, h0.x, h0.y, h0.z, h0.w, h1.x, h1.y, h1.z, h1.w};
#pragma unroll
            for (int i = 0; i < 16; ++i) mx = bmax2(mx, all[i] & 0x7fff7fffu);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] += s2[i];
        amax = fmaxf(__uint_as_float(mx << 16), __uint_as_float(mx & 0xffff0000u));
        if ((mx & 0x7fffu) > 0x7f80u || (mx >> 16) > 0x7f80u) amax = INFINITY;      // not a number: no bound on the error
        const int r0 = first + gid, r1 = r0 + 8;
        if (p.group_sum) {
            float x = s[0] + s[1], y = s[2] + s[3];
            x += __shfl_xor_sync(0xffffffffu, x, 1); y += __shfl_xor_sync(0xffffffffu, y, 1);
            x += __shfl_xor_sync(0xffffffffu, x, 2); y += __shfl_xor_sync(0xffffffffu, y, 2);
            const float f = p.k_scale ? __ldg(p.k_scale + g) : 1.f;
            float* row = p.scores + ((long long)b * c.Hkv + g) * p.stride;
            if (tig == 0) {
                if (r0 < nblk) row[r0] = x * f;
                if (r1 < nblk) row[r1] = y * f;
            }
        } else {
            float* row = p.scores + ((long long)b * c.Hq + g * c.G) * p.stride;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = 2 * tig + i;
                if (col < c.G) {
                    if (r0 < nblk) row[col * p.stride + r0] = s[i];
                    if (r1 < nblk) row[col * p.stride + r1] = s[2 + i];
                }
            }
        }
    }
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, sh));
    if (lane == 0) s_amax[warp] = amax;
    __syncthreads();
    if (threadIdx.x == 0) {
        float m = s_amax[0];
#pragma unroll
        for (int w = 1; w < BS_WARPS; ++w) m = fmaxf(m, s_amax[w]);
        p.amax[(long long)pair * p.chunks + chunk] = m;
    }
}

// ---- the m best blocks -----------------------------------------------------------------------------------------
// One CTA per (sequence, index head), sixteen scores per thread in registers. The set is the one that the scores in 64 bits
// give. From the fp32 scores x, each within e of its true value, one histogram over the row's range gives the bin of the
// need-th largest x, t say: a block with bin(x - 2e) > t is in for certain (x - 2e exceeds the need-th largest x,
// whose true value exceeds no less than need true values by more than e), one with bin(x + 2e) < t is out for certain;
// bin() is monotone, so rounding in it does no harm. What is left, a handful of blocks next to the border, is evaluated in 64 bits
// from the bounds and ranked by (score, lower block first).
//   e: a matrix instruction adds 16 exact products and an accumulator with an error of at most 2^-22 of the sum of their
// magnitudes; at most 16 follow each other, the final additions (a group's heads, KV heads, their factors) add 2^-24
// each: together below 2^-17 of sum_c |q_c| max|bound|, taken as 2^-16.
// Rows whose scores or error bound are not finite, or whose range is empty, evaluate every block in 64 bits.
struct TopBlocksParams {
    BlockCache c;
    const __nv_bfloat16* q;
    const __nv_bfloat16* bounds;
    const float* k_scale;                                   // as in ScoreParams
    const float* scores;
    long long stride;
    const float* amax;
    int chunks;
    int rows, Hi;                                           // score rows per sequence, index heads
    int m, keep_first, keep_last;
    int* idx;
    int* idx_count;
    unsigned long long* wide;                               // [batch, Hi, max_blocks] keys in 64 bits where they do not fit shared memory
    int* wide_blk;
};

constexpr int TB_BINS = 2048;
constexpr int TB_PER = 16;                                  // blocks per thread
constexpr int TB_CAND = 1024;                               // candidates kept in shared memory
constexpr int TB_RANK = 192;                                // candidates ranked by counting

// Larger double <=> larger key; not-a-number above everything, -0 as +0.
__device__ __forceinline__ unsigned long long wide_key(double s) {
    s += 0.0;
    if (s != s) return ~0ull;
    const unsigned long long u = (unsigned long long)__double_as_longlong(s);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}

template <int NT>
__device__ __forceinline__ int block_scan(int v, int* s_part, int& total) {        // exclusive prefix sum over the CTA
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int x = v;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, x, sh);
        if (lane >= sh) x += y;
    }
    __syncthreads();                                        // s_part may still be read from the last call
    if (lane == 31) s_part[warp] = x;
    __syncthreads();
    int w = lane < NT / 32 ? s_part[lane] : 0;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, w, sh);
        if (lane >= sh) w += y;
    }
    total = __shfl_sync(0xffffffffu, w, NT / 32 - 1);
    const int before = __shfl_sync(0xffffffffu, w, max(warp - 1, 0));
    return x - v + (warp > 0 ? before : 0);
}

// One candidate's score in 64 bits, by a warp: every lane four channels of each member head.
__device__ __forceinline__ double wide_score(const TopBlocksParams& p, int b, int h0, int h1, int blk, int lane) {
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
        const uint2 l2 = __ldg(bp), h2 = __ldg(bp + 32);
        double lo[4], hi[4], part = 0.0;
        const uint32_t lw[2] = {l2.x, l2.y}, hw[2] = {h2.x, h2.y};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            lo[2 * i] = __uint_as_float(lw[i] << 16); lo[2 * i + 1] = __uint_as_float(lw[i] & 0xffff0000u);
            hi[2 * i] = __uint_as_float(hw[i] << 16); hi[2 * i + 1] = __uint_as_float(hw[i] & 0xffff0000u);
        }
        for (; h < h1 && h < (g + 1) * c.G; ++h) {
            const uint2 q2 = __ldg(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h) * HEAD_DIM) + lane);
            const uint32_t qw[2] = {q2.x, q2.y};
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const double q0 = __uint_as_float(qw[i] << 16), q1 = __uint_as_float(qw[i] & 0xffff0000u);
                const double x0 = q0 * lo[2 * i], y0 = q0 * hi[2 * i], x1 = q1 * lo[2 * i + 1], y1 = q1 * hi[2 * i + 1];
                part += (x0 > y0 || x0 != x0) ? x0 : y0;
                part += (x1 > y1 || x1 != x1) ? x1 : y1;
            }
        }
        acc += p.k_scale ? part * (double)__ldg(p.k_scale + g) : part;
    }
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, sh);
    return acc;
}

template <int NT>
__global__ void __launch_bounds__(NT) block_topk_kernel(const TopBlocksParams p) {
    const BlockCache& c = p.c;
    constexpr int NW = NT / 32;
    __shared__ unsigned s_hist[TB_BINS];
    __shared__ unsigned long long s_key[TB_CAND];
    __shared__ int s_blk[TB_CAND];
    __shared__ unsigned s_take[NT * TB_PER / 32];           // candidates that made it, one bit per block
    __shared__ unsigned s_tie[NT * TB_PER / 32];
    __shared__ float s_red[3][NW];
    __shared__ int s_part[NW];
    __shared__ int s_bin;
    __shared__ unsigned s_digit[256];
    __shared__ unsigned long long s_prefix;
    __shared__ int s_need;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int b = blockIdx.x / p.Hi, hi = blockIdx.x - b * p.Hi;
#pragma unroll
    for (int i = tid; i < TB_BINS; i += NT) s_hist[i] = 0;
    if (tid < NT * TB_PER / 32) { s_take[tid] = 0; s_tie[tid] = 0; }
    if (tid == 0) s_bin = 0;
    pdl_wait();
    pdl_trigger();
    const int n = (cached_len(c, b) + TILE - 1) / TILE;
    const int kk = min(p.m, n);
    const int members = c.Hq / p.Hi, h0 = hi * members, h1 = h0 + members;
    int* const out = p.idx + ((long long)b * p.Hi + hi) * p.m;
    if (hi == 0 && tid == 0 && p.idx_count) p.idx_count[b] = kk;
    for (int i = kk + tid; i < p.m; i += NT) out[i] = -1;
    const int base = tid * TB_PER;
    // blocks that are kept whatever they score
    auto forced = [&](int blk) { return blk < p.keep_first || blk >= n - p.keep_last; };
    const int nforced = min((long long)n, (long long)p.keep_first + p.keep_last);
    unsigned mine = 0;                                      // bit i: block base + i is in
    if (kk == n || nforced >= kk) {
        // every block, or the first kk of the kept ones
        int have = 0;
        for (int i = 0; i < TB_PER; ++i) if (base + i < n && (kk == n || forced(base + i))) { mine |= 1u << i; ++have; }
        int total;
        const int before = block_scan<NT>(have, s_part, total);
        int at = before;
        for (int i = 0; i < TB_PER; ++i) if ((mine >> i) & 1u) { if (at < kk) out[at] = base + i; ++at; }
        return;
    }
    const int need = kk - nforced;

    float x[TB_PER];
    unsigned there = 0;                                     // bit i: an unforced block of the row
    {
        const float* row = p.scores + (p.rows == p.Hi ? (long long)b * p.rows + hi : (long long)b * p.rows) * p.stride;
        const int sum_rows = p.rows / p.Hi;
#pragma unroll
        for (int i = 0; i < TB_PER; i += 4) {
            float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
            if (base + i < n) {                             // rows are padded to 16 scores: whole vectors may be read
                for (int r = 0; r < sum_rows; ++r) {
                    const float4 u = __ldcg(reinterpret_cast<const float4*>(row + r * p.stride + base + i));
                    t.x += u.x; t.y += u.y; t.z += u.z; t.w += u.w;
                }
            }
            x[i] = t.x; x[i + 1] = t.y; x[i + 2] = t.z; x[i + 3] = t.w;
        }
#pragma unroll
        for (int i = 0; i < TB_PER; ++i) if (base + i < n && !forced(base + i)) there |= 1u << i;
    }
    // range of the scores, and the error bound
    float mn = INFINITY, mx = -INFINITY, err = 0.f;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < TB_PER; ++i) {
        if ((there >> i) & 1u) {
            mn = fminf(mn, x[i]); mx = fmaxf(mx, x[i]);
            odd |= !(fabsf(x[i]) <= 3.4e38f);
        }
    }
    {
        // sum over member KV heads of factor * max|bound| * sum |q|
        const int g0 = h0 / c.G, g1 = (h1 - 1) / c.G;
        const int used = (n + BS_BLOCKS - 1) / BS_BLOCKS;
        for (int g = g0 + warp; g <= g1; g += NW) {
            float big = 0.f, l1 = 0.f;
            for (int i = lane; i < used; i += 32) big = fmaxf(big, __ldcg(p.amax + ((long long)b * c.Hkv + g) * p.chunks + i));
            for (int h = max(h0, g * c.G); h < min(h1, (g + 1) * c.G); ++h) {
                const uint2 q2 = __ldg(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h) * HEAD_DIM) + lane);
                l1 += fabsf(__uint_as_float(q2.x << 16)) + fabsf(__uint_as_float(q2.x & 0xffff0000u)) +
                      fabsf(__uint_as_float(q2.y << 16)) + fabsf(__uint_as_float(q2.y & 0xffff0000u));
            }
#pragma unroll
            for (int sh = 16; sh >= 1; sh >>= 1) {
                big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, sh));
                l1 += __shfl_xor_sync(0xffffffffu, l1, sh);
            }
            err += big * l1 * (p.k_scale ? fabsf(__ldg(p.k_scale + g)) : 1.f);
        }
    }
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) {
        mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, sh));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, sh));
    }
    if (lane == 0) { s_red[0][warp] = mn; s_red[1][warp] = mx; s_red[2][warp] = err; }
    odd = __syncthreads_or(odd);
    mn = s_red[0][0]; mx = s_red[1][0]; err = s_red[2][0];
#pragma unroll
    for (int w = 1; w < NW; ++w) { mn = fminf(mn, s_red[0][w]); mx = fmaxf(mx, s_red[1][w]); err += s_red[2][w]; }
    const float two_e = err * (2.1f / 65536.f);
    const float inv = (float)(TB_BINS - 1) / (mx - mn);
    const bool all = odd || !(two_e <= 3.4e38f) || !(mx > mn) || !(inv <= 3.4e38f);
    auto bin = [&](float v) { return max(0, min(TB_BINS - 1, __float2int_rd((v - mn) * inv))); };

    unsigned cand = there;
    if (!all) {
#pragma unroll
        for (int i = 0; i < TB_PER; ++i) if ((there >> i) & 1u) atomicAdd(&s_hist[bin(x[i])], 1u);
        __syncthreads();
        // the bin of the need-th largest: counts from the top
        constexpr int PER = TB_BINS / NT;
        int cnt = 0;
#pragma unroll
        for (int u = 0; u < PER; ++u) cnt += s_hist[TB_BINS - 1 - (tid * PER + u)];
        int total;
        int above = block_scan<NT>(cnt, s_part, total);
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int h = s_hist[TB_BINS - 1 - (tid * PER + u)];
            if (above < need && above + h >= need) s_bin = TB_BINS - 1 - (tid * PER + u);
            above += h;
        }
        __syncthreads();
        const int t = s_bin;
#pragma unroll
        for (int i = 0; i < TB_PER; ++i) {
            if ((there >> i) & 1u) {
                if (bin(x[i] - two_e) > t) { mine |= 1u << i; cand &= ~(1u << i); }
                else if (bin(x[i] + two_e) < t) cand &= ~(1u << i);
            }
        }
    }
    int winners;
    block_scan<NT>(__popc(mine), s_part, winners);
    int ncand;
    int at = block_scan<NT>(__popc(cand), s_part, ncand);
    const int want = need - winners;                        // of the candidates; 0 <= want <= ncand
    const bool spill = ncand > TB_CAND;
    const long long wrow = ((long long)b * p.Hi + hi) * c.max_blocks;
    unsigned long long* key = spill ? p.wide + wrow : s_key;
    int* cblk = spill ? p.wide_blk + wrow : s_blk;
    for (unsigned m = cand; m; m &= m - 1) cblk[at++] = base + __ffs(m) - 1;      // in ascending order
    __syncthreads();
    if (want > 0 && want < ncand) {
        for (int i = warp; i < ncand; i += NW) {
            const double s = wide_score(p, b, h0, h1, cblk[i], lane);
            if (lane == 0) key[i] = wide_key(s);
        }
        __syncthreads();
    }
    auto take = [&](unsigned* bits, int blk) { atomicOr(&bits[blk >> 5], 1u << (blk & 31)); };
    if (want >= ncand) {
        for (int i = tid; i < ncand; i += NT) take(s_take, cblk[i]);
    } else if (want > 0 && ncand <= TB_RANK) {
        // a candidate's place is the number of candidates before it: larger, or equal and lower (the list ascends)
        for (int i = tid; i < ncand; i += NT) {
            const unsigned long long k = key[i];
            int before = 0;
            for (int j = 0; j < ncand; ++j) before += (key[j] > k) || (key[j] == k && j < i);
            if (before < want) take(s_take, cblk[i]);
        }
    } else if (want > 0) {
        // the want-th largest key, eight bits at a time from the top
        if (tid == 0) { s_prefix = 0ull; s_need = want; }
        for (int shift = 56; shift >= 0; shift -= 8) {
            if (tid < 256) s_digit[tid] = 0;
            __syncthreads();
            const unsigned long long prefix = s_prefix;
            for (int i = tid; i < ncand; i += NT) {
                const unsigned long long k = key[i];
                if (shift == 56 || (k >> (shift + 8)) == prefix) atomicAdd(&s_digit[(unsigned)(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                int left = s_need, d = 255;
                while (d > 0 && (int)s_digit[d] < left) left -= s_digit[d--];
                s_prefix = (prefix << 8) | (unsigned)d;
                s_need = left;
            }
            __syncthreads();
        }
        const unsigned long long border = s_prefix;
        const int ties = s_need;                            // how many of those equal to the border are in: the lowest
        for (int i = tid; i < ncand; i += NT) {
            if (key[i] > border) take(s_take, cblk[i]);
            else if (key[i] == border) take(s_tie, cblk[i]);
        }
        __syncthreads();
        const unsigned tie = (s_tie[base >> 5] >> (base & 31)) & 0xffffu;
        int total;
        int before = block_scan<NT>(__popc(tie), s_part, total);
        for (unsigned m = tie; m; m &= m - 1) if (before++ < ties) mine |= m & (~m + 1u);
    }
    __syncthreads();
    mine |= (s_take[base >> 5] >> (base & 31)) & 0xffffu;
#pragma unroll
    for (int i = 0; i < TB_PER; ++i) if (base + i < n && forced(base + i)) mine |= 1u << i;
    int total;
    int pos = block_scan<NT>(__popc(mine), s_part, total);
    for (unsigned m = mine; m; m &= m - 1) out[pos++] = base + __ffs(m) - 1;
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

__device__ __forceinline__ float ld_cluster(uint32_t addr, int rank) {
    uint32_t a;
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(a) : "r"(addr), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;\n" ::: "memory");
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
    cluster_barrier();
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
    cluster_barrier();                                      // nobody leaves while its shared memory is read
}

}  // namespace tidal
