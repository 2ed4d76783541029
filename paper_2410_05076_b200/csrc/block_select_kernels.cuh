// The m best blocks per index head: scores of all blocks of 16 positions from their key bounds, ranked exactly.
//
// Scores. sum_c max(q_c lo_c, q_c hi_c) = q+ . hi + q- . lo with q+ = max(q, 0), q- = min(q, 0): two products, so 16 matrix
// instructions serve 16 blocks and the whole group of query heads. A warp takes 16 blocks x 512 bytes straight into the
// registers that are its A fragments (the contraction index may be relabelled: lane (gid, tig) holds the 16-byte
// pieces tig + 4 j of rows gid and gid + 8). Bound by memory: 512 bytes per block and KV head.
//
// Ranking. The set is the one that the scores in 64 bits give. Every matrix instruction starts from zero and its results are
// added in fp32: aligned to its largest product and cut at 2^-23 of that, 16 products lose at most 2^-19 of it, 16
// instructions 2^-15; the additions (16 per score, three over a group, one per KV head) lose 2^-24 of sum_c |q_c| max|bound|
// each. Call that e. One histogram over the row's range gives the bin t of the need-th largest fp32 score x; a block with
// x more than 2e above that bin is in for certain (its true value exceeds all but need - 1 others'), one more than 2e
// below it is out. What is left, a few blocks, is ranked by x; if the gap at the border is not more than 2e, those
// within 2e of it are evaluated in 64 bits and ranked by (score, lower block first). Rows that have no finite range or error
// bound, or too many blocks at the border, are evaluated in 64 bits wherever undecided.
//
// Two ways to run it (rule in tidal_api.cu):
//   block_select_kernel   one launch, no scratch memory, for short contexts: a thread-block cluster scores an item's blocks, pushes
//                         the scores into the shared memory of the CTAs that own the rows, and these rank them
//   block_score_kernel, block_rank_kernel   for long ones: scores by the whole GPU into scratch memory, then a CTA per row
#pragma once

#include "block_kernels.cuh"

namespace tidal {

struct SelectBlocksParams {
    BlockCache c;
    const __nv_bfloat16* q;
    const __nv_bfloat16* bounds;
    const float* k_scale;                                   // factors of the KV heads where several are added up (or null)
    int mode;                                               // TIDAL_SEL_*: a row per query head, per KV head (its heads' sum), or per sequence
    int m, keep_first, keep_last;
    int npad;                                               // blocks a score row has room for (a multiple of 32)
    int* idx;
    int* idx_count;
    // two launches:
    float* scores;                                          // [batch, query heads or KV heads, npad]
    float* amax;                                            // [batch, Hkv, chunks] largest |bound| of a chunk of blocks
    int chunks;
};

constexpr int SB_BINS = 2048;
constexpr int SB_CAND = 256;                                // border blocks ranked directly
constexpr int SB_MAX_CLUSTER = 16;
constexpr int SB_QROW = HEAD_DIM + 8;                       // padded query row in shared memory (elements)

// Larger double <=> larger key; not-a-number above everything, -0 as +0.
__device__ __forceinline__ unsigned long long wide_key(double s) {
    s += 0.0;
    if (s != s) return ~0ull;
    const unsigned long long u = (unsigned long long)__double_as_longlong(s);
    return (u >> 63) ? ~u : (u | 0x8000000000000000ull);
}
__device__ __forceinline__ unsigned float_key(float f) {
    const unsigned u = __float_as_uint(f);
    return (u >> 31) ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float key_float(unsigned k) { return __uint_as_float((k >> 31) ? k & 0x7fffffffu : ~k); }

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

// One block's score in 64 bits for query heads h0 .. h1 - 1, by a warp: four channels per lane and head. The queries are
// read from shared memory (rows of SB_QROW from head h0 on) where a group's are there, else from global memory.
__device__ __noinline__ double wide_score(const SelectBlocksParams& p, const __nv_bfloat16* group_q, int b, int h0, int h1, int blk, int lane) {
    const BlockCache& c = p.c;
    int page = 0;
    if (c.paged) {
        page = __ldg(c.page_table + (long long)b * c.max_pages + blk);
        if ((unsigned)page >= (unsigned)c.num_pages) return 0.0;
    }
    double acc = 0.0;
    int h = h0;
#pragma unroll 1
    for (int g = h0 / c.G; h < h1; ++g) {
        const uint2* bp = reinterpret_cast<const uint2*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS) + lane;
        const uint2 lo = __ldg(bp), hi = __ldg(bp + 32);
        double part = 0.0;
#pragma unroll 1
        for (; h < h1 && h < (g + 1) * c.G; ++h) {
            const __nv_bfloat16* qrow = group_q ? group_q + (h - h0) * SB_QROW : p.q + ((long long)b * c.Hq + h) * HEAD_DIM;
            const uint2 q = reinterpret_cast<const uint2*>(qrow)[lane];
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

// What one head adds to e per unit of the largest |bound|: 2^-15 max|q| + (24 + Hkv) 2^-24 sum|q|, by a warp that holds four
// elements of the row per lane.
__device__ __forceinline__ float query_part(uint2 q, int Hkv) {
    const float v[4] = {fabsf(__uint_as_float(q.x << 16)), fabsf(__uint_as_float(q.x & 0xffff0000u)),
                        fabsf(__uint_as_float(q.y << 16)), fabsf(__uint_as_float(q.y & 0xffff0000u))};
    float sum = (v[0] + v[1]) + (v[2] + v[3]);
    // (magnitudes order like their bits; not-a-number is the largest, and shows in the scores too)
    const float big = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])))));
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
    return big * (1.f / 32768.f) + sum * (float)(24 + Hkv) * (1.f / 16777216.f);
}

// The scores of a tile of 16 blocks against a group of query heads: s[0], s[1] for row gid and heads 2 tig, 2 tig + 1; s[2], s[3]
// for row gid + 8. neg / pos: the lane's pieces tig + 4 j of q-, q+ of head gid (zero beyond the group). x0, x1: the lane's
// pieces of rows gid and gid + 8. Raises amax to the largest magnitude seen, infinity where that is not finite.
template <typename Q>
__device__ __forceinline__ void score_tile(const uint4 (&x0)[8], const uint4 (&x1)[8], Q&& query, float (&s)[4], float& amax) {
    s[0] = s[1] = s[2] = s[3] = 0.f;
    uint32_t top = 0u, least = 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint4 q4 = query(j >> 2, j & 3);
        float d[4] = {0.f, 0.f, 0.f, 0.f}, e[4] = {0.f, 0.f, 0.f, 0.f};
        mma_bf16_16816(d, x0[j].x, x1[j].x, x0[j].y, x1[j].y, q4.x, q4.y);
        mma_bf16_16816(e, x0[j].z, x1[j].z, x0[j].w, x1[j].w, q4.z, q4.w);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] += d[i] + e[i];
        // the greatest of hi and of -lo bounds both in magnitude
        const uint32_t all[8] = {x0[j].x, x0[j].y, x0[j].z, x0[j].w, x1[j].x, x1[j].y, x1[j].z, x1[j].w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { if (j < 4) least = bmin2(least, all[i]); else top = bmax2(top, all[i]); }
    }
    const float t = fmaxf(fmaxf(__uint_as_float(top << 16), __uint_as_float(top & 0xffff0000u)),
                          -fminf(__uint_as_float(least << 16), __uint_as_float(least & 0xffff0000u)));
    const uint32_t a = (top & 0x7f807f80u) ^ 0x7f807f80u, b = (least & 0x7f807f80u) ^ 0x7f807f80u;
    const bool finite = (a & 0xffffu) && (a >> 16) && (b & 0xffffu) && (b >> 16);
    amax = fmaxf(amax, finite ? t : INFINITY);
}

// ---- ranking one row ---------------------------------------------------------------------------------------------
template <int NT, int V>
struct RankShared {
    static constexpr int WORDS = V * NT * 4 / 32;
    unsigned hist[SB_BINS];                                 // (first: aligned for vector loads)
    unsigned take[WORDS], cand[WORDS];                      // one bit per block: in, undecided
    unsigned long long key[SB_CAND], prefix;
    float x[SB_CAND], edge[2];
    int blk[SB_CAND];
    unsigned digit[256], range[3][NT / 32];
    int part[2][NT / 32];
    int ncand, winners, bin, left;
};

// v[j][u]: the score of block (j NT + tid) 4 + u (anything where there is none). err: e of the row is at most the largest
// of the threads' err. keys: room for 8 bytes per block of the row. All NT threads; returns with the shared memory in use.
template <int NT, int V>
__device__ __forceinline__ void rank_row(const SelectBlocksParams& p, RankShared<NT, V>& sh, float (&v)[V][4], float err,
                                         const __nv_bfloat16* group_q, unsigned long long* keys, int b, int h0, int h1, int n, int* out) {
    constexpr int NW = NT / 32;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int kk = min(p.m, n), words = (n + 31) / 32;
    const int nforced = (int)min((long long)n, (long long)p.keep_first + p.keep_last), need = kk - nforced;
    const int last = max(n - p.keep_last, 0);               // first block of those kept at the end
    auto forced = [&](int blk) { return blk < p.keep_first || blk >= last; };
#pragma unroll
    for (int i = tid * 4; i < SB_BINS; i += NT * 4) *reinterpret_cast<uint4*>(&sh.hist[i]) = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
    for (int w = tid; w < words; w += NT) {
        auto span = [&](int from, int to) -> unsigned {     // bits of this word for blocks from .. to - 1
            const int f = max(from - 32 * w, 0), t = min(to - 32 * w, 32);
            return f < t ? (0xffffffffu >> (32 - (t - f))) << f : 0u;
        };
        sh.take[w] = kk == n ? span(0, n) : span(0, min(p.keep_first, n)) | span(last, n);
        sh.cand[w] = 0;
    }
    if (tid == 0) { sh.ncand = 0; sh.winners = 0; }
#pragma unroll 1
    for (int i = kk + tid; i < p.m; i += NT) out[i] = -1;
    if (need > 0 && kk < n) {                               // else: every block, or the first kk of the kept ones
        // ---- range and error bound. Blocks that may not be chosen (kept ones, places behind the row) become -inf ------------
        float lo = INFINITY, hi = -INFINITY, odd = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = (j * NT + tid) * 4;
            if (at < p.keep_first || at + 4 > last) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (forced(at + u)) v[j][u] = -INFINITY;             // (last <= n)
                    else { lo = fminf(lo, v[j][u]); hi = fmaxf(hi, v[j][u]); odd = fmaf(v[j][u], 0.f, odd); }
                }
            } else {
#pragma unroll
                for (int u = 0; u < 4; ++u) { lo = fminf(lo, v[j][u]); hi = fmaxf(hi, v[j][u]); odd = fmaf(v[j][u], 0.f, odd); }
            }
        }
        if (odd != 0.f) hi = INFINITY;                      // (0 times an infinity or a not-a-number)
        {
            const unsigned a = __reduce_max_sync(0xffffffffu, float_key(-lo)), d = __reduce_max_sync(0xffffffffu, float_key(hi));
            const unsigned e = __reduce_max_sync(0xffffffffu, float_key(err));
            if (lane == 0) { sh.range[0][warp] = a; sh.range[1][warp] = d; sh.range[2][warp] = e; }
        }
        __syncthreads();
        lo = -key_float(__reduce_max_sync(0xffffffffu, lane < NW ? sh.range[0][lane] : 0u));
        hi = key_float(__reduce_max_sync(0xffffffffu, lane < NW ? sh.range[1][lane] : 0u));
        const float two_e = 2.01f * key_float(__reduce_max_sync(0xffffffffu, lane < NW ? sh.range[2][lane] : 0u));
        const float width = __fdividef(hi - lo, (float)(SB_BINS - 2)), inv = __fdividef(1.f, width);
        const bool all = !(hi <= 3.4e38f) || !(lo >= -3.4e38f) || !(two_e <= 3.4e38f) || !(width > 1e-30f) || !(width < 1e30f);
        float sure = INFINITY, least = -3.4e38f;            // above the first: in; below the second: out
        if (!all) {
            // (-inf converts to 0: it counts in the lowest bin, and is out by `least` even if that bin is t)
#pragma unroll
            for (int j = 0; j < V; ++j)
                if ((j * NT + warp * 32) * 4 < n) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) atomicAdd(&sh.hist[min(__float2uint_rd((v[j][u] - lo) * inv), (unsigned)(SB_BINS - 1))], 1u);
                }
            __syncthreads();
            // the bin t of the need-th largest: counts from the top
            constexpr int PER = SB_BINS / NT < 4 ? 4 : SB_BINS / NT;      // (the first SB_BINS / PER threads)
            int cnt = 0;
            if (tid * PER < SB_BINS) {
#pragma unroll
                for (int u = 0; u < PER; u += 4) {
                    const uint4 w = *reinterpret_cast<const uint4*>(&sh.hist[SB_BINS - 4 - (tid * PER + u)]);
                    cnt += w.x + w.y + w.z + w.w;
                }
            }
            int above = cta_scan<NT>(cnt, sh.part[0]);
            if (above < need && above + cnt >= need) {      // (one thread)
#pragma unroll 1
                for (int i = SB_BINS - 1 - tid * PER;; --i) {
                    above += sh.hist[i];
                    if (above >= need) { sh.bin = i; break; }
                }
            }
            __syncthreads();
            // Edges of the bin, moved outwards by 2 e and by more than what the binning rounds: (v - lo) inv and lo + t width
            // are each within a few 2^-23 of |lo| + |hi| in terms of v.
            const int t = sh.bin;
            const float slack = two_e + (fabsf(lo) + fabsf(hi)) * (1.f / 1048576.f);
            if (t < SB_BINS - 1) sure = lo + (float)(t + 1) * width + slack;
            if (t > 0) least = lo + (float)t * width - slack;
        }
        // ---- in, out or undecided --------------------------------------------------------------------------------------------
        int winners = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = (j * NT + tid) * 4;
            unsigned in = 0, und = 0;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                if (all ? !forced(at + u) : v[j][u] >= least) und |= 1u << u;
                if (!all && v[j][u] > sure) in |= 1u << u;
            }
            und &= ~in;
            if (in) { atomicOr(&sh.take[at >> 5], in << (at & 31)); winners += __popc(in); }
            if (und) {
                atomicOr(&sh.cand[at >> 5], und << (at & 31));
                int place = atomicAdd(&sh.ncand, __popc(und));
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if ((und >> u) & 1u) {
                        if (place < SB_CAND) { sh.x[place] = v[j][u]; sh.blk[place] = at + u; }
                        ++place;
                    }
            }
        }
        winners = __reduce_add_sync(0xffffffffu, winners);
        if (lane == 0 && winners) atomicAdd(&sh.winners, winners);
        __syncthreads();
        const int ncand = sh.ncand, want = need - sh.winners;           // 1 <= want <= ncand
        auto take = [&](int blk) { atomicOr(&sh.take[blk >> 5], 1u << (blk & 31)); };
        if (want == ncand) {
#pragma unroll 1
            for (int w = tid; w < words; w += NT) sh.take[w] |= sh.cand[w];
        } else if (!all && ncand <= SB_CAND) {
            // ranks by x; the want-th and the next
            int place = 0;
            if (tid < ncand) {
                const float mine = sh.x[tid];
                const int blk = sh.blk[tid];
#pragma unroll 4
                for (int j = 0; j < ncand; ++j) place += sh.x[j] > mine || (sh.x[j] == mine && sh.blk[j] < blk);
                if (place == want - 1) sh.edge[0] = mine;
                if (place == want) sh.edge[1] = mine;
            }
            __syncthreads();
            const float edge = sh.edge[0];
            if (edge - sh.edge[1] > two_e) {
                if (tid < ncand && place < want) take(sh.blk[tid]);
            } else {
                // 64 bits for those within 2e of the border; the others are certain
#pragma unroll 1
                for (int i = warp; i < ncand; i += NW) {
                    const float d = sh.x[i] - edge;
                    unsigned long long k = d > 0.f ? ~0ull : 0ull;
                    if (fabsf(d) <= two_e) k = wide_key(wide_score(p, group_q, b, h0, h1, sh.blk[i], lane));
                    if (lane == 0) sh.key[i] = k;
                }
                __syncthreads();
                if (tid < ncand) {
                    const unsigned long long k = sh.key[tid];
                    const int blk = sh.blk[tid];
                    int before = 0;
#pragma unroll 4
                    for (int j = 0; j < ncand; ++j) before += sh.key[j] > k || (sh.key[j] == k && sh.blk[j] < blk);
                    if (before < want) take(blk);
                }
            }
        } else {
            // ---- all undecided blocks in 64 bits; the want-th largest key eight bits at a time from the top --------------------
#pragma unroll 1
            for (int w = warp; w < words; w += NW)
#pragma unroll 1
                for (unsigned m = sh.cand[w]; m; m &= m - 1) {
                    const int blk = w * 32 + __ffs(m) - 1;
                    const unsigned long long k = wide_key(wide_score(p, group_q, b, h0, h1, blk, lane));
                    if (lane == 0) keys[blk] = k;
                }
            if (tid == 0) { sh.prefix = 0ull; sh.left = want; }
#pragma unroll 1
            for (int shift = 56; shift >= 0; shift -= 8) {
                if (tid < 256) sh.digit[tid] = 0;
                __syncthreads();
                const unsigned long long prefix = sh.prefix;
#pragma unroll 1
                for (int i = tid; i < n; i += NT) {
                    if (!((sh.cand[i >> 5] >> (i & 31)) & 1u)) continue;
                    const unsigned long long k = keys[i];
                    if (shift == 56 || (k >> (shift + 8)) == prefix) atomicAdd(&sh.digit[(unsigned)(k >> shift) & 255u], 1u);
                }
                __syncthreads();
                if (tid == 0) {
                    int left = sh.left, d = 255;
                    while (d > 0 && (int)sh.digit[d] < left) left -= sh.digit[d--];
                    sh.prefix = (prefix << 8) | (unsigned)d;
                    sh.left = left;
                }
                __syncthreads();
            }
            // larger ones are in, and as many of the equal ones as are wanted, the lower first
            const unsigned long long border = sh.prefix;
            const int ties = sh.left;
            static_assert(RankShared<NT, V>::WORDS <= NT, "a word per thread");
            unsigned in = 0, equal = 0;
            if (tid < words)
#pragma unroll 1
                for (unsigned m = sh.cand[tid]; m; m &= m - 1) {
                    const unsigned long long k = keys[tid * 32 + __ffs(m) - 1];
                    if (k > border) in |= m & (~m + 1u);
                    else if (k == border) equal |= m & (~m + 1u);
                }
            int before = cta_scan<NT>(__popc(equal), sh.part[0]);
#pragma unroll 1
            for (unsigned m = equal; m; m &= m - 1) if (before++ < ties) in |= m & (~m + 1u);
            if (tid < words) sh.take[tid] |= in;
        }
    }
    __syncthreads();
    // ---- the chosen blocks in ascending order ------------------------------------------------------------------------------------
    const unsigned bits = tid < words ? sh.take[tid] : 0u;
    int pos = cta_scan<NT>(__popc(bits), sh.part[1]);
#pragma unroll 1
    for (unsigned m = bits; m && pos < kk; m &= m - 1) out[pos++] = tid * 32 + __ffs(m) - 1;
}

// ---- short contexts: one launch ----------------------------------------------------------------------------------
constexpr int SC_THREADS = 256, SC_WARPS = SC_THREADS / 32;
constexpr int SC_MAX_BLOCKS = SC_THREADS * 4;
// Dynamic shared memory: the rows that a CTA owns, then 8 bytes per block for keys.
__host__ __device__ constexpr size_t sc_smem(int npad, int rows_per_cta) { return (size_t)npad * (8 + 4 * (size_t)rows_per_cta); }

__global__ void __launch_bounds__(SC_THREADS, 2) block_select_kernel(const __grid_constant__ SelectBlocksParams p) {
    constexpr int NT = SC_THREADS, NW = SC_WARPS;
    const BlockCache& c = p.c;
    extern __shared__ __align__(16) uint8_t sc_rows[];
    __shared__ __align__(16) RankShared<NT, 1> sh;
    __shared__ __align__(16) __nv_bfloat16 s_q[3][8][SB_QROW];        // q-, q+ and q of a group
    __shared__ float s_amax[SB_MAX_CLUSTER * NW], s_qpart[8];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    int rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    cluster_arrive();                                       // waited for before the first write to another CTA
    const bool shared_set = p.mode == 2, per_qhead = p.mode == 0;
    const int item = blockIdx.x / size;
    const int b = shared_set ? item : item / c.Hkv, g0 = shared_set ? 0 : item - b * c.Hkv, g1 = shared_set ? c.Hkv : g0 + 1;
    const int rows = per_qhead ? c.G : 1, owners = min(rows, size), slots = (rows + size - 1) / size;
    unsigned long long* const keys = reinterpret_cast<unsigned long long*>(sc_rows + (size_t)slots * p.npad * 4);
    pdl_wait();
    pdl_trigger();
    const int n = (cached_len(c, b) + TILE - 1) / TILE;
    const uint32_t a_rows = smem_u32(sc_rows);

    float amax = 0.f;
    bool first_write = true;
#pragma unroll 1
    for (int g = g0; g < g1; ++g) {
        if (g > g0) __syncthreads();
        for (int i = tid; i < 8 * HEAD_DIM / 2; i += NT) {
            const int h = i / (HEAD_DIM / 2), w = i % (HEAD_DIM / 2);
            const uint32_t x = h < c.G ? __ldg(reinterpret_cast<const uint32_t*>(p.q + ((long long)b * c.Hq + g * c.G + h) * HEAD_DIM) + w) : 0u;
            *reinterpret_cast<uint32_t*>(&s_q[0][h][2 * w]) = bmin2(x, 0u);
            *reinterpret_cast<uint32_t*>(&s_q[1][h][2 * w]) = bmax2(x, 0u);
            *reinterpret_cast<uint32_t*>(&s_q[2][h][2 * w]) = x;
        }
        const float factor = p.k_scale ? __ldg(p.k_scale + g) : 1.f;
        float gmax = 0.f;
        bool staged = false;
#pragma unroll 1
        for (int first = (rank * NW + warp) * 16; first < n; first += size * NW * 16) {
            const int r0 = first + gid, r1 = r0 + 8;
            auto source = [&](int blk) -> const uint4* {    // null: zeros
                if (blk >= n) return nullptr;
                int page = 0;
                if (c.paged) {
                    page = __ldg(c.page_table + (long long)b * c.max_pages + blk);
                    if ((unsigned)page >= (unsigned)c.num_pages) { atomicOr(c.status, STATUS_BAD_PAGE); return nullptr; }
                }
                return reinterpret_cast<const uint4*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS) + tig;
            };
            const uint4 *src0 = source(r0), *src1 = source(r1);
            uint4 x0[8], x1[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                x0[j] = src0 ? __ldg(src0 + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
                x1[j] = src1 ? __ldg(src1 + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
            }
            if (!staged) { asm volatile("bar.sync 1, %0;\n" ::"n"(NT) : "memory"); staged = true; }      // s_q is there
            float s[4];
            score_tile(x0, x1, [&](int half, int j) { return *reinterpret_cast<const uint4*>(&s_q[half][gid][8 * (tig + 4 * j)]); }, s, gmax);
            if (first_write) { cluster_wait(); first_write = false; }
            if (per_qhead) {
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int col = 2 * tig + i;
                    if (col < c.G) {
                        const uint32_t at = a_rows + (uint32_t)(col / size) * p.npad * 4;
                        if (r0 < n) st_cluster(at + 4 * r0, col % size, s[i]);
                        if (r1 < n) st_cluster(at + 4 * r1, col % size, s[2 + i]);
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
                }
            }
        }
        if (!staged) asm volatile("bar.sync 1, %0;\n" ::"n"(NT) : "memory");
        amax = fmaxf(amax, gmax * fabsf(factor));
        if ((shared_set || g == g1 - 1) && rank < owners && warp < c.G) {
            const float part = query_part(reinterpret_cast<const uint2*>(s_q[2][warp])[lane], c.Hkv);
            if (lane == 0) s_qpart[warp] = g > g0 ? s_qpart[warp] + part : part;
        }
    }
    if (first_write) cluster_wait();
    amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));       // (not negative: ordered like its bits)
    if (lane < owners) st_cluster(smem_u32(s_amax) + 4 * (rank * NW + warp), lane, amax);
    cluster_arrive();                                       // every score of the item is where it belongs ...
    if (g0 == 0 && rank == 0 && tid == 0 && p.idx_count) p.idx_count[b] = min(p.m, n);
    cluster_wait();                                         // ... and nobody touches another CTA's memory from here on
    if (rank >= owners) return;
#pragma unroll 1
    for (int row = rank, slot = 0; row < rows; row += size, ++slot) {
        if (slot > 0) __syncthreads();
        const int h0 = per_qhead ? g0 * c.G + row : g0 * c.G, h1 = per_qhead ? h0 + 1 : g1 * c.G;
        const int hi = per_qhead ? h0 : (shared_set ? 0 : g0), Hi = per_qhead ? c.Hq : (shared_set ? 1 : c.Hkv);
        float v[1][4] = {{0.f, 0.f, 0.f, 0.f}}, err = 0.f, qsum = 0.f;
        if (tid * 4 < n) {                                  // rows have room for a multiple of 32 blocks
            const float4 t = *reinterpret_cast<const float4*>(sc_rows + (size_t)slot * p.npad * 4 + tid * 16);
            v[0][0] = t.x; v[0][1] = t.y; v[0][2] = t.z; v[0][3] = t.w;
        }
        for (int i = tid; i < size * NW; i += NT) err = fmaxf(err, s_amax[i]);
        if (per_qhead) qsum = s_qpart[row];
        else for (int h = 0; h < c.G; ++h) qsum += s_qpart[h];
        rank_row<NT, 1>(p, sh, v, err * qsum, shared_set ? nullptr : &s_q[2][h0 - g0 * c.G][0], keys, b, h0, h1, n,
                        p.idx + ((long long)b * Hi + hi) * p.m);
    }
}

// ---- long contexts: scores by the whole GPU, then a CTA per row ----------------------------------------------------
constexpr int SS_WARPS = 4;
constexpr int SS_BLOCKS = SS_WARPS * 16;                    // blocks per CTA of the score kernel: a chunk

__global__ void __launch_bounds__(SS_WARPS * 32) block_score_kernel(const __grid_constant__ SelectBlocksParams p) {
    const BlockCache& c = p.c;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    const int pair = blockIdx.x / p.chunks, chunk = blockIdx.x - pair * p.chunks;
    const int b = pair / c.Hkv, g = pair - b * c.Hkv;
    const int r0 = chunk * SS_BLOCKS + warp * 16 + gid, r1 = r0 + 8;
    __shared__ float s_amax[SS_WARPS];
    pdl_wait();
    pdl_trigger();
    // Nothing waits for the length: bounds (and table entries) up to max_blocks may be read whatever they hold, and the
    // rows beyond the length become zeros before they count.
    const int len = c.ctx_lens[b];
    int page0 = 0, page1 = 0;
    if (c.paged) {
        const int* row = c.page_table + (long long)b * c.max_pages;
        page0 = r0 < c.max_blocks ? __ldg(row + r0) : -1;
        page1 = r1 < c.max_blocks ? __ldg(row + r1) : -1;
    }
    auto source = [&](int blk, int page) -> const uint4* {
        if (blk >= c.max_blocks || (c.paged && (unsigned)page >= (unsigned)c.num_pages)) return nullptr;
        return reinterpret_cast<const uint4*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS) + tig;
    };
    const uint4 *src0 = source(r0, page0), *src1 = source(r1, page1);
    uint4 x0[8], x1[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x0[j] = src0 ? __ldg(src0 + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
        x1[j] = src1 ? __ldg(src1 + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
    }
    uint4 q4[4];
    const uint4* qp = reinterpret_cast<const uint4*>(p.q + ((long long)b * c.Hq + g * c.G + min(gid, c.G - 1)) * HEAD_DIM) + tig;
#pragma unroll
    for (int j = 0; j < 4; ++j) q4[j] = __ldg(qp + 4 * j);
    const int n = (max(min(len, c.max_ctx), 0) + TILE - 1) / TILE;
    if (chunk * SS_BLOCKS >= n) return;
    if ((r0 < n && !src0) || (r1 < n && !src1)) atomicOr(c.status, STATUS_BAD_PAGE);
    const bool on = gid < c.G;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (r0 >= n) x0[j] = make_uint4(0u, 0u, 0u, 0u);
        if (r1 >= n) x1[j] = make_uint4(0u, 0u, 0u, 0u);
    }
    float s[4], amax = 0.f;
    score_tile(x0, x1, [&](int half, int j) {
        uint4 r;
        r.x = on ? (half ? bmax2(q4[j].x, 0u) : bmin2(q4[j].x, 0u)) : 0u;
        r.y = on ? (half ? bmax2(q4[j].y, 0u) : bmin2(q4[j].y, 0u)) : 0u;
        r.z = on ? (half ? bmax2(q4[j].z, 0u) : bmin2(q4[j].z, 0u)) : 0u;
        r.w = on ? (half ? bmax2(q4[j].w, 0u) : bmin2(q4[j].w, 0u)) : 0u;
        return r;
    }, s, amax);
    if (p.mode == 0) {
        float* row = p.scores + ((long long)b * c.Hq + g * c.G) * p.npad;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int col = 2 * tig + i;
            if (col < c.G) {
                if (r0 < n) row[(long long)col * p.npad + r0] = s[i];
                if (r1 < n) row[(long long)col * p.npad + r1] = s[2 + i];
            }
        }
    } else {
        float x = s[0] + s[1], y = s[2] + s[3];
        x += __shfl_xor_sync(0xffffffffu, x, 1); y += __shfl_xor_sync(0xffffffffu, y, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2); y += __shfl_xor_sync(0xffffffffu, y, 2);
        const float f = p.k_scale ? __ldg(p.k_scale + g) : 1.f;
        float* row = p.scores + ((long long)b * c.Hkv + g) * p.npad;
        if (tig == 0 && r0 < n) row[r0] = x * f;
        if (tig == 0 && r1 < n) row[r1] = y * f;
    }
    amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
    if (lane == 0) s_amax[warp] = amax;
    __syncthreads();
    if (threadIdx.x == 0) {
        float m = s_amax[0];
#pragma unroll
        for (int w = 1; w < SS_WARPS; ++w) m = fmaxf(m, s_amax[w]);
        p.amax[(long long)pair * p.chunks + chunk] = m;
    }
}

// Dynamic shared memory: 8 bytes per block for keys.
template <int NT, int V>
__global__ void __launch_bounds__(NT) block_rank_kernel(const __grid_constant__ SelectBlocksParams p) {
    constexpr int NW = NT / 32;
    const BlockCache& c = p.c;
    extern __shared__ __align__(16) uint8_t rk_keys[];
    __shared__ __align__(16) RankShared<NT, V> sh;
    __shared__ __align__(16) __nv_bfloat16 s_q[8][SB_QROW];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const bool shared_set = p.mode == 2, per_qhead = p.mode == 0;
    const int Hi = per_qhead ? c.Hq : (shared_set ? 1 : c.Hkv);
    const int b = blockIdx.x / Hi, hi = blockIdx.x - b * Hi;
    const int members = c.Hq / Hi, h0 = hi * members, h1 = h0 + members;
    pdl_wait();
    pdl_trigger();
    // (rows of npad scores: what lies behind the length is read, and ignored when the length is there)
    const int len = c.ctx_lens[b];
    const int sum_rows = shared_set ? c.Hkv : 1;
    const float* row = p.scores + ((long long)b * (per_qhead ? c.Hq : c.Hkv) + (shared_set ? 0 : hi)) * p.npad;
    float v[V][4];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int at = (j * NT + tid) * 4;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at < p.npad) t = __ldcg(reinterpret_cast<const float4*>(row + at));
        v[j][0] = t.x; v[j][1] = t.y; v[j][2] = t.z; v[j][3] = t.w;
    }
#pragma unroll 1
    for (int r = 1; r < sum_rows; ++r)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int at = (j * NT + tid) * 4;
            if (at < p.npad) {
                const float4 t = __ldcg(reinterpret_cast<const float4*>(row + (long long)r * p.npad + at));
                v[j][0] += t.x; v[j][1] += t.y; v[j][2] += t.z; v[j][3] += t.w;
            }
        }
    const int n = (max(min(len, c.max_ctx), 0) + TILE - 1) / TILE, used = (n + SS_BLOCKS - 1) / SS_BLOCKS;
    // e: the sum over the member heads is at most their number times the largest
    float err = 0.f;
#pragma unroll 1
    for (int h = h0 + warp; h < h1; h += NW) {
        const int g = h / c.G;
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h) * HEAD_DIM) + lane);
        float big = 0.f;
        const float* am = p.amax + ((long long)b * c.Hkv + g) * p.chunks;
#pragma unroll 4
        for (int i = lane; i < used; i += 32) big = fmaxf(big, __ldcg(am + i));
        big = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(big)));
        if (!shared_set) reinterpret_cast<uint2*>(s_q[h - h0])[lane] = q;
        err = fmaxf(err, (float)members * big * query_part(q, c.Hkv) * (p.k_scale ? fabsf(__ldg(p.k_scale + g)) : 1.f));
    }
    if (hi == 0 && tid == 0 && p.idx_count) p.idx_count[b] = min(p.m, n);
    rank_row<NT, V>(p, sh, v, err, shared_set ? nullptr : &s_q[0][0], reinterpret_cast<unsigned long long*>(rk_keys), b, h0, h1, n,
                    p.idx + ((long long)b * Hi + hi) * p.m);
}

}  // namespace tidal
