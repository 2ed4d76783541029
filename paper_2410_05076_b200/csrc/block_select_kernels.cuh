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
//   block_select_kernel   one launch, no scratch memory, for short contexts: a CTA or a thread-block cluster scores an item's blocks,
//                         pushes the scores into the shared memory of the CTAs that own the rows, and these rank them, with a warp
//                         per row or all together
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
    float* err;                                             // [the same rows, chunks] e over a chunk of blocks
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

// One block's score in 64 bits, by a warp: every lane four channels of each head. near_bounds: the bounds of the lane's channels
// (zero without a page); near_score: `heads` query heads of one KV head, their rows in shared memory; wide_score: query heads h0 ..
// h1 - 1 of any KV heads.
__device__ __forceinline__ void near_bounds(const SelectBlocksParams& p, int b, int g, int blk, int lane, uint2& lo, uint2& hi) {
    const BlockCache& c = p.c;
    int page = 0;
    if (c.paged) {
        page = read_global(c.page_table + (long long)b * c.max_pages + blk);
        if ((unsigned)page >= (unsigned)c.num_pages) { lo = hi = make_uint2(0u, 0u); return; }
    }
    const uint2* bp = reinterpret_cast<const uint2*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS) + lane;
    lo = read_global(bp);
    hi = read_global(bp + 32);
}
// A bf16 number, as the upper half of an fp32's bits, in 64 bits: its fields put into place are its value times 2^-896, subnormal ones
// included (infinities and not-a-numbers become 2^128 and more). Two integer instructions and a product; the
// conversion instruction has an eighth of their rate.
__device__ __forceinline__ double widen(uint32_t w) {
    return __hiloint2double(((int)w >> 3) & (int)0x8fffffff, 0) * 0x1p896;
}
__device__ __forceinline__ void wide_add(double (&sum)[4], uint2 q, uint2 lo, uint2 hi) {      // four chains: the latency is what counts
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t qw = i & 2 ? q.y : q.x, lw = i & 2 ? lo.y : lo.x, hw = i & 2 ? hi.y : hi.x;
        const uint32_t bw = (i & 1 ? qw : qw << 16) >> 31 ? lw : hw;              // a negative q takes the least key
        sum[i] = fma(widen(i & 1 ? qw & 0xffff0000u : qw << 16), widen(i & 1 ? bw & 0xffff0000u : bw << 16), sum[i]);
    }
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) x += __shfl_xor_sync(0xffffffffu, x, sh);
    return x;
}
__device__ __forceinline__ double near_score(const __nv_bfloat16* group_q, int heads, uint2 lo, uint2 hi, int lane) {
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 2
    for (int h = 0; h < heads; ++h) wide_add(sum, reinterpret_cast<const uint2*>(group_q + h * SB_QROW)[lane], lo, hi);
    return warp_sum((sum[0] + sum[1]) + (sum[2] + sum[3]));
}
__device__ __noinline__ double wide_score(const SelectBlocksParams& p, const __nv_bfloat16* group_q, int b, int h0, int h1, int blk, int lane) {
    const BlockCache& c = p.c;
    double acc = 0.0;
    int h = h0;
#pragma unroll 1
    for (int g = h0 / c.G; h < h1; ++g) {
        uint2 lo, hi;
        near_bounds(p, b, g, blk, lane, lo, hi);
        double sum[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
        for (; h < h1 && h < (g + 1) * c.G; ++h) {
            const __nv_bfloat16* qrow = group_q ? group_q + (h - h0) * SB_QROW : p.q + ((long long)b * c.Hq + h) * HEAD_DIM;
            wide_add(sum, reinterpret_cast<const uint2*>(qrow)[lane], lo, hi);
        }
        const double part = (sum[0] + sum[1]) + (sum[2] + sum[3]);
        acc += p.k_scale ? part * (double)read_global(p.k_scale + g) : part;
    }
    return warp_sum(acc);
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

// A matrix instruction that starts from zero; its results as two pairs of fp32.
__device__ __forceinline__ void mma_from_zero(f32pair (&d)[2], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    float r[4];
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};\n"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
    d[0] = pair2(r[0], r[1]);
    d[1] = pair2(r[2], r[3]);
}
// The scores of a tile of 16 blocks against a group of query heads: s[0], s[1] for row gid and heads 2 tig, 2 tig + 1; s[2], s[3]
// for row gid + 8. query(half, j): the lane's piece tig + 4 j of q- (half 0) or q+ (1) of head gid, zero beyond the group. x0, x1:
// the lane's pieces of rows gid and gid + 8. low, high: running maxima of the bits of the least and of the greatest keys,
// from which largest_bound() tells the largest magnitude: as unsigned numbers the bits of the least keys are largest for the
// most negative one (or, if there is none, for the largest), as signed numbers those of the greatest for the largest.
template <typename Q>
__device__ __forceinline__ void score_tile(const uint4 (&x0)[8], const uint4 (&x1)[8], Q&& query, float (&s)[4], uint32_t& low, uint32_t& high) {
    f32pair sum[2] = {0ull, 0ull};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint4 q4 = query(j >> 2, j & 3);
        f32pair d[2], e[2];
        mma_from_zero(d, x0[j].x, x1[j].x, x0[j].y, x1[j].y, q4.x, q4.y);
        mma_from_zero(e, x0[j].z, x1[j].z, x0[j].w, x1[j].w, q4.z, q4.w);
#pragma unroll
        for (int i = 0; i < 2; ++i) sum[i] = add2(sum[i], add2(d[i], e[i]));
        if (j < 4) {
            low = __vimax3_u16x2(low, x0[j].x, x0[j].y); low = __vimax3_u16x2(low, x0[j].z, x0[j].w);
            low = __vimax3_u16x2(low, x1[j].x, x1[j].y); low = __vimax3_u16x2(low, x1[j].z, x1[j].w);
        } else {
            high = __vimax3_s16x2(high, x0[j].x, x0[j].y); high = __vimax3_s16x2(high, x0[j].z, x0[j].w);
            high = __vimax3_s16x2(high, x1[j].x, x1[j].y); high = __vimax3_s16x2(high, x1[j].z, x1[j].w);
        }
    }
    s[0] = half2(sum[0], 0); s[1] = half2(sum[0], 1);
    s[2] = half2(sum[1], 0); s[3] = half2(sum[1], 1);
}
// Start: low = 0, high = 0x80008000. Infinity where a bound is not finite: there is no error bound then.
__device__ __forceinline__ float largest_bound(uint32_t low, uint32_t high) {
    const uint32_t a = max(low & 0x7fffu, (low >> 16) & 0x7fffu);
    // (a negative greatest key is smaller in magnitude than its least one)
    const uint32_t b = max((high & 0x8000u) ? 0u : high & 0x7fffu, (high >> 31) ? 0u : high >> 16);
    const uint32_t m = max(a, b);
    return m >= 0x7f80u ? INFINITY : __uint_as_float(m << 16);
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

// Keys of the candidates of a set that all heads share, by all NW warps: those within two_e of the edge in 64 bits, each warp
// some of the KV heads of every block, with the loads of four under way together. parts: room for SB_BINS / 2 numbers.
template <int NW>
__device__ __noinline__ void shared_keys(const SelectBlocksParams& p, const float* x, const int* blks, float edge, float two_e, int ncand,
                                         unsigned long long* keys, double* parts, int b) {
    const BlockCache& c = p.c;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int AHEAD = 4, ROUND = SB_BINS / 2 / NW;
#pragma unroll 1
    for (int i0 = 0; i0 < ncand; i0 += ROUND) {
        const int i1 = min(ncand, i0 + ROUND);
#pragma unroll 1
        for (int i = i0; i < i1; ++i) {
            if (!(fabsf(x[i] - edge) <= two_e)) continue;
            double acc = 0.0;
#pragma unroll 1
            for (int g = warp; g < c.Hkv; g += NW * AHEAD) {
                uint2 lo[AHEAD], hi[AHEAD];
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) near_bounds(p, b, min(g + a * NW, c.Hkv - 1), blks[i], lane, lo[a], hi[a]);
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    const int ga = g + a * NW;
                    if (ga >= c.Hkv) break;
                    double sum[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
                    for (int h = 0; h < c.G; ++h)
                        wide_add(sum, read_global(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + ga * c.G + h) * HEAD_DIM) + lane), lo[a], hi[a]);
                    const double part = (sum[0] + sum[1]) + (sum[2] + sum[3]);
                    acc += p.k_scale ? part * (double)read_global(p.k_scale + ga) : part;
                }
            }
            acc = warp_sum(acc);
            if (lane == 0) parts[(i - i0) * NW + warp] = acc;
        }
        __syncthreads();
        if (tid < i1 - i0) {
            const float d = x[i0 + tid] - edge;
            unsigned long long k = d > 0.f ? ~0ull : 0ull;
            if (fabsf(d) <= two_e) {
                double sum = 0.0;
#pragma unroll 1
                for (int w = 0; w < NW; ++w) sum += parts[tid * NW + w];
                k = wide_key(sum);
            }
            keys[i0 + tid] = k;
        }
        __syncthreads();
    }
}

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
            // (A warp per candidate asks for its bounds already: if 64 bits are needed, they are there when the ranks are.)
            const bool early = group_q != nullptr && ncand <= NW;
            uint2 near_lo = make_uint2(0u, 0u), near_hi = near_lo;
            if (early && warp < ncand) near_bounds(p, b, h0 / p.c.G, sh.blk[warp], lane, near_lo, near_hi);
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
                if (early) {
                    if (warp < ncand) {
                        const float d = sh.x[warp] - edge;
                        unsigned long long k = d > 0.f ? ~0ull : 0ull;
                        if (fabsf(d) <= two_e) k = wide_key(near_score(group_q, h1 - h0, near_lo, near_hi, lane));
                        if (lane == 0) sh.key[warp] = k;
                    }
                } else if (!group_q) {
                    shared_keys<NW>(p, sh.x, sh.blk, edge, two_e, ncand, sh.key, reinterpret_cast<double*>(sh.hist), b);
                } else {
#pragma unroll 1
                    for (int i = warp; i < ncand; i += NW) {
                        const float d = sh.x[i] - edge;
                        unsigned long long k = d > 0.f ? ~0ull : 0ull;
                        if (fabsf(d) <= two_e) k = wide_key(wide_score(p, group_q, b, h0, h1, sh.blk[i], lane));
                        if (lane == 0) sh.key[i] = k;
                    }
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
// The scores in 64 bits of two blocks for heads h0 .. h1 - 1 of one KV head (a negative number: no block), by a warp. One call's code is
// run rarely and so fetched anew: it is short, and what it loads is loaded at once.
__device__ __noinline__ double2 near_pair(const SelectBlocksParams& p, int b, int h0, int h1, int blk0, int blk1, int lane) {
    const BlockCache& c = p.c;
    const int g = h0 / c.G;
    uint2 lo[2], hi[2];
    near_bounds(p, b, g, max(blk0, 0), lane, lo[0], hi[0]);
    near_bounds(p, b, g, max(blk1, 0), lane, lo[1], hi[1]);
    double x[4] = {0.0, 0.0, 0.0, 0.0}, y[4] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 1
    for (int h = h0; h < h1; ++h) {
        const uint2 q = read_global(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h) * HEAD_DIM) + lane);
        wide_add(x, q, lo[0], hi[0]);
        wide_add(y, q, lo[1], hi[1]);
    }
    double s = (x[0] + x[1]) + (x[2] + x[3]), t = (y[0] + y[1]) + (y[2] + y[3]);
#pragma unroll
    for (int sh = 16; sh >= 1; sh >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, sh);
        t += __shfl_xor_sync(0xffffffffu, t, sh);
    }
    return make_double2(s, t);
}

// Ranks one row by one warp, which keeps the whole row in registers: no barriers, so that the chain of a short row is short, and a CTA's
// rows at once. Instead of the histogram a bisection for a threshold that exactly the wanted number of scores exceeds (a count per
// step; about as many steps as the row's length has bits, and a few), or until the interval is no wider than 2e. v[j]: the score of
// block 32 j + lane. keys: room for 8 bytes per block; the warp's alone.
template <int V>
__device__ __forceinline__ void rank_row_warp(const SelectBlocksParams& p, float (&v)[V], float two_e, unsigned long long* keys, int b, int h0,
                                              int h1, int n, int* out) {
    const int lane = threadIdx.x & 31;
    const int kk = min(p.m, n);
    const int nforced = (int)min((long long)n, (long long)p.keep_first + p.keep_last), need = kk - nforced;
    const int last = max(n - p.keep_last, 0);               // first block of those kept at the end
    unsigned take = 0, can = 0;                             // a bit per j: chosen, to be ranked
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int blk = j * 32 + lane;
        if (blk < n) {
            if (kk == n || blk < p.keep_first || blk >= last) take |= 1u << j;
            else can |= 1u << j;
        }
    }
    if (need > 0 && kk < n) {                               // else: every block, or the first kk of the kept ones
        float lo = INFINITY, hi = -INFINITY, odd = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if ((can >> j) & 1u) { lo = fminf(lo, v[j]); hi = fmaxf(hi, v[j]); odd = fmaf(v[j], 0.f, odd); }
            else v[j] = -INFINITY;
        }
        if (odd != 0.f) hi = INFINITY;                      // (0 times an infinity or a not-a-number)
        lo = -key_float(__reduce_max_sync(0xffffffffu, float_key(-lo)));
        hi = key_float(__reduce_max_sync(0xffffffffu, float_key(hi)));
        unsigned in = 0, und = can;
        if (hi <= 3.4e38f && lo >= -3.4e38f && two_e <= 3.4e38f) {
            // more than `need` scores are above a, or exactly as many; fewer are above c
            float a = lo - (two_e + fabsf(lo) * 1e-6f + 1e-37f), c = hi, t = 0.f;
            bool exact = false;
#pragma unroll 1
            for (int step = 0; step < 64 && c - a > two_e; ++step) {
                t = a + (c - a) * 0.5f;
                if (!(t > a && t < c)) break;
                int some[2] = {0, 0};
#pragma unroll
                for (int j = 0; j < V; ++j) some[j & 1] += v[j] > t;
                const int above = __reduce_add_sync(0xffffffffu, some[0] + some[1]);
                if (above == need) { exact = true; break; }
                if (above > need) a = t; else c = t;
            }
            // above: no less than the (need + 1)-th largest; below: no more than the need-th
            float above = c, below = a;
            if (exact) {
                float next = -INFINITY, least = INFINITY;
#pragma unroll
                for (int j = 0; j < V; ++j) { if (v[j] > t) least = fminf(least, v[j]); else next = fmaxf(next, v[j]); }
                above = key_float(__reduce_max_sync(0xffffffffu, float_key(next)));
                below = -key_float(__reduce_max_sync(0xffffffffu, float_key(-least)));
            }
            const bool clear = exact && below - above > two_e;
            und = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (clear ? v[j] > t : v[j] - above > two_e) in |= 1u << j;
                else if (!clear && !(below - v[j] > two_e)) und |= 1u << j;
            }
            und &= can;
        }
        take |= in;
        const int nund = __reduce_add_sync(0xffffffffu, __popc(und)), want = need - __reduce_add_sync(0xffffffffu, __popc(in));
        if (nund == want) {
            take |= und;
        } else if (nund <= 32) {
            // lane i keeps the i-th of them
            int* const list = reinterpret_cast<int*>(keys);
            __syncwarp();                                   // (the scores may lie where the list goes)
            int at = 0;
#pragma unroll 1
            for (int j = 0; j < V; ++j) {
                const unsigned bits = __ballot_sync(0xffffffffu, (und >> j) & 1u);
                if ((und >> j) & 1u) list[at + __popc(bits & ((1u << lane) - 1u))] = j * 32 + lane;
                at += __popc(bits);
            }
            __syncwarp();
            const int mine = lane < nund ? list[lane] : -1;
            unsigned long long key = 0ull;
#pragma unroll 1
            for (int i = 0; i < nund; i += 2) {
                const int blk0 = __shfl_sync(0xffffffffu, mine, i), blk1 = __shfl_sync(0xffffffffu, mine, i + 1);       // (i + 1 < 32)
                const double2 k = near_pair(p, b, h0, h1, blk0, blk1, lane);
                if ((lane & ~1) == i) key = wide_key(lane & 1 ? k.y : k.x);
            }
            int before = 0;
#pragma unroll 1
            for (int i = 0; i < nund; ++i) {
                const unsigned long long k = __shfl_sync(0xffffffffu, key, i);
                before += k > key || (k == key && i < lane);          // (the list ascends)
            }
            unsigned chosen = __ballot_sync(0xffffffffu, lane < nund && before < want);
#pragma unroll 1
            for (; chosen; chosen &= chosen - 1) {
                const int blk = __shfl_sync(0xffffffffu, mine, __ffs(chosen) - 1);
                if ((blk & 31) == lane) take |= 1u << (blk >> 5);
            }
        } else {
            // all undecided blocks in 64 bits; the want-th largest key bit by bit from the top
            __syncwarp();
#pragma unroll 1
            for (int j = 0; j < V; ++j) {
                const unsigned bits = __ballot_sync(0xffffffffu, (und >> j) & 1u);
#pragma unroll 1
                for (int i = 0; i < 32; i += 2) {
                    if (!((bits >> i) & 3u)) continue;
                    const double2 k = near_pair(p, b, h0, h1, j * 32 + min(i, n - 1 - j * 32), j * 32 + min(i + 1, n - 1 - j * 32), lane);
                    if ((lane & ~1) == i && ((und >> j) & 1u)) keys[j * 32 + lane] = wide_key(lane & 1 ? k.y : k.x);
                }
            }
            __syncwarp();
            unsigned long long border = 0ull;
#pragma unroll 1
            for (int bit = 63; bit >= 0; --bit) {
                const unsigned long long t = border | (1ull << bit);
                int some = 0;
#pragma unroll 2
                for (int j = 0; j < V; ++j) if ((und >> j) & 1u) some += keys[j * 32 + lane] >= t;
                if (__reduce_add_sync(0xffffffffu, some) >= want) border = t;
            }
            unsigned equal = 0, larger = 0;
#pragma unroll 1
            for (int j = 0; j < V; ++j)
                if ((und >> j) & 1u) {
                    const unsigned long long k = keys[j * 32 + lane];
                    if (k > border) larger |= 1u << j;
                    if (k == border) equal |= 1u << j;
                }
            take |= larger;
            int ties = want - __reduce_add_sync(0xffffffffu, __popc(larger));         // the lower ones of the equal
#pragma unroll 1
            for (int j = 0; j < V; ++j) {
                const unsigned bits = __ballot_sync(0xffffffffu, (equal >> j) & 1u);
                if (((equal >> j) & 1u) && __popc(bits & ((1u << lane) - 1u)) < ties) take |= 1u << j;
                ties -= __popc(bits);
            }
        }
    }
    // the chosen blocks in ascending order
    int at = 0;
#pragma unroll 4
    for (int j = 0; j < V; ++j) {
        const unsigned bits = __ballot_sync(0xffffffffu, (take >> j) & 1u);
        const int pos = at + __popc(bits & ((1u << lane) - 1u));
        if (((take >> j) & 1u) && pos < kk) out[pos] = j * 32 + lane;
        at += __popc(bits);
    }
}

template <int V>
struct RankByCta {};                                        // nothing for rows that a warp ranks
template <>
struct RankByCta<0> {
    RankShared<256, 1> rank;
    __nv_bfloat16 q[8][SB_QROW];
};

// An item is a (sequence, KV head), or a sequence where all heads share a set. The warps of a CTA, or of a thread-block cluster, score
// its tiles of 16 blocks and push the scores into the shared memory of the CTAs that own the rows. These are ranked by a warp each, V
// scores per lane, or (V = 0) by the CTA one after the other.
// A shared set adds up its KV heads: as many warps as there are take the heads of a tile in slices, and the slices' sums are added
// before the ranking.
constexpr int SC_THREADS = 256, SC_WARPS = SC_THREADS / 32;
constexpr int SC_MAX_BLOCKS = SC_THREADS * 4;
// Dynamic shared memory: 8 bytes per block (the score, later a key) of the rows that a CTA owns; or the slices' sums.
__host__ __device__ constexpr size_t sc_smem(int npad, int rows_per_cta, int sums) {
    return (size_t)npad * 8 * (size_t)rows_per_cta > (size_t)sums * 64 ? (size_t)npad * 8 * (size_t)rows_per_cta : (size_t)sums * 64;
}

template <int V, bool SHARED>
__global__ void __launch_bounds__(SC_THREADS, 2) block_select_kernel(const __grid_constant__ SelectBlocksParams p) {
    static_assert(V == 0 || !SHARED, "a set that all heads share is ranked by a CTA");
    const BlockCache& c = p.c;
    extern __shared__ __align__(16) uint8_t sc_rows[];
    __shared__ __align__(16) RankByCta<V> sh;
    __shared__ float2 s_part[SB_MAX_CLUSTER * SC_WARPS];    // per warp: largest bound, share of the members' query_part
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, gid = lane >> 2, tig = lane & 3;
    int rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    if (size > 1) cluster_arrive();                         // waited for before the first write to another CTA
    const bool per_qhead = !SHARED && p.mode == 0;
    const int item = blockIdx.x / size, NW = blockDim.x / 32, W = size * NW, wid = rank * NW + warp;
    const int b = SHARED ? item : item / c.Hkv, g0 = SHARED ? 0 : item - b * c.Hkv;
    const int rows = per_qhead ? c.G : 1, owners = min(rows, size), my_row = rank + warp * size;       // (a CTA has a warp for each of its rows)
    const bool mine = my_row < rows;                        // this warp's row is one
    pdl_wait();
    pdl_trigger();
    const int n = (cached_len(c, b) + TILE - 1) / TILE, tiles = (n + 15) / 16;
    const uint32_t a_rows = smem_u32(sc_rows);
    const int h0 = per_qhead ? g0 * c.G + my_row : g0 * c.G, h1 = per_qhead ? h0 + 1 : (SHARED ? c.Hq : h0 + c.G);       // its heads
    float amax = 0.f, qsum = 0.f;
    bool first = true;

    auto load = [&](int tile, int g, uint4 (&x0)[8], uint4 (&x1)[8]) {
        auto entry = [&](int blk) -> int {                  // (does not wait for the length)
            return c.paged && blk < c.max_blocks ? read_global(c.page_table + (long long)b * c.max_pages + blk) : 0;
        };
        const int page0 = entry(tile * 16 + gid), page1 = entry(tile * 16 + gid + 8);
        auto source = [&](int blk, int page) -> const uint4* {         // null: zeros
            if (blk >= n) return nullptr;
            if (c.paged && (unsigned)page >= (unsigned)c.num_pages) { atomicOr(c.status, STATUS_BAD_PAGE); return nullptr; }
            return reinterpret_cast<const uint4*>(p.bounds + bounds_row(c, b, blk, page, g) * BOUND_ELEMS) + tig;
        };
        const uint4 *src0 = source(tile * 16 + gid, page0), *src1 = source(tile * 16 + gid + 8, page1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x0[j] = src0 ? read_global(src0 + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
            x1[j] = src1 ? read_global(src1 + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
        }
    };
    auto load_query = [&](int g, uint4 (&q4)[4]) {
        const uint4* qp = reinterpret_cast<const uint4*>(p.q + ((long long)b * c.Hq + g * c.G + min(gid, c.G - 1)) * HEAD_DIM) + tig;
#pragma unroll
        for (int j = 0; j < 4; ++j) q4[j] = gid < c.G ? read_global(qp + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
    };
    auto part_of = [](const uint4 (&q4)[4]) {
        return [&](int half, int j) -> uint4 {              // q-, q+
            const uint4 x = q4[j];
            return half ? make_uint4(bmax2(x.x, 0u), bmax2(x.y, 0u), bmax2(x.z, 0u), bmax2(x.w, 0u))
                        : make_uint4(bmin2(x.x, 0u), bmin2(x.y, 0u), bmin2(x.z, 0u), bmin2(x.w, 0u));
        };
    };
    auto heads_sum = [&](const float (&s)[4], float& x, float& y) {
        x = s[0] + s[1]; y = s[2] + s[3];
        x += __shfl_xor_sync(0xffffffffu, x, 1); y += __shfl_xor_sync(0xffffffffu, y, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2); y += __shfl_xor_sync(0xffffffffu, y, 2);
    };
    // what the row's heads add to e, by the warp that ranks the row, or a share of them by every warp
    auto query_share = [&]() {
        if (per_qhead) {
            if (mine) qsum = query_part(read_global(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h0) * HEAD_DIM) + lane), c.Hkv);
        } else {
#pragma unroll 1
            for (int h = h0 + wid; h < h1; h += W) qsum += query_part(read_global(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h) * HEAD_DIM) + lane), c.Hkv);
        }
    };
    int slices = 1;
    if constexpr (!SHARED) {
        uint4 q4[4];
        load_query(g0, q4);
        uint32_t low = 0u, high = 0x80008000u;
        uint32_t at[2];
        int dst[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int col = 2 * tig + i;
            dst[i] = col % size;
            at[i] = a_rows + (uint32_t)(col / size) * p.npad * 8;
        }
#pragma unroll 1
        for (int tile = wid; tile < tiles; tile += W) {
            uint4 x0[8], x1[8];
            load(tile, g0, x0, x1);
            if (first) query_share();
            float s[4];
            score_tile(x0, x1, part_of(q4), s, low, high);
            if (first && size > 1) cluster_wait();
            first = false;
            const int r0 = tile * 16 + gid;                 // (rows have room for whole tiles)
            if (per_qhead) {
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (2 * tig + i < c.G) {
                        st_cluster(at[i] + 4 * r0, dst[i], s[i]);
                        st_cluster(at[i] + 4 * (r0 + 8), dst[i], s[2 + i]);
                    }
            } else {
                float x, y;
                heads_sum(s, x, y);
                if (tig == 0) { st_cluster(a_rows + 4 * r0, 0, x); st_cluster(a_rows + 4 * (r0 + 8), 0, y); }
            }
        }
        amax = largest_bound(low, high);
    } else {
        slices = max(min(W / max(tiles, 1), c.Hkv), 1);
        const int per = (c.Hkv + slices - 1) / slices;
        slices = (c.Hkv + per - 1) / per;
#pragma unroll 1
        for (int task = wid; task < slices * tiles; task += W) {
            const int slice = task / tiles, tile = task - slice * tiles;
            float sx = 0.f, sy = 0.f;
#pragma unroll 1
            for (int g = slice * per; g < min((slice + 1) * per, c.Hkv); ++g) {
                uint4 x0[8], x1[8], q4[4];
                load(tile, g, x0, x1);
                load_query(g, q4);
                const float factor = p.k_scale ? read_global(p.k_scale + g) : 1.f;
                if (first) { query_share(); first = false; if (size > 1) cluster_wait(); }
                uint32_t low = 0u, high = 0x80008000u;
                float s[4], x, y;
                score_tile(x0, x1, part_of(q4), s, low, high);
                heads_sum(s, x, y);
                sx += x * factor; sy += y * factor;
                amax = fmaxf(amax, largest_bound(low, high) * fabsf(factor));
            }
            if (tig == 0) {
                const uint32_t to = a_rows + 4 * (uint32_t)(task * 16 + gid);
                st_cluster(to, 0, sx);
                st_cluster(to + 32, 0, sy);
            }
        }
    }
    if (first) { query_share(); if (size > 1) cluster_wait(); }
    amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));       // (not negative: ordered like its bits)
    if (lane < owners) {
        st_cluster(smem_u32(&s_part[wid].x), lane, amax);
        st_cluster(smem_u32(&s_part[wid].y), lane, qsum);
    }
    if constexpr (V == 0 && !SHARED) {                      // the group's queries, for scores in 64 bits
        for (int i = tid; i < c.G * (HEAD_DIM / 4); i += SC_THREADS)
            reinterpret_cast<uint2*>(sh.q[i / (HEAD_DIM / 4)])[i % (HEAD_DIM / 4)] =
                read_global(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + g0 * c.G) * HEAD_DIM) + i);
    }
    if (size > 1) cluster_arrive();                         // every score of the item is where it belongs ...
    if (g0 == 0 && rank == 0 && tid == 0 && p.idx_count) p.idx_count[b] = min(p.m, n);
    const int Hi = per_qhead ? c.Hq : (SHARED ? 1 : c.Hkv), hi0 = per_qhead ? g0 * c.G : g0;
    if (V > 0)                                              // (rank_row does it itself)
        for (int row = rank; row < rows; row += size) {
            int* const out = p.idx + ((long long)b * Hi + hi0 + row) * p.m;
            for (int i = min(p.m, n) + tid; i < p.m; i += blockDim.x) out[i] = -1;
        }
    if (size > 1) cluster_wait();                           // ... and nobody touches another CTA's memory from here on
    else __syncthreads();
    if (rank >= owners) return;
    float err = 0.f;
    const int padded = tiles * 16;
    if constexpr (V > 0) {
        if (!mine) return;
        float* const row = reinterpret_cast<float*>(sc_rows + (size_t)warp * p.npad * 8);
        float v[V], sum = 0.f;
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = j * 32 + lane < padded ? row[j * 32 + lane] : 0.f;
        for (int i = lane; i < W; i += 32) { err = fmaxf(err, s_part[i].x); sum += s_part[i].y; }
        err = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(err)));
        if (!per_qhead) {
#pragma unroll
            for (int sh = 16; sh >= 1; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
            qsum = sum;
        }
        rank_row_warp<V>(p, v, 2.01f * (err * qsum), reinterpret_cast<unsigned long long*>(row), b, h0, h1, n,
                         p.idx + ((long long)b * Hi + hi0 + my_row) * p.m);
    } else {
        if (tid < W) err = s_part[tid].x;
        float sum = 0.f;
        if (!per_qhead) for (int i = 0; i < W; ++i) sum += s_part[i].y;
#pragma unroll 1
        for (int r = rank, slot = 0; r < rows; r += size, ++slot) {
            if (slot > 0) __syncthreads();
            const float* row = reinterpret_cast<const float*>(sc_rows + (size_t)slot * p.npad * 8);
            float v[1][4] = {{0.f, 0.f, 0.f, 0.f}};
            if (tid * 4 < padded) {
                const float4 t = *reinterpret_cast<const float4*>(row + tid * 4);
                v[0][0] = t.x; v[0][1] = t.y; v[0][2] = t.z; v[0][3] = t.w;
                if constexpr (SHARED) {
#pragma unroll 4
                    for (int i = 1; i < slices; ++i) {
                        const float4 t = *reinterpret_cast<const float4*>(row + i * padded + tid * 4);
                        v[0][0] += t.x; v[0][1] += t.y; v[0][2] += t.z; v[0][3] += t.w;
                    }
                }
            }
            const int first_head = g0 * c.G + (per_qhead ? r : 0), end = per_qhead ? first_head + 1 : (SHARED ? c.Hq : first_head + c.G);
            if (per_qhead) sum = s_part[rank * NW + slot].y;            // (this CTA's warp `slot` worked it out)
            rank_row<SC_THREADS, 1>(p, sh.rank, v, err * sum, SHARED ? nullptr : &sh.q[per_qhead ? r : 0][0],
                                    reinterpret_cast<unsigned long long*>(sc_rows + (size_t)slot * p.npad * 8), b, first_head, end, n,
                                    p.idx + ((long long)b * Hi + hi0 + r) * p.m);
        }
    }
}

// ---- long contexts: scores by the whole GPU, then a CTA per row ----------------------------------------------------
// The scores are a stream of 8 KB tiles (16 blocks of one KV head). A warp, which is a CTA (so that what is left at the end is small),
// has SS_TILES of them in a row and a cp.async ring in shared memory; a slot is free as soon as its tile is in registers, so
// that two tiles are under way while one is worked on. (With loads straight into registers a warp had nothing under way while it
// worked. Four warps to a CTA and two slots: 12.8 and 23.3 us for the whole selection of 131072 positions and of a ragged batch of
// 8 x 65536; a warp and three slots: 12.4 and 22.8; four slots, with fewer CTAs per SM: 13.7 and 23.7.)
constexpr int SS_TILES = 4, SS_STAGES = 3;
constexpr int SS_BLOCKS = SS_TILES * 16;                    // blocks per warp: a chunk
constexpr int SS_ROW = BOUND_ELEMS * 2;                     // bytes of a block's bounds
constexpr int SS_SLOT = 16 * SS_ROW;
constexpr size_t SS_SMEM = (size_t)SS_STAGES * SS_SLOT;

__global__ void __launch_bounds__(32, 9) block_score_kernel(const __grid_constant__ SelectBlocksParams p) {
    const BlockCache& c = p.c;
    extern __shared__ __align__(128) uint8_t ss_ring[];
    const int lane = threadIdx.x, gid = lane >> 2, tig = lane & 3;
    // KV heads innermost: the CTAs that run together then read neighbouring 512 bytes of the same physical pages.
    const int part = blockIdx.x / c.Hkv, g = blockIdx.x - part * c.Hkv;
    const int b = part / p.chunks, chunk = part - b * p.chunks;
    const int blk0 = chunk * SS_BLOCKS;                     // the first block
    pdl_wait();
    pdl_trigger();
    const int len = c.ctx_lens[b];
    // Rows of the bounds, in units of `pitch`, of the chunk's blocks: lane l keeps blocks l, l + 32, ... Table entries are read along
    // with the length, as far as the table goes, whatever it holds there.
    constexpr int PER = SS_TILES / 2;
    int at[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        at[i] = blk0 + lane + 32 * i;
        if (c.paged) at[i] = at[i] < c.max_blocks ? read_global(c.page_table + (long long)b * c.max_pages + at[i]) : -1;
    }
    uint4 q4[4];
    const uint4* qp = reinterpret_cast<const uint4*>(p.q + ((long long)b * c.Hq + g * c.G + min(gid, c.G - 1)) * HEAD_DIM) + tig;
    const bool on = gid < c.G;
#pragma unroll
    for (int j = 0; j < 4; ++j) q4[j] = on ? read_global(qp + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
    const int n = (max(min(len, c.max_ctx), 0) + TILE - 1) / TILE;
    if (blk0 >= n) return;
    if (c.paged) {
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (blk0 + lane + 32 * i < n && (unsigned)at[i] >= (unsigned)c.num_pages) {
                atomicOr(c.status, STATUS_BAD_PAGE);
                at[i] = 0;                                  // (any page: a block without one has no score to speak of)
            }
    }
    const uint8_t* base = reinterpret_cast<const uint8_t*>(p.bounds) + (c.paged ? (long long)g : ((long long)b * c.Hkv + g) * c.bound_blocks) * SS_ROW + lane * 16;
    const long long pitch = c.paged ? (long long)c.Hkv * SS_ROW : SS_ROW;
    const uint32_t ring = smem_u32(ss_ring);
    const int valid = min(SS_BLOCKS, n - blk0), tiles = (valid + 15) / 16;
    // One instruction copies a block's 512 bytes; piece c of row r goes to c ^ ((r & 1) << 2), so that the fragment reads
    // below (two rows, four pieces per eight lanes) meet no bank twice. The last block stands in for those behind it.
    auto issue = [&](int t, uint32_t slot) {
        int mine = at[0];
#pragma unroll
        for (int i = 1; i < PER; ++i) if ((t >> 1) == i) mine = at[i];
        const int first = (t & 1) * 16, last = min(15, valid - 1 - t * 16);
        const uint32_t even = slot + lane * 16, odd = slot + (lane ^ 4) * 16;
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const int row = __shfl_sync(0xffffffffu, mine, first + min(r, last));
            cp_async16_full((r & 1 ? odd : even) + r * SS_ROW, base + row * pitch);
        }
    };
    uint4 qs[2][4];                                         // q-, q+
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        qs[0][j] = make_uint4(bmin2(q4[j].x, 0u), bmin2(q4[j].y, 0u), bmin2(q4[j].z, 0u), bmin2(q4[j].w, 0u));
        qs[1][j] = make_uint4(bmax2(q4[j].x, 0u), bmax2(q4[j].y, 0u), bmax2(q4[j].z, 0u), bmax2(q4[j].w, 0u));
    }
    uint32_t low = 0u, high = 0x80008000u;
    const float f = p.k_scale ? read_global(p.k_scale + g) : 1.f;
    float* const row = p.scores + (p.mode == 0 ? (long long)b * c.Hq + g * c.G : (long long)b * c.Hkv + g) * p.npad;
#pragma unroll
    for (int t = 0; t < SS_STAGES; ++t) {
        if (t < tiles) issue(t, ring + t * SS_SLOT);
        cp_async_commit();
    }
    uint32_t slot = ring;
#pragma unroll 1
    for (int t = 0; t < tiles; ++t) {
        cp_async_wait<SS_STAGES - 1>();
        __syncwarp();
        uint4 x0[8], x1[8];
        const uint32_t frag = slot + gid * SS_ROW, swz = (gid & 1) << 2;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            uint32_t a[4], d[4];
            lds128(frag + (((tig + 4 * j) ^ swz) << 4), a);
            lds128(frag + 8 * SS_ROW + (((tig + 4 * j) ^ swz) << 4), d);
            x0[j] = make_uint4(a[0], a[1], a[2], a[3]);
            x1[j] = make_uint4(d[0], d[1], d[2], d[3]);
        }
        __syncwarp();                                       // every lane has its pieces: the slot is free
        if (t + SS_STAGES < tiles) issue(t + SS_STAGES, slot);
        cp_async_commit();
        slot = slot == ring + (SS_STAGES - 1) * SS_SLOT ? ring : slot + SS_SLOT;
        float s[4];
        score_tile(x0, x1, [&](int half, int j) { return qs[half][j]; }, s, low, high);
        const int r0 = blk0 + t * 16 + gid, r1 = r0 + 8;
        if (p.mode == 0) {
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
            if (tig == 0 && r0 < n) row[r0] = x * f;
            if (tig == 0 && r1 < n) row[r1] = y * f;
        }
    }
    // ---- the chunk's share of e, per row ---------------------------------------------------------------------------------
    const float amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(largest_bound(low, high))));
    // 2^-15 max|q| + (24 + Hkv) 2^-24 sum|q| of head gid, whose row the four lanes of a gid hold between them
    float big = 0.f, sum = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w[4] = {q4[j].x, q4[j].y, q4[j].z, q4[j].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float lo = fabsf(__uint_as_float(w[i] << 16)), hi = fabsf(__uint_as_float(w[i] & 0xffff0000u));
            big = fmaxf(big, fmaxf(lo, hi));
            sum += lo + hi;
        }
    }
#pragma unroll
    for (int sh = 1; sh <= 2; sh <<= 1) {
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, sh));
        sum += __shfl_xor_sync(0xffffffffu, sum, sh);
    }
    float e = on ? amax * (big * (1.f / 32768.f) + sum * (float)(24 + c.Hkv) * (1.f / 16777216.f)) * fabsf(f) : 0.f;
    if (p.mode == 0) {
        if (on && tig == 0) p.err[((long long)b * c.Hq + g * c.G + gid) * p.chunks + chunk] = e;
    } else {
#pragma unroll
        for (int sh = 4; sh <= 16; sh <<= 1) e += __shfl_xor_sync(0xffffffffu, e, sh);
        if (lane == 0) p.err[((long long)b * c.Hkv + g) * p.chunks + chunk] = e;
    }
}

// Dynamic shared memory: 8 bytes per block for keys.
// (A bound on the CTAs per SM for the sake of the registers: without it the compiler stops at 64 and spills, 25.3 us against 23.4 for the
// 256 rows of a ragged batch of 8 x 65536.)
template <int NT, int V>
__global__ void __launch_bounds__(NT, 512 / NT) block_rank_kernel(const __grid_constant__ SelectBlocksParams p) {
    const BlockCache& c = p.c;
    extern __shared__ __align__(16) uint8_t rk_keys[];
    __shared__ __align__(16) RankShared<NT, V> sh;
    __shared__ __align__(16) __nv_bfloat16 s_q[8][SB_QROW];
    const int tid = threadIdx.x;
    const bool shared_set = p.mode == 2, per_qhead = p.mode == 0;
    const int Hi = per_qhead ? c.Hq : (shared_set ? 1 : c.Hkv);
    const int b = blockIdx.x / Hi, hi = blockIdx.x - b * Hi;
    const int members = c.Hq / Hi, h0 = hi * members, h1 = h0 + members;
    pdl_wait();
    pdl_trigger();
    // (rows of npad scores: what lies behind the length is read, and ignored when the length is there)
    const int len = c.ctx_lens[b];
    const int sum_rows = shared_set ? c.Hkv : 1;
    const long long row0 = (long long)b * (per_qhead ? c.Hq : c.Hkv) + (shared_set ? 0 : hi);
    const float* row = p.scores + row0 * p.npad;
    float v[V][4];
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const int at = (j * NT + tid) * 4;
        float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
        if (at < p.npad) t = __ldcg(reinterpret_cast<const float4*>(row + at));
        v[j][0] = t.x; v[j][1] = t.y; v[j][2] = t.z; v[j][3] = t.w;
    }
    const int errs = sum_rows * p.chunks;
    const float err0 = tid < errs ? __ldcg(p.err + row0 * p.chunks + tid) : 0.f;
    if (!shared_set)                                        // the members' queries, for scores in 64 bits
        for (int i = tid; i < members * (HEAD_DIM / 4); i += NT)
            reinterpret_cast<uint2*>(s_q[i / (HEAD_DIM / 4)])[i % (HEAD_DIM / 4)] =
                read_global(reinterpret_cast<const uint2*>(p.q + ((long long)b * c.Hq + h0) * HEAD_DIM) + i);
#pragma unroll 2
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
    // e: the sum over the rows added up is at most their number times the largest
    float err = tid < errs && tid % p.chunks < used ? err0 : 0.f;
#pragma unroll 4
    for (int i = tid + NT; i < errs; i += NT) if (i % p.chunks < used) err = fmaxf(err, __ldcg(p.err + row0 * p.chunks + i));
    err *= (float)sum_rows;
    if (hi == 0 && tid == 0 && p.idx_count) p.idx_count[b] = min(p.m, n);
    rank_row<NT, V>(p, sh, v, err, shared_set ? nullptr : &s_q[0][0], reinterpret_cast<unsigned long long*>(rk_keys), b, h0, h1, n,
                    p.idx + ((long long)b * Hi + hi) * p.m);
}

}  // namespace tidal
