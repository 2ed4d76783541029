// The attention weight that every cached position receives from a chunk of new tokens, given the chunk's log-sum-exps.
//
//   w[b, head, j] = decay w[b, head, j] + sum over queries t and query heads of the head of exp(scale q_t . k_j - lse_t),  j <= position of t
//
// A persistent CTA takes tiles of 128 positions one after the other: S^T = K Q^T into TMEM, positions as rows, so that a thread
// owns a position and adds up along its row in registers; no atomics, the same sum in the same order every time. Keys are
// read once. Two pairs of warpgroups take the tiles in turn, a pair's warpgroups its products (an accumulator in TMEM each), so that the
// exponentials of four run beside the products and loads of the next. Single tokens (64 sequences of up to 16384 in
// pages: 209 us, 5.2 TB/s) are bound by the copies of 16 rows of 128 bytes, of which an SM takes 27 bytes a clock, and by the issuing warp's turns; many
// queries (64 of 131072: 92 us) by the exponential unit, 16 a clock and SM.
#pragma once

#include "chunk_kernels.cuh"

namespace tidal {

struct WeightParams {
    BlockCache c;
    int page_mul, batch_mul, head_mul;
    const int* q_offsets;
    int num_tokens, tile_tokens;                            // tokens per product
    int causal, window, last;                               // last > 0: only a chunk's last so many queries count
    float scale_log2, decay;
    const float* k_scale;
    const float* lse;
    float* weights;
    long long stride;
    int heads;                                              // Hkv, or 1: all heads together
    int strided;                                            // a CTA takes every gridDim.x-th tile instead of a run of them
};

constexpr int CW_THREADS = 640, CW_THREADS8 = 768, CW_RING = 3, CW_QRING = 3, CW_QRING8 = 2, CW_BUFS = 4;
constexpr size_t cw_smem(bool kv8) { return 1024 + (size_t)(CW_RING + (kv8 ? CW_QRING8 : CW_QRING)) * CH_MAT + (kv8 ? CH_RAW * CH_HALF : 0); }

struct WeightShared {
    unsigned long long k_full[CW_RING], k_empty[CW_RING], q_full[CW_QRING], q_empty[CW_QRING], d_full[CW_BUFS], d_empty[CW_BUFS], raw_full[CH_RAW], raw_empty[CH_RAW];
    uint32_t tmem;
    int gave_up;
    // Per tile of positions with products, bit i: its i-th page is not one. Read before the warpgroup arrives for the last of its products with the tile: until
    // then its pair's next-but-one product waits, so that tiles up to four further on are in work and five more on their way.
    unsigned bad_pages[CH_TAGS];
    alignas(16) float lse2[4][2][CH_TILE];                  // per warpgroup and turn: minus a row's log-sum-exp in base 2 (read four at a time), and what it sees
    int2 sees[4][2][CH_TILE];
    float sums[2][2][CH_TILE];                              // per pair: the second warpgroup's part of a tile
};

// A walk over a CTA's tiles of positions. A run of all sequences' and weight heads' tiles, so that it meets few
// sequences and their queries stay; where new tokens are a good part of the context, so that the tiles they see are not alike, every gridDim.x-th.
struct WeightWalk {
    long long left;                                         // tiles to come
    int step, b, ctx, tiles, first, begin, chunk;           // first: position of the first new token; begin: its row; chunk: new tokens
    int head, tile, key0, g0, g1, t0, q0, q1, all_q;        // the tile; KV heads; first query, products that see the tile, products of the sequence
    int alike;                                              // tiles of the head before this one differ in their place only: all queries see them, or the one product
};

__device__ __forceinline__ void weight_sequence(const WeightParams& p, WeightWalk& w, int b) {
    w.b = b;
    w.ctx = cached_len(p.c, b);
    w.tiles = (w.ctx + CH_TILE - 1) / CH_TILE;
    w.begin = max(min(read_global(p.q_offsets + b), p.num_tokens), 0);
    w.chunk = max(min(read_global(p.q_offsets + b + 1), p.num_tokens), w.begin) - w.begin;
    w.first = w.ctx - w.chunk;
}
// From tile w.tile of head w.head on to one that is there (both may stand behind the sequence's last).
__device__ __forceinline__ void weight_settle(const WeightParams& p, WeightWalk& w) {
    while (w.tile >= w.tiles) {
        w.tile -= w.tiles;
        if (++w.head < p.heads && w.tiles > 0) continue;
        w.head = 0;
        if (w.b + 1 >= p.c.batch) { w.left = 0; return; }
        weight_sequence(p, w, w.b + 1);
    }
}
// All lanes of a warp together.
__device__ __forceinline__ void weight_start(const WeightParams& p, WeightWalk& w, int lane) {
    long long all = 0;
    for (int b0 = 0; b0 < p.c.batch; b0 += 32) {
        int n = b0 + lane < p.c.batch ? (cached_len(p.c, b0 + lane) + CH_TILE - 1) / CH_TILE : 0;
#pragma unroll
        for (int sh = 16; sh; sh >>= 1) n += __shfl_xor_sync(0xffffffffu, n, sh);
        all += n;
    }
    all *= p.heads;
    long long at = blockIdx.x;
    w.step = (int)gridDim.x;
    w.left = at < all ? (all - at + w.step - 1) / w.step : 0;
    if (!p.strided) {
        at = all * blockIdx.x / gridDim.x;
        w.left = all * (blockIdx.x + 1) / gridDim.x - at;
        w.step = 1;
    }
    // the sequence it lies in: whole ones are passed 32 at a time
    int b = 0;
    for (int b0 = 0; b0 < p.c.batch; b0 += 32) {
        const int n = b0 + lane < p.c.batch ? (cached_len(p.c, b0 + lane) + CH_TILE - 1) / CH_TILE * p.heads : 0;
        int x = n;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, sh); if (lane >= sh) x += y; }
        const unsigned over = __ballot_sync(0xffffffffu, x > at);
        const int last = over ? __ffs(over) - 1 : 31;
        b = min(b0 + last, p.c.batch - 1);
        at -= __shfl_sync(0xffffffffu, over ? x - n : x, last);
        if (over) break;
    }
    weight_sequence(p, w, b);
    w.alike = 0;
    w.head = w.tiles > 0 ? (int)(at / w.tiles) : 0;
    w.tile = (int)(at - (long long)w.head * w.tiles);
}
// The next tile; false behind the last.
__device__ __forceinline__ bool weight_tile(const WeightParams& p, WeightWalk& w) {
    if (w.left <= 0) return false;
    if (w.tile < w.alike) {                                 // (few instructions: the issuing warp's turns are the bound)
        --w.left;
        w.key0 = w.tile * CH_TILE;
        return true;
    }
    w.alike = 0;
    weight_settle(p, w);
    if (w.left <= 0) return false;
    --w.left;
    w.key0 = w.tile * CH_TILE;
    w.g0 = p.heads > 1 ? w.head : 0;
    w.g1 = p.heads > 1 ? w.head + 1 : p.c.Hkv;
    w.t0 = p.last > 0 ? max(w.chunk - p.last, 0) : 0;
    const int from = w.first + w.t0, n = w.chunk - w.t0;     // position of the first query that counts, how many
    w.q0 = 0;
    w.q1 = n <= p.tile_tokens ? (n > 0) : (n + p.tile_tokens - 1) / p.tile_tokens;
    w.all_q = w.q1;
    if (p.causal && w.key0 > from) w.q0 = (w.key0 - from) / p.tile_tokens;
    if (p.window > 0) {
        const long long last = (long long)w.key0 + CH_TILE - 1 + p.window - 1 - from;      // the last query whose window reaches the tile
        w.q1 = last < 0 ? 0 : (int)min((long long)w.q1, last / p.tile_tokens + 1);
    }
    w.q0 = min(w.q0, w.q1);
    // (a lone product's last query stands in the sequence's last tile; of several the first sees the tiles up to its own)
    if (p.window <= 0 && w.q0 == 0) w.alike = w.all_q <= 1 || !p.causal ? w.tiles : min(w.tiles, max(from, 0) / CH_TILE + 1);
    return true;
}

template <bool KV8>
__global__ void __launch_bounds__(KV8 ? CW_THREADS8 : CW_THREADS, 1)
chunk_weights_kernel(const __grid_constant__ WeightParams p, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map) {
    extern __shared__ unsigned char cw_raw_smem[];
    constexpr int QRING = KV8 ? CW_QRING8 : CW_QRING;
    __shared__ WeightShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t k_ring = (smem_u32(cw_raw_smem) + 1023u) & ~1023u, q_ring = k_ring + CW_RING * CH_MAT, raw = q_ring + QRING * CH_MAT;
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n");
    }
    if (tid == 32) {
        for (int i = 0; i < CW_RING; ++i) {
            bar_init(smem_u32(&sh.k_full[i]), KV8 ? 4 : 1); bar_init(smem_u32(&sh.k_empty[i]), 1);
        }
        for (int i = 0; i < QRING; ++i) { bar_init(smem_u32(&sh.q_full[i]), 1); bar_init(smem_u32(&sh.q_empty[i]), 1); }
        for (int i = 0; i < CW_BUFS; ++i) { bar_init(smem_u32(&sh.d_full[i]), 1); bar_init(smem_u32(&sh.d_empty[i]), 4); }
        for (int i = 0; i < CH_RAW; ++i) { bar_init(smem_u32(&sh.raw_full[i]), 1); bar_init(smem_u32(&sh.raw_empty[i]), 4); }
        sh.gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    pdl_wait();
    pdl_trigger();
    const uint32_t tmem = sh.tmem;
    volatile int* const gave_up = &sh.gave_up;
    const int G = p.c.G, tt = p.tile_tokens;
    bool ok = true;
    WeightWalk w;
    weight_start(p, w, lane);

    if (warp < 16) {
        // ---- sums ----
        // (Nothing here hangs on how a wait ended: warps meet at named barriers, which know no limit, so all of them take all steps, whatever has run out.)
        const int wg = warp >> 2, pair = wg >> 1, s = wg & 1, row = tid & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        if (blockIdx.x == 0)                                // offsets that are cut are reported
            for (int b = tid; b < p.c.batch; b += 512) {
                const int x = read_global(p.q_offsets + b), y = read_global(p.q_offsets + b + 1);
                if (x < 0 || y < x || y > p.num_tokens) atomicOr(p.c.status, STATUS_BAD_INDEX);
            }
        int step = 0, tag = 0, turn = 0, item = 0, count = 0;           // the pair's products, tiles with products, own fillings, the pair's joined tiles, tiles of positions
        long long filled = -1;                              // the queries whose sums are in shared memory
        for (; weight_tile(p, w); w.tile += w.step) {
            const int key = w.key0 + row, steps = (w.q1 - w.q0) * (w.g1 - w.g0), first_step = step;
            float acc = 0.f;
            if ((count++ & 1) != pair) {                    // the other pair's
                tag += w.q1 > w.q0;
                continue;
            }
            for (int g = w.g0; g < w.g1; ++g) {
                float part = 0.f;
                unsigned skip = 0;
                for (int q = w.q0; q < w.q1; ++q, ++step) {
                    if ((step & 1) != s) continue;
                    const int t = w.t0 + q * tt, rows = min(tt, w.chunk - t) * G;      // first token, rows that count
                    const int buf = wg, cols = (rows + 31) & ~31;
                    const float scale = p.scale_log2 * (KV8 && p.k_scale ? read_global(p.k_scale + g) : 1.f);
                    const long long these = ((long long)w.b * p.c.Hkv + g) << 32 | q;
                    if (these != filled) {                  // (a run of tiles has the same queries)
                        filled = these;
                        ++turn;
                        const int pos = w.first + t + row / G;
                        const bool counts = row < rows;
                        sh.lse2[wg][turn & 1][row] = counts ? read_global(p.lse + (long long)(w.begin + t + row / G) * p.c.Hq + g * G + row % G) * -1.4426950408889634f : 0.f;
                        sh.sees[wg][turn & 1][row] = counts ? make_int2(p.window > 0 ? max(pos - p.window + 1, 0) : 0, p.causal ? min(pos + 1, w.ctx) : w.ctx) : make_int2(0, 0);
                        asm volatile("bar.sync %0, 128;\n" ::"r"(1 + wg) : "memory");
                    }
                    const float* const lse2 = sh.lse2[wg][turn & 1];
                    const int2* const sees = sh.sees[wg][turn & 1];
                    bar_pass<true>(smem_u32(&sh.d_full[buf]), (step >> 1) & 1, gave_up);
                    tmem_fence_after();
                    const bool all = (!p.causal || w.key0 + CH_TILE - 1 <= w.first + t) && (p.window <= 0 || w.first + t + (rows - 1) / G - p.window < w.key0);
                    const f32pair scale2 = pair2(scale, scale);
                    for (int c = 0; c < cols; c += 32) {
                        uint32_t x[32];
                        __syncwarp();
                        tmem_ld32(tmem + lanes + buf * CH_TILE + c, x);
                        tmem_wait_ld();
                        tmem_loaded32(x);
                        if (all && c + 32 <= rows) {
                            f32pair sum0 = pair2(0.f, 0.f), sum1 = sum0;
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const float4 l = *reinterpret_cast<const float4*>(lse2 + c + j);
                                const f32pair a = fma2(pair2(__uint_as_float(x[j]), __uint_as_float(x[j + 1])), scale2, pair2(l.x, l.y));
                                const f32pair b = fma2(pair2(__uint_as_float(x[j + 2]), __uint_as_float(x[j + 3])), scale2, pair2(l.z, l.w));
                                sum0 = add2(sum0, pair2(fast_exp2(half2(a, 0)), fast_exp2(half2(a, 1))));
                                sum1 = add2(sum1, pair2(fast_exp2(half2(b, 0)), fast_exp2(half2(b, 1))));
                            }
                            sum0 = add2(sum0, sum1);
                            part += half2(sum0, 0) + half2(sum0, 1);
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                const int2 range = sees[c + j];
                                const float e = fast_exp2(fmaf(__uint_as_float(x[j]), scale, lse2[c + j]));
                                if (key >= range.x && key < range.y) part += e;
                            }
                        }
                    }
                    skip = *(volatile unsigned*)&sh.bad_pages[tag % CH_TAGS];
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&sh.d_empty[buf]));
                }
                // a page id outside the pool: its positions receive nothing
                if ((skip >> (row / TILE)) & 1) part = 0.f;
                acc += part;
            }
            tag += w.q1 > w.q0;
            bool writes = steps == 0 ? s == 0 : (first_step & 1) == s;
            if (steps > 1) {
                // the second warpgroup leaves its part and goes on, the first adds it (barriers 5 + 4 pair: a part is there; two further on: its
                // place is free again)
                const int there = 5 + 4 * pair + (item & 1), free = there + 2;
                if (s == 1) {
                    if (item >= 2) asm volatile("bar.sync %0, 256;\n" ::"r"(free) : "memory");
                    sh.sums[pair][item & 1][row] = acc;
                    asm volatile("bar.arrive %0, 256;\n" ::"r"(there) : "memory");
                } else {
                    asm volatile("bar.sync %0, 256;\n" ::"r"(there) : "memory");
                    acc += sh.sums[pair][item & 1][row];
                    asm volatile("bar.arrive %0, 256;\n" ::"r"(free) : "memory");
                }
                writes = s == 0;
                ++item;
            }
            if (writes && key < w.ctx) {
                float* const to = p.weights + ((long long)w.b * p.heads + w.head) * p.stride + key;
                if (p.decay != 0.f && key < w.first) acc = fmaf(p.decay, read_global(to), acc);
                *to = acc;
            }
        }
    } else if (warp == 16) {
        // ---- products: the whole warp walks, one lane issues (see chunk_attn_kernel) ----
        const uint32_t d = uniform(tmem);
        int steps[2] = {0, 0}, count = 0, ks = 0, kp = 0;
        unsigned held = 0, qp = 0;                          // slots of queries that stay, parities of the slots' next fillings
        long long group = -1;
        for (; ok && weight_tile(p, w); w.tile += w.step) {
            const int pair = count++ & 1;
            for (int g = w.g0; g < w.g1 && ok && w.q0 < w.q1; ++g) {
                if (const long long these = (long long)w.b * p.c.Hkv + g; these != group) {
                    if (elected())
                        for (int i = 0; i < QRING; ++i) if ((held >> i) & 1) mma_commit(smem_u32(&sh.q_empty[i]));
                    __syncwarp();
                    held = 0;
                    group = these;
                }
                ok = bar_wait<false>(smem_u32(&sh.k_full[ks]), kp, gave_up);
                for (int q = w.q0; q < w.q1 && ok; ++q) {
                    const int step = pair ? steps[1]++ : steps[0]++, buf = 2 * pair + (step & 1);
                    const int rows = min(tt, w.chunk - w.t0 - q * tt) * G, cols = (rows + 31) & ~31;
                    // Queries have the slot of their number; where a sequence and head has no more than there are slots they stay while it does.
                    const int qs = q % QRING;
                    const bool stay = w.all_q <= QRING, fresh = !((held >> qs) & 1);
                    ok = (!fresh || bar_wait<false>(smem_u32(&sh.q_full[qs]), (qp >> qs) & 1, gave_up)) &&
                         (step < 2 || bar_wait<false>(smem_u32(&sh.d_empty[buf]), ((step >> 1) - 1) & 1, gave_up));
                    if (!ok) break;
                    tmem_fence_after();
                    const uint64_t a = smem_matrix(k_ring + ks * CH_MAT, 16), b = smem_matrix(q_ring + qs * CH_MAT, 16);
                    const uint32_t shape = mma_shape(true, uniform(cols), false);
                    if (elected()) {
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk) {
                            const uint32_t off = ((kk >> 2) * CH_HALF + (kk & 3) * 32) >> 4;
                            mma_ss(d + buf * CH_TILE, a + off, b + off, shape, kk > 0);
                        }
                        mma_commit(smem_u32(&sh.d_full[buf]));
                        if (!stay) mma_commit(smem_u32(&sh.q_empty[qs]));
                        if (q == w.q1 - 1) mma_commit(smem_u32(&sh.k_empty[ks]));
                    }
                    __syncwarp();
                    if (fresh) qp ^= 1u << qs;
                    if (stay) held |= 1u << qs;
                }
                if (++ks == CW_RING) { ks = 0; kp ^= 1; }
            }
        }
    } else if (warp == 17 || warp == 18) {
        // ---- keys in: two warps, a tile each in turn; the pages of a warp's next tile are looked up before it waits for this one's place ----
        int tile = 0, tag = 0;                              // of all (tile, KV head) so far; of tiles with products
        auto lookup = [&](unsigned& bad) {
            int page = 0;
            bad = 0;
            if (p.c.paged) {
                page = p.c.num_pages;                       // (out of range: filled with zeros)
                const int blk = w.key0 / TILE + (lane & 7);
                if (blk * TILE < w.ctx) {
                    page = read_global(p.c.page_table + (long long)w.b * p.c.max_pages + blk);
                    if ((unsigned)page >= (unsigned)p.c.num_pages) { page = p.c.num_pages; bad = 1; }
                }
            }
            return page;
        };
        bool more = weight_tile(p, w);
        unsigned bad = 0;
        int page = more ? lookup(bad) : 0;
        while (more && ok) {
            const int b = w.b, key0 = w.key0, g0 = w.g0, g1 = w.q0 < w.q1 ? w.g1 : w.g0, here = page;
            const unsigned skip = __ballot_sync(0xffffffffu, bad) & 0xffu;
            if (skip && g1 > g0) {                          // pages before the first query's window are nobody's
                const int before = p.window > 0 ? min(max((w.first + w.t0 - p.window + 1 - key0) / TILE, 0), 8) : 0;
                if (lane == 0 && skip >> before) atomicOr(p.c.status, STATUS_BAD_PAGE);
            }
            w.tile += w.step;
            more = weight_tile(p, w);
            if (more) page = lookup(bad);
            for (int g = g0; g < g1 && ok; ++g, ++tile) {
                if ((tile & 1) != warp - 17) continue;
                const int slot = KV8 ? tile % CH_RAW : tile % CW_RING;
                if constexpr (KV8) { if (tile >= CH_RAW) ok = bar_wait<false>(smem_u32(&sh.raw_empty[slot]), (tile / CH_RAW - 1) & 1, gave_up); }
                else { if (tile >= CW_RING) ok = bar_wait<false>(smem_u32(&sh.k_empty[slot]), (tile / CW_RING - 1) & 1, gave_up); }
                if (!ok) break;
                const uint32_t dst = KV8 ? raw + slot * CH_HALF : k_ring + slot * CH_MAT, bar = smem_u32(KV8 ? &sh.raw_full[slot] : &sh.k_full[slot]);
                if (lane == 0) {
                    sh.bad_pages[tag % CH_TAGS] = skip;
                    bar_expect(bar, KV8 ? CH_HALF : CH_MAT);
                }
                __syncwarp();
                constexpr int HALVES = KV8 ? 1 : 2;
                if (p.c.paged) {
                    if (lane < 8 * HALVES)
                        tma_load4(dst + (lane >> 3) * CH_HALF + (lane & 7) * 2048, &k_map, bar, (lane >> 3) * 64, 0, g * p.head_mul,
                                  here * p.page_mul + (here == p.c.num_pages && !p.page_mul ? 1 : 0));
                } else if (lane < HALVES) {
                    tma_load4(dst + lane * CH_HALF, &k_map, bar, lane * 64, key0, g * p.head_mul, b * p.batch_mul);
                }
            }
            tag += g1 > g0;
        }
    } else if (warp == 19) {
        // ---- queries in, unless they are there ----
        unsigned held = 0, used = 0, parity = 0;
        long long group = -1;
        for (; ok && weight_tile(p, w); w.tile += w.step)
            for (int g = w.g0; g < w.g1 && ok && w.q0 < w.q1; ++g) {
                if (const long long these = (long long)w.b * p.c.Hkv + g; these != group) { group = these; held = 0; }
                for (int q = w.q0; q < w.q1 && ok; ++q) {
                    const int qs = q % QRING;
                    if ((held >> qs) & 1) continue;
                    if ((used >> qs) & 1) {
                        ok = bar_wait<false>(smem_u32(&sh.q_empty[qs]), (parity >> qs) & 1, gave_up);
                        parity ^= 1u << qs;
                    }
                    if (!ok) break;
                    if (elected()) {
                        bar_expect(smem_u32(&sh.q_full[qs]), 2 * G * tt * 128);
                        for (int h = 0; h < 2; ++h)
                            tma_load3(q_ring + qs * CH_MAT + h * CH_HALF, &q_map, smem_u32(&sh.q_full[qs]), h * 64, g * G, w.begin + w.t0 + q * tt);
                    }
                    __syncwarp();
                    used |= 1u << qs;
                    if (w.all_q <= QRING) held |= 1u << qs;
                }
            }
    } else if (KV8) {
        // ---- codes to bf16 ----
        const int l = tid - 640;
        int tile = 0;
        for (; ok && weight_tile(p, w); w.tile += w.step)
            for (int g = w.g0; g < w.g1 && ok && w.q0 < w.q1; ++g, ++tile) {
                const int rs = tile % CH_RAW, slot = tile % CW_RING;
                ok = bar_wait<false>(smem_u32(&sh.raw_full[rs]), (tile / CH_RAW) & 1, gave_up) &&
                     (tile < CW_RING || bar_wait<false>(smem_u32(&sh.k_empty[slot]), (tile / CW_RING - 1) & 1, gave_up));
                if (!ok) break;
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const int k = u * 128 + l, r = k >> 3, c = k & 7;
                    uint32_t x[4], y[8];
                    lds128(raw + rs * CH_HALF + r * 128 + ((c ^ (r & 7)) << 4), x);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        e4m3x4_to_f16x2x2(x[j], y[2 * j], y[2 * j + 1]);
                        y[2 * j] = f16x2_to_bf16x2(y[2 * j]);
                        y[2 * j + 1] = f16x2_to_bf16x2(y[2 * j + 1]);
                    }
                    const uint32_t to = k_ring + slot * CH_MAT + (c >> 2) * CH_HALF + r * 128;
                    const int c0 = 2 * (c & 3);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(to + ((c0 ^ (r & 7)) << 4)), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(to + (((c0 + 1) ^ (r & 7)) << 4)), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
                }
                smem_to_async();
                __syncwarp();
                if (lane == 0) { bar_arrive(smem_u32(&sh.k_full[slot])); bar_arrive(smem_u32(&sh.raw_empty[rs])); }
            }
    }
    __syncwarp();
    if (sh.gave_up) let_land();
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem));
    if (tid == 0 && sh.gave_up) atomicOr(p.c.status, STATUS_WAITED_OUT);
}

}  // namespace tidal
