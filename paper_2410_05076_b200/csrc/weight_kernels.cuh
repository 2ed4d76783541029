// The attention weight that every cached position receives from a chunk of new tokens, given the chunk's log-sum-exps.
//
//   w[b, head, j] = decay w[b, head, j] + sum over queries t and query heads of the head of exp(scale q_t . k_j - lse_t),  j <= position of t
//
// A persistent CTA takes tiles of 128 positions one after the other: S^T = K Q^T into TMEM, positions as rows, so that a thread
// owns a position and adds up along its row in registers; no atomics, the same sum in the same order every time. Keys are
// read once. Two warpgroups take the products in turn (four accumulators in TMEM), so that the exponentials of one run beside the products and
// loads of the next. Bound by memory where a sequence has few new tokens, by the exponentials (16 a clock and SM) where it has many.
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
};

constexpr int CW_THREADS = 320, CW_THREADS8 = 448, CW_RING = 3, CW_QRING = 3, CW_QRING8 = 2, CW_BUFS = 4;
constexpr size_t cw_smem(bool kv8) { return 1024 + (size_t)(CW_RING + (kv8 ? CW_QRING8 : CW_QRING)) * CH_MAT + (kv8 ? CH_RAW * CH_HALF : 0); }

struct WeightShared {
    unsigned long long k_full[CW_RING], k_empty[CW_RING], q_full[CW_QRING], q_empty[CW_QRING], d_full[CW_BUFS], d_empty[CW_BUFS], raw_full[CH_RAW], raw_empty[CH_RAW];
    uint32_t tmem;
    int gave_up;
    unsigned bad_pages[CH_TAGS];
    alignas(16) float lse2[2][2][CH_TILE];                  // per warpgroup and turn: a row's log-sum-exp in base 2 (read four at a time), and what it sees
    int2 sees[2][2][CH_TILE];
    float sums[2][CH_TILE];
};

// A walk over a CTA's tiles of positions: every gridDim.x-th of all sequences' and weight heads'.
struct WeightWalk {
    long long at, end;                                      // the tile's number among all, where its sequence ends
    int b, ctx, tiles, first, begin, chunk;                 // first: position of the first new token; begin: its row; chunk: new tokens
    int head, key0, g0, g1, t0, q0, q1;                     // the tile; KV heads; first query, products that see the tile
};

__device__ __forceinline__ void weight_sequence(const WeightParams& p, WeightWalk& w, int b) {
    w.b = b;
    w.ctx = cached_len(p.c, b);
    w.tiles = (w.ctx + CH_TILE - 1) / CH_TILE;
    w.begin = max(min(read_global(p.q_offsets + b), p.num_tokens), 0);
    w.chunk = max(min(read_global(p.q_offsets + b + 1), p.num_tokens), w.begin) - w.begin;
    w.first = w.ctx - w.chunk;
}
__device__ __forceinline__ void weight_start(const WeightParams& p, WeightWalk& w) {
    w.at = blockIdx.x;
    weight_sequence(p, w, 0);
    w.end = (long long)w.tiles * p.heads;
}
// The tile at w.at; false behind the last.
__device__ __forceinline__ bool weight_tile(const WeightParams& p, WeightWalk& w) {
    while (w.at >= w.end) {
        if (w.b + 1 >= p.c.batch) return false;
        weight_sequence(p, w, w.b + 1);
        w.end += (long long)w.tiles * p.heads;
    }
    const int i = (int)(w.at - (w.end - (long long)w.tiles * p.heads));
    w.head = i / w.tiles;
    w.key0 = (i - w.head * w.tiles) * CH_TILE;
    w.g0 = p.heads > 1 ? w.head : 0;
    w.g1 = p.heads > 1 ? w.head + 1 : p.c.Hkv;
    w.t0 = p.last > 0 ? max(w.chunk - p.last, 0) : 0;
    const int from = w.first + w.t0, n = w.chunk - w.t0;     // position of the first query that counts, how many
    w.q0 = 0;
    w.q1 = (n + p.tile_tokens - 1) / p.tile_tokens;
    if (p.causal) w.q0 = max(w.key0 - from, 0) / p.tile_tokens;
    if (p.window > 0) {
        const long long last = (long long)w.key0 + CH_TILE - 1 + p.window - 1 - from;      // the last query whose window reaches the tile
        w.q1 = last < 0 ? 0 : (int)min((long long)w.q1, last / p.tile_tokens + 1);
    }
    w.q0 = min(w.q0, w.q1);
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
    weight_start(p, w);

    if (warp < 8) {
        // ---- sums ----
        const int s = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        int step = 0, tile = 0, turn = 0, item = 0;          // products and key tiles so far, own turns, joined tiles
        for (; ok && weight_tile(p, w); w.at += gridDim.x) {
            const int key = w.key0 + row, steps = (w.q1 - w.q0) * (w.g1 - w.g0), first_step = step;
            float acc = 0.f;
            for (int g = w.g0; g < w.g1 && ok; ++g) {
                float part = 0.f;
                for (int q = w.q0; q < w.q1 && ok; ++q, ++step) {
                    if ((step & 1) != s) continue;
                    const int t = w.t0 + q * tt, rows = min(tt, w.chunk - t) * G;      // first token, rows that count
                    const int buf = step % CW_BUFS, cols = (rows + 31) & ~31;
                    const float scale = p.scale_log2 * (KV8 && p.k_scale ? read_global(p.k_scale + g) : 1.f);
                    float* const lse2 = sh.lse2[s][turn & 1];
                    int2* const sees = sh.sees[s][turn & 1];
                    ++turn;
                    const int pos = w.first + t + row / G;
                    const bool counts = row < rows;
                    lse2[row] = counts ? read_global(p.lse + (long long)(w.begin + t + row / G) * p.c.Hq + g * G + row % G) * 1.4426950408889634f : 0.f;
                    sees[row] = counts ? make_int2(p.window > 0 ? max(pos - p.window + 1, 0) : 0, p.causal ? min(pos + 1, w.ctx) : w.ctx) : make_int2(0, 0);
                    asm volatile("bar.sync %0, 128;\n" ::"r"(1 + s) : "memory");
                    ok = bar_wait(smem_u32(&sh.d_full[buf]), (step / CW_BUFS) & 1, gave_up);
                    if (!ok) break;
                    tmem_fence_after();
                    const bool all = rows == cols && (!p.causal || w.key0 + CH_TILE - 1 <= w.first + t) &&
                                     (p.window <= 0 || w.first + t + (rows - 1) / G - p.window < w.key0);
                    for (int c = 0; c < cols; c += 32) {
                        uint32_t x[32];
                        __syncwarp();
                        tmem_ld32(tmem + lanes + buf * CH_TILE + c, x);
                        tmem_wait_ld();
                        tmem_loaded32(x);
                        float sum0 = 0.f, sum1 = 0.f;
                        if (all) {
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const float4 l = *reinterpret_cast<const float4*>(lse2 + c + j);
                                sum0 += fast_exp2(fmaf(__uint_as_float(x[j]), scale, -l.x));
                                sum1 += fast_exp2(fmaf(__uint_as_float(x[j + 1]), scale, -l.y));
                                sum0 += fast_exp2(fmaf(__uint_as_float(x[j + 2]), scale, -l.z));
                                sum1 += fast_exp2(fmaf(__uint_as_float(x[j + 3]), scale, -l.w));
                            }
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                const int2 range = sees[c + j];
                                const float e = fast_exp2(fmaf(__uint_as_float(x[j]), scale, -lse2[c + j]));
                                if (key >= range.x && key < range.y) sum0 += e;
                            }
                        }
                        part += sum0 + sum1;
                    }
                    tmem_fence_before();
                    __syncwarp();
                    if (lane == 0) bar_arrive(smem_u32(&sh.d_empty[buf]));
                }
                // a page id outside the pool: its positions receive nothing
                if (steps > 0 && ((sh.bad_pages[tile % CH_TAGS] >> (row / TILE)) & 1)) part = 0.f;
                if (w.q1 > w.q0) ++tile;
                acc += part;
            }
            if (!ok) break;
            bool writes = steps == 0 ? s == 0 : (first_step & 1) == s;
            if (steps > 1) {
                if (s == 1) sh.sums[item & 1][row] = acc;
                asm volatile("bar.sync 3, 256;\n" ::: "memory");
                if (s == 0) acc += sh.sums[item & 1][row];
                writes = s == 0;
                ++item;
            }
            if (writes && key < w.ctx) {
                float* const to = p.weights + ((long long)w.b * p.heads + w.head) * p.stride + key;
                if (p.decay != 0.f && key < w.first) acc = fmaf(p.decay, read_global(to), acc);
                *to = acc;
            }
        }
    } else if (warp == 8) {
        // ---- products ----
        if (lane == 0) {
            int step = 0, tile = 0;
            for (; ok && weight_tile(p, w); w.at += gridDim.x)
                for (int g = w.g0; g < w.g1 && ok && w.q0 < w.q1; ++g, ++tile) {
                    const int ks = tile % CW_RING;
                    ok = bar_wait(smem_u32(&sh.k_full[ks]), (tile / CW_RING) & 1, gave_up);
                    for (int q = w.q0; q < w.q1 && ok; ++q, ++step) {
                        const int qs = step % QRING, buf = step % CW_BUFS;
                        const int rows = min(tt, w.chunk - w.t0 - q * tt) * G, cols = (rows + 31) & ~31;
                        ok = bar_wait(smem_u32(&sh.q_full[qs]), (step / QRING) & 1, gave_up) &&
                             (step < CW_BUFS || bar_wait(smem_u32(&sh.d_empty[buf]), (step / CW_BUFS - 1) & 1, gave_up));
                        if (!ok) break;
                        tmem_fence_after();
                        const uint32_t a = k_ring + ks * CH_MAT, b = q_ring + qs * CH_MAT, shape = mma_shape(true, cols, false);
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk) {
                            const uint32_t off = (kk >> 2) * CH_HALF + (kk & 3) * 32;
                            mma_ss(tmem + buf * CH_TILE, smem_matrix(a + off, 16), smem_matrix(b + off, 16), shape, kk > 0);
                        }
                        mma_commit(smem_u32(&sh.d_full[buf]));
                        mma_commit(smem_u32(&sh.q_empty[qs]));
                        if (q == w.q1 - 1) mma_commit(smem_u32(&sh.k_empty[ks]));
                    }
                }
        }
    } else if (warp == 9) {
        // ---- copies in ----
        int step = 0, tile = 0;
        for (; ok && weight_tile(p, w); w.at += gridDim.x)
            for (int g = w.g0; g < w.g1 && ok && w.q0 < w.q1; ++g, ++tile) {
                int page = 0;
                unsigned bad = 0;
                if (p.c.paged) {
                    page = p.c.num_pages;                   // (out of range: filled with zeros)
                    const int blk = w.key0 / TILE + (lane & 7);
                    if (blk * TILE < w.ctx) {
                        page = read_global(p.c.page_table + (long long)w.b * p.c.max_pages + blk);
                        if ((unsigned)page >= (unsigned)p.c.num_pages) { page = p.c.num_pages; bad = 1; }
                    }
                    bad = __ballot_sync(0xffffffffu, bad) & 0xffu;
                    if (bad && lane == 0) atomicOr(p.c.status, STATUS_BAD_PAGE);
                }
                const int slot = KV8 ? tile % CH_RAW : tile % CW_RING;
                if constexpr (KV8) { if (tile >= CH_RAW) ok = bar_wait(smem_u32(&sh.raw_empty[slot]), (tile / CH_RAW - 1) & 1, gave_up); }
                else { if (tile >= CW_RING) ok = bar_wait(smem_u32(&sh.k_empty[slot]), (tile / CW_RING - 1) & 1, gave_up); }
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t dst = KV8 ? raw + slot * CH_HALF : k_ring + slot * CH_MAT, bar = smem_u32(KV8 ? &sh.raw_full[slot] : &sh.k_full[slot]);
                if (lane == 0) {
                    sh.bad_pages[tile % CH_TAGS] = bad;
                    bar_expect(bar, KV8 ? CH_HALF : CH_MAT);
                }
                __syncwarp();
                constexpr int HALVES = KV8 ? 1 : 2;
                if (p.c.paged) {
                    if (lane < 8 * HALVES)
                        tma_load4(dst + (lane >> 3) * CH_HALF + (lane & 7) * 2048, &k_map, bar, (lane >> 3) * 64, 0, g * p.head_mul,
                                  page * p.page_mul + (page == p.c.num_pages && !p.page_mul ? 1 : 0));
                } else if (lane < HALVES) {
                    tma_load4(dst + lane * CH_HALF, &k_map, bar, lane * 64, w.key0, g * p.head_mul, w.b * p.batch_mul);
                }
                for (int q = w.q0; q < w.q1 && ok; ++q, ++step) {
                    const int qs = step % QRING;
                    if (step >= QRING) ok = bar_wait(smem_u32(&sh.q_empty[qs]), (step / QRING - 1) & 1, gave_up);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (lane == 0) {
                        bar_expect(smem_u32(&sh.q_full[qs]), 2 * G * tt * 128);
                        for (int h = 0; h < 2; ++h)
                            tma_load3(q_ring + qs * CH_MAT + h * CH_HALF, &q_map, smem_u32(&sh.q_full[qs]), h * 64, g * G, w.begin + w.t0 + q * tt);
                    }
                }
            }
    } else if (KV8) {
        // ---- codes to bf16 ----
        const int l = tid - 320;
        int tile = 0;
        for (; ok && weight_tile(p, w); w.at += gridDim.x)
            for (int g = w.g0; g < w.g1 && ok && w.q0 < w.q1; ++g, ++tile) {
                const int rs = tile % CH_RAW, slot = tile % CW_RING;
                ok = bar_wait(smem_u32(&sh.raw_full[rs]), (tile / CH_RAW) & 1, gave_up) &&
                     (tile < CW_RING || bar_wait(smem_u32(&sh.k_empty[slot]), (tile / CW_RING - 1) & 1, gave_up));
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
    if (sh.gave_up) for (int i = 0; i < 50; ++i) __nanosleep(20000);      // (copies that are still on their way land meanwhile)
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem));
    if (tid == 0 && sh.gave_up) atomicOr(p.c.status, STATUS_WAITED_OUT);
}

}  // namespace tidal
