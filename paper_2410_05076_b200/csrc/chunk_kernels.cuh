// Attention of chunks of new tokens over the cache (chunk_attn_kernel) on the fifth-generation tensor cores: operands come by
// TMA into 128-byte-swizzled shared memory, products accumulate in TMEM, one thread issues them.
#pragma once

#include <cuda.h>

#include <type_traits>

#include "page_kernels.cuh"

namespace tidal {

enum { STATUS_WAITED_OUT = 16 };          // a wait on a copy or a product ran out: results are invalid

// ---- barriers, copies, products ------------------------------------------------------------------------------------
#ifndef TIDAL_WAIT_TRIES
#define TIDAL_WAIT_TRIES (1 << 22)
#endif
constexpr int WAIT_TRIES = TIDAL_WAIT_TRIES;       // each try sleeps for up to a microsecond or so

__device__ __forceinline__ void bar_init(uint32_t bar, int count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(bar) : "memory"); }
__device__ __forceinline__ void bar_expect(uint32_t bar, int bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0;
}
// Waits for the phase of that parity to end; a whole warp together, with one answer for its lanes. False once a wait of this CTA has run out: the warp
// then leaves its loop. APART: the first try stands before the loop of the others, after which the compiler orders what follows differently; each kernel
// takes what it is faster with (attention over 16 bits 7.33 ms with it and 7.40 without, weights of single tokens 215 and 207 us).
template <bool APART>
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (APART && __all_sync(0xffffffffu, bar_try(bar, parity))) return true;
    for (int i = 0; i < WAIT_TRIES; ++i) {
        if (APART && __any_sync(0xffffffffu, *gave_up)) break;
        if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
        if (!APART && __any_sync(0xffffffffu, *gave_up)) break;
    }
    *gave_up = 1;
    return false;
}
// The same without the vote, which costs the attention kernel a tenth of its speed where its products and its softmax wait (4096 tokens after 131072: 7.39
// and 8.12 ms). Lanes may then have different answers, so that no branch that the warp takes together may hang on one: what waits here goes
// on through all its steps, with results that are none.
template <bool APART>
__device__ __forceinline__ bool bar_pass(uint32_t bar, uint32_t parity, volatile int* gave_up) {
    if (APART && bar_try(bar, parity)) return true;
    for (int i = 0; i < WAIT_TRIES; ++i) {
        if (APART && *gave_up) break;
        if (bar_try(bar, parity)) return true;
        if (!APART && *gave_up) break;
    }
    *gave_up = 1;
    return false;
}
// A millisecond after a wait has run out: copies and products that are still on their way land before the CTA gives its memory back.
__device__ __noinline__ void let_land() {
    unsigned long long t0, t;
    asm volatile("mov.u64 %0, %%globaltimer;\n" : "=l"(t0));
    for (int i = 0; i < 100000; ++i) {
        __nanosleep(10000);
        asm volatile("mov.u64 %0, %%globaltimer;\n" : "=l"(t));
        if (t - t0 >= 1000000) return;
    }
}
__device__ __forceinline__ void tma_load4(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];\n"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3) : "memory");
}
__device__ __forceinline__ void tma_load3(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];\n"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
// Matrix in shared memory, 128-byte swizzle, 8-row groups 1024 bytes apart. `block`: bytes between blocks of 64 elements along
// the contiguous direction, used where that direction is not the contracted one.
__device__ __forceinline__ uint64_t smem_matrix(uint32_t addr, uint32_t block) {
    return (uint64_t)((addr >> 4) & 0x3fff) | ((uint64_t)(block >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// Instruction descriptor: 128 rows, N columns, fp32 accumulator, both operands bf16 or fp16; cols_major: the second operand's rows
// (N) are its contiguous direction.
__device__ __forceinline__ uint32_t mma_shape(bool bf16, int n, bool cols_major) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (cols_major ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n"
                 ::"r"(d), "l"(a), "l"(b), "r"(shape), "r"((int)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t shape, bool add) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.b32 p, %4, 0;\ntcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}\n"
                 ::"r"(d), "r"(a), "l"(b), "r"(shape), "r"((int)add) : "memory");
}
// The barrier completes when all products issued so far by this thread have.
__device__ __forceinline__ void mma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(bar) : "memory");
}
// One lane of a warp whose lanes are together, the same one every time.
__device__ __forceinline__ bool elected() {
    uint32_t e;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}\n" : "=r"(e));
    return e != 0;
}
// A value that all lanes of a warp share, as one that the compiler knows they do: descriptors and addresses of products live in uniform registers,
// and moving them there one by one costs more than a product takes.
__device__ __forceinline__ int uniform(int x) { return __shfl_sync(0xffffffffu, x, 0); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void smem_to_async() { asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory"); }

#define TMEM_REGS32(r, o) r(o + 0), r(o + 1), r(o + 2), r(o + 3), r(o + 4), r(o + 5), r(o + 6), r(o + 7), r(o + 8), r(o + 9), r(o + 10), r(o + 11), \
    r(o + 12), r(o + 13), r(o + 14), r(o + 15), r(o + 16), r(o + 17), r(o + 18), r(o + 19), r(o + 20), r(o + 21), r(o + 22), r(o + 23), r(o + 24), \
    r(o + 25), r(o + 26), r(o + 27), r(o + 28), r(o + 29), r(o + 30), r(o + 31)

// 32 columns of this thread's lane (row) of TMEM.
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* x) {
#define R(i) "=r"(x[i])
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
                 "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
                 : TMEM_REGS32(R, 0) : "r"(addr) : "memory");
#undef R
}
__device__ __forceinline__ void tmem_st32(uint32_t addr, const uint32_t* x) {
#define R(i) "r"(x[i])
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
                 "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};\n"
                 :: TMEM_REGS32(R, 0), "r"(addr) : "memory");
#undef R
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* x) {
#define R(i) "r"(x[i])
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};\n"
                 :: R(0), R(1), R(2), R(3), R(4), R(5), R(6), R(7), R(8), R(9), R(10), R(11), R(12), R(13), R(14), R(15), "r"(addr) : "memory");
#undef R
}
// (the loads above are done: their registers may be read)
__device__ __forceinline__ void tmem_loaded32(uint32_t* x) {
#define R(i) "+r"(x[i])
    asm volatile("" : TMEM_REGS32(R, 0));
#undef R
}

__device__ __forceinline__ float max3(float a, float b, float c) {         // not-a-number if one is
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

// ---- attention -------------------------------------------------------------------------------------------------------
// A CTA takes up to 256 rows (token, query head of a KV head's group), two streams of 128, over a range of the cache in tiles of 128
// positions. Per tile and stream: S = Q K^T into TMEM, a softmax warpgroup turns it into weights in place (a row per
// thread; running maximum in base 2, raised only when it is passed by 2^8, so that the output is hardly ever rescaled), and
// O += P V. One stream's softmax runs beside the other's products. Where a sequence has no more than one stream's rows, both streams
// take them, every other tile each. Long axes are cut over the CTAs of a cluster (and the two streams), whose partial results are joined
// through shared memory.
//
// 4096 tokens at the end of 16384: 814 us, 1180 TFLOP/s, tensor pipe at 65 % (over E4M3 898 us, 57 %); at the end of 131072 under the power limit 7.0 to 7.9 ms. Bound by
// what lies between products: a stream's scores wait for its weights, the exponential unit (2048 clocks for a pair of tiles, as long as their
// products) and the issuing warp's turns beside the softmax warps. One warp issues for both streams in turn, which keeps one's softmax beside the
// other's products; a warp for each lets them fall into step (1090 us).
//
// Rounding: weights enter the second product as bf16 (fp16 over an 8-bit cache, whose codes are widened exactly); sums of weights, maxima and
// outputs are fp32.
struct ChunkParams {
    BlockCache c;
    int page_mul, batch_mul, head_mul;                      // 0 where a coordinate has no stride
    const __nv_bfloat16* q;
    long long q_stride;
    const int* q_offsets;                                   // [batch + 1]
    int num_tokens, tile_tokens;                            // tokens per stream (128 / G)
    int q_tiles;                                            // bound of the CTA tiles of all sequences together
    int causal, window;
    float scale_log2;
    const float* k_scale;
    const float* v_scale;
    float* out;
    int out_bf16;
    float* lse;
};

constexpr int CH_TILE = 128;                                // positions per tile, rows per stream
constexpr int CH_HALF = CH_TILE * 128;                      // bytes of 64 channels of a tile's rows, 16 bits each
constexpr int CH_MAT = 2 * CH_HALF;
constexpr int CH_TAGS = 16, CH_MAX_TILES = 2048;            // tiles of the longest context
constexpr int CH_THREADS = 384, CH_THREADS8 = 512;
constexpr int CH_RING = 5, CH_RING8 = 4;                       // operand slots: keys and values of a tile take one each
constexpr int CH_MOST = 6;                                  // of eight products of weights and values, those that begin before all weights are there
constexpr int CH_RAW = 2;                                   // 8-bit caches: tiles of codes in flight
template <bool KV8> constexpr size_t ch_smem() { return 1024 + 2 * CH_MAT + (size_t)(KV8 ? CH_RING8 : CH_RING) * CH_MAT + (KV8 ? CH_RAW * CH_HALF : 0); }

struct ChunkShared {
    unsigned long long q_full, full[5], empty[5], raw_full[2], raw_empty[2], s_full[2], p_most[2], p_full[2], o_done[2];
    uint32_t tmem;
    int gave_up, seq, tile;
    int any_odd;                                            // a tile that not all rows of a stream see whole has values that are not finite:
    unsigned odd[CH_MAX_TILES / 32];                        // bit i: the CTA's i-th
    unsigned bad_pages[CH_TAGS];                            // per tile, bit i: its i-th page is not one
};
// Partial results take the operands' place: 2 x 128 rows of 128 outputs, then their maxima and sums.
constexpr uint32_t CH_PART_MAX = 2 * CH_TILE * HEAD_DIM * 4, CH_PART_SUM = CH_PART_MAX + 2 * CH_TILE * 4;

// What a CTA works on; every warp works it out for itself.
struct ChunkWork {
    int b, g, t0, new_tokens, first, ctx, q_row;            // sequence, KV head, first token, tokens of the chunk, its first position, length
    int tile0, tiles;                                       // this CTA's tiles of positions
    int twin;                                               // both streams take the same rows, every other tile each
    int stream_tiles[2];
    // the tile that a stream's i-th step is about
    __device__ __forceinline__ int at(int s, int i) const { return twin ? 2 * i + s : i; }
};

__device__ __forceinline__ bool chunk_work(const ChunkParams& p, const ChunkShared& sh, int rank, int ranks, int g, ChunkWork& w) {
    const int tt = p.tile_tokens;
    w.b = sh.seq; w.g = g;
    const int begin = max(min(read_global(p.q_offsets + w.b), p.num_tokens), 0);
    const int end = max(min(read_global(p.q_offsets + w.b + 1), p.num_tokens), begin);
    w.new_tokens = end - begin;
    w.ctx = cached_len(p.c, w.b);
    w.first = w.ctx - w.new_tokens;
    w.t0 = sh.tile * 2 * tt;
    w.q_row = begin + w.t0;
    const int rows = min(2 * tt, w.new_tokens - w.t0);      // tokens here
    // positions that some row of each stream sees
    const int first_pos = w.first + w.t0;
    const int lo = p.window > 0 ? max(first_pos - p.window + 1, 0) : 0;
    int hi[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int last = first_pos + min(rows, (s + 1) * tt) - 1;
        hi[s] = p.causal ? min(last + 1, w.ctx) : w.ctx;
    }
    w.twin = rows <= tt;
    const int from = lo / CH_TILE;
    const int all[2] = {max((hi[0] + CH_TILE - 1) / CH_TILE - from, 0), max((hi[1] + CH_TILE - 1) / CH_TILE - from, 0)};
    const int per = (all[1] + ranks - 1) / ranks, mine = min(rank * per, all[1]);
    w.tile0 = from + mine;
    w.tiles = min(per, all[1] - mine);
    if (w.twin) {
        w.stream_tiles[0] = (w.tiles + 1) / 2;
        w.stream_tiles[1] = w.tiles / 2;
    } else {
        w.stream_tiles[0] = max(min(all[0] - mine, w.tiles), 0);
        w.stream_tiles[1] = w.tiles;
    }
    return w.tiles > 0;
}

// One CTA tile of a sequence: which of all of them it is. The last tokens of a sequence, which see most, first; up to 32 sequences by their
// lengths, the longest first, so that no long tile begins when the others are nearly done (8 sequences of 8192 to 65536 with chunks of 1000 down
// to 1, 8 bits: 1.93 -> 1.55 ms); more of them in order.
__device__ __forceinline__ void chunk_find(const ChunkParams& p, int want, int lane, int& seq, int& tile, bool& damaged) {
    const int per = 2 * p.tile_tokens;
    int before = 0;
    seq = -1; tile = 0; damaged = false;
    for (int b0 = 0; b0 < p.c.batch; b0 += 32) {
        int b = b0 + lane, n = 0, len = -1;
        bool bad = false;
        if (b < p.c.batch) {
            const int x = read_global(p.q_offsets + b), y = read_global(p.q_offsets + b + 1);
            const int lo = max(min(x, p.num_tokens), 0), hi = max(min(y, p.num_tokens), lo);
            bad = lo != x || hi != y;
            n = (hi - lo + per - 1) / per;
            len = cached_len(p.c, b);
        }
        damaged |= __any_sync(0xffffffffu, bad);
        if (p.c.batch > 1 && p.c.batch <= 32) {
            int place = 0;                                  // lanes in order of their lengths
#pragma unroll 1
            for (int i = 0; i < p.c.batch; ++i) {
                const int other = __shfl_sync(0xffffffffu, len, i);
                place += other > len || (other == len && i < lane);
            }
            int from = lane;
#pragma unroll 1
            for (int i = 0; i < p.c.batch; ++i) from = __shfl_sync(0xffffffffu, place, i) == lane ? i : from;
            b = from;
            n = __shfl_sync(0xffffffffu, n, from);
        }
        int x = n;
#pragma unroll
        for (int sft = 1; sft < 32; sft <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, sft); if (lane >= sft) x += y; }
        const unsigned hit = __ballot_sync(0xffffffffu, before + x > want);
        if (hit && seq < 0) {
            const int src = __ffs(hit) - 1;
            const int here = __shfl_sync(0xffffffffu, x, src), size = __shfl_sync(0xffffffffu, n, src);
            seq = __shfl_sync(0xffffffffu, b, src);
            tile = size - 1 - (want - (before + here - size));
            if (want > 0) return;                           // (the first CTAs look at all offsets)
        }
        before += __shfl_sync(0xffffffffu, x, 31);
    }
}

// Eight 16-bit numbers with zeros for those that are not finite; whether there were any.
template <bool HALF>
__device__ __forceinline__ bool drop_odd(uint32_t (&x)[4]) {
    constexpr uint32_t EXP = HALF ? 0x7c007c00u : 0x7f807f80u, ONE = HALF ? 0x04000400u : 0x00800080u;
    uint32_t any = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t full = ((x[j] & EXP) + ONE) & 0x80008000u;          // a full exponent carries
        any |= full;
        x[j] &= ~((full >> 15) * 0xffffu);
    }
    return any != 0;
}

// What the values that were left out of a stream's products (see the kernel) add to its rows, a quarter of them per warp: infinities and not-a-numbers to the
// channels of the rows that see their position, and that have a weight at all (`lives`), whatever is there already. Four channels per lane; into the partial results
// where they are joined.
template <bool KV8>
__device__ __noinline__ void chunk_odd_values(const ChunkParams& p, const ChunkShared& sh, uint32_t base, int rank, int ranks, int g, int s, int quarter, int lane, unsigned lives) {
    ChunkWork w;
    chunk_work(p, sh, rank, ranks, g, w);
    const bool joined = ranks > 1 || w.twin;
    const int G = p.c.G, tt = p.tile_tokens;
    for (int tile = 0; tile < w.tiles; ++tile) {
        const unsigned word = sh.odd[tile >> 5];
        if (!word) { tile |= 31; continue; }
        if (!((word >> (tile & 31)) & 1) || (w.twin && (tile & 1) != s)) continue;
        const int key0 = (w.tile0 + tile) * CH_TILE;
        for (int key = key0; key < min(key0 + CH_TILE, w.ctx); ++key) {
            long long row = (long long)w.b * p.c.stride_b + key * p.c.stride_pos;
            if (p.c.paged) {
                const int page = read_global(p.c.page_table + (long long)w.b * p.c.max_pages + key / TILE);
                if ((unsigned)page >= (unsigned)p.c.num_pages) continue;
                row = page * p.c.stride_page + key % TILE * p.c.stride_pos;
            }
            row += w.g * p.c.stride_head + lane * 4;
            uint32_t a, b;
            if constexpr (KV8) {
                e4m3x4_to_f16x2x2(read_global(reinterpret_cast<const uint32_t*>(p.c.v + row)), a, b);
                a = f16x2_to_bf16x2(a);
                b = f16x2_to_bf16x2(b);
            } else {
                const uint2 y = read_global(reinterpret_cast<const uint2*>(p.c.v + row * 2));
                a = y.x; b = y.y;
            }
            float v[4] = {__uint_as_float(a << 16), __uint_as_float(a & 0xffff0000u), __uint_as_float(b << 16), __uint_as_float(b & 0xffff0000u)};
            bool any = false;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (isfinite(v[c])) v[c] = 0.f;
                else any = true;
            }
            if (!__any_sync(0xffffffffu, any)) continue;
            for (int i = 0; i < 32; ++i) {
                const int r = quarter * 32 + i, token = w.t0 + (w.twin ? 0 : s * tt) + r / G, head = w.g * G + r % G, pos = w.first + token;
                if (!any || !((lives >> i) & 1) || key >= (p.causal ? min(pos + 1, w.ctx) : w.ctx) || (p.window > 0 && key <= pos - p.window)) continue;
                const long long at = ((long long)(w.q_row + token - w.t0) * p.c.Hq + head) * HEAD_DIM + lane * 4;
                if (joined) {
                    const uint32_t to = base + ((s * CH_TILE + r) * 32 + (lane ^ i)) * 16;
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float x;
                        asm volatile("ld.shared.f32 %0, [%1];\n" : "=f"(x) : "r"(to + 4 * c) : "memory");
                        asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(to + 4 * c), "f"(x + v[c]) : "memory");
                    }
                } else if (p.out_bf16) {
                    uint2* const to = reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at);
                    const uint2 x = read_global(to);
                    *to = make_uint2(pack_bf16(__uint_as_float(x.x << 16) + v[0], __uint_as_float(x.x & 0xffff0000u) + v[1]),
                                     pack_bf16(__uint_as_float(x.y << 16) + v[2], __uint_as_float(x.y & 0xffff0000u) + v[3]));
                } else {
                    float4* const to = reinterpret_cast<float4*>(p.out + at);
                    const float4 x = read_global(to);
                    *to = make_float4(x.x + v[0], x.y + v[1], x.z + v[2], x.w + v[3]);
                }
            }
        }
    }
}

template <bool KV8>
__global__ void __launch_bounds__(KV8 ? CH_THREADS8 : CH_THREADS, 1)
chunk_attn_kernel(const __grid_constant__ ChunkParams p, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                  const __grid_constant__ CUtensorMap v_map) {
    extern __shared__ unsigned char ch_raw_smem[];
    __shared__ ChunkShared sh;
    constexpr int RING = KV8 ? CH_RING8 : CH_RING;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t base = (smem_u32(ch_raw_smem) + 1023u) & ~1023u;
    const uint32_t q_smem = base, ring = base + 2 * CH_MAT, raw = ring + RING * CH_MAT;
    int ranks, rank;
    asm volatile("mov.u32 %0, %%cluster_nctarank;\n" : "=r"(ranks));
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    const int unit = (int)blockIdx.x / ranks, g = unit % p.c.Hkv;

    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&sh.tmem)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n");
    }
    if (tid == 32) {
        bar_init(smem_u32(&sh.q_full), 1);
        for (int i = 0; i < RING; ++i) { bar_init(smem_u32(&sh.full[i]), KV8 ? 4 : 1); bar_init(smem_u32(&sh.empty[i]), 1); }
        for (int i = 0; i < 2; ++i) {
            bar_init(smem_u32(&sh.raw_full[i]), 1); bar_init(smem_u32(&sh.raw_empty[i]), 4);
            bar_init(smem_u32(&sh.s_full[i]), 1); bar_init(smem_u32(&sh.p_most[i]), 4); bar_init(smem_u32(&sh.p_full[i]), 4);
            bar_init(smem_u32(&sh.o_done[i]), 1);
        }
        sh.gave_up = sh.any_odd = 0;
        for (unsigned& x : sh.odd) x = 0;
        asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    }
    pdl_wait();
    pdl_trigger();
    if (warp == 2) {
        int seq, tile;
        bool damaged;
        chunk_find(p, unit / p.c.Hkv, lane, seq, tile, damaged);
        if (lane == 0) {
            sh.seq = seq; sh.tile = tile;
            if (damaged) atomicOr(p.c.status, STATUS_BAD_INDEX);
        }
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = sh.tmem;
    if (sh.seq < 0) {                                       // (the whole cluster)
        if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem));
        return;
    }
    ChunkWork w;
    const bool busy = chunk_work(p, sh, rank, ranks, g, w);
    const bool joined = ranks > 1 || w.twin;                // (the same for the cluster)
    volatile int* const gave_up = &sh.gave_up;
    const int G = p.c.G, tt = p.tile_tokens;

    // Registers: the softmax warpgroups hold a row of scores each, the others need few. The shares add up to what the launch has.
    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;\n" ::"n"(KV8 ? 208 : 216));
        // ---- softmax ----
        const int s = warp >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t S = tmem + lanes + s * CH_TILE, O = tmem + lanes + 256 + s * CH_TILE;
        const int token = w.t0 + (w.twin ? 0 : s * tt) + row / G, head = w.g * G + row % G;
        const bool valid = row < tt * G && token < w.new_tokens;
        const int pos = w.first + token;
        const int hi = p.causal ? min(pos + 1, w.ctx) : w.ctx, lo = p.window > 0 ? max(pos - p.window + 1, 0) : 0;
        const int s_first = w.first + w.t0 + (w.twin ? 0 : s * tt), s_last = w.first + min(w.t0 + (w.twin ? 0 : s * tt) + tt, w.new_tokens) - 1;
        const float scale = p.scale_log2 * (KV8 && p.k_scale ? read_global(p.k_scale + w.g) : 1.f);
        const int n = w.stream_tiles[s];
        float m = -INFINITY, l = 0.f;
        if constexpr (KV8) {                                // queries as fp16
            if (busy) {
                bar_pass<true>(smem_u32(&sh.q_full), 0, gave_up);
                for (int i = tid & 127; i < CH_MAT / 16; i += 128) {
                    const uint32_t a = q_smem + s * CH_MAT + i * 16;
                    uint32_t x[4];
                    lds128(a, x);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = bf16x2_to_f16x2(x[j]);
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(a), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
                }
                smem_to_async();
                __syncwarp();
                if (lane == 0) bar_arrive(smem_u32(&sh.p_full[s]));
            }
        }
        for (int i = 0; i < n; ++i) {
            const int tile = w.at(s, i), key0 = (w.tile0 + tile) * CH_TILE;
            bar_pass<true>(smem_u32(&sh.s_full[s]), i & 1, gave_up);
            tmem_fence_after();
            uint32_t x[CH_TILE];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(S + c * 32, x + c * 32);
            tmem_wait_ld();
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_loaded32(x + c * 32);
            const unsigned bad = sh.bad_pages[tile % CH_TAGS];
            const bool ragged = key0 + CH_TILE > w.ctx;
            const bool partly = (p.causal && key0 + CH_TILE - 1 > s_first) || (p.window > 0 && key0 <= s_last - p.window);
            if (ragged || partly || bad) {
#pragma unroll
                for (int j = 0; j < CH_TILE; ++j) {
                    const bool seen = key0 + j >= lo && key0 + j < hi && !((bad >> (j / TILE)) & 1);
                    x[j] = seen ? x[j] : 0xff800000u;
                }
                if (ragged) {
                    // what lies behind the sequence may be anything, and zero times infinity is not zero
                    const int item = 2 * tile + 1, slot = item % RING;
                    bar_pass<true>(smem_u32(&sh.full[slot]), (item / RING) & 1, gave_up);
                    const int from = max(w.ctx - key0, 0);
                    for (int k = from * 8 + (tid & 127); k < CH_TILE * 8; k += 128)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};\n" ::"r"(ring + slot * CH_MAT + h * CH_HALF + k * 16), "r"(0) : "memory");
                    smem_to_async();
                }
            }
            if (i == 0) {
                float top = -INFINITY;
#pragma unroll
                for (int j = 0; j < CH_TILE; j += 2) top = max3(top, __uint_as_float(x[j]), __uint_as_float(x[j + 1]));
                m = top == top ? top : -INFINITY;
            }
            if (partly) {
                // A weight of zero times a value that is not finite would spoil rows that do not see it: such values are left out of the product and
                // added at the end to the rows that do. (Every stream writes back what it has looked at, since its own product has to find it so; the other
                // stream, whose rows may all see the tile, meets such a value or zero, and is given it at the end in both cases.)
                const int item = 2 * tile + 1, slot = item % RING;
                bar_pass<true>(smem_u32(&sh.full[slot]), (item / RING) & 1, gave_up);
                bool odd = false;
                for (int k = tid & 127; k < min(w.ctx - key0, CH_TILE) * 8; k += 128)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const uint32_t at = ring + slot * CH_MAT + h * CH_HALF + k * 16;
                        uint32_t v[4];
                        lds128(at, v);
                        odd |= drop_odd<KV8>(v);
                        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
                    }
                smem_to_async();
                if (odd) {
                    atomicOr(&sh.odd[tile >> 5], 1u << (tile & 31));
                    sh.any_odd = 1;
                }
            }
            // Weights by the maximum so far, while this tile's own is looked for: it is raised, and the weights are worked out again, only
            // where that leaves one above 2^8.
            f32pair sum0, sum1;
            float top;
            auto weights = [&](auto) -> bool {
                const float shift = m == -INFINITY ? 0.f : -m * scale;
                const f32pair scale2 = pair2(scale, scale), shift2 = pair2(shift, shift);
                sum0 = sum1 = pair2(0.f, 0.f);
                top = -INFINITY;
                float other = -INFINITY;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t y[16];
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const int at = c * 32 + 2 * j;
                        if (c < 2) {
                            top = max3(top, __uint_as_float(x[2 * at]), __uint_as_float(x[2 * at + 1]));
                            other = max3(other, __uint_as_float(x[2 * at + 2]), __uint_as_float(x[2 * at + 3]));
                        }
                        const f32pair t = fma2(pair2(__uint_as_float(x[at]), __uint_as_float(x[at + 1])), scale2, shift2);
                        const f32pair e = pair2(fast_exp2(half2(t, 0)), fast_exp2(half2(t, 1)));
                        if (j & 1) sum1 = add2(sum1, e); else sum0 = add2(sum0, e);
                        y[j] = KV8 ? pack_f16(half2(e, 0), half2(e, 1)) : pack_bf16(half2(e, 0), half2(e, 1));
                    }
                    tmem_st16(S + c * 16, y);
                    if (c == CH_MOST / 2 - 1) {                           // the products with three quarters of the positions may begin
                        top = max3(top, other, other);
                        if (__any_sync(0xffffffffu, valid && (top - m) * scale > 8.f)) return false;      // (rows that are none must not change others' rounding)
                        tmem_wait_st();
                        tmem_fence_before();
                        __syncwarp();
                        if (lane == 0) bar_arrive(smem_u32(&sh.p_most[s]));
                    }
                }
                return true;
            };
            // (two copies of the same code, one of them for whole tiles alone: the compiler schedules that one better when the masked tiles' paths do
            // not lead into it: 817 against 844 us, over E4M3 975 against 1074, when that was tried)
            const bool whole = !(ragged || partly || bad);
            while (!(whole ? weights(std::true_type()) : weights(std::false_type()))) {
                const float up = fmaxf(m, top), f = m == up ? 1.f : fast_exp2((m - up) * scale);
                l *= f;
                m = up;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t y[32];
                    tmem_ld32(O + c * 32, y);
                    tmem_wait_ld();
                    tmem_loaded32(y);
#pragma unroll
                    for (int j = 0; j < 32; ++j) y[j] = __float_as_uint(__uint_as_float(y[j]) * f);
                    tmem_st32(O + c * 32, y);
                }
            }
            sum0 = add2(sum0, sum1);
            l += half2(sum0, 0) + half2(sum0, 1);
            if (!(top == top)) l = top;                     // (the row's result is not a number)
            tmem_wait_st();
            tmem_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(smem_u32(&sh.p_full[s]));
        }
        // ---- results ----
        if (n > 0) bar_pass<true>(smem_u32(&sh.o_done[s]), 0, gave_up);
        tmem_fence_after();
        const float vs = KV8 && p.v_scale ? read_global(p.v_scale + w.g) : 1.f;
        if (joined && w.stream_tiles[1 - s] > 0) bar_pass<true>(smem_u32(&sh.o_done[1 - s]), 0, gave_up);    // (partial results take the operands' place)
        if (!joined) {
            const bool some = l != 0.f;                     // (a sum that is not a number is some)
            const float inv = some ? vs / l : 0.f;
            const long long at = ((long long)(w.q_row + token - w.t0) * p.c.Hq + head);
            if (valid && p.lse) p.lse[at] = some ? (m * scale + log2f(l)) * 0.6931471805599453f : -INFINITY;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t y[32];
                if (n > 0) {
                    __syncwarp();
                    tmem_ld32(O + c * 32, y);
                    tmem_wait_ld();
                    tmem_loaded32(y);
                }
                float z[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) z[j] = some ? __uint_as_float(y[j]) * inv : 0.f;
                if (valid && p.out_bf16) {
                    uint4* to = reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at * HEAD_DIM + c * 32);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        to[j] = make_uint4(pack_bf16(z[8 * j], z[8 * j + 1]), pack_bf16(z[8 * j + 2], z[8 * j + 3]), pack_bf16(z[8 * j + 4], z[8 * j + 5]),
                                           pack_bf16(z[8 * j + 6], z[8 * j + 7]));
                } else if (valid) {
                    float4* to = reinterpret_cast<float4*>(p.out + at * HEAD_DIM + c * 32);
#pragma unroll
                    for (int j = 0; j < 8; ++j) to[j] = make_float4(z[4 * j], z[4 * j + 1], z[4 * j + 2], z[4 * j + 3]);
                }
            }
        } else {
            // partial results to shared memory
            asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(base + CH_PART_MAX + (s * CH_TILE + row) * 4), "f"(m == -INFINITY ? m : m * scale) : "memory");
            asm volatile("st.shared.f32 [%0], %1;\n" ::"r"(base + CH_PART_SUM + (s * CH_TILE + row) * 4), "f"(l) : "memory");
            if (n > 0 && __any_sync(0xffffffffu, valid)) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t y[32];
                    __syncwarp();
                    tmem_ld32(O + c * 32, y);
                    tmem_wait_ld();
                    tmem_loaded32(y);
                    if (valid)
#pragma unroll
                        for (int j = 0; j < 8; ++j)
                            asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(base + ((s * CH_TILE + row) * 32 + ((c * 8 + j) ^ (row & 31))) * 16),
                                         "r"(y[4 * j]), "r"(y[4 * j + 1]), "r"(y[4 * j + 2]), "r"(y[4 * j + 3]) : "memory");
                }
            }
        }
        const unsigned lives = __ballot_sync(0xffffffffu, valid && l != 0.f);
        asm volatile("bar.sync 1, 256;\n" ::: "memory");    // both streams' results stand, and what they have left out is known
        if (*(volatile int*)&sh.any_odd) chunk_odd_values<KV8>(p, sh, base, rank, ranks, g, s, warp & 3, lane, lives);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;\n" ::"n"(KV8 ? 48 : 72));
    }
    if (warp == 8) {
        // ---- products: the whole warp walks, one lane issues (nothing more once a wait of its own has run out) ----
        if (busy) {
            const uint32_t first = mma_shape(!KV8, CH_TILE, false), second = mma_shape(!KV8, HEAD_DIM, true);
            const uint32_t acc = uniform(tmem);
            const int twin = uniform(w.twin), n0 = uniform(w.stream_tiles[0]), n1 = uniform(w.stream_tiles[1]);
            // Few instructions between products: every one of them waits its turn beside the softmax warps', and the unit's own queue
            // is two or three products deep.
            const uint32_t s_full = smem_u32(sh.s_full), p_most = smem_u32(sh.p_most), p_full = smem_u32(sh.p_full), o_done = smem_u32(sh.o_done), full = smem_u32(sh.full), empty = smem_u32(sh.empty);
            const uint64_t q = smem_matrix(q_smem, 16);
            auto scores = [&](int s, uint64_t a, int slot) {
                const uint64_t k = smem_matrix(ring + slot * CH_MAT, 16);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    const uint32_t off = ((kk >> 2) * CH_HALF + (kk & 3) * 32) >> 4;
                    mma_ss(acc + s * CH_TILE, a + off, k + off, first, kk > 0);
                }
                mma_commit(s_full + 8 * s);
            };
            // (positions 16 k0 .. 16 k1 - 1 of the tile)
            auto values = [&](int s, int slot, bool add, int k0, int k1) {
                const uint64_t v = smem_matrix(ring + slot * CH_MAT, CH_HALF);
#pragma unroll
                for (int kk = k0; kk < k1; ++kk)
                    mma_ts(acc + 256 + s * CH_TILE, acc + s * CH_TILE + kk * 8, v + (kk * 2048 >> 4), second, add || kk > 0);
            };
            bool ok = bar_pass<!KV8>(smem_u32(&sh.q_full), 0, gave_up);
            if (KV8) for (int s = 0; s < 2; ++s) ok = bar_pass<!KV8>(p_full + 8 * s, 0, gave_up) && ok;
            int slot = 0, parity = 0;                       // of the next ring item to be looked for
            auto next = [&]() {                             // waits for it; its slot
                ok = bar_pass<!KV8>(full + 8 * slot, parity, gave_up) && ok;
                const int at = slot;
                if (++slot == RING) { slot = 0; parity ^= 1; }
                return at;
            };
            int most = 0, turn = KV8;                                 // parity of the weights to come
            if (!twin) {
                int k = next();
                tmem_fence_after();
                if (elected() && ok) {
                    if (n0 > 0) scores(0, q, k);
                    scores(1, q + (CH_MAT >> 4), k);
                    mma_commit(empty + 8 * k);
                }
                __syncwarp();
                int v = next();
                if (n1 > 1) k = next();
                for (int i = 0; i < n1; ++i, turn ^= 1, most ^= 1) {
                    if (i < n0) {
                        ok = bar_pass<!KV8>(p_most, most, gave_up) && ok;
                        tmem_fence_after();
                        if (elected() && ok) values(0, v, i > 0, 0, CH_MOST);
                        __syncwarp();
                        ok = bar_pass<!KV8>(p_full, turn, gave_up) && ok;
                        tmem_fence_after();
                        if (elected() && ok) {
                            values(0, v, true, CH_MOST, 8);
                            if (i + 1 < n0) scores(0, q, k);
                            else mma_commit(o_done);
                        }
                        __syncwarp();
                    }
                    ok = bar_pass<!KV8>(p_most + 8, most, gave_up) && ok;
                    tmem_fence_after();
                    if (elected() && ok) values(1, v, i > 0, 0, CH_MOST);
                    __syncwarp();
                    ok = bar_pass<!KV8>(p_full + 8, turn, gave_up) && ok;
                    tmem_fence_after();
                    if (elected() && ok) {
                        values(1, v, true, CH_MOST, 8);
                        mma_commit(empty + 8 * v);
                        if (i + 1 < n1) {
                            scores(1, q + (CH_MAT >> 4), k);
                            mma_commit(empty + 8 * k);
                        } else {
                            mma_commit(o_done + 8);
                        }
                    }
                    __syncwarp();
                    if (i + 1 < n1) {
                        v = next();
                        if (i + 2 < n1) k = next();
                    }
                }
            } else {
                int vs = 1, vp = 0, ks = 0, kp = 0;         // slots and parities of the values of tile t and of the keys of tile t + 2
                auto on = [&](int& at, int& par) { at += 2; if (at >= RING) { at -= RING; par ^= 1; } };
                const int tiles = n0 + n1;
                auto keys = [&](int s) {
                    ok = bar_pass<!KV8>(full + 8 * ks, kp, gave_up) && ok;
                    tmem_fence_after();
                    if (elected() && ok) {
                        scores(s, q, ks);
                        mma_commit(empty + 8 * ks);
                    }
                    __syncwarp();
                    on(ks, kp);
                };
                for (int t = 0; t < min(tiles, 2); ++t) keys(t);
                for (int t = 0; t < tiles; ++t) {
                    const int s = t & 1;
                    ok = bar_pass<!KV8>(full + 8 * vs, vp, gave_up) && ok;
                    ok = bar_pass<!KV8>(p_full + 8 * s, turn, gave_up) && ok;
                    tmem_fence_after();
                    if (elected() && ok) {
                        values(s, vs, t > 1, 0, 8);
                        mma_commit(empty + 8 * vs);
                        if (t + 2 >= tiles) mma_commit(o_done + 8 * s);
                    }
                    __syncwarp();
                    on(vs, vp);
                    if (t + 2 < tiles) keys(s);
                    turn ^= s;
                }
            }
        }
    } else if (warp == 9 && busy) {
        // ---- copies in ----
        if (lane == 0) {
            const int bytes = 2 * G * tt * 128;
            bar_expect(smem_u32(&sh.q_full), w.twin ? bytes : 2 * bytes);
            for (int s = 0; s < (w.twin ? 1 : 2); ++s)
                for (int h = 0; h < 2; ++h)
                    tma_load3(q_smem + s * CH_MAT + h * CH_HALF, &q_map, smem_u32(&sh.q_full), h * 64, w.g * G, w.q_row + s * tt);
        }
        const int hcoord = w.g * p.head_mul, lo = p.window > 0 ? max(w.first + w.t0 - p.window + 1, 0) : 0;     // (pages before the first row's window are nobody's)
        for (int tile = 0; tile < w.tiles; ++tile) {
            const int key0 = (w.tile0 + tile) * CH_TILE;
            int page = 0;
            unsigned bad = 0;
            if (p.c.paged) {
                page = p.c.num_pages;                       // (out of range: filled with zeros)
                const int blk = key0 / TILE + (lane & 7);
                if (blk * TILE < w.ctx && blk * TILE + TILE > lo) {
                    page = read_global(p.c.page_table + (long long)w.b * p.c.max_pages + blk);
                    if ((unsigned)page >= (unsigned)p.c.num_pages) { page = p.c.num_pages; bad = 1; }
                }
                bad = __ballot_sync(0xffffffffu, bad) & 0xffu;
                if (bad && lane == 0) atomicOr(p.c.status, STATUS_BAD_PAGE);
            }
            if (lane == 0) sh.bad_pages[tile % CH_TAGS] = bad;
            bool ok = true;
            for (int kv = 0; kv < 2 && ok; ++kv) {
                const int item = 2 * tile + kv;
                const CUtensorMap* map = kv ? &v_map : &k_map;
                uint32_t dst, bar;
                if constexpr (KV8) {
                    const int slot = item % CH_RAW;
                    if (item >= CH_RAW) ok = bar_wait<!KV8>(smem_u32(&sh.raw_empty[slot]), (item / CH_RAW - 1) & 1, gave_up);
                    dst = raw + slot * CH_HALF; bar = smem_u32(&sh.raw_full[slot]);
                } else {
                    const int slot = item % RING;
                    if (item >= RING) ok = bar_wait<!KV8>(smem_u32(&sh.empty[slot]), (item / RING - 1) & 1, gave_up);
                    dst = ring + slot * CH_MAT; bar = smem_u32(&sh.full[slot]);
                }
                if (!ok) break;
                if (lane == 0) bar_expect(bar, KV8 ? CH_HALF : CH_MAT);
                __syncwarp();
                constexpr int HALVES = KV8 ? 1 : 2;
                if (p.c.paged) {
                    if (lane < 8 * HALVES)
                        tma_load4(dst + (lane >> 3) * CH_HALF + (lane & 7) * 2048, map, bar, (lane >> 3) * 64, 0, hcoord, page * p.page_mul + (page == p.c.num_pages && !p.page_mul ? 1 : 0));
                } else if (lane < HALVES) {
                    tma_load4(dst + lane * CH_HALF, map, bar, lane * 64, key0, hcoord, w.b * p.batch_mul);
                }
            }
            if (!ok) break;
        }
    } else if (KV8 && warp >= 12 && busy) {
        // ---- codes to fp16 ----
        const int l = tid & 127;
        for (int item = 0; item < 2 * w.tiles; ++item) {
            const int rs = item % CH_RAW, slot = item % RING;
            if (!bar_wait<false>(smem_u32(&sh.raw_full[rs]), (item / CH_RAW) & 1, gave_up)) break;
            if (item >= RING && !bar_wait<false>(smem_u32(&sh.empty[slot]), (item / RING - 1) & 1, gave_up)) break;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int k = u * 128 + l, r = k >> 3, c = k & 7;           // sixteen channels of a position
                uint32_t x[4], y[8];
                lds128(raw + rs * CH_HALF + r * 128 + ((c ^ (r & 7)) << 4), x);
#pragma unroll
                for (int j = 0; j < 4; ++j) e4m3x4_to_f16x2x2(x[j], y[2 * j], y[2 * j + 1]);
                const uint32_t to = ring + slot * CH_MAT + (c >> 2) * CH_HALF + r * 128;
                const int c0 = 2 * (c & 3);
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(to + ((c0 ^ (r & 7)) << 4)), "r"(y[0]), "r"(y[1]), "r"(y[2]), "r"(y[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(to + (((c0 + 1) ^ (r & 7)) << 4)), "r"(y[4]), "r"(y[5]), "r"(y[6]), "r"(y[7]) : "memory");
            }
            smem_to_async();
            __syncwarp();
            if (lane == 0) { bar_arrive(smem_u32(&sh.full[slot])); bar_arrive(smem_u32(&sh.raw_empty[rs])); }
        }
    }
    __syncwarp();
    if (joined) {
        // ---- partial results of the streams and of the cluster's CTAs ----
        if (ranks > 1) { cluster_arrive(); cluster_wait(); } else __syncthreads();
        const int here = min(2 * tt, w.new_tokens - w.t0) * G;              // rows of this CTA tile, the same for the cluster
        const int warps = (KV8 ? CH_THREADS8 : CH_THREADS) / 32, parts = w.twin ? 2 * ranks : ranks;
        const float vs = KV8 && p.v_scale ? read_global(p.v_scale + w.g) : 1.f;
        for (int r = rank + warp * ranks; r < here; r += warps * ranks) {
            const int s = w.twin ? 0 : r / (tt * G), row = w.twin ? r : r % (tt * G);
            const int token = w.t0 + r / G, head = w.g * G + r % G;
            auto ld = [&](uint32_t a) { float v; asm volatile("ld.shared::cluster.f32 %0, [%1];\n" : "=f"(v) : "r"(a) : "memory"); return v; };
            float mi = -INFINITY, li = 0.f;                 // lane i holds part i's (at most 32)
            if (lane < parts) {
                const int st = w.twin ? lane & 1 : s;
                const uint32_t at = base + (st * CH_TILE + row) * 4;
                mi = ld(cluster_addr(at + CH_PART_MAX, w.twin ? lane >> 1 : lane));
                li = ld(cluster_addr(at + CH_PART_SUM, w.twin ? lane >> 1 : lane));
            }
            float m = mi;
#pragma unroll
            for (int sft = 16; sft; sft >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, sft));
            // (a part with weights counts for something however far it stands below the others: an infinity among its values is still one)
            const float f = mi == -INFINITY && li == 0.f ? 0.f : (mi == m || li != li ? 1.f : fmaxf(fast_exp2(mi - m), 0x1p-120f));
            float l = f == 0.f ? 0.f : li * f;
#pragma unroll
            for (int sft = 16; sft; sft >>= 1) l += __shfl_xor_sync(0xffffffffu, l, sft);
            float o[4] = {0.f, 0.f, 0.f, 0.f};
            for (int i = 0; i < parts; ++i) {
                const float fi = __shfl_sync(0xffffffffu, f, i);
                if (fi == 0.f) continue;                    // (its rows may never have been written)
                const int st = w.twin ? i & 1 : s;
                const uint32_t a = cluster_addr(base + ((st * CH_TILE + row) * 32 + (lane ^ (row & 31))) * 16, w.twin ? i >> 1 : i);
                float v[4];
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];\n" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(a) : "memory");
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] = fmaf(fi, v[j], o[j]);
            }
            const bool some = l != 0.f;
            const long long at = (long long)(w.q_row + token - w.t0) * p.c.Hq + head;
            const float inv = some ? vs / l : 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = some ? o[j] * inv : 0.f;
            if (p.out_bf16) *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(p.out) + at * HEAD_DIM + lane * 4) = make_uint2(pack_bf16(o[0], o[1]), pack_bf16(o[2], o[3]));
            else *reinterpret_cast<float4*>(p.out + at * HEAD_DIM + lane * 4) = make_float4(o[0], o[1], o[2], o[3]);
            if (lane == 0 && p.lse) p.lse[at] = some ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
        }
        if (ranks > 1) { cluster_arrive(); cluster_wait(); }               // nobody leaves while its results are read
    }
    if (sh.gave_up) let_land();
    tmem_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(tmem));
    if (tid == 0 && sh.gave_up) atomicOr(p.c.status, STATUS_WAITED_OUT);
}

}  // namespace tidal
