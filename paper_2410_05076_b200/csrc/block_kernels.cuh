// Block-sparse decode attention: blocks of 16 positions (one page) ranked by an upper bound of their logits.
//
//   block_bounds_kernel  per block and KV head the channelwise least and greatest key (lo, hi), in bf16 (exact)
//   block_select_kernels.cuh   s = sum_c max(q_c lo_c, q_c hi_c) >= q . k for every key k of a block, and per index head the
//                        m blocks with the largest s, exactly, ties toward the lower block
//   block_attn_kernels.cuh     softmax attention over the cached positions of the listed blocks
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
// by shuffles. Bound by memory: the keys are read once, 512 bytes are written per 16 rows (131072 positions of 8 heads 44 us,
// 6.9 TB/s).
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
    const int start = p.start_lens ? max(min(p.start_lens[b], n), 0) : 0;      // (shorter now: its last block has lost keys)
    const long long blk_l = (long long)(start / TILE) + (w - pair * p.blocks);
    if (blk_l * TILE >= n) return;
    const int blk = (int)blk_l, rows = min(TILE, n - blk * TILE);
    int page = 0;
    long long off = (long long)g * c.stride_head;
    if (c.paged) {
        page = read_global(c.page_table + (long long)b * c.max_pages + blk);
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
            if (r0 + 2 * i < rows) x[i] = read_global(reinterpret_cast<const uint4*>(src + 2 * i * c.stride_pos));
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
            if (r0 + 4 * i < rows) x[i] = read_global(reinterpret_cast<const uint4*>(src + 4 * i * c.stride_pos));
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

// ---- pairs of fp32 in one instruction --------------------------------------------------------------------------
using f32pair = unsigned long long;
__device__ __forceinline__ f32pair pair2(float lo, float hi) {
    f32pair d;
    asm("mov.b64 %0, {%1, %2};\n" : "=l"(d) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ float half2(f32pair v, int i) {
    float lo, hi;
    asm("mov.b64 {%0, %1}, %2;\n" : "=f"(lo), "=f"(hi) : "l"(v));
    return i ? hi : lo;
}
__device__ __forceinline__ f32pair add2(f32pair a, f32pair b) {
    f32pair d;
    asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32pair mul2(f32pair a, f32pair b) {
    f32pair d;
    asm("mul.rn.f32x2 %0, %1, %2;\n" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32pair fma2(f32pair a, f32pair b, f32pair c) {
    f32pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32pair fma2_rm(f32pair a, f32pair b, f32pair c) {       // rounded downwards: x - x is -0
    f32pair d;
    asm("fma.rm.f32x2 %0, %1, %2, %3;\n" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}

// ---- thread-block clusters -----------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_addr(uint32_t addr, int rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;\n" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, int rank, float v) {
    asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(cluster_addr(addr, rank)), "f"(v) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;\n" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;\n" ::: "memory"); }

}  // namespace tidal
