// Paged caches filled on the device: page tables and slot maps from request lengths (page_map_kernel) and
// the rows of many tokens written through a slot map (kv_write_kernel).
#pragma once

#include <cooperative_groups.h>
#include <cuda_fp8.h>

#include "attn_kernels.cuh"

namespace tidal {

enum { STATUS_NO_PAGES = 8 };            // page_map: the request cannot be met, nothing was changed

// ---- page tables and slot maps ---------------------------------------------------------------------------
// With P(x) = ceil(x / 16), sequence b gives back rel_b = max(P(old) - P(new), 0) pages, takes
// grow_b = max(P(new) - P(old), 0) and writes tok_b = max(new - old, 0) tokens. The pages given back are pushed on the
// stack of free pages in the order (sequence, logical page), then the growing sequences pop theirs in the same
// order: with F free pages and R pushed, the i-th page taken is element F + R - 1 - i of the stack after the
// push, which is free_pages[.] below F and the (. - F)-th page given back from F on. So every page is known from three
// prefix sums over the sequences and nothing has to be moved before it is read.
//
// One launch of one thread-block cluster: every CTA computes the prefix sums and the checks for itself (a few
// thousand lengths), the cluster's barrier separates all reads of what is written in place (num_free, the stack's upper
// part) from the writes, and tables and slots are then dealt out over the cluster's threads.
constexpr int PM_THREADS = 1024;
constexpr int PM_PER = 4;                                   // sequences per thread
constexpr int PM_MAX_BATCH = PM_THREADS * PM_PER;

struct PageMapParams {
    int batch, max_pages, num_pages, max_tokens;
    const int* old_lens;
    const int* new_lens;
    int* page_table;
    int* free_pages;
    const int* num_free;
    int* num_free_out;
    long long* slots;
    int* positions;
    int* token_offsets;
    int* status;
};

// The sequence that element `i` of a packed list belongs to: the last one that starts at or before it.
__device__ __forceinline__ int owner_of(const int* starts, int batch, int i) {
    int lo = 0, hi = batch;                                 // starts[lo] <= i < starts[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= i) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(PM_THREADS) page_map_kernel(const PageMapParams p) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    extern __shared__ int pm_smem[];
    int* s_tok = pm_smem;                                   // [batch + 1] prefix sums
    int* s_grow = s_tok + p.batch + 1;
    int* s_rel = s_grow + p.batch + 1;
    __shared__ long long s_part[3][PM_THREADS / 32];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid == 0) s_bad = 0;
    pdl_wait();
    pdl_trigger();
    __syncthreads();

    const long long limit = (long long)p.max_pages * TILE;
    long long v[PM_PER][3], sum[3] = {0, 0, 0};
    bool bad = false;
#pragma unroll
    for (int u = 0; u < PM_PER; ++u) {
        const int b = tid * PM_PER + u;
        v[u][0] = v[u][1] = v[u][2] = 0;
        if (b < p.batch) {
            const int o = p.old_lens[b], n = p.new_lens[b];
            if (o < 0 || n < 0 || o > limit || n > limit) {
                bad = true;
            } else {
                const int d = (n + TILE - 1) / TILE - (o + TILE - 1) / TILE;
                v[u][0] = max(n - o, 0); v[u][1] = max(d, 0); v[u][2] = max(-d, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) sum[i] += v[u][i];
    }
    if (bad) s_bad = 1;
    long long inc[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        long long x = sum[i];
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, sh);
            if (lane >= sh) x += y;
        }
        inc[i] = x;
        if (lane == 31) s_part[i][warp] = x;
    }
    __syncthreads();
    if (warp < 3) {
        long long x = s_part[warp][lane];
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
            const long long y = __shfl_up_sync(0xffffffffu, x, sh);
            if (lane >= sh) x += y;
        }
        s_part[warp][lane] = x;
    }
    __syncthreads();
    const long long T = s_part[0][31], N = s_part[1][31], R = s_part[2][31];
    long long at[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) at[i] = inc[i] - sum[i] + (warp > 0 ? s_part[i][warp - 1] : 0);
#pragma unroll
    for (int u = 0; u < PM_PER; ++u) {
        const int b = tid * PM_PER + u;
        // (sums that pass 32 bits fail the checks below and are not used)
        if (b <= p.batch) { s_tok[b] = (int)at[0]; s_grow[b] = (int)at[1]; s_rel[b] = (int)at[2]; }
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] += v[u][i];
    }
    if (tid == PM_THREADS - 1 && p.batch == PM_MAX_BATCH) { s_tok[p.batch] = (int)T; s_grow[p.batch] = (int)N; s_rel[p.batch] = (int)R; }
    const long long F = *p.num_free;
    const bool fits = F >= 0 && F <= p.num_pages && T <= p.max_tokens && F + R <= p.num_pages && N <= F + R;
    __syncthreads();
    // the j-th page given back, in the order (sequence, logical page)
    auto released = [&](int j) -> int {
        const int b = owner_of(s_rel, p.batch, j);
        return p.page_table[(long long)b * p.max_pages + (p.new_lens[b] + TILE - 1) / TILE + (j - s_rel[b])];
    };
    if (fits && !s_bad)
        for (int j = tid; j < (int)R; j += PM_THREADS)
            if ((unsigned)released(j) >= (unsigned)p.num_pages) s_bad = 1;
    __syncthreads();
    const bool ok = fits && !s_bad;
    cluster.sync();                                         // everything that is overwritten below has been read

    const int gtid = (int)cluster.block_rank() * PM_THREADS + tid, gsize = (int)cluster.num_blocks() * PM_THREADS;
    if (!ok) {
        for (int t = gtid; t < p.max_tokens; t += gsize) { p.slots[t] = -1; if (p.positions) p.positions[t] = -1; }
        if (p.token_offsets) for (int b = gtid; b <= p.batch; b += gsize) p.token_offsets[b] = 0;
        if (gtid == 0) { *p.num_free_out = (int)F; atomicOr(p.status, STATUS_NO_PAGES); }
        return;
    }
    const int top = (int)(F + R);
    auto taken = [&](int i) -> int {                        // the i-th page taken
        const int e = top - 1 - i;
        return e < F ? p.free_pages[e] : released(e - (int)F);
    };
    for (int i = gtid; i < (int)N; i += gsize) {
        const int b = owner_of(s_grow, p.batch, i);
        const int page = taken(i);
        if ((unsigned)page >= (unsigned)p.num_pages) atomicOr(p.status, STATUS_BAD_PAGE);
        p.page_table[(long long)b * p.max_pages + (p.old_lens[b] + TILE - 1) / TILE + (i - s_grow[b])] = page;
    }
    for (int t = gtid; t < p.max_tokens; t += gsize) {
        long long slot = -1;
        int pos = -1;
        if (t < (int)T) {
            const int b = owner_of(s_tok, p.batch, t);
            const int o = p.old_lens[b], held = (o + TILE - 1) / TILE;
            pos = o + (t - s_tok[b]);
            const int blk = pos / TILE;
            const int page = blk < held ? p.page_table[(long long)b * p.max_pages + blk] : taken(s_grow[b] + blk - held);
            if ((unsigned)page < (unsigned)p.num_pages) slot = (long long)page * TILE + (pos & (TILE - 1));
            else atomicOr(p.status, STATUS_BAD_PAGE);
        }
        p.slots[t] = slot;
        if (p.positions) p.positions[t] = pos;
    }
    // pages given back and not taken again stay on the stack: elements F .. F + R - N - 1, which nobody reads
    for (int j = gtid; j < (int)(R - N); j += gsize) p.free_pages[F + j] = released(j);
    if (p.token_offsets) for (int b = gtid; b <= p.batch; b += gsize) p.token_offsets[b] = s_tok[b];
    if (gtid == 0) *p.num_free_out = (int)(F + R - N);
}

// ---- rows of many tokens into the cache ------------------------------------------------------------------
// One warp per (token, KV head): lanes 0-15 move the key row, lanes 16-31 the value row, eight elements each; four such
// units per warp, so that every lane has four loads in flight. Bound by memory: every row is read and written once.
struct KvWriteParams {
    uint8_t* k;
    uint8_t* v;
    const __nv_bfloat16* k_new;
    const __nv_bfloat16* v_new;
    long long k_stride, v_stride;         // elements between tokens of k_new / v_new
    const long long* slots;
    int num_tokens, Hkv, paged, max_ctx;
    long long num_slots;
    long long stride_b, stride_pos, stride_head, stride_page;
    const float* k_scale;
    const float* v_scale;
    int* status;
};

// code = the E4M3 value nearest to x / scale (the quotient in fp32, correctly rounded), saturated at +-448.
__device__ __forceinline__ uint2 quantise8(uint4 w, float scale) {
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t out[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        uint32_t half[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint32_t x = in[2 * i + j];
            const float lo = __fdiv_rn(__uint_as_float(x << 16), scale), hi = __fdiv_rn(__uint_as_float(x & 0xffff0000u), scale);
            half[j] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
        }
        out[i] = half[0] | (half[1] << 16);
    }
    return make_uint2(out[0], out[1]);
}

constexpr int KW_UNITS = 4, KW_WARPS = 8;

template <bool KV8>
__global__ void __launch_bounds__(KW_WARPS * 32) kv_write_kernel(const KvWriteParams p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int piece = lane & 15;
    const bool value = lane >= 16;
    const long long units = (long long)p.num_tokens * p.Hkv;
    const long long u0 = ((long long)blockIdx.x * KW_WARPS + warp) * KW_UNITS;
    pdl_wait();
    pdl_trigger();
    if (u0 >= units) return;
    const __nv_bfloat16* src = value ? p.v_new : p.k_new;
    const long long stride = value ? p.v_stride : p.k_stride;
    uint8_t* dst = value ? p.v : p.k;
    uint4 row[KW_UNITS];
    long long slot[KW_UNITS];
    int head[KW_UNITS];
    long long t = u0 / p.Hkv;
    int g = (int)(u0 - t * p.Hkv);
#pragma unroll
    for (int i = 0; i < KW_UNITS; ++i) {
        slot[i] = -1;
        head[i] = g;
        if (u0 + i < units) {
            slot[i] = __ldg(p.slots + t);
            row[i] = __ldg(reinterpret_cast<const uint4*>(src + t * stride + g * HEAD_DIM) + piece);
        }
        if (++g == p.Hkv) { g = 0; ++t; }
    }
#pragma unroll
    for (int i = 0; i < KW_UNITS; ++i) {
        const long long s = slot[i];
        if (s < 0 || s >= p.num_slots) {
            if (s != -1 && lane == 0) atomicOr(p.status, STATUS_BAD_INDEX);      // -1: padding
            continue;
        }
        long long off = (long long)head[i] * p.stride_head;
        if (p.paged) off += (s / TILE) * p.stride_page + (s % TILE) * p.stride_pos;
        else off += (s / p.max_ctx) * p.stride_b + (s % p.max_ctx) * p.stride_pos;
        if constexpr (KV8) {
            const float* sc = value ? p.v_scale : p.k_scale;
            *reinterpret_cast<uint2*>(dst + off + piece * 8) = quantise8(row[i], sc ? __ldg(sc + head[i]) : 1.f);
        } else {
            *reinterpret_cast<uint4*>(dst + 2 * off + piece * 16) = row[i];
        }
    }
}

}  // namespace tidal
