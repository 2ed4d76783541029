// Eviction from a cache by accumulated weight: which positions stay (evict_select_kernel), and their rows and weights moved
// together (gather_copy_kernel into another cache, gather_inplace_kernel within one).
#pragma once

#include "block_kernels.cuh"

namespace tidal {

// ---- the m positions with the largest weights ------------------------------------------------------------------
// A cluster per (sequence, weight head): every CTA keeps the order-preserving keys of its slice of the row in shared memory (one
// read of memory in all), and three rounds of 2048, 2048 and 1024 bins over the cluster's histograms find the m-th largest key and how many of
// the positions that share it still belong to the set. In a round every CTA counts its slice, adds up its share of the
// bins over all CTAs and hands the sums to all, so that each finds the bin for itself. Then each CTA counts what it
// keeps and writes it behind what the CTAs before it keep, in ascending order; of equal weights the lower positions.
// Bound by that chain of barriers and by the instructions of three counts, not by its 4 bytes a position: 8 rows of 131072 16.7 us in clusters of
// eight (clusters of sixteen do not all find room at once: half as long again on some GPUs), 64 rows of up to 65536 21 us in clusters of two.
struct EvictParams {
    const float* weights;                                   // [batch][heads][stride]
    long long stride;
    const int* ctx_lens;
    int max_ctx, heads, m, keep_first, keep_last;
    int* kept;                                              // [batch][heads][m]
    int* new_lens;                                          // [batch]
};

constexpr int EV_THREADS = 1024, EV_WARPS = EV_THREADS / 32, EV_BINS = 2048, EV_MAX_CLUSTER = 8, EV_BATCH = 4, EV_TLOG = 10;
constexpr int EV_MERGE = EV_BINS / EV_THREADS;               // counts that a thread merges, bins that it scans
constexpr size_t EV_SMEM_MAX = 160 * 1024;

// Order-preserving: larger weight, larger key; -0 as 0; not-a-number below everything. Kept positions are above everything.
__device__ __forceinline__ uint32_t evict_key(float w) {
    if (!(w == w)) return 1u;                               // (0: no position)
    const uint32_t b = __float_as_uint(w + 0.f);
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}
__device__ __forceinline__ int ld_cluster(uint32_t addr, int rank) {
    int v;
    asm volatile("ld.shared::cluster.s32 %0, [%1];\n" : "=r"(v) : "r"(cluster_addr(addr, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_int(uint32_t addr, int rank, int v) {
    asm volatile("st.shared::cluster.s32 [%0], %1;\n" ::"r"(cluster_addr(addr, rank)), "r"(v) : "memory");
}

__global__ void __launch_bounds__(EV_THREADS) evict_select_kernel(const EvictParams p) {
    extern __shared__ __align__(16) uint32_t ev_keys[];
    __shared__ int s_hist[EV_BINS], s_all[EV_BINS], s_part[EV_WARPS], s_found[2], s_mine[2];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int C, rank;
    asm volatile("mov.u32 %0, %%cluster_nctarank;\n" : "=r"(C));
    asm volatile("mov.u32 %0, %%cluster_ctarank;\n" : "=r"(rank));
    const int clog = 31 - __clz(C), row = blockIdx.x >> clog, b = row / p.heads;          // (cluster sizes are powers of two)
    pdl_wait();
    pdl_trigger();
    const int n = max(min(read_global(p.ctx_lens + b), p.max_ctx), 0);
    const int want = min(p.m, n);
    int* const kept = p.kept + (long long)row * p.m;
    if (rank == 0 && tid == 0 && row == b * p.heads) p.new_lens[b] = want;
    for (int i = want + rank * EV_THREADS + tid; i < p.m; i += C * EV_THREADS) kept[i] = -1;
    if (want == n) {                                        // everything stays
        for (int i = rank * EV_THREADS + tid; i < n; i += C * EV_THREADS) kept[i] = i;
        return;                                             // (the whole cluster)
    }
    const int slice = (((n + C - 1) >> clog) + 3) & ~3, lo = min(rank * slice, n), cnt = min(slice, n - lo);
    const float* const w = p.weights + (long long)row * p.stride + lo;
    // four positions at a time, counted by their top digit on the way; behind the slice's end keys below every other
    const int groups = (cnt + 3) >> 2;
    uint4* const keys4 = reinterpret_cast<uint4*>(ev_keys);
    const bool aligned = ((uintptr_t)w & 15) == 0;
    for (int i = tid; i < EV_BINS; i += EV_THREADS) s_hist[i] = 0;
    __syncthreads();
    for (int i0 = tid; i0 < groups; i0 += EV_BATCH * EV_THREADS) {
        float4 x[EV_BATCH];
#pragma unroll
        for (int u = 0; u < EV_BATCH; ++u) {
            const int i = 4 * (i0 + u * EV_THREADS);
            x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (aligned && i + 4 <= cnt) {
                x[u] = read_global(reinterpret_cast<const float4*>(w + i));
            } else if (i < cnt) {
                x[u].x = read_global(w + i);
                if (i + 1 < cnt) x[u].y = read_global(w + i + 1);
                if (i + 2 < cnt) x[u].z = read_global(w + i + 2);
                if (i + 3 < cnt) x[u].w = read_global(w + i + 3);
            }
        }
#pragma unroll
        for (int u = 0; u < EV_BATCH; ++u) {
            const int i = 4 * (i0 + u * EV_THREADS);
            if (i >= cnt) break;
            const float y[4] = {x[u].x, x[u].y, x[u].z, x[u].w};
            uint32_t key[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int pos = lo + i + v;
                const bool keep = pos < p.keep_first || pos >= n - p.keep_last;
                key[v] = i + v >= cnt ? 0u : keep ? 0xffffffffu : evict_key(y[v]);
                atomicAdd(&s_hist[key[v] >> 21], 1);        // (keys of no position are below what is looked for)
            }
            keys4[i >> 2] = make_uint4(key[0], key[1], key[2], key[3]);
        }
    }
    // the want-th largest key, digit by digit from the top
    uint32_t prefix = 0, known = 0;
    int left = want;                                        // of the keys that share the prefix
    const uint32_t all_addr = smem_u32(s_all), hist_addr = smem_u32(s_hist), mine_addr = smem_u32(s_mine);
#pragma unroll 1
    for (int round = 0; round < 3; ++round) {
        const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bins = round == 2 ? 1024 : 2048;
        if (round > 0) {
            for (int i = tid; i < bins; i += EV_THREADS) s_hist[i] = 0;
            __syncthreads();
            for (int i = tid; i < groups; i += EV_THREADS) {
                const uint4 k = keys4[i];
                const uint32_t key[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    if ((key[v] & known) == prefix) atomicAdd(&s_hist[(key[v] >> shift) & (bins - 1)], 1);
            }
        }
        if (C > 1) {
            cluster_arrive(); cluster_wait();
            // this CTA's share of the bins, several threads to a bin with one or two CTAs' counts each
            const int tlog = max(clog + EV_TLOG - (round == 2 ? 10 : 11), 0), team = 1 << tlog, sub = tid & (team - 1);
            for (int own = tid >> tlog; own < bins >> clog; own += EV_THREADS >> tlog) {
                const uint32_t at = (uint32_t)(rank * (bins >> clog) + own) * 4;
                int sum = 0;
#pragma unroll
                for (int u = 0; u < EV_MERGE; ++u) if (sub + u * team < C) sum += ld_cluster(hist_addr + at, sub + u * team);
                for (int sh = team >> 1; sh; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
#pragma unroll
                for (int u = 0; u < EV_MERGE; ++u) if (sub + u * team < C) st_cluster_int(all_addr + at, sub + u * team, sum);
            }
            cluster_arrive(); cluster_wait();
        } else {
            __syncthreads();
            for (int i = tid; i < bins; i += EV_THREADS) s_all[i] = s_hist[i];
            __syncthreads();
        }
        // bins from the top: thread t holds bins bins - 1 - 2 t and the one below it (bins - 1 - t in the last round)
        const int per = bins >> EV_TLOG;
        int v[EV_MERGE], sum = 0;
#pragma unroll
        for (int u = 0; u < EV_MERGE; ++u) { v[u] = u < per ? s_all[bins - 1 - tid * per - u] : 0; sum += v[u]; }
        int x = sum;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, sh); if (lane >= sh) x += y; }
        if (lane == 31) s_part[warp] = x;
        __syncthreads();
        int y = lane < EV_WARPS ? s_part[lane] : 0;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) { const int z = __shfl_up_sync(0xffffffffu, y, sh); if (lane >= sh) y += z; }
        const int before = __shfl_sync(0xffffffffu, y, max(warp - 1, 0));
        int above = x - sum + (warp ? before : 0);
#pragma unroll
        for (int u = 0; u < EV_MERGE; ++u) {
            if (u < per && above < left && above + v[u] >= left) { s_found[0] = bins - 1 - tid * per - u; s_found[1] = left - above; }
            above += v[u];
        }
        __syncthreads();
        prefix |= (uint32_t)s_found[0] << shift;
        known |= (uint32_t)(bins - 1) << shift;
        left = s_found[1];
    }
    // every warp a run of the slice: how much it keeps for certain, and how much shares the last key (both in one word, 16 bits each)
    const int run = ((groups + EV_WARPS - 1) / EV_WARPS + 31) & ~31, from = min(warp * run, groups), to = min(from + run, groups);
    auto counts = [&](const uint4& k) {
        int c = 0;
        const uint32_t key[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
        for (int v = 0; v < 4; ++v) c += (key[v] > prefix ? 1 : 0) + (key[v] == prefix ? 0x10000 : 0);
        return c;
    };
    int both = 0;
    for (int i = from + lane; i < to; i += 32) both += counts(keys4[i]);
    int more = both & 0xffff, same = both >> 16;
#pragma unroll
    for (int sh = 16; sh; sh >>= 1) { more += __shfl_xor_sync(0xffffffffu, more, sh); same += __shfl_xor_sync(0xffffffffu, same, sh); }
    __shared__ int s_more[EV_WARPS], s_same[EV_WARPS];
    if (lane == 0) { s_more[warp] = more; s_same[warp] = same; }
    __syncthreads();
    int a = lane < EV_WARPS ? s_more[lane] : 0, e = lane < EV_WARPS ? s_same[lane] : 0;
#pragma unroll
    for (int sh = 1; sh < 32; sh <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, a, sh), z = __shfl_up_sync(0xffffffffu, e, sh);
        if (lane >= sh) { a += y; e += z; }
    }
    if (tid == 31) { s_mine[0] = a; s_mine[1] = e; }
    int more_at = __shfl_sync(0xffffffffu, a, max(warp - 1, 0)), same_at = __shfl_sync(0xffffffffu, e, max(warp - 1, 0));
    if (warp == 0) more_at = same_at = 0;
    if (C > 1) {
        cluster_arrive(); cluster_wait();
        int x = 0, y = 0;                                   // what the CTAs before this one keep
        if (lane < rank) { x = ld_cluster(mine_addr, lane); y = ld_cluster(mine_addr + 4, lane); }
#pragma unroll
        for (int sh = 8; sh; sh >>= 1) { x += __shfl_xor_sync(0xffffffffu, x, sh); y += __shfl_xor_sync(0xffffffffu, y, sh); }
        more_at += __shfl_sync(0xffffffffu, x, 0);
        same_at += __shfl_sync(0xffffffffu, y, 0);
        cluster_arrive();                                   // (waited for at the end: nobody leaves while it is read)
    }
    for (int i = from; i < to; i += 32) {
        const uint4 k = i + lane < to ? keys4[i + lane] : make_uint4(0, 0, 0, 0);
        const int mine = counts(k);
        int x = mine;
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) { const int y = __shfl_up_sync(0xffffffffu, x, sh); if (lane >= sh) x += y; }
        if (mine) {
            int m_at = more_at + ((x - mine) & 0xffff), e_at = same_at + ((x - mine) >> 16);
            const uint32_t key[4] = {k.x, k.y, k.z, k.w};
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const bool certain = key[v] > prefix, shares = key[v] == prefix;
                if (certain || (shares && e_at < left)) kept[m_at + min(e_at, left)] = lo + 4 * (i + lane) + v;
                m_at += certain;
                e_at += shares;
            }
        }
        const int all = __shfl_sync(0xffffffffu, x, 31);
        more_at += all & 0xffff;
        same_at += all >> 16;
    }
    if (C > 1) cluster_wait();
}

// ---- rows of listed positions moved to the front -----------------------------------------------------------------
struct GatherParams {
    BlockCache from;
    uint8_t* k;                                             // where the rows go: another cache, or this one
    uint8_t* v;
    long long stride_b, stride_pos, stride_head, stride_page;
    const int* page_table;
    int max_pages, num_pages, paged, max_ctx;
    const int* kept;                                        // [batch][heads][m]
    const int* counts;                                      // [batch]
    int heads, m, row_bytes;
    const float* weights;
    float* weights_out;
    long long w_stride, wo_stride;
};

constexpr int GA_WARPS = 8, GA_ROWS = 16, GA_UNROLL = 8;

// Byte offset of position pos (element offset times the element's size), -1 where a page id is outside the pool.
__device__ __forceinline__ long long cache_row(const int* table, int max_pages, int num_pages, int paged, long long stride_b, long long stride_pos,
                                               long long stride_page, int b, int pos, int* status) {
    if (!paged) return b * stride_b + pos * stride_pos;
    const int page = read_global(table + (long long)b * max_pages + pos / TILE);
    if ((unsigned)page >= (unsigned)num_pages) { atomicOr(status, STATUS_BAD_PAGE); return -1; }
    return page * stride_page + (pos % TILE) * stride_pos;
}

// How many rows of sequence b are moved, and the source of the j-th (-1: none).
__device__ __forceinline__ int gather_count(const GatherParams& p, int b) { return max(min(read_global(p.counts + b), p.m), 0); }
__device__ __forceinline__ int gather_source(const GatherParams& p, int b, int g, int j, int n) {
    const int pos = read_global(p.kept + ((long long)b * p.heads + (p.heads > 1 ? g : 0)) * p.m + j);
    if ((unsigned)pos >= (unsigned)n) { if (pos != -1) atomicOr(p.from.status, STATUS_BAD_INDEX); return -1; }
    return pos;
}

// Into another cache: a warp takes sixteen rows. A lane works out one row's two places, and the warp moves them row by row (16 bits: a position's key and value
// row fill a warp with 16 bytes per lane; 8 bits: half of one), eight loads in flight. Bound by memory: 98000 rows of eight heads from pages into
// pages 127 us, 6.3 TB/s (with every lane working out every row's places 158).
template <bool KV8>
__global__ void __launch_bounds__(GA_WARPS * 32) gather_copy_kernel(const GatherParams p) {
    constexpr int ROWS = KV8 ? 2 : 1, LANES = 32 / ROWS, STEPS = GA_ROWS / ROWS;
    constexpr int ESZ = KV8 ? 1 : 2;
    const int lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES, piece = l % (LANES / 2);
    const bool value = l >= LANES / 2;
    const BlockCache& c = p.from;
    const long long unit = (long long)blockIdx.x * GA_WARPS + (threadIdx.x >> 5);
    const int groups = (p.m + GA_ROWS - 1) / GA_ROWS;
    const long long pair = unit / groups;
    pdl_wait();
    pdl_trigger();
    if (pair >= (long long)c.batch * c.Hkv) return;
    const int b = (int)(pair / c.Hkv), g = (int)(pair - (long long)b * c.Hkv);
    const int j0 = (int)(unit - pair * groups) * GA_ROWS, j = j0 + (lane & (GA_ROWS - 1));
    // (the list's entry is asked for together with the lengths that say which of them count)
    const long long row = (long long)b * p.heads + (p.heads > 1 ? g : 0);
    const int pos = j < p.m ? read_global(p.kept + row * p.m + j) : -1;
    const int all = gather_count(p, b), cnt = min(all, p.max_ctx), n = cached_len(c, b);
    if (j0 >= all) return;
    long long src = -1, dst = -1;
    if (j < all) {
        if (j >= cnt || (unsigned)pos >= (unsigned)n) {     // (behind cnt there is no place for it)
            if (pos != -1 && lane < GA_ROWS) atomicOr(c.status, STATUS_BAD_INDEX);
        } else {
            if (p.weights && lane < GA_ROWS && (p.heads > 1 || g == 0)) p.weights_out[row * p.wo_stride + j] = read_global(p.weights + row * p.w_stride + pos);
            src = cache_row(c.page_table, c.max_pages, c.num_pages, c.paged, c.stride_b, c.stride_pos, c.stride_page, b, pos, c.status);
            dst = cache_row(p.page_table, p.max_pages, p.num_pages, p.paged, p.stride_b, p.stride_pos, p.stride_page, b, j, c.status);
            if (src < 0 || dst < 0) src = -1;
        }
    }
    const uint8_t* const from = (value ? c.v : c.k) + g * c.stride_head * ESZ + piece * 16;
    uint8_t* const to = (value ? p.v : p.k) + g * p.stride_head * ESZ + piece * 16;
#pragma unroll
    for (int u0 = 0; u0 < STEPS; u0 += GA_UNROLL) {
        if (j0 + u0 * ROWS >= cnt) break;
        uint4 w[GA_UNROLL];
        long long at[GA_UNROLL];
#pragma unroll
        for (int u = 0; u < GA_UNROLL; ++u) {
            const int r = (u0 + u) * ROWS + sub;
            const long long s = __shfl_sync(0xffffffffu, src, r);
            at[u] = s < 0 ? -1 : 0;
            if (s >= 0) w[u] = read_global(reinterpret_cast<const uint4*>(from + s * ESZ));
        }
#pragma unroll
        for (int u = 0; u < GA_UNROLL; ++u) {
            const long long d = __shfl_sync(0xffffffffu, dst, (u0 + u) * ROWS + sub);
            if (at[u] >= 0) *reinterpret_cast<uint4*>(to + d * ESZ) = w[u];
        }
    }
}

// Within a cache: the j-th listed position is never below j (the list is ascending), so a row may be written once all rows up to it
// have been read. A CTA takes a column of 32 bytes of all rows of a sequence and KV head, so that this order is its own affair: it reads
// GI_ROWS rows, waits for its threads, writes them. The last CTAs move the weights in the same way. 64 sequences of eight heads that lose 1 to 16 of about 2056
// positions, one list for all heads: 276 us for 461 MB that move (both ways 3.3 TB/s), over E4M3 144 us; where one of the 64 loses any, 77 us, of
// which reading every list once per column is most.
constexpr int GI_THREADS = 512, GI_COLUMN = 32, GI_UNROLL = 4;
constexpr int GI_ROWS = GI_THREADS / (GI_COLUMN / 16) * GI_UNROLL;

__global__ void __launch_bounds__(GI_THREADS) gather_inplace_kernel(const GatherParams p) {
    const int esz = p.row_bytes / HEAD_DIM;
    const BlockCache& c = p.from;
    const int columns = 2 * p.row_bytes / GI_COLUMN, tid = threadIdx.x;
    const long long moves = (long long)c.batch * c.Hkv * columns;
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x >= moves) {                              // weights
        const int row = (int)(blockIdx.x - moves), b = row / p.heads, g = row - b * p.heads;
        const int n = cached_len(c, b), cnt = min(gather_count(p, b), n);
        float* const w = p.weights_out + (long long)row * p.wo_stride;
        const float* const from = p.weights + (long long)row * p.w_stride;
        for (int j0 = 0; j0 < cnt; j0 += GI_THREADS) {
            const int j = j0 + tid, pos = j < cnt ? gather_source(p, b, g, j, n) : -1;
            float x = 0.f;
            if (pos >= 0) x = read_global(from + pos);
            __syncthreads();
            if (pos >= 0) w[j] = x;
        }
        return;
    }
    const int col = (int)(blockIdx.x % columns);
    const long long pair = blockIdx.x / columns;
    const int b = (int)(pair / c.Hkv), g = (int)(pair - (long long)b * c.Hkv);
    const int all = gather_count(p, b), n = cached_len(c, b), cnt = min(all, n);       // (an ascending list has no more)
    if (col == 0)
        for (int j = cnt + tid; j < all; j += GI_THREADS) gather_source(p, b, g, j, 0);    // (what it has all the same is reported)
    const int byte = col * GI_COLUMN + (tid % (GI_COLUMN / 16)) * 16;
    const bool value = byte >= p.row_bytes;
    uint8_t* const base = (value ? p.v : p.k) + (long long)g * c.stride_head * esz + (value ? byte - p.row_bytes : byte);
    for (int j0 = 0; j0 < cnt; j0 += GI_ROWS) {
        uint4 w[GI_UNROLL];
        long long to[GI_UNROLL];
#pragma unroll
        for (int u = 0; u < GI_UNROLL; ++u) {
            const int j = j0 + u * (GI_ROWS / GI_UNROLL) + tid / (GI_COLUMN / 16);
            to[u] = -1;
            const int pos = j < cnt ? gather_source(p, b, g, j, n) : -1;
            if (pos < 0 || pos == j) continue;              // (a row that stays where it is)
            const long long src = cache_row(c.page_table, c.max_pages, c.num_pages, c.paged, c.stride_b, c.stride_pos, c.stride_page, b, pos, c.status);
            const long long dst = cache_row(c.page_table, c.max_pages, c.num_pages, c.paged, c.stride_b, c.stride_pos, c.stride_page, b, j, c.status);
            if (src < 0 || dst < 0) continue;
            w[u] = read_global(reinterpret_cast<const uint4*>(base + src * esz));
            to[u] = dst * esz;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < GI_UNROLL; ++u)
            if (to[u] >= 0) *reinterpret_cast<uint4*>(base + to[u]) = w[u];
    }
}

}  // namespace tidal
