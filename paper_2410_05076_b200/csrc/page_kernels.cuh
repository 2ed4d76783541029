// Paged caches filled on the device: page tables and slot maps from request lengths (page_map_kernel) and
// the rows of many tokens written through a slot map (kv_write_kernel).
#pragma once

#include <cuda_fp8.h>

#include "block_kernels.cuh"

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
// One launch. Every CTA computes the prefix sums and the checks for itself (a few thousand lengths, all in 32 bits: at most
// 4096 x 262144 tokens) and takes its share of the pages and tokens. What is written in place does not meet
// what is read: the stack is read below F and written from F on, a table is read below P(old) and for shrinking
// sequences, and written from P(old) on for growing ones. The one word that may be both is num_free: the last CTA to have read it
// writes it (an arrival count, nobody waits).
//
// Bound by its chain (lengths, scan, barrier, search, table, slot), not by its 12 bytes a token: 64 requests' decode step 3.1 us,
// 295 K tokens of 8 prompts 4.9 us.
constexpr int PM_PER = 4;                                   // sequences per thread
constexpr int PM_THREADS = 1024, PM_THREADS_SMALL = 256;        // by the number of sequences (rule in tidal_api.cu)
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
    int* arrivals;                       // zero between launches
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

template <int NT>
__global__ void __launch_bounds__(NT) page_map_kernel(const PageMapParams p) {
    extern __shared__ int pm_smem[];
    int* s_tok = pm_smem;                                   // [batch + 1] prefix sums
    int* s_grow = s_tok + p.batch + 1;
    int* s_rel = s_grow + p.batch + 1;
    __shared__ int s_part[3][NT / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_wait();
    pdl_trigger();

    const int F = *p.num_free;
    const int limit = p.max_pages * TILE;                   // at most 262144
    int v[PM_PER][3], sum[3] = {0, 0, 0};
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
    int inc[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        int x = sum[i];
#pragma unroll
        for (int sh = 1; sh < 32; sh <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, sh);
            if (lane >= sh) x += y;
        }
        inc[i] = x;
        if (lane == 31) s_part[i][warp] = x;
    }
    bad = __syncthreads_or(bad);
    int total[3], at[3];
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        int x = lane < NT / 32 ? s_part[i][lane] : 0;
#pragma unroll
        for (int sh = 1; sh < NT / 32; sh <<= 1) {
            const int y = __shfl_up_sync(0xffffffffu, x, sh);
            if (lane >= sh) x += y;
        }
        total[i] = __shfl_sync(0xffffffffu, x, NT / 32 - 1);
        const int before = __shfl_sync(0xffffffffu, x, max(warp - 1, 0));
        at[i] = inc[i] - sum[i] + (warp > 0 ? before : 0);
    }
    const int T = total[0], N = total[1], R = total[2];
#pragma unroll
    for (int u = 0; u < PM_PER; ++u) {
        const int b = tid * PM_PER + u;
        if (b <= p.batch) { s_tok[b] = at[0]; s_grow[b] = at[1]; s_rel[b] = at[2]; }
#pragma unroll
        for (int i = 0; i < 3; ++i) at[i] += v[u][i];
    }
    if (tid == NT - 1 && p.batch == NT * PM_PER) { s_tok[p.batch] = T; s_grow[p.batch] = N; s_rel[p.batch] = R; }
    const long long top = (long long)F + R;                 // the stack's height after the push
    __syncthreads();
    // the j-th page given back, in the order (sequence, logical page)
    auto released = [&](int j) -> int {
        const int b = owner_of(s_rel, p.batch, j);
        return p.page_table[(long long)b * p.max_pages + (p.new_lens[b] + TILE - 1) / TILE + (j - s_rel[b])];
    };
    bool ok = !bad && F >= 0 && F <= p.num_pages && T <= p.max_tokens && top <= p.num_pages && N <= top;
    if (ok && R > 0) {
        for (int j = tid; j < R; j += NT) bad |= (unsigned)released(j) >= (unsigned)p.num_pages;
        ok = !__syncthreads_or(bad);
    }

    const int gtid = (int)blockIdx.x * NT + tid, gsize = (int)gridDim.x * NT;
    if (ok) {
        auto taken = [&](int i) -> int {                    // the i-th page taken
            const int e = (int)top - 1 - i;
            return e < F ? p.free_pages[e] : released(e - F);
        };
        for (int i = gtid; i < N; i += gsize) {
            const int b = owner_of(s_grow, p.batch, i);
            const int page = taken(i);
            if ((unsigned)page >= (unsigned)p.num_pages) atomicOr(p.status, STATUS_BAD_PAGE);
            p.page_table[(long long)b * p.max_pages + (p.old_lens[b] + TILE - 1) / TILE + (i - s_grow[b])] = page;
        }
        for (unsigned t = gtid; t < (unsigned)p.max_tokens; t += gsize) {          // (max_tokens + gsize may pass 2^31)
            long long slot = -1;
            int pos = -1;
            if (t < (unsigned)T) {
                const int b = owner_of(s_tok, p.batch, (int)t);
                const int o = p.old_lens[b], held = (o + TILE - 1) / TILE;
                pos = o + ((int)t - s_tok[b]);
                const int blk = pos / TILE;
                const int page = blk < held ? p.page_table[(long long)b * p.max_pages + blk] : taken(s_grow[b] + blk - held);
                if ((unsigned)page < (unsigned)p.num_pages) slot = (long long)page * TILE + (pos & (TILE - 1));
                else atomicOr(p.status, STATUS_BAD_PAGE);
            }
            p.slots[t] = slot;
            if (p.positions) p.positions[t] = pos;
        }
        // pages given back and not taken again stay on the stack: elements F .. F + R - N - 1, which nobody reads
        for (int j = gtid; j < R - N; j += gsize) p.free_pages[F + j] = released(j);
    } else {
        for (unsigned t = gtid; t < (unsigned)p.max_tokens; t += gsize) { p.slots[t] = -1; if (p.positions) p.positions[t] = -1; }
        if (gtid == 0) atomicOr(p.status, STATUS_NO_PAGES);
    }
    if (p.token_offsets) for (int b = gtid; b <= p.batch; b += gsize) p.token_offsets[b] = ok ? s_tok[b] : 0;
    if (tid == 0) {
        bool last = gridDim.x == 1;
        if (!last) {
            int old;
            asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;\n" : "=r"(old) : "l"(p.arrivals) : "memory");
            last = old == (int)gridDim.x - 1;
            if (last) *p.arrivals = 0;
        }
        if (last) *p.num_free_out = ok ? (int)(top - N) : F;
    }
}

// ---- rows of many tokens into the cache ------------------------------------------------------------------
// One warp per KV head and run of four tokens: lanes 0-15 move key rows, lanes 16-31 value rows, eight elements each, so that
// every lane has four loads in flight and one scale for all of them. Bound by memory, every row is read and written once: 65536
// tokens of 8 heads into a bf16 cache 82 us, 6.55 TB/s; into an E4M3 cache, quantised, 62 us at full clock (6.5 TB/s), 72 us under
// the power limit.
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
    unsigned page_bytes, pos_bytes;       // the two strides in bytes where both fit 32 bits, else page_bytes = 0
    const float* k_scale;
    const float* v_scale;
    int* status;
};

// Eight elements' codes: the E4M3 values nearest to x / scale (the quotient in fp32, correctly rounded), saturated at +-448.
// Not a division each: with r the correctly rounded reciprocal of s, q0 = x r and the exact remainder x - q0 s, q0 + r (x - q0 s)
// rounds to x / s (P. Markstein, "Computation of elementary functions on the IBM RISC System/6000 processor", 1990) as
// long as nothing leaves the range. So it is used where s is between 2^-60 and 2^60 and the eight elements are below 2^65 (a
// remainder that underflows then belongs to a quotient below 2^-40, whose code is zero); a division otherwise. The remainder
// is rounded downwards, which changes nothing but the sign of a zero: -0, unlike +0, leaves the sign of q0 as it is. Two
// elements per instruction, and few instructions besides: under load the power limit holds the SM clock at 1.6 GHz and it is the
// instructions that bound this kernel.
__device__ __forceinline__ uint32_t babs_max2(uint32_t a, uint32_t b) {
    uint32_t d;
    asm("max.NaN.xorsign.abs.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __noinline__ uint2 quantise8_unusual(uint4 w, float scale) {
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t half[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float lo = __fdiv_rn(__uint_as_float(in[i] << 16), scale), hi = __fdiv_rn(__uint_as_float(in[i] & 0xffff0000u), scale);
        half[i] = __nv_cvt_float2_to_fp8x2(make_float2(lo, hi), __NV_SATFINITE, __NV_E4M3);
    }
    return make_uint2(half[0] | (half[1] << 16), half[2] | (half[3] << 16));
}
__device__ __forceinline__ uint2 quantise8(uint4 w, float scale, float inv, bool usual) {
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
    uint32_t half[4];
    // the largest magnitude of either half; 2^65 and more, infinities and not-a-numbers have both upper exponent bits set
    const uint32_t most = babs_max2(babs_max2(w.x, w.y), babs_max2(w.z, w.w));
    if (usual && !(most & (most << 1) & 0x40004000u)) {
        const f32pair r2 = pair2(inv, inv), s2 = pair2(-scale, -scale);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32pair x = pair2(__uint_as_float(in[i] << 16), __uint_as_float(in[i] & 0xffff0000u)), q0 = mul2(x, r2);
            const f32pair q = fma2(fma2_rm(q0, s2, x), r2, q0);
            half[i] = __nv_cvt_float2_to_fp8x2(make_float2(half2(q, 0), half2(q, 1)), __NV_SATFINITE, __NV_E4M3);
        }
    } else {
        return quantise8_unusual(w, scale);
    }
    return make_uint2(half[0] | (half[1] << 16), half[2] | (half[3] << 16));
}

constexpr int KW_TOKENS = 4, KW_WARPS = 8;

template <bool KV8>
__global__ void __launch_bounds__(KW_WARPS * 32, 6) kv_write_kernel(const KvWriteParams p) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int piece = lane & 15;
    const bool value = lane >= 16;
    const unsigned w = blockIdx.x * KW_WARPS + warp;         // (the host keeps them below 2^32)
    const unsigned run = w / (unsigned)p.Hkv;
    const int g = (int)(w - run * (unsigned)p.Hkv);
    const long long t0 = (long long)run * KW_TOKENS;
    pdl_wait();
    pdl_trigger();
    if (t0 >= p.num_tokens) return;
    const long long stride = value ? p.v_stride : p.k_stride;
    const uint4* src = reinterpret_cast<const uint4*>((value ? p.v_new : p.k_new) + t0 * stride + (long long)g * HEAD_DIM) + piece;
    uint8_t* const dst = value ? p.v : p.k;
    uint4 row[KW_TOKENS];
    long long slot[KW_TOKENS];
#pragma unroll
    for (int i = 0; i < KW_TOKENS; ++i) {
        slot[i] = -1;
        if (t0 + i < p.num_tokens) {
            slot[i] = read_global(p.slots + t0 + i);
            row[i] = read_global(src + i * (stride >> 3));
        }
    }
    float scale = 1.f, inv = 1.f;
    if constexpr (KV8) {
        const float* sc = value ? p.v_scale : p.k_scale;
        if (sc) { scale = read_global(sc + g); inv = __frcp_rn(scale); }
    }
    const bool usual = scale >= 0x1p-60f && scale <= 0x1p60f;
    constexpr int ESZ = KV8 ? 1 : 2;
    uint8_t* const base = dst + (long long)g * p.stride_head * ESZ + piece * (KV8 ? 8 : 16);
#pragma unroll
    for (int i = 0; i < KW_TOKENS; ++i) {
        const unsigned long long s = (unsigned long long)slot[i];
        if (s >= (unsigned long long)p.num_slots) {
            if (slot[i] != -1 && lane == 0) atomicOr(p.status, STATUS_BAD_INDEX);      // -1: padding
            continue;
        }
        uint8_t* to;
        if (p.paged) {                                      // (page numbers fit 32 bits; so do the strides, mostly)
            const unsigned page = (unsigned)(s / TILE), place = (unsigned)s % TILE;
            if (p.page_bytes) to = base + (unsigned long long)page * p.page_bytes + (unsigned long long)place * p.pos_bytes;
            else to = base + ((long long)page * p.stride_page + (long long)place * p.stride_pos) * ESZ;
        } else {
            to = base + ((long long)(s / (unsigned)p.max_ctx) * p.stride_b + (long long)(s % (unsigned)p.max_ctx) * p.stride_pos) * ESZ;
        }
        if constexpr (KV8) *reinterpret_cast<uint2*>(to) = quantise8(row[i], scale, inv, usual);
        else *reinterpret_cast<uint4*>(to) = row[i];
    }
}

}  // namespace tidal
