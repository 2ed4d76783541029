// Attention over listed blocks of 16 positions (see block_kernels.cuh).
#pragma once

#include "block_kernels.cuh"

namespace tidal {

// ---- attention over listed blocks ------------------------------------------------------------------------------
// Item = (sequence, KV head), or (sequence, query head) where every query head has its own list. A thread-block cluster
// serves an item: its warps take the listed blocks in turn, each with a private cp.async ring (no CTA barrier on the
// streaming path). At the end every warp pushes its (max, sum, O) into the shared memory of the CTAs that finish the
// output, a slice each; one cluster barrier later they add up what they received. So the kernel needs no scratch
// memory, no counters and no second launch.
// The matrix instructions have positions as rows and the group's heads as columns: S^T = K Q^T, O^T += V^T P^T, so K and V are read
// once per KV head. The softmax weights enter the second product as a sum of 16-bit numbers, three of bf16 over a bf16 cache (2^-24
// relative), two of fp16 over an 8-bit one (2^-22): the path waits for memory, and the further matrix instructions cost it
// 1 to 2 % (131072 positions, 256 blocks per KV head: 8.8 us) where one bf16 would leave 2^-8.
struct BlockAttnParams {
    BlockCache c;
    const __nv_bfloat16* q;
    void* out;
    int out_bf16;
    const int* idx;
    const int* idx_count;
    int m, Hi;
    int over_ring;                                          // the inbox lies over the rings (see ba_over_ring)
    float scale_log2;
    const float* k_scale;
    const float* v_scale;
};

// Weights that are split into fp16 numbers carry a factor 2^14 (which the sums share, so it cancels): the second number of a weight
// below 2^-13 would otherwise fall below fp16's normal range.
constexpr float W16_SHIFT = 14.f;

template <int N>
struct IntConst { static constexpr int value = N; };

// Softmax state of a warp: running maxima (base 2) and sums of this lane's heads 2 tig, 2 tig + 1; o[t][0] their O^T elements in the first
// fragment row of run t, o[t][1] in the second, as pairs of fp32. A block's products go into fresh accumulators that are then added:
// the matrix instruction cuts what it adds to an accumulator, always downwards, which over the 32 blocks of a warp
// left 1.1e-6 relative instead of 0.3e-6.
struct BlockAcc {
    float m[2], l[2];
    f32pair o[8][2];
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
        const f32pair a = pair2(a0, a1);
#pragma unroll
        for (int t = 0; t < 8; ++t) { acc.o[t][0] = mul2(acc.o[t][0], a); acc.o[t][1] = mul2(acc.o[t][1], a); }
        acc.m[0] = g0;
        acc.m[1] = g1;
    }
}

// Softmax weights of one block from its scaled logits t (rows gid, gid + 8; this lane's two heads).
template <bool W16>
__device__ __forceinline__ void block_weights(BlockAcc& acc, const float (&s)[4], float scale_log2, int nvalid, int gid, float (&w)[4]) {
    const bool v0 = gid < nvalid, v1 = gid + 8 < nvalid;
    const float t0 = v0 ? s[0] * scale_log2 : -INFINITY, t1 = v0 ? s[1] * scale_log2 : -INFINITY;
    const float t2 = v1 ? s[2] * scale_log2 : -INFINITY, t3 = v1 ? s[3] * scale_log2 : -INFINITY;
    raise_max(acc, fmaxf(t0, t2), fmaxf(t1, t3));
    const float shift = W16 ? W16_SHIFT : 0.f;
    const float m0 = ((acc.m[0] == -INFINITY) ? 0.f : acc.m[0]) - shift, m1 = ((acc.m[1] == -INFINITY) ? 0.f : acc.m[1]) - shift;
    w[0] = fast_exp2(t0 - m0); w[1] = fast_exp2(t1 - m1);
    w[2] = fast_exp2(t2 - m0); w[3] = fast_exp2(t3 - m1);
    acc.l[0] += w[0] + w[2];
    acc.l[1] += w[1] + w[3];
}

__device__ __forceinline__ void add_block(BlockAcc& acc, const float (&d)[8][4]) {
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        acc.o[t][0] = add2(acc.o[t][0], pair2(d[t][0], d[t][1]));
        acc.o[t][1] = add2(acc.o[t][1], pair2(d[t][2], d[t][3]));
    }
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
    block_weights<false>(acc, s, scale_log2, nvalid, gid, w);
    // the weights as h + l + r, each rounded to bf16
    auto low = [](uint32_t v) { return __uint_as_float(v << 16); };
    auto high = [](uint32_t v) { return __uint_as_float(v & 0xffff0000u); };
    const uint32_t h0 = pack_bf16(w[0], w[1]), h1 = pack_bf16(w[2], w[3]);
    w[0] -= low(h0); w[1] -= high(h0); w[2] -= low(h1); w[3] -= high(h1);
    const uint32_t l0 = pack_bf16(w[0], w[1]), l1 = pack_bf16(w[2], w[3]);
    const uint32_t r0 = pack_bf16(w[0] - low(l0), w[1] - high(l0)), r1 = pack_bf16(w[2] - low(l1), w[3] - high(l1));
    const uint32_t ph0 = movmatrix_trans(h0), ph1 = movmatrix_trans(h1), pl0 = movmatrix_trans(l0), pl1 = movmatrix_trans(l1);
    const uint32_t pr0 = movmatrix_trans(r0), pr1 = movmatrix_trans(r1);
    const int rr = lane & 7, mb = (lane >> 3) & 1;
    const uint32_t vl = vs + (rr + ((lane >> 4) << 3)) * 256 + ((rr ^ mb) << 4);
    // all of the value fragments first, then the products part by part: three in a row into one accumulator would wait for
    // each other
    uint32_t a[8][4];
#pragma unroll
    for (int t = 0; t < 8; ++t) ldmatrix_x4_trans(vl ^ (t << 5), a[t]);
    float d[8][4];
#pragma unroll
    for (int t = 0; t < 8; ++t) { d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.f; mma_bf16_16816(d[t], a[t][0], a[t][1], a[t][2], a[t][3], pr0, pr1); }
#pragma unroll
    for (int t = 0; t < 8; ++t) mma_bf16_16816(d[t], a[t][0], a[t][1], a[t][2], a[t][3], pl0, pl1);
#pragma unroll
    for (int t = 0; t < 8; ++t) mma_bf16_16816(d[t], a[t][0], a[t][1], a[t][2], a[t][3], ph0, ph1);
    add_block(acc, d);
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
    block_weights<true>(acc, s, scale_log2, nvalid, gid, w);
    const uint32_t h0 = pack_f16(w[0], w[1]), h1 = pack_f16(w[2], w[3]);
    const uint32_t l0 = pack_f16(w[0] - f16_lo(h0), w[1] - f16_hi(h0)), l1 = pack_f16(w[2] - f16_lo(h1), w[3] - f16_hi(h1));
    const uint32_t ph0 = movmatrix_trans(h0), ph1 = movmatrix_trans(h1), pl0 = movmatrix_trans(l0), pl1 = movmatrix_trans(l1);
    const int rr = lane & 7, mi = lane >> 3;
    const uint32_t vbase = vs + (rr + ((mi >> 1) << 3)) * ROW_BYTES8;
    uint32_t a[8][4];                                       // as in consume_block: fragments first, then products part by part
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        uint32_t m[4];
        ldmatrix_x4_trans(vbase + ((uint32_t)((2 * u + (mi & 1)) ^ rr) << 4), m);
        e4m3x4_to_f16x2x2(__byte_perm(m[0], 0, 0x3120), a[2 * u][0], a[2 * u][1]);
        e4m3x4_to_f16x2x2(__byte_perm(m[2], 0, 0x3120), a[2 * u][2], a[2 * u][3]);
        e4m3x4_to_f16x2x2(__byte_perm(m[1], 0, 0x3120), a[2 * u + 1][0], a[2 * u + 1][1]);
        e4m3x4_to_f16x2x2(__byte_perm(m[3], 0, 0x3120), a[2 * u + 1][2], a[2 * u + 1][3]);
    }
    float d[8][4];
#pragma unroll
    for (int t = 0; t < 8; ++t) { d[t][0] = d[t][1] = d[t][2] = d[t][3] = 0.f; mma_f16_16816(d[t], a[t][0], a[t][1], a[t][2], a[t][3], pl0, pl1); }
#pragma unroll
    for (int t = 0; t < 8; ++t) mma_f16_16816(d[t], a[t][0], a[t][1], a[t][2], a[t][3], ph0, ph1);
    add_block(acc, d);
}

constexpr int BA_STAGES = 3, BA_STAGES8 = 6;                // the same bytes in flight
// Shapes: eight warps with an SM to themselves, or smaller CTAs that share one, eight warps in all (rule in tidal_api.cu).
constexpr int BA_MAX_CLUSTER = 16;
constexpr int BA_MAX_LIST = 1 << 30;                        // entries of a list: 32 bits hold an entry number and a round of all warps besides

template <bool KV8>
constexpr size_t ba_ring(int warps) { return (size_t)warps * (KV8 ? BA_STAGES8 * STAGE_BYTES8 : BA_STAGES * STAGE_BYTES); }
// Elements of an output slice: whole runs of 16 of a row, so that a fragment goes to one CTA.
__host__ __device__ constexpr int ba_slice(int ncols, int cluster) { return (ncols * (HEAD_DIM / 16) + cluster - 1) / cluster * 16; }
// What the warps of a cluster push into one CTA: a row of O (padded so that four sources' rows lie in different banks) and
// (max, sum) per column each. It lies behind
// the rings, or over them where there is no room behind (and in a cluster of one).
__host__ __device__ constexpr size_t ba_inbox(int ncols, int cluster, int warps) {
    return (size_t)cluster * warps * ((size_t)(ba_slice(ncols, cluster) + 8) * sizeof(float) + ncols * sizeof(float2)) + 8;
}
constexpr size_t BA_SLACK = 256;                            // ring slots start on 256-byte boundaries
constexpr size_t ba_smem_most(int warps) { return (size_t)(warps == 8 ? 227 : warps == 4 ? 113 : warps == 2 ? 56 : 28) * 1024; }
template <bool KV8>
constexpr bool ba_over_ring(int ncols, int cluster, int warps) {
    return cluster == 1 || ba_ring<KV8>(warps) + ba_inbox(ncols, cluster, warps) + BA_SLACK > ba_smem_most(warps);
}
template <bool KV8>
constexpr size_t ba_smem(int ncols, int cluster, int warps) {
    return ba_ring<KV8>(warps) + (ba_over_ring<KV8>(ncols, cluster, warps) ? 0 : ba_inbox(ncols, cluster, warps)) + BA_SLACK;
}

template <bool KV8, int NW>
__global__ void __launch_bounds__(NW * 32, 8 / NW) block_attn_kernel(const BlockAttnParams p) {
    constexpr int STAGES = KV8 ? BA_STAGES8 : BA_STAGES, SLOT = KV8 ? STAGE_BYTES8 : STAGE_BYTES;
    const BlockCache& c = p.c;
    extern __shared__ __align__(128) uint8_t smem_raw[];
    uint8_t* smem = smem_raw + ((BA_SLACK - (smem_u32(smem_raw) & (BA_SLACK - 1))) & (BA_SLACK - 1));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    int rank, size;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank));
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
    if (size > 1) cluster_arrive();                         // waited for before the first write to another CTA
    const bool per_qhead = p.Hi == c.Hq;
    const int IY = per_qhead ? c.Hq : c.Hkv;
    const int item = blockIdx.x / size, b = item / IY, y = item - b * IY;
    const int g = per_qhead ? y / c.G : y;
    const int head0 = per_qhead ? y : g * c.G, ncols = per_qhead ? 1 : c.G;
    const int* row = p.idx + ((long long)b * p.Hi + (per_qhead ? y : (p.Hi == c.Hkv ? g : 0))) * p.m;
    const int stride = size * NW, me = rank * NW + warp;
    pdl_wait();
    pdl_trigger();

    // Blocks of this warp: list entries me + i * stride; lane l keeps what entry l of a run of 32 needs. (A run's entries are
    // read one run ahead, the first along with the lengths: the list has m of them whatever the count says.)
    const long long e0 = (long long)me + (long long)lane * stride;
    int next_blk = e0 < p.m ? read_global(row + e0) : -1;
    const int n = cached_len(c, b);
    const int cnt = p.idx_count ? min(p.idx_count[b], p.m) : p.m;
    const int count = cnt > me ? (cnt - me + stride - 1) / stride : 0;
    long long my_off = 0;
    int my_rows = 0;
    const uint32_t ring = smem_u32(smem) + warp * STAGES * SLOT;
    const uint64_t policy = l2_evict_first_policy();
    const int c16 = lane & 15, rhalf = lane >> 4;           // bf16: piece c16 of rows rhalf + 2 i
    const int p8 = lane & 7, r8 = lane >> 3;                // codes: piece p8 of rows r8 + 4 i
    // Copies block `i` of this warp into a slot; returns its valid rows.
    auto issue = [&](int i, uint32_t slot) -> int {
        if ((i & 31) == 0) {
            const long long e = e0 + (long long)i * stride;
            const int blk = e < cnt ? next_blk : -1;
            const long long ahead = e + 32ll * stride;
            next_blk = ahead < p.m ? read_global(row + ahead) : -1;
            my_rows = 0;
            my_off = 0;
            if (blk < -1 || (blk >= 0 && (long long)blk * TILE >= n)) atomicOr(c.status, STATUS_BAD_INDEX);
            else if (blk >= 0) {
                my_rows = min(TILE, n - blk * TILE);
                my_off = (long long)g * c.stride_head;
                if (c.paged) {
                    const int page = read_global(c.page_table + (long long)b * c.max_pages + blk);
                    if ((unsigned)page < (unsigned)c.num_pages) my_off += (long long)page * c.stride_page;
                    else { my_rows = 0; my_off = 0; atomicOr(c.status, STATUS_BAD_PAGE); }
                } else {
                    my_off += (long long)b * c.stride_b + (long long)blk * TILE * c.stride_pos;
                }
            }
            __syncwarp();
        }
        const int rows = __shfl_sync(0xffffffffu, my_rows, i & 31);
        const long long off = __shfl_sync(0xffffffffu, my_off, i & 31);
        if (rows > 0) {
            if constexpr (KV8) {
                const long long src = off + r8 * c.stride_pos + p8 * 16;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int r = r8 + 4 * j;
                    const bool on = r < rows;
                    const long long o = on ? src + 4 * j * c.stride_pos : 0;
                    cp_async16_hint(slot + r * ROW_BYTES8 + ((p8 ^ ((r & 1) << 2)) << 4), c.k + o, on ? 16 : 0, policy);
                    cp_async16_hint(slot + TILE_BYTES8 + r * ROW_BYTES8 + ((p8 ^ (r & 7)) << 4), c.v + o, on ? 16 : 0, policy);
                }
            } else {
                const long long src = 2 * (off + rhalf * c.stride_pos + c16 * 8);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int r = rhalf + 2 * j;
                    const bool on = r < rows;
                    const long long o = on ? src + 4 * j * c.stride_pos : 0;
                    const uint32_t d = slot + r * 256 + ((c16 ^ (r & 7)) << 4);
                    cp_async16_hint(d, c.k + o, on ? 16 : 0, policy);
                    cp_async16_hint(d + TILE_BYTES, c.v + o, on ? 16 : 0, policy);
                }
            }
        }
        return rows;
    };

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
                const uint4 t0 = read_global(qp + 2 * pc), t1 = read_global(qp + 2 * pc + 1);
                const uint32_t w[8] = {t0.x, t0.y, t0.z, t0.w, t1.x, t1.y, t1.z, t1.w};
#pragma unroll
                for (int i = 0; i < 8; ++i) qf8[sl][i] = on ? bf16x2_to_f16x2(w[i]) : 0u;
            }
        } else {
            const uint32_t* qw = reinterpret_cast<const uint32_t*>(qrow);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t w0 = read_global(qw + 8 * j + tig), w1 = read_global(qw + 8 * j + 4 + tig);
                qf[j][0] = on ? w0 : 0u;
                qf[j][1] = on ? w1 : 0u;
            }
        }
    }
    const float scale_log2 = p.scale_log2 * ((KV8 && p.k_scale) ? read_global(p.k_scale + g) : 1.f);
    const float vscale = (KV8 && p.v_scale) ? read_global(p.v_scale + g) : 1.f;
    BlockAcc acc;
    acc.m[0] = acc.m[1] = -INFINITY;
    acc.l[0] = acc.l[1] = 0.f;
#pragma unroll
    for (int t = 0; t < 8; ++t) acc.o[t][0] = acc.o[t][1] = 0ull;

    // One rolled loop, which first fills the ring and then refills it one block behind: unrolled over the slots the code does
    // not fit the instruction cache (a line fetched costs as much as the instructions in it twice over). The valid
    // rows of the blocks in flight are kept in one word, five bits a slot.
    static_assert(STAGES * 5 <= 32, "rows in flight");
    uint32_t flying = 0;
    uint32_t in_slot = ring, out_slot = ring;
#pragma unroll 1
    for (int it = 1 - STAGES; it < count; ++it) {
        const int i = it + STAGES - 1;
        __syncwarp();                                       // every lane is done with the slot that is refilled
        uint32_t rows = 0;
        if (i < count) rows = issue(i, in_slot);
        cp_async_commit();
        in_slot = in_slot == ring + (STAGES - 1) * SLOT ? ring : in_slot + SLOT;
        const uint32_t nvalid = (flying >> (5 * (STAGES - 2))) & 31u;       // of the block issued STAGES - 1 rounds ago
        flying = (flying << 5) | rows;
        if (it < 0) continue;
        cp_async_wait<STAGES - 1>();
        __syncwarp();
        if (nvalid > 0) {
            if constexpr (KV8) consume_block8(out_slot, out_slot + TILE_BYTES8, qf8, acc, scale_log2, (int)nvalid, lane);
            else consume_block(out_slot, out_slot + TILE_BYTES, qf, acc, scale_log2, (int)nvalid, lane);
        }
        out_slot = out_slot == ring + (STAGES - 1) * SLOT ? ring : out_slot + SLOT;
    }
    cp_async_wait<0>();
#pragma unroll
    for (int sh = 4; sh <= 16; sh <<= 1) {
        acc.l[0] += __shfl_xor_sync(0xffffffffu, acc.l[0], sh);
        acc.l[1] += __shfl_xor_sync(0xffffffffu, acc.l[1], sh);
    }

    // ---- every warp's part to the CTAs that finish the output ------------------------------------------------------
    // CTA r finishes elements r * slice .. of the item's rows [ncols][128]. Inbox: [warp of the cluster][slice + 8] of O, then
    // [warp][column] (max, sum).
    const int slice = ba_slice(ncols, size), pitch = slice + 8, sources = size * NW;
    if (size > 1) cluster_wait();                           // every CTA of the cluster has started
    if (p.over_ring) {                                      // ... and every warp that writes there has drained its ring
        if (size == 1) __syncthreads();
        else { cluster_arrive(); cluster_wait(); }
    }
    const int behind = p.over_ring ? 0 : NW * STAGES * SLOT;
    const uint32_t box = smem_u32(smem) + behind;
    const uint32_t box_ml = (box + 4 * (uint32_t)(sources * pitch) + 7) & ~7u;
    {
        const int runs = slice / 16, magic = (65536 + runs - 1) / runs;       // run q belongs to CTA q / runs, q < 64
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int col = 2 * tig + u;
            if (col < ncols) {
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    const int q = col * 8 + t, dst = (q * magic) >> 16;
                    const uint32_t at = cluster_addr(box + 4 * (uint32_t)(me * pitch + (q - dst * runs) * 16), dst);
                    // fragment rows: gid and gid + 8 of the run; over an 8-bit cache 2 gid and 2 gid + 1
                    const int d0 = KV8 ? 2 * gid : gid, d1 = KV8 ? d0 + 1 : d0 + 8;
                    asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(at + 4 * d0), "f"(half2(acc.o[t][0], u) * vscale) : "memory");
                    asm volatile("st.shared::cluster.f32 [%0], %1;\n" ::"r"(at + 4 * d1), "f"(half2(acc.o[t][1], u) * vscale) : "memory");
                }
            }
        }
        for (int col = 0; col < ncols; ++col) {
            const float m = __shfl_sync(0xffffffffu, (col & 1) ? acc.m[1] : acc.m[0], col >> 1);
            const float l = __shfl_sync(0xffffffffu, (col & 1) ? acc.l[1] : acc.l[0], col >> 1);
            if (lane < size) {
                const uint32_t at = cluster_addr(box_ml + 8 * (uint32_t)(me * ncols + col), lane);
                asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};\n" ::"r"(at), "f"(m), "f"(l) : "memory");
            }
        }
    }
    if (size == 1) __syncthreads();
    else { cluster_arrive(); cluster_wait(); }              // (nobody touches another CTA's memory from here on)
    const uint8_t* base = smem + behind;
    const float* in_o = reinterpret_cast<const float*>(base);
    const float2* in_ml = reinterpret_cast<const float2*>(base + (box_ml - box));
    // An element each for TPE threads, which share the sources; each works out the sources' factors for itself: a shared table of
    // them would be a longer chain of shuffles and another barrier.
    auto finish = [&](auto tpe) {
        constexpr int TPE = decltype(tpe)::value;
        const int sub = threadIdx.x & (TPE - 1);
#pragma unroll 1
        for (int i = threadIdx.x / TPE; i < slice && rank * slice + i < ncols * HEAD_DIM; i += NW * 32 / TPE) {      // (the same for TPE lanes)
            const int e = rank * slice + i;
            const float2* ml = in_ml + (e >> 7);
            const unsigned mask = ((1u << TPE) - 1u) << (lane & ~(TPE - 1));
            float M = -INFINITY, L = 0.f, O = 0.f;
#pragma unroll 4
            for (int w = sub; w < sources; w += TPE) M = fmaxf(M, ml[w * ncols].x);
#pragma unroll
            for (int sh = 1; sh < TPE; sh <<= 1) M = fmaxf(M, __shfl_xor_sync(mask, M, sh));
            // (a warp whose logits are all NaN has no maximum but a sum that is NaN: it goes in with factor 0)
#pragma unroll 4
            for (int w = sub; w < sources; w += TPE) {
                const float2 v = ml[w * ncols];
                const float f = (v.x == -INFINITY) ? 0.f : fast_exp2(v.x - M);
                L = fmaf(v.y, f, L);
                O = fmaf(in_o[w * pitch + i], f, O);
            }
#pragma unroll
            for (int sh = 1; sh < TPE; sh <<= 1) {
                L += __shfl_xor_sync(mask, L, sh);
                O += __shfl_xor_sync(mask, O, sh);
            }
            if (sub == 0) {
                const float r = (L != 0.f) ? O / L : 0.f;
                const long long at = ((long long)b * c.Hq + head0) * HEAD_DIM + e;
                if (p.out_bf16) reinterpret_cast<__nv_bfloat16*>(p.out)[at] = __float2bfloat16_rn(r);
                else reinterpret_cast<float*>(p.out)[at] = r;
            }
        }
    };
    if (sources <= 8) finish(IntConst<1>());
    else finish(IntConst<4>());
}

}  // namespace tidal
