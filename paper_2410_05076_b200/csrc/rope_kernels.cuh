// Queries and keys of new tokens on their way to the cache: RMS norm of every head (optional), rotation to the token's position, and
// either back to memory (rope_kernel<..., ROPE_BACK>) or, keys and values, into the cache through a slot map.
//
// Norm: x w / sqrt(mean(x^2) + eps) over a head's 128 channels. Rotation: a pair (a, b) of channels at position p becomes
// (a c - b s, b c + a s) with c, s = scale cos, sin(p f). A row's result is then r (x_j C_j + x'_j S_j) with x' the
// other channel of the pair, r the row's norm and C, S the same for all rows of a token: cosine and sine with the weights (own and the
// other channel's) taken in.
//
// Angles: p f / 2 pi mod 1 in fixed point, p times a 64-bit fraction of a turn, wrapped. The product's upper 32 bits are
// the turn to 2^-32 (p 2^-65 from the fraction's rounding besides), whatever the position; fp32 products would be off by
// p 2^-24 radians, 2^-6 at position 262144. All arithmetic is fp32 and rounded once, to the type that is stored.
//
// A half-warp holds a row. A lane has four pairs of channels (4 l .. and half + 4 l .., or 8 l .. interleaved), so that nothing is
// exchanged but the norm's sums; lanes behind the turning channels hold eight that stay. A warp takes the rows of one token (or a part of them)
// four pairs of rows at a time, and the sines are worked out once. Bound by memory where there are many tokens (16384 normed
// 58 us, 5.8 TB/s; 32768 into an E4M3 cache 135 us, 5.5 TB/s, instructions then nearly as long), by the chain position -> sine -> row for few (64: 2.6 us).
#pragma once

#include "../../include/tidal.h"
#include "page_kernels.cuh"

#include <type_traits>

namespace tidal {

enum { ROPE_BACK = 0, ROPE_CACHE = 1, ROPE_CACHE8 = 2 };

struct RopeParams {
    tidal_rope_t rope;
    const __nv_bfloat16* q;
    const __nv_bfloat16* k;
    const __nv_bfloat16* v;
    long long q_stride, k_stride, v_stride;                  // elements between tokens
    __nv_bfloat16* q_out;
    __nv_bfloat16* k_out;
    long long qo_stride, ko_stride;
    const int* positions;
    const __nv_bfloat16* q_weight;
    const __nv_bfloat16* k_weight;
    float eps;
    int num_tokens, Hq, Hkv;
    int parts;                                               // warps per token
    // the cache (ROPE_CACHE*)
    uint8_t* ck;
    uint8_t* cv;
    const long long* slots;
    long long num_slots;
    int paged, max_ctx;
    long long stride_b, stride_pos, stride_head, stride_page;
    const float* k_scale;
    const float* v_scale;
    int* status;
};

constexpr int RO_WARPS = 8, RO_UNROLL = 4;                          // (rope_norms takes four rows)

// Four fp32 numbers' codes, as quantise8 for bf16 ones (the correctly rounded quotient, saturated, to the nearest code).
__device__ __noinline__ uint32_t quantise4_f32_unusual(float x0, float x1, float x2, float x3, float scale) {
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(x0, scale), __fdiv_rn(x1, scale)), __NV_SATFINITE, __NV_E4M3) |
           ((uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(x2, scale), __fdiv_rn(x3, scale)), __NV_SATFINITE, __NV_E4M3) << 16);
}
__device__ __forceinline__ uint32_t quantise4_f32(f32pair x, f32pair y, float scale, float inv, bool usual) {
    const float most = fmaxf(fmaxf(fabsf(half2(x, 0)), fabsf(half2(x, 1))), fmaxf(fabsf(half2(y, 0)), fabsf(half2(y, 1))));
    if (!usual || !(most < 0x1p65f)) return quantise4_f32_unusual(half2(x, 0), half2(x, 1), half2(y, 0), half2(y, 1), scale);
    const f32pair r2 = pair2(inv, inv), s2 = pair2(-scale, -scale);
    const f32pair p0 = mul2(x, r2), p1 = mul2(y, r2);
    const f32pair a = fma2(fma2_rm(p0, s2, x), r2, p0), b = fma2(fma2_rm(p1, s2, y), r2, p1);
    return (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(half2(a, 0), half2(a, 1)), __NV_SATFINITE, __NV_E4M3) |
           ((uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(half2(b, 0), half2(b, 1)), __NV_SATFINITE, __NV_E4M3) << 16);
}

// A lane's four pairs of channels (a[0], b[0]) .. (a[3], b[3]) as two pairs of numbers each.
struct RopeRow { f32pair a[2], b[2]; };
struct RopeFactors { f32pair ca[2], cb[2], sa[2], sb[2]; };    // a' = a ca - b sb, b' = b cb + a sa

// Words of eight channels: HALF keeps a's in x, y and b's in z, w; interleaved, a's are the lower halves.
template <bool HALF>
__device__ __forceinline__ RopeRow rope_unpack(const uint4& w) {
    auto lo = [](uint32_t x) { return __uint_as_float(x << 16); };
    auto hi = [](uint32_t x) { return __uint_as_float(x & 0xffff0000u); };
    RopeRow r;
    if constexpr (HALF) {
        r.a[0] = pair2(lo(w.x), hi(w.x)); r.a[1] = pair2(lo(w.y), hi(w.y));
        r.b[0] = pair2(lo(w.z), hi(w.z)); r.b[1] = pair2(lo(w.w), hi(w.w));
    } else {
        r.a[0] = pair2(lo(w.x), lo(w.y)); r.a[1] = pair2(lo(w.z), lo(w.w));
        r.b[0] = pair2(hi(w.x), hi(w.y)); r.b[1] = pair2(hi(w.z), hi(w.w));
    }
    return r;
}
template <bool HALF>
__device__ __forceinline__ uint4 rope_pack(const RopeRow& r) {
    if constexpr (HALF)
        return make_uint4(pack_bf16(half2(r.a[0], 0), half2(r.a[0], 1)), pack_bf16(half2(r.a[1], 0), half2(r.a[1], 1)),
                          pack_bf16(half2(r.b[0], 0), half2(r.b[0], 1)), pack_bf16(half2(r.b[1], 0), half2(r.b[1], 1)));
    return make_uint4(pack_bf16(half2(r.a[0], 0), half2(r.b[0], 0)), pack_bf16(half2(r.a[0], 1), half2(r.b[0], 1)),
                      pack_bf16(half2(r.a[1], 0), half2(r.b[1], 0)), pack_bf16(half2(r.a[1], 1), half2(r.b[1], 1)));
}
// A lane's words of a row of 16-bit numbers: two pieces of eight bytes at channels c0 and c1, or one of sixteen at c0.
template <bool HALF>
__device__ __forceinline__ uint4 rope_load(const __nv_bfloat16* row, int c0, int c1) {
    if constexpr (!HALF) return read_global(reinterpret_cast<const uint4*>(row + c0));
    const uint2 a = read_global(reinterpret_cast<const uint2*>(row + c0)), b = read_global(reinterpret_cast<const uint2*>(row + c1));
    return make_uint4(a.x, a.y, b.x, b.y);
}
template <bool HALF>
__device__ __forceinline__ void rope_store(__nv_bfloat16* row, int c0, int c1, const uint4& w) {
    if constexpr (!HALF) {
        *reinterpret_cast<uint4*>(row + c0) = w;
    } else {
        *reinterpret_cast<uint2*>(row + c0) = make_uint2(w.x, w.y);
        *reinterpret_cast<uint2*>(row + c1) = make_uint2(w.z, w.w);
    }
}

// Cosines and sines with the norm's weights taken in.
template <bool HALF>
__device__ __forceinline__ RopeFactors rope_factors(const f32pair (&c)[2], const f32pair (&s)[2], const __nv_bfloat16* weight, int c0, int c1) {
    RopeFactors f;
    RopeRow w;
    w.a[0] = w.a[1] = w.b[0] = w.b[1] = pair2(1.f, 1.f);
    if (weight) w = rope_unpack<HALF>(rope_load<HALF>(weight, c0, c1));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        f.ca[i] = mul2(c[i], w.a[i]); f.cb[i] = mul2(c[i], w.b[i]);
        f.sa[i] = mul2(s[i], w.a[i]); f.sb[i] = mul2(mul2(s[i], pair2(-1.f, -1.f)), w.b[i]);
    }
    return f;
}

// One row's rotation (and the norm's weights).
__device__ __forceinline__ RopeRow rope_row(const RopeRow& x, const RopeFactors& f, bool turns) {
    RopeRow y;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        y.a[i] = mul2(x.a[i], f.ca[i]);
        y.b[i] = mul2(x.b[i], f.cb[i]);
        if (turns) {                                        // (channels that stay must not meet 0 times infinity)
            y.a[i] = fma2(x.b[i], f.sb[i], y.a[i]);
            y.b[i] = fma2(x.a[i], f.sa[i], y.b[i]);
        }
    }
    return y;
}
__device__ __forceinline__ float rope_squares(const RopeRow& x) {
    const f32pair q = fma2(x.b[1], x.b[1], fma2(x.b[0], x.b[0], fma2(x.a[1], x.a[1], mul2(x.a[0], x.a[0]))));
    return half2(q, 0) + half2(q, 1);
}
// 1 / sqrt(mean square + eps) of four rows, from each lane's part of their sums of squares: the sixteen lanes of a row end up with a quarter of the
// rows each, so that the four sums take nine exchanges and one root.
__device__ __forceinline__ void rope_norms(float (&v)[4], int lane, float eps) {
    const bool b = lane & 8, d = lane & 4;
    const float x0 = (b ? v[2] : v[0]) + __shfl_xor_sync(0xffffffffu, b ? v[0] : v[2], 8);
    const float x1 = (b ? v[3] : v[1]) + __shfl_xor_sync(0xffffffffu, b ? v[1] : v[3], 8);
    float x = (d ? x1 : x0) + __shfl_xor_sync(0xffffffffu, d ? x0 : x1, 4);
    x += __shfl_xor_sync(0xffffffffu, x, 2);
    x += __shfl_xor_sync(0xffffffffu, x, 1);
    x = x * (1.f / HEAD_DIM) + eps;
    float r = rsqrtf(x);
    const float e = fmaf(-x * r, r, 1.f);                   // one step of Newton's method: to about an fp32 step
    if (e > -1.f && e < 1.f) r = fmaf(0.5f * r, e, r);       // (not for 0 and infinity)
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = __shfl_sync(0xffffffffu, r, (lane & 16) + (u >> 1) * 8 + (u & 1) * 4);
}

template <bool HALF, bool NORM, int MODE>
__global__ void __launch_bounds__(RO_WARPS * 32, 4) rope_kernel(const __grid_constant__ RopeParams p) {
    __shared__ unsigned long long s_step[HEAD_DIM / 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane & 15, side = lane >> 4;
    if (threadIdx.x < HEAD_DIM / 2) s_step[threadIdx.x] = p.rope.step[threadIdx.x];
    __syncthreads();
    const long long unit = (long long)blockIdx.x * RO_WARPS + warp;
    const int t = (int)(unit / p.parts), part = (int)(unit - (long long)t * p.parts);
    pdl_wait();
    pdl_trigger();
    if (t >= p.num_tokens) return;
    const int pos = read_global(p.positions + t);
    if (pos < 0) return;                                    // padding

    const int half = p.rope.rotary_dim / 2;
    const bool turns = 4 * piece < half;
    const int c0 = HALF && turns ? 4 * piece : 8 * piece, c1 = HALF && turns ? half + 4 * piece : 8 * piece + 4;
    f32pair c[2], s[2];
    {
        float cs[4], sn[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            cs[j] = 1.f; sn[j] = 0.f;
            if (turns) {
                // the turn in quarters, so that what is left, at most an eighth either way, keeps its 24 bits
                const unsigned turn = (unsigned)(((unsigned long long)(unsigned)pos * s_step[4 * piece + j]) >> 32);
                const unsigned quarter = (turn + 0x20000000u) >> 30;
                float x, y;
                sincospif((float)(int)(turn - (quarter << 30)) * 0x1p-31f, &y, &x);
                const float u = quarter & 1 ? y : x, v = quarter & 1 ? x : y;
                cs[j] = ((quarter + 1) & 2 ? -u : u) * p.rope.scale;
                sn[j] = (quarter & 2 ? -v : v) * p.rope.scale;
            }
        }
        c[0] = pair2(cs[0], cs[1]); c[1] = pair2(cs[2], cs[3]);
        s[0] = pair2(sn[0], sn[1]); s[1] = pair2(sn[2], sn[3]);
    }
    // pairs of rows: queries, keys, then values (which are only moved)
    const int nq = (p.Hq + 1) / 2, nk = (p.Hkv + 1) / 2, all = nq + nk + (MODE != ROPE_BACK ? nk : 0);
    const int lo = (int)((long long)all * part / p.parts), hi = (int)((long long)all * (part + 1) / p.parts);

    // Pairs of rows i0 .. end - 1 of `heads` rows; what becomes of a row is the caller's
    auto rows = [&](const __nv_bfloat16* src, int i0, int end, int heads, const __nv_bfloat16* weight, auto store) {
        const RopeFactors f = rope_factors<HALF>(c, s, NORM ? weight : nullptr, c0, c1);
        const bool norm = NORM && weight;
        auto group = [&](int i, auto whole) {               // (whole: all four pairs are there)
            uint4 w[RO_UNROLL];
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                if (decltype(whole)::value || (i + u < end && h < heads)) w[u] = rope_load<HALF>(src + h * HEAD_DIM, c0, c1);
                else w[u] = make_uint4(0, 0, 0, 0);
            }
            float r[RO_UNROLL];
            if (norm) {
#pragma unroll
                for (int u = 0; u < RO_UNROLL; ++u) r[u] = rope_squares(rope_unpack<HALF>(w[u]));
                rope_norms(r, lane, p.eps);
            }
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                RopeRow y = rope_row(rope_unpack<HALF>(w[u]), f, turns);
                if (norm) {
                    const f32pair r2 = pair2(r[u], r[u]);
#pragma unroll
                    for (int j = 0; j < 2; ++j) { y.a[j] = mul2(y.a[j], r2); y.b[j] = mul2(y.b[j], r2); }
                }
                if (decltype(whole)::value || (i + u < end && h < heads)) store(h, y);
            }
        };
        int i = i0;
        for (; i + RO_UNROLL <= end && 2 * (i + RO_UNROLL) <= heads; i += RO_UNROLL) group(i, std::true_type());
        if (i < end) group(i, std::false_type());
    };
    if (lo < nq) {
        __nv_bfloat16* dst = p.q_out + (long long)t * p.qo_stride;
        rows(p.q + (long long)t * p.q_stride, lo, min(hi, nq), p.Hq, p.q_weight,
             [&](int h, const RopeRow& y) { rope_store<HALF>(dst + h * HEAD_DIM, c0, c1, rope_pack<HALF>(y)); });
    }
    if (hi <= nq) return;

    long long row = 0;
    if constexpr (MODE != ROPE_BACK) {
        const long long slot = read_global(p.slots + t);
        if ((unsigned long long)slot >= (unsigned long long)p.num_slots) {
            if (slot != -1 && lane == 0) atomicOr(p.status, STATUS_BAD_INDEX);
            return;
        }
        row = p.paged ? (slot / TILE) * p.stride_page + (slot % TILE) * p.stride_pos : (slot / p.max_ctx) * p.stride_b + (slot % p.max_ctx) * p.stride_pos;
    }
    if (max(lo, nq) < min(hi, nq + nk)) {
        rows(p.k + (long long)t * p.k_stride, max(lo - nq, 0), min(hi, nq + nk) - nq, p.Hkv, p.k_weight, [&](int h, const RopeRow& y) {
            if constexpr (MODE == ROPE_CACHE8) {
                const float scale = p.k_scale ? read_global(p.k_scale + h) : 1.f, inv = __frcp_rn(scale);
                const bool usual = scale >= 0x1p-60f && scale <= 0x1p60f;
                uint8_t* const to = p.ck + row + h * p.stride_head;
                const uint32_t a = quantise4_f32(y.a[0], y.a[1], scale, inv, usual), b = quantise4_f32(y.b[0], y.b[1], scale, inv, usual);
                if constexpr (HALF) {
                    *reinterpret_cast<uint32_t*>(to + c0) = a;
                    *reinterpret_cast<uint32_t*>(to + c1) = b;
                } else {                                    // codes of a's and b's in turn
                    *reinterpret_cast<uint2*>(to + c0) = make_uint2(__byte_perm(a, b, 0x5140), __byte_perm(a, b, 0x7362));
                }
            } else {
                __nv_bfloat16* dst = MODE == ROPE_BACK ? p.k_out + (long long)t * p.ko_stride + h * HEAD_DIM
                                                       : reinterpret_cast<__nv_bfloat16*>(p.ck) + row + h * p.stride_head;
                rope_store<HALF>(dst, c0, c1, rope_pack<HALF>(y));
            }
        });
    }
    if constexpr (MODE != ROPE_BACK) {
        const int ch = 8 * piece;
        const __nv_bfloat16* src = p.v + (long long)t * p.v_stride + ch;
        const int end = hi - nq - nk;
        for (int i = max(lo - nq - nk, 0); i < end; i += RO_UNROLL) {
            uint4 w[RO_UNROLL];
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                if (i + u < end && h < p.Hkv) w[u] = read_global(reinterpret_cast<const uint4*>(src + h * HEAD_DIM));
            }
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                if (i + u < end && h < p.Hkv) {
                    if constexpr (MODE == ROPE_CACHE8) {
                        const float scale = p.v_scale ? read_global(p.v_scale + h) : 1.f;
                        *reinterpret_cast<uint2*>(p.cv + row + h * p.stride_head + ch) = quantise8(w[u], scale, __frcp_rn(scale), scale >= 0x1p-60f && scale <= 0x1p60f);
                    } else {
                        *reinterpret_cast<uint4*>(reinterpret_cast<__nv_bfloat16*>(p.cv) + row + h * p.stride_head + ch) = w[u];
                    }
                }
            }
        }
    }
}

}  // namespace tidal
