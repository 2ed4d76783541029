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
// A half-warp holds a row, eight channels per lane; a warp takes the rows of one token (or a part of them) four pairs at a time, so
// that four 16-byte loads per lane are in flight and the sines are worked out once. Bound by memory where there are many
// tokens, by the chain position -> sine -> row for few.
#pragma once

#include "../../include/tidal.h"
#include "page_kernels.cuh"

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

constexpr int RO_WARPS = 8, RO_UNROLL = 4;

// Eight fp32 numbers' codes, as quantise8 for bf16 ones: x / scale saturated and rounded to E4M3. With a reciprocal the quotient
// may be off by an fp32 step, which is as far off as x is already.
__device__ __noinline__ uint2 quantise8_f32_unusual(const float (&x)[8], float scale) {
    uint32_t half[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        half[i] = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(x[2 * i], scale), __fdiv_rn(x[2 * i + 1], scale)), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(half[0] | (half[1] << 16), half[2] | (half[3] << 16));
}
__device__ __forceinline__ uint2 quantise8_f32(const float (&x)[8], float scale, float inv, bool usual) {
    if (!usual) return quantise8_f32_unusual(x, scale);
    uint32_t half[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        half[i] = __nv_cvt_float2_to_fp8x2(make_float2(x[2 * i] * inv, x[2 * i + 1] * inv), __NV_SATFINITE, __NV_E4M3);
    return make_uint2(half[0] | (half[1] << 16), half[2] | (half[3] << 16));
}

__device__ __forceinline__ void unpack8(const uint4& w, float (&x)[8]) {
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(in[i] << 16); x[2 * i + 1] = __uint_as_float(in[i] & 0xffff0000u); }
}

// Cosines and sines of a lane's eight channels with the norm's weights taken in.
template <bool HALF, bool NORM>
__device__ __forceinline__ void rope_factors(const float (&c)[8], const float (&s)[8], const __nv_bfloat16* weight, int ch, int other, float (&C)[8],
                                             float (&S)[8]) {
#pragma unroll
    for (int j = 0; j < 8; ++j) { C[j] = c[j]; S[j] = s[j]; }
    if constexpr (NORM) {
        if (weight) {
            float w[8], o[8];
            unpack8(read_global(reinterpret_cast<const uint4*>(weight + ch)), w);
            unpack8(read_global(reinterpret_cast<const uint4*>(weight + other)), o);
#pragma unroll
            for (int j = 0; j < 8; ++j) { C[j] *= w[j]; S[j] *= HALF ? o[j] : w[j ^ 1]; }
        }
    }
}

// One row: norm and rotation of a lane's eight channels.
template <bool HALF, bool NORM>
__device__ __forceinline__ void rope_row(const uint4& w, const float (&C)[8], const float (&S)[8], bool turns, int partner, float eps, float (&y)[8]) {
    float x[8], z[8];
    unpack8(w, x);
    if constexpr (HALF) {
        uint4 o;
        o.x = __shfl_sync(0xffffffffu, w.x, partner); o.y = __shfl_sync(0xffffffffu, w.y, partner);
        o.z = __shfl_sync(0xffffffffu, w.z, partner); o.w = __shfl_sync(0xffffffffu, w.w, partner);
        unpack8(o, z);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) z[j] = x[j ^ 1];
    }
    float r = 1.f;
    if constexpr (NORM) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum += x[j] * x[j];
#pragma unroll
        for (int sh = 8; sh; sh >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, sh);
        r = rsqrtf(sum * (1.f / HEAD_DIM) + eps);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        y[j] = x[j] * C[j];
        if (turns) y[j] = fmaf(z[j], S[j], y[j]);           // (the other channels must not meet 0 times infinity)
        if constexpr (NORM) y[j] *= r;
    }
}

template <bool HALF, bool NORM, int MODE>
__global__ void __launch_bounds__(RO_WARPS * 32) rope_kernel(const __grid_constant__ RopeParams p) {
    __shared__ unsigned long long s_step[HEAD_DIM / 2];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, piece = lane & 15, ch = piece * 8, side = lane >> 4;
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
    const bool turns = ch < 2 * half;
    const int partner = HALF && turns ? side * 16 + (ch < half ? piece + half / 8 : piece - half / 8) : lane;
    float c[8], s[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        c[j] = 1.f; s[j] = 0.f;
        if (turns) {
            if (HALF || (j & 1) == 0) {
                const int i = HALF ? (ch < half ? ch : ch - half) + j : (ch + j) / 2;
                const unsigned turn = (unsigned)(((unsigned long long)(unsigned)pos * s_step[i]) >> 32);
                sincospif((float)(int)turn * 0x1p-31f, &s[j], &c[j]);
                c[j] *= p.rope.scale; s[j] *= p.rope.scale;
                if (HALF && ch < half) s[j] = -s[j];
            } else {
                c[j] = c[j - 1]; s[j] = s[j - 1];
                s[j - 1] = -s[j];
            }
        }
    }
    // pairs of rows: queries, keys, then values (which are only moved)
    const int nq = (p.Hq + 1) / 2, nk = (p.Hkv + 1) / 2, all = nq + nk + (MODE != ROPE_BACK ? nk : 0);
    const int lo = (int)((long long)all * part / p.parts), hi = (int)((long long)all * (part + 1) / p.parts);
    float C[8], S[8], y[8];

    if (lo < nq) {
        rope_factors<HALF, NORM>(c, s, p.q_weight, ch, (partner & 15) * 8, C, S);
        const bool norm = NORM && p.q_weight;
        const __nv_bfloat16* src = p.q + (long long)t * p.q_stride + ch;
        __nv_bfloat16* dst = p.q_out + (long long)t * p.qo_stride + ch;
        for (int i = lo; i < min(hi, nq); i += RO_UNROLL) {
            uint4 w[RO_UNROLL];
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                w[u] = make_uint4(0, 0, 0, 0);
                if (i + u < min(hi, nq) && h < p.Hq) w[u] = read_global(reinterpret_cast<const uint4*>(src + h * HEAD_DIM));
            }
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                if (norm) rope_row<HALF, NORM>(w[u], C, S, turns, partner, p.eps, y);
                else rope_row<HALF, false>(w[u], C, S, turns, partner, p.eps, y);
                if (i + u < min(hi, nq) && h < p.Hq)
                    *reinterpret_cast<uint4*>(dst + h * HEAD_DIM) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
            }
        }
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
        rope_factors<HALF, NORM>(c, s, p.k_weight, ch, (partner & 15) * 8, C, S);
        const bool norm = NORM && p.k_weight;
        const __nv_bfloat16* src = p.k + (long long)t * p.k_stride + ch;
        const int end = min(hi, nq + nk) - nq;
        for (int i = max(lo - nq, 0); i < end; i += RO_UNROLL) {
            uint4 w[RO_UNROLL];
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                w[u] = make_uint4(0, 0, 0, 0);
                if (i + u < end && h < p.Hkv) w[u] = read_global(reinterpret_cast<const uint4*>(src + h * HEAD_DIM));
            }
#pragma unroll
            for (int u = 0; u < RO_UNROLL; ++u) {
                const int h = 2 * (i + u) + side;
                if (norm) rope_row<HALF, NORM>(w[u], C, S, turns, partner, p.eps, y);
                else rope_row<HALF, false>(w[u], C, S, turns, partner, p.eps, y);
                if (i + u < end && h < p.Hkv) {
                    if constexpr (MODE == ROPE_CACHE8) {
                        const float scale = p.k_scale ? read_global(p.k_scale + h) : 1.f;
                        *reinterpret_cast<uint2*>(p.ck + row + h * p.stride_head + ch) = quantise8_f32(y, scale, __frcp_rn(scale), scale >= 0x1p-60f && scale <= 0x1p60f);
                    } else {
                        __nv_bfloat16* dst = MODE == ROPE_BACK ? p.k_out + (long long)t * p.ko_stride + h * HEAD_DIM
                                                               : reinterpret_cast<__nv_bfloat16*>(p.ck) + row + h * p.stride_head;
                        *reinterpret_cast<uint4*>(dst + ch) = make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
                    }
                }
            }
        }
    }
    if constexpr (MODE != ROPE_BACK) {
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
