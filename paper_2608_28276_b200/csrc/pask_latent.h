// RETAIN-LOW of latent caches: quantising a group of 32 values, reading it back, and where its codes lie in a page
// (pask_layout.h).  Shared by the append kernels, the read-back and decode attention.
#pragma once
#include <cuda_bf16.h>

#include "pask_layout.h"

namespace pask {
namespace {

constexpr float kMinScale = 1.17549435e-38f;      // 2^-126: a smaller scale is stored as zero

// levels on each side of zero; the offset that makes codes unsigned; the largest scale: bf16(levels * scale) has to be finite,
// and the next bf16 number above 36.25 * 2^120 (2 * 2^120 for 127 levels) times the levels rounds to 2^128
template <int BITS> struct Codes;
template <> struct Codes<2> { static constexpr int kLevels = 1, kOffset = 2; static constexpr float kMaxScale = 3.3895314e38f; };
template <> struct Codes<4> { static constexpr int kLevels = 7, kOffset = 8; static constexpr float kMaxScale = 36.25f * 0x1p120f; };
template <> struct Codes<8> { static constexpr int kLevels = 127, kOffset = 128; static constexpr float kMaxScale = 2.0f * 0x1p120f; };

__device__ __forceinline__ float latent_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float latent_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The 32 values of one group (16 bf16 pairs) -> BITS packed words and the scale's bf16 bits.
// scale = bf16(amax / levels), at most kMaxScale (zero unless a normal number), code = x / scale to the nearest integer, ties to
// even, at most `levels` in magnitude.
// x and scale have 8 significant bits each, so a quotient that is no tie is at least 2^-9 away from one: rounding
// x * (1 / scale) to a multiple of 2^-10 (the first addition, 1.5 * 2^13) removes the error of the reciprocal and leaves
// exact ties exact; the second addition (up to 1.5 * 2^23 + offset) rounds to the integer, ties to even.  |x / scale| is
// at most levels * (1 + 2^-8), which rounds to levels; only under kMaxScale can it be more: 255 / 36.25 rounds to 7 all the same,
// 255 / 2 to 128, so that with eight-bit codes limit_group moves those values to 254 first (rarely: a limit on every code
// cost 2 us of a bulk append's 76).
struct GroupScale { float inv; uint32_t bits; };
template <int BITS>
__device__ __forceinline__ GroupScale group_scale(float amax) {
    float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(amax, (float)Codes<BITS>::kLevels)));
    s = s >= kMinScale ? fminf(s, Codes<BITS>::kMaxScale) : 0.0f;
    return {s == 0.0f ? 0.0f : __fdiv_rn(1.0f, s), __float_as_uint(s) >> 16};
}
template <int BITS>
__device__ __forceinline__ uint32_t code_of(float x, float inv) {
    const float grid = __fmaf_rn(x, inv, 12288.0f);
    return __float_as_uint(__fadd_rn(grid, 12582912.0f - 12288.0f + (float)Codes<BITS>::kOffset)) & ((1u << BITS) - 1u);
}
template <int BITS, int N>
__device__ __forceinline__ void limit_group(float amax, uint32_t (&xs)[N]) {
    constexpr float kTop = Codes<8>::kLevels * Codes<8>::kMaxScale;
    if (BITS == 8 && amax > kTop) {
        const __nv_bfloat162 top = __float2bfloat162_rn(kTop), bottom = __float2bfloat162_rn(-kTop);
#pragma unroll
        for (int e = 0; e < N; e++) {
            const __nv_bfloat162 x = __hmin2(__hmax2(*reinterpret_cast<const __nv_bfloat162 *>(&xs[e]), bottom), top);
            xs[e] = *reinterpret_cast<const uint32_t *>(&x);
        }
    }
}
template <int BITS>
__device__ __forceinline__ uint32_t quantise_group(uint32_t (&xs)[16], uint32_t (&words)[BITS]) {
    __nv_bfloat162 m2 = __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&xs[0]));
#pragma unroll
    for (int e = 1; e < 16; e++) m2 = __hmax2(m2, __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&xs[e])));
    const uint32_t m = *reinterpret_cast<const uint32_t *>(&m2);
    const float amax = fmaxf(latent_lo(m), latent_hi(m));
    const GroupScale sc = group_scale<BITS>(amax);
    limit_group<BITS>(amax, xs);
    uint32_t code[32];
#pragma unroll
    for (int e = 0; e < 32; e++) code[e] = code_of<BITS>((e & 1) ? latent_hi(xs[e >> 1]) : latent_lo(xs[e >> 1]), sc.inv);
#pragma unroll
    for (int j = 0; j < BITS; j++) words[j] = 0;
#pragma unroll
    for (int e = 0; e < 32; e++) {
        if (BITS == 4) words[e >> 3] |= code[e] << (4 * ((e & 7) >> 1) + 16 * (e & 1));
        else if (BITS == 2) words[e >> 4] |= code[e] << ((e & 14) + 16 * (e & 1));
        else words[e >> 2] |= code[e] << (8 * (e & 3));
    }
    return sc.bits;
}

// BITS packed words of a group and its scale -> 16 bf16 pairs: bf16((code - offset) * scale), one rounding each.
// Two- and four-bit codes: 0x4300 | code is the bf16 number 128 + code, the difference is exact and the product rounded
// once.  Eight-bit codes go through fp32 (0x4B000000 | code = 2^23 + code; the product of 7 and 8 bits is exact there).
template <int BITS>
__device__ __forceinline__ void dequantise_group(const uint32_t (&words)[BITS], uint32_t scale_bits, uint32_t (&xs)[16]) {
    constexpr int kOffset = Codes<BITS>::kOffset;
    if (BITS == 8) {
        const float s = __uint_as_float(scale_bits << 16);
#pragma unroll
        for (int p = 0; p < 16; p++) {
            const uint32_t w = words[(p >> 1) < BITS ? p >> 1 : 0];
            const float a = (__uint_as_float(__byte_perm(w, 0x4B000000u, (p & 1) ? 0x7442 : 0x7440)) - (8388608.0f + kOffset)) * s;
            const float b = (__uint_as_float(__byte_perm(w, 0x4B000000u, (p & 1) ? 0x7443 : 0x7441)) - (8388608.0f + kOffset)) * s;
            const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
            xs[p] = *reinterpret_cast<const uint32_t *>(&r);
        }
        return;
    }
    const __nv_bfloat162 s2 = __bfloat162bfloat162(__ushort_as_bfloat16((unsigned short)scale_bits));
    const __nv_bfloat162 off = __float2bfloat162_rn(128.0f + kOffset);
#pragma unroll
    for (int p = 0; p < 16; p++) {
        const uint32_t w = BITS == 4 ? words[(p >> 2) < BITS ? p >> 2 : 0] >> (4 * (p & 3)) : words[(p >> 3) < BITS ? p >> 3 : 0] >> (2 * (p & 7));
        const uint32_t v = (w & (BITS == 4 ? 0x000F000Fu : 0x00030003u)) | 0x43004300u;
        const __nv_bfloat162 r = __hmul2(__hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&v), off), s2);
        xs[p] = *reinterpret_cast<const uint32_t *>(&r);
    }
}

// the packed codes of (token, group) of a LOW page
template <int BITS>
__device__ __forceinline__ void load_codes(const uint8_t *page, int tau, int group, uint32_t (&words)[BITS]) {
    const uint8_t *p = page + latent_code_off(tau, group, BITS);
    if (BITS == 2) {
        const uint2 a = *reinterpret_cast<const uint2 *>(p);
        words[0] = a.x; words[1] = a.y;
    } else {
#pragma unroll
        for (int h = 0; h < BITS / 4; h++) {
            const uint4 a = *reinterpret_cast<const uint4 *>(p + h * kPageTokens * 16);
            words[(4 * h) % BITS] = a.x; words[(4 * h + 1) % BITS] = a.y; words[(4 * h + 2) % BITS] = a.z; words[(4 * h + 3) % BITS] = a.w;
        }
    }
}
template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t *page, int tau, int group, const uint32_t (&words)[BITS], uint32_t scale_bits) {
    uint8_t *p = page + latent_code_off(tau, group, BITS);
    if (BITS == 2) {
        *reinterpret_cast<uint2 *>(p) = make_uint2(words[0], words[1]);
    } else {
#pragma unroll
        for (int h = 0; h < BITS / 4; h++)
            *reinterpret_cast<uint4 *>(p + h * kPageTokens * 16) =
                make_uint4(words[(4 * h) % BITS], words[(4 * h + 1) % BITS], words[(4 * h + 2) % BITS], words[(4 * h + 3) % BITS]);
    }
    *reinterpret_cast<uint16_t *>(page + latent_scale_off(tau, group, BITS)) = (uint16_t)scale_bits;
}

// The same from one 16-byte chunk (8 values) a lane: the four lanes of a group are adjacent and call together, with the whole
// warp.  Lanes without `write` only lend their chunk to the group's amax.
template <int BITS>
__device__ __forceinline__ void store_chunk(uint8_t *page, int tau, int chunk, const uint4 x, bool write) {
    uint32_t xs[4] = {x.x, x.y, x.z, x.w};
    float amax = 0.0f;
#pragma unroll
    for (int e = 0; e < 4; e++) amax = fmaxf(amax, fmaxf(fabsf(latent_lo(xs[e])), fabsf(latent_hi(xs[e]))));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 1));
    amax = fmaxf(amax, __shfl_xor_sync(0xffffffffu, amax, 2));
    const GroupScale sc = group_scale<BITS>(amax);
    limit_group<BITS>(amax, xs);
    uint32_t code[8];
#pragma unroll
    for (int e = 0; e < 8; e++) code[e] = code_of<BITS>((e & 1) ? latent_hi(xs[e >> 1]) : latent_lo(xs[e >> 1]), sc.inv);
    if (!write) return;
    const int group = chunk >> 2, q = chunk & 3;
    uint8_t *p = page + latent_code_off(tau, group, BITS);
    if (BITS == 4) {
        uint32_t w = 0;
#pragma unroll
        for (int e = 0; e < 8; e++) w |= code[e] << (4 * (e >> 1) + 16 * (e & 1));
        reinterpret_cast<uint32_t *>(p)[q] = w;
    } else if (BITS == 2) {                        // half of a word of 16 values: a byte of its even dims, a byte of its odd dims
        p += 4 * (q >> 1) + (q & 1);
        p[0] = (uint8_t)(code[0] | code[2] << 2 | code[4] << 4 | code[6] << 6);
        p[2] = (uint8_t)(code[1] | code[3] << 2 | code[5] << 4 | code[7] << 6);
    } else {
        *reinterpret_cast<uint2 *>(p + (q >> 1) * kPageTokens * 16 + (q & 1) * 8) =
            make_uint2(code[0] | code[1] << 8 | code[2] << 16 | code[3] << 24, code[4] | code[5] << 8 | code[6] << 16 | code[7] << 24);
    }
    if (q == 0) *reinterpret_cast<uint16_t *>(page + latent_scale_off(tau, group, BITS)) = (uint16_t)sc.bits;
}

// zeros in place of what row tau of a page holds; thread `tid` of `threads`
__device__ __forceinline__ void clear_high_row(uint8_t *page, int tau, int tid, int threads) {
    for (int ch = tid; ch < kLatentChunks; ch += threads) *reinterpret_cast<uint4 *>(page + latent_chunk_off(tau, ch)) = make_uint4(0, 0, 0, 0);
}
__device__ __forceinline__ void clear_low_row(uint8_t *page, int tau, int bits, int tid, int threads) {
    for (int g = tid; g < kLatentGroups; g += threads) {
        uint8_t *p = page + latent_code_off(tau, g, bits);
        if (bits == 2) *reinterpret_cast<uint2 *>(p) = make_uint2(0, 0);
        else *reinterpret_cast<uint4 *>(p) = make_uint4(0, 0, 0, 0);
        if (bits == 8) *reinterpret_cast<uint4 *>(p + kPageTokens * 16) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint16_t *>(page + latent_scale_off(tau, g, bits)) = 0;
    }
}

}  // namespace
}  // namespace pask
