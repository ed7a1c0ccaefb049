// The quantizer of one group of 64 binary16 values in eight consecutive lanes (Sec. 3.2), shared by the flat and the paged
// kernels of codec.hip and by the head preparation of head_append.hip.
#pragma once
#include "q4_device.h"

namespace q4kv {
namespace {

#pragma clang fp contract(off)

// fl(h + a) in binary32 for the low / the high binary16 half h of a word: the mixed-precision fused multiply-add
// h * 1.0 + a converts and adds in one instruction (the product is exact, so the one rounding is that of the sum)
__device__ __forceinline__ float half_lo_plus(uint32_t pair, float a)
{
    float d;
    asm("v_fma_mix_f32 %0, %1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(d) : "v"(pair), "v"(a));
    return d;
}
__device__ __forceinline__ float half_hi_plus(uint32_t pair, float a)
{
    float d;
    asm("v_fma_mix_f32 %0, %1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(d) : "v"(pair), "v"(a));
    return d;
}

// min over the 8 lanes of an octet of both halves of a packed binary16 pair: two quad permutes and a mirror
// inside each half row, on the vector ALU's data-parallel-primitive lanes (every lane has a source lane, so the
// previous value of the destination is never used)
__device__ __forceinline__ uint32_t octet_pk_min(uint32_t v)
{
    v = pk_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xB1, 0xF, 0xF, true));  // quad_perm [1,0,3,2]
    v = pk_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4E, 0xF, 0xF, true));  // quad_perm [2,3,0,1]
    v = pk_min(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xF, 0xF, true)); // row_half_mirror
    return v;
}

// Quantize the 8 elements held by this lane; the 8 lanes of an octet form one group.
// Returns the packed word; *scale_bits / *bias_bits are the group's stored parameters: binary16, or bfloat16 when
// BF.  The codes are taken against the stored parameters; a bfloat16 bias is in general not the minimum itself, so
// quotients may fall below 0 or above 15 and are clamped.
template <bool BF>
__device__ __forceinline__ uint32_t quantize_octet(uint4 raw, int lane_in_octet, uint16_t *scale_bits,
                                                   uint16_t *bias_bits)
{
    const uint32_t wds[4] = {raw.x, raw.y, raw.z, raw.w};
    uint16_t xb[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        xb[2 * i] = (uint16_t)(wds[i] & 0xffffu);
        xb[2 * i + 1] = (uint16_t)(wds[i] >> 16);
    }
    // min and max of the group in packed binary16 (exact: the inputs are binary16), carried together as
    // (min, -max) so that one packed minimum per exchange serves both
    const uint32_t lo2 = pk_min(pk_min(wds[0], wds[1]), pk_min(wds[2], wds[3]));
    const uint32_t hi2 = pk_max(pk_max(wds[0], wds[1]), pk_max(wds[2], wds[3]));
    const half2_t l2 = bits_to_half2(lo2), h2 = bits_to_half2(hi2);
    half2_t mm = {l2.x < l2.y ? l2.x : l2.y, -(h2.x > h2.y ? h2.x : h2.y)};
    mm = bits_to_half2(octet_pk_min(half2_to_bits(mm)));
    const float mn = (float)mm.x, mx = -(float)mm.y;
    // The stored bias is the bit pattern of the first minimal element.  Only a zero minimum has two
    // encodings; then the sign of the first zero in the group decides.
    uint16_t bb = float_to_half_bits(mn);
    if (mn == 0.0f) {
        uint32_t key = 0xffffffffu; // (position << 1) | sign of the first zero seen by this lane
#pragma unroll
        for (int i = 7; i >= 0; --i)
            if ((xb[i] & 0x7fffu) == 0) key = ((uint32_t)(lane_in_octet * 8 + i) << 1) | (uint32_t)(xb[i] >> 15);
#pragma unroll
        for (int off = 4; off >= 1; off >>= 1) key = min(key, (uint32_t)__shfl_xor((int)key, off, 8));
        bb = (key & 1u) ? 0x8000u : 0x0000u;
    }
    if (BF && mn != 0.0f) bb = float_to_bf16_bits(mn); // +-0 has the same bits in both types
    const float b = BF ? bf16_bits_to_float(bb) : mn;  // what a decoder adds back
    // scale = fl((max - min) / 15), the correctly rounded binary32 quotient, without the division sequence: with
    // c = fl(1/15), q0 = fl(r * c), e = fma(-15, q0, r) and q = fma(e, c, q0), q equals fl(r / 15) for every
    // binary32 r in [2^-24, 2^17] (checked value by value on the host); r = max - min of finite binary16 values
    // is 0 or lies in that range
    const float r = mx - mn, q0 = r * (1.0f / 15.0f);
    float scale32 = __builtin_fmaf(__builtin_fmaf(-15.0f, q0, r), 1.0f / 15.0f, q0);
    asm("" : "+v"(scale32)); // the binary32 value itself is rounded next: keeps that rounding a step of its own
    const uint16_t sb = BF ? float_to_bf16_bits(scale32) : float_to_half_bits(scale32);
    const float s = param_bits_to_float<BF>(sb);
    uint32_t word = 0;
    if (s != 0.0f) {
        // code = clamp(rint(fl(d / s)), 0, 15) with a correctly rounded binary32 division.  The division is the
        // expensive part, so the quotient is first approximated as t = d * rcp(s): rcp is within 1 ulp and d / s < 32
        // here (d <= max - min, and s is (max - min) / 15 rounded to binary16, at worst halved when it is a binary16
        // subnormal), so |t - fl(d / s)| <= 32 * (2^-23 + 2^-24 + 2^-24) = 2^-17.  rint(t) can differ from
        // rint(fl(d / s)) only if a half-integer lies within that distance of t; such octets (about one element in
        // 2^15, and exact ties) look closer, and divide where that does not settle it.  v_cvt_pk_u8_f32 rounds to nearest
        // even and saturates at 0 (checked on the device); quotients reach 15.5 only where they are divided and clamped.
        // With bfloat16 parameters the bias may lie above the minimum or far below it (|d / s| is then unbounded):
        // groups whose quotients leave [-0.4, 15.4] take the careful path as well.
        const float inv = __builtin_amdgcn_rcpf(s);
        float d[8], t[8];
        const float minus_b = -b;
        // the upper clamp only matters when the stored scale was rounded down a lot (a binary16 subnormal); then too
        // the lane takes the careful path
        bool careful = (mx - b) * inv >= 15.4f;
        if (BF) careful |= (mn - b) * inv <= -0.4f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            d[i] = (i & 1) ? half_hi_plus(wds[i / 2], minus_b) : half_lo_plus(wds[i / 2], minus_b); // fl(x - b)
            t[i] = d[i] * inv;
            careful |= fabsf(__builtin_amdgcn_fractf(t[i]) - 0.5f) <= 0x1p-16f;
        }
        if (careful) {
            // Most of these are exact ties: inputs and parameters of few bits, with bfloat16 parameters or inputs in nearly every
            // wave.  One Newton step brings t within 2^-21 of d / s (half an ulp below 16, and an error of 2^-17 times inv's 2^-22); so
            // where t is more than 2^-17 from a half-integer fl(d / s) rounds to the same integer, and where t s = d without a
            // remainder (one fused operation, zero only if exact) t is the quotient.  The rest is divided.  9,000 rows of 16 128-wide
            // heads, four layers, with bfloat16 parameters 66 -> 51 us, with bfloat16 inputs 58 -> 51, with both 70 -> 56.
            bool divide = (mx - b) * inv >= 15.4f || (BF && (mn - b) * inv <= -0.4f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[i] = __builtin_fmaf(__builtin_fmaf(-t[i], s, d[i]), inv, t[i]);
                divide |= fabsf(__builtin_amdgcn_fractf(t[i]) - 0.5f) <= 0x1p-17f && __builtin_fmaf(-t[i], s, d[i]) != 0.0f;
            }
            if (divide) {
#pragma unroll
                for (int i = 0; i < 8; ++i) t[i] = fminf(BF ? fmaxf(d[i] / s, 0.0f) : d[i] / s, 15.0f);
            }
        }
        uint32_t even = 0, odd = 0; // codes 0,2,4,6 and 1,3,5,7 as bytes
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            even = __builtin_amdgcn_cvt_pk_u8_f32(t[2 * i], i, even);
            odd = __builtin_amdgcn_cvt_pk_u8_f32(t[2 * i + 1], i, odd);
        }
        word = even | (odd << 4);
    }
    *scale_bits = sb;
    *bias_bits = bb;
    return word;
}

} // namespace
} // namespace q4kv
