// Stochastic rounding to FP8 and its random bits (gfx950).
#pragma once

#include "fp8_encode.hpp"

namespace fp8mm {
namespace {

// ------------------------------------------------------------------------------------------
// Stochastic rounding.  For lo <= |y| < hi adjacent FP8 values, t = (|y| - lo)/(hi - lo),
// T = floor(t * 2^16): the result is hi iff T + r >= 2^16, r = 16 random bits of the element.
// In the bits of y: for results in the normal range T is the 16 bits below the kept mantissa and
// the carry of T + r is added to the truncated code (a mantissa carry bumps the exponent as it
// should); below the smallest normal value the grid is uniform, |y| / step is taken as a fixed-point
// number with 16 fraction bits and r is added to it.
// ------------------------------------------------------------------------------------------
template <int FMT>
__device__ __forceinline__ unsigned encode_sr_bits(float y, unsigned r16)
{
    constexpr int MB = FMT == FP8_E4M3 ? 3 : 2;
    constexpr int BIAS = FMT == FP8_E4M3 ? 7 : 15;
    constexpr unsigned DROP = 23 - MB;
    constexpr unsigned REBIAS = (unsigned)(127 - BIAS) << 23;
    constexpr unsigned MIN_NORMAL = (unsigned)(127 + 1 - BIAS) << 23;
    constexpr unsigned TO_FIXED = (unsigned)(127 + 16 - (1 - BIAS - MB)) << 23;     // 2^16 / step
    constexpr unsigned MAX_BITS = FMT == FP8_E4M3 ? 0x43E00000u : 0x47600000u;
    constexpr unsigned MAX_CODE = FMT == FP8_E4M3 ? 0x7Eu : 0x7Bu;
    constexpr unsigned INF_CODE = FMT == FP8_E4M3 ? 0x7Fu : 0x7Cu;
    const unsigned u = as_u32(y);
    const unsigned a = u & 0x7fffffffu;
    const unsigned sign = (u >> 24) & 0x80u;
    const unsigned T = (a >> (DROP - 16)) & 0xffffu;
    const unsigned normal = ((a - REBIAS) >> DROP) + ((T + r16) >> 16);
    const unsigned fixed = (unsigned)(as_f32(a < MIN_NORMAL ? a : 0u) * as_f32(TO_FIXED));   // truncates
    const unsigned sub = (fixed + r16) >> 16;
    unsigned code = a < MIN_NORMAL ? sub : normal;
    code = a >= MAX_BITS ? MAX_CODE : code;
    code = a >= 0x7f800000u ? INF_CODE : code;
    code = a > 0x7f800000u ? 0x7Fu : code;
    return sign | code;
}

// The same rule through the converter instructions of gfx950 (v_cvt_sr_fp8_f32 / v_cvt_sr_bf8_f32:
// the random operand's upper bits are added below the kept mantissa; with the 16 random bits in
// its upper half and zeros below, the carry is exactly that of T + r; subnormal results included.
// Checked against the integer form on the GPU test inputs and on constructed carry boundaries).
// The instructions do not saturate (a magnitude beyond the largest value comes out as NaN / inf), so
// the value is clamped first; NaN and infinities take the integer form.
// Four scaled values and their four 16-bit fields (r01 = fields 0, 1; r23 = fields 2, 3) -> 4 bytes.
template <int FMT>
__device__ __forceinline__ unsigned encode_sr4(float y0, float y1, float y2, float y3, unsigned r01, unsigned r23)
{
    if (is_special(y0) | is_special(y1) | is_special(y2) | is_special(y3))
        return encode_sr_bits<FMT>(y0, r01 & 0xffffu) | (encode_sr_bits<FMT>(y1, r01 >> 16) << 8) |
               (encode_sr_bits<FMT>(y2, r23 & 0xffffu) << 16) | (encode_sr_bits<FMT>(y3, r23 >> 16) << 24);
    constexpr float FMAX = FMT == FP8_E4M3 ? 448.0f : 57344.0f;
    y0 = __builtin_amdgcn_fmed3f(y0, FMAX, -FMAX); y1 = __builtin_amdgcn_fmed3f(y1, FMAX, -FMAX);
    y2 = __builtin_amdgcn_fmed3f(y2, FMAX, -FMAX); y3 = __builtin_amdgcn_fmed3f(y3, FMAX, -FMAX);
    int w = 0;
    if (FMT == FP8_E4M3) {
        w = __builtin_amdgcn_cvt_sr_fp8_f32(y0, r01 << 16, w, 0);
        w = __builtin_amdgcn_cvt_sr_fp8_f32(y1, r01 & 0xffff0000u, w, 1);
        w = __builtin_amdgcn_cvt_sr_fp8_f32(y2, r23 << 16, w, 2);
        w = __builtin_amdgcn_cvt_sr_fp8_f32(y3, r23 & 0xffff0000u, w, 3);
    } else {
        w = __builtin_amdgcn_cvt_sr_bf8_f32(y0, r01 << 16, w, 0);
        w = __builtin_amdgcn_cvt_sr_bf8_f32(y1, r01 & 0xffff0000u, w, 1);
        w = __builtin_amdgcn_cvt_sr_bf8_f32(y2, r23 << 16, w, 2);
        w = __builtin_amdgcn_cvt_sr_bf8_f32(y3, r23 & 0xffff0000u, w, 3);
    }
    return (unsigned)w;
}

// Philox4x32-10 (Salmon et al., SC 2011): counter (c0, c1, c2, c3), key (k0, k1).
__device__ __forceinline__ void philox4x32_10(unsigned c0, unsigned c1, unsigned c2, unsigned c3, unsigned k0, unsigned k1, unsigned (&out)[4])
{
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const unsigned hi0 = __umulhi(0xD2511F53u, c0), lo0 = 0xD2511F53u * c0;
        const unsigned hi1 = __umulhi(0xCD9E8D57u, c2), lo1 = 0xCD9E8D57u * c2;
        c0 = __builtin_amdgcn_bitop3_b32(hi1, c1, k0, 0x96);        // the three exclusive ored
        c1 = lo1;
        c2 = __builtin_amdgcn_bitop3_b32(hi0, c3, k1, 0x96);
        c3 = lo0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    out[0] = c0; out[1] = c1; out[2] = c2; out[3] = c3;
}

}  // namespace
}  // namespace fp8mm
