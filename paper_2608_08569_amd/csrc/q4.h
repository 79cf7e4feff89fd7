// The 4-bit cache's format, shared by the kernels that write and read it.
//
// A row of d channels is d / 2 bytes of e2m1 codes (0, 1/2, 1, 3/2, 2, 3, 4, 6
// and their negatives; the even channel in a byte's low half) and one scale
// byte per block of 32 channels: byte b scales its block by 2^(b - 127), and
// 255 marks a block that held something not finite and reads as NaN.  This is
// the form gfx950 converts in one instruction per two elements, scale included
// (v_cvt_scalef32_pk_bf16_fp4, at the full VALU rate), and every value is exact
// in bfloat16, so the matrix cores take the cache as it stands.  Codes and
// scales lie in planes of their own ([..][slot][d / 2] and [..][slot][d / 32]):
// rows of 64 and 4 bytes (d = 128) keep 16- and 4-byte accesses aligned, where
// rows of 68 would not.
#pragma once

#include "vz_internal.h"

namespace vz_q4 {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

constexpr int kBlock = 32;  // channels per scale
constexpr int kNoScale = 255;
constexpr int kMinExp = -125, kMaxExp = 125;  // every value a normal float32 and bfloat16

// ---- reading ----
// Two codes (byte SEL of w) as packed bfloat16, low code first.  Only the
// exponent field of the scale operand counts: its sign and mantissa bits may
// hold anything (checked for every scale byte and code).
template <int SEL>
__device__ __forceinline__ uint32_t pair_bf16(uint32_t w, float scale) {
    const bf16x2_t r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL);
    uint32_t u;
    __builtin_memcpy(&u, &r, 4);
    return u;
}
// Byte b of a word of scales as a scale operand: one rotation that brings it to
// the exponent field (rot = scale_rot(b)).
__device__ __forceinline__ int scale_rot(int b) { return 9 + 8 * b; }
__device__ __forceinline__ float scale_of(uint32_t w, int rot) {
    return __uint_as_float(__builtin_amdgcn_alignbit(w, w, rot));
}

// ---- writing ----
// The block's scale from top = max |x| over its channels (INFINITY when one is
// not finite), where the values are x / n: the smallest 2^e with
// max |x| / n <= 7 2^e, within [kMinExp, kMaxExp] (7 rounds to the largest
// code, 6, with no more error than a value between 4 and 6 can have).
// Thresholds are compared with n 2^e times the code borders instead of dividing
// by n, so a mean that lies on a border is recognised whatever n is.
struct Scale {
    int byte;
    double unit;  // n 2^e
};
__device__ __forceinline__ Scale scale_for(double top, double n) {
    Scale s;
    if (!(top < INFINITY)) {
        s.byte = kNoScale;
        s.unit = NAN;  // no code passes a border
        return s;
    }
    // top = a 2^x, 7 n = b 2^y with a, b in [1/2, 1): top / (7 n) = (a / b) 2^(x - y), a / b in (1/2, 2)
    const double n7 = 7.0 * n;
    int e = __builtin_amdgcn_frexp_exp(top) - __builtin_amdgcn_frexp_exp(n7) +
            (__builtin_amdgcn_frexp_mant(top) > __builtin_amdgcn_frexp_mant(n7) ? 1 : 0);
    e = top > 0.0 ? min(max(e, kMinExp), kMaxExp) : kMinExp;
    s.byte = e + 127;
    s.unit = __builtin_ldexp(n, e);
    return s;
}
// The nearest code of x / n: ties to the even code, at most 6; a sign only for x < 0.
__device__ __forceinline__ uint32_t code_of(double x, double unit) {
    const double a = __builtin_fabs(x);
    uint32_t c = a > 0.25 * unit ? 1u : 0u;
    c += a >= 0.75 * unit ? 1u : 0u;
    c += a > 1.25 * unit ? 1u : 0u;
    c += a >= 1.75 * unit ? 1u : 0u;
    c += a > 2.5 * unit ? 1u : 0u;
    c += a >= 3.5 * unit ? 1u : 0u;
    c += a > 5.0 * unit ? 1u : 0u;
    return c | (x < 0.0 ? 8u : 0u);
}

// Byte offsets of the rows of a cache.
template <int D>
struct Rows {
    static constexpr int kCodes = D / 2;       // bytes of a row's codes
    static constexpr int kScales = D / kBlock;  // bytes of a row's scales
};

}  // namespace vz_q4
