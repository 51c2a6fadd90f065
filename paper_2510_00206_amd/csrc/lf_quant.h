// Numbers held in fewer bits than bf16, with a power of two that they share: the smallest that keeps the largest magnitude in range, so that
// the scale costs no rounding of its own and what is read back is exact in bf16.
//   fp8   e4m3 (up to 448), one power of two for a token's head
//   fp4   e2m1 (0, 0.5, 1, 1.5, 2, 3, 4, 6), one for 32 entries, which lie in four lanes of eight; two codes to a byte, the first in the low half
#pragma once
#include "lf_device.h"

namespace lf {

// The smallest biased exponents: the least code times the power of two is still a normal bf16 (2^-9 of e4m3, 0.5 of e2m1).
constexpr int kLeastFp8 = 127 - 117, kLeastFp4 = 127 - 125;
constexpr int kNanFp4 = 255;                     // a group of codes with a value that is not finite: all of it reads as NaN (e2m1 has no code for one)

__device__ __forceinline__ float exp2_of_biased(uint32_t e) { return __builtin_bit_cast(float, e << 23); }

// x (32 bits) of a 64-bit value, what is left of it kept in the last bit: rounded again, to fewer bits, it gives what the 64-bit value would.
__device__ __forceinline__ float round_to_odd(double x) {
    const float f = (float)x;
    const uint32_t bits = __builtin_bit_cast(uint32_t, f);
    if ((bits & 0x7F800000u) == 0x7F800000u) return f;
    const double gone = __builtin_fabs(x) - (double)__builtin_fabsf(f);
    const uint32_t odd = gone > 0.0 ? bits + 1u : bits - 1u;
    return __builtin_bit_cast(float, gone != 0.0 && !(bits & 1u) ? odd : bits);
}

// Eight entries of a head that lies in LANES lanes: codes, and the biased exponent.  Largest magnitudes come from the bit patterns (integers in the
// order of the values).  What is not finite becomes the format's NaN, and does not count for the exponent.
template <int LANES>
__device__ __forceinline__ u32x2 to_fp8(const float (&x)[8], uint32_t& exponent) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu);
    // (of the wave; without such values they are not looked for entry by entry: 2085 tokens of 8 heads of 128 to the cache 4.75 us, always 5.3)
    const bool odd = __any(top >= 0x7F800000u);
    if (odd) {
        top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t b = __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu;
            top = max(top, b < 0x7F800000u ? b : 0u);
        }
    }
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o));
    const int e = top ? max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u), kLeastFp8) : 127;      // 448 = 1.75 x 2^8
    const float scale = exp2_of_biased(254 - e);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * scale;
    if (odd)
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = (__builtin_bit_cast(uint32_t, x[i]) & 0x7F800000u) == 0x7F800000u ? __builtin_nanf("") : y[i];
    u32x2 code;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        code[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], v, true);
    }
    exponent = (uint32_t)e;
    return code;
}

// Eight entries of a group that lies in four lanes.
__device__ __forceinline__ uint32_t to_fp4(const float (&x)[8], uint32_t& exponent) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7FFFFFFFu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    top = max(top, (uint32_t)__shfl_xor((int)top, 2));
    if (top >= 0x7F800000u) {
        exponent = kNanFp4;
        return 0u;
    }
    const int e = top ? max((int)(top >> 23) - 2 + ((top & 0x7FFFFFu) > 0x400000u), kLeastFp4) : 127;      // 6 = 1.5 x 2^2
    const float scale = exp2_of_biased(254 - e);
    uint32_t code = 0;
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[0] * scale, x[1] * scale, 1.f, 0);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[2] * scale, x[3] * scale, 1.f, 1);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[4] * scale, x[5] * scale, 1.f, 2);
    code = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(code, x[6] * scale, x[7] * scale, 1.f, 3);
    exponent = (uint32_t)e;
    return code;
}

// Eight values of a word of codes, exact: e2m1 times a power of two (255: NaN).
__device__ __forceinline__ bf16x8 from_fp4(uint32_t code, float scale) {
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

}  // namespace lf
