// 8-bit floating point (OCP e4m3: 4 exponent bits, 3 mantissa bits, largest 448, no
// infinity) with a scale for each block of 128 values along a row.
//
// A block's scale is the least power of two with which its largest magnitude fits
// e4m3, at least 2^-126.  e4m3 floats, so a power of two costs no precision against
// amax / 448 (the step of a value relative to it is the same; only values 2^-13 of
// the largest and less lose a bit of their subnormal steps), and dividing by it is
// exact: every value is rounded once, to nearest even, and codes do not depend on
// how a quotient was rounded.
#pragma once

#include <type_traits>

#include "cap_device.hpp"

namespace cap {
namespace {

constexpr uint32_t kF32Inf = 0x7F800000u;

// Magnitude bits of a finite v, 0 for infinities and NaN (they take no part in a
// block's largest value and become NaN codes by themselves).
__device__ __forceinline__ uint32_t finite_magnitude(float v) {
    const uint32_t m = __float_as_uint(v) & 0x7FFFFFFFu;
    return m < kF32Inf ? m : 0u;
}

// Biased exponent of the scale for a block whose largest magnitude has these bits:
// amax = m 2^e with 1 <= m < 2 fits 448 = 1.75 x 2^8 with the scale 2^(e-8) if m <=
// 1.75, and with 2^(e-7) if not; the addition carries into the exponent just then.
__device__ __forceinline__ uint32_t f8_scale_exponent(uint32_t amax_bits) {
    const int e = static_cast<int>((amax_bits + 0x1FFFFFu) >> 23) - 8;
    return static_cast<uint32_t>(e < 1 ? 1 : e);
}
__device__ __forceinline__ float f8_scale(uint32_t exponent) { return __uint_as_float(exponent << 23); }
// 1 / scale, also a power of two (254 - exponent is 6 to 253: a normal number).
__device__ __forceinline__ float f8_inverse(uint32_t exponent) { return __uint_as_float((254u - exponent) << 23); }

// Four values to e4m3 codes, the first in the lowest byte.  Products with `inv` are
// at most 448 for finite values; what is not finite becomes NaN.
__device__ __forceinline__ uint32_t f8_pack4(float a, float b, float c, float d, float inv) {
    auto f = [&](float v) {
        v *= inv;
        return (__float_as_uint(v) & 0x7FFFFFFFu) < kF32Inf ? v : __builtin_nanf("");
    };
    int p = __builtin_amdgcn_cvt_pk_fp8_f32(f(a), f(b), 0, false);
    return static_cast<uint32_t>(__builtin_amdgcn_cvt_pk_fp8_f32(f(c), f(d), p, true));
}

// Largest of a value over the 16 lanes of a DPP row (every lane gets it).
__device__ __forceinline__ uint32_t row16_max(uint32_t v) {
    auto step = [&](auto ctrl) {
        const uint32_t o = static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), ctrl.value, 0xF, 0xF, true));
        v = o > v ? o : v;
    };
    step(std::integral_constant<int, 0xB1>{});     // quad_perm xor 1
    step(std::integral_constant<int, 0x4E>{});     // quad_perm xor 2
    step(std::integral_constant<int, 0x141>{});    // row_half_mirror: 8 lanes
    step(std::integral_constant<int, 0x140>{});    // row_mirror: 16 lanes
    return v;
}

}  // namespace
}  // namespace cap
