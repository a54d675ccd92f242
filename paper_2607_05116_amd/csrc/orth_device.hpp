// What the two forms of the orthogonalisation share (gfx950): loading U, values
// split over two fp16, and the transpose that mirrors a symmetric product.
#pragma once

#include "mfma_tile.hpp"

namespace cap {
namespace {

// A value as fp16 plus what is left of it in a second fp16, scaled so that what the
// smallest normal values leave is normal too.
constexpr float kLoScale = 2048.0f;

// (The packed bits are opaque to the compiler.  From a product that is rounded to fp16 and
// back it makes two conversions, one of the fp32 product and one that rounds once, and where
// the first is a tie they differ: what was left over was then that of another value.)
__device__ __forceinline__ uint32_t pack_f16x2(float a, float b) {
    typedef _Float16 h2 __attribute__((ext_vector_type(2)));
    const h2 v = {static_cast<_Float16>(a), static_cast<_Float16>(b)};
    uint32_t bits = __builtin_bit_cast(uint32_t, v);
    asm("" : "+v"(bits));
    return bits;
}
__device__ __forceinline__ float f16_to_f32(uint16_t b) { return static_cast<float>(__builtin_bit_cast(_Float16, b)); }
// value e = 0..3 of four packed fp16
__device__ __forceinline__ float f16_at(const u32x2& v, int e) {
    return f16_to_f32(static_cast<uint16_t>(v[e >> 1] >> (16 * (e & 1))));
}
// Split over both, to 22 bits.
__device__ __forceinline__ void split4(const float (&v)[4], u32x2& hi, u32x2& lo) {
    hi = u32x2{pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3])};
    float d[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = (v[e] - f16_at(hi, e)) * kLoScale;
    lo = u32x2{pack_f16x2(d[0], d[1]), pack_f16x2(d[2], d[3])};
}
// Split with rounding toward zero (one instruction for two values): both halves are
// always used, the second takes up what the first leaves, and 21 bits remain.
__device__ __forceinline__ uint32_t pack_f16x2_rtz(float a, float b) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
}
__device__ __forceinline__ void split4_rtz(const float (&v)[4], u32x2& hi, u32x2& lo) {
    hi = u32x2{pack_f16x2_rtz(v[0], v[1]), pack_f16x2_rtz(v[2], v[3])};
    float d[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = __builtin_fmaf(f16_at(hi, e), -kLoScale, v[e] * kLoScale);
    lo = u32x2{pack_f16x2_rtz(d[0], d[1]), pack_f16x2_rtz(d[2], d[3])};
}

// 4 x 4 transpose of 16-bit values within each quad of lanes: lane r holds four
// columns of row r; afterwards lane r holds four rows of column r % 4.
__device__ __forceinline__ u32x2 quad_transpose(const u32x2& v, int lane) {
    const uint32_t p0 = __builtin_amdgcn_mov_dpp(v[0], 0xB1, 0xF, 0xF, true);              // lane ^ 1
    const uint32_t p1 = __builtin_amdgcn_mov_dpp(v[1], 0xB1, 0xF, 0xF, true);
    // even lanes: the low halves of their own and the partner's pair; odd: the high ones
    const uint32_t pick = 0x05040100u ^ ((0u - (lane & 1)) & (0x05040100u ^ 0x03020706u));
    const uint32_t x0 = __builtin_amdgcn_perm(p0, v[0], pick), x1 = __builtin_amdgcn_perm(p1, v[1], pick);
    const uint32_t up = 0u - ((lane >> 1) & 1);
    const uint32_t y = __builtin_amdgcn_mov_dpp(x1 ^ (up & (x0 ^ x1)), 0x4E, 0xF, 0xF, true);   // lane ^ 2
    return u32x2{x0 ^ (up & (x0 ^ y)), y ^ (up & (x1 ^ y))};
}

// Block (i, j), j <= i, of the t-th block on or below the diagonal.
__device__ __forceinline__ void triangle(int t, int& i, int& j) {
    i = static_cast<int>((sqrtf(8.0f * static_cast<float>(t) + 1.0f) - 1.0f) * 0.5f);
    while (i * (i + 1) / 2 > t) --i;
    while ((i + 1) * (i + 2) / 2 <= t) ++i;
    j = t - i * (i + 1) / 2;
}

// The matrix to orthogonalise: U = G, or G + mu M / M with M the new momentum
// (which the first pass writes: M <- mu M + G).
struct Source {
    const void* g;
    float* mom;
    float mu;
    int nesterov;
    int bf16;
};
template <bool BF16>
__device__ __forceinline__ float load_g(const void* g, size_t i) {
    if constexpr (BF16) return bf16_to_f32(static_cast<const uint16_t*>(g)[i]);
    else return static_cast<const float*>(g)[i];
}
// Raw values of four consecutive elements (the gradient's, the momentum's) and U from
// them, apart so that loads can be under way while something else is computed.  vec: 16-byte
// (fp32) and 8-byte (bf16) aligned; step: distance of the elements; n: how many there are.
struct Raw4 {
    f32x4 g, m;
};
template <bool BF16, bool MOM>
__device__ __forceinline__ void load_raw(const Source& s, size_t i, size_t step, int n, bool vec, Raw4& x) {
    x.g = x.m = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (vec) {
        if (n <= 0) return;
        if constexpr (BF16) {
            const u32x2 v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(s.g) + i);
            x.g = f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xFFFF0000u), __uint_as_float(v[1] << 16),
                        __uint_as_float(v[1] & 0xFFFF0000u)};
        } else {
            x.g = *reinterpret_cast<const f32x4*>(static_cast<const float*>(s.g) + i);
        }
        if constexpr (MOM) x.m = *reinterpret_cast<const f32x4*>(s.mom + i);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < n) {
                x.g[e] = load_g<BF16>(s.g, i + e * step);
                if constexpr (MOM) x.m[e] = s.mom[i + e * step];
            }
    }
}
template <bool MOM, bool FIRST>
__device__ __forceinline__ f32x4 finish_u(const Source& s, size_t i, size_t step, int n, bool vec, const Raw4& x) {
    if constexpr (!MOM) return x.g;
    f32x4 m = x.m;
    if constexpr (FIRST) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = __builtin_fmaf(s.mu, m[e], x.g[e]);
        if (vec) {
            if (n > 0) *reinterpret_cast<f32x4*>(s.mom + i) = m;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < n) s.mom[i + e * step] = m[e];
        }
    }
    if (s.nesterov) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = __builtin_fmaf(s.mu, m[e], x.g[e]);
    }
    return m;
}
template <bool BF16, bool MOM, bool FIRST>
__device__ __forceinline__ float load_u(const Source& s, size_t i) {
    const float g = load_g<BF16>(s.g, i);
    if constexpr (!MOM) return g;
    float m = s.mom[i];
    if constexpr (FIRST) {
        m = __builtin_fmaf(s.mu, m, g);
        s.mom[i] = m;
    }
    return s.nesterov ? __builtin_fmaf(s.mu, m, g) : m;
}
// Four consecutive values, 16-byte (fp32) and 8-byte (bf16) aligned.
template <bool BF16, bool MOM, bool FIRST>
__device__ __forceinline__ f32x4 load_u4(const Source& s, size_t i) {
    f32x4 g;
    if constexpr (BF16) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(static_cast<const uint16_t*>(s.g) + i);
        g = f32x4{__uint_as_float(v[0] << 16), __uint_as_float(v[0] & 0xFFFF0000u), __uint_as_float(v[1] << 16),
                  __uint_as_float(v[1] & 0xFFFF0000u)};
    } else {
        g = *reinterpret_cast<const f32x4*>(static_cast<const float*>(s.g) + i);
    }
    if constexpr (!MOM) return g;
    f32x4 m = *reinterpret_cast<const f32x4*>(s.mom + i);
    if constexpr (FIRST) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = __builtin_fmaf(s.mu, m[e], g[e]);
        *reinterpret_cast<f32x4*>(s.mom + i) = m;
    }
    if (s.nesterov) {
#pragma unroll
        for (int e = 0; e < 4; ++e) m[e] = __builtin_fmaf(s.mu, m[e], g[e]);
    }
    return m;
}

// Whether every run of four columns may be loaded as one vector.
inline bool vector_rows(const Source& s, int cols) {
    return cols % 4 == 0 && (reinterpret_cast<uintptr_t>(s.g) & (s.bf16 ? 7 : 15)) == 0 &&
           (reinterpret_cast<uintptr_t>(s.mom) & 15) == 0;
}

}  // namespace

struct StepCoef {
    float v[kMaxOrthSteps][3];
};

size_t gram_form_bytes(int batch, int rows, int cols);
cap_status gram_form_launch(int batch, int rows, int cols, const void* g, bool bf16, float* momentum, float mu,
                            int nesterov, int steps, const StepCoef& coef, float eps, void* out, void* workspace,
                            hipStream_t stream);

}  // namespace cap
