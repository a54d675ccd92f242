// Gradient of the router logits through the gates of the routing by scores (Eq. 1): of the
// quotient w = scale s / (sum of the kept s) or of w = scale s, and of the scores.
//
// It writes a row of E values a token and reads as many (the logits of an unnormalised
// softmax, the gradient that it adds), so memory bounds it.
#pragma clang fp contract(off)

#include <hip/hip_runtime.h>
#include <math.h>

#include <type_traits>

#include "cap_device.hpp"

namespace cap {
namespace {

struct ScoreGradArgs {
    const float* logits;
    const int32_t* idx;
    const uint8_t* keep;
    const float* w;
    const float* d_w;
    const float* d_add;
    void* out;
    int T, E, k, sigmoid, normalise;
    float inv_scale;             // 1 / scale in two factors, inv_scale 2^-scale_exponent: of the least scales it is infinite
    int scale_exponent;
};

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(uint16_t* p, float v) {
    // round to nearest even, once
    *p = static_cast<uint16_t>(pack_bf16x2_rne(v, v));
}

// A wave takes eight tokens: first their slots, one a lane, whose gradients it puts in place in
// rows in LDS; then the rows, L lanes (four experts each) a row, whose loads were under way
// meanwhile.  VEC: rows of whole aligned vectors.  One token a wave took 19.4 us for 32,768
// tokens of 256 experts with d_add and a bf16 result (its chain of loads by itself), this
// 12.1 us: 4.5 TB/s, where a large copy reaches 4.85.
template <int L, typename OUT, bool VEC>
__global__ __launch_bounds__(256) void route_scores_grad_kernel(const ScoreGradArgs a) {
    constexpr int kRounds = L / 8, kRows = 64 / L;       // kRounds times kRows rows
    __shared__ __align__(16) float rows[4][8][4 * L];
    __shared__ float totals[4][8];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long long t0 = (static_cast<long long>(blockIdx.x) * 4 + wave) * 8;
    if (t0 >= a.T) return;
    const bool full = !a.sigmoid && !a.normalise;        // the softmax's other experts have a gradient too
    const int e0 = 4 * (lane & (L - 1));                 // the lane's experts in the rows

    // rows' loads
    auto row_of = [&](int r) {
        const long long t = t0 + r * kRows + lane / L;
        return static_cast<size_t>(t < a.T ? t : a.T - 1) * a.E;
    };
    auto load4 = [&](const float* p, float (&v)[4], float none) {
        if constexpr (VEC) {
            const f32x4 q = *reinterpret_cast<const f32x4*>(p + (e0 < a.E ? e0 : 0));
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = e0 < a.E ? q[i] : none;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = e0 + i < a.E ? p[e0 + i] : none;
        }
    };
    float add[kRounds][4], x[kRounds][4];
    if (a.d_add) {
#pragma unroll
        for (int r = 0; r < kRounds; ++r) load4(a.d_add + row_of(r), add[r], 0.0f);
    } else {
#pragma unroll
        for (int r = 0; r < kRounds; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) add[r][i] = 0.0f;
    }
    if (full) {
#pragma unroll
        for (int r = 0; r < kRounds; ++r) load4(a.logits + row_of(r), x[r], -INFINITY);
    }

    // slots: lane 8 n + j has slot j of token t0 + n
    float g = 0.0f, wk = 0.0f, one_less = 1.0f;
    int e = -1;
    {
        const long long t = t0 + (lane >> 3);
        const int j = lane & 7;
        if (t < a.T && j < a.k) {
            const size_t at = static_cast<size_t>(t) * a.k + j;
            const int ei = a.idx[at];
            if ((!a.keep || a.keep[at]) && ei >= 0 && ei < a.E) {
                e = ei;
                wk = a.w[at];
                g = wk * a.d_w[at];
                if (a.sigmoid) one_less = 1.0f / (1.0f + expf(a.logits[static_cast<size_t>(t) * a.E + ei]));   // 1 - s
            }
        }
    }
    float total = g;
#pragma unroll
    for (int d = 1; d < 8; d *= 2) total += __shfl_xor(total, d);
    const float slot = (a.normalise ? g - wk * __builtin_ldexpf(total * a.inv_scale, -a.scale_exponent) : g) * one_less;
    float(*const mine)[4 * L] = rows[wave];
    const f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < kRounds; ++r) *reinterpret_cast<f32x4*>(&mine[r * kRows + lane / L][e0]) = zero;
    __builtin_amdgcn_wave_barrier();                     // a wave's LDS accesses stay in order
    if (e >= 0) mine[lane >> 3][e] = slot;
    // (0 where no slot is kept: the token may hold anything)
    if ((lane & 7) == 0) totals[wave][lane >> 3] = total;
    __builtin_amdgcn_wave_barrier();

#pragma unroll
    for (int r = 0; r < kRounds; ++r) {
        const int n = r * kRows + lane / L;
        f32x4 d = *reinterpret_cast<const f32x4*>(&mine[n][e0]);
        if (full) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[r][i] = fabsf(x[r][i]) < INFINITY ? x[r][i] : -INFINITY;     // not finite: off
                top = fmaxf(top, x[r][i]);
            }
#pragma unroll
            for (int s = 1; s < L; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
            top = top > -INFINITY ? top : 0.0f;
            float p[4], sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = expf(x[r][i] - top);
                sum += p[i];
            }
#pragma unroll
            for (int s = 1; s < L; s *= 2) sum += __shfl_xor(sum, s);
            const float f = sum > 0.0f ? totals[wave][n] / sum : 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] -= f * p[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] += add[r][i];
        if (t0 + n >= a.T || e0 >= a.E) continue;
        OUT* const out = static_cast<OUT*>(a.out) + row_of(r) + e0;
        if constexpr (VEC) {
            if constexpr (std::is_same<OUT, float>::value) *reinterpret_cast<f32x4*>(out) = d;
            else *reinterpret_cast<u32x2*>(out) = u32x2{pack_bf16x2_rne(d[0], d[1]), pack_bf16x2_rne(d[2], d[3])};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (e0 + i < a.E) store_value(out + i, d[i]);
        }
    }
}

template <typename OUT>
void launch_grad(const ScoreGradArgs& a, hipStream_t st) {
    auto aligned = [](const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; };
    const bool vec = a.E % 4 == 0 && aligned(a.logits, 16) && aligned(a.d_add, 16) && aligned(a.out, 4 * sizeof(OUT));
    auto go = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        const int blocks = (a.T + 31) / 32;
        if (vec) route_scores_grad_kernel<L, OUT, true><<<blocks, 256, 0, st>>>(a);
        else route_scores_grad_kernel<L, OUT, false><<<blocks, 256, 0, st>>>(a);
    };
    if (a.E <= 32) go(std::integral_constant<int, 8>{});
    else if (a.E <= 64) go(std::integral_constant<int, 16>{});
    else if (a.E <= 128) go(std::integral_constant<int, 32>{});
    else go(std::integral_constant<int, 64>{});
}

}  // namespace

cap_status route_scores_grad_launch(int T, int k, int E, const float* logits, const int32_t* idx, const uint8_t* keep,
                                    const float* w, const float* d_w, const cap_score_options* opt, const float* d_add,
                                    cap_dtype dtype, void* d_logits, hipStream_t st) {
    ScoreGradArgs a;
    a.logits = logits;
    a.idx = idx;
    a.keep = keep;
    a.w = w;
    a.d_w = d_w;
    a.d_add = d_add;
    a.out = d_logits;
    a.T = T;
    a.E = E;
    a.k = k;
    a.sigmoid = opt->kind == CAP_SCORE_SIGMOID;
    a.normalise = opt->normalise != 0;
    a.inv_scale = 0.5f / frexpf(opt->scale, &a.scale_exponent);
    a.scale_exponent -= 1;
    if (dtype == CAP_DTYPE_BF16) launch_grad<uint16_t>(a, st);
    else launch_grad<float>(a, st);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
