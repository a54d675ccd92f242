// Routing by scores: sigmoid or softmax over a token's experts, a bias for balance,
// groups of experts, top-k, gates, and the communication-aware pruning of Eq. 6
// (Sec. VI) on the gates' shares.  (Built without NaN semantics: whether a logit is finite
// is asked of its bits.)
//
// Decisions (groups, experts, kept devices) are those of the real numbers for all but values
// within about 2^-43 of each other: in fp32 the scores of two experts at a border of the choice
// are equal or exchanged once in some hundred thousand tokens.  The choice is made in fp32, with
// a bound on its error, and again in fp64 for the tokens that this leaves unsure; gates and
// pruning are in fp64.
//
// Selection keys are the packed doubles of route_device.hpp: the high word is the logit
// (without a bias, within groups) or the biased score as fp32, the low word breaks ties (the
// larger double is the lower expert).  The exact choice's keys are biased scores in fp64 whose
// low 8 bits hold the expert: 44 bits of the score are left.  An expert that is off (its logit
// is not finite, or its token masked) has a key below all scores, one of a closed group a key
// below that.
#pragma clang fp contract(off)

#include <math.h>

#include <type_traits>

#include "route_device.hpp"

namespace cap {
namespace {

constexpr int kQuadLanes = 4;
// Values in the place of logits or scores: of an expert that is off (the lowest finite float:
// the operator takes finite logits to lie above it), and of one of a closed group (-inf).  As
// high words of keys both are finite doubles, whose exponent has three bits more, below all others.
constexpr uint32_t kInfBits = 0x7F800000u;
constexpr float kOff = -3.402823466e38f;
constexpr uint32_t kOffHigh = 0xFF7FFFFFu, kClosedHigh = 0xFF800000u;
__device__ __forceinline__ bool key_is_on(uint32_t high) { return high < kOffHigh; }
__device__ __forceinline__ bool finite_bits(float v) { return (__float_as_uint(v) & kInfBits) != kInfBits; }

struct ScoreArgs {
    const float* logits;
    const float* bias;
    const uint8_t* token_mask;
    const int32_t* expert_rank;
    int32_t* idx;
    float* w;
    uint8_t* keep;
    uint64_t* mask;
    int T, E, R, k, ranks_per_node, tokens_per_rank;
    int groups, group_size, open_groups, group_top, sigmoid, normalise;
    float scale, p, inter_node_cost;
};

// e^x in fp64 for x <= 709 (0 below -700): n = round(x / ln 2), r = x - n ln 2 with
// ln 2 in two parts (the first of 32 bits, so n times it is exact), the Taylor
// polynomial of degree 12 (|r| <= 0.347: the next term is 2^-53 of the sum), times 2^n.
__device__ __forceinline__ double exp64(double x) {
    const double n = __builtin_rint(x * 1.4426950408889634);
    double r = __builtin_fma(-n, 0x1.62e42feep-1, x);
    r = __builtin_fma(-n, 0x1.a39ef35793c76p-33, r);
    double q = 1.0 / 479001600.0;
    q = __builtin_fma(q, r, 1.0 / 39916800.0);
    q = __builtin_fma(q, r, 1.0 / 3628800.0);
    q = __builtin_fma(q, r, 1.0 / 362880.0);
    q = __builtin_fma(q, r, 1.0 / 40320.0);
    q = __builtin_fma(q, r, 1.0 / 5040.0);
    q = __builtin_fma(q, r, 1.0 / 720.0);
    q = __builtin_fma(q, r, 1.0 / 120.0);
    q = __builtin_fma(q, r, 1.0 / 24.0);
    q = __builtin_fma(q, r, 1.0 / 6.0);
    q = __builtin_fma(q, r, 0.5);
    q = __builtin_fma(q, r, 1.0);
    q = __builtin_fma(q, r, 1.0);
    const double e = __builtin_ldexp(q, static_cast<int>(n));
    return x >= -700.0 ? e : 0.0;
}

// 1 / a for 1 <= a < 2^1022: the hardware's estimate and two Newton steps.
__device__ __forceinline__ double reciprocal64(double a) {
    double y = __builtin_amdgcn_rcp(a);
    y = __builtin_fma(__builtin_fma(-a, y, 1.0), y, y);
    return __builtin_fma(__builtin_fma(-a, y, 1.0), y, y);
}

// 1 / (1 + e^-x); 0 below -700.
__device__ __forceinline__ double sigmoid64(float x) {
    const float y = -x < 700.0f ? -x : 700.0f;
    const double s = reciprocal64(1.0 + exp64(static_cast<double>(y)));
    return -x < 700.0f ? s : 0.0;
}

template <int S>
__device__ __forceinline__ int quad_at(int v) {
    return __builtin_amdgcn_mov_dpp(v, S | (S << 2) | (S << 4) | (S << 6), 0xF, 0xF, true);
}
template <int S>
__device__ __forceinline__ double quad_at(double v) {
    const long long b = __double_as_longlong(v);
    const int lo = quad_at<S>(static_cast<int>(b)), hi = quad_at<S>(static_cast<int>(b >> 32));
    return __longlong_as_double((static_cast<long long>(hi) << 32) | static_cast<uint32_t>(lo));
}
template <int CTRL>
__device__ __forceinline__ float dpp_swap_f32(float v) {
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}

__device__ __forceinline__ double words(uint32_t hi, uint32_t lo) {
    return __longlong_as_double(static_cast<long long>((static_cast<uint64_t>(hi) << 32) | lo));
}
__device__ __forceinline__ uint32_t high_word(double v) {
    return static_cast<uint32_t>(static_cast<uint64_t>(__double_as_longlong(v)) >> 32);
}
__device__ __forceinline__ uint32_t low_word(double v) {
    return static_cast<uint32_t>(static_cast<uint64_t>(__double_as_longlong(v)));
}

// Key of a value that is not -0.
__device__ __forceinline__ double value_key(float v, uint32_t tie) {
    const uint32_t hi = __float_as_uint(v);
    return words(hi, tie ^ static_cast<uint32_t>(static_cast<int32_t>(hi) >> 31));
}

// Best two of a group so far, with one more value.
__device__ __forceinline__ void best_two(double& a, double& b, double v) {
    b = __builtin_fmax(b, __builtin_fmin(a, v));
    a = __builtin_fmax(a, v);
}
// A group's score from its best two: -infinity without an expert that is on.
__device__ __forceinline__ double group_total(double a, double b, int top) {
    return top > 1 && b > kNoKey ? a + b : a;
}

// Tokens up to which eight lanes take one, not four: they fill the chip sooner, at the price of
// one join more.  us with eight and with four: 256 experts in 8 groups, 32 tokens 7.5 and 9.4,
// 8,192 11.8 and 13.6, 12,288 14.3 and 13.5, 32,768 21.0 and 18.7; 96 experts in 12 groups
// (through LDS) 9.2 and 13.0, 13.2 and 17.9, 13.2 and 18.0, 22.0 and 22.8.
constexpr int kTokens8 = 12288;

// Slots of the routing: s = 0 .. N - 1 as a compile-time loop.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each_slot(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each_slot<N, I + 1>(f);
    }
}

// ------------------------------------------------------------------ exact choice
// How far two biased scores v may lie apart, relative to 1 + |v|, and not be ordered for
// certain by their fp32 values: twice their error, and twice that for a margin.  A sigmoid's
// error is below 2^-22 (in units of 2^-24: 0.3 from the rounded argument, weighed with
// s (1 - s) |x| < 0.23; 0.5 from the exponential's ulp, 1 from 1 + e, 2 from the reciprocal's
// ulp), a softmax probability's 2^-20 of it (that of its sum, see below); the sum with the
// bias rounds by 2^-24 |v|.
constexpr float kUnsureSigmoid = 0x1p-20f, kUnsureSoftmax = 0x1p-18f;

constexpr int kExactValues = kMaxE;
struct ExactSpace {
    double value[kExactValues];
    int chosen[kMaxK];
};

// Joins over a wave: DPP within rows of 16 lanes, then the four rows' first lanes.
__device__ __forceinline__ double lane_f64(double v, int l) {
    const long long b = __double_as_longlong(v);
    return words(static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b >> 32), l)),
                 static_cast<uint32_t>(__builtin_amdgcn_readlane(static_cast<int>(b), l)));
}
template <typename F>
__device__ __forceinline__ double over_wave(double v, F&& join) {
    v = join(v, dpp_swap<kDppXor1>(v));
    v = join(v, dpp_swap<kDppXor2>(v));
    v = join(v, dpp_swap<kDppHalfMirror>(v));
    v = join(v, dpp_swap<0x140>(v));                   // row_mirror
    return join(join(lane_f64(v, 0), lane_f64(v, 16)), join(lane_f64(v, 32), lane_f64(v, 48)));
}

// The choice of one token by the whole wave, on fp64 scores: for the few tokens that fp32
// leaves unsure, and for ties.  Leaves expert | on << 16 of each slot in space.chosen.
__device__ __forceinline__ void exact_choice(const ScoreArgs& a, int t, ExactSpace& space) {
    const int lane = threadIdx.x & 63;
    const float* row = a.logits + static_cast<size_t>(t) * a.E;
    const bool counted = !a.token_mask || a.token_mask[t] != 0;
    float x[4], b[4];
    bool on[4];
    double top_x = kNoKey;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 4 * lane + i < a.E ? 4 * lane + i : a.E - 1;
        x[i] = row[e];
        b[i] = a.bias ? a.bias[e] : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        on[i] = 4 * lane + i < a.E && counted && finite_bits(x[i]) && x[i] > kOff;
        top_x = on[i] ? __builtin_fmax(top_x, static_cast<double>(x[i])) : top_x;
    }
    double inv_sum = 1.0;
    if (!a.sigmoid) {
        top_x = over_wave(top_x, [](double p, double q) { return __builtin_fmax(p, q); });
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += on[i] ? exp64(static_cast<double>(x[i]) - top_x) : 0.0;
        sum = over_wave(sum, [](double p, double q) { return p + q; });
        inv_sum = sum > 0.0 ? 1.0 / sum : 0.0;
    }
    double key[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int e = 4 * lane + i;
        double v = 0.0;
        if (on[i])
            v = a.sigmoid ? sigmoid64(x[i]) : exp64(static_cast<double>(x[i]) - top_x) * inv_sum;
        v += static_cast<double>(b[i]);
        space.value[4 * lane + i] = on[i] ? words(high_word(v), low_word(v) & ~255u) : kNoKey;
        const uint32_t tie = 255u - static_cast<uint32_t>(e);
        const uint32_t hi = high_word(v), sign = static_cast<uint32_t>(static_cast<int32_t>(hi) >> 31);
        // (without a bias, the choice within groups goes by the logits)
        key[i] = !on[i] ? words(kOffHigh, ~tie) : a.bias ? words(hi, (low_word(v) & ~255u) | ((tie ^ sign) & 255u)) : value_key(x[i] + 0.0f, tie);
        key[i] = e < a.E ? key[i] : kNoKey;
    }
    if (a.open_groups < a.groups) {
        __builtin_amdgcn_wave_barrier();               // one wave: its LDS accesses stay in order
        double b1 = kNoKey, b2 = kNoKey;
        if (lane < a.groups)
#pragma unroll 8
            for (int i = 0; i < a.group_size; ++i) best_two(b1, b2, space.value[lane * a.group_size + i]);
        const double total = group_total(b1, b2, a.group_top);
        int ahead = 0;
        for (int o = 0; o < a.groups; ++o) {
            const double other = lane_f64(total, o);
            ahead += (o < lane ? other >= total : other > total) ? 1 : 0;
        }
        const Bits open = split_bits(__ballot(lane < a.groups && ahead < a.open_groups));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = 4 * lane + i;
            key[i] = e < a.E && has_bit(open, small_quotient(e, a.group_size)) ? key[i] : kNoKey;
        }
    }
    for (int s = 0; s < a.k; ++s) {
        const double best = over_wave(__builtin_fmax(__builtin_fmax(key[0], key[1]), __builtin_fmax(key[2], key[3])),
                                      [](double p, double q) { return __builtin_fmax(p, q); });
#pragma unroll
        for (int i = 0; i < 4; ++i) key[i] = key[i] == best ? kNoKey : key[i];     // keys are distinct
        if (lane == 0) space.chosen[s] = key_expert(best) | (high_word(best) != kOffHigh ? 1 << 16 : 0);
    }
    __builtin_amdgcn_wave_barrier();
}

// ------------------------------------------------------------------ routing
// Joins over the L lanes of a token (4 or 8).
template <int L, typename F>
__device__ __forceinline__ void over_lanes(F&& step) {
    step(std::integral_constant<int, kDppXor1>{});
    step(std::integral_constant<int, kDppXor2>{});
    if constexpr (L == 8) step(std::integral_constant<int, kDppHalfMirror>{});
}
template <int CTRL>
__device__ __forceinline__ int dpp_swap_i32(int v) { return __builtin_amdgcn_mov_dpp(v, CTRL, 0xF, 0xF, true); }

// L lanes per token; lane h holds experts c * 4 L + h * 4 + [0, 4), c < V / 4; the lanes h of
// a quad own slots h and h + 4 (of 8 lanes, both quads work them out, and the first writes).
//   SCORE   the choice goes by biased scores, first in fp32; tokens whose order that leaves
//           unsure (about one of 2000) are chosen by exact_choice.  Else it goes by logits.
//   GROUPS  0: one group (or all of them open); 1: groups of 4 L CPG experts, which are whole
//           values of c; 2: any, through LDS
// What bounds it: instruction issue.  32,768 tokens of 256 experts in 8 groups, sigmoid with a
// bias, pruned: 18.8 us (35.8 with all scores in fp64: one wave a SIMD, for the registers of 64
// keys a lane; keys are formed block by block now, and fp64 is left to the chosen slots); to read
// and write 36 MB takes 8.  A wave has 2,852 vector instructions.  The routing by the chosen
// logits' softmax, whose selection network is the same and which takes 8.0 us for these logits, has
// 1,314: the others are around the network, where every value is asked whether it is finite, scored,
// biased, compared for its group, closed with it and counted if it is within reach of the last.
// Unsure tokens cost under 0.2 us, but if every token is one (all logits alike), 32,768 take 90 us.
// 32 tokens: 7.5 us, a chain of joins.  Through LDS (GROUPS 2), with loads of single values: 96
// experts in 12 groups 22.8 us, 160 in 8 groups 43 us.
template <int L, int V, int KP, bool SCORE, bool VEC, int GROUPS, int CPG>
__global__ __launch_bounds__(256) void route_scores_kernel(const ScoreArgs a) {
    constexpr int C = V / 4, kTokens = 256 / L;
    constexpr int NS = (KP + 3) / 4;
    __shared__ ExactSpace exact[SCORE ? 4 : 1];
    const int h = threadIdx.x & (L - 1), hq = h & 3;
    const int t = blockIdx.x * kTokens + threadIdx.x / L;
    const bool live = t < a.T;
    const int tc = live ? t : a.T - 1;
    const float* row = a.logits + static_cast<size_t>(tc) * a.E;
    auto expert = [&](int j) { return (j >> 2) * (4 * L) + h * 4 + (j & 3); };

    // v: what the choice goes by, never -0
    float v[V];
    const bool counted = !a.token_mask || a.token_mask[tc] != 0;
    auto load_row = [&]() {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            if constexpr (VEC) {
                const f32x4 q = *reinterpret_cast<const f32x4*>(row + c * (4 * L) + h * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[c * 4 + i] = q[i];
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = expert(c * 4 + i);
                    v[c * 4 + i] = e < a.E ? row[e] : kOff;
                }
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = counted & finite_bits(v[j]) ? v[j] + 0.0f : kOff;
    };
    load_row();

    // ---- softmax: the row's maximum, and the sum of fp32 exponentials in fp64.  With z = l -
    // max, a term is off by 2^-23 (its ulp) and 2.5 |z| 2^-24 (z, log2 e and their product
    // rounded); |z| is at most ln 256 on average under the softmax: the sum is within 2^-20.
    constexpr float kLog2E = 1.44269504088896340736f;
    float top_x = 0.0f;
    double inv_sum = 1.0;
    const bool need_sum = !a.sigmoid && (SCORE || !a.normalise);
    if (need_sum) {
        top_x = v[0];
#pragma unroll
        for (int j = 1; j < V; ++j) top_x = fmaxf(top_x, v[j]);
        over_lanes<L>([&](auto ctrl) { top_x = fmaxf(top_x, dpp_swap_f32<ctrl.value>(top_x)); });
        top_x = top_x > kOff ? top_x : 0.0f;
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j)
            sum += static_cast<double>(__builtin_amdgcn_exp2f((v[j] - top_x) * kLog2E));         // 0 if off
        over_lanes<L>([&](auto ctrl) { sum += dpp_swap<ctrl.value>(sum); });
        inv_sum = sum > 0.0 ? 1.0 / sum : 0.0;
    }
    const float inv_sum32 = static_cast<float>(inv_sum);
    if constexpr (SCORE) {
        // (each branch for all values at once: one around every value would keep the loads apart)
        if (a.sigmoid) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float p = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-v[j] * kLog2E));
                v[j] = v[j] > kOff ? p : kOff;
            }
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float p = __builtin_amdgcn_exp2f((v[j] - top_x) * kLog2E) * inv_sum32;
                v[j] = v[j] > kOff ? p : kOff;
            }
        }
        if (a.bias) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[j] += a.bias[VEC || expert(j) < a.E ? expert(j) : 0];       // kOff stays: |b| is below half its ulp
        }
    }

    // ---- groups: experts of closed ones leave the choice
    const float closed = -INFINITY;
    bool unsure = false;
    const float reach_of = a.sigmoid ? kUnsureSigmoid : kUnsureSoftmax;
    // with scores: totals of two values, of magnitudes up to `size`, each unsure by itself
    auto gap_unsure = [&](float lowest_open, float highest_closed, float size) {
        return (highest_closed > kOff) & lowest_open - highest_closed <= 2.0f * reach_of * (1.0f + size);
    };
    if constexpr (GROUPS == 1) {
        constexpr int G = C / CPG;
        float total[G], size = 0.0f;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float b1 = kOff, b2 = kOff;
#pragma unroll
            for (int j = g * CPG * 4; j < (g + 1) * CPG * 4; ++j) {
                b2 = fmaxf(b2, fminf(b1, v[j]));
                b1 = fmaxf(b1, v[j]);
            }
            over_lanes<L>([&](auto ctrl) {
                const float p1 = dpp_swap_f32<ctrl.value>(b1), p2 = dpp_swap_f32<ctrl.value>(b2);
                b2 = fmaxf(fminf(b1, p1), fmaxf(b2, p2));
                b1 = fmaxf(b1, p1);
            });
            total[g] = (a.group_top > 1) & (b2 > kOff) ? b1 + b2 : b1;
            size = fmaxf(size, b1 > kOff ? fabsf(b1) : 0.0f);
            size = fmaxf(size, b2 > kOff ? fabsf(b2) : 0.0f);
        }
        uint32_t open = 0;
        float lowest = INFINITY, highest = kOff;
#pragma unroll
        for (int g = 0; g < G; ++g) {
            int ahead = 0;
#pragma unroll
            for (int o = 0; o < G; ++o)
                if (o != g) ahead += (o < g ? total[o] >= total[g] : total[o] > total[g]) ? 1 : 0;
            const bool is_open = ahead < a.open_groups;
            open |= is_open ? 1u << g : 0u;
            lowest = is_open ? fminf(lowest, total[g]) : lowest;
            highest = is_open ? highest : fmaxf(highest, total[g]);
        }
        if (SCORE) {
            unsure = gap_unsure(lowest, highest, size);
            if (!a.bias) load_row();                   // within groups the choice goes by the logits
        }
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (open >> (j / (4 * CPG))) & 1u ? v[j] : closed;
    }
    if constexpr (GROUPS == 2) {
        // pitches are odd: a token's lanes, and the tokens, fall into different banks
        constexpr int kPitch = L * V + 1;
        __shared__ float value[kTokens * kPitch];
        __shared__ float total[kTokens * (kMaxScoreGroups + 1)];
        float* const mine = value + threadIdx.x / L * kPitch;
        float* const sums = total + threadIdx.x / L * (kMaxScoreGroups + 1);
#pragma unroll
        for (int j = 0; j < V; ++j) mine[expert(j)] = v[j];
        __syncthreads();
        float size = 0.0f;
        for (int g = h; g < a.groups; g += L) {
            float b1 = kOff, b2 = kOff;
            for (int i = 0; i < a.group_size; ++i) {
                const float x = mine[g * a.group_size + i];
                b2 = fmaxf(b2, fminf(b1, x));
                b1 = fmaxf(b1, x);
            }
            sums[g] = (a.group_top > 1) & (b2 > kOff) ? b1 + b2 : b1;
            size = fmaxf(size, b1 > kOff ? fabsf(b1) : 0.0f);
            size = fmaxf(size, b2 > kOff ? fabsf(b2) : 0.0f);
        }
        __syncthreads();
        uint64_t open = 0;
        float lowest = INFINITY, highest = kOff;
        for (int g = h; g < a.groups; g += L) {
            const float s = sums[g];
            int ahead = 0;
            for (int o = 0; o < a.groups; ++o) ahead += (o < g ? sums[o] >= s : sums[o] > s) ? 1 : 0;
            const bool is_open = ahead < a.open_groups;
            open |= bit64(g, is_open);
            lowest = is_open ? fminf(lowest, s) : lowest;
            highest = is_open ? highest : fmaxf(highest, s);
        }
        over_lanes<L>([&](auto ctrl) {
            open |= dpp_swap_u64<ctrl.value>(open);
            lowest = fminf(lowest, dpp_swap_f32<ctrl.value>(lowest));
            highest = fmaxf(highest, dpp_swap_f32<ctrl.value>(highest));
            size = fmaxf(size, dpp_swap_f32<ctrl.value>(size));
        });
        if (SCORE) {
            unsure = gap_unsure(lowest, highest, size);
            if (!a.bias) load_row();
        }
        const Bits opened = split_bits(open);
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const int e = expert(j);
            v[j] = e < a.E && has_bit(opened, small_quotient(e, a.group_size)) ? v[j] : closed;
        }
    }

    // ---- the KP largest keys of the lane, then of the token's lanes
    auto key_of = [&](int j) {
        const double key = value_key(v[j], 255u - static_cast<uint32_t>(expert(j)));
        return VEC || expert(j) < a.E ? key : kNoKey;
    };
    double top[KP];
#pragma unroll
    for (int s = 0; s < KP; ++s) top[s] = s < V ? key_of(s < V ? s : 0) : kNoKey;
    sort_desc<KP>(top);
#pragma unroll
    for (int b0 = KP; b0 < V; b0 += KP) {
        double blk[KP];
#pragma unroll
        for (int s = 0; s < KP; ++s) blk[s] = key_of(b0 + s);
        sort_desc<KP>(blk);
        merge_top<KP>(top, blk);
    }
    over_lanes<L>([&](auto ctrl) { merge_with_partner<ctrl.value, KP>(top); });

    // ---- is the order sure?  Neighbours among the chosen lie far enough apart, and so does
    // what comes next: no more than k values within reach of the last one
    if constexpr (SCORE) {
        if (GROUPS == 0 || a.bias) {
            float last = INFINITY;
#pragma unroll
            for (int s = 0; s < KP; ++s) {
                const bool on = key_is_on(high_word(top[s]));
                const float x = key_logit(top[s]);
                if (s + 1 < KP) {
                    const bool next_on = key_is_on(high_word(top[s + 1 < KP ? s + 1 : s]));
                    unsure |= (s + 1 < a.k) & on & next_on & (x - key_logit(top[s + 1 < KP ? s + 1 : s]) <= reach_of * (1.0f + fabsf(x)));
                }
                last = (s + 1 == a.k) & on ? x - reach_of * (1.0f + fabsf(x)) : last;
            }
            int reach = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) reach += v[j] >= last ? 1 : 0;
            over_lanes<L>([&](auto ctrl) { reach += dpp_swap_i32<ctrl.value>(reach); });
            unsure |= (last < INFINITY) & (reach > a.k);
        }
    }

    // ---- the lane's slots hq + 4 u
    bool has[NS], on[NS];
    int my_e[NS];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
        double m = top[4 * u];
#pragma unroll
        for (int s = 1; s < kQuadLanes && 4 * u + s < KP; ++s) m = (hq == s) ? top[4 * u + s] : m;
        has[u] = hq + 4 * u < a.k;
        my_e[u] = key_expert(m);
        on[u] = key_is_on(high_word(m));
    }
    if constexpr (SCORE) {
        ExactSpace& space = exact[threadIdx.x >> 6];
        uint64_t left = __ballot(unsure && live && h == 0);
        while (left) {                                 // wave-uniform
            const int l = __ffsll(static_cast<unsigned long long>(left)) - 1;
            left &= left - 1;
            exact_choice(a, __builtin_amdgcn_readlane(t, l), space);
            const bool here = ((threadIdx.x & 63) ^ h) == l;
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                const int c = space.chosen[hq + 4 * u];
                my_e[u] = here ? c & 0xFFFF : my_e[u];
                on[u] = here ? (c >> 16) != 0 : on[u];
            }
            __builtin_amdgcn_wave_barrier();
        }
    }

    // ---- their devices and scores
    int my_dev[NS];
    double q[NS];
    float my_l[NS];
#pragma unroll
    for (int u = 0; u < NS; ++u) {
        my_e[u] = has[u] && my_e[u] < a.E ? my_e[u] : a.E - 1;
        on[u] = on[u] && has[u];
        my_dev[u] = has[u] ? a.expert_rank[my_e[u]] & 63 : -1;
        my_l[u] = row[my_e[u]];
    }
    float lead = -INFINITY;                            // normalised over the chosen: relative to the largest of them
#pragma unroll
    for (int u = 0; u < NS; ++u) lead = on[u] ? fmaxf(lead, my_l[u]) : lead;
    lead = fmaxf(lead, dpp_swap_f32<kDppXor1>(lead));
    lead = fmaxf(lead, dpp_swap_f32<kDppXor2>(lead));
    const float base = a.normalise ? lead : top_x;
#pragma unroll
    for (int u = 0; u < NS; ++u) {
        const double s = a.sigmoid ? sigmoid64(my_l[u])
                                   : exp64(static_cast<double>(my_l[u]) - static_cast<double>(base)) *
                                         (a.normalise ? 1.0 : inv_sum);
        q[u] = on[u] ? s : 0.0;
    }
    double qs[KP];
    int devs[KP];
    each_slot<KP>([&](auto S) {
        constexpr int s = decltype(S)::value;
        qs[s] = quad_at<s % 4>(q[s / 4]);
        devs[s] = quad_at<s % 4>(on[s / 4] ? my_dev[s / 4] : -1);
    });
    double sum = qs[0];
#pragma unroll
    for (int s = 1; s < KP; ++s) sum += qs[s];
    const double inv = sum > 0.0 ? 1.0 / sum : 0.0;

    // ---- pruning (Eq. 6): a device's share a_d over its cost; devices are kept in
    // descending order until the kept shares reach 1 - p.  A lane works out, for the
    // devices of its slots, the share of those that come before.
    bool kept[NS];
    if (a.p == 0.0f) {
#pragma unroll
        for (int u = 0; u < NS; ++u) kept[u] = on[u];
    } else {
        const int src = small_quotient(tc, a.tokens_per_rank);
        const int src_node = small_quotient(src, a.ranks_per_node);
        double share[NS], ratio[NS];
        bool first[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u) {
            double sh = 0.0;
            bool repeat = false;
#pragma unroll
            for (int s = 0; s < KP; ++s) {
                const bool same = on[u] && devs[s] == my_dev[u];
                sh += same ? qs[s] : 0.0;
                repeat = repeat || (same && s < hq + 4 * u);
            }
            share[u] = sh * inv;
            first[u] = on[u] && !repeat;
            ratio[u] = share[u];
            if (my_dev[u] == src) ratio[u] = __builtin_inf();
            else if (a.R > a.ranks_per_node && small_quotient(my_dev[u] & 63, a.ranks_per_node) != src_node)
                ratio[u] = share[u] / static_cast<double>(a.inter_node_cost);
        }
        const double target = 1.0 - static_cast<double>(a.p);
        double before[NS];
#pragma unroll
        for (int u = 0; u < NS; ++u) before[u] = 0.0;
        each_slot<KP>([&](auto S) {
            constexpr int s = decltype(S)::value;
            const double r = quad_at<s % 4>(first[s / 4] ? ratio[s / 4] : kNoKey);
            const double sh = quad_at<s % 4>(share[s / 4]);
#pragma unroll
            for (int u = 0; u < NS; ++u) {
                // without a candidate r is -infinity, below every ratio
                const bool ahead = r > ratio[u] || (r == ratio[u] && devs[s] < my_dev[u]);
                before[u] += ahead ? sh : 0.0;
            }
        });
        // every slot of a device has the same share, ratio and sum before it
#pragma unroll
        for (int u = 0; u < NS; ++u) kept[u] = on[u] && before[u] < target;
    }
    uint64_t mask = 0;
    double kept_sum = 0.0;
#pragma unroll
    for (int u = 0; u < NS; ++u) mask |= bit64(my_dev[u], kept[u]);
    mask |= dpp_swap_u64<kDppXor1>(mask);
    mask |= dpp_swap_u64<kDppXor2>(mask);
    each_slot<KP>([&](auto S) {
        constexpr int s = decltype(S)::value;
        kept_sum += quad_at<s % 4>(kept[s / 4] ? q[s / 4] : 0.0);
    });
    const double factor = static_cast<double>(a.scale) *
                          (a.normalise ? (kept_sum > 0.0 ? 1.0 / kept_sum : 0.0) : 1.0);
    if (!live || h >= 4) return;
#pragma unroll
    for (int u = 0; u < NS; ++u)
        if (has[u]) {
            const size_t at = static_cast<size_t>(t) * a.k + hq + 4 * u;
            a.idx[at] = my_e[u];
            a.w[at] = kept[u] ? static_cast<float>(q[u] * factor) : 0.0f;
            a.keep[at] = kept[u] ? 1 : 0;
        }
    if (h == 0) a.mask[t] = mask;
}

template <int L, int V, int KP, bool SCORE, bool VEC, int GROUPS, int CPG = 1>
void launch(const ScoreArgs& a, hipStream_t st) {
    constexpr int tokens = 256 / L;
    route_scores_kernel<L, V, KP, SCORE, VEC, GROUPS, CPG><<<(a.T + tokens - 1) / tokens, 256, 0, st>>>(a);
}

template <int L, int V, int KP, bool SCORE>
void launch_groups(const ScoreArgs& a, bool vec, hipStream_t st) {
    if (a.open_groups >= a.groups) {
        if (vec) launch<L, V, KP, SCORE, true, 0>(a, st);
        else launch<L, V, KP, SCORE, false, 0>(a, st);
        return;
    }
    if (vec && a.group_size % (4 * L) == 0) {
        const int cpg = a.group_size / (4 * L);
        if constexpr (V >= 8) if (cpg == 1) return launch<L, V, KP, SCORE, true, 1, 1>(a, st);
        if constexpr (V >= 16) if (cpg == 2) return launch<L, V, KP, SCORE, true, 1, 2>(a, st);
        if constexpr (V >= 32) if (cpg == 4) return launch<L, V, KP, SCORE, true, 1, 4>(a, st);
        if constexpr (V >= 64) if (cpg == 8) return launch<L, V, KP, SCORE, true, 1, 8>(a, st);
    }
    launch<L, V, KP, SCORE, false, 2>(a, st);
}

template <int L, int V>
void launch_keys(const ScoreArgs& a, bool vec, hipStream_t st) {
    // logits order experts and groups alike where nothing is added to scores
    const bool grouped = a.open_groups < a.groups;
    const bool score = a.bias || (grouped && a.group_top > 1 && a.group_size > 1);
    if (a.k <= 4) {
        if (score) launch_groups<L, V, 4, true>(a, vec, st);
        else launch_groups<L, V, 4, false>(a, vec, st);
    } else {
        if (score) launch_groups<L, V, 8, true>(a, vec, st);
        else launch_groups<L, V, 8, false>(a, vec, st);
    }
}

}  // namespace

cap_status route_scores_launch(const cap_topology* tp, const float* logits, const cap_score_options* opt, float p,
                               int32_t* idx, float* w, uint8_t* keep, uint64_t* mask, hipStream_t st) {
    ScoreArgs a;
    a.logits = logits;
    a.bias = opt->bias;
    a.token_mask = opt->token_mask;
    a.expert_rank = tp->expert_rank;
    a.idx = idx;
    a.w = w;
    a.keep = keep;
    a.mask = mask;
    a.T = tp->T;
    a.E = tp->E;
    a.R = tp->R;
    a.k = tp->k;
    a.ranks_per_node = tp->ranks_per_node;
    a.tokens_per_rank = tp->tokens_per_rank;
    a.groups = opt->n_groups;
    a.group_size = tp->E / opt->n_groups;
    a.open_groups = opt->topk_groups;
    a.group_top = opt->group_top;
    a.sigmoid = opt->kind == CAP_SCORE_SIGMOID;
    a.normalise = opt->normalise != 0;
    a.scale = opt->scale;
    a.p = p;
    a.inter_node_cost = tp->inter_node_cost;
    auto go = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        int V = 4;
        while (L * V < a.E) V *= 2;
        const bool vec = a.E == L * V && (reinterpret_cast<uintptr_t>(logits) & 15) == 0;
        if (V == 4) return launch_keys<L, 4>(a, vec, st);
        if (V == 8) return launch_keys<L, 8>(a, vec, st);
        if (V == 16) return launch_keys<L, 16>(a, vec, st);
        if (V == 32) return launch_keys<L, 32>(a, vec, st);
        if constexpr (L == 4) if (V == 64) return launch_keys<L, 64>(a, vec, st);
    };
    if (a.E > 16 && a.T <= kTokens8) go(std::integral_constant<int, 8>{});
    else go(std::integral_constant<int, 4>{});
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
