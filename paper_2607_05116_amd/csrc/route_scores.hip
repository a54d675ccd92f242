// Routing by scores: sigmoid or softmax over a token's experts, a bias for balance,
// groups of experts, top-k, gates, and the communication-aware pruning of Eq. 6
// (Sec. VI) on the gates' shares; and the gradient of the logits through the gates.
//
// Decisions (groups, experts, kept devices) are taken on values in 64 bits, so that
// they are those of the real numbers for all but values within about 2^-43 of each
// other: in 32 bits the scores of two experts at a border of the choice are equal or
// exchanged once in some hundred thousand tokens.
//
// Selection keys are the packed doubles of route_device.hpp.  Without a bias the choice
// goes by the logits (the high word), and so do groups by their best expert; else the
// key is the biased score in fp64, whose low 8 bits hold the expert
// (255 - e, or e below zero, so that the larger double is the lower expert among
// equal scores): 44 bits of the score are left.  An expert that is off (logit -inf
// or NaN, or a masked token) has a key below all scores, one of a closed group
// -infinity.
#pragma clang fp contract(off)

#include <math.h>

#include <type_traits>

#include "route_device.hpp"

namespace cap {
namespace {

constexpr int kQuadLanes = 4;               // lanes of a token
constexpr uint32_t kOffHigh = 0xFFEFFFFFu;  // high word of an off expert's key: about the lowest double

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

// Key of a logit (-0 as +0).
__device__ __forceinline__ double logit_key(float l, uint32_t tie) {
    const uint32_t hi = __float_as_uint(l + 0.0f);
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

// Slots of the routing: s = 0 .. N - 1 as a compile-time loop.
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each_slot(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each_slot<N, I + 1>(f);
    }
}

// Four lanes per token; lane h holds experts c * 16 + h * 4 + [0, 4), c < V / 4, and
// owns slots h and h + 4.
//   SCORE   keys are biased scores (else logits)
//   GROUPS  0: one group (or all of them open); 1: groups of 16 * CPG experts, which
//           are whole values of c; 2: any, through LDS (one wave per workgroup)
template <int V, int KP, bool SCORE, bool VEC, int GROUPS, int CPG>
__global__ __launch_bounds__(GROUPS == 2 ? 64 : 256) void route_scores_kernel(const ScoreArgs a) {
    constexpr int kThreads = GROUPS == 2 ? 64 : 256;
    constexpr int C = V / 4;
    constexpr int NS = (KP + 3) / 4;
    const int h = threadIdx.x & 3;
    const int t = blockIdx.x * (kThreads / kQuadLanes) + (threadIdx.x >> 2);
    const bool live = t < a.T;
    const int tc = live ? t : a.T - 1;
    const float* row = a.logits + static_cast<size_t>(tc) * a.E;

    float x[V];
#pragma unroll
    for (int c = 0; c < C; ++c) {
        if constexpr (VEC) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(row + c * 16 + h * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) x[c * 4 + i] = v[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int e = c * 16 + h * 4 + i;
                x[c * 4 + i] = e < a.E ? row[e] : -INFINITY;
            }
        }
    }
    const bool counted = !a.token_mask || a.token_mask[tc] != 0;
    // off: -inf; NaN too (the comparison is false)
#pragma unroll
    for (int j = 0; j < V; ++j) x[j] = (counted && x[j] > -INFINITY) ? x[j] : -INFINITY;

    // ---- softmax: the row's maximum and sum (in fp64 where keys take them)
    float top_x = 0.0f;
    double inv_sum = 1.0;
    const bool need_sum = !a.sigmoid && (SCORE || !a.normalise);
    if (need_sum) {
        top_x = x[0];
#pragma unroll
        for (int j = 1; j < V; ++j) top_x = fmaxf(top_x, x[j]);
        top_x = fmaxf(top_x, dpp_swap_f32<kDppXor1>(top_x));
        top_x = fmaxf(top_x, dpp_swap_f32<kDppXor2>(top_x));
        top_x = top_x > -INFINITY ? top_x : 0.0f;
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < V; ++j)
            sum += x[j] > -INFINITY ? exp64(static_cast<double>(x[j]) - static_cast<double>(top_x)) : 0.0;
        sum += dpp_swap<kDppXor1>(sum);
        sum += dpp_swap<kDppXor2>(sum);
        inv_sum = sum > 0.0 ? 1.0 / sum : 0.0;
    }
    auto score_of = [&](float l) {             // of an expert that is on
        return a.sigmoid ? sigmoid64(l) : exp64(static_cast<double>(l) - static_cast<double>(top_x)) * inv_sum;
    };

    // ---- keys
    double keys[V];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int j = c * 4 + i, e = c * 16 + h * 4 + i;
            const bool on = x[j] > -INFINITY;
            const uint32_t tie = 255u - static_cast<uint32_t>(e);
            double key;
            if constexpr (SCORE) {
                double v = score_of(on ? x[j] : 0.0f);
                if (a.bias) v += static_cast<double>(a.bias[VEC || e < a.E ? e : 0]);
                const uint32_t hi = high_word(v), sign = static_cast<uint32_t>(static_cast<int32_t>(hi) >> 31);
                key = words(hi, (low_word(v) & ~255u) | ((tie ^ sign) & 255u));
            } else {
                key = logit_key(x[j], tie);
            }
            key = on ? key : words(kOffHigh, ~tie);
            keys[j] = (VEC || e < a.E) ? key : kNoKey;
        }

    // ---- groups: the experts of closed ones leave the choice
    if constexpr (GROUPS != 0) {
        // what a key stands for in its group's score
        auto value_of = [&](double key) {
            const uint32_t hi = high_word(key);
            const double v = words(hi, SCORE ? low_word(key) & ~255u : 0u);
            return hi == kOffHigh ? kNoKey : v;
        };
        uint64_t open = 0;
        if constexpr (GROUPS == 1) {
            constexpr int G = C / CPG;
            double total[G];
#pragma unroll
            for (int g = 0; g < G; ++g) {
                double b1 = kNoKey, b2 = kNoKey;
#pragma unroll
                for (int j = g * CPG * 4; j < (g + 1) * CPG * 4; ++j) best_two(b1, b2, value_of(keys[j]));
                auto join = [&](double p1, double p2) {
                    b2 = __builtin_fmax(__builtin_fmin(b1, p1), __builtin_fmax(b2, p2));
                    b1 = __builtin_fmax(b1, p1);
                };
                join(dpp_swap<kDppXor1>(b1), dpp_swap<kDppXor1>(b2));
                join(dpp_swap<kDppXor2>(b1), dpp_swap<kDppXor2>(b2));
                total[g] = group_total(b1, b2, a.group_top);
            }
            uint32_t bits = 0;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                int ahead = 0;
#pragma unroll
                for (int o = 0; o < G; ++o)
                    if (o != g) ahead += (o < g ? total[o] >= total[g] : total[o] > total[g]) ? 1 : 0;
                bits |= ahead < a.open_groups ? 1u << g : 0u;
            }
            open = bits;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    keys[c * 4 + i] = (bits >> (c / CPG)) & 1u ? keys[c * 4 + i] : kNoKey;
        } else {
            // 16 tokens a workgroup of one wave; pitches are odd, so a token's lanes and
            // the tokens fall into different banks
            constexpr int kPitch = 4 * V + 1;
            __shared__ double value[16 * kPitch];
            __shared__ double total[16 * 65];
            double* mine = value + (threadIdx.x >> 2) * kPitch;
            double* sums = total + (threadIdx.x >> 2) * 65;
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) mine[c * 16 + h * 4 + i] = value_of(keys[c * 4 + i]);
            __syncthreads();
            for (int g = h; g < a.groups; g += 4) {
                double b1 = kNoKey, b2 = kNoKey;
                for (int i = 0; i < a.group_size; ++i) best_two(b1, b2, mine[g * a.group_size + i]);
                sums[g] = group_total(b1, b2, a.group_top);
            }
            __syncthreads();
            for (int g = h; g < a.groups; g += 4) {
                const double s = sums[g];
                int ahead = 0;
                for (int o = 0; o < a.groups; ++o) ahead += (o < g ? sums[o] >= s : sums[o] > s) ? 1 : 0;
                open |= ahead < a.open_groups ? 1ull << g : 0ull;
            }
            open |= dpp_swap_u64<kDppXor1>(open);
            open |= dpp_swap_u64<kDppXor2>(open);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int e = c * 16 + h * 4 + i;
                    const bool in = e < a.E && ((open >> small_quotient(e, a.group_size)) & 1ull);
                    keys[c * 4 + i] = in ? keys[c * 4 + i] : kNoKey;
                }
        }
    }

    // without a bias the choice within groups goes by the logits, which tell apart what
    // scores of 64 bits may not (the row is read again: keeping it costs V registers)
    const bool by_logit = !SCORE || (GROUPS != 0 && !a.bias);
    if constexpr (SCORE && GROUPS != 0) {
        if (!a.bias) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int e = (j / 4) * 16 + h * 4 + j % 4;
                const float l = row[VEC || e < a.E ? e : 0];
                const bool on = high_word(keys[j]) != kOffHigh && keys[j] > kNoKey;
                keys[j] = on ? logit_key(l, 255u - static_cast<uint32_t>(e)) : keys[j];
            }
        }
    }

    // ---- the KP largest keys of the lane, then of the quad
    double top[KP];
#pragma unroll
    for (int s = 0; s < KP; ++s) top[s] = s < V ? keys[s < V ? s : 0] : kNoKey;
    sort_desc<KP>(top);
#pragma unroll
    for (int b0 = KP; b0 < V; b0 += KP) {
        double blk[KP];
#pragma unroll
        for (int s = 0; s < KP; ++s) blk[s] = keys[b0 + s];
        sort_desc<KP>(blk);
        merge_top<KP>(top, blk);
    }
    merge_with_partner<kDppXor1, KP>(top);
    merge_with_partner<kDppXor2, KP>(top);

    // ---- the lane's slots h + 4 u: expert, device, score
    bool has[NS], on[NS];
    int my_e[NS], my_dev[NS];
    double q[NS];
    const float lead = key_logit(top[0]);                     // logit keys: the largest chosen logit
#pragma unroll
    for (int u = 0; u < NS; ++u) {
        double m = top[4 * u];
#pragma unroll
        for (int s = 1; s < kQuadLanes && 4 * u + s < KP; ++s) m = (h == s) ? top[4 * u + s] : m;
        has[u] = h + 4 * u < a.k;
        const int e = key_expert(m);
        my_e[u] = e < a.E ? e : a.E - 1;
        on[u] = has[u] && high_word(m) != kOffHigh;
        my_dev[u] = has[u] ? a.expert_rank[my_e[u]] & 63 : -1;
        double s = 0.0;
        if (on[u]) {
            const float l = by_logit ? key_logit(m) : row[my_e[u]];
            // softmax that is normalised over the chosen: relative to the largest of them
            s = a.sigmoid || need_sum ? score_of(l) : exp64(static_cast<double>(l) - static_cast<double>(lead));
        }
        q[u] = s;
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
                repeat = repeat || (same && s < h + 4 * u);
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
    for (int u = 0; u < NS; ++u) mask |= kept[u] ? 1ull << (my_dev[u] & 63) : 0ull;
    mask |= dpp_swap_u64<kDppXor1>(mask);
    mask |= dpp_swap_u64<kDppXor2>(mask);
#pragma unroll
    for (int s = 0; s < KP; ++s) kept_sum += devs[s] >= 0 && ((mask >> (devs[s] & 63)) & 1ull) ? qs[s] : 0.0;
    const double factor = static_cast<double>(a.scale) *
                          (a.normalise ? (kept_sum > 0.0 ? 1.0 / kept_sum : 0.0) : 1.0);
    if (!live) return;
#pragma unroll
    for (int u = 0; u < NS; ++u)
        if (has[u]) {
            const size_t at = static_cast<size_t>(t) * a.k + h + 4 * u;
            a.idx[at] = my_e[u];
            a.w[at] = kept[u] ? static_cast<float>(q[u] * factor) : 0.0f;
            a.keep[at] = kept[u] ? 1 : 0;
        }
    if (h == 0) a.mask[t] = mask;
}

template <int V, int KP, bool SCORE, bool VEC, int GROUPS, int CPG>
void launch(const ScoreArgs& a, hipStream_t st) {
    const int tokens = GROUPS == 2 ? 16 : 64;
    route_scores_kernel<V, KP, SCORE, VEC, GROUPS, CPG>
        <<<(a.T + tokens - 1) / tokens, GROUPS == 2 ? 64 : 256, 0, st>>>(a);
}

template <int V, int KP, bool SCORE>
void launch_groups(const ScoreArgs& a, bool vec, hipStream_t st) {
    if (a.open_groups >= a.groups) {
        if (vec) launch<V, KP, SCORE, true, 0, 1>(a, st);
        else launch<V, KP, SCORE, false, 0, 1>(a, st);
        return;
    }
    if constexpr (V >= 16) {
        if (vec && a.group_size % 16 == 0 && a.groups > 1) {
            const int cpg = a.group_size / 16;
            if (cpg == 1) return launch<V, KP, SCORE, true, 1, 1>(a, st);
            if constexpr (V >= 16) if (cpg == 2) return launch<V, KP, SCORE, true, 1, 2>(a, st);
            if constexpr (V >= 32) if (cpg == 4) return launch<V, KP, SCORE, true, 1, 4>(a, st);
            if constexpr (V >= 64) if (cpg == 8) return launch<V, KP, SCORE, true, 1, 8>(a, st);
        }
    }
    launch<V, KP, SCORE, false, 2, 1>(a, st);
}

template <int V>
void launch_keys(const ScoreArgs& a, bool vec, hipStream_t st) {
    // logits order experts and groups alike where nothing is added to scores
    const bool grouped = a.open_groups < a.groups;
    const bool score = a.bias || (grouped && a.group_top > 1 && a.group_size > 1);
    if (a.k <= 4) {
        if (score) launch_groups<V, 4, true>(a, vec, st);
        else launch_groups<V, 4, false>(a, vec, st);
    } else {
        if (score) launch_groups<V, 8, true>(a, vec, st);
        else launch_groups<V, 8, false>(a, vec, st);
    }
}

// ------------------------------------------------------------------ gradient
struct ScoreGradArgs {
    const float* logits;
    const int32_t* idx;
    const uint8_t* keep;
    const float* w;
    const float* d_w;
    const float* d_add;
    void* out;
    int T, E, k, sigmoid, normalise;
    float inv_scale;
};

__device__ __forceinline__ void store_value(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_value(uint16_t* p, float v) {
    // round to nearest even, once (a NaN stays one)
    *p = static_cast<uint16_t>(pack_bf16x2_rne(v, v));
}

// L lanes per token (a power of two, at least 8), four experts a lane.  The slots'
// gradients are worked out by the token's first k lanes and put in place through LDS.
template <int L, typename OUT>
__global__ __launch_bounds__(256) void route_scores_grad_kernel(const ScoreGradArgs a) {
    constexpr int kTokens = 256 / L;
    __shared__ float slot_row[kTokens][4 * L];
    const int j = threadIdx.x & (L - 1), tl = threadIdx.x / L;
    const long long t = static_cast<long long>(blockIdx.x) * kTokens + tl;
    const bool live = t < a.T;
    const bool full = !a.sigmoid && !a.normalise;        // the softmax's other experts have a gradient too
    const size_t row = static_cast<size_t>(live ? t : 0) * a.E;

    // the slot's part
    float g = 0.0f, wk = 0.0f, one_less = 1.0f;
    int e = -1;
    if (live && j < a.k) {
        const size_t at = static_cast<size_t>(t) * a.k + j;
        const int ei = a.idx[at];
        if ((!a.keep || a.keep[at]) && ei >= 0 && ei < a.E) {
            e = ei;
            wk = a.w[at];
            g = wk * a.d_w[at];
            if (a.sigmoid) one_less = 1.0f / (1.0f + expf(a.logits[row + ei]));   // 1 - s
        }
    }
    float total = g;
#pragma unroll
    for (int d = 1; d < 8; d *= 2) total += __shfl_xor(total, d);      // within the first 8 lanes
    total = __shfl(total, 0, L);                                       // to the token's lanes
    const uint64_t any_kept = __ballot(e >= 0);
    const int lane = threadIdx.x & 63;
    const bool some = ((any_kept >> (lane & ~(L - 1))) & 0xFFull) != 0;
    float slot = a.normalise ? g - wk * (total * a.inv_scale) : g;
    slot *= one_less;

    f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    *reinterpret_cast<f32x4*>(&slot_row[tl][4 * j]) = zero;
    __builtin_amdgcn_wave_barrier();                 // a token's lanes are of one wave, whose LDS accesses stay in order
    if (e >= 0) slot_row[tl][e] = slot;
    __builtin_amdgcn_wave_barrier();
    f32x4 d = *reinterpret_cast<const f32x4*>(&slot_row[tl][4 * j]);

    if (full) {
        float x[4], top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int ei = 4 * j + i;
            x[i] = live && ei < a.E ? a.logits[row + ei] : -INFINITY;
            x[i] = x[i] > -INFINITY ? x[i] : -INFINITY;          // NaN is off
            top = fmaxf(top, x[i]);
        }
#pragma unroll
        for (int s = 1; s < L; s *= 2) top = fmaxf(top, __shfl_xor(top, s));
        float p[4], sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            p[i] = x[i] > -INFINITY ? expf(x[i] - top) : 0.0f;
            sum += p[i];
        }
#pragma unroll
        for (int s = 1; s < L; s *= 2) sum += __shfl_xor(sum, s);
#pragma unroll
        for (int i = 0; i < 4; ++i) d[i] -= some && sum > 0.0f ? total * (p[i] / sum) : 0.0f;
    }
    if (!live) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int ei = 4 * j + i;
        if (ei < a.E) {
            float v = d[i];
            if (a.d_add) v += a.d_add[row + ei];
            store_value(static_cast<OUT*>(a.out) + row + ei, v);
        }
    }
}

template <typename OUT>
void launch_grad(const ScoreGradArgs& a, hipStream_t st) {
    auto go = [&](auto lanes) {
        constexpr int L = decltype(lanes)::value;
        constexpr int tokens = 256 / L;
        route_scores_grad_kernel<L, OUT><<<(a.T + tokens - 1) / tokens, 256, 0, st>>>(a);
    };
    if (a.E <= 32) go(std::integral_constant<int, 8>{});
    else if (a.E <= 64) go(std::integral_constant<int, 16>{});
    else if (a.E <= 128) go(std::integral_constant<int, 32>{});
    else go(std::integral_constant<int, 64>{});
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
    int V = 4;
    while (kQuadLanes * V < a.E) V *= 2;
    const bool vec = a.E == kQuadLanes * V && (reinterpret_cast<uintptr_t>(logits) & 15) == 0;
    switch (V) {
        case 4: launch_keys<4>(a, vec, st); break;
        case 8: launch_keys<8>(a, vec, st); break;
        case 16: launch_keys<16>(a, vec, st); break;
        case 32: launch_keys<32>(a, vec, st); break;
        default: launch_keys<64>(a, vec, st); break;
    }
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

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
    a.inv_scale = 1.0f / opt->scale;
    if (dtype == CAP_DTYPE_BF16) launch_grad<uint16_t>(a, st);
    else launch_grad<float>(a, st);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
