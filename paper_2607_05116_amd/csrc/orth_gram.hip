// Orthogonalised gradients of few rows (or columns): the steps in the space of
// the Gram matrix.
//
// Every step multiplies X by a polynomial of S = X X^T, and polynomials of one
// symmetric matrix commute, so with S_0 = U U^T / |U|^2 (n x n, n the shorter side)
//   P = a I + b S + c S S;   Q <- Q P  (Q_0 = I);   S <- P S P
// for each step, and the result is Q X_0.  U is read twice whatever the number of
// steps, and the trace of U U^T is the norm.  What the short form costs is
// precision: S has the squares of the singular values, so its rounding reaches
// directions of sqrt(2^-p) of the largest one.  S_0 is summed in fp32 and the n x n
// products are taken on values of 21 bits (fp16 pairs, three MFMAs a product), which
// leaves 1e-6 to 1e-3 of the result's norm over spectra that fall by e^-12 and low ranks;
// with plain fp16 it would be 1e-3 to 2e-1.
//
//   1. gram_partial_kernel   lower blocks of U U^T over a run of the longer side, fp32
//                            MFMAs straight from global memory; the momentum update
//   2. gram_reduce_kernel    (128 rows, many runs) sums the runs
//   3. gram_steps_kernel     one workgroup per matrix: the sum, the norm, all the steps
//   4. gram_apply_kernel     Q X_0, rounded to bf16 once
// Three or four launches, against two or more for every step of the general form.
// Bound by the latency of the steps' chain of n x n products (four a step) for few
// matrices, by U's way from HBM for many: 1 x 128 x 2048 bf16 10.4 + 4.6 + 47.3 + 10.2 us
// (102 us in the general form), 1 x 64 x 2048 6.5 + 15.3 + 5.3, 40 x 20 x 300 3.5 + 9.4 + 4.1,
// 14 x 4433 x 111 fp32 22 + 5 + 48 + 25 (its 28 MB in at 1.25 TB/s, the products on values of
// 24 bits taking as long as the loads).
#include "orth_device.hpp"

namespace cap {
namespace {

constexpr int kGramWaves = 4;
constexpr int kGramThreads = kGramWaves * kWave;
constexpr int kMaxSplits = 64;

constexpr int blocks_of(int NB) { return NB * (NB + 1) / 2; }

// Sum over the runs' parts: block t of the lower triangle, lane l: rows 16 i + 4 (l /
// 16) + 0..3, column 16 j + l % 16.
template <int NB, bool BF16, bool MOM>
__global__ __launch_bounds__(kGramThreads) void gram_partial_kernel(Source src, int n, int m, int tall, int vec,
                                                                    int run, f32x4* __restrict__ part) {
    constexpr int NT = blocks_of(NB);
    __shared__ f32x4 sums[NT][kWave];
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const int r = lane & 15, kq = lane >> 4;
    const size_t base = static_cast<size_t>(blockIdx.y) * n * m;
    const int k_end = min(m, static_cast<int>(blockIdx.x + 1) * run);
    f32x4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // this lane's four positions along the longer side, of row 16 i + r
    const bool rows_vec = !tall && vec;
    const size_t step = tall ? n : 1;
    auto place = [&](int k, int i) __attribute__((always_inline)) {
        return base + (tall ? static_cast<size_t>(k) * n + 16 * i + r : static_cast<size_t>(16 * i + r) * m + k);
    };
    Raw4 raw[NB];
    auto load = [&](int k) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < NB; ++i)
            load_raw<BF16, MOM>(src, place(k, i), step, 16 * i + r < n ? k_end - k : 0, rows_vec, raw[i]);
    };
    int k = blockIdx.x * run + wave * 16 + 4 * kq;
    // the next positions are on their way during the products (with 128 rows there are no
    // registers for them)
    constexpr bool kAhead = NB < 8;
    if (kAhead && k - 4 * kq < k_end) load(k);
    for (; k - 4 * kq < k_end; k += kGramWaves * 16) {
        f32x4 u[NB];
#pragma unroll
        for (int i = 0; i < NB; ++i) {
            const int count = 16 * i + r < n ? k_end - k : 0;
            Raw4 x;
            if constexpr (kAhead) x = raw[i];
            else load_raw<BF16, MOM>(src, place(k, i), step, count, rows_vec, x);
            u[i] = finish_u<MOM, true>(src, place(k, i), step, count, rows_vec, x);
        }
        if (kAhead && k - 4 * kq + kGramWaves * 16 < k_end) load(k + kGramWaves * 16);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int j = 0; j <= i; ++j)
                    acc[i * (i + 1) / 2 + j] =
                        __builtin_amdgcn_mfma_f32_16x16x4f32(u[i][e], u[j][e], acc[i * (i + 1) / 2 + j], 0, 0, 0);
    }
    // the waves add their sums in turn
    for (int w = 0; w < kGramWaves; ++w) {
        if (wave == w) {
#pragma unroll
            for (int t = 0; t < NT; ++t) sums[t][lane] = w ? sums[t][lane] + acc[t] : acc[t];
        }
        __syncthreads();
    }
    f32x4* out = part + (static_cast<size_t>(blockIdx.y) * gridDim.x + blockIdx.x) * NT * kWave;
    for (int i = threadIdx.x; i < NT * kWave; i += kGramThreads) out[i] = sums[i / kWave][i % kWave];
}

__global__ __launch_bounds__(kGramThreads) void gram_reduce_kernel(int items, int splits, const f32x4* __restrict__ part,
                                                                   f32x4* __restrict__ sum) {
    const int i = blockIdx.x * kGramThreads + threadIdx.x;
    if (i >= items) return;
    const f32x4* p = part + static_cast<size_t>(blockIdx.y) * splits * items + i;
    f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int k = 0; k < splits; ++k) s += p[static_cast<size_t>(k) * items];
    sum[static_cast<size_t>(blockIdx.y) * items + i] = s;
}

// An n x n matrix of value pairs, rows of NP fp16 padded by 16 bytes (fragment reads,
// 16 rows at one chunk, then hit distinct banks).
template <int NP>
struct Pair {
    static constexpr int kPitch = NP * 2 + 16;
    uint8_t hi[NP * kPitch];
    uint8_t lo[NP * kPitch];
};

template <int NP>
__device__ __forceinline__ f16x8 pair_frag(const uint8_t* p, int row, int chunk) {
    return *reinterpret_cast<const f16x8*>(p + row * Pair<NP>::kPitch + chunk * 16);
}

// The steps of one matrix, in one workgroup: a wave for each lower block (pair of
// blocks a side at 128 rows) of the products.  Q P and P S of a step are one phase.  Up
// to 64 rows S, P S, P and two Q are in LDS and a phase ends in one barrier; at 128
// rows S and P take 139 of the 160 KB: P S replaces S behind a second barrier, and Q
// stays in the waves' registers, a block each, and passes through the place of S while
// the next S waits in registers (through the workspace Q P took 18,000 of a step's
// 33,000 cycles).
template <int NP>
constexpr int step_waves() { return blocks_of(NP == 128 ? 4 : NP / 16); }
template <int NP>
constexpr int step_threads() { return kWave * (step_waves<NP>() < 4 ? 4 : step_waves<NP>()); }

template <int NP, int NB>
__global__ __launch_bounds__(step_threads<NP>()) void gram_steps_kernel(int n, int splits, int steps, StepCoef coef, float eps,
                                                                       const f32x4* __restrict__ part,
                                                                       uint16_t* __restrict__ q_ws,
                                                                       float* __restrict__ scale_out) {
    constexpr int NT = blocks_of(NB);
    constexpr int WB = NP == 128 ? 2 : 1;                    // 16 x 16 blocks of a wave, each way
    constexpr int KS = NP / 32;
    constexpr bool kSmall = NP <= 64;
    constexpr int THREADS = step_threads<NP>();
    __shared__ __attribute__((aligned(16))) Pair<NP> M[kSmall ? 5 : 2];
    __shared__ float red[THREADS / kWave], abc[3 * kMaxOrthSteps];
    constexpr int kSumAhead = NP == 128 ? 4 : 16;            // runs on their way at once
    Pair<NP>&S = M[0], &P = M[1];
    Pair<NP>& T = M[kSmall ? 2 : 0];
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const int r = lane & 15, g = lane >> 4;
    uint16_t* const qw = q_ws + static_cast<size_t>(blockIdx.x) * 2 * NP * NP;   // the result, high and low halves

    // S_0 = U U^T / |U|^2, with |U|^2 its trace.  What does not depend on the runs' sums (block
    // numbers, coefficients) is found while they are on their way.
    constexpr int ITEMS = NT * kWave, PER = (ITEMS + THREADS - 1) / THREADS;
    f32x4 s[PER];
    float trace = 0.0f;
    const f32x4* p[PER];
    int bi[PER], bj[PER];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int it = x * THREADS + threadIdx.x;
        p[x] = part + static_cast<size_t>(blockIdx.x) * splits * ITEMS + (it < ITEMS ? it : ITEMS - 1);
        s[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        triangle(it / kWave, bi[x], bj[x]);
    }
    int si = 0, sj = 0;
    const bool mine = wave < step_waves<NP>();
    if (mine) triangle(wave, si, sj);
    si = __builtin_amdgcn_readfirstlane(si);
    sj = __builtin_amdgcn_readfirstlane(sj);
    if (threadIdx.x < 3 * kMaxOrthSteps) abc[threadIdx.x] = coef.v[threadIdx.x / 3][threadIdx.x % 3];
    for (int k = 0; k < splits; k += kSumAhead) {
        f32x4 v[kSumAhead][PER];
#pragma unroll
        for (int i = 0; i < kSumAhead; ++i)
#pragma unroll
            for (int x = 0; x < PER; ++x) {
                v[i][x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                if (k + i < splits) v[i][x] = p[x][static_cast<size_t>(k + i) * ITEMS];
            }
#pragma unroll
        for (int i = 0; i < kSumAhead; ++i)
#pragma unroll
            for (int x = 0; x < PER; ++x) s[x] += v[i][x];
    }
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int it = x * THREADS + threadIdx.x;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (it < ITEMS && bi[x] == bj[x] && 4 * g + e == r) trace += s[x][e];
    }
    if constexpr (16 * NB < NP)
        for (int i = threadIdx.x; i < static_cast<int>(sizeof(Pair<NP>)) / 16; i += THREADS)
            reinterpret_cast<u32x4*>(&S)[i] = u32x4{0, 0, 0, 0};
#pragma unroll
    for (int o = 32; o; o >>= 1) trace += __shfl_xor(trace, o);
    if (lane == 0) red[wave] = trace;
    __syncthreads();
    trace = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / kWave; ++w) trace += red[w];
    const float norm = sqrtf(trace), scale = 1.0f / (norm + eps);

    auto to_lds = [](Pair<NP>& D) {
        return [&D](int row, int col, const u32x2& hi, const u32x2& lo) __attribute__((always_inline)) {
            *reinterpret_cast<u32x2*>(D.hi + row * Pair<NP>::kPitch + col * 2) = hi;
            *reinterpret_cast<u32x2*>(D.lo + row * Pair<NP>::kPitch + col * 2) = lo;
        };
    };
    auto to_ws = [qw](int row, int col, const u32x2& hi, const u32x2& lo) __attribute__((always_inline)) {
        *reinterpret_cast<u32x2*>(qw + row * NP + col) = hi;
        *reinterpret_cast<u32x2*>(qw + NP * NP + row * NP + col) = lo;
    };
    // four values of row 16 bi + r, columns 16 bj + 4 g .., bj <= bi, and their mirror image.
    // What is stored is symmetric to the last bit: of a block on the diagonal the lower
    // triangle, mirrored.  (P, S and Q commute only up to rounding; with both triangles of such
    // blocks as computed, that difference grew with every step to 1e-1 of the result's norm on
    // matrices of rank 1.)
    auto put = [&](int bi, int bj, const float (&v)[4], auto&& store) __attribute__((always_inline)) {
        u32x2 hi, lo;
        split4_rtz(v, hi, lo);
        const u32x2 th = quad_transpose(hi, lane), tl = quad_transpose(lo, lane);
        const int below = bi != bj ? 1 : (r >> 2) - g;       // of the diagonal: this lane's 4 x 4 values
        if (below == 0) {
            const u32x2 own = {(r & 3) >= 1 ? ~0u : 0xFFFFu, (r & 3) == 3 ? ~0u : (r & 3) == 2 ? 0xFFFFu : 0u};
            hi = (hi & own) | (th & ~own);
            lo = (lo & own) | (tl & ~own);
        }
        if (below >= 0) store(16 * bi + r, 16 * bj + 4 * g, hi, lo);
        if (below > 0) store(16 * bj + 4 * g + (r & 3), 16 * bi + 4 * (r >> 2), th, tl);
    };
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int it = x * THREADS + threadIdx.x;
        if (it >= ITEMS) continue;
        // row 16 bj + r, columns 16 bi + 4 g .. (S is symmetric, each sum the same both ways), and
        // their mirror image
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = s[x][e] * scale * scale;
        u32x2 hi, lo;
        split4_rtz(v, hi, lo);
        to_lds(S)(16 * bj[x] + r, 16 * bi[x] + 4 * g, hi, lo);
        if (bi[x] != bj[x])
            to_lds(S)(16 * bi[x] + 4 * g + (r & 3), 16 * bj[x] + 4 * (r >> 2), quad_transpose(hi, lane), quad_transpose(lo, lane));
    }
    __syncthreads();

    // lower super-block of A B: lane (r, g) holds columns 4 g .. of row r of each block
    typedef float Block[WB][WB][4];
    auto product = [&](const Pair<NP>& A, const Pair<NP>& B, Block& v) __attribute__((always_inline)) {
        f32x4 main[WB][WB], corr[WB][WB];
#pragma unroll
        for (int i = 0; i < WB; ++i)
#pragma unroll
            for (int j = 0; j < WB; ++j) main[i][j] = corr[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            f16x8 ah[WB], al[WB], bh[WB], bl[WB];
#pragma unroll
            for (int i = 0; i < WB; ++i) {
                ah[i] = pair_frag<NP>(A.hi, (si * WB + i) * 16 + r, ks * 4 + g);
                al[i] = pair_frag<NP>(A.lo, (si * WB + i) * 16 + r, ks * 4 + g);
                bh[i] = pair_frag<NP>(B.hi, (sj * WB + i) * 16 + r, ks * 4 + g);
                bl[i] = pair_frag<NP>(B.lo, (sj * WB + i) * 16 + r, ks * 4 + g);
            }
#pragma unroll
            for (int i = 0; i < WB; ++i)
#pragma unroll
                for (int j = 0; j < WB; ++j) {
                    main[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bh[j], ah[i], main[i][j], 0, 0, 0);
                    corr[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bl[j], ah[i], corr[i][j], 0, 0, 0);
                    corr[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(bh[j], al[i], corr[i][j], 0, 0, 0);
                }
        }
#pragma unroll
        for (int i = 0; i < WB; ++i)
#pragma unroll
            for (int j = 0; j < WB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[i][j][e] = __builtin_fmaf(corr[i][j][e], 1.0f / kLoScale, main[i][j][e]);
    };
    auto each = [&](const Block& v, auto&& store) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < WB; ++i)
#pragma unroll
            for (int j = 0; j < WB; ++j)
                if (si * WB + i >= sj * WB + j) put(si * WB + i, sj * WB + j, v[i][j], store);
    };

    Block q;                                                 // at 128 rows
    auto copy = [](const Block& from, Block& to) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < WB; ++i)
#pragma unroll
            for (int j = 0; j < WB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) to[i][j][e] = from[i][j][e];
    };
    for (int it = 0; it < steps; ++it) {
        const float a = abc[3 * it], b = abc[3 * it + 1], c = abc[3 * it + 2];
        const bool last = it + 1 == steps;
        if (mine) {
            Block v;
            product(S, S, v);
#pragma unroll
            for (int i = 0; i < WB; ++i)
#pragma unroll
                for (int j = 0; j < WB; ++j) {
                    const int row = (si * WB + i) * 16 + r, col = (sj * WB + j) * 16 + 4 * g;
                    const u32x2 hi = *reinterpret_cast<const u32x2*>(S.hi + row * Pair<NP>::kPitch + col * 2);
                    const u32x2 lo = *reinterpret_cast<const u32x2*>(S.lo + row * Pair<NP>::kPitch + col * 2);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float sv = __builtin_fmaf(f16_at(lo, e), 1.0f / kLoScale, f16_at(hi, e));
                        const float d = row == col + e && row < n ? a : 0.0f;
                        v[i][j][e] = __builtin_fmaf(c, v[i][j][e], __builtin_fmaf(b, sv, d));
                    }
                }
            each(v, to_lds(P));
            if (it == 0) {                                   // Q = P
                if constexpr (kSmall) {
                    if (last) each(v, to_ws);
                    else each(v, to_lds(M[3]));
                } else {
                    copy(v, q);
                }
            }
        }
        __syncthreads();
        Block t;
        if constexpr (kSmall) {
            if (mine) {
                if (it > 0) {                                // Q <- Q P
                    product(M[3 + ((it - 1) & 1)], P, t);
                    if (last) each(t, to_ws);
                    else each(t, to_lds(M[3 + (it & 1)]));
                }
                if (!last) product(P, S, t);                 // S <- P S P
            }
            if (last) break;
            if (mine) each(t, to_lds(T));
            __syncthreads();
            if (mine) {
                product(T, P, t);
                each(t, to_lds(S));
            }
            __syncthreads();
        } else {
            if (!last) {                                     // t = P S P
                if (mine) product(P, S, t);
                __syncthreads();
                if (mine) each(t, to_lds(T));
                __syncthreads();
                if (mine) product(T, P, t);
                __syncthreads();
            }
            if (it > 0) {                                    // Q <- Q P
                if (mine) each(q, to_lds(T));
                __syncthreads();
                if (mine) product(T, P, q);
                __syncthreads();
            }
            if (last) break;
            if (mine) each(t, to_lds(S));
            __syncthreads();
        }
    }
    if constexpr (!kSmall)
        if (mine) each(q, to_ws);
    // X_0 = |X_0| U / |U|: the applying kernel splits values of U / |U| into fp16, however small
    // an eps well above |U| makes X_0.  (At its place above the next barrier would wait for it.)
    if (threadIdx.x == 0) {
        scale_out[2 * blockIdx.x] = trace == 0.0f ? 0.0f : 1.0f / norm;
        scale_out[2 * blockIdx.x + 1] = norm / (norm + eps);
    }
}

// Q X_0: a wave takes 16 positions of the longer side at a time.
template <int NP, bool BF16, bool MOM>
__global__ __launch_bounds__(kGramThreads) void gram_apply_kernel(Source src, int n, int m, int tall, int vec, int run,
                                                                  const uint16_t* __restrict__ q_ws, int q_stride,
                                                                  const float* __restrict__ scales,
                                                                  uint16_t* __restrict__ out) {
    constexpr int KS = NP / 32;
    __shared__ __attribute__((aligned(16))) Pair<NP> Q;
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const int r = lane & 15, g = lane >> 4;
    const uint16_t* qh = q_ws + static_cast<size_t>(blockIdx.y) * q_stride;
    const uint16_t* ql = qh + NP * NP;
    const float scale = scales[2 * blockIdx.y], size = scales[2 * blockIdx.y + 1];
    const size_t base = static_cast<size_t>(blockIdx.y) * n * m;
    const int end = min(m, static_cast<int>(blockIdx.x + 1) * run);
    // position c0 + r of the longer side, values 32 ks + 8 g + 4 h .. of the shorter
    const bool rows_vec = tall && vec;
    const size_t step = tall ? 1 : m;
    Raw4 raw[KS][2];
    auto place = [&](int c, int k) __attribute__((always_inline)) {
        return base + (tall ? static_cast<size_t>(c) * n + k : static_cast<size_t>(k) * m + c);
    };
    auto load = [&](int c) __attribute__((always_inline)) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = ks * 32 + g * 8 + 4 * h;
                load_raw<BF16, MOM>(src, place(c, k), step, c < end ? n - k : 0, rows_vec, raw[ks][h]);
            }
    };
    int c0 = blockIdx.x * run + wave * 16;
    if (c0 < end) load(c0 + r);
    // all of Q on its way at once
    constexpr int ITEMS = NP * NP / 8, PER = (ITEMS + kGramThreads - 1) / kGramThreads;
    u32x4 q[PER][2];
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = x * kGramThreads + threadIdx.x, at = (i < ITEMS ? i : 0) * 8;
        q[x][0] = *reinterpret_cast<const u32x4*>(qh + at);
        q[x][1] = *reinterpret_cast<const u32x4*>(ql + at);
    }
#pragma unroll
    for (int x = 0; x < PER; ++x) {
        const int i = x * kGramThreads + threadIdx.x, row = i / (NP / 8), c = i % (NP / 8);
        if (i < ITEMS) {
            *reinterpret_cast<u32x4*>(Q.hi + row * Pair<NP>::kPitch + c * 16) = q[x][0];
            *reinterpret_cast<u32x4*>(Q.lo + row * Pair<NP>::kPitch + c * 16) = q[x][1];
        }
    }
    __syncthreads();
    for (; c0 < end; c0 += kGramWaves * 16) {
        f16x8 vh[KS], vl[KS];
        const int c = c0 + r;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            u32x2 hi[2], lo[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const f32x4 u = finish_u<MOM, false>(src, 0, step, 0, rows_vec, raw[ks][h]);
                const float x[4] = {u[0] * scale, u[1] * scale, u[2] * scale, u[3] * scale};
                split4(x, hi[h], lo[h]);
            }
            vh[ks] = __builtin_bit_cast(f16x8, u32x4{hi[0][0], hi[0][1], hi[1][0], hi[1][1]});
            vl[ks] = __builtin_bit_cast(f16x8, u32x4{lo[0][0], lo[0][1], lo[1][0], lo[1][1]});
        }
        // the next are on their way during the products
        if (c0 + kGramWaves * 16 < end) load(c + kGramWaves * 16);
#pragma unroll 2
        for (int i = 0; i < NP / 16; ++i) {
            if (i * 16 >= n) break;
            f32x4 main = {0.0f, 0.0f, 0.0f, 0.0f}, corr = main;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const f16x8 h = pair_frag<NP>(Q.hi, i * 16 + r, ks * 4 + g), l = pair_frag<NP>(Q.lo, i * 16 + r, ks * 4 + g);
                if (tall) {
                    main = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, vh[ks], main, 0, 0, 0);
                    corr = __builtin_amdgcn_mfma_f32_16x16x32_f16(l, vh[ks], corr, 0, 0, 0);
                    corr = __builtin_amdgcn_mfma_f32_16x16x32_f16(h, vl[ks], corr, 0, 0, 0);
                } else {
                    main = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh[ks], h, main, 0, 0, 0);
                    corr = __builtin_amdgcn_mfma_f32_16x16x32_f16(vh[ks], l, corr, 0, 0, 0);
                    corr = __builtin_amdgcn_mfma_f32_16x16x32_f16(vl[ks], h, corr, 0, 0, 0);
                }
            }
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = size * __builtin_fmaf(corr[e], 1.0f / kLoScale, main[e]);
            const u32x2 o = {pack_bf16x2_rne(v[0], v[1]), pack_bf16x2_rne(v[2], v[3])};
            // tall: row c, columns 16 i + 4 g ..; wide: row 16 i + r, columns c0 + 4 g ..
            const int row = tall ? c : i * 16 + r, col = tall ? i * 16 + 4 * g : c0 + 4 * g;
            const int rows_end = tall ? end : n, cols_end = tall ? n : end, pitch = tall ? n : m;
            if (row >= rows_end) continue;
            uint16_t* dst = out + base + static_cast<size_t>(row) * pitch + col;
            if (col + 3 < cols_end && (reinterpret_cast<uintptr_t>(dst) & 7) == 0) {
                *reinterpret_cast<u32x2*>(dst) = o;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < cols_end) dst[e] = static_cast<uint16_t>(o[e >> 1] >> (16 * (e & 1)));
            }
        }
    }
}

struct GramPlan {
    int n, m, NB, NP, splits, run, items, q_values;
    bool reduce;
};

GramPlan gram_plan(int batch, int rows, int cols) {
    GramPlan p;
    p.n = rows < cols ? rows : cols;
    p.m = rows < cols ? cols : rows;
    p.NB = p.n <= 16 ? 1 : p.n <= 32 ? 2 : p.n <= 64 ? 4 : 8;
    p.NP = p.NB < 2 ? 32 : 16 * p.NB;
    p.items = blocks_of(p.NB) * kWave;
    p.q_values = 2 * p.NP * p.NP;                            // of a matrix: high and low halves
    // runs of at least 64 positions (one step of the four waves); about two
    // workgroups a CU over the batch, and no more parts than one workgroup sums soon
    int splits = (512 + batch - 1) / batch;
    // (the steps' kernel has sixteen runs on their way at once, four at 128 rows: few of them up to 64
    // rows, whose runs are short work, 32 x 4096 16.3 us against 17.1 with 64, but 64 x 7168
    // 30.6 with 32 against 32.6 with 16; with 128 rows many, behind a kernel of their own:
    // 128 x 7168 75 us against 90 with 16)
    const int most_splits = p.NB == 8 ? kMaxSplits : p.m > 2048 ? 32 : 16;
    if (splits > most_splits) splits = most_splits;
    const int most = (p.m + 63) / 64;
    if (splits > most) splits = most;
    p.run = ((p.m + splits - 1) / splits + 63) / 64 * 64;
    p.splits = (p.m + p.run - 1) / p.run;
    p.reduce = p.NB == 8 && p.splits > 8;
    return p;
}

size_t align_up(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace

size_t gram_form_bytes(int batch, int rows, int cols) {
    const GramPlan p = gram_plan(batch, rows, cols);
    const size_t b = batch;
    return align_up(b * p.splits * p.items * 16) + align_up(p.reduce ? b * p.items * 16 : 0) +
           align_up(b * p.q_values * 2) + align_up(b * 8);
}

cap_status gram_form_launch(int batch, int rows, int cols, const void* g, bool bf16, float* momentum, float mu,
                            int nesterov, int steps, const StepCoef& coef, float eps, void* out, void* workspace,
                            hipStream_t stream) {
    const GramPlan p = gram_plan(batch, rows, cols);
    const size_t b = batch;
    char* at = static_cast<char*>(workspace);
    f32x4* part = reinterpret_cast<f32x4*>(at);
    at += align_up(b * p.splits * p.items * 16);
    f32x4* sum = reinterpret_cast<f32x4*>(at);
    at += align_up(p.reduce ? b * p.items * 16 : 0);
    uint16_t* q = reinterpret_cast<uint16_t*>(at);
    at += align_up(b * p.q_values * 2);
    float* scale = reinterpret_cast<float*>(at);
    const Source src{g, momentum, mu, nesterov, bf16 ? 1 : 0};
    const int tall = rows > cols, vec = vector_rows(src, cols);
    uint16_t* o = static_cast<uint16_t*>(out);
    // the applying kernel: a workgroup loads Q once for its run; about two workgroups a CU
    int arun = 64;
    while (arun < p.m && static_cast<size_t>((p.m + arun - 1) / arun) * batch > 512) arun += 64;
    const dim3 agrid((p.m + arun - 1) / arun, batch);

    auto go = [&](auto NBc, auto NPc, auto BF, auto MO) {
        constexpr int NB = decltype(NBc)::value, NP = decltype(NPc)::value;
        constexpr bool bf = decltype(BF)::value, mo = decltype(MO)::value;
        gram_partial_kernel<NB, bf, mo><<<dim3(p.splits, batch), kGramThreads, 0, stream>>>(src, p.n, p.m, tall, vec, p.run, part);
        if (p.reduce)
            gram_reduce_kernel<<<dim3((p.items + kGramThreads - 1) / kGramThreads, batch), kGramThreads, 0, stream>>>(
                p.items, p.splits, part, sum);
        gram_steps_kernel<NP, NB><<<batch, step_threads<NP>(), 0, stream>>>(p.n, p.reduce ? 1 : p.splits, steps, coef, eps,
                                                                           p.reduce ? sum : part, q, scale);
        gram_apply_kernel<NP, bf, mo><<<agrid, kGramThreads, 0, stream>>>(src, p.n, p.m, tall, vec, arun, q, p.q_values, scale, o);
    };
    auto by_type = [&](auto NBc, auto NPc) {
        if (bf16 && momentum) go(NBc, NPc, std::true_type{}, std::true_type{});
        else if (bf16) go(NBc, NPc, std::true_type{}, std::false_type{});
        else if (momentum) go(NBc, NPc, std::false_type{}, std::true_type{});
        else go(NBc, NPc, std::false_type{}, std::false_type{});
    };
    using std::integral_constant;
    if (p.NB == 1) by_type(integral_constant<int, 1>{}, integral_constant<int, 32>{});
    else if (p.NB == 2) by_type(integral_constant<int, 2>{}, integral_constant<int, 32>{});
    else if (p.NB == 4) by_type(integral_constant<int, 4>{}, integral_constant<int, 64>{});
    else by_type(integral_constant<int, 8>{}, integral_constant<int, 128>{});
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
