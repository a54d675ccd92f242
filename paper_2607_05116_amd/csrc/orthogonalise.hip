// Orthogonalised gradients: Newton-Schulz steps on a batch of matrices, as
// optimizers that bound an update's spectral norm take them, with the momentum
// that feeds them.
//
//   U  = G                                   (cap_orthogonalise)
//   M <- mu M + G,  U = G + mu M  or  M      (cap_muon_update)
//   X0 = U / (|U|_F + eps);   S = X X^T;   X <- (a I + b S + c S S) X,  steps times
//
// X is held with the shorter side n as its rows ([n][m], transposed on the way in
// and out when the matrix has more rows than columns), so S is n x n.
//
// A step is three products:
//   S (n^2 m);   R = P - p I with P = a I + b S + c S S (n^3);   X <- p X + R X (n^2 m).
// S and R are symmetric: tiles on and below the diagonal, mirrored.  (Two steps in one, with
// S of the second as P S P, would save a product of X each, but their common polynomial is
// a difference of numbers ten times its size where singular values are 1 among others of 0:
// matrices of one to three unequal rows came out with errors of 1e-2 to 2e-2.)
//
// Every product is an MFMA product of fp16 values with fp32 sums whose operands
// are both contiguous along the contraction: S from rows of X, the n x n ones from
// rows of symmetric matrices, the last from rows of Q and rows of X^T, of which a
// second copy is kept.  What is rounded to fp16, and why that is enough:
//   * fp16, not bf16: the singular values stay below 1.3, so the range is known, and
//     steps amplify what rounding adds to small singular values (by a each).
//   * S and R are carried as a multiple of I and the rest (S = s I + D, with s their mean
//     diagonal, in fp32), and only the rest is rounded: with m >> n, or once the singular
//     values are near 1, it is several times smaller.  What rounding takes from R's diagonal
//     is kept in fp32 and joins p: where few rows hold the matrix, R is little else.
//   * X is carried as fp16 and its rounding error, in fp16 too (22 bits), where it is multiplied
//     by p: that error passes on undamped, and in directions whose singular value is 0 each
//     step multiplies it by a.
//   * What is carried is Y = X / u, with u a number of each matrix.  u = 2^-12 (values of X up
//     to 16, and 20 bits of one down to 2^-16, which 65536 x 65536 values of equal size have)
//     while X may have a norm of 1 or more; below, as an eps well above |U| makes it, u
//     follows a bound of |X|, since with a fixed one X would leave the range of fp16.
// Together 3e-4 to 1e-3 of the result's norm for five steps on full ranks, 1e-3 to 3.5e-3 on
// low ones; where two or three unequal rows hold everything a few roundings may agree, and
// 1 in 1000 such matrices has more than 5e-3, none of 12,800 more than 9e-3 (emulated; bf16
// products leave 1e-2 to 1e-1).
//
// Bound by the matrix cores and, where X is the operand, by the results' way through
// memory beside them.  8 x 2048 x 7168 in bf16: 4.6 ms, of which the five Gram products
// take 214 us each (240 of their 481 GFLOP done, the rest mirrored: 1.12 PFLOP/s), the five
// n x n products 87 us and 10 us for joining their parts, the four updates of X 562 us
// each (481 GFLOP, 0.86 PFLOP/s; 2.0 GB read and written) and the last one 455 us (1.06).
// A 8192^3 product of the library reaches 1.39 PFLOP/s on the same card.  A single matrix
// of 256 x 7168 takes 149 us for 22 launches, each 5 to 11 us of latency.
//
// Matrices of at most 128 rows or columns take the Gram form (orth_gram.hip), unless the
// steps' gain is too large for it: 1 x 128 x 2048 takes 71 us there and 102 us here, 40 x 20 x
// 300 16 and 100.
#include "orth_device.hpp"

#include <algorithm>
#include <cmath>

namespace cap {
namespace {

constexpr int kPad = 128;                  // n and m in the workspace are multiples of this

// Tiles of the products, a workgroup's: ROWS x COLS in WM x WN waves.
template <int ROWS_, int COLS_, int WM_, int WN_>
struct Shape {
    static constexpr int ROWS = ROWS_, COLS = COLS_, WM = WM_, WN = WN_, WAVES = WM * WN;
    static constexpr int WR = ROWS / WM, WC = COLS / WN;     // of a wave
    static constexpr int MI = WR / 16, NJ = WC / 16;         // 16 x 16 blocks of a wave
    static constexpr int STEPS = (MI / 2) * (NJ / 2);        // its results' way out (Out)
    static constexpr int BLOCK = ROWS < 128 ? ROWS : 128;    // symmetric products: left out or mirrored by blocks
};
using Big = Shape<256, 256, 4, 2>;
using Mid = Shape<128, 256, 2, 4>;
using Small = Shape<64, 64, 2, 2>;
constexpr int kNormThreads = 256;
constexpr int kMaxNormParts = 256;
// Up to this many rows (or columns) the Gram form (orth_gram.hip) is taken.
constexpr int kGramRows = 128;
constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};

// What the steps may make of noise where the singular value is 0: each multiplies it by a.
float steps_gain(const StepCoef& c, int steps) {
    float now = 0.0f, most = 0.0f;
    for (int i = 0; i < steps; ++i) {
        now = std::fabs(c.v[i][0]) * std::max(now, 1.0f);
        most = std::max(most, now);
    }
    return most;
}
// Up to this gain (five steps of the default have 485) the last product takes X in 11 bits and
// the Gram form may be used.  Past it X's error, the lower 11 bits, is an operand too, and the
// Gram form, whose S takes the gain squared, is left.  Both sides, six and eight steps of the
// default, error by the norm after rounding to bf16 (1.7e-3):
//   256 x 1024 of rank 128   11 bits 8.4e-3, 9.5e-2   both parts 1.9e-3, 2.1e-3
//   64 x 200 of rank 1       Gram 2.8e-3, 8.4e3       here 1.8e-3, 2.4e-3
// and in us for six: 16 x 768 x 2048 851, 1220; 1 x 256 x 7168 176, 182; 8 x 2048 x 7168 5440,
// 9440 (no 256 x 256 tiles); in the Gram form and here: 1 x 128 x 2048 80, 127; 40 x 20 x 300
// 17, 126.
constexpr float kMostGain = 512.0f;

struct OrthWs {
    uint16_t *xh, *xl, *xt[2];             // Y [n][m] in fp16 and its error; Y^T [m][n] (its error beside
                                           // it in rows of 2 n where that is an operand), in turn
    uint16_t* sq[2];                       // D and R, n x n
    float* diag;                           // [batch][np] what rounding took from the diagonal of R
    float* norm;                           // [batch][parts] sums of squares of U
    float* trace;                          // [batch][trace_cap] parts of the next trace
    float* scal;                           // [batch][4] s of the step, |Y|^2, and the units u in turn
    f32x4* sums;                           // of the tiles computed in parts
    int n, m, np, mp;                      // sides, and as padded with zeros
    int parts, trace_cap;
};

int up_to(int v, int q) { return (v + q - 1) / q * q; }

// Parts of a matrix for its norm, of at least 2048 values: two vectors a thread (eight
// single values where the matrices are not aligned, for which a part of 8192 took 12 us on
// 3 x 333 x 517 with momentum).
size_t norm_per_part(int rows, int cols) {
    const size_t size = static_cast<size_t>(rows) * cols;
    const size_t per = (size + kMaxNormParts - 1) / kMaxNormParts;
    return per < 2048 ? 2048 : (per + 3) / 4 * 4;
}
int norm_parts(int rows, int cols) {
    const size_t per = norm_per_part(rows, cols);
    return static_cast<int>((static_cast<size_t>(rows) * cols + per - 1) / per);
}

// How a product runs.  Tiles of a symmetric product that do not fill a round of the chip
// may be computed in parts along K, whose fp32 sums a second kernel joins.
struct ProductPlan {
    int shape, tiles;                      // 0 Big, 1 Mid, 2 Small; tiles of one matrix
    int whole, split;                      // tiles of all matrices computed whole; parts of each of the others
    int grid;
    int traces;                            // places of a trace's parts, of one matrix
    size_t sums;                           // bytes of the parts' sums
    double us;                             // estimated
};

// Tiles of a matrix: all of them, or those with a block on or below the diagonal.
template <typename S>
int count_tiles(bool square, int np, int mp) {
    const int r = (np + S::ROWS - 1) / S::ROWS, c = ((square ? np : mp) + S::COLS - 1) / S::COLS;
    if (!square) return r * c;
    if (S::ROWS == S::COLS) return r * (r + 1) / 2;
    return r / 2 * (r / 2 + 1) + (r % 2 ? r / 2 + 1 : 0);
}

// The rule: the estimated time of each shape, whole or with its last round in `split`
// parts, from what a stage of K = 64 and the way in and out of a tile take (us, measured
// on 2 to 576 tiles of K = 256 to 7168).  Both sides, in us for a whole call:
//                      Big only  Mid only  Small only  by the rule
//   8 x 2048 x 7168      4545      5484      9770        4534 (Big)
//   8 x 1408 x 2048      1003      1064      1262         989 (Big; Mid for X)
//   16 x 768 x 2048       839       712       828         713 (Mid)
//   1 x 256 x 7168        306       232       149         149 (Small)
// and without parts 5016, 993, 714 and 262 (for one Gram product of the first and the
// last: 310 against 214 + 11, 35 against 7 + 5).
ProductPlan plan_product(bool square, int np, int mp, int K, int batch, bool big = true) {
    const int cus = device_cu_count(), KT = K / kStageK;
    ProductPlan best{};
    auto consider = [&](auto shape, int id, int per_cu, double stage, double fixed) {
        using S = decltype(shape);
        const int tiles = count_tiles<S>(square, np, mp), slots = per_cu * cus;
        const long long total = static_cast<long long>(tiles) * batch;
        const long long rounds = total / slots;
        const int rest = static_cast<int>(total % slots);
        const double tile_us = S::ROWS * S::COLS * 4 / 4e6;  // a part's sums one way, 4 MB a us
        for (int split = 1; split <= (square && rest ? 16 : 1); ++split) {
            if (split > 1 && (split * rest > slots || split > KT / 2)) break;
            double us = rounds * (KT * stage + fixed);
            if (rest && split == 1) us += KT * stage + fixed;
            if (split > 1) us += (KT / 2 + split - 1) / split * 2 * stage + fixed + 5.0 + 2.0 * rest * split * tile_us;
            if (best.us > 0.0 && us >= best.us) continue;
            best.us = us;
            best.shape = id;
            best.tiles = tiles;
            best.whole = static_cast<int>(split > 1 ? total - rest : total);
            best.split = split;
            const long long units = best.whole + (split > 1 ? static_cast<long long>(rest) * split : 0);
            best.grid = static_cast<int>(std::min<long long>(units, slots));
            best.traces = tiles * S::WAVES;
            best.sums = split > 1 ? static_cast<size_t>(rest) * split * S::ROWS * S::COLS * 4 : 0;
        }
    };
    if (big) consider(Big{}, 0, 1, 1.42, square ? 10.0 : 22.0);
    consider(Mid{}, 1, 1, 1.05, square ? 7.0 : 12.0);
    consider(Small{}, 2, 2, 0.5, square ? 4.0 : 6.0);
    return best;
}
struct Plans {
    ProductPlan gram, sym, apply, apply2;  // apply2: with X in two parts
};
Plans plan_all(int np, int mp, int batch) {
    return {plan_product(true, np, mp, mp, batch), plan_product(true, np, mp, np, batch),
            plan_product(false, np, mp, np, batch), plan_product(false, np, mp, 2 * np, batch, false)};
}

size_t orth_layout(int batch, int rows, int cols, void* base, OrthWs* w) {
    const int n = rows < cols ? rows : cols, m = rows < cols ? cols : rows;
    const size_t np = up_to(n, kPad), mp = up_to(m, kPad);
    size_t at = 0;
    char* p = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        char* q = p + at;
        at += (bytes + 255) & ~size_t(255);
        return q;
    };
    const size_t x = 2 * batch * np * mp, q = 2 * batch * np * np;
    // tiles of 256 may read 128 rows past a matrix (never used): of the next one, or of
    // what follows here; each kind of matrix is followed by one at least as large
    char* v[6];
    for (int i = 4; i < 6; ++i) v[i] = take(q);
    for (int i = 0; i < 4; ++i) v[i] = take(i < 2 ? x : 2 * x);
    take(static_cast<size_t>(kPad) * np * 4);
    char* d = take(static_cast<size_t>(batch) * np * 4);
    const int parts = norm_parts(rows, cols);
    char* f = take(static_cast<size_t>(batch) * parts * 4);
    const Plans plans = plan_all(static_cast<int>(np), static_cast<int>(mp), batch);
    const size_t cap = std::max(plans.apply.traces, plans.apply2.traces);
    char* t = take(static_cast<size_t>(batch) * cap * 4);
    char* c = take(static_cast<size_t>(batch) * 16);
    char* sums = take(std::max(plans.gram.sums, plans.sym.sums));
    if (w) {
        w->sums = reinterpret_cast<f32x4*>(sums);
        w->xh = reinterpret_cast<uint16_t*>(v[0]);
        w->xl = reinterpret_cast<uint16_t*>(v[1]);
        for (int i = 0; i < 2; ++i) w->xt[i] = reinterpret_cast<uint16_t*>(v[2 + i]);
        for (int i = 0; i < 2; ++i) w->sq[i] = reinterpret_cast<uint16_t*>(v[4 + i]);
        w->diag = reinterpret_cast<float*>(d);
        w->norm = reinterpret_cast<float*>(f);
        w->trace = reinterpret_cast<float*>(t);
        w->scal = reinterpret_cast<float*>(c);
        w->n = n;
        w->m = m;
        w->np = static_cast<int>(np);
        w->mp = static_cast<int>(mp);
        w->parts = parts;
        w->trace_cap = static_cast<int>(cap);
    }
    return at;
}

// ------------------------------------------------------------------ norm and momentum
// Sum of squares of U over this block's part of its matrix; writes the momentum.  Bound by
// HBM: 50 us for 235 MB (4.7 TB/s), 40 us for 46 MB of gradient and 185 MB of momentum.
template <bool BF16, bool MOM>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(Source src, size_t size, size_t per, int parts, int vec,
                                                            float* __restrict__ norm) {
    __shared__ float red[kNormThreads / kWave];
    const size_t base = blockIdx.y * size;
    const size_t a = blockIdx.x * per, b = a + per < size ? a + per : size;
    float sum = 0.0f;
    if (vec) {                                               // per and size are multiples of 4
#pragma unroll 4
        for (size_t i = a + 4 * threadIdx.x; i < b; i += 4 * kNormThreads) {
            const f32x4 u = load_u4<BF16, MOM, true>(src, base + i);
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(u[e], u[e], sum);
        }
    } else {
        // (in the same order: an odd address changes no bit of the result)
        for (size_t i = a + 4 * threadIdx.x; i < b; i += 4 * kNormThreads) {
            float u[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) u[e] = i + e < b ? load_u<BF16, MOM, true>(src, base + i + e) : 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(u[e], u[e], sum);
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        float t = 0.0f;
        for (int w = 0; w < kNormThreads / kWave; ++w) t += red[w];
        norm[static_cast<size_t>(blockIdx.y) * parts + blockIdx.x] = t;
    }
}

constexpr float kUnit = 4096.0f;           // 1 / u, unless X is small
// y = fp16 + fp16, the second unscaled
__device__ __forceinline__ void split_y(const float (&v)[4], u32x2& hi, u32x2& err) {
    hi = u32x2{pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3])};
    float d[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = v[e] - f16_at(hi, e);
    err = u32x2{pack_f16x2(d[0], d[1]), pack_f16x2(d[2], d[3])};
}

// Y0 in both orientations, padded with zeros: 64 x 64 tiles of U through LDS, four
// values a thread at a time.  Bound by HBM: 253 us for 235 MB read and 705 MB written
// (3.7 TB/s; a large copy reaches 5.1).
template <bool BF16, bool MOM>
__global__ __launch_bounds__(256) void start_kernel(Source src, int rows, int cols, int vec, float eps, int two, OrthWs w) {
    __shared__ float tile[64][65];
    __shared__ float scale_s;
    const bool tall = rows > cols;
    const int batch = blockIdx.z;
    const size_t base = static_cast<size_t>(batch) * rows * cols;
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;      // in the matrix as given
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    f32x4 u[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) {
        const int row = r0 + 16 * x + ty, col = c0 + 4 * tx;
        u[x] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (row < rows) {
            const size_t i = base + static_cast<size_t>(row) * cols + col;
            if (vec) {
                if (col < cols) u[x] = load_u4<BF16, MOM, false>(src, i);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (col + e < cols) u[x][e] = load_u<BF16, MOM, false>(src, i + e);
            }
        }
    }
    if (threadIdx.x < kWave) {
        float t = 0.0f;
        for (int i = threadIdx.x; i < w.parts; i += kWave) t += w.norm[static_cast<size_t>(batch) * w.parts + i];
#pragma unroll
        for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
        if (threadIdx.x == 0) {
            const float norm = sqrtf(t), scale = t == 0.0f ? 0.0f : kUnit / norm;
            scale_s = scale;
            if (blockIdx.x == 0 && blockIdx.y == 0) {
                w.trace[static_cast<size_t>(batch) * w.trace_cap] = t * scale * scale;
                w.scal[4 * static_cast<size_t>(batch) + 2] = norm / (norm + eps) / kUnit;
            }
        }
    }
    __syncthreads();
    const float scale = scale_s;
    // as given, [rows][cols] is X of a wide matrix and X^T of a tall one
    const size_t t_pitch = two ? 2 * w.np : w.np;
    uint16_t* const x = w.xh + static_cast<size_t>(batch) * w.np * w.mp;
    uint16_t* const x_err = w.xl + static_cast<size_t>(batch) * w.np * w.mp;
    uint16_t* const xt = w.xt[0] + static_cast<size_t>(batch) * w.mp * t_pitch;
    auto store = [&](const float (&v)[4], bool transposed, int row, int col) __attribute__((always_inline)) {
        u32x2 hi, err;
        split_y(v, hi, err);
        const size_t at = static_cast<size_t>(row) * (transposed ? t_pitch : w.mp) + col;
        *reinterpret_cast<u32x2*>((transposed ? xt : x) + at) = hi;
        if (!transposed) *reinterpret_cast<u32x2*>(x_err + at) = err;
        else if (two) *reinterpret_cast<u32x2*>(xt + w.np + at) = err;
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = u[i][e] * scale;
            tile[16 * i + ty][4 * tx + e] = v[e];
        }
        store(v, tall, r0 + 16 * i + ty, c0 + 4 * tx);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = tile[4 * tx + e][16 * i + ty];
        store(v, !tall, c0 + 16 * i + ty, r0 + 4 * tx);
    }
}

// ------------------------------------------------------------------ products
// The products of a step, with p = a + b s + c s^2 and X = u Y:
//   kGram   D  = u^2 Y Y^T - s I                  s = u^2 |Y|^2 / n
//   kSym    R  = (b + 2 c s) D + c D D            P = p I + R; what rounding takes from R's diagonal
//   kApply  Y <- (u / u') (p Y + R Y): Y, its error, Y^T and the parts of |Y|^2
//   kFinal  u (p Y + R Y) to the bf16 result, in the orientation it is wanted
//   kApply2, kFinal2  the same with Y in two parts: R [Y Y_err], along 2 n
enum Product { kGram, kSym, kApply, kFinal, kApply2, kFinal2 };
constexpr bool is_square(Product m) { return m == kGram || m == kSym; }
constexpr bool is_two(Product m) { return m == kApply2 || m == kFinal2; }
constexpr bool is_final(Product m) { return m == kFinal || m == kFinal2; }
constexpr bool is_apply(Product m) { return m == kApply || m == kApply2; }

struct ProductArgs {
    OrthWs w;
    const uint16_t *A, *B;                 // rows of the left operand; rows (of the transpose) of the right
    uint16_t* D;                           // result; kApply: X^T
    int traces;                            // kGram: parts of |Y|^2
    int turn;                              // which of the two units is the step's
    float coef[3];                         // of the step
    int whole, split;                      // tiles (of all matrices) computed whole, parts of each of the others
    uint16_t* out;
    int rows, cols, batch;
};

struct Scalars {
    float ab, a, i;                        // of A B, A (kApply: Y) and I
    float out;                             // kApply, kFinal: of the sum
};

// Sum of `count` parts by the whole workgroup, in a fixed order.
template <int THREADS>
__device__ __forceinline__ float sum_parts(const float* parts, int count, float* red) {
    float t = 0.0f;
    for (int i = threadIdx.x; i < count; i += THREADS) t += parts[i];
#pragma unroll
    for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
    __syncthreads();
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = t;
    __syncthreads();
    t = 0.0f;
#pragma unroll
    for (int i = 0; i < THREADS / kWave; ++i) t += red[i];
    return t;
}

__device__ __forceinline__ float poly(const float (&c)[3], float s) { return __builtin_fmaf(__builtin_fmaf(c[2], s, c[1]), s, c[0]); }

// The scalars of a product of matrix `batch`; kGram finds its s from the parts and (tile 0
// of the matrix) keeps it for the products after it; so does kApply with the next unit.
// KNOWN: they are kept.
template <Product MODE, int THREADS, bool KNOWN = false>
__device__ __forceinline__ Scalars scalars(const ProductArgs& q, int batch, bool first_tile, float* red) {
    Scalars c{};
    float* k = q.w.scal + 4 * static_cast<size_t>(batch);
    c.ab = 1.0f;
    if constexpr (MODE == kGram) {
        const float* parts = q.w.trace + static_cast<size_t>(batch) * q.w.trace_cap;
        const float t = KNOWN ? k[1] : sum_parts<THREADS>(parts, q.traces, red);
        c.ab = k[2 + q.turn] * k[2 + q.turn];
        const float s = c.ab * t / static_cast<float>(q.w.n);
        if (!KNOWN && first_tile && threadIdx.x == 0) {
            k[0] = s;
            k[1] = t;
        }
        c.i = -s;
    } else if constexpr (MODE == kSym) {
        c.ab = q.coef[2];
        c.a = __builtin_fmaf(2.0f * q.coef[2], k[0], q.coef[1]);
    } else {
        c.a = poly(q.coef, k[0]);
        const float u = k[2 + q.turn];
        c.out = u;
        if constexpr (is_apply(MODE)) {
            // |X'| <= u f, since every singular value's square is at most |X|^2
            const float t = u * u * k[1];
            const float f = __builtin_fmaf(__builtin_fmaf(fabsf(q.coef[2]), t, fabsf(q.coef[1])), t, fabsf(q.coef[0])) * sqrtf(k[1]);
            float next = u;
            c.out = 1.0f;
            if (u * f >= 1.0f) {
                next = 1.0f / kUnit;
                c.out = u * kUnit;
            } else if (f > 0.0f) {
                next = u * f / kUnit;
                c.out = kUnit / f;
            }
            if (first_tile && threadIdx.x == 0) k[2 + (q.turn ^ 1)] = next;
        }
    }
    return c;
}

// LDS row of an operand's tile that holds its row v (0 .. 31) of a pair of 16-row
// blocks, the other way round: LDS row 16 i + r holds row 8 (r / 4) + 4 i + r % 4, so
// that after a transpose within the quads a lane's values of both blocks are eight
// consecutive rows.
__device__ __forceinline__ int paired_row(int v) {
    return (v & ~31) | ((v & 12) << 1) | ((v >> 2) & 4) | (v & 3);
}

// A vector at a scalar base and a lane's 32-bit offset, in global memory.
typedef __attribute__((address_space(1))) char global_char;
template <typename V = u32x4>
__device__ __forceinline__ __attribute__((address_space(1))) V* lane_ptr(const void* base, uint32_t off) {
    return reinterpret_cast<__attribute__((address_space(1))) V*>(
        reinterpret_cast<global_char*>(reinterpret_cast<uint64_t>(uniform_ptr(base))) + off);
}

// What a step of the results adds to: 8 columns a lane of two rows, of A or of X and its
// error, and (kApply) what joins p in these rows.
struct Added {
    u32x4 first[2], second[2];
    float diag[2];
};

// Results leave a wave in steps of 32 x 32 values: two row blocks and two column
// blocks, at (row0, col0) of the matrix.  Lane (r, g) holds columns 4 g .. + 3 of each 16
// x 16 block, of row paired_row.  Two adjacent blocks trade halves (permlane16_swap), so
// that a lane reads and writes 8 consecutive columns: columns 8 (g / 2) .. of block g % 2.
// Addresses are a scalar base for the step and a 32-bit lane offset.

template <Product MODE>
struct Out {
    static constexpr bool kSquare = is_square(MODE);
    static constexpr int kIn = MODE == kGram ? 0 : MODE == kSym ? 1 : 2;      // matrices the results add to
    const ProductArgs& q;
    const Scalars& c;
    int batch, lane, pitch;
    bool mirror;
    uint32_t lane_at, lane_t;
    const uint16_t* p0;

    __device__ __forceinline__ Out(const ProductArgs& q_, const Scalars& c_, int batch_, bool mirror_, int lane_)
        : q(q_), c(c_), batch(batch_), lane(lane_), pitch(kSquare ? q_.w.np : q_.w.mp), mirror(mirror_) {
        const int r = lane & 15, g = lane >> 4;
        lane_at = 2u * ((8 * (r >> 2) + (r & 3)) * pitch + 16 * (g & 1) + 8 * (g >> 1));
        lane_t = 2u * ((4 * g + (r & 3)) * t_pitch() + 8 * (r >> 2));
        p0 = kSquare ? q.A : q.w.xh;
    }
    __device__ __forceinline__ auto at(const uint16_t* p, int row0, int col0, int ii) const {
        return lane_ptr(p + (static_cast<size_t>(batch) * q.w.np + row0 + 4 * ii) * pitch + col0, lane_at);
    }
    __device__ __forceinline__ int t_pitch() const { return is_two(MODE) ? 2 * q.w.np : q.w.np; }
    // of the lane's row ii
    __device__ __forceinline__ int row_of(int row0, int ii) const {
        const int r = lane & 15;
        return row0 + 8 * (r >> 2) + 4 * ii + (r & 3);
    }
    // What N steps side by side add to; steps that share lines of 128 bytes are loaded
    // together, a row block at a time (apart, each line came twice: 467 -> 446 us for the last
    // product of 8 x 2048 x 7168).
    template <int N>
    __device__ __forceinline__ void fetch(Added (&in)[N], int row0, int col0) const {
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
            if constexpr (kIn > 0) {
#pragma unroll
                for (int x = 0; x < N; ++x) in[x].first[ii] = *at(p0, row0, col0 + 32 * x, ii);
            }
            if constexpr (kIn > 1) {
#pragma unroll
                for (int x = 0; x < N; ++x) in[x].second[ii] = *at(q.w.xl, row0, col0 + 32 * x, ii);
                const float d = q.w.diag[static_cast<size_t>(batch) * q.w.np + row_of(row0, ii)];
#pragma unroll
                for (int x = 0; x < N; ++x) in[x].diag[ii] = d;
            }
        }
    }
    // 8 consecutive columns of a row <-> the lane's halves of two blocks
    static __device__ __forceinline__ void halves(const u32x4& v, u32x2& x, u32x2& y) {
        const auto s0 = __builtin_amdgcn_permlane16_swap(v[0], v[2], false, false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(v[1], v[3], false, false);
        x = u32x2{s0[0], s1[0]};
        y = u32x2{s0[1], s1[1]};
    }
    static __device__ __forceinline__ u32x4 join(const u32x2& x, const u32x2& y) {
        const auto s0 = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
        return u32x4{s0[0], s1[0], s0[1], s1[1]};
    }
    __device__ __forceinline__ void bf16_out(int row, int col, const u32x4& y) const {
        if (row >= q.rows) return;
        uint16_t* o = q.out + (static_cast<size_t>(batch) * q.rows + row) * q.cols + col;
        if (col + 7 < q.cols && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
            *reinterpret_cast<u32x4*>(o) = y;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (col + e < q.cols) o[e] = static_cast<uint16_t>(y[e >> 1] >> (16 * (e & 1)));
        }
    }

    // One step: acc[row block][column block], what fetch() brought; returns its part of
    // |Y|^2.
    __device__ __forceinline__ float store(const f32x4 (&acc)[2][2], const Added& in, int row0, int col0) const {
        const int r = lane & 15, g = lane >> 4;
        float sum = 0.0f;
        u32x2 t[2][2], t_err[2][2];                                // transposed
#pragma unroll
        for (int ii = 0; ii < 2; ++ii) {
            const int row = row_of(row0, ii);
            float v[2][4];
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[b][e] = acc[ii][b][e];
            u32x2 hi[2], i0[2], i1[2];
            if constexpr (kIn > 0) halves(in.first[ii], i0[0], i0[1]);
            if constexpr (kIn > 1) halves(in.second[ii], i1[0], i1[1]);
            if constexpr (kSquare) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int d = row - (col0 + 16 * b + 4 * g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        v[b][e] *= c.ab;
                        if constexpr (kIn > 0) v[b][e] = __builtin_fmaf(c.a, f16_at(i0[b], e), v[b][e]);
                        else if (!mirror && d == e && row < q.w.n) v[b][e] += c.i;
                    }
                    hi[b] = u32x2{pack_f16x2(v[b][0], v[b][1]), pack_f16x2(v[b][2], v[b][3])};
                    if constexpr (MODE == kSym) {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (!mirror && d == e)
                                q.w.diag[static_cast<size_t>(batch) * q.w.np + row] = v[b][e] - f16_at(hi[b], e);
                    }
                }
                *at(q.D, row0, col0, ii) = join(hi[0], hi[1]);
            } else {
                const float p = c.a + in.diag[ii];
                u32x2 err[2];
#pragma unroll
                for (int b = 0; b < 2; ++b) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = f16_at(i0[b], e) + f16_at(i1[b], e);
                        v[b][e] = c.out * __builtin_fmaf(p, y, v[b][e]);
                    }
                    if constexpr (is_apply(MODE)) {
                        split_y(v[b], hi[b], err[b]);
                        if constexpr (is_two(MODE)) t_err[ii][b] = quad_transpose(err[b], lane);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(v[b][e], v[b][e], sum);
                    } else {
                        hi[b] = u32x2{pack_bf16x2_rne(v[b][0], v[b][1]), pack_bf16x2_rne(v[b][2], v[b][3])};
                    }
                }
                if constexpr (is_apply(MODE)) {
                    *at(q.w.xh, row0, col0, ii) = join(hi[0], hi[1]);
                    *at(q.w.xl, row0, col0, ii) = join(err[0], err[1]);
                } else if (q.rows <= q.cols) {
                    bf16_out(row, col0 + 16 * (g & 1) + 8 * (g >> 1), join(hi[0], hi[1]));
                }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) t[ii][b] = quad_transpose(hi[b], lane);
        }
        // transposed: row col0 + .. + 4 g + r % 4, eight columns
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const u32x4 y = {t[0][b][0], t[0][b][1], t[1][b][0], t[1][b][1]};
            if constexpr (is_final(MODE)) {
                if (q.rows > q.cols) bf16_out(col0 + 16 * b + 4 * g + (r & 3), row0 + 8 * (r >> 2), y);
            } else if (is_apply(MODE) || mirror) {
                const size_t rows = kSquare ? q.w.np : q.w.mp;
                uint16_t* const d = q.D + (batch * rows + col0 + 16 * b) * t_pitch() + row0;
                *lane_ptr(d, lane_t) = y;
                if constexpr (is_two(MODE))
                    *lane_ptr(d + q.w.np, lane_t) = u32x4{t_err[0][b][0], t_err[0][b][1], t_err[1][b][0], t_err[1][b][1]};
            }
        }
        return sum;
    }
};

// All results of a wave at (row0, col0).  What a pair of steps adds to is loaded a pair
// before, since the loads' way is as long as several steps.  The steps are kept apart
// (sched_barrier): mixed, they need more registers than there are.
template <Product MODE, typename S>
__device__ __forceinline__ float store_wave(const ProductArgs& q, const Scalars& c, f32x4 (&acc)[S::MI][S::NJ], int batch,
                                            int row0, int col0, bool mirror, int lane) {
    constexpr int kAcross = S::NJ / 2, kPair = kAcross < 2 ? 1 : 2;           // steps that share lines
    const Out<MODE> out(q, c, batch, mirror, lane);
    Added in[2][kPair];
    auto fetch = [&](auto X) __attribute__((always_inline)) {
        constexpr int x = decltype(X)::value;
        out.fetch(in[x / kPair % 2], row0 + 32 * (x / kAcross), col0 + 32 * (x % kAcross));
    };
    float sum = 0.0f;
    fetch(std::integral_constant<int, 0>{});
    __builtin_amdgcn_sched_barrier(0);
    static_for<S::STEPS>([&](auto X) __attribute__((always_inline)) {
        constexpr int x = decltype(X)::value, ip = x / kAcross, pr = x % kAcross;
        if constexpr (x % kPair == 0 && x + kPair < S::STEPS) fetch(std::integral_constant<int, x + kPair>{});
        const f32x4 v[2][2] = {{acc[2 * ip][2 * pr], acc[2 * ip][2 * pr + 1]},
                               {acc[2 * ip + 1][2 * pr], acc[2 * ip + 1][2 * pr + 1]}};
        sum += out.store(v, in[x / kPair % 2][x % kPair], row0 + 32 * ip, col0 + 32 * pr);
        __builtin_amdgcn_sched_barrier(0);
    });
    return sum;
}

// The fp32 sums of a part of a product, as a wave holds them: [step][block][lane].
template <typename S>
__device__ __forceinline__ void store_sums(const OrthWs& w, int part, int wave, const f32x4 (&acc)[S::MI][S::NJ], int lane) {
    constexpr int kAcross = S::NJ / 2;
    f32x4* dst = w.sums + (static_cast<size_t>(part) * S::WAVES + wave) * S::STEPS * 4 * kWave;
    static_for<S::STEPS>([&](auto X) __attribute__((always_inline)) {
        constexpr int x = decltype(X)::value, ip = x / kAcross, pr = x % kAcross;
#pragma unroll
        for (int e = 0; e < 4; ++e) dst[(4 * x + e) * kWave + lane] = acc[2 * ip + e / 2][2 * pr + e % 2];
    });
}

// A wave's part of |Y|^2.
__device__ __forceinline__ void store_trace(const ProductArgs& q, int batch, int place, float sum, int lane) {
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) q.w.trace[static_cast<size_t>(batch) * q.w.trace_cap + place] = sum;
}

// The u-th unit of a product's tiles (of all matrices, the matrix outermost): whole
// tiles, then parts along K of the rest.  Parts are runs of an even number of stages.
struct Unit {
    int tile, part;                        // part -1: whole
    int kt0, kt1;                          // stages
};
template <Product MODE>
__device__ __forceinline__ Unit unit_of(const ProductArgs& q, int u, int KT) {
    Unit x{u, -1, 0, KT};
    if constexpr (is_square(MODE)) {
        if (u >= q.whole) {
            const int v = u - q.whole, t = v / q.split, p = v - t * q.split;
            x.tile = q.whole + t;
            x.part = v;
            x.kt0 = (KT / 2) * p / q.split * 2;
            x.kt1 = (KT / 2) * (p + 1) / q.split * 2;
        }
    }
    return x;
}

// Tile t of a matrix: of all, or of those on and below the diagonal.
template <Product MODE, typename S>
__device__ __forceinline__ void decode_tile(const ProductArgs& q, int t, int& ti, int& tj) {
    if constexpr (!is_square(MODE)) {
        const int tm = (q.w.np + S::ROWS - 1) / S::ROWS;
        ti = t % tm;
        tj = t / tm;
    } else if constexpr (S::ROWS == S::COLS) {
        triangle(t, ti, tj);
    } else {                                                 // row tiles 2 p and 2 p + 1 have p + 1 each
        static_assert(S::COLS == 2 * S::ROWS, "row tiles in pairs");
        int p = static_cast<int>((sqrtf(4.0f * static_cast<float>(t) + 1.0f) - 1.0f) * 0.5f);
        while (p * (p + 1) > t) --p;
        while ((p + 1) * (p + 2) <= t) ++p;
        const int rest = t - p * (p + 1), second = rest > p;
        ti = 2 * p + second;
        tj = rest - second * (p + 1);
    }
}

// What becomes of a wave's block at (row0, col0): in a symmetric product the blocks above
// the diagonal are left out, those below it mirrored.
template <Product MODE, typename S>
struct Place {
    bool store, mirror;
    __device__ __forceinline__ Place(const OrthWs& w, int row0, int col0) {
        const int r = row0 / S::BLOCK, c = col0 / S::BLOCK;
        if constexpr (is_square(MODE)) {
            store = row0 < w.np && col0 < w.np && c <= r;
            mirror = c < r;
        } else {
            store = row0 < w.np && col0 < w.mp;
            mirror = true;
        }
    }
};

// ---- Mid and Small: a ring of K = 64 stages that runs on across the tiles of a workgroup,
// all but one of them in flight.  (The two waves of a SIMD taking turns at reading fragments
// and multiplying, a barrier apart, were 2 to 7 % slower on the 128 x 256 tiles.)
template <typename S>
struct Ring {
    static constexpr int kStages = S::ROWS == 64 ? 4 : 3;                     // 64 or 144 KB
    static constexpr int kStageB = (S::ROWS + S::COLS) * kRowB;
    static constexpr int kA = S::ROWS / kRowsPerLoad / S::WAVES, kB = S::COLS / kRowsPerLoad / S::WAVES;   // loads of a wave
    static constexpr int kPerCu = S::ROWS == 64 ? 2 : 1;
};

template <Product MODE, typename S>
__global__ __launch_bounds__(S::WAVES * kWave, Ring<S>::kPerCu) void product_ring_kernel(ProductArgs q, int tiles, int units) {
    using R = Ring<S>;
    constexpr int THREADS = S::WAVES * kWave;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[R::kStages * R::kStageB];
    __shared__ float red[S::WAVES];
    const OrthWs& w = q.w;
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const int wm = wave / S::WN, wn = wave % S::WN;
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    constexpr int kParts = is_two(MODE) ? 2 : 1;                     // of the right operand, along K
    const int lead = MODE == kGram ? w.mp : w.np, KT = kParts * lead / kStageK;
    const uint32_t pitch = static_cast<uint32_t>(lead) * 2u;
    const LaneMap lm = lane_map(lane);
    const int G = gridDim.x;
    int unit = G % 8 == 0 ? (blockIdx.x % 8) * (G / 8) + blockIdx.x / 8 : blockIdx.x;
    if (unit >= units) return;

    struct Tile { int batch, t, ti, tj, part, kt0, stages; };
    auto decode = [&](int x) __attribute__((always_inline)) {
        const Unit u = unit_of<MODE>(q, x, KT);
        Tile T;
        T.part = __builtin_amdgcn_readfirstlane(u.part);
        T.kt0 = __builtin_amdgcn_readfirstlane(u.kt0);
        T.stages = __builtin_amdgcn_readfirstlane(u.kt1 - u.kt0);
        T.batch = __builtin_amdgcn_readfirstlane(u.tile / tiles);
        T.t = __builtin_amdgcn_readfirstlane(u.tile) - T.batch * tiles;
        int ti, tj;
        decode_tile<MODE, S>(q, T.t, ti, tj);
        T.ti = __builtin_amdgcn_readfirstlane(ti);
        T.tj = __builtin_amdgcn_readfirstlane(tj);
        return T;
    };
    // the load cursor, all but one stage ahead: a wave brings kA (kB) runs of eight rows
    uint32_t a_off[R::kA], b_off[R::kB];
#pragma unroll
    for (int i = 0; i < R::kA; ++i)
        a_off[i] = paired_row((wave * R::kA + i) * kRowsPerLoad + lm.ld_row) * pitch + lm.col_b[(wave * R::kA + i) & 1];
#pragma unroll
    for (int i = 0; i < R::kB; ++i)
        b_off[i] = ((wave * R::kB + i) * kRowsPerLoad + lm.ld_row) * kParts * pitch + lm.col_b[(wave * R::kB + i) & 1];
    const char *pa = nullptr, *pb = nullptr;
    int it_unit = unit, it_left = 0, it_buf = 0;
    auto cursor = [&]() __attribute__((always_inline)) {
        const Tile T = decode(it_unit);
        const size_t b_rows = is_square(MODE) ? w.np : w.mp;
        pa = reinterpret_cast<const char*>(q.A + (static_cast<size_t>(T.batch) * w.np + T.ti * S::ROWS) * lead + T.kt0 * kStageK);
        pb = reinterpret_cast<const char*>(q.B + (T.batch * b_rows + T.tj * S::COLS) * kParts * lead + T.kt0 * kStageK);
        it_left = T.stages;
    };
    auto issue = [&]() __attribute__((always_inline)) {
        const uint32_t at = lds_base + it_buf * R::kStageB;
        static_for<R::kA>([&](auto I) { lds_dma16(pa, a_off[I.value], at + (wave * R::kA + I.value) * 1024); });
        static_for<R::kB>(
            [&](auto I) { lds_dma16(pb, b_off[I.value], at + S::ROWS * kRowB + (wave * R::kB + I.value) * 1024); });
        it_buf = it_buf + 1 == R::kStages ? 0 : it_buf + 1;
        if (--it_left > 0) {
            pa += kRowB;
            pb += kRowB;
            if constexpr (is_two(MODE))
                if (it_left == KT / 2) pa -= pitch;                  // the left operand again, for the second part
        } else if (it_unit + G < units) {
            it_unit += G;
            cursor();
        } else {
            it_left = 1;                   // past the end: the last stage again, so that the counts of loads in flight hold
        }
    };
    cursor();
#pragma unroll 1
    for (int i = 0; i < R::kStages - 1; ++i) issue();
    int buf = 0;
    const int pc[2] = {(lm.fr_kc ^ lm.fr_swz) << 4, ((lm.fr_kc ^ lm.fr_swz) << 4) ^ 64};
    for (; unit < units; unit += G) {
        const Tile T = decode(unit);
        const int row0 = T.ti * S::ROWS + wm * S::WR, col0 = T.tj * S::COLS + wn * S::WC;
        const Place<MODE, S> place(w, row0, col0);
        f32x4 acc[S::MI][S::NJ];
#pragma unroll
        for (int i = 0; i < S::MI; ++i)
#pragma unroll
            for (int j = 0; j < S::NJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
        for (int kt = 0; kt < T.stages; ++kt) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the stage before has been read
            wait_vm<(R::kStages - 2) * (R::kA + R::kB)>();                                 // this wave's part of this one has landed
            block_barrier();
            issue();                                                 // into the buffer of the stage before
            const uint8_t* la = lds + buf * R::kStageB + (wm * S::WR + lm.fr_row) * kRowB;
            const uint8_t* lb = lds + buf * R::kStageB + (S::ROWS + wn * S::WC + lm.fr_row) * kRowB;
            buf = buf + 1 == R::kStages ? 0 : buf + 1;
            if (!place.store) continue;                              // wave-uniform
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                f16x8 a[S::MI], b[S::NJ];
#pragma unroll
                for (int i = 0; i < S::MI; ++i) a[i] = frag_at<f16x8>(la + i * 16 * kRowB + pc[ks]);
#pragma unroll
                for (int j = 0; j < S::NJ; ++j) b[j] = frag_at<f16x8>(lb + j * 16 * kRowB + pc[ks]);
#pragma unroll
                for (int i = 0; i < S::MI; ++i)
#pragma unroll
                    for (int j = 0; j < S::NJ; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[j], a[i], acc[i][j], 0, 0, 0);
            }
        }
        if (is_square(MODE) && T.part >= 0) {
            store_sums<S>(w, T.part, wave, acc, lane);
            if (T.t == 0 && T.kt0 == 0) scalars<MODE, THREADS>(q, T.batch, true, red);
            continue;
        }
        const Scalars c = scalars<MODE, THREADS>(q, T.batch, T.t == 0, red);
        float sum = 0.0f;
        if (place.store) sum = store_wave<MODE, S>(q, c, acc, T.batch, row0, col0, place.mirror, lane);
        if constexpr (is_apply(MODE)) store_trace(q, T.batch, T.t * S::WAVES + wave, sum, lane);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// ---- Big: the K loop of mfma_tile.hpp
static_assert(Big::ROWS == kBM && Big::COLS == kBN && Big::WM == kWavesM && Big::WN == kWavesN, "the K loop's tile");

template <Product MODE>
__global__ __launch_bounds__(kNW * kWave, 1) void product_big_kernel(ProductArgs q, int tiles, int units) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[kStages * kStageBytes];
    __shared__ float red[kNW];
    const OrthWs& w = q.w;
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const bool loader = wave < kNL;
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    const uint32_t a_lds = lds_base + wave * kALd * 1024;
    const uint32_t b_lds = lds_base + (kBM + (wave >> 1) * kWN + (wave & 1) * 16) * kRowB;
    const int KT = (MODE == kGram ? w.mp : w.np) / kStageK, lead = MODE == kGram ? w.mp : w.np;
    // block b runs on XCD b % 8: each XCD gets a run of tiles, mostly of one matrix
    const int G = gridDim.x;
    int tile = G % 8 == 0 ? (blockIdx.x % 8) * (G / 8) + blockIdx.x / 8 : blockIdx.x;
    int batch = 0, t = 0, ti = 0, tj = 0, part = -1, stages = KT;
    bool first = true;
    Loads ld;
    auto start_tile = [&](int x) __attribute__((always_inline)) {
        const Unit u = unit_of<MODE>(q, x, KT);
        part = __builtin_amdgcn_readfirstlane(u.part);
        first = u.kt0 == 0;
        stages = __builtin_amdgcn_readfirstlane(u.kt1 - u.kt0);
        batch = __builtin_amdgcn_readfirstlane(u.tile / tiles);
        t = __builtin_amdgcn_readfirstlane(u.tile) - batch * tiles;
        decode_tile<MODE, Big>(q, t, ti, tj);
        ti = __builtin_amdgcn_readfirstlane(ti);
        tj = __builtin_amdgcn_readfirstlane(tj);
        if (!loader) return;
        const LaneMap lm = lane_map(opaque(lane));
        const uint32_t pitch = static_cast<uint32_t>(lead) * 2u;
        const size_t b_rows = is_square(MODE) ? w.np : w.mp;
        const uint16_t* A = q.A + (static_cast<size_t>(batch) * w.np + static_cast<size_t>(ti) * kBM) * lead;
        const uint16_t* B = q.B + (batch * b_rows + static_cast<size_t>(tj) * kBN + (wave >> 1) * kWN + (wave & 1) * 16) * lead;
        const int k0 = is_square(MODE) ? u.kt0 * kStageK : 0;
        ld.a = reinterpret_cast<const char*>(A + k0);
        ld.a_on = ti * kBM + wave / kWavesN * kWM < w.np;
        ld.b0 = reinterpret_cast<const char*>(B + k0);
        ld.b1 = ld.b0 + static_cast<size_t>(32) * pitch;
        ld.c0 = ld.b0 + static_cast<size_t>(64) * pitch;
        ld.c1 = ld.b0 + static_cast<size_t>(96) * pitch;
#pragma unroll
        for (int i = 0; i < 2; ++i) ld.b_off[i] = (i * kRowsPerLoad + lm.ld_row) * pitch + lm.col_b[i];
        // (a loader whose own rows lie past the end loads none: its rows come after them)
#pragma unroll
        for (int i = 0; i < kALd; ++i)
            ld.a_off[i] = static_cast<uint32_t>(paired_row(wave * kALd * kRowsPerLoad + i * kRowsPerLoad + lm.ld_row)) * pitch +
                          lm.col_b[i & 1];
        load_half0(ld, ld.a_on, a_lds, b_lds, 0);
        load_half1(ld, b_lds, 0);
    };
    if (tile < units) start_tile(tile);
    while (tile < units) {
        f32x4 acc[kMI][kNJ];
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
            for (int j = 0; j < kNJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
        const bool cfirst = first;
        const int cb = batch, ct = t, ci = ti, cj = tj, cp = part, ck = is_square(MODE) ? stages : KT;
        const int next = tile + G;
        // in the last stage buffer 0 is free: the next tile's stage 0 lands during the
        // rest of that stage and the results' way out
        auto hook = [&](auto step) {
            if constexpr (decltype(step)::value == kLast) {
                if (next < units) start_tile(next);
            }
        };
        const bool active = ci * kBM + wm * kWM < w.np;
        run_k_loop<f16x8>(ck, lds, wm, wn, lane, loader, active, acc, ld, a_lds, b_lds, hook, hook);
        if (is_square(MODE) && cp >= 0) {
            store_sums<Big>(w, cp, wave, acc, lane);
            if (ct == 0 && cfirst) scalars<MODE, kNW * kWave>(q, cb, true, red);
            tile = next;
            continue;
        }
        const Scalars c = scalars<MODE, kNW * kWave>(q, cb, ct == 0, red);
        const int row0 = ci * kBM + wm * kWM, col0 = cj * kBN + wn * kWN;
        const Place<MODE, Big> place(w, row0, col0);
        float sum = 0.0f;
        if (place.store) sum = store_wave<MODE, Big>(q, c, acc, cb, row0, col0, place.mirror, opaque(lane));
        if constexpr (is_apply(MODE)) store_trace(q, cb, ct * Big::WAVES + wave, sum, lane);
        tile = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Joins the parts of the tiles computed in parts: one wave for a step of a wave of the
// tile.
template <Product MODE, typename S>
__global__ __launch_bounds__(kWave) void join_kernel(ProductArgs q, int tiles) {
    const int lane = threadIdx.x;
    const int wave = blockIdx.x / S::STEPS, x = blockIdx.x % S::STEPS;
    const int tile = q.whole + blockIdx.y, batch = tile / tiles, t = tile - batch * tiles;
    int ti, tj;
    decode_tile<MODE, S>(q, t, ti, tj);
    const int row0 = ti * S::ROWS + wave / S::WN * S::WR + 32 * (x / (S::NJ / 2));
    const int col0 = tj * S::COLS + wave % S::WN * S::WC + 32 * (x % (S::NJ / 2));
    const Scalars c = scalars<MODE, kWave, true>(q, batch, false, nullptr);
    const Place<MODE, S> place(q.w, row0, col0);
    if (place.store) {
        const Out<MODE> out(q, c, batch, place.mirror, lane);
        Added in[1];
        out.fetch(in, row0, col0);
        f32x4 acc[2][2] = {};
        const f32x4* p = q.w.sums + ((static_cast<size_t>(blockIdx.y) * q.split * S::WAVES + wave) * S::STEPS + x) * 4 * kWave + lane;
#pragma unroll 4
        for (int i = 0; i < q.split; ++i) {
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[e / 2][e % 2] += p[e * kWave];
            p += static_cast<size_t>(S::WAVES) * S::STEPS * 4 * kWave;
        }
        out.store(acc, in[0], row0, col0);
    }
}

template <Product MODE>
void launch_product(const ProductArgs& args, const ProductPlan& p, hipStream_t stream) {
    ProductArgs q = args;
    q.whole = p.whole;
    q.split = p.split;
    const int rest = p.tiles * q.batch - p.whole, units = p.whole + rest * p.split;
    auto join = [&](auto shape) {
        using S = decltype(shape);
        if constexpr (is_square(MODE))
            if (rest) join_kernel<MODE, S><<<dim3(S::WAVES * S::STEPS, rest), kWave, 0, stream>>>(q, p.tiles);
    };
    if (p.shape == 0) {
        if constexpr (!is_two(MODE)) {
            product_big_kernel<MODE><<<p.grid, Big::WAVES * kWave, 0, stream>>>(q, p.tiles, units);
            join(Big{});
        }
    } else if (p.shape == 1) {
        product_ring_kernel<MODE, Mid><<<p.grid, Mid::WAVES * kWave, 0, stream>>>(q, p.tiles, units);
        join(Mid{});
    } else {
        product_ring_kernel<MODE, Small><<<p.grid, Small::WAVES * kWave, 0, stream>>>(q, p.tiles, units);
        join(Small{});
    }
}

// Matrices of at most 128 rows or columns that the Gram form leaves are taken in parts of the
// batch whose workspace stays below this (or one by one), since their sides are padded to 128.
constexpr size_t kMostPadded = size_t(256) << 20;
int batch_part(int batch, int rows, int cols) {
    if ((rows < cols ? rows : cols) > kGramRows) return batch;
    const size_t one = orth_layout(1, rows, cols, nullptr, nullptr);
    return static_cast<int>(std::max<size_t>(1, std::min<size_t>(batch, kMostPadded / one)));
}

void general_launch(bool bf16, int batch, int rows, int cols, const void* g, float* momentum, float mu, int nesterov, int steps,
                    const StepCoef& sc, bool two, float eps, void* out, void* workspace, hipStream_t stream) {
    const Source src{g, momentum, mu, nesterov, bf16 ? 1 : 0};
    ProductArgs q{};
    orth_layout(batch, rows, cols, workspace, &q.w);
    const OrthWs& w = q.w;
    q.out = static_cast<uint16_t*>(out);
    q.rows = rows;
    q.cols = cols;
    q.batch = batch;
    const size_t size = static_cast<size_t>(rows) * cols;
    const bool tall = rows > cols;
    const dim3 ngrid(w.parts, batch);
    const dim3 sgrid((tall ? w.np : w.mp) / 64, (tall ? w.mp : w.np) / 64, batch);
    auto begin = [&](auto BF, auto MOM) {
        constexpr bool bf = decltype(BF)::value, mo = decltype(MOM)::value;
        norm_kernel<bf, mo><<<ngrid, kNormThreads, 0, stream>>>(src, size, norm_per_part(rows, cols), w.parts,
                                                               vector_rows(src, size % 4 == 0 ? 4 : 1), w.norm);
        start_kernel<bf, mo><<<sgrid, 256, 0, stream>>>(src, rows, cols, vector_rows(src, cols), eps, two, w);
    };
    if (bf16 && momentum) begin(std::true_type{}, std::true_type{});
    else if (bf16) begin(std::true_type{}, std::false_type{});
    else if (momentum) begin(std::false_type{}, std::true_type{});
    else begin(std::false_type{}, std::false_type{});
    const Plans plans = plan_all(w.np, w.mp, batch);
    int from = 0, traces = 1;
    auto set = [&](uint16_t* A, uint16_t* B, uint16_t* D) {
        q.A = A;
        q.B = B;
        q.D = D;
    };
    for (int i = 0; i < steps; ++i) {
        for (int j = 0; j < 3; ++j) q.coef[j] = sc.v[i][j];
        q.traces = traces;
        q.turn = i & 1;
        set(w.xh, w.xh, w.sq[0]);
        launch_product<kGram>(q, plans.gram, stream);                    // D
        set(w.sq[0], w.sq[0], w.sq[1]);
        launch_product<kSym>(q, plans.sym, stream);                      // R
        set(w.sq[1], w.xt[from], w.xt[from ^ 1]);
        if (two) {
            if (i + 1 < steps) launch_product<kApply2>(q, plans.apply2, stream);
            else launch_product<kFinal2>(q, plans.apply2, stream);
        } else {
            if (i + 1 < steps) launch_product<kApply>(q, plans.apply, stream);
            else launch_product<kFinal>(q, plans.apply, stream);
        }
        from ^= 1;
        traces = two ? plans.apply2.traces : plans.apply.traces;
    }
}

}  // namespace

size_t orthogonalise_workspace_bytes(int batch, int rows, int cols) {
    const int part = batch_part(batch, rows, cols);
    size_t bytes = std::max(orth_layout(part, rows, cols, nullptr, nullptr),
                            orth_layout(batch % part ? batch % part : part, rows, cols, nullptr, nullptr));
    // (the form goes by the coefficients too)
    if ((rows < cols ? rows : cols) <= kGramRows) bytes = std::max(bytes, gram_form_bytes(batch, rows, cols));
    return bytes;
}

cap_status orthogonalise_launch(cap_dtype dtype, int batch, int rows, int cols, const void* g, float* momentum, float mu,
                                int nesterov, int steps, const float* coef, float eps, void* out, void* workspace,
                                hipStream_t stream) {
    StepCoef sc;
    for (int i = 0; i < kMaxOrthSteps; ++i)
        for (int j = 0; j < 3; ++j) sc.v[i][j] = coef && i < steps ? coef[3 * i + j] : kQuintic[j];
    const bool bf16 = dtype == CAP_DTYPE_BF16;
    const bool two = !(steps_gain(sc, steps) <= kMostGain);
    if ((rows < cols ? rows : cols) <= kGramRows && !two)
        return gram_form_launch(batch, rows, cols, g, bf16, momentum, mu, nesterov, steps, sc, eps, out, workspace, stream);
    const int part = batch_part(batch, rows, cols);
    for (int from = 0; from < batch; from += part) {
        const size_t at = static_cast<size_t>(from) * rows * cols;
        general_launch(bf16, std::min(part, batch - from), rows, cols, static_cast<const char*>(g) + at * (bf16 ? 2 : 4),
                       momentum ? momentum + at : nullptr, mu, nesterov, steps, sc, two, eps, static_cast<uint16_t*>(out) + at,
                       workspace, stream);
        CAP_LAUNCH_CHECK();
    }
    return CAP_OK;
}

}  // namespace cap
