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
// Steps go in groups of one or two: the first two and the last two are pairs, the
// others single.  A pair needs X once, since S of its second step is P S P with P =
// a I + b S + c S S (polynomials of one symmetric matrix commute):
//   S (n^2 m), then n x n products:  R = P - p I;   T = P S;   S' = T P;  R' = P' - p' I;
//   Q = P P';   X <- Q X (2 n^2 m).
// All n x n products are symmetric: tiles on and below the diagonal, mirrored.  Five
// steps take 9 n^2 m + 11 n^3 multiply-adds, single steps 15 n^2 m + 5 n^3, and X is
// read and written three times instead of five.
//
// Every product is an MFMA product of fp16 values with fp32 sums whose operands
// are both contiguous along the contraction: S from rows of X, the n x n ones from
// rows of symmetric matrices, the last from rows of Q and rows of X^T, of which a
// second copy is kept.  What is rounded to fp16, and why that is enough:
//   * fp16, not bf16: the singular values stay below 1.3, so the range is known, and
//     steps amplify what rounding adds to small singular values (by a each).
//   * S, P, T and Q are carried as a multiple of I and the rest (S = s I + D, with s
//     their mean diagonal, in fp32), and only the rest is rounded: with m >> n, or once
//     the singular values are near 1, it is several times smaller.
//   * X is carried to 22 bits (a second fp16 with its rounding error, scaled by 2^11)
//     where it is multiplied by the multiple of I, which passes its error on undamped.
// Together 3e-4 to 1.3e-3 of the result's norm on square, wide, low-rank and 1/i spectra,
// 2.5e-3 where they fall by e^-12; bf16 products leave 1e-2 to 1e-1.  A pair in the middle
// or three steps in one group lose more (up to 3e-3 and 2e-2): the noise of S' grows by
// a^2 with each step taken on it.
//
// Matrices of at most 128 rows or columns take the Gram form (orth_gram.hip).
#include "orth_device.hpp"

namespace cap {
namespace {

constexpr int kPad = 128;                  // n and m in the workspace are multiples of this
constexpr int kNormThreads = 256;
constexpr int kMaxNormParts = 256;
// Up to this many rows (or columns) the Gram form (orth_gram.hip) is taken.
constexpr int kGramRows = 128;
constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};

struct OrthWs {
    uint16_t *xh, *xl, *xt[2];             // X [n][m]: fp16 and its scaled error; X^T [m][n], in turn
    uint16_t* sq[3];                       // n x n
    float* norm;                           // [batch][parts] sums of squares of U
    float* trace;                          // [batch][trace_cap] parts of the next trace
    float* center;                         // [batch][2] s of the group's first and second step
    int n, m, np, mp, parts, trace_cap;
};

int up_to(int v, int q) { return (v + q - 1) / q * q; }

int norm_parts(int rows, int cols) {
    const long long per = 64 * 1024;       // values per block
    const long long want = (static_cast<long long>(rows) * cols + per - 1) / per;
    return static_cast<int>(want < kMaxNormParts ? want : kMaxNormParts);
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
    char* v[7];
    for (int i = 4; i < 7; ++i) v[i] = take(q);
    for (int i = 0; i < 4; ++i) v[i] = take(x);
    take(static_cast<size_t>(kPad) * mp * 2);
    const int parts = norm_parts(rows, cols);
    char* f = take(static_cast<size_t>(batch) * parts * 4);
    const size_t cap = (np / 128) * (mp / 128);
    char* t = take(static_cast<size_t>(batch) * cap * 4);
    char* c = take(static_cast<size_t>(batch) * 8);
    if (w) {
        w->xh = reinterpret_cast<uint16_t*>(v[0]);
        w->xl = reinterpret_cast<uint16_t*>(v[1]);
        for (int i = 0; i < 2; ++i) w->xt[i] = reinterpret_cast<uint16_t*>(v[2 + i]);
        for (int i = 0; i < 3; ++i) w->sq[i] = reinterpret_cast<uint16_t*>(v[4 + i]);
        w->norm = reinterpret_cast<float*>(f);
        w->trace = reinterpret_cast<float*>(t);
        w->center = reinterpret_cast<float*>(c);
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
// Sum of squares of U over this block's part of its matrix; writes the momentum.
template <bool BF16, bool MOM>
__global__ __launch_bounds__(kNormThreads) void norm_kernel(Source src, size_t size, int parts,
                                                            float* __restrict__ norm) {
    __shared__ float red[kNormThreads / kWave];
    const size_t base = blockIdx.y * size;
    const size_t per = (size + parts - 1) / parts;
    const size_t a = blockIdx.x * per, b = a + per < size ? a + per : size;
    float sum = 0.0f;
    for (size_t i = a + threadIdx.x; i < b; i += kNormThreads) {
        const float u = load_u<BF16, MOM, true>(src, base + i);
        sum = __builtin_fmaf(u, u, sum);
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

// X0 in both orientations, padded with zeros: 64 x 64 tiles of U through LDS.
template <bool BF16, bool MOM>
__global__ __launch_bounds__(256) void start_kernel(Source src, int rows, int cols, float eps, OrthWs w) {
    __shared__ float tile[64][65];
    __shared__ float scale_s;
    const bool tall = rows > cols;
    const int batch = blockIdx.z;
    if (threadIdx.x < kWave) {
        float t = 0.0f;
        for (int i = threadIdx.x; i < w.parts; i += kWave) t += w.norm[static_cast<size_t>(batch) * w.parts + i];
#pragma unroll
        for (int o = 32; o; o >>= 1) t += __shfl_xor(t, o);
        if (threadIdx.x == 0) {
            const float scale = 1.0f / (sqrtf(t) + eps);
            scale_s = scale;
            // the trace of S_0
            if (blockIdx.x == 0 && blockIdx.y == 0) w.trace[static_cast<size_t>(batch) * w.trace_cap] = t * scale * scale;
        }
    }
    __syncthreads();
    const float scale = scale_s;
    const size_t base = static_cast<size_t>(batch) * rows * cols;
    const int r0 = blockIdx.y * 64, c0 = blockIdx.x * 64;      // in the matrix as given
    const int tx = threadIdx.x % 64, ty = threadIdx.x / 64;
    for (int r = ty; r < 64; r += 4) {
        float u = 0.0f;
        if (r0 + r < rows && c0 + tx < cols) {
            const size_t i = base + static_cast<size_t>(r0 + r) * cols + c0 + tx;
            u = load_u<BF16, MOM, false>(src, i);
        }
        tile[r][tx] = u * scale;
    }
    __syncthreads();
    const size_t xb = static_cast<size_t>(batch) * w.np * w.mp;
    // as given: [rows][cols] goes to X (wide) or to X^T (tall)
    for (int r = ty; r < 64; r += 4) {
        const float v = tile[r][tx], u = tile[tx][r];
        const _Float16 hv = static_cast<_Float16>(v), hu = static_cast<_Float16>(u);
        const int ra = r0 + r, ca = c0 + tx;                   // element v
        const int rb = c0 + r, cb = r0 + tx;                   // element u, transposed
        const float x = tall ? u : v;
        const _Float16 h = tall ? hu : hv;
        const size_t nat = tall ? xb + static_cast<size_t>(rb) * w.mp + cb : xb + static_cast<size_t>(ra) * w.mp + ca;
        const size_t tra = tall ? xb + static_cast<size_t>(ra) * w.np + ca : xb + static_cast<size_t>(rb) * w.np + cb;
        w.xh[nat] = __builtin_bit_cast(uint16_t, h);
        w.xl[nat] = __builtin_bit_cast(uint16_t, static_cast<_Float16>((x - static_cast<float>(h)) * kLoScale));
        w.xt[0][tra] = __builtin_bit_cast(uint16_t, tall ? hv : hu);
    }
}

// ------------------------------------------------------------------ products
// kGram:  D = X X^T - s I, s = its trace / n
// kSym:   one of the group's n x n products (Sym)
// kApply: X <- p X + Q X: X, its error, X^T and the parts of |X|^2
// kFinal: the same to the bf16 result, in the orientation it is wanted
enum Product { kGram, kSym, kApply, kFinal };

// The n x n products of a group, with p = a + b s + c s^2 of the first step's
// coefficients and s, p' of the second's:
//   kSymFirst:  R  = (b + 2 c s) D + c D D               (P = p I + R)
//   kSymMix:    T  = p D + s R + R D                     (P S = p s I + T), parts of tr(P S P)
//   kSymNext:   D' = p T + p s R + T R + (p^2 s - s') I  (P S P = s' I + D')
//   kSymSecond: R' = kSymFirst of the second step
//   kSymJoin:   Q  = p R' + p' R + R R'                  (P P' = p p' I + Q)
enum Sym { kSymFirst, kSymMix, kSymNext, kSymSecond, kSymJoin };

struct ProductArgs {
    OrthWs w;
    const uint16_t *A, *B;                 // rows of the left operand; rows (of the transpose) of the right
    uint16_t* D;                           // kSym, kGram: result; kApply: X^T
    int sym, traces;                       // kSym: which; kGram, kSymNext: parts of the trace
    float coef[2][3];                      // of the group's steps
    int pair;
    uint16_t* out;
    int rows, cols, batch;
};

struct Scalars {
    float ab, a, b, i;                     // of A B, A, B and I
    float s1;                              // kSymNext: s'
    float p, ps;                           // kSymMix: the multiples of I in P and T
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

// The scalars of a product of matrix `batch`; kGram and kSymNext find their s from the
// parts and (tile 0 of the matrix) keep it for the products after them.
template <Product MODE, int THREADS>
__device__ __forceinline__ Scalars scalars(const ProductArgs& q, int batch, bool first_tile, float* red) {
    Scalars c{};
    float* center = q.w.center + 2 * static_cast<size_t>(batch);
    const float* parts = q.w.trace + static_cast<size_t>(batch) * q.w.trace_cap;
    c.ab = 1.0f;
    if constexpr (MODE == kGram) {
        const float s = sum_parts<THREADS>(parts, q.traces, red) / static_cast<float>(q.w.n);
        if (first_tile && threadIdx.x == 0) center[0] = s;
        c.i = -s;
    } else {
        const float s = center[0];
        const float p = poly(q.coef[0], s);
        if constexpr (MODE == kSym) {
            if (q.sym == kSymFirst) {
                c.ab = q.coef[0][2];
                c.a = __builtin_fmaf(2.0f * q.coef[0][2], s, q.coef[0][1]);
            } else if (q.sym == kSymMix) {
                c.a = s;
                c.b = p;
                c.p = p;
                c.ps = p * s;
            } else if (q.sym == kSymNext) {
                c.s1 = sum_parts<THREADS>(parts, q.traces, red) / static_cast<float>(q.w.n);
                if (first_tile && threadIdx.x == 0) center[1] = c.s1;
                c.a = p;
                c.b = p * s;
                c.i = p * p * s - c.s1;
            } else if (q.sym == kSymSecond) {
                c.ab = q.coef[1][2];
                c.a = __builtin_fmaf(2.0f * q.coef[1][2], center[1], q.coef[1][1]);
            } else {
                c.a = poly(q.coef[1], center[1]);
                c.b = p;
            }
        } else {
            c.a = q.pair ? p * poly(q.coef[1], center[1]) : p;
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

// Results of a wave's 64 x 16 NJ block at (row0, col0) of the matrix.  Lane (r, g)
// holds columns 4 g .. + 3 of each 16 x 16 block, of row paired_row.  Two adjacent
// blocks trade halves (permlane16_swap), so that a lane reads and writes 8 consecutive
// columns: columns 8 (g / 2) .. of block g % 2.
template <Product MODE, int NJ>
__device__ __forceinline__ float store_wave(const ProductArgs& q, const Scalars& c, f32x4 (&acc)[4][NJ], int batch, int row0,
                                            int col0, bool mirror, int lane) {
    const OrthWs& w = q.w;
    const int r = lane & 15, g = lane >> 4;
    constexpr bool kSquare = MODE == kGram || MODE == kSym;
    const size_t pitch = kSquare ? w.np : w.mp;
    const size_t xb = static_cast<size_t>(batch) * w.np * w.mp, sb = static_cast<size_t>(batch) * w.np * w.np;
    const size_t base = kSquare ? sb : xb;
    const bool use_a = MODE == kSym, use_b = MODE == kSym && c.b != 0.0f;
    float sum = 0.0f;
    // 8 consecutive columns of a row: the lane's halves of two blocks
    auto load_pair = [&](const uint16_t* p, size_t at, u32x2& x, u32x2& y) __attribute__((always_inline)) {
        const u32x4 v = *reinterpret_cast<const u32x4*>(p + at);
        const auto s0 = __builtin_amdgcn_permlane16_swap(v[0], v[2], false, false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(v[1], v[3], false, false);
        x = u32x2{s0[0], s1[0]};
        y = u32x2{s0[1], s1[1]};
    };
    auto join_pair = [&](const u32x2& x, const u32x2& y) __attribute__((always_inline)) {
        const auto s0 = __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false);
        return u32x4{s0[0], s1[0], s0[1], s1[1]};
    };
#pragma unroll
    for (int ip = 0; ip < 2; ++ip)
#pragma unroll
        for (int pr = 0; pr < NJ / 2; ++pr) {
            u32x2 t[2][2];                                         // [row block][column block], transposed
#pragma unroll
            for (int ii = 0; ii < 2; ++ii) {
                const int row = row0 + 32 * ip + 8 * (r >> 2) + 4 * ii + (r & 3);
                const int c8 = col0 + 32 * pr + 16 * (g & 1) + 8 * (g >> 1);
                const size_t at = base + static_cast<size_t>(row) * pitch + c8;
                float v[2][4];
#pragma unroll
                for (int b = 0; b < 2; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[b][e] = acc[2 * ip + ii][2 * pr + b][e];
                u32x2 hi[2], lo[2];
                if constexpr (kSquare) {
                    u32x2 ea[2], eb[2];
                    if (use_a) load_pair(q.A, at, ea[0], ea[1]);
                    if (use_b) load_pair(q.B, at, eb[0], eb[1]);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int col = col0 + 32 * pr + 16 * b + 4 * g + e;
                            const bool diag = row == col && row < w.n;
                            float x = c.ab * v[b][e];
                            if (use_a) x = __builtin_fmaf(c.a, f16_at(ea[b], e), x);
                            if (use_b) x = __builtin_fmaf(c.b, f16_at(eb[b], e), x);
                            if (diag) x += c.i;
                            if constexpr (MODE == kSym)
                                if (q.sym == kSymMix)                  // P and T whole
                                    sum = __builtin_fmaf(diag ? x + c.ps : x, f16_at(ea[b], e) + (diag ? c.p : 0.0f), sum);
                            v[b][e] = x;
                        }
                        hi[b] = u32x2{pack_f16x2(v[b][0], v[b][1]), pack_f16x2(v[b][2], v[b][3])};
                    }
                    *reinterpret_cast<u32x4*>(q.D + at) = join_pair(hi[0], hi[1]);
                    if (mirror) {
#pragma unroll
                        for (int b = 0; b < 2; ++b) t[ii][b] = quad_transpose(hi[b], lane);
                    }
                } else {
                    u32x2 xh[2], xl[2];
                    load_pair(w.xh, at, xh[0], xh[1]);
                    load_pair(w.xl, at, xl[0], xl[1]);
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float x = __builtin_fmaf(f16_at(xl[b], e), 1.0f / kLoScale, f16_at(xh[b], e));
                            v[b][e] = __builtin_fmaf(c.a, x, v[b][e]);
                        }
                        if constexpr (MODE == kApply) {
                            split4(v[b], hi[b], lo[b]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum = __builtin_fmaf(v[b][e], v[b][e], sum);
                            t[ii][b] = quad_transpose(hi[b], lane);
                        } else {
                            hi[b] = u32x2{pack_bf16x2_rne(v[b][0], v[b][1]), pack_bf16x2_rne(v[b][2], v[b][3])};
                            if (q.rows > q.cols) t[ii][b] = quad_transpose(hi[b], lane);
                        }
                    }
                    if constexpr (MODE == kApply) {
                        *reinterpret_cast<u32x4*>(w.xh + at) = join_pair(hi[0], hi[1]);
                        *reinterpret_cast<u32x4*>(w.xl + at) = join_pair(lo[0], lo[1]);
                    } else if (q.rows <= q.cols) {
                        const u32x4 y = join_pair(hi[0], hi[1]);
                        if (row < q.rows) {
                            uint16_t* o = q.out + (static_cast<size_t>(batch) * q.rows + row) * q.cols + c8;
                            if (c8 + 7 < q.cols && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
                                *reinterpret_cast<u32x4*>(o) = y;
                            } else {
#pragma unroll
                                for (int e = 0; e < 8; ++e)
                                    if (c8 + e < q.cols) o[e] = static_cast<uint16_t>(y[e >> 1] >> (16 * (e & 1)));
                            }
                        }
                    }
                }
            }
            // transposed: row col0 + .. + 4 g + r % 4, eight columns
            const int tc = row0 + 32 * ip + 8 * (r >> 2);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int tr = col0 + 32 * pr + 16 * b + 4 * g + (r & 3);
                const u32x4 y = {t[0][b][0], t[0][b][1], t[1][b][0], t[1][b][1]};
                if constexpr (kSquare) {
                    if (mirror) *reinterpret_cast<u32x4*>(q.D + sb + static_cast<size_t>(tr) * w.np + tc) = y;
                } else if constexpr (MODE == kApply) {
                    *reinterpret_cast<u32x4*>(q.D + xb + static_cast<size_t>(tr) * w.np + tc) = y;
                } else if (q.rows > q.cols && tr < q.rows) {
                    uint16_t* o = q.out + (static_cast<size_t>(batch) * q.rows + tr) * q.cols + tc;
                    if (tc + 7 < q.cols && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
                        *reinterpret_cast<u32x4*>(o) = y;
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (tc + e < q.cols) o[e] = static_cast<uint16_t>(y[e >> 1] >> (16 * (e & 1)));
                    }
                }
            }
        }
    return sum;
}

// This tile's part of a trace (off the diagonal it stands for two tiles).
template <int THREADS>
__device__ __forceinline__ void store_part(const ProductArgs& q, int batch, int tile, float sum, float* red) {
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    __syncthreads();
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        float t = 0.0f;
        for (int i = 0; i < THREADS / kWave; ++i) t += red[i];
        q.w.trace[static_cast<size_t>(batch) * q.w.trace_cap + tile] = t;
    }
}

template <Product MODE>
__device__ __forceinline__ void decode_tile(const ProductArgs& q, int t, int tile_rows, int& ti, int& tj) {
    if constexpr (MODE == kGram || MODE == kSym) {
        triangle(t, ti, tj);
    } else {
        const int tm = (q.w.np + tile_rows - 1) / tile_rows;
        ti = t % tm;
        tj = t / tm;
    }
}

// ---- tiles of 128 x 128: four waves of 64 x 64, two workgroups a CU
constexpr int kT = 128;
constexpr int kThreads = 256;
constexpr int kTileStageB = 2 * kT * kRowB;

template <Product MODE>
__global__ __launch_bounds__(kThreads, 2) void product128_kernel(ProductArgs q) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kTileStageB];
    __shared__ float red[kThreads / kWave];
    const OrthWs& w = q.w;
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const int wm = wave >> 1, wn = wave & 1;
    const int batch = blockIdx.y;
    int ti, tj;
    decode_tile<MODE>(q, blockIdx.x, kT, ti, tj);
    const size_t xb = static_cast<size_t>(batch) * w.np * w.mp, sb = static_cast<size_t>(batch) * w.np * w.np;
    const int K = MODE == kGram ? w.mp : w.np;
    const uint16_t* A = q.A + (MODE == kGram ? xb : sb);
    const uint16_t* B = q.B + (MODE == kSym ? sb : xb);
    const uint32_t pitch = static_cast<uint32_t>(K) * 2u;
    const LaneMap lm = lane_map(lane);
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    // wave w brings rows 32 w .. + 31 of both operands, eight at a time
    const char* pa = reinterpret_cast<const char*>(A + (static_cast<size_t>(ti) * kT + wave * 32) * K);
    const char* pb = reinterpret_cast<const char*>(B + (static_cast<size_t>(tj) * kT + wave * 32) * K);
    uint32_t a_off[4], b_off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a_off[i] = paired_row(i * 8 + lm.ld_row) * pitch + lm.col_b[i & 1];
        b_off[i] = (i * 8 + lm.ld_row) * pitch + lm.col_b[i & 1];
    }
    auto issue = [&](int buf) __attribute__((always_inline)) {
        const uint32_t at = lds_base + buf * kTileStageB + wave * 32 * kRowB;
        static_for<4>([&](auto I) { lds_dma16(pa, a_off[I.value], at + I.value * 1024); });
        static_for<4>([&](auto I) { lds_dma16(pb, b_off[I.value], at + kT * kRowB + I.value * 1024); });
        pa += kRowB;
        pb += kRowB;
    };
    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
    const int KT = K / kStageK;
    const int pc[2] = {(lm.fr_kc ^ lm.fr_swz) << 4, ((lm.fr_kc ^ lm.fr_swz) << 4) ^ 64};
    issue(0);
    for (int kt = 0; kt < KT; ++kt) {
        const int buf = kt & 1;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // the stage before has been read
        wait_vm<0>();                                            // this wave's part of the stage has landed
        block_barrier();
        if (kt + 1 < KT) issue(buf ^ 1);
        const uint8_t* la = lds + buf * kTileStageB + (wm * 64 + lm.fr_row) * kRowB;
        const uint8_t* lb = lds + buf * kTileStageB + (kT + wn * 64 + lm.fr_row) * kRowB;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            f16x8 a[4], b[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = frag_at<f16x8>(la + i * 16 * kRowB + pc[ks]);
#pragma unroll
            for (int j = 0; j < 4; ++j) b[j] = frag_at<f16x8>(lb + j * 16 * kRowB + pc[ks]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(b[j], a[i], acc[i][j], 0, 0, 0);
        }
    }
    const Scalars c = scalars<MODE, kThreads>(q, batch, blockIdx.x == 0, red);
    const float sum = store_wave<MODE, 4>(q, c, acc, batch, ti * kT + wm * 64, tj * kT + wn * 64, ti != tj, lane);
    if (MODE == kApply || (MODE == kSym && q.sym == kSymMix))
        store_part<kThreads>(q, batch, blockIdx.x, MODE == kSym && ti != tj ? 2.0f * sum : sum, red);
}

// ---- tiles of 256 x 256: the K loop of mfma_tile.hpp, persistent, one workgroup a CU
template <Product MODE>
__global__ __launch_bounds__(kNW * kWave, 1) void product256_kernel(ProductArgs q, int tiles) {
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
    const int K = MODE == kGram ? w.mp : w.np;
    const int KT = K / kStageK;
    const size_t xb = static_cast<size_t>(w.np) * w.mp, sb = static_cast<size_t>(w.np) * w.np;
    const int total = tiles * q.batch;
    // block b runs on XCD b % 8: each XCD gets a run of tiles, mostly of one matrix
    const int G = gridDim.x;
    int tile = G % 8 == 0 ? (blockIdx.x % 8) * (G / 8) + blockIdx.x / 8 : blockIdx.x;
    int batch = 0, t = 0, ti = 0, tj = 0;
    Loads ld;
    auto start_tile = [&](int x) __attribute__((always_inline)) {
        batch = __builtin_amdgcn_readfirstlane(x / tiles);
        t = x - batch * tiles;
        decode_tile<MODE>(q, t, kBM, ti, tj);
        ti = __builtin_amdgcn_readfirstlane(ti);
        tj = __builtin_amdgcn_readfirstlane(tj);
        if (!loader) return;
        const LaneMap lm = lane_map(opaque(lane));
        const uint32_t pitch = static_cast<uint32_t>(K) * 2u;
        const uint16_t* A = q.A + batch * (MODE == kGram ? xb : sb) + static_cast<size_t>(ti) * kBM * K;
        const uint16_t* B = q.B + batch * (MODE == kSym ? sb : xb) +
                            (static_cast<size_t>(tj) * kBN + (wave >> 1) * kWN + (wave & 1) * 16) * K;
        ld.a = reinterpret_cast<const char*>(A);
        ld.a_on = ti * kBM + wave / kWavesN * kWM < w.np;
        ld.b0 = reinterpret_cast<const char*>(B);
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
    if (tile < total) start_tile(tile);
    while (tile < total) {
        f32x4 acc[kMI][kNJ];
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
            for (int j = 0; j < kNJ; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][j][e] = 0.0f;
        const int cb = batch, ct = t, ci = ti, cj = tj;
        const int next = tile + G;
        // in the last stage buffer 0 is free: the next tile's stage 0 lands during the
        // rest of that stage and the results' way out
        auto hook = [&](auto step) {
            if constexpr (decltype(step)::value == kLast) {
                if (next < total) start_tile(next);
            }
        };
        const bool active = ci * kBM + wm * kWM < w.np;
        run_k_loop<f16x8>(KT, lds, wm, wn, lane, loader, active, acc, ld, a_lds, b_lds, hook, hook);
        const Scalars c = scalars<MODE, kNW * kWave>(q, cb, ct == 0, red);
        float sum = 0.0f;
        if (active && cj * kBN + wn * kWN < (MODE == kGram || MODE == kSym ? w.np : w.mp))
            sum = store_wave<MODE, kNJ>(q, c, acc, cb, ci * kBM + wm * kWM, cj * kBN + wn * kWN, ci != cj, opaque(lane));
        if (MODE == kApply || (MODE == kSym && q.sym == kSymMix))
            store_part<kNW * kWave>(q, cb, ct, MODE == kSym && ci != cj ? 2.0f * sum : sum, red);
        tile = next;
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

// Which tiles a product runs on: 256 x 256 (one workgroup a CU) or 128 x 128 (two).
bool wide_tiles(int big, int small, int batch) {
    const long long cus = device_cu_count();
    const long long rounds256 = (static_cast<long long>(big) * batch + cus - 1) / cus;
    const long long rounds128 = (static_cast<long long>(small) * batch + 2 * cus - 1) / (2 * cus);
    return rounds256 * 24 <= rounds128 * 16;
}

template <Product MODE>
void launch_product(const ProductArgs& q, hipStream_t stream) {
    const OrthWs& w = q.w;
    constexpr bool square = MODE == kGram || MODE == kSym;
    auto tiles = [&](int t) {
        const int r = (w.np + t - 1) / t, c = ((square ? w.np : w.mp) + t - 1) / t;
        return square ? r * (r + 1) / 2 : r * c;
    };
    const int big = tiles(kBM);
    if (wide_tiles(big, tiles(kT), q.batch)) {
        const long long total = static_cast<long long>(big) * q.batch;
        const int cus = device_cu_count();
        product256_kernel<MODE><<<total < cus ? static_cast<int>(total) : cus, kNW * kWave, 0, stream>>>(q, big);
    } else {
        product128_kernel<MODE><<<dim3(tiles(kT), q.batch), kThreads, 0, stream>>>(q);
    }
}

}  // namespace

size_t orthogonalise_workspace_bytes(int batch, int rows, int cols) {
    if ((rows < cols ? rows : cols) <= kGramRows) return gram_form_bytes(batch, rows, cols);
    return orth_layout(batch, rows, cols, nullptr, nullptr);
}

cap_status orthogonalise_launch(cap_dtype dtype, int batch, int rows, int cols, const void* g, float* momentum, float mu,
                                int nesterov, int steps, const float* coef, float eps, void* out, void* workspace,
                                hipStream_t stream) {
    StepCoef sc;
    for (int i = 0; i < kMaxOrthSteps; ++i)
        for (int j = 0; j < 3; ++j) sc.v[i][j] = coef && i < steps ? coef[3 * i + j] : kQuintic[j];
    const bool bf16 = dtype == CAP_DTYPE_BF16;
    if ((rows < cols ? rows : cols) <= kGramRows)
        return gram_form_launch(batch, rows, cols, g, bf16, momentum, mu, nesterov, steps, sc, eps, out, workspace, stream);
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
        norm_kernel<bf, mo><<<ngrid, kNormThreads, 0, stream>>>(src, size, w.parts, w.norm);
        start_kernel<bf, mo><<<sgrid, 256, 0, stream>>>(src, rows, cols, eps, w);
    };
    if (bf16 && momentum) begin(std::true_type{}, std::true_type{});
    else if (bf16) begin(std::true_type{}, std::false_type{});
    else if (momentum) begin(std::false_type{}, std::true_type{});
    else begin(std::false_type{}, std::false_type{});
    CAP_LAUNCH_CHECK();
    auto tri_tiles = [&](int side) { return side * (side + 1) / 2; };
    const int t256 = (w.np + kBM - 1) / kBM, t128 = w.np / kT;
    const int sym_tiles = wide_tiles(tri_tiles(t256), tri_tiles(t128), batch) ? tri_tiles(t256) : tri_tiles(t128);
    const int a256 = t256 * ((w.mp + kBN - 1) / kBN), a128 = t128 * (w.mp / kT);
    const int apply_tiles = wide_tiles(a256, a128, batch) ? a256 : a128;
    int from = 0, traces = 1;
    auto sym = [&](int which, uint16_t* A, uint16_t* B, uint16_t* D) {
        q.sym = which;
        q.A = A;
        q.B = B;
        q.D = D;
        q.traces = sym_tiles;
        launch_product<kSym>(q, stream);
    };
    for (int i = 0; i < steps;) {
        q.pair = (i == 0 && steps >= 4) || i == steps - 2;
        for (int h = 0; h < 2; ++h)
            for (int j = 0; j < 3; ++j) q.coef[h][j] = sc.v[q.pair ? i + h : i][j];
        q.A = q.B = w.xh;
        q.D = w.sq[0];
        q.traces = traces;
        launch_product<kGram>(q, stream);                          // D
        sym(kSymFirst, w.sq[0], w.sq[0], w.sq[1]);                   // R
        uint16_t* Q = w.sq[1];
        if (q.pair) {
            sym(kSymMix, w.sq[1], w.sq[0], w.sq[2]);                  // T
            sym(kSymNext, w.sq[2], w.sq[1], w.sq[0]);                 // D'
            sym(kSymSecond, w.sq[0], w.sq[0], w.sq[2]);               // R'
            sym(kSymJoin, w.sq[1], w.sq[2], w.sq[0]);                 // Q
            Q = w.sq[0];
        }
        q.A = Q;
        q.B = w.xt[from];
        q.D = w.xt[from ^ 1];
        i += q.pair ? 2 : 1;
        if (i < steps) launch_product<kApply>(q, stream);
        else launch_product<kFinal>(q, stream);
        from ^= 1;
        traces = apply_tiles;
    }
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
