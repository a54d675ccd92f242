// Orthogonalised gradients: Newton-Schulz steps on a batch of matrices, as
// optimizers that bound an update's spectral norm take them, with the momentum
// that feeds them.
//
//   U  = G                                   (cap_orthogonalise)
//   M <- mu M + G,  U = G + mu M  or  M      (cap_muon_update)
//   X0 = U / (|U|_F + eps);   S = X X^T;   X <- a X + (b S + c S S) X,  steps times
//
// X is held with the shorter side n as its rows ([n][m], transposed on the way in
// and out when the matrix has more rows than columns), so S is n x n and a step
// costs 3 n^2 m + n^3 multiply-adds with both symmetric products (S and S S)
// computed on and below the diagonal and mirrored.
//
// Every product is an MFMA product of fp16 values with fp32 sums whose operands
// are both contiguous along the contraction: S from rows of X; S S from rows of S
// (it is symmetric); the last from rows of b S + c S S and rows of X^T, of which a
// second copy is kept.  fp16, not bf16: |X|_2 <= 1.3 at every step, so the range
// is known, and the steps amplify what rounding adds to small singular values;
// its 11 bits leave 1 to 2e-3 of the result's norm where bf16 leaves 1 to 3e-2.
// X itself is carried to 22 bits (a second fp16 with the rounding error, scaled by
// 2^11), because a X passes its rounding on undamped: rounding X to fp16 at each
// step doubles the error on square or decaying spectra.
#include "orth_device.hpp"

namespace cap {
namespace {

constexpr int kPad = 128;                  // n and m in the workspace are multiples of this
constexpr int kT = 128;                    // tile of the products
constexpr int kThreads = 256;              // four waves of 64 x 64
constexpr int kTileStageB = 2 * kT * kRowB;
constexpr int kNormThreads = 256;
constexpr int kMaxNormParts = 256;
// Up to this many rows (or columns) the Gram form (orth_gram.hip) is taken.
constexpr int kGramRows = 128;
constexpr float kQuintic[3] = {3.4445f, -4.7750f, 2.0315f};

struct OrthWs {
    uint16_t *xh, *xl, *xt[2], *s, *p;
    float* norm;                           // [batch][parts] sums of squares
    int n, m, np, mp, parts;
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
    char* v[6];
    for (int i = 0; i < 4; ++i) v[i] = take(x);
    for (int i = 4; i < 6; ++i) v[i] = take(q);
    const int parts = norm_parts(rows, cols);
    char* f = take(static_cast<size_t>(batch) * parts * 4);
    if (w) {
        w->xh = reinterpret_cast<uint16_t*>(v[0]);
        w->xl = reinterpret_cast<uint16_t*>(v[1]);
        w->xt[0] = reinterpret_cast<uint16_t*>(v[2]);
        w->xt[1] = reinterpret_cast<uint16_t*>(v[3]);
        w->s = reinterpret_cast<uint16_t*>(v[4]);
        w->p = reinterpret_cast<uint16_t*>(v[5]);
        w->norm = reinterpret_cast<float*>(f);
        w->n = n;
        w->m = m;
        w->np = static_cast<int>(np);
        w->mp = static_cast<int>(mp);
        w->parts = parts;
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
        if (threadIdx.x == 0) scale_s = 1.0f / (sqrtf(t) + eps);
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
// kGram: S = X X^T; kPoly: P = b S + c S S; kApply: X <- a X + P X (X, its error
// and X^T); kFinal: the same to the bf16 result, in the orientation it is wanted.
enum Product { kGram, kPoly, kApply, kFinal };

struct ProductArgs {
    OrthWs w;
    int from;                              // X^T buffer that holds X
    float a, b, c;
    uint16_t* out;
    int rows, cols;
};

template <Product MODE>
__global__ __launch_bounds__(kThreads, 2) void product_kernel(ProductArgs q) {
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kTileStageB];
    const OrthWs& w = q.w;
    const int lane = threadIdx.x % kWave;
    const int wave = static_cast<int>(__builtin_amdgcn_readfirstlane(threadIdx.x / kWave));
    const int wm = wave >> 1, wn = wave & 1;
    const size_t xb = static_cast<size_t>(blockIdx.y) * w.np * w.mp, sb = static_cast<size_t>(blockIdx.y) * w.np * w.np;
    int ti, tj;
    if constexpr (MODE == kGram || MODE == kPoly) {
        triangle(blockIdx.x, ti, tj);
    } else {
        const int tm = w.np / kT;
        ti = blockIdx.x % tm;
        tj = blockIdx.x / tm;
    }
    const int K = MODE == kGram ? w.mp : w.np;
    const uint16_t* A = MODE == kGram ? w.xh + xb : MODE == kPoly ? w.s + sb : w.p + sb;
    const uint16_t* B = MODE == kGram ? w.xh + xb : MODE == kPoly ? w.s + sb : w.xt[q.from] + xb;
    const uint32_t pitch = static_cast<uint32_t>(K) * 2u;
    const LaneMap lm = lane_map(lane);
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    // wave w brings rows 32 w .. + 31 of both operands, eight at a time
    const char* pa = reinterpret_cast<const char*>(A + (static_cast<size_t>(ti) * kT + wave * 32) * K);
    const char* pb = reinterpret_cast<const char*>(B + (static_cast<size_t>(tj) * kT + wave * 32) * K);
    uint32_t off[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) off[i] = (i * 8 + lm.ld_row) * pitch + lm.col_b[i & 1];
    auto issue = [&](int buf) __attribute__((always_inline)) {
        const uint32_t at = lds_base + buf * kTileStageB + wave * 32 * kRowB;
        static_for<4>([&](auto I) { lds_dma16(pa, off[I.value], at + I.value * 1024); });
        static_for<4>([&](auto I) { lds_dma16(pb, off[I.value], at + kT * kRowB + I.value * 1024); });
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
    // lane (r, g) holds columns 4 g .. + 3 of row r of each 16 x 16 block
    const int r = lm.fr_row, g = lane >> 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int row = ti * kT + wm * 64 + i * 16 + r, col = tj * kT + wn * 64 + j * 16 + 4 * g;
            const int trow = ti * kT + wm * 64 + i * 16 + 4 * (r >> 2), tcol = col + (r & 3);    // after quad_transpose
            float v[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = acc[i][j][e];
            if constexpr (MODE == kGram || MODE == kPoly) {
                if constexpr (MODE == kPoly) {
                    const u32x2 s = *reinterpret_cast<const u32x2*>(w.s + sb + static_cast<size_t>(row) * w.np + col);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        v[e] = __builtin_fmaf(q.c, v[e], q.b * f16_at(s, e));
                }
                uint16_t* out = MODE == kGram ? w.s : w.p;
                const u32x2 h = {pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3])};
                *reinterpret_cast<u32x2*>(out + sb + static_cast<size_t>(row) * w.np + col) = h;
                if (ti != tj)
                    *reinterpret_cast<u32x2*>(out + sb + static_cast<size_t>(tcol) * w.np + trow) = quad_transpose(h, lane);
            } else {
                const size_t at = xb + static_cast<size_t>(row) * w.mp + col;
                const u32x2 h = *reinterpret_cast<const u32x2*>(w.xh + at), l = *reinterpret_cast<const u32x2*>(w.xl + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float x = __builtin_fmaf(f16_at(l, e), 1.0f / kLoScale, f16_at(h, e));
                    v[e] = __builtin_fmaf(q.a, x, v[e]);
                }
                if constexpr (MODE == kApply) {
                    u32x2 hi, lo;
                    split4(v, hi, lo);
                    *reinterpret_cast<u32x2*>(w.xh + at) = hi;
                    *reinterpret_cast<u32x2*>(w.xl + at) = lo;
                    *reinterpret_cast<u32x2*>(w.xt[q.from ^ 1] + xb + static_cast<size_t>(tcol) * w.np + trow) =
                        quad_transpose(hi, lane);
                } else {
                    u32x2 y = {pack_bf16x2_rne(v[0], v[1]), pack_bf16x2_rne(v[2], v[3])};
                    uint16_t* out = q.out + static_cast<size_t>(blockIdx.y) * q.rows * q.cols;
                    int orow = row, ocol = col;
                    if (q.rows > q.cols) {
                        y = quad_transpose(y, lane);
                        orow = tcol;
                        ocol = trow;
                    }
                    if (orow < q.rows) {
                        uint16_t* o = out + static_cast<size_t>(orow) * q.cols + ocol;
                        if (ocol + 3 < q.cols && (reinterpret_cast<uintptr_t>(o) & 7) == 0) {
                            *reinterpret_cast<u32x2*>(o) = y;
                        } else {
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                if (ocol + e < q.cols) o[e] = static_cast<uint16_t>(y[e >> 1] >> (16 * (e & 1)));
                        }
                    }
                }
            }
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
    const int tn = w.np / kT, tm = w.mp / kT;
    const dim3 tri(tn * (tn + 1) / 2, batch), all(tn * tm, batch);
    for (int i = 0; i < steps; ++i) {
        q.from = i & 1;
        q.a = sc.v[i][0];
        q.b = sc.v[i][1];
        q.c = sc.v[i][2];
        product_kernel<kGram><<<tri, kThreads, 0, stream>>>(q);
        product_kernel<kPoly><<<tri, kThreads, 0, stream>>>(q);
        if (i + 1 < steps) product_kernel<kApply><<<all, kThreads, 0, stream>>>(q);
        else product_kernel<kFinal><<<all, kThreads, 0, stream>>>(q);
    }
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
