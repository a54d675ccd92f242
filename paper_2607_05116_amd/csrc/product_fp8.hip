// Products of rows with their expert's weights, both in e4m3 with an fp32 scale for
// each block of 128 along K (and, for weights, of 128 outputs):
//   y[i][n] = sum over blocks b of  sx[i][b] sw[n / 128][b] (sum over k in b of x[i][k] w[n][k]),
// and the experts' SwiGLU feed-forward made of two of them.
//
// One v_mfma_f32_16x16x128_f8f6f4 sums a block of 16 x 16 outputs over exactly one
// scale block, so its result, started from zero, is scaled and added to the fp32
// accumulators by one FMA a value.  The instruction aligns each eight neighbouring
// products to the largest of them and drops what lies 2^-13 below it (1.4e-5 of the
// result on normal values, measured; what follows is fp32): far below a bf16 result's
// rounding, but not an fp32 one's, so products with an fp32 result are taken on the
// bf16 instructions, at half the rate: a code's value is a bf16 value, and those
// products are exact.  H, whose codes an error of 1.4e-5 moves across a border once in some
// thousands, is taken so for few rows (1 to 2 % of the time), but not for many: there exact
// products take 2.60 ms instead of 1.36 for 33,234 rows of d = 7168, inter = 2048 (and 92 us
// instead of 55 for 3,001 of d = 2048, inter = 1408), and y, in bf16, is then off by 0.00167 of
// its norm against 64 bits instead of 0.0020 (0.0021).  The weights are the MFMA's first operand: a lane
// then holds four consecutive outputs n of one row, one activation scale a lane and
// block of rows, and the weights' scale is the same for a wave.
#pragma clang fp contract(off)

#include <hip/hip_runtime.h>
#include <math.h>

#include "fp8_device.hpp"
#include "mfma_tile.hpp"

namespace cap {

cap_status quantise_fp8_launch(cap_dtype, int, int, int, int, const void*, void*, float*, hipStream_t);

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct F8Args {
    const uint8_t* x;            // [x_rows][K]
    const float* sx;             // of row r, block b: sx[r * sx_row + b * sx_block]
    const int32_t* row_src;      // nullable
    const int32_t* offsets;
    const uint8_t *w1, *w3;      // [E_loc][N][K]; w3 for SwiGLU only
    const float *s1, *s3;        // [E_loc][ceil(N / 128)][KT]
    void* out;                   // [max_rows][N]
    float* out_scale;            // SwiGLU: [N / 128][scale_pitch]
    size_t sx_row, sx_block, scale_pitch;
    int x_rows, E_loc, max_rows, N, KT;
    bool sx_in_order;            // wide: sx is [KT][sx_block] in the rows' order
};

// 4-byte form of lds_dma16: lane i's dword lands at LDS byte lds_addr + 4 i.
__device__ __forceinline__ void lds_dma4(const void* base, uint32_t off, uint32_t lds_addr) {
    uint64_t b;
    asm volatile("s_mov_b64 %0, %2\n\tglobal_load_lds_dword %1, %0"
                 : "=&s"(b)
                 : "v"(off), "s"(uniform_ptr(base)), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr))
                 : "memory");
}

// Eight codes of a fragment (registers 2 s, 2 s + 1) as bf16, exactly.
typedef __bf16 bf16x2_f8 __attribute__((ext_vector_type(2)));
template <int S>
__device__ __forceinline__ bf16x8 widen8(const i32x8& f) {
    const bf16x2_f8 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * S], 1.0f, false);
    const bf16x2_f8 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * S], 1.0f, true);
    const bf16x2_f8 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * S + 1], 1.0f, false);
    const bf16x2_f8 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(f[2 * S + 1], 1.0f, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The sum over a scale block.
template <bool PRECISE>
__device__ __forceinline__ f32x4 block_sum(const i32x8& w, const i32x8& x) {
    f32x4 zero = {0.0f, 0.0f, 0.0f, 0.0f};
    if constexpr (PRECISE) {
        static_for<4>([&](auto S) {
            zero = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen8<S.value>(w), widen8<S.value>(x), zero, 0, 0, 0);
        });
        return zero;
    }
    // both operands e4m3 (formats 0), no hardware scales
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, zero, 0, 0, 0, 0, 0, 0);
}

// 32 bytes of a stage row: 16-byte chunks kc and kc + 4 (both operands take the same
// chunks, so the products pair up whatever order the hardware sums K in).
__device__ __forceinline__ i32x8 frag8(const uint8_t* p0, const uint8_t* p1) {
    const i32x4 lo = *reinterpret_cast<const i32x4*>(p0), hi = *reinterpret_cast<const i32x4*>(p1);
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Rows of expert e: [lo, lo + n) of the expert-sorted rows, within max_rows.
__device__ __forceinline__ void expert_rows(const F8Args& a, int e, int& lo, int& n) {
    const int base = a.offsets[0];
    auto at = [&](int i) {
        const int v = a.offsets[i] - base;
        return v < 0 ? 0 : v > a.max_rows ? a.max_rows : v;
    };
    lo = at(e);
    const int hi = at(e + 1);
    n = hi > lo ? hi - lo : 0;
}

struct Tile {
    int e, m0, end, nt;          // expert, first row, end of the expert's rows, column tile
};

// Four neighbouring results of a row from column n on, those that are there.
template <typename OUT>
__device__ __forceinline__ void store4(const F8Args& a, OUT* out, int row, int n, const f32x4& v) {
    if (n >= a.N) return;
    OUT* const p = out + static_cast<size_t>(row) * a.N + n;
    // rows of whole, aligned groups of four
    if ((a.N & 3) == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(OUT) - 1)) == 0) {
        if constexpr (std::is_same<OUT, float>::value) *reinterpret_cast<f32x4*>(p) = v;
        else *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2_rne(v[0], v[1]), pack_bf16x2_rne(v[2], v[3])};
        return;
    }
#pragma unroll
    for (int c = 0; c < 4; ++c)
        if (n + c < a.N) {
            if constexpr (std::is_same<OUT, float>::value) p[c] = v[c];
            else p[c] = static_cast<uint16_t>(pack_bf16x2_rne(v[c], v[c]));
        }
}

// ------------------------------------------------------------------ tiles of 128 x 128
constexpr int kTile = 128;

// The tile of a workgroup; false for surplus ones.  Workgroups go to the XCDs in
// turn: each XCD gets a contiguous run of tiles, in which groups of four row tiles
// go through all column tiles together (their operands then meet in its L2).
__device__ __forceinline__ bool find_tile(const F8Args& a, int NT, Tile& out) {
    constexpr int BM = kTile;
    const int lane = threadIdx.x & 63;
    int total = 0;
    for (int c = 0; c < a.E_loc; c += 64) {
        int lo, n = 0;
        if (c + lane < a.E_loc) expert_rows(a, c + lane, lo, n);
        int m = (n + BM - 1) / BM;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) m += __shfl_xor(m, d);
        total += m;
    }
    total = __builtin_amdgcn_readfirstlane(total) * NT;      // the tile stays in scalar registers
    const int per = (total + 7) / 8;
    const int slot = blockIdx.x / 8;
    const int id = (blockIdx.x % 8) * per + slot;
    if (slot >= per || id >= total) return false;
    int before = 0;
    for (int c = 0; c < a.E_loc; c += 64) {
        int lo = 0, n = 0;
        if (c + lane < a.E_loc) expert_rows(a, c + lane, lo, n);
        const int m = (n + BM - 1) / BM;
        int upto = m;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        const uint64_t hit = __ballot(id < before + upto * NT);
        if (hit) {
            const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
            const int mt = __builtin_amdgcn_readlane(m, l);
            const int first = before + (__builtin_amdgcn_readlane(upto, l) - mt) * NT;
            const int local = id - first;
            const int g = local / (4 * NT);
            const int gm = mt - 4 * g < 4 ? mt - 4 * g : 4;
            const int r = local - g * 4 * NT;
            const int start = __builtin_amdgcn_readlane(lo, l);
            out.e = c + l;
            out.nt = r / gm;
            out.m0 = start + (4 * g + r % gm) * BM;
            out.end = start + __builtin_amdgcn_readlane(n, l);
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63) * NT;
    }
    return false;
}

// Barrier that publishes LDS writes and leaves direct loads under way.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    block_barrier();
}

// One tile of 128 rows x 128 weight rows, four waves of 64 x 64; K in stages of 128, two of
// them on their way: a stage's fragments are read at once, then its buffer is filled again.  For fp32 results, and for bf16 ones whose rows the wide
// kernel cannot load or store (n % 8 or y's address).  OUT: uint16_t (bf16) or float.  33,234 rows
// of 8 experts, kdim = 2048: n = 7165 in bf16 730 us (1.34 PFLOP/s, half of the 8-bit library
// product's), n = 7168 in fp32 991 us (0.98, 0.7 of the bf16 library product's, whose instructions it
// uses): a stage's LDS reads lie between two barriers before its first MFMA, and every wave converts
// its own fragments.
template <typename OUT>
__global__ __launch_bounds__(256) void f8_tile_kernel(const F8Args a) {
    constexpr int NW = 4, WM = 64, WN = 64, MI = WM / 16, NJ = WN / 16;
    constexpr int kChunksW = 2 * kTile / 8 / NW;        // 1 KiB loads of a wave per stage
    constexpr int kStage = 2 * kTile * 128;
    __shared__ __align__(16) uint8_t lds[2 * kStage];
    __shared__ float lds_sx[2 * kTile];
    __shared__ float lds_sw[kF8MaxStages];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / 2, wn = wave % 2;
    const int KT = a.KT, K = KT * 128, NT = (a.N + kTile - 1) / kTile;
    Tile tile;
    if (!find_tile(a, NT, tile)) return;
    const int n0 = tile.nt * kTile;

    // the weights' scales of the tile: one row of blocks
    for (int i = threadIdx.x; i < KT; i += 64 * NW) lds_sw[i] = a.s1[(static_cast<size_t>(tile.e) * NT + tile.nt) * KT + i];

    // direct loads: lane l of a load writes row l / 8 of its 8 rows, chunk l % 8
    const LaneMap lm = lane_map(lane);
    const uint32_t col_b = wave & 1 ? lm.col_b[1] : lm.col_b[0];
    auto source_row = [&](int r) {               // tile row -> row of x; rows past the end repeat the last
        int row = tile.m0 + r;
        row = row < tile.end ? row : tile.end - 1;
        if (a.row_src) {
            row = a.row_src[row];
            row = row < 0 ? 0 : row < a.x_rows ? row : a.x_rows - 1;
        }
        return row;
    };
    const char* base[kChunksW];
    uint32_t off[kChunksW], dst[kChunksW];
#pragma unroll
    for (int i = 0; i < kChunksW; ++i) {
        const int c = wave + NW * i;
        dst[i] = c * 1024;
        if (c < kTile / 8) {
            base[i] = reinterpret_cast<const char*>(a.x);
            off[i] = static_cast<uint32_t>(source_row(8 * c + lm.ld_row)) * static_cast<uint32_t>(K) + col_b;
        } else {
            int n = n0 + 8 * (c - kTile / 8) + lm.ld_row;
            n = n < a.N ? n : a.N - 1;
            base[i] = reinterpret_cast<const char*>(a.w1 + static_cast<size_t>(tile.e) * a.N * K);
            off[i] = static_cast<uint32_t>(n) * static_cast<uint32_t>(K) + col_b;
        }
    }
    uint32_t sx_off = 0;
    if (wave < kTile / 64) sx_off = static_cast<uint32_t>(source_row(64 * wave + lane)) * static_cast<uint32_t>(a.sx_row) * 4u;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    const uint32_t sx0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds_sx));
    auto issue = [&](int kt, int buf) {
#pragma unroll
        for (int i = 0; i < kChunksW; ++i)
            lds_dma16(base[i] + static_cast<size_t>(kt) * 128, off[i], lds0 + buf * kStage + dst[i]);
        if (wave < kTile / 64)
            lds_dma4(a.sx + kt * a.sx_block, sx_off, sx0 + buf * kTile * 4 + wave * 256);
    };

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int pc0 = (lm.fr_kc ^ lm.fr_swz) << 4, pc1 = pc0 ^ 64;
    const uint8_t* const la = lds + (wm * WM + lm.fr_row) * 128;
    const uint8_t* const lb = lds + (kTile + wn * WN + lm.fr_row) * 128;
    __syncthreads();                                   // the weights' scales; no load of ours is under way yet
    issue(0, 0);
    if (KT > 1) issue(1, 1);
    for (int kt = 0; kt < KT; ++kt) {
        const int buf = kt & 1;
        if (kt + 1 < KT) wait_vm<kChunksW>();          // stage kt has landed (the next, of as many loads or one more, may not have)
        else wait_vm<0>();
        block_barrier();
        float s[MI];
        i32x8 xf[MI], wf[NJ];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            s[i] = lds_sx[buf * kTile + wm * WM + 16 * i + lm.fr_row] * lds_sw[kt];
            xf[i] = frag8(la + buf * kStage + i * 2048 + pc0, la + buf * kStage + i * 2048 + pc1);
        }
#pragma unroll
        for (int j = 0; j < NJ; ++j) wf[j] = frag8(lb + buf * kStage + j * 2048 + pc0, lb + buf * kStage + j * 2048 + pc1);
        lds_barrier();                                 // read by all waves
        if (kt + 2 < KT) issue(kt + 2, buf);
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const f32x4 d = block_sum<std::is_same<OUT, float>::value>(wf[j], xf[i]);
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(d[v], s[i], acc[i][j][v]);
            }
    }

    // out by rows: a wave turns 16 of its rows at a time, in LDS of its own
    constexpr int kPitch = WN + 4;
    float* const mine = reinterpret_cast<float*>(lds) + wave * 16 * kPitch;
    OUT* const out = static_cast<OUT*>(a.out);
    const int n = n0 + wn * WN;
    const bool fours = (a.N & 3) == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(OUT) - 1)) == 0;
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int m = tile.m0 + wm * WM + 16 * i;
#pragma unroll
        for (int j = 0; j < NJ; ++j)
            *reinterpret_cast<f32x4*>(mine + lm.fr_row * kPitch + 16 * j + (lane >> 4) * 4) = acc[i][j];
        __builtin_amdgcn_wave_barrier();
        if (fours) {
#pragma unroll
            for (int r = lane >> 4; r < 16; r += 4) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(mine + r * kPitch + 4 * (lane & 15));
                if (m + r < tile.end) store4(a, out, m + r, n + 4 * (lane & 15), v);
            }
        } else if (n + lane < a.N) {
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float v = mine[r * kPitch + lane];
                OUT* const p = out + static_cast<size_t>(m + r) * a.N + n + lane;
                if (m + r >= tile.end) break;
                if constexpr (std::is_same<OUT, float>::value) *p = v;
                else *p = static_cast<uint16_t>(pack_bf16x2_rne(v, v));
            }
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// ------------------------------------------------------------------ wide tiles
// 256 x 256, eight waves of 64 x 128, in the four quarters a stage of mfma_tile.hpp's K
// loop (its barriers a and c, LDS layout and fragment reads, with 128 8-bit values in a
// stage row instead of 64 of 16 bits: a quarter is 4 x 2 MFMAs of K = 128).  What differs:
//   - The FMAs that scale and add an MFMA's sums follow two MFMAs later, so that they never
//     wait for it (right after the next one they did, for 28 cycles of every 64).
//   - All waves load: each 32 rows of A and 8 of each quarter of B a stage.
//   - Activation scales come with a stage's B quarters 0, 1: in place ([rows][KT], 256 cache
//     lines a stage, half as many as its operands), or, in long calls with long rows, from
//     [KT][rows] in the rows' order, 256 bytes a wave; the weights' are in LDS.
//   - KT may be odd: stage kt sits in buffer (kt + KT) % 2, so the last is in buffer 1.
// 33,234 rows of 8 experts, n = 7168, kdim = 2048: 450 us, 2.17 PFLOP/s (tiles of 128 x 128
// 727 us; one tile a workgroup, not a run of them, 520); the feed-forward of the same sizes
// 1.33 ms, 2.2 PFLOP/s.  The chip's power bounds it: its clock falls to 1.6 to 1.9 GHz, and
// with operands of zeros the same feed-forward takes 1.09 ms.  At that clock the MFMAs are
// busy for 55 % of the time; without the FMAs' three quarters it takes 1.16 ms.
constexpr int kALdF8 = kBM / kRowsPerLoad / kNW;       // direct loads of A per wave and stage
static_assert(kALdF8 == 4 && kNW == 8, "32 rows of A, 8 of each B quarter");

struct WideLoads {
    const char *a, *b[4], *s;    // at the stage to be loaded next (b: one for each quarter)
    size_t s_step;               // bytes of the scales from stage to stage
    uint32_t a_off[kALdF8], b_off, s_off;      // the lane's
    uint32_t a_lds, b_lds, s_lds;              // in buffer 0
};
// Direct loads and waits of a stage that may lie past the last (left: stages from it to the
// last, < 1 past it): left out by a branch
// inside the statement, so that the loop's body stays one block for the compiler (with
// branches of its own it spilled hundreds of registers; a copy of the body for the last
// stages cost more in the instruction cache).
__device__ __forceinline__ void lds_dma16_if(int left, const void* base, uint32_t off, uint32_t lds_addr) {
    uint64_t b;
    asm volatile("s_cmp_lt_i32 %4, 1\n\ts_cbranch_scc1 .Lskip%=\n\ts_mov_b64 %0, %2\n\t"
                 "global_load_lds_dwordx4 %1, %0\n.Lskip%=:"
                 : "=&s"(b)
                 : "v"(off), "s"(uniform_ptr(base)), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr)), "s"(__builtin_amdgcn_readfirstlane(left))
                 : "memory", "scc");
}
__device__ __forceinline__ void lds_dma4_if(int left, const void* base, uint32_t off, uint32_t lds_addr) {
    uint64_t b;
    asm volatile("s_cmp_lt_i32 %4, 1\n\ts_cbranch_scc1 .Lskip%=\n\ts_mov_b64 %0, %2\n\t"
                 "global_load_lds_dword %1, %0\n.Lskip%=:"
                 : "=&s"(b)
                 : "v"(off), "s"(uniform_ptr(base)), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr)), "s"(__builtin_amdgcn_readfirstlane(left))
                 : "memory", "scc");
}
// At most N loads under way if the stage is there, else at most M < N.
template <int N, int M>
__device__ __forceinline__ void wait_vm_if(int left) {
    asm volatile("s_cmp_gt_i32 %0, 0\n\ts_cbranch_scc1 .Lmore%=\n\ts_waitcnt vmcnt(%2)\n.Lmore%=:\n\ts_waitcnt vmcnt(%1)"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(left)), "n"(N), "n"(M)
                 : "memory", "scc");
}
template <int I>
__device__ __forceinline__ void wide_a(const WideLoads& l, int left, uint32_t buf) {
    lds_dma16_if(left, l.a, l.a_off[I], l.a_lds + buf * kStageBytes + I * 1024);
}
template <int Q>
__device__ __forceinline__ void wide_b(WideLoads& l, int left, uint32_t buf) {
    lds_dma16_if(left, l.b[Q], l.b_off, l.b_lds + buf * kStageBytes + Q * 32 * kRowB);
    l.b[Q] += kRowB;
}
__device__ __forceinline__ void wide_s(WideLoads& l, int left, uint32_t buf) {
    lds_dma4_if(left, l.s, l.s_off, l.s_lds + buf * kBM * 4);
    l.s += l.s_step;
}

// sx: LDS [2][256], at the wave's rows and the lane's row of 16; sw: LDS, the scales of the
// wave's weights (SwiGLU: W1's, W3's KT further).  The caller has issued stage 0, whole.
template <bool SWIGLU, bool ACTIVE>
__device__ __forceinline__ void f8_k_loop(int KT, const uint8_t* lds, const float* sx, const float* sw, int wm, int wn,
                                          int lane, f32x4 (&acc)[kMI][kNJ], WideLoads& ld) {
    i32x8 a[kMI], b0[2], b1[2];
    f32x4 d[4] = {};
    float s[kMI] = {}, fac[4] = {};
    uint32_t buf = KT & 1;                             // of stage kt
    const LaneMap lm = lane_map(opaque(lane));
    const int pc0 = (lm.fr_kc ^ lm.fr_swz) << 4;
    // LDS offsets of the wave's fragments in the buffer that is read (chunks pc0, pc0 ^ 64)
    uint32_t la0 = (wm * kWM + lm.fr_row) * kRowB + pc0 + buf * kStageBytes, la1 = la0 ^ 64;
    uint32_t lb0 = (kBM + wn * kWN + lm.fr_row) * kRowB + pc0 + buf * kStageBytes, lb1 = lb0 ^ 64;
    auto read_a = [&](auto In) {
        constexpr int i = decltype(In)::value;
        a[i] = frag8(lds + la0 + i * 16 * kRowB, lds + la1 + i * 16 * kRowB);
    };
    auto read_b = [&](i32x8 (&b)[2], auto Qn, auto Jn) {
        constexpr int at = (2 * decltype(Qn)::value + decltype(Jn)::value) * 16 * kRowB;
        b[decltype(Jn)::value] = frag8(lds + lb0 + at, lds + lb1 + at);
    };
    auto read_s = [&](int kt, bool up) {
        const float w = sw[up ? KT + kt : kt];
#pragma unroll
        for (int i = 0; i < kMI; ++i) s[i] = sx[buf * kBM + 16 * i] * w;
    };
    // MFMA m = 8 q + 2 g + jj of the stage (A block g, B block 2 q + jj), then the scaling of
    // MFMA m - 2 (of the stage before for m = 0, 1)
    auto add = [&](auto Mn) {
        constexpr int m = decltype(Mn)::value, i = (m >> 1) & 3, j = 2 * (m >> 3) + (m & 1);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(d[m & 3][v], fac[m & 3], acc[i][j][v]);
    };
    auto group = [&](i32x8 (&b)[2], auto Qn, auto Gn) {
        constexpr int q = decltype(Qn)::value, g = decltype(Gn)::value;
        static_for<2>([&](auto J) {
            constexpr int m = 8 * q + 2 * g + J.value;
            d[m & 3] = block_sum<false>(b[J.value], a[g]);
            fac[m & 3] = s[g];
            __builtin_amdgcn_sched_barrier(0);
            add(std::integral_constant<int, (m + 30) % 32>{});
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    auto N0 = std::integral_constant<int, 0>{};
    auto N1 = std::integral_constant<int, 1>{};
    auto N2 = std::integral_constant<int, 2>{};
    auto N3 = std::integral_constant<int, 3>{};
    wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    block_barrier();                                   // stage 0 and the weights' scales are visible; the other buffer is free
    {
        const int more = KT - 1;
        static_for<kALdF8>([&](auto I) { wide_a<I.value>(ld, more, buf ^ 1); });
        ld.a += kRowB;
        wide_s(ld, more, buf ^ 1);
        wide_b<0>(ld, more, buf ^ 1);
        wide_b<1>(ld, more, buf ^ 1);
    }
    if constexpr (ACTIVE) {
        static_for<2>([&](auto N) { read_b(b0, N0, N); });
        static_for<2>([&](auto N) { read_a(N); });
    }
    for (int kt = 0; kt < KT; ++kt) {
        const int next1 = KT - kt - 1, next2 = next1 - 1;      // stages from kt + 1, kt + 2 on
        if constexpr (ACTIVE) read_s(kt, false);
        static_for<4>([&](auto G) {                                            // quarter 0
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) read_a(std::integral_constant<int, 2 + G.value>{});
                else read_b(b1, N1, std::integral_constant<int, G.value - 2>{});
                group(b0, N0, G);
            }
            if constexpr (G.value < 2) wide_b<2 + G.value>(ld, next1, buf ^ 1);
            __builtin_amdgcn_sched_barrier(0);
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // A, quarters 0 and 1 read
        wait_vm_if<kALdF8 + 5, 0>(next1);                        // quarters 2, 3 of stage kt landed
        block_barrier();                                         // barrier a
        static_for<4>([&](auto G) {                                            // quarter 1
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) read_b(b0, N2, G);
                group(b1, N1, G);
            }
            if constexpr (G.value % 2 == 1) wide_a<G.value / 2>(ld, next2, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (ACTIVE && SWIGLU) read_s(kt, true);
        static_for<4>([&](auto G) {                                            // quarter 2
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) read_b(b1, N3, G);
                group(b0, N2, G);
            }
            if constexpr (G.value % 2 == 1) wide_a<2 + G.value / 2>(ld, next2, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        ld.a += kRowB;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // quarters 2, 3 and the scales read
        wait_vm_if<kALdF8 + 2, 2>(next2);                        // A, quarters 0, 1, scales of stage kt + 1 landed
        block_barrier();                                         // barrier c
        la0 ^= kStageBytes;
        la1 ^= kStageBytes;
        lb0 ^= kStageBytes;
        lb1 ^= kStageBytes;
        static_for<4>([&](auto G) {                                            // quarter 3
            if constexpr (ACTIVE) {
                // (after the last stage what is read here is not used)
                if constexpr (G.value < 2) read_b(b0, N0, G);
                else read_a(std::integral_constant<int, G.value - 2>{});
                group(b1, N3, G);
            }
            if constexpr (G.value == 0) wide_s(ld, next2, buf);
            else if constexpr (G.value < 3) wide_b<G.value - 1>(ld, next2, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        buf ^= 1;
    }
    if constexpr (ACTIVE) {
        add(std::integral_constant<int, 30>{});
        add(std::integral_constant<int, 31>{});
    }
}

// A wide tile's way out: each wave turns its 64 x 128 results, 32 rows at a time, in 8 KB
// of the stages of its own, and writes 256 bytes of a row together (chunk c of row r at c
// ^ r: a wave's accesses fall on all banks alike).  Every wave is past its last read of a
// stage.
__device__ __forceinline__ void store_wide(const F8Args& a, const Tile& tile, int n0, int wm, int wn, int wave, int lane,
                                           const f32x4 (&acc)[kMI][kNJ], uint8_t* lds) {
    uint8_t* const mine = lds + wave * 8192;
    const int r16 = lane & 15, q = lane >> 4;
    uint16_t* const out = static_cast<uint16_t*>(a.out);
    const int n = n0 + wn * kWN + 8 * r16;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int ii = 0; ii < 2; ++ii)
#pragma unroll
            for (int j = 0; j < kNJ; ++j) {
                const f32x4 v = acc[2 * half + ii][j];
                const int chunk = (2 * j + (q >> 1)) ^ r16;
                *reinterpret_cast<u32x2*>(mine + (16 * ii + r16) * 256 + chunk * 16 + (q & 1) * 8) =
                    u32x2{pack_bf16x2_rne(v[0], v[1]), pack_bf16x2_rne(v[2], v[3])};
            }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const int r = 4 * p + q;                   // of 32
            const u32x4 v = *reinterpret_cast<const u32x4*>(mine + r * 256 + (r16 ^ (r & 15)) * 16);
            const int row = tile.m0 + wm * kWM + 32 * half + r;
            if (row < tile.end && n < a.N) *reinterpret_cast<u32x4*>(out + static_cast<size_t>(row) * a.N + n) = v;
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// A wide SwiGLU tile's way out: H quantised to e4m3 by rows, with its scales.  `lds` (the
// other buffer's stage) is free but for reads that other waves may still make.
__device__ __forceinline__ void store_h(const F8Args& a, const Tile& tile, int n0, int wm, int wn, int lane,
                                        f32x4 (&acc)[kMI][kNJ], uint8_t* lds) {
    const int fr_row = lane & 15;
    const int q4 = (lane >> 4) * 4;                    // the lane's four outputs within a block of 16
    constexpr int kHCols = kWN / 2;                    // H columns of a wave
    float* const row_max = reinterpret_cast<float*>(lds);            // [kWavesN][kBM]
    uint8_t* const codes = lds + kWavesN * kBM * 4;                  // [kBM][kPitch]
    constexpr int kPitch = 128 + 16;
    static_assert(kWavesN * kBM * 4 + kBM * kPitch <= kStageBytes, "epilogue in one stage");
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNJ / 2; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float g = acc[i][j][v];
                acc[i][j][v] = g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * acc[i][j + kNJ / 2][v];
            }
    lds_barrier();                                     // the last stage is read
    uint32_t m[kMI];
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        m[i] = 0;
#pragma unroll
        for (int j = 0; j < kNJ / 2; ++j)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const uint32_t b = finite_magnitude(acc[i][j][v]);
                m[i] = b > m[i] ? b : m[i];
            }
#pragma unroll
        for (int d = 16; d < 64; d *= 2) {
            const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(m[i]), d));
            m[i] = o > m[i] ? o : m[i];
        }
        if (lane < 16) row_max[wn * kBM + wm * kWM + 16 * i + lane] = __uint_as_float(m[i]);
    }
    lds_barrier();
#pragma unroll
    for (int i = 0; i < kMI; ++i) {
        const int r = wm * kWM + 16 * i + fr_row;
        uint32_t top = 0;
#pragma unroll
        for (int c = 0; c < kWavesN; ++c) {
            const uint32_t o = __float_as_uint(row_max[c * kBM + r]);
            top = o > top ? o : top;
        }
        const uint32_t ex = f8_scale_exponent(top);
        const float inv = f8_inverse(ex);
#pragma unroll
        for (int j = 0; j < kNJ / 2; ++j) {
            const f32x4 v = acc[i][j];
            *reinterpret_cast<uint32_t*>(codes + r * kPitch + wn * kHCols + 16 * j + q4) =
                f8_pack4(v[0], v[1], v[2], v[3], inv);
        }
        if (wn == 0 && lane < 16 && tile.m0 + r < tile.end)
            a.out_scale[tile.nt * a.scale_pitch + tile.m0 + r] = f8_scale(ex);
    }
    lds_barrier();
    uint8_t* const out = static_cast<uint8_t*>(a.out);
    for (int c = threadIdx.x; c < kBM * 8; c += 64 * kNW) {
        const int r = c >> 3;
        if (tile.m0 + r < tile.end)
            *reinterpret_cast<u32x4*>(out + static_cast<size_t>(tile.m0 + r) * a.N + n0 + (c & 7) * 16) =
                *reinterpret_cast<const u32x4*>(codes + r * kPitch + (c & 7) * 16);
    }
}

// Tiles of the wide kernel: experts' row tiles and rows, once a workgroup.
struct WideTable {
    int upto[kMaxE];             // row tiles of the experts up to and with e
    int start[kMaxE], end[kMaxE];
};
__device__ __forceinline__ int fill_table(const F8Args& a, WideTable& t, int lane, bool writes) {
    int before = 0;
    for (int c = 0; c < a.E_loc; c += 64) {
        int lo = 0, n = 0;
        if (c + lane < a.E_loc) expert_rows(a, c + lane, lo, n);
        int upto = (n + kBM - 1) / kBM;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        if (writes && c + lane < a.E_loc) {
            t.upto[c + lane] = before + upto;
            t.start[c + lane] = lo;
            t.end[c + lane] = lo + n;
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return before;
}
// Tile `id`: groups of four row tiles of an expert go through all column tiles together
// (the workgroups of an XCD then meet on their operands in its L2).
__device__ __forceinline__ Tile tile_at(const WideTable& t, int E_loc, int NT, int id, int lane) {
    int e = 0;
    for (int c = 0; c < E_loc; c += 64)
        e += __popcll(__ballot(c + lane < E_loc && t.upto[c + lane < E_loc ? c + lane : 0] * NT <= id));
    const int first = e ? __builtin_amdgcn_readfirstlane(t.upto[e - 1]) : 0;
    const int mt = __builtin_amdgcn_readfirstlane(t.upto[e]) - first;
    const int start = __builtin_amdgcn_readfirstlane(t.start[e]);
    const int local = id - first * NT;
    const int g = local / (4 * NT);
    const int gm = mt - 4 * g < 4 ? mt - 4 * g : 4;
    const int r = local - g * 4 * NT;
    Tile out;
    out.e = e;
    out.nt = r / gm;
    out.m0 = start + (4 * g + r % gm) * kBM;
    out.end = __builtin_amdgcn_readfirstlane(t.end[e]);
    return out;
}

// N % 8 == 0: the 8 weight rows of a load are all there or all past the end (then those of
// the last 8 outputs are loaded, and nothing of them stored).  A workgroup goes through
// the tiles of its XCD's run; the next tile's first stage and weight scales are on their
// way while a tile's results go out through the other buffer.
template <typename OUT>
__global__ __launch_bounds__(512) void f8_wide_kernel(const F8Args a) {
    constexpr bool kSwiglu = std::is_same<OUT, uint8_t>::value;
    constexpr int kCols = kSwiglu ? kBN / 2 : kBN;
    __shared__ __align__(16) uint8_t lds[2 * kStageBytes];
    __shared__ float lds_sx[2 * kBM];
    __shared__ float lds_sw[2][2 * kF8MaxStages];
    __shared__ WideTable table;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const int KT = a.KT, K = KT * 128, NT = (a.N + kCols - 1) / kCols, NB = (a.N + 127) / 128, first = KT & 1;
    const int total = __builtin_amdgcn_readfirstlane(fill_table(a, table, lane, wave == 0)) * NT;
    const int per = (total + 7) / 8, xcd = blockIdx.x % 8, step = gridDim.x / 8;
    const int last = (xcd + 1) * per < total ? (xcd + 1) * per : total;
    int id = xcd * per + blockIdx.x / 8;
    if (id >= last) return;
    __syncthreads();

    const LaneMap lm = lane_map(lane);
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    const int col = wave >> 2, sub = wave & 3;         // B: wave column and eighths of a quarter's 32 rows
    WideLoads ld = {};
    ld.s_step = a.sx_block * 4;
    ld.a_lds = lds_base + wave * kALdF8 * 1024;
    ld.b_lds = lds_base + (kBM + col * kWN + sub * kRowsPerLoad) * kRowB;
    ld.s_lds = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds_sx)) + (wave >> 1) * kWM * 4;
    ld.b_off = lm.ld_row * K + (sub & 1 ? lm.col_b[1] : lm.col_b[0]);
    const float* const sx = lds_sx + wm * kWM + lm.fr_row;
    auto source_row = [&](const Tile& tile, int r) {   // rows past the end repeat the last
        int row = tile.m0 + r;
        row = row < tile.end ? row : tile.end - 1;
        if (a.row_src) {
            row = a.row_src[row];
            row = row < 0 ? 0 : row < a.x_rows ? row : a.x_rows - 1;
        }
        return row;
    };
    // a tile's operands, its first stage, and the weights' scales
    auto begin = [&](const Tile& tile, float* sw) {
        const int n0 = tile.nt * kCols;
        const size_t expert = static_cast<size_t>(tile.e) * a.N;
        auto rows_at = [&](const uint8_t* w, int n) {
            n = n < a.N ? n : a.N - kRowsPerLoad;
            return reinterpret_cast<const char*>(w + (expert + n) * K);
        };
        const int n = n0 + (kSwiglu ? 64 : 128) * col + sub * kRowsPerLoad;
        ld.b[0] = rows_at(a.w1, n);
        ld.b[1] = rows_at(a.w1, n + 32);
        ld.b[2] = rows_at(kSwiglu ? a.w3 : a.w1, kSwiglu ? n : n + 64);
        ld.b[3] = rows_at(kSwiglu ? a.w3 : a.w1, kSwiglu ? n + 32 : n + 96);
        ld.a = reinterpret_cast<const char*>(a.x);
        if (a.sx_in_order) {
            ld.s = reinterpret_cast<const char*>(a.sx + tile.m0 + (wave >> 1) * kWM);
            ld.s_off = lane * 4;
        } else {
            ld.s = reinterpret_cast<const char*>(a.sx);
            ld.s_off = static_cast<uint32_t>(source_row(tile, (wave >> 1) * kWM + lane)) * KT * 4;
        }
#pragma unroll
        for (int i = 0; i < kALdF8; ++i)
            ld.a_off[i] = static_cast<uint32_t>(source_row(tile, wave * 8 * kALdF8 + i * kRowsPerLoad + lm.ld_row)) * K +
                          lm.col_b[i & 1];
        const size_t at = (static_cast<size_t>(tile.e) * NB + n0 / 128) * KT;
        float w0 = 0.0f, w1 = 0.0f;
        if (static_cast<int>(threadIdx.x) < KT) {
            w0 = a.s1[at + threadIdx.x];
            w1 = kSwiglu ? a.s3[at + threadIdx.x] : a.s1[(n0 / 128 + 1 < NB ? at + KT : at) + threadIdx.x];
        }
        static_for<kALdF8>([&](auto I) { wide_a<I.value>(ld, 1, first); });
        ld.a += kRowB;
        wide_s(ld, 1, first);
        static_for<4>([&](auto Q) { wide_b<Q.value>(ld, 1, first); });
        if (static_cast<int>(threadIdx.x) < KT) {
            sw[threadIdx.x] = w0;
            sw[KT + threadIdx.x] = w1;
        }
    };
    Tile tile = tile_at(table, a.E_loc, NT, id, lane);
    int set = 0;
    begin(tile, lds_sw[0]);
    while (true) {
        const float* const sw = lds_sw[set] + (kSwiglu ? 0 : wn * KT);
        f32x4 acc[kMI][kNJ];
#pragma unroll
        for (int i = 0; i < kMI; ++i)
#pragma unroll
            for (int j = 0; j < kNJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        if (tile.m0 + wm * kWM < tile.end) f8_k_loop<kSwiglu, true>(KT, lds, sx, sw, wm, wn, lane, acc, ld);
        else f8_k_loop<kSwiglu, false>(KT, lds, sx, sw, wm, wn, lane, acc, ld);
        id += step;
        const bool more = id < last;
        const Tile done = tile;
        if (more) {
            tile = tile_at(table, a.E_loc, NT, id, lane);
            set ^= 1;
            begin(tile, lds_sw[set]);
        }
        uint8_t* const out_lds = lds + (first ^ 1) * kStageBytes;
        if constexpr (kSwiglu)
            store_h(a, done, done.nt * kCols, wm, wn, lane, acc, out_lds);
        else
            store_wide(a, done, done.nt * kCols, wm, wn, wave, lane, acc, out_lds);
        if (!more) return;
    }
}

template <typename OUT>
cap_status launch_tiles(const F8Args& a, hipStream_t st) {
    const long long rows = a.max_rows / kTile + (a.E_loc < a.max_rows ? a.E_loc : a.max_rows);
    const long long blocks = (rows * ((a.N + kTile - 1) / kTile) + 7) / 8 * 8;
    if (blocks * 256 >= (1ll << 32)) return CAP_ERR_UNSUPPORTED;
    f8_tile_kernel<OUT><<<static_cast<unsigned>(blocks), 256, 0, st>>>(a);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

// ------------------------------------------------------------------ few rows
// Up to some tens of rows an expert: every weight is read once for little arithmetic, and
// its way from memory is all that counts.  A workgroup takes 16 I rows of an expert and 16 J
// of its outputs (within one scale block); its eight waves share the blocks of K among
// them, load their weights straight into the MFMA's registers, a block ahead, and join
// their sums in LDS in the waves' order.  SwiGLU: four waves take W1 and four W3, and H
// leaves in fp32: quantising it takes 128 of its columns, and workgroups of so many leave
// half of the compute units without one.  The weights' bytes bound it: 8 rows of 8 experts,
// d = 7168, inter = 2048: 71 us for 352 MB, 4.95 TB/s (weights through LDS in tiles 120 us).
template <int BM>
__device__ __forceinline__ bool find_rows(const F8Args& a, int NT, Tile& out) {
    const int lane = threadIdx.x & 63, id = blockIdx.x;
    int lo[kMaxE / 64], n[kMaxE / 64];
    const int base = a.offsets[0];
#pragma unroll
    for (int c = 0; c < kMaxE / 64; ++c) {             // all on their way together; experts past the last are empty
        const int e = 64 * c + lane;
        lo[c] = a.offsets[e < a.E_loc ? e : a.E_loc];
        n[c] = a.offsets[e < a.E_loc ? e + 1 : a.E_loc];
    }
#pragma unroll
    for (int c = 0; c < kMaxE / 64; ++c) {
        auto within = [&](int v) { return v < 0 ? 0 : v > a.max_rows ? a.max_rows : v; };
        lo[c] = within(lo[c] - base);
        const int hi = within(n[c] - base);
        n[c] = hi > lo[c] ? hi - lo[c] : 0;
    }
    int before = 0;
#pragma unroll
    for (int c = 0; c < kMaxE / 64; ++c) {
        if (64 * c >= a.E_loc) break;
        const int m = (n[c] + BM - 1) / BM;
        int upto = m;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(upto, d);
            upto += lane >= d ? o : 0;
        }
        const uint64_t hit = __ballot(id < before + upto * NT);
        if (hit) {
            const int l = __ffsll(static_cast<unsigned long long>(hit)) - 1;
            const int mt = __builtin_amdgcn_readlane(m, l);
            const int local = id - before - (__builtin_amdgcn_readlane(upto, l) - mt) * NT;
            const int start = __builtin_amdgcn_readlane(lo[c], l);
            out.e = 64 * c + l;
            out.nt = local / mt;                       // an output block's row tiles side by side: its weights meet in a cache
            out.m0 = start + (local % mt) * BM;
            out.end = start + __builtin_amdgcn_readlane(n[c], l);
            return true;
        }
        before += __builtin_amdgcn_readlane(upto, 63) * NT;
    }
    return false;
}

template <int I, int J, bool H32>
struct FewStage {
    i32x4 w[J][2], x[I][2];
    float sx[I], sw;
};
template <int I, int J>
struct FewStage<I, J, true> {
    i32x4 w[J][2];
    f32x4 x[I][8];
    float sw;
};

// H32: the rows are H in fp32, quantised on their way to the MFMA, each block of 128 by the four
// lanes that hold it (as the quantisation's kernel does, to the bit).
template <int I, int J, typename OUT, bool kSwiglu, bool H32>
__global__ __launch_bounds__(512) void f8_few_kernel(const F8Args a) {
    constexpr bool kPrecise = std::is_same<OUT, float>::value;         // H too: its error moves codes across a border
    constexpr int kParts = kSwiglu ? 4 : 8;            // waves that share K
    constexpr int kCols = 16 * J, kRows = 16 * I;
    constexpr int kPitch = kCols + 4;                  // of a row of sums in LDS
    __shared__ __align__(16) float sums[8][kRows][kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int part = wave % kParts;
    const bool up = kSwiglu && wave >= kParts;
    const int KT = a.KT, NT = (a.N + kCols - 1) / kCols, NB = (a.N + 127) / 128;
    const size_t K = static_cast<size_t>(KT) * 128;
    Tile tile;
    if (!find_rows<kRows>(a, NT, tile)) return;
    const int n0 = tile.nt * kCols, r16 = lane & 15, g = lane >> 4;
    const uint8_t* const w = (up ? a.w3 : a.w1) + static_cast<size_t>(tile.e) * a.N * K;
    const float* const sw = (up ? a.s3 : a.s1) + (static_cast<size_t>(tile.e) * NB + n0 / 128) * KT;
    uint32_t w_off[J], x_off[I];
    size_t s_off[I];
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int n = n0 + 16 * j + r16;
        w_off[j] = static_cast<uint32_t>(n < a.N ? n : a.N - 1) * static_cast<uint32_t>(K) + 16 * g;
    }
    FewStage<I, J, H32> st[2];
    auto load_w = [&](FewStage<I, J, H32>& s, int kt) {
        const uint8_t* const p = w + static_cast<size_t>(kt) * 128;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) s.w[j][h] = *reinterpret_cast<const i32x4*>(p + w_off[j] + 64 * h);
        s.sw = sw[kt];
    };
    auto load_x = [&](FewStage<I, J, H32>& s, int kt) {
        const uint8_t* const p = a.x + static_cast<size_t>(kt) * (H32 ? 512 : 128);
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (H32) {
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    s.x[i][c] = *reinterpret_cast<const f32x4*>(p + x_off[i] + 256 * (c >> 2) + 16 * (c & 3));
            } else {
#pragma unroll
                for (int h = 0; h < 2; ++h) s.x[i][h] = *reinterpret_cast<const i32x4*>(p + x_off[i] + 64 * h);
                s.sx[i] = a.sx[s_off[i] + kt * a.sx_block];
            }
        }
    };
    if (part < KT) load_w(st[0], part);                // before the rows' sources are known
#pragma unroll
    for (int i = 0; i < I; ++i) {
        int row = tile.m0 + 16 * i + r16;              // rows past the end repeat the last
        row = row < tile.end ? row : tile.end - 1;
        if (a.row_src) {
            row = a.row_src[row];
            row = row < 0 ? 0 : row < a.x_rows ? row : a.x_rows - 1;
        }
        x_off[i] = (static_cast<uint32_t>(row) * static_cast<uint32_t>(K) + 16 * g) * (H32 ? 4 : 1);
        s_off[i] = row * a.sx_row;
    }
    f32x4 acc[I][J];
#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    auto add = [&](const FewStage<I, J, H32>& s) {
        i32x8 xf[I];
        float sx[I];
#pragma unroll
        for (int i = 0; i < I; ++i) {
            if constexpr (H32) {
                uint32_t m = 0;
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const uint32_t b = finite_magnitude(s.x[i][c][v]);
                        m = b > m ? b : m;
                    }
#pragma unroll
                for (int d = 16; d < 64; d *= 2) {
                    const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d));
                    m = o > m ? o : m;
                }
                const uint32_t ex = f8_scale_exponent(m);
                const float inv = f8_inverse(ex);
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    xf[i][c] = static_cast<int>(f8_pack4(s.x[i][c][0], s.x[i][c][1], s.x[i][c][2], s.x[i][c][3], inv));
                sx[i] = f8_scale(ex);
            } else {
                xf[i] = __builtin_shufflevector(s.x[i][0], s.x[i][1], 0, 1, 2, 3, 4, 5, 6, 7);
                sx[i] = s.sx[i];
            }
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const i32x8 wf = __builtin_shufflevector(s.w[j][0], s.w[j][1], 0, 1, 2, 3, 4, 5, 6, 7);
#pragma unroll
            for (int i = 0; i < I; ++i) {
                const f32x4 d = block_sum<kPrecise>(wf, xf[i]);
                const float f = sx[i] * s.sw;
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(d[v], f, acc[i][j][v]);
            }
        }
    };
    if (part < KT) load_x(st[0], part);
    int kt = part;
    for (; kt + kParts < KT; kt += 2 * kParts) {
        load_w(st[1], kt + kParts);
        load_x(st[1], kt + kParts);
        add(st[0]);
        if (kt + 2 * kParts < KT) {
            load_w(st[0], kt + 2 * kParts);
            load_x(st[0], kt + 2 * kParts);
        }
        add(st[1]);
    }
    if (kt < KT) add(st[0]);

#pragma unroll
    for (int i = 0; i < I; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) *reinterpret_cast<f32x4*>(&sums[wave][16 * i + r16][16 * j + 4 * g]) = acc[i][j];
    __syncthreads();
    // four neighbouring outputs a thread
    constexpr int kQuads = kRows * kCols / 4;
    for (int t = threadIdx.x; t < (kQuads + 63) / 64 * 64; t += 512) {
        const int r = t / (kCols / 4), c = t % (kCols / 4) * 4;
        const int row = tile.m0 + r, n = n0 + c;
        const bool there = t < kQuads && row < tile.end;
        auto join = [&](int first) {
            f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int p = 0; p < kParts; ++p) v += *reinterpret_cast<const f32x4*>(&sums[first + p][t < kQuads ? r : 0][c]);
            return v;
        };
        f32x4 v = join(0);
        if constexpr (kSwiglu) {
            const f32x4 u = join(kParts);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = v[i] * __builtin_amdgcn_rcpf(1.0f + __expf(-v[i])) * u[i];
        }
        if (there) store4(a, static_cast<OUT*>(a.out), row, n, v);
    }
}

long long few_blocks(const F8Args& a, int rows, int cols) {
    const long long tiles = a.max_rows / rows + (a.E_loc < a.max_rows ? a.E_loc : a.max_rows);
    return tiles * ((a.N + cols - 1) / cols);
}
bool few_launches(long long blocks) { return blocks * 512 < (1ll << 32); }     // threads of a launch

template <int I, int J, typename OUT, bool SWIGLU, bool H32 = false>
cap_status launch_few(const F8Args& a, hipStream_t st) {
    const long long blocks = few_blocks(a, 16 * I, 16 * J);
    if (!few_launches(blocks)) return CAP_ERR_UNSUPPORTED;
    f8_few_kernel<I, J, OUT, SWIGLU, H32><<<static_cast<unsigned>(blocks), 512, 0, st>>>(a);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

// Scales of the rows in expert-sorted order, [KT][pitch]; a lane takes a row.
__global__ __launch_bounds__(256) void f8_gather_scales_kernel(const F8Args a, float* __restrict__ out, size_t pitch) {
    const int i = blockIdx.x * 64 + (threadIdx.x & 63);
    if (i >= a.max_rows) return;
    int row = i;
    if (a.row_src) {
        row = a.row_src[i];
        row = row < 0 ? 0 : row < a.x_rows ? row : a.x_rows - 1;
    }
    const float* const p = a.sx + row * a.sx_row;
    for (int kt = threadIdx.x >> 6; kt < a.KT; kt += 4) out[kt * pitch + i] = p[kt];
}

// Floats between the scales of two blocks: whole tiles of rows.
size_t f8_scale_pitch(int max_rows) { return (static_cast<size_t>(max_rows) + 2 * kBM - 1) / kBM * kBM; }
size_t f8_scales_bytes(int k, int max_rows) { return f8_scale_pitch(max_rows) * (k / 128) * 4; }

// Which kernel a call takes goes by estimates of its time in microseconds, from its sizes
// alone (max_rows for the rows, as if they fell about evenly; every kernel is right for any).
// Measured, estimates in brackets: E = 8, n = 2048, kdim = 7168, 64 rows: few 21.7 (27), wide 56
// (61); 256 rows: 47 (50), 57 (61); n = 7168, kdim = 2048, 64 rows: few 24.5 (27), wide 22.9 (28);
// 256 rows: 42 (50), 23.7 (28); E = 7, 6,126 rows, n = 267, kdim = 2304: few 36 (31), tiles 26.5
// (26).
constexpr int kFewFfnRows = 8192;                      // the feed-forward's workspace has room for so many rows of H in fp32
long long likely_tiles(const F8Args& a, int rows) {    // row tiles, experts' sizes differing by a factor of three
    const long long some = a.E_loc < a.max_rows ? a.E_loc : a.max_rows, more = a.max_rows - 8ll * a.E_loc;
    return some + (more > 0 ? more / rows : 0);
}
// Enough workgroups of 16 J outputs for three of four compute units.
bool few_fill(const F8Args& a, int rows, int cols) {
    return 4 * likely_tiles(a, rows) * ((a.N + cols - 1) / cols) >= 3 * device_cu_count();
}
// 32 rows a workgroup once most experts have more than 8 rows.
bool few_take_32(const F8Args& a) { return a.max_rows > 8ll * a.E_loc && few_fill(a, 32, 64); }
// Rows and outputs of a workgroup.
struct FewForm {
    int rows, cols;
};
FewForm few_form(const F8Args& a) {
    if (few_take_32(a)) return {32, 64};
    // the more outputs a workgroup, the fewer bytes of x it reads beside its weights; with W1
    // and W3, a wave has twice the blocks of K (128 outputs: 78 us for 8 rows of 8 experts of
    // d = 7168, inter = 2048 in 128 workgroups, 64: 47 us)
    if (!a.w3 && likely_tiles(a, 16) * ((a.N + 127) / 128) >= device_cu_count()) return {16, 128};
    if (few_fill(a, 16, 64)) return {16, 64};
    // a compute unit has so much on its way at most: below half of them, 16 outputs each (8 rows of
    // 6 experts, d = 6400, inter = 384 27.1 -> 21.5 us; 13 experts, 71 rows, d = 2176, in 156
    // workgroups or 312: 17.5 or 18.7)
    if (2 * likely_tiles(a, 16) * ((a.N + 31) / 32) < device_cu_count()) return {16, 16};
    return {16, 32};
}
double weight_bytes(const F8Args& a) { return static_cast<double>(a.w3 ? 2 : 1) * a.N * a.KT * 128; }
double few_time(const F8Args& a) {                     // the weights' way, again for each row tile, and that of the rows (from nearer)
    const FewForm f = few_form(a);
    if (!few_launches(few_blocks(a, f.rows, f.cols))) return HUGE_VAL;
    const int rows = f.rows;
    const double row_bytes = static_cast<double>(rows) * a.KT * 128 * ((a.N + 63) / 64);
    return 3.5 + static_cast<double>(likely_tiles(a, rows)) * (weight_bytes(a) + 0.5 * row_bytes) / 5.5e6;
}
// Tiles: a round of them takes so long a stage, but no less than the weights' way.
double tiles_time(const F8Args& a, int rows, int cols, int at_once, double stage) {
    const long long tiles = likely_tiles(a, rows) * ((a.N + cols - 1) / cols);
    const double stages = stage * a.KT * static_cast<double>((tiles + at_once - 1) / at_once);
    const double bytes = static_cast<double>(a.E_loc < a.max_rows ? a.E_loc : a.max_rows) * weight_bytes(a) / 5.0e6;
    return 5.0 + (stages > bytes ? stages : bytes);
}
double wide_time(const F8Args& a) { return tiles_time(a, kBM, a.w3 ? kBN / 2 : kBN, device_cu_count(), 1.0); }
double tile_time(const F8Args& a) { return 1.5 + tiles_time(a, kTile, kTile, device_cu_count(), 1.1); }

// From so many stages on a launch that puts the scales in order is worth its 5 us, if a row's
// scales are more than a line of 128 bytes (d = 7168, 33,234 rows: the feed-forward 1.36 ms, in
// place 1.40; the product of kdim = 2048 468 us, in place 459).
constexpr int kStagesInOrder = 128;
template <typename OUT>
cap_status launch_wide(F8Args a, float* scales, hipStream_t st) {
    constexpr int cols = std::is_same<OUT, uint8_t>::value ? kBN / 2 : kBN;
    const long long rows = a.max_rows / kBM + (a.E_loc < a.max_rows ? a.E_loc : a.max_rows);
    const long long tiles = rows * ((a.N + cols - 1) / cols);
    if (tiles >= (1ll << 31)) return CAP_ERR_UNSUPPORTED;
    const long long cus = (device_cu_count() + 7) / 8 * 8;             // one workgroup a CU
    const long long blocks = tiles < cus ? (tiles + 7) / 8 * 8 : cus;
    const long long ordering = (a.max_rows + 63) / 64;                 // workgroups that put the scales in order
    if (!a.sx_in_order && a.KT > 32 && ordering * 256 < (1ll << 32) && (tiles + cus - 1) / cus * a.KT >= kStagesInOrder) {
        const size_t pitch = f8_scale_pitch(a.max_rows);
        f8_gather_scales_kernel<<<static_cast<unsigned>(ordering), 256, 0, st>>>(a, scales, pitch);
        a.sx = scales;
        a.sx_row = 1;
        a.sx_block = pitch;
        a.sx_in_order = true;
    }
    f8_wide_kernel<OUT><<<static_cast<unsigned>(blocks), 512, 0, st>>>(a);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace

size_t product_fp8_workspace_bytes(int, int kdim, int max_rows) {
    return f8_scales_bytes(kdim, max_rows);
}

// H's codes and its scales, [KT][rows], then scales in the rows' order (of x, or of H quantised
// from fp32) and H in fp32, which few rows need.
struct FfnSpace {
    size_t codes, h_scales, scales, h, end;
};
FfnSpace ffn_space(int d, int inter, int max_rows) {
    FfnSpace s;
    s.codes = 0;
    s.h_scales = (static_cast<size_t>(max_rows) * inter + 255) & ~size_t(255);
    s.scales = s.h_scales + f8_scales_bytes(inter, max_rows);
    s.h = s.scales + f8_scales_bytes(d > inter ? d : inter, max_rows);
    s.end = s.h + (max_rows <= kFewFfnRows ? static_cast<size_t>(max_rows) * inter * 4 : 0);
    return s;
}
size_t ffn_fp8_workspace_bytes(int d, int inter, int max_rows) { return ffn_space(d, inter, max_rows).end; }

namespace {

template <typename OUT, bool SWIGLU>
cap_status launch_few_rows(const F8Args& a, hipStream_t st) {
    const FewForm f = few_form(a);
    if (f.rows == 32) return launch_few<2, 4, OUT, SWIGLU>(a, st);
    if constexpr (!SWIGLU)
        if (f.cols == 128) return launch_few<1, 8, OUT, SWIGLU>(a, st);
    if (f.cols == 64) return launch_few<1, 4, OUT, SWIGLU>(a, st);
    if (f.cols == 32) return launch_few<1, 2, OUT, SWIGLU>(a, st);
    return launch_few<1, 1, OUT, SWIGLU>(a, st);
}

// y from H in fp32.
constexpr double kH32Bytes = 8e6;
cap_status launch_few_h32(const F8Args& a, hipStream_t st) {
    if (few_fill(a, 16, 64)) return launch_few<1, 4, uint16_t, false, true>(a, st);
    return launch_few<1, 2, uint16_t, false, true>(a, st);
}

// scales: room for those of the rows in their order.
cap_status product(cap_dtype out_dtype, const F8Args& a, float* scales, hipStream_t st) {
    if (out_dtype == CAP_DTYPE_F32) {
        if (few_time(a) < tile_time(a)) return launch_few_rows<float, false>(a, st);
        return launch_tiles<float>(a, st);
    }
    const bool wide = a.N % 8 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
    if (few_time(a) < (wide ? wide_time(a) : tile_time(a))) return launch_few_rows<uint16_t, false>(a, st);
    if (wide) return launch_wide<uint16_t>(a, scales, st);
    return launch_tiles<uint16_t>(a, st);
}

}  // namespace

cap_status product_fp8_launch(cap_dtype out_dtype, int E_loc, int n, int kdim, int max_rows, const void* x,
                              const float* x_scale, int x_rows, const int32_t* row_src, const int32_t* row_offsets,
                              const void* w, const float* w_scale, void* y, void* ws, hipStream_t st) {
    F8Args a = {};
    a.x = static_cast<const uint8_t*>(x);
    a.sx = x_scale;
    a.sx_row = kdim / 128;
    a.sx_block = 1;
    a.row_src = row_src;
    a.offsets = row_offsets;
    a.w1 = static_cast<const uint8_t*>(w);
    a.s1 = w_scale;
    a.out = y;
    a.x_rows = x_rows;
    a.E_loc = E_loc;
    a.max_rows = max_rows;
    a.N = n;
    a.KT = kdim / 128;
    return product(out_dtype, a, static_cast<float*>(ws), st);
}

cap_status expert_ffn_fp8_launch(int E_loc, int d, int inter, int max_rows, const void* x, const float* x_scale,
                                 int x_rows, const int32_t* row_src, const int32_t* row_offsets, const void* w1,
                                 const float* s1, const void* w3, const float* s3, const void* w2, const float* s2,
                                 void* y, void* ws, hipStream_t st) {
    const FfnSpace space = ffn_space(d, inter, max_rows);
    uint8_t* const at = static_cast<uint8_t*>(ws);
    uint8_t* const codes = at + space.codes;
    float* const h_scales = reinterpret_cast<float*>(at + space.h_scales);
    float* const scales = reinterpret_cast<float*>(at + space.scales);
    float* const h = reinterpret_cast<float*>(at + space.h);
    F8Args a = {};
    a.x = static_cast<const uint8_t*>(x);
    a.sx = x_scale;
    a.sx_row = d / 128;
    a.sx_block = 1;
    a.row_src = row_src;
    a.offsets = row_offsets;
    a.w1 = static_cast<const uint8_t*>(w1);
    a.w3 = static_cast<const uint8_t*>(w3);
    a.s1 = s1;
    a.s3 = s3;
    a.out = codes;
    a.out_scale = h_scales;
    a.scale_pitch = f8_scale_pitch(max_rows);
    a.x_rows = x_rows;
    a.E_loc = E_loc;
    a.max_rows = max_rows;
    a.N = inter;
    a.KT = d / 128;
    // few rows: H in fp32, quantised by the product that reads it, or, for more rows, by itself
    const bool few = max_rows <= kFewFfnRows && few_time(a) < wide_time(a);
    cap_status done;
    if (few) {
        a.out = h;
        done = launch_few_rows<float, true>(a, st);
    } else {
        done = launch_wide<uint8_t>(a, scales, st);
    }
    if (done != CAP_OK) return done;
    a.x = codes;
    a.sx = h_scales;
    a.sx_row = few ? inter / 128 : 1;
    a.sx_block = few ? 1 : a.scale_pitch;
    a.sx_in_order = !few;
    a.row_src = nullptr;
    a.w1 = static_cast<const uint8_t*>(w2);
    a.s1 = s2;
    a.w3 = nullptr;
    a.out = y;
    a.x_rows = max_rows;
    a.N = d;
    a.KT = inter / 128;
    if (few) {
        // (the kernel that quantises by itself reads H again with every block of outputs: 10 rows of 13
        // experts, d = 384, inter = 896 8.8 us instead of 10.3, but 8 rows of 8 experts, d = 7168,
        // inter = 2048 75 instead of 71.4; of the cases timed it is ahead below 11 MB of weights)
        if (!few_take_32(a) && static_cast<double>(likely_tiles(a, 16)) * weight_bytes(a) < kH32Bytes) {
            a.x = reinterpret_cast<const uint8_t*>(h);
            return launch_few_h32(a, st);
        }
        done = quantise_fp8_launch(CAP_DTYPE_F32, 1, max_rows, inter, 1, h, codes, h_scales, st);
        if (done != CAP_OK) return done;
    }
    return product(CAP_DTYPE_BF16, a, scales, st);
}

}  // namespace cap
