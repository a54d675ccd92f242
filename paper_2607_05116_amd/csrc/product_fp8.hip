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
// products are exact.  The weights are the MFMA's first operand: a lane
// then holds four consecutive outputs n of one row, one activation scale a lane and
// block of rows, and the weights' scale is the same for a wave.
#pragma clang fp contract(off)

#include <hip/hip_runtime.h>

#include "fp8_device.hpp"
#include "mfma_tile.hpp"

namespace cap {
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

// The tile of a workgroup; false for surplus ones.  Workgroups go to the XCDs in
// turn: each XCD gets a contiguous run of tiles, in which groups of four row tiles
// go through all column tiles together (their operands then meet in its L2).
template <int BM>
__device__ __forceinline__ bool find_tile(const F8Args& a, int NT, Tile& out) {
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

// A tile's way out: y, or H with its scales.  `lds` (the stages) is free but for reads
// of the last stage that other waves may still make.
template <int BM, int BN, int NWM, int NWN, typename OUT>
__device__ __forceinline__ void finish_tile(const F8Args& a, const Tile& tile, int n0, int wm, int wn, int lane,
                                            f32x4 (&acc)[BM / NWM / 16][BN / NWN / 16], uint8_t* lds) {
    constexpr bool kSwiglu = std::is_same<OUT, uint8_t>::value;
    constexpr int NW = NWM * NWN, WM = BM / NWM, WN = BN / NWN, MI = WM / 16, NJ = WN / 16;
    const int NB = (a.N + 127) / 128, fr_row = lane & 15;
    const int q4 = (lane >> 4) * 4;                    // the lane's four outputs within a block of 16
    if constexpr (!kSwiglu) {
        OUT* const out = static_cast<OUT*>(a.out);
        // rows of whole, aligned groups of four
        const bool whole = (a.N & 3) == 0 && (reinterpret_cast<uintptr_t>(out) & (4 * sizeof(OUT) - 1)) == 0;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int row = tile.m0 + wm * WM + 16 * i + fr_row;
            if (row >= tile.end) continue;
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                const int n = n0 + wn * WN + 16 * j + q4;
                OUT* const p = out + static_cast<size_t>(row) * a.N + n;
                const f32x4 v = acc[i][j];
                if (whole) {
                    if (n < a.N) {
                        if constexpr (std::is_same<OUT, float>::value) *reinterpret_cast<f32x4*>(p) = v;
                        else *reinterpret_cast<u32x2*>(p) = u32x2{pack_bf16x2_rne(v[0], v[1]), pack_bf16x2_rne(v[2], v[3])};
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (n + c < a.N) {
                            if constexpr (std::is_same<OUT, float>::value) p[c] = v[c];
                            else p[c] = static_cast<uint16_t>(pack_bf16x2_rne(v[c], v[c]));
                        }
                }
            }
        }
    } else {
        constexpr int HC = WN / 2;                     // H columns of a wave
        float* const row_max = reinterpret_cast<float*>(lds);                    // [NWN][BM]
        uint8_t* const codes = lds + NWN * BM * 4;                               // [BM][kPitch]
        constexpr int kPitch = 128 + 16;
        static_assert(NWN * BM * 4 + BM * kPitch <= 2 * (BM + BN) * 128, "epilogue in the stages");
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NJ / 2; ++j)
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float g = acc[i][j][v];
                    acc[i][j][v] = g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)) * acc[i][j + NJ / 2][v];
                }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        block_barrier();                               // the last stage is read
        uint32_t m[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            m[i] = 0;
#pragma unroll
            for (int j = 0; j < NJ / 2; ++j)
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
            if (lane < 16) row_max[wn * BM + wm * WM + 16 * i + lane] = __uint_as_float(m[i]);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const int r = wm * WM + 16 * i + fr_row;
            uint32_t top = 0;
#pragma unroll
            for (int c = 0; c < NWN; ++c) {
                const uint32_t o = __float_as_uint(row_max[c * BM + r]);
                top = o > top ? o : top;
            }
            const uint32_t ex = f8_scale_exponent(top);
            const float inv = f8_inverse(ex);
#pragma unroll
            for (int j = 0; j < NJ / 2; ++j) {
                const f32x4 v = acc[i][j];
                *reinterpret_cast<uint32_t*>(codes + r * kPitch + wn * HC + 16 * j + q4) =
                    f8_pack4(v[0], v[1], v[2], v[3], inv);
            }
            if (wn == 0 && lane < 16 && tile.m0 + r < tile.end)
                a.out_scale[tile.nt * a.scale_pitch + tile.m0 + r] = f8_scale(ex);
        }
        __syncthreads();
        uint8_t* const out = static_cast<uint8_t*>(a.out);
        for (int c = threadIdx.x; c < BM * 8; c += 64 * NW) {
            const int r = c >> 3;
            if (tile.m0 + r < tile.end)
                *reinterpret_cast<u32x4*>(out + static_cast<size_t>(tile.m0 + r) * a.N + n0 + (c & 7) * 16) =
                    *reinterpret_cast<const u32x4*>(codes + r * kPitch + (c & 7) * 16);
        }
    }
}

// One tile of BM rows x BN weight rows; K in stages of 128, double buffered, one
// barrier a stage.  OUT: uint16_t (bf16), float, or uint8_t: SwiGLU, whose BN weight
// rows are 128 of W1 and the same 128 of W3, those of each wave half and half, and
// whose result is quantised to e4m3 by rows.
template <int BM, int BN, int NWM, int NWN, typename OUT>
__global__ __launch_bounds__(64 * NWM * NWN) void f8_tile_kernel(const F8Args a) {
    constexpr bool kSwiglu = std::is_same<OUT, uint8_t>::value;
    constexpr int NW = NWM * NWN, WM = BM / NWM, WN = BN / NWN, MI = WM / 16, NJ = WN / 16;
    constexpr int kChunksW = (BM + BN) / 8 / NW;        // 1 KiB loads of a wave per stage
    constexpr int kStage = (BM + BN) * 128;
    constexpr int kCols = kSwiglu ? BN / 2 : BN;        // outputs of the tile
    static_assert((BM + BN) % (8 * NW) == 0 && BM % 64 == 0 && BM / 64 <= NW, "load split");
    static_assert(kSwiglu ? BN == 256 : BN <= 256, "scale blocks of a tile");
    __shared__ __align__(16) uint8_t lds[2 * kStage];
    __shared__ float lds_sx[2 * BM];
    __shared__ float lds_sw[2 * kF8MaxStages];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / NWN, wn = wave % NWN;
    const int KT = a.KT, K = KT * 128, NT = (a.N + kCols - 1) / kCols;
    Tile tile;
    if (!find_tile<BM>(a, NT, tile)) return;
    const int n0 = tile.nt * kCols, NB = (a.N + 127) / 128;

    // the weights' scales of the tile: one row of blocks of W1 and of W3, or BN / 128 rows
    {
        const size_t first = (static_cast<size_t>(tile.e) * NB + n0 / 128) * KT;
        for (int i = threadIdx.x; i < KT; i += 64 * NW) {
            lds_sw[i] = a.s1[first + i];
            if constexpr (kSwiglu) lds_sw[KT + i] = a.s3[first + i];
            else if constexpr (BN > 128) lds_sw[KT + i] = a.s1[(n0 / 128 + 1 < NB ? first + KT : first) + i];
        }
    }

    // direct loads: lane l of a load writes row l / 8 of its 8 rows, chunk l % 8
    const LaneMap lm = lane_map(lane);
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
        if (c < BM / 8) {
            base[i] = reinterpret_cast<const char*>(a.x);
            off[i] = static_cast<uint32_t>(source_row(8 * c + lm.ld_row)) * static_cast<uint32_t>(K) + lm.col_b[c & 1];
        } else {
            const int b = 8 * (c - BM / 8) + lm.ld_row;               // row of the B tile
            const size_t expert = static_cast<size_t>(tile.e) * a.N * K;
            int n = b;
            base[i] = reinterpret_cast<const char*>(a.w1 + expert);
            if constexpr (kSwiglu) {
                const int col = b / WN, in = b % WN;
                n = col * (WN / 2) + in % (WN / 2);
                if (in >= WN / 2) base[i] = reinterpret_cast<const char*>(a.w3 + expert);
            }
            n = n0 + n < a.N ? n0 + n : a.N - 1;
            off[i] = static_cast<uint32_t>(n) * static_cast<uint32_t>(K) + lm.col_b[c & 1];
        }
    }
    uint32_t sx_off = 0;
    if (wave < BM / 64) sx_off = static_cast<uint32_t>(source_row(64 * wave + lane)) * static_cast<uint32_t>(a.sx_row) * 4u;
    const uint32_t lds0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    const uint32_t sx0 = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds_sx));
    auto issue = [&](int kt, int buf) {
#pragma unroll
        for (int i = 0; i < kChunksW; ++i)
            lds_dma16(base[i] + static_cast<size_t>(kt) * 128, off[i], lds0 + buf * kStage + dst[i]);
        if (wave < BM / 64)
            lds_dma4(a.sx + kt * a.sx_block, sx_off, sx0 + buf * BM * 4 + wave * 256);
    };

    f32x4 acc[MI][NJ];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

    const int pc0 = (lm.fr_kc ^ lm.fr_swz) << 4, pc1 = pc0 ^ 64;
    const uint8_t* const la = lds + (wm * WM + lm.fr_row) * 128;
    const uint8_t* const lb = lds + (BM + wn * WN + lm.fr_row) * 128;
    __syncthreads();                                   // the weights' scales; no load of ours is under way yet
    issue(0, 0);
    for (int kt = 0; kt < KT; ++kt) {
        const int buf = kt & 1;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        wait_vm<0>();
        block_barrier();                               // stage kt is complete, stage kt - 1 read
        if (kt + 1 < KT) issue(kt + 1, buf ^ 1);
        float s[MI], su[MI];
        const float sw = lds_sw[(!kSwiglu && BN > 128 ? (wn * WN / 128) * KT : 0) + kt];
        const float sw3 = kSwiglu ? lds_sw[KT + kt] : 0.0f;
#pragma unroll
        for (int i = 0; i < MI; ++i) {
            const float v = lds_sx[buf * BM + wm * WM + 16 * i + lm.fr_row];
            s[i] = v * sw;
            su[i] = v * sw3;
        }
        i32x8 xf[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i)
            xf[i] = frag8(la + buf * kStage + i * 2048 + pc0, la + buf * kStage + i * 2048 + pc1);
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
            const i32x8 wf = frag8(lb + buf * kStage + j * 2048 + pc0, lb + buf * kStage + j * 2048 + pc1);
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const f32x4 d = block_sum<std::is_same<OUT, float>::value>(wf, xf[i]);
                const float f = kSwiglu && j >= NJ / 2 ? su[i] : s[i];
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[i][j][v] = __builtin_fmaf(d[v], f, acc[i][j][v]);
            }
        }
    }

    finish_tile<BM, BN, NWM, NWN, OUT>(a, tile, n0, wm, wn, lane, acc, lds);
}

// ------------------------------------------------------------------ wide tiles
// 256 x 256 in the four quarters a stage of mfma_tile.hpp's K loop (its barriers, loads
// and fragment reads, with 128 8-bit values in a stage row instead of 64 of 16 bits: a
// quarter is 4 x 2 MFMAs of K = 128).  What differs: a group of two MFMAs (A block g,
// both B blocks) leaves its sums in one of two register sets, and the FMAs that scale
// and add those of the one before run meanwhile.  Activation scales come with a stage's
// B quarters 0, 1, from [KT][rows] in the rows' order: 256 bytes a wave (read in place,
// [rows][KT], they are 256 cache lines a stage, half as many as its operands: 5 to 9 % of
// the time); the weights' are in LDS for the tile.
// KT may be odd: the stages sit in buffers so that the last is in buffer 1.
struct WideScales {
    const char* src;             // of the wave's 64 rows, at the stage to be loaded next
    size_t step;                 // bytes from stage to stage
    uint32_t off, dst;           // the lane's four bytes; LDS of the wave's rows
    const float* sx;             // LDS: [2][256], at the wave's rows and the lane's row of 16
    const float* sw;             // LDS: scales of the wave's weights; SwiGLU: W1's, W3's KT further
};

template <bool SWIGLU, bool LOADER, bool ACTIVE>
__device__ __forceinline__ void f8_k_loop(int KT, const uint8_t* lds, int wm, int wn, int lane, f32x4 (&acc)[kMI][kNJ],
                                          Loads& ld, WideScales& sc, uint32_t a_lds, uint32_t b_lds) {
    constexpr bool LOAD_A = LOADER && ACTIVE;
    constexpr int kA = LOAD_A ? kALd : 0, kS = LOAD_A ? 1 : 0;      // loads of A and of scales a stage
    i32x8 a[kMI], b0[2], b1[2];
    f32x4 d[2] = {};
    float s[kMI], pf = 0.0f;
    const LaneMap lm = lane_map(opaque(lane));
    const int pc0 = (lm.fr_kc ^ lm.fr_swz) << 4, pc1 = pc0 ^ 64;
    const uint8_t* const la = lds + (wm * kWM + lm.fr_row) * kRowB;
    const uint8_t* const lb = lds + (kBM + wn * kWN + lm.fr_row) * kRowB;
    auto read_a = [&](int buf, auto In) {
        constexpr int i = decltype(In)::value;
        const uint8_t* p = la + buf * kStageBytes + i * 16 * kRowB;
        a[i] = frag8(p + pc0, p + pc1);
    };
    auto read_b = [&](i32x8 (&b)[2], int buf, int q, auto Jn) {
        constexpr int j = decltype(Jn)::value;
        const uint8_t* p = lb + buf * kStageBytes + (2 * q + j) * 16 * kRowB;
        b[j] = frag8(p + pc0, p + pc1);
    };
    auto read_s = [&](int buf, int kt, bool up) {
        const float w = sc.sw[up ? KT + kt : kt];
#pragma unroll
        for (int i = 0; i < kMI; ++i) s[i] = sc.sx[buf * kBM + 16 * i] * w;
    };
    // group g of quarter q; the sums of the MFMA before each are scaled and added while it runs
    auto group = [&](i32x8 (&b)[2], auto Qn, auto Gn) {
        constexpr int q = decltype(Qn)::value, g = decltype(Gn)::value;
        constexpr int pg = g ? g - 1 : 3, pq = g ? q : (q + 3) % 4;
        d[0] = block_sum<false>(b[0], a[g]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[pg][2 * pq + 1][v] = __builtin_fmaf(d[1][v], pf, acc[pg][2 * pq + 1][v]);
        __builtin_amdgcn_sched_barrier(0);
        d[1] = block_sum<false>(b[1], a[g]);
        __builtin_amdgcn_sched_barrier(0);
        pf = s[g];
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[g][2 * q][v] = __builtin_fmaf(d[0][v], pf, acc[g][2 * q][v]);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto load_s = [&](int buf) {
        if constexpr (LOAD_A) {
            lds_dma4(sc.src, sc.off, sc.dst + buf * kBM * 4);
            sc.src += sc.step;
        }
    };
    auto N0 = std::integral_constant<int, 0>{};
    auto N1 = std::integral_constant<int, 1>{};
    auto N2 = std::integral_constant<int, 2>{};
    auto N3 = std::integral_constant<int, 3>{};
    const int first = KT & 1;
    load_s(first);
    if constexpr (LOADER) {
        load_half0(ld, LOAD_A, a_lds, b_lds, first);
        load_half1(ld, b_lds, first);
        wait_vm<0>();
    }
    block_barrier();                                   // the first stage is visible
    if constexpr (LOADER) {
        if (KT > 1) {
            load_s(first ^ 1);
            load_half0(ld, LOAD_A, a_lds, b_lds, first ^ 1);
        }
    }
    if constexpr (ACTIVE) {
        static_for<2>([&](auto N) { read_b(b0, first, 0, N); });
        static_for<2>([&](auto N) { read_a(first, N); });
    }
    int kt = 0;
    auto stage = [&](auto BUF, auto STEP) {
        constexpr int buf = decltype(BUF)::value;
        constexpr KStep step = decltype(STEP)::value;
        constexpr bool next1 = step != kLast, next2 = next1 && step != kLast2;   // stages kt + 1, kt + 2 exist
        if constexpr (ACTIVE) read_s(buf, kt, false);
        static_for<4>([&](auto G) {                                            // quarter 0
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) read_a(buf, std::integral_constant<int, 2 + G.value>{});
                else read_b(b1, buf, 1, std::integral_constant<int, G.value - 2>{});
                group(b0, N0, G);
            }
            if constexpr (LOADER && next1) load_b<1, G.value>(ld, b_lds, buf ^ 1);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (LOADER && next1) step_half1(ld);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // A, quarters 0 and 1 read
        if constexpr (LOADER) wait_vm<next1 ? kA + kS + 8 : 0>();   // quarters 2, 3 of stage kt landed
        block_barrier();                                         // barrier a
        static_for<4>([&](auto G) {                                            // quarter 1
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) read_b(b0, buf, 2, G);
                group(b1, N1, G);
            }
            if constexpr (LOAD_A && next2) load_a<G.value>(ld, a_lds, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (ACTIVE && SWIGLU) read_s(buf, kt, true);
        static_for<4>([&](auto G) {                                            // quarter 2
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) read_b(b1, buf, 3, G);
                group(b0, N2, G);
            }
            if constexpr (LOAD_A && next2) load_a<4 + G.value>(ld, a_lds, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // quarters 2, 3 and the scales read
        if constexpr (LOADER && next1) wait_vm<next2 ? kA + 4 : 4>();   // A, quarters 0, 1, scales of stage kt + 1 landed
        block_barrier();                                         // barrier c
        static_for<4>([&](auto G) {                                            // quarter 3
            if constexpr (ACTIVE) {
                if constexpr (next1) {
                    if constexpr (G.value < 2) read_b(b0, buf ^ 1, 0, G);
                    else read_a(buf ^ 1, std::integral_constant<int, G.value - 2>{});
                }
                group(b1, N3, G);
            }
            if constexpr (LOADER && next2) load_b<0, G.value>(ld, b_lds, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (LOADER && next2) {
            load_s(buf);
            step_half0(ld);
        }
        ++kt;
    };
    auto M = std::integral_constant<KStep, kMiddle>{};
    if (KT == 1) {
        stage(N1, std::integral_constant<KStep, kLast>{});
    } else {
        if (first) stage(N1, M);
        while (kt + 2 < KT) {
            stage(N0, M);
            stage(N1, M);
        }
        stage(N0, std::integral_constant<KStep, kLast2>{});
        stage(N1, std::integral_constant<KStep, kLast>{});
    }
    if constexpr (ACTIVE) {
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[3][7][v] = __builtin_fmaf(d[1][v], pf, acc[3][7][v]);
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

// N % 16 == 0: a loader's 16 weight rows of a quarter are all there or all past the end
// (then those of the last 16 outputs are loaded, and nothing of them stored).
template <typename OUT>
__global__ __launch_bounds__(512) void f8_wide_kernel(const F8Args a) {
    constexpr bool kSwiglu = std::is_same<OUT, uint8_t>::value;
    constexpr int kCols = kSwiglu ? kBN / 2 : kBN;
    __shared__ __align__(16) uint8_t lds[2 * kStageBytes];
    __shared__ float lds_sx[2 * kBM];
    __shared__ float lds_sw[2 * kF8MaxStages];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave / kWavesN, wn = wave % kWavesN;
    const int KT = a.KT, K = KT * 128, NT = (a.N + kCols - 1) / kCols;
    Tile tile;
    if (!find_tile<kBM>(a, NT, tile)) return;
    const int n0 = tile.nt * kCols, NB = (a.N + 127) / 128;
    {
        const size_t first = (static_cast<size_t>(tile.e) * NB + n0 / 128) * KT;
        for (int i = threadIdx.x; i < KT; i += 512) {
            lds_sw[i] = a.s1[first + i];
            lds_sw[KT + i] = kSwiglu ? a.s3[first + i] : a.s1[(n0 / 128 + 1 < NB ? first + KT : first) + i];
        }
    }
    const bool loader = wave < kNL, active = tile.m0 + wm * kWM < tile.end;
    Loads ld = {};
    WideScales sc = {};
    const LaneMap lm = lane_map(lane);
    if (loader) {
        ld.a_on = tile.m0 + wave / kWavesN * kWM < tile.end;
        const size_t expert = static_cast<size_t>(tile.e) * a.N;
        const int c = wave >> 1, h = (wave & 1) * 16;
        auto rows_at = [&](const uint8_t* w, int n) {
            n = n < a.N ? n : a.N - 16;
            return reinterpret_cast<const char*>(w + (expert + n) * K);
        };
        if constexpr (kSwiglu) {                       // 64 of W1, then 64 of W3, for each of the two wave columns
            const int n = n0 + 64 * c + h;
            ld.b0 = rows_at(a.w1, n);
            ld.b1 = rows_at(a.w1, n + 32);
            ld.c0 = rows_at(a.w3, n);
            ld.c1 = rows_at(a.w3, n + 32);
        } else {
            const int n = n0 + 128 * c + h;
            ld.b0 = rows_at(a.w1, n);
            ld.b1 = rows_at(a.w1, n + 32);
            ld.c0 = rows_at(a.w1, n + 64);
            ld.c1 = rows_at(a.w1, n + 96);
        }
        auto source_row = [&](int r) {                 // rows past the end repeat the last
            int row = tile.m0 + r;
            row = row < tile.end ? row : tile.end - 1;
            if (a.row_src) {
                row = a.row_src[row];
                row = row < 0 ? 0 : row < a.x_rows ? row : a.x_rows - 1;
            }
            return static_cast<uint32_t>(row);
        };
        ld.a = reinterpret_cast<const char*>(a.x);
#pragma unroll
        for (int i = 0; i < 2; ++i) ld.b_off[i] = (i * kRowsPerLoad + lm.ld_row) * K + lm.col_b[i];
#pragma unroll
        for (int i = 0; i < kALd; ++i)
            ld.a_off[i] = source_row(wave * kWM + i * kRowsPerLoad + lm.ld_row) * K + lm.col_b[i & 1];
        sc.src = reinterpret_cast<const char*>(a.sx + tile.m0 + wave * kWM);
        sc.step = a.sx_block * 4;
        sc.off = lane * 4;
        sc.dst = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds_sx)) + wave * kWM * 4;
    }
    sc.sx = lds_sx + wm * kWM + lm.fr_row;
    sc.sw = lds_sw + (kSwiglu ? 0 : wn * KT);
    const uint32_t lds_base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>((lds_void*)lds));
    const uint32_t a_lds = lds_base + wave * kALd * 1024;
    const uint32_t b_lds = lds_base + (kBM + (wave >> 1) * kWN + (wave & 1) * 16) * kRowB;
    f32x4 acc[kMI][kNJ];
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNJ; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();                                   // the weights' scales; no load of the loop is under way yet
    if (loader) {
        if (active) f8_k_loop<kSwiglu, true, true>(KT, lds, wm, wn, lane, acc, ld, sc, a_lds, b_lds);
        else f8_k_loop<kSwiglu, true, false>(KT, lds, wm, wn, lane, acc, ld, sc, a_lds, b_lds);
    } else {
        if (active) f8_k_loop<kSwiglu, false, true>(KT, lds, wm, wn, lane, acc, ld, sc, a_lds, b_lds);
        else f8_k_loop<kSwiglu, false, false>(KT, lds, wm, wn, lane, acc, ld, sc, a_lds, b_lds);
    }
    if constexpr (kSwiglu) finish_tile<kBM, kBN, kWavesM, kWavesN, OUT>(a, tile, n0, wm, wn, lane, acc, lds);
    else store_wide(a, tile, n0, wm, wn, wave, lane, acc, lds);
}

template <int BM, int BN, int NWM, int NWN, typename OUT>
cap_status launch_tiles(const F8Args& a, hipStream_t st) {
    constexpr int cols = std::is_same<OUT, uint8_t>::value ? BN / 2 : BN;
    const long long rows = a.max_rows / BM + (a.E_loc < a.max_rows ? a.E_loc : a.max_rows);
    const long long blocks = (rows * ((a.N + cols - 1) / cols) + 7) / 8 * 8;
    if (blocks * (64 * NWM * NWN) >= (1ll << 32)) return CAP_ERR_UNSUPPORTED;
    f8_tile_kernel<BM, BN, NWM, NWN, OUT><<<static_cast<unsigned>(blocks), 64 * NWM * NWN, 0, st>>>(a);
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

// Wide tiles: enough rows that their weights' passes through the tiles count for less
// than the halves of tiles that stay empty.
bool wide_rows(int max_rows) { return max_rows >= 8192; }

template <typename OUT>
cap_status launch_wide(F8Args a, float* scales, hipStream_t st) {
    constexpr int cols = std::is_same<OUT, uint8_t>::value ? kBN / 2 : kBN;
    const long long rows = a.max_rows / kBM + (a.E_loc < a.max_rows ? a.E_loc : a.max_rows);
    const long long blocks = (rows * ((a.N + cols - 1) / cols) + 7) / 8 * 8;
    if (blocks * 512 >= (1ll << 32)) return CAP_ERR_UNSUPPORTED;
    if (a.sx_row != 1) {
        const size_t pitch = f8_scale_pitch(a.max_rows);
        f8_gather_scales_kernel<<<(a.max_rows + 63) / 64, 256, 0, st>>>(a, scales, pitch);
        a.sx = scales;
        a.sx_row = 1;
        a.sx_block = pitch;
    }
    f8_wide_kernel<OUT><<<static_cast<unsigned>(blocks), 512, 0, st>>>(a);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace

size_t product_fp8_workspace_bytes(int, int kdim, int max_rows) {
    return wide_rows(max_rows) ? f8_scales_bytes(kdim, max_rows) : 0;
}

// H's codes, its scales, and the scales of x in the rows' order.
size_t ffn_fp8_workspace_bytes(int d, int inter, int max_rows) {
    const size_t codes = (static_cast<size_t>(max_rows) * inter + 255) & ~size_t(255);
    return codes + f8_scales_bytes(inter, max_rows) + (wide_rows(max_rows) ? f8_scales_bytes(d, max_rows) : 0);
}

namespace {

cap_status product(cap_dtype out_dtype, const F8Args& a, float* scales, hipStream_t st) {
    if (out_dtype == CAP_DTYPE_F32) return launch_tiles<128, 128, 2, 2, float>(a, st);
    if (wide_rows(a.max_rows) && a.N % 16 == 0 && (reinterpret_cast<uintptr_t>(a.out) & 15) == 0)
        return launch_wide<uint16_t>(a, scales, st);
    return launch_tiles<128, 128, 2, 2, uint16_t>(a, st);
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
    uint8_t* const h = static_cast<uint8_t*>(ws);
    float* const sh = reinterpret_cast<float*>(h + ((static_cast<size_t>(max_rows) * inter + 255) & ~size_t(255)));
    float* const sxt = sh + f8_scales_bytes(inter, max_rows) / 4;
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
    a.out = h;
    a.out_scale = sh;
    a.scale_pitch = f8_scale_pitch(max_rows);
    a.x_rows = x_rows;
    a.E_loc = E_loc;
    a.max_rows = max_rows;
    a.N = inter;
    a.KT = d / 128;
    const cap_status first = wide_rows(max_rows) ? launch_wide<uint8_t>(a, sxt, st) : launch_tiles<128, 256, 2, 4, uint8_t>(a, st);
    if (first != CAP_OK) return first;
    a.x = h;
    a.sx = sh;
    a.sx_row = 1;
    a.sx_block = a.scale_pitch;
    a.row_src = nullptr;
    a.w1 = static_cast<const uint8_t*>(w2);
    a.s1 = s2;
    a.out = y;
    a.x_rows = max_rows;
    a.N = d;
    a.KT = inter / 128;
    return product(CAP_DTYPE_BF16, a, nullptr, st);
}

}  // namespace cap
