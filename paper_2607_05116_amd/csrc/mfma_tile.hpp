// Building blocks of the 16-bit matrix kernels (gfx950 MFMA, fp32 accumulation):
// direct-to-LDS loads, the LDS stage layout and its swizzle, fragment reads, and
// the K loop of a 256 x 256 tile.  Fragment type F is bf16x8 or f16x8.
#pragma once

#include "cap_device.hpp"

#include <type_traits>

namespace cap {
namespace {

// Compile-time loop: f(std::integral_constant<int, 0>) ... f(<N - 1>).
template <int N, int I = 0, typename F>
__device__ __forceinline__ void static_for(F&& f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<N, I + 1>(f);
    }
}

// Scalar base of a direct load: uniform by construction; readfirstlane keeps it
// in scalar registers (widening through uint32_t so the low word is never
// sign-extended).
__device__ __forceinline__ const void* uniform_ptr(const void* p) {
    const uint64_t b = reinterpret_cast<uint64_t>(p);
    const uint64_t lo = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b)));
    const uint64_t hi = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<uint32_t>(b >> 32)));
    return reinterpret_cast<const void*>((hi << 32) | lo);
}

// Wave-wide copies global -> LDS (gfx950 global_load_lds_dwordx4): lane i
// reads 16 bytes at base + voff_i and they land at LDS byte M0 + 16 * i; base
// is a scalar register pair, voff a 32-bit per-lane byte offset, and the
// instruction's immediate offset stays 0 (it would shift the LDS address too).
// They are inline assembly so that the compiler's wait-count pass does not
// treat every later LDS read as aliasing them (it would drain all in-flight
// stages); the kernel waits on them explicitly.  Because the compiler does not
// see the instruction, it also does not insert the wait states the hardware
// needs before it: a VALU write of an SGPR (v_readfirstlane of the base, or a
// reload of a spilled scalar) needs 5 wait states before a vector-memory
// instruction reads it, and an SALU write of M0 needs 1 before an LDS DMA.  The
// statement copies the base with s_mov_b64, which waits for the VALU write by
// itself, is no hazard for the load, and separates it from the M0 write: 3
// issue slots, where an s_nop 4 took 7.
__device__ __forceinline__ void lds_dma16(const void* base, uint32_t off, uint32_t lds_addr) {
    uint64_t b;
    asm volatile("s_mov_b64 %0, %2\n\tglobal_load_lds_dwordx4 %1, %0"
                 : "=&s"(b)
                 : "v"(off), "s"(uniform_ptr(base)), "{m0}"(__builtin_amdgcn_readfirstlane(lds_addr))
                 : "memory");
}

// ------------------------------------------------------------------ 16-bit MFMA GEMM
// LDS holds kStages stages; a stage is the A tile [BM][64] and the B tile
// [BN][64] (bf16 or fp16, 128-byte rows).  A stage row is one whole 128-byte line of
// the K-contiguous operand: the direct-to-LDS path moves full lines at about
// twice the rate of half lines, which is what sets the stage depth to K = 64.
// 16-byte chunk c of row r sits at physical chunk c ^ lds_swz(r); fragment
// reads (16 consecutive rows, one chunk) then hit distinct banks for both 128-
// and 256-byte bank windows.
constexpr int kStageK = 64;                 // K per stage
constexpr int kStages = 2;                  // stage kt lives in buffer kt % 2
constexpr int kRowB = kStageK * 2;          // bytes per LDS row
constexpr int kChunks = kRowB / 16;         // 16-byte chunks per row

__device__ __forceinline__ int lds_swz(int r) { return (r & 7) ^ ((r >> 3) & 1); }

// Workgroup barrier without the memory fence that __syncthreads() carries (the
// fence would drain every in-flight prefetch).  LDS visibility is ensured by
// explicit waits: vmcnt for the direct-to-LDS loads, and lgkmcnt(0) before a
// barrier that publishes ds_write data (staged outputs, broadcast values); the
// empty asm statements keep memory accesses from being moved across the
// barrier.
__device__ __forceinline__ void block_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

typedef __attribute__((address_space(3))) void lds_void;


// ------------------------------------------------------------------ shared tile pieces
// Block tile 256 x 256, eight waves in a 4 x 2 grid, each wave 64 x 128.
constexpr int kBM = 256, kBN = 256, kWavesM = 4, kWavesN = 2;
constexpr int kNW = kWavesM * kWavesN;
constexpr int kNL = kNW / 2;                          // loader waves; the rest are storers
constexpr int kWM = kBM / kWavesM, kWN = kBN / kWavesN;
constexpr int kMI = kWM / 16, kNJ = kWN / 16;         // 16 x 16 MFMA blocks per wave
constexpr int kRowsPerLoad = 1024 / kRowB;            // rows one wave-wide 16-byte load covers
constexpr int kALd = kBM / kRowsPerLoad / kNL;        // direct loads per loader wave per stage
constexpr int kBLd = kBN / kRowsPerLoad / kNL;
constexpr int kStageBytes = (kBM + kBN) * kRowB;
static_assert(kNL % 4 == 0, "one loader and one storer wave per SIMD");
static_assert(kBM % (kRowsPerLoad * kNL) == 0 && kBN % (kRowsPerLoad * kNL) == 0, "load split");
static_assert(kALd + kBLd <= 60, "loads per stage must fit the vmcnt field");
static_assert(kWN % 64 == 0, "gate/up pairs need 64-column wave tiles");
static_assert(kNL == 4 && kBLd == 8 && kRowsPerLoad == 8, "a loader takes 16 rows of each B quarter");
static_assert(kMI == 4 && kNJ == 8, "quarters of two B blocks, A blocks in pairs");
static_assert(kALd * kRowsPerLoad == kWM, "loader wave w loads the A rows that waves of row w read");
static_assert(kStageK == 64, "a stage is two MFMA K steps of 32");
static_assert(kStages == 2, "staging lives in stage buffer 1");

// Per-lane constants of the direct loads and the fragment reads.
struct LaneMap {
    int ld_row;          // direct loads: lane l writes row l / 8 of its 1 KiB block ...
    uint32_t col_b[2];   // ... at physical chunk l % 8, fetching logical chunk (l % 8) ^ swz(row):
                         // the swizzle of row (8 * blk + l / 8) is swz(l / 8) ^ (blk & 1)
    int fr_row, fr_swz, fr_kc;     // fragment reads: row r = ... + lane % 16, K chunk kc(lane / 16)
};
__device__ __forceinline__ LaneMap lane_map(int lane) {
    LaneMap m;
    m.ld_row = lane >> 3;
    const int pc = lane & (kChunks - 1);
    m.col_b[0] = static_cast<uint32_t>((pc ^ lds_swz(m.ld_row)) * 16);
    m.col_b[1] = static_cast<uint32_t>((pc ^ lds_swz(kRowsPerLoad + m.ld_row)) * 16);
    m.fr_row = lane & 15;
    m.fr_swz = lds_swz(m.fr_row);
    // K chunk of lane group g = lane / 16 within a K step: 0, 2, 1, 3, so
    // that lanes l and l + 32 (read in one LDS pass) take chunks of opposite
    // parity and, under the row swizzle, distinct banks
    m.fr_kc = ((lane >> 3) & 2) | (lane >> 5);
    return m;
}

// The same value, opaque to the compiler: what is derived from it is formed
// where it is used, per tile, and not kept in registers across the K loop.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}

// Fragments and MFMAs.  One MFMA K step is K = 32 (two per stage).  Lane
// (r, g) = (lane % 16, lane / 16) reads row r of each 16-row block at 16-byte
// chunk 4 ks + kc(g) of K step ks, kc = (0, 2, 1, 3) (8 consecutive K; A and
// B take the same K positions, so the contraction pairs them correctly
// whatever order the hardware sums them in).  The MFMA takes the weight fragment as its first
// operand, so a lane's 4 accumulators of block (i, j) hold output columns
// 16 j + 4 q + 0..3 of tile row 16 i + r.
template <typename F>
__device__ __forceinline__ const F& frag_at(const uint8_t* p) { return *reinterpret_cast<const F*>(p); }

// Loads of one tile for one loader wave.  A: rows wave * 64 .. + 63, 8 loads a
// stage (lane l of load i: byte offset a_off[i] from the operand base: a tile
// row, clamped to the expert's last, or a gathered row of x), none of them by
// a loader whose own wave computes nothing (a_on: wave row w / 2 has rows; the
// rows 64 w .. it loads come after those).  B: of quarter q
// (rows wn * 128 + 32 q .. + 31 of both wave columns wn) the 16 rows wn =
// wave / 2, 16 (wave % 2) ..: 2 loads a quarter.  The pointers run along K:
// a and b0 / b1 (quarters 0, 1) one stage ahead of c0 / c1 (quarters 2, 3).
struct Loads {
    const char *a, *b0, *b1, *c0, *c1;
    uint32_t a_off[kALd];
    uint32_t b_off[2];
    bool a_on;
};

template <int I>
__device__ __forceinline__ void load_a(const Loads& s, uint32_t a_lds, int buf) {
    lds_dma16(s.a, s.a_off[I], a_lds + buf * kStageBytes + I * 1024);
}
// load I = 0..3 of quarters 0, 1 (half 0) or 2, 3 (half 1)
template <int HALF, int I>
__device__ __forceinline__ void load_b(const Loads& s, uint32_t b_lds, int buf) {
    const char* p = HALF ? (I / 2 ? s.c1 : s.c0) : (I / 2 ? s.b1 : s.b0);
    lds_dma16(p, s.b_off[I % 2],
              b_lds + buf * kStageBytes + (HALF * 64 + (I / 2) * 32 + (I % 2) * kRowsPerLoad) * kRowB);
}
__device__ __forceinline__ void step_half0(Loads& s) { s.a += kRowB; s.b0 += kRowB; s.b1 += kRowB; }
__device__ __forceinline__ void step_half1(Loads& s) { s.c0 += kRowB; s.c1 += kRowB; }
__device__ __forceinline__ void load_half0(Loads& s, bool a_on, uint32_t a_lds, uint32_t b_lds, int buf) {
    if (a_on) static_for<kALd>([&](auto I) { load_a<I.value>(s, a_lds, buf); });
    static_for<4>([&](auto I) { load_b<0, I.value>(s, b_lds, buf); });
    step_half0(s);
}
__device__ __forceinline__ void load_half1(Loads& s, uint32_t b_lds, int buf) {
    static_for<4>([&](auto I) { load_b<1, I.value>(s, b_lds, buf); });
    step_half1(s);
}

// The K loop of one tile: KT stages of K = 64 (KT is even: d % 256 == 0 and
// inter % 128 == 0), stage kt in buffer kt % 2.  A stage is computed in four
// quarters (Q = 0..3: all A blocks with B blocks 2 Q, 2 Q + 1), and each
// quarter's B fragments are read during the quarter before it (two register
// sets in turn).  The A fragments of the next stage replace this one's in
// place: blocks 0, 1 after their last MFMA in quarter 3, blocks 2, 3 at the
// start of the next quarter 0.  So a part of a stage stays in LDS only while
// one or two quarters read it, and its space takes the loads of the stage two
// ahead from then on:
//   barrier a (after quarter 0):  A and B quarters 0, 1 of stage kt are read;
//                                 B quarters 2, 3 of stage kt are complete.
//   barrier c (after quarter 2):  B quarters 2, 3 of stage kt are read; A and
//                                 B quarters 0, 1 of stage kt + 1 are complete.
// A quarter is four groups of four MFMAs; a group starts with its fragment
// reads and ends, in a loader wave, with its direct loads, spread so that the
// address path takes them while the MFMAs run: A of stage kt + 2 in quarters
// 1, 2, its B quarters 0, 1 in quarter 3, its B quarters 2, 3 in quarter 0 of
// stage kt + 1.
//   hook(step)       bookkeeping of the caller, none of it in the middle of the
//                    loop: after barrier a of the first (kFirst) and second
//                    stage (kSecond; both only if KT > 2), of the last but one
//                    (kLast2), before (kPreLast) and after (kLast) that of the
//                    last.
// On entry stage 0 has been issued whole; on return every wave is past its
// last LDS read of the tile (barrier c of the last stage), and buffer 0 was
// free from barrier a of the last stage (the hook may issue the next tile's
// stage 0).
// What bounds it: the board's power (under the counters the MFMA pipes are 73 %
// busy at 1.7 GHz on the 33,234 rows of d = 7168, inter = 2048, where loading
// each stage whole behind one barrier kept them 62 % busy at 1.8 GHz), then the
// LDS, whose fragment reads and direct writes need 256 KB a stage, the time of
// its MFMAs at 128 bytes a clock; on tiles of few stages (a down tile of inter =
// 768 has twelve) also the next tile's stage 1, which cannot be issued before
// the epilogue has given its buffer back.  That call 2328 -> 2131 us, 44,420
// rows of d = 2048, inter = 768 393 -> 358 us, 3,001 rows of d = 2048, inter =
// 1408 98 -> 89 us.  Issuing twelve of a stage's sixteen loads in quarters 1 and
// 2 was no faster, nor a raised wave priority around the MFMAs or for the
// loaders (0 to 2 % slower).
// A wave whose 64 rows all lie past the tile's valid rows (active = false)
// computes nothing: its accumulators stay zero and are never stored.  A loader
// among them loads no A either, and its waits count without those loads: tiles
// of 64 rows or fewer then bring 16 KB of A a stage instead of 32.  (A third
// form of the loop for the loaders of which only the rows they load lie past
// the end was 1 to 4 % slower on 300 rows an expert of d = 7168.)
template <int N>
__device__ __forceinline__ void wait_vm() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

// acc += b a^T in place, as inline assembly: with most of the registers taken,
// the register allocator otherwise moves accumulators about (24 spilled
// registers and copies at every tile's end; 2172 -> 2131 us on the 33,234 rows
// of d = 7168, inter = 2048, 372 -> 358 us on 44,420 rows of d = 2048, inter =
// 768).  The compiler inserts no wait states around it: acc_pin and the s_nop
// before and after the K loop separate the MFMAs from the code that writes and
// reads the accumulators; fragment operands come from LDS reads, whose wait it
// does insert.
__device__ __forceinline__ void mfma_acc(f32x4& acc, const bf16x8& b, const bf16x8& a) {
    asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc) : "v"(b), "v"(a));
}
__device__ __forceinline__ void mfma_acc(f32x4& acc, const f16x8& b, const f16x8& a) {
    asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+v"(acc) : "v"(b), "v"(a));
}
__device__ __forceinline__ void acc_pin(f32x4 (&acc)[kMI][kNJ]) {
#pragma unroll
    for (int i = 0; i < kMI; ++i)
#pragma unroll
        for (int j = 0; j < kNJ; ++j) asm volatile("" : "+v"(acc[i][j]));
}
enum KStep { kMiddle, kFirst, kSecond, kLast2, kPreLast, kLast };

template <typename F, bool LOADER, bool ACTIVE, typename Hook>
__device__ __forceinline__ void k_loop(int KT, const uint8_t* lds, int wm, int wn, int lane, f32x4 (&acc)[kMI][kNJ], Loads& ld, uint32_t a_lds, uint32_t b_lds,
                                       Hook&& hook) {
    constexpr bool LOAD_A = LOADER && ACTIVE;
    constexpr int kA = LOAD_A ? kALd : 0;              // this wave's A loads of a stage
    F a[kMI][2], b0[2][2], b1[2][2];
    const LaneMap lm = lane_map(opaque(lane));
    const int pc0 = (lm.fr_kc ^ lm.fr_swz) << 4, pc1 = pc0 ^ 64;
    const uint8_t* const la = lds + (wm * kWM + lm.fr_row) * kRowB;
    const uint8_t* const lb = lds + (kBM + wn * kWN + lm.fr_row) * kRowB;
    // fragment n = 0..3 of A blocks i0, i0 + 1 / of quarter q: K step n / 2
    auto read_a = [&](int buf, int i0, auto Nn) {
        constexpr int n = decltype(Nn)::value;
        a[i0 + n % 2][n / 2] = frag_at<F>(la + buf * kStageBytes + (i0 + n % 2) * 16 * kRowB + (n / 2 ? pc1 : pc0));
    };
    auto read_b = [&](F (&b)[2][2], int buf, int q, auto Nn) {
        constexpr int n = decltype(Nn)::value;
        b[n % 2][n / 2] = frag_at<F>(lb + buf * kStageBytes + (2 * q + n % 2) * 16 * kRowB + (n / 2 ? pc1 : pc0));
    };
    // MFMA group g = 0..3 of quarter Q.  Quarters 1, 2: K step g / 2, A blocks
    // 2 (g % 2) ..; quarters 0, 3: A blocks 2 (g / 2) .., K step g % 2 (the A
    // fragments change hands half way).
    auto mfma4 = [&](F (&b)[2][2], auto Qn, auto Gn) {
        constexpr int q = decltype(Qn)::value, g = decltype(Gn)::value;
        constexpr bool by_k = q == 1 || q == 2;
        constexpr int ks = by_k ? g / 2 : g % 2, i0 = 2 * (by_k ? g % 2 : g / 2);
#pragma unroll
        for (int i = i0; i < i0 + 2; ++i)
#pragma unroll
            for (int jj = 0; jj < 2; ++jj)
                mfma_acc(acc[i][2 * q + jj], b[jj][ks], a[i][ks]);
    };
    auto N0 = std::integral_constant<int, 0>{};
    auto N1 = std::integral_constant<int, 1>{};
    auto N2 = std::integral_constant<int, 2>{};
    auto N3 = std::integral_constant<int, 3>{};
    acc_pin(acc);
    asm volatile("s_nop 7");
    if (LOADER) wait_vm<0>();
    block_barrier();                                   // stage 0 visible; buffer 1 free
    if (LOADER) load_half0(ld, LOAD_A, a_lds, b_lds, 1);
    if constexpr (ACTIVE)
        static_for<4>([&](auto N) {
            read_b(b0, 0, 0, N);
            read_a(0, 0, N);
        });
    auto stage = [&](auto BUF, auto STEP) {
        constexpr int buf = decltype(BUF)::value;
        constexpr KStep step = decltype(STEP)::value;
        constexpr bool next1 = step != kLast, next2 = next1 && step != kLast2;   // stages kt + 1, kt + 2 exist
        static_for<4>([&](auto G) {                                            // quarter 0
            if constexpr (ACTIVE) {
                if constexpr (G.value < 2) {
                    read_a(buf, 2, std::integral_constant<int, 2 * G.value>{});
                    read_a(buf, 2, std::integral_constant<int, 2 * G.value + 1>{});
                } else {
                    read_b(b1, buf, 1, std::integral_constant<int, 2 * G.value - 4>{});
                    read_b(b1, buf, 1, std::integral_constant<int, 2 * G.value - 3>{});
                }
                mfma4(b0, N0, G);
            }
            if constexpr (LOADER && next1) load_b<1, G.value>(ld, b_lds, buf ^ 1);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (LOADER && next1) step_half1(ld);
        if constexpr (step == kLast) hook(std::integral_constant<KStep, kPreLast>{});
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // A, quarters 0 and 1 read
        if constexpr (LOADER) {                                  // quarters 2, 3 of stage kt landed
            wait_vm<next1 ? kA + 8 : 0>();
        }
        block_barrier();                                         // barrier a
        if constexpr (step != kMiddle) hook(STEP);
        static_for<4>([&](auto G) {                                            // quarter 1
            if constexpr (ACTIVE) {
                read_b(b0, buf, 2, G);
                mfma4(b1, N1, G);
            }
            if constexpr (LOAD_A && next2) load_a<G.value>(ld, a_lds, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        static_for<4>([&](auto G) {                                            // quarter 2
            if constexpr (ACTIVE) {
                read_b(b1, buf, 3, G);
                mfma4(b0, N2, G);
            }
            if constexpr (LOAD_A && next2) load_a<4 + G.value>(ld, a_lds, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");       // quarters 2, 3 read
        if constexpr (LOADER && next1) {                         // A, quarters 0, 1 of stage kt + 1 landed
            wait_vm<next2 ? kA + 4 : 4>();
        }
        block_barrier();                                         // barrier c
        static_for<4>([&](auto G) {                                            // quarter 3
            if constexpr (ACTIVE) {
                if constexpr (next1) {
                    if constexpr (G.value < 2) {
                        read_b(b0, buf ^ 1, 0, std::integral_constant<int, 2 * G.value>{});
                        read_b(b0, buf ^ 1, 0, std::integral_constant<int, 2 * G.value + 1>{});
                    } else if constexpr (G.value == 2) {
                        static_for<4>([&](auto N) { read_a(buf ^ 1, 0, N); });
                    }
                }
                mfma4(b1, N3, G);
            }
            if constexpr (LOADER && next2) load_b<0, G.value>(ld, b_lds, buf);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (LOADER && next2) step_half0(ld);
    };
    int kt = 0;
    if constexpr (!LOADER) {
        if (KT > 2) {
            stage(N0, std::integral_constant<KStep, kFirst>{});
            stage(N1, std::integral_constant<KStep, kSecond>{});
            kt = 2;
        }
    }
    for (; kt + 2 < KT; kt += 2) {
        stage(N0, std::integral_constant<KStep, kMiddle>{});
        stage(N1, std::integral_constant<KStep, kMiddle>{});
    }
    stage(N0, std::integral_constant<KStep, kLast2>{});
    stage(N1, std::integral_constant<KStep, kLast>{});
    asm volatile("s_nop 15\n\ts_nop 15");             // the last MFMAs' results are written
    acc_pin(acc);
}

// The four roles of a wave in a tile (wave-uniform): each has a loop of its
// own, all with the same barriers.
template <typename F, typename LoadHook, typename StoreHook>
__device__ __forceinline__ void run_k_loop(int KT, const uint8_t* lds, int wm, int wn, int lane,
                                           bool loader, bool active, f32x4 (&acc)[kMI][kNJ], Loads& ld,
                                           uint32_t a_lds, uint32_t b_lds, LoadHook&& load_hook,
                                           StoreHook&& store_hook) {
    if (loader) {
        if (active) k_loop<F, true, true>(KT, lds, wm, wn, lane, acc, ld, a_lds, b_lds, load_hook);
        else k_loop<F, true, false>(KT, lds, wm, wn, lane, acc, ld, a_lds, b_lds, load_hook);
    } else {
        if (active) k_loop<F, false, true>(KT, lds, wm, wn, lane, acc, ld, a_lds, b_lds, store_hook);
        else k_loop<F, false, false>(KT, lds, wm, wn, lane, acc, ld, a_lds, b_lds, store_hook);
    }
}

}  // namespace
}  // namespace cap
