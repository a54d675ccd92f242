// Device-side helpers shared by the CAP kernels (gfx950 / CDNA4, wave64).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cap.h"

namespace cap {

constexpr int kWave = 64;
constexpr int kMaxK = 8;
constexpr int kMaxE = 256;
constexpr int kMaxR = 64;
constexpr int kMaxLossTokens = INT32_MAX - 4095, kMaxLossSequences = 1 << 30;   // of the router's training
constexpr int kMaxOrthSide = 65536, kMaxOrthBatch = 65535, kMaxOrthSteps = 16;
constexpr int kMaxScoreGroups = 64;                   // groups of cap_route_scores: one bit each
constexpr int kF8Block = 128;                         // values that share a scale in 8-bit floating point
constexpr int kF8MaxK = 1 << 15, kF8MaxStages = kF8MaxK / kF8Block;   // K of the products in 8 bits
constexpr int kMaxDevices = 64;                       // per-device caches of host code
constexpr size_t kLayoutScratchBytes = size_t(4) << 20;   // cap_dispatch_layout_static's workspace

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
// 16- and 8-byte raw vectors (native clang vector: stay in registers, unlike HIP's uint4 struct)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// bf16 <-> fp32 on raw 16-bit patterns.
__device__ __forceinline__ float bf16_to_f32(uint16_t b) {
    return __uint_as_float(static_cast<uint32_t>(b) << 16);
}

// Round to nearest, ties to even (finite inputs).
__device__ __forceinline__ uint16_t f32_to_bf16(float f) {
    uint32_t u = __float_as_uint(f);
    u += 0x7FFFu + ((u >> 16) & 1u);
    return static_cast<uint16_t>(u >> 16);
}

// Two fp32 -> packed bf16x2 (low half = a).
__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    return static_cast<uint32_t>(f32_to_bf16(a)) | (static_cast<uint32_t>(f32_to_bf16(b)) << 16);
}

// Two fp32 -> packed bf16x2 with the hardware conversion (v_cvt_pk_bf16_f32,
// round to nearest even: the same bits as pack_bf16x2 for finite inputs).
typedef __bf16 bf16x2_hw __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_bf16x2_rne(float a, float b) {
    const bf16x2_hw v = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
    return __builtin_bit_cast(uint32_t, v);
}

__device__ __forceinline__ int lane_id() { return __lane_id(); }

// 64-bit masks by a lane's own bit number, in shifts of 32 bits.  A 64-bit shift whose amount is the last vector
// register that the kernel has is taken to give wrong results now and then, in whole waves: of 2,406 such shifts by
// a register in the 172 kernels of the routing by scores 7 were of that form, one each in 7 kernels, and the drawn
// cases whose gates came out wrong (9 of 19,800) all ran kernels among these 7.  Which register it is, is the
// compiler's choice, so no kernel of this library shifts 64 bits by one.
struct Bits {
    uint32_t lo, hi;
};
// (Two words for the compiler too, which would put 64-bit shifts together again.)
__device__ __forceinline__ void keep_apart(Bits& b) { asm("" : "+v"(b.lo), "+v"(b.hi)); }
__device__ __forceinline__ Bits split_bits(uint64_t m) {
    Bits b = {static_cast<uint32_t>(m), static_cast<uint32_t>(m >> 32)};
    keep_apart(b);
    return b;
}
__device__ __forceinline__ uint64_t join_bits(Bits b) {
    keep_apart(b);
    return static_cast<uint64_t>(b.hi) << 32 | b.lo;
}
// Bit i.  (A choice between the two words by a condition is one between their addresses for the compiler, which
// then keeps them in memory: in LDS, at a place that it works out from the dispatch packet, which lies in host memory.)
__device__ __forceinline__ bool has_bit(const Bits& m, int i) {
    const uint32_t high = 0u - (static_cast<uint32_t>(i) >> 5 & 1u);
    return ((m.hi & high) | (m.lo & ~high)) >> (i & 31) & 1u;
}
__device__ __forceinline__ bool has_bit(uint64_t m, int i) { return has_bit(split_bits(m), i); }
__device__ __forceinline__ uint64_t bit64(int i, bool set = true) {
    const uint32_t b = (set ? 1u : 0u) << (i & 31), high = 0u - (static_cast<uint32_t>(i) >> 5 & 1u);
    return join_bits(Bits{b & ~high, b & high});
}
// Bits 0 .. i - 1 (of 0 <= i < 64), and 0 .. i.
__device__ __forceinline__ Bits bits_below(int i) {
    const uint32_t part = (1u << (i & 31)) - 1u, high = 0u - (static_cast<uint32_t>(i) >> 5 & 1u);
    return Bits{part | high, part & high};
}
__device__ __forceinline__ Bits bits_through(int i) {
    const uint32_t part = (2u << (i & 31)) - 1u, high = 0u - (static_cast<uint32_t>(i) >> 5 & 1u);
    return Bits{part | high, part & high};
}
// How many of the bits in `of` are set.
__device__ __forceinline__ int count_bits(const Bits& m, const Bits& of) {
    return __popc(m.lo & of.lo) + __popc(m.hi & of.hi);
}

// Mask of lanes below the calling lane.
__device__ __forceinline__ Bits lanemask_lt() { return bits_below(lane_id()); }

// floor(n / d) for 0 <= n < 2^31 and 1 <= d < 2^31 with a quotient below
// 2^16: the fp32 estimate n * rcp(d) is within 2^-21 of n / d relative (so
// within one of the quotient), and one correction step each way makes it exact.
__device__ __forceinline__ int small_quotient(int n, int d) {
    int q = static_cast<int>(static_cast<float>(n) * __builtin_amdgcn_rcpf(static_cast<float>(d)));
    const long long r = static_cast<long long>(n) - static_cast<long long>(q) * d;
    q += (r >= d) ? 1 : 0;
    q -= (r < 0) ? 1 : 0;
    return q;
}

// Grid-wide launch helpers: compute units and XCDs of the current device.
int device_cu_count();
int device_xcc_count();

}  // namespace cap

#define CAP_LAUNCH_CHECK()                                      \
    do {                                                        \
        if (hipGetLastError() != hipSuccess) return CAP_ERR_HIP; \
    } while (0)
