// Quantisation to e4m3 with a power-of-two scale for each block of 128 (see
// fp8_device.hpp): blocks of 1 x 128 (rows of activations) or 128 x 128 (weights).
//
// Both read each value once and write each code once, so memory bounds them: 32,768 rows of
// 7168 in bf16 126 us (5.6 TB/s of 712 MB), weights of 16 x 768 x 2048 in fp32 26 us (4.8
// TB/s of 126 MB; 21.8 us if they were read just before, and lie in the last-level cache); a copy
// reaches 4.85 TB/s, writing alone 6.9.
#include <hip/hip_runtime.h>

#include "fp8_device.hpp"

namespace cap {
namespace {

// Eight consecutive values as fp32.
template <typename X>
__device__ __forceinline__ void load8(const X* p, float (&v)[8]) {
    if constexpr (std::is_same<X, float>::value) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(p), b = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[i] = a[i];
            v[4 + i] = b[i];
        }
    } else {
        const u32x4 a = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(a[i] << 16);
            v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
        }
    }
}
__device__ __forceinline__ uint32_t magnitude8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t b = finite_magnitude(v[i]);
        m = b > m ? b : m;
    }
    return m;
}
__device__ __forceinline__ u32x2 codes8(const float (&v)[8], float inv) {
    return u32x2{f8_pack4(v[0], v[1], v[2], v[3], inv), f8_pack4(v[4], v[5], v[6], v[7], inv)};
}

// 1 x 128: 16 lanes a block, 8 values a lane; a thread takes kEach blocks a pass.
constexpr int kEach = 4;
template <typename X>
__global__ __launch_bounds__(256) void quantise_rows_kernel(const X* __restrict__ x, uint8_t* __restrict__ q,
                                                            float* __restrict__ scale, long long blocks) {
    const int lane16 = threadIdx.x & 15;
    const long long b0 = static_cast<long long>(blockIdx.x) * (16 * kEach) + (threadIdx.x >> 4);
    float v[kEach][8];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long b = b0 + 16 * i;
        if (b < blocks) load8(x + b * kF8Block + lane16 * 8, v[i]);
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const long long b = b0 + 16 * i;
        if (b >= blocks) break;                     // the 16 lanes of a block go together
        const uint32_t e = f8_scale_exponent(row16_max(magnitude8(v[i])));
        *reinterpret_cast<u32x2*>(q + b * kF8Block + lane16 * 8) = codes8(v[i], f8_inverse(e));
        if (lane16 == 0) scale[b] = f8_scale(e);
    }
}

// 128 x 128: one workgroup a block, 64 values a thread, kept in registers between
// the maximum and the rounding.
template <typename X>
__global__ __launch_bounds__(256) void quantise_blocks_kernel(const X* __restrict__ x, uint8_t* __restrict__ q,
                                                              float* __restrict__ scale, int rows, int cols,
                                                              int row_blocks) {
    __shared__ uint32_t wave_max[4];
    const int col_blocks = cols / kF8Block;
    const int cb = blockIdx.x % col_blocks;
    const long long rest = blockIdx.x / col_blocks;
    const int rb = static_cast<int>(rest % row_blocks);
    const long long batch = rest / row_blocks;
    const int r0 = rb * kF8Block + (threadIdx.x >> 4);
    const long long at = (batch * rows + r0) * cols + cb * kF8Block + (threadIdx.x & 15) * 8;
    float v[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (r0 + 16 * i < rows) load8(x + at + static_cast<long long>(16 * i) * cols, v[i]);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (r0 + 16 * i < rows) {
            const uint32_t b = magnitude8(v[i]);
            m = b > m ? b : m;
        }
    m = row16_max(m);
#pragma unroll
    for (int d = 16; d < 64; d *= 2) {
        const uint32_t o = static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), d));
        m = o > m ? o : m;
    }
    if ((threadIdx.x & 63) == 0) wave_max[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) m = wave_max[w] > m ? wave_max[w] : m;
    const uint32_t e = f8_scale_exponent(m);
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (r0 + 16 * i < rows)
            *reinterpret_cast<u32x2*>(q + at + static_cast<long long>(16 * i) * cols) = codes8(v[i], f8_inverse(e));
    if (threadIdx.x == 0) scale[blockIdx.x] = f8_scale(e);
}

template <typename X>
void launch(int batch, int rows, int cols, int block_rows, const void* x, void* q, float* scale, hipStream_t st) {
    const X* xs = static_cast<const X*>(x);
    uint8_t* qs = static_cast<uint8_t*>(q);
    const int col_blocks = cols / kF8Block;
    if (block_rows == 1) {
        const long long blocks = static_cast<long long>(batch) * rows * col_blocks;
        quantise_rows_kernel<X><<<static_cast<unsigned>((blocks + 16 * kEach - 1) / (16 * kEach)), 256, 0, st>>>(
            xs, qs, scale, blocks);
    } else {
        const int row_blocks = (rows + kF8Block - 1) / kF8Block;
        quantise_blocks_kernel<X><<<static_cast<unsigned>(static_cast<long long>(batch) * row_blocks * col_blocks), 256,
                                    0, st>>>(xs, qs, scale, rows, cols, row_blocks);
    }
}

}  // namespace

cap_status quantise_fp8_launch(cap_dtype dtype, int batch, int rows, int cols, int block_rows, const void* x, void* q,
                               float* scale, hipStream_t st) {
    if (dtype == CAP_DTYPE_BF16) launch<uint16_t>(batch, rows, cols, block_rows, x, q, scale, st);
    else launch<float>(batch, rows, cols, block_rows, x, q, scale, st);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
