// Load-balance loss of a batch's routing with per-sequence expert counts, and the
// gradient of the router logits (the router's training; Eq. 1 gates).
//
// With P_te = exp(l_te - lse_t), n_s the valid tokens of sequence s, S_a the
// sequences that have one, N their sum, c_se the kept slots of s at expert e and
// p_se = (1 / n_s) sum_t P_te:
//   balance = 1 / S_a  sum_s E / (k n_s) sum_e c_se p_se
//   z       = 1 / N    sum_t lse_t^2
//   d l_te  = P_te (C_se - sum_f P_tf C_sf) + P_te 2 z_coef lse_t / N
//             + w_ts (dw_ts - sum_kept w dw) at the expert of each kept slot s,
//   C_se    = balance_coef E c_se / (k n_s^2 S_a).
//
// A row of at most 256 logits is held by 16 lanes (16 values each at most), so a
// wave works on four tokens and every reduction over a row is four DPP steps.
// One pass over the logits in either direction; probabilities are never stored.
// Both are bound by the logits' way from HBM and, for small batches, by launches.
//
// The forward sums over tokens in a fixed order: a wave owns `per_wave`
// consecutive tokens, walks the sequences they belong to and leaves one partial
// row (a "piece") per sequence.  Piece (wave v, sequence s) has slot v + s: along
// the tokens v and s only grow and one of them does at every piece, so slots are
// distinct and there are at most waves + sequences of them, however the batch is
// cut.  A block whose tokens all belong to one sequence joins its waves' rows in
// LDS and leaves one piece.  The second kernel sums a sequence's pieces; the last
// of its blocks sums the losses over the sequences.
#include "cap_device.hpp"

#include <type_traits>

namespace cap {
namespace {

constexpr int kRowLanes = 16;                        // lanes that hold one token's row
constexpr int kTokPerStep = kWave / kRowLanes;       // tokens of a wave at a time
constexpr int kLossWaves = 4;                        // waves per block, both directions
constexpr int kLossThreads = kLossWaves * kWave;
constexpr int kSumThreads = 1024;
constexpr int kSumWaves = kSumThreads / kWave;

// All-reduce over the 16 lanes of a row (rotations within the row: every lane
// adds the same pairs, so all lanes hold the same bits).
template <int N>
__device__ __forceinline__ float row_ror(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x120 + N, 0xF, 0xF, false));
}
__device__ __forceinline__ float row_sum(float x) {
    x += row_ror<8>(x);
    x += row_ror<4>(x);
    x += row_ror<2>(x);
    x += row_ror<1>(x);
    return x;
}
__device__ __forceinline__ float row_max(float x) {
    x = fmaxf(x, row_ror<8>(x));
    x = fmaxf(x, row_ror<4>(x));
    x = fmaxf(x, row_ror<2>(x));
    x = fmaxf(x, row_ror<1>(x));
    return x;
}

// Lane j of a row holds columns 64 c + 4 j .. + 3, c < NV.  VEC: rows are 16-byte
// aligned and E is a multiple of 4.  Columns past E are -inf.
template <int NV, bool VEC>
__device__ __forceinline__ void load_row(const float* __restrict__ row, int E, int j, float (&v)[NV][4]) {
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int col = 64 * c + 4 * j;
        if constexpr (VEC) {
            f32x4 q = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
            if (col < E) q = *reinterpret_cast<const f32x4*>(row + col);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] = q[i];
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[c][i] = col + i < E ? row[col + i] : -INFINITY;
        }
    }
}

// v -> exp(v - max); returns the row's maximum and sum.
template <int NV>
__device__ __forceinline__ void row_exp(float (&v)[NV][4], float& top, float& total) {
    float m = -INFINITY;
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = fmaxf(m, v[c][i]);
    m = row_max(m);
    float s = 0.0f;
#pragma unroll
    for (int c = 0; c < NV; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[c][i] = __expf(v[c][i] - m);
            s += v[c][i];
        }
    top = m;
    total = row_sum(s);
}

// Sequence of token t among sequences lo .. hi (it is known to be one of them):
// the last whose offset is <= t, so an empty sequence never has a token.
__device__ __forceinline__ int find_sequence(const int32_t* __restrict__ offs, int t, int lo, int hi) {
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (offs[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// Sequences of tokens t0 and t1 (-1: before the first offset, S: at or past the
// last), found by the whole block: the offsets <= t are counted.  Ends in a barrier.
__device__ __forceinline__ void block_sequences(const int32_t* __restrict__ offs, int S, int t0, int t1, int* shared2,
                                                int& s0, int& s1) {
    if (!offs) {
        s0 = s1 = 0;
        return;
    }
    if (threadIdx.x < 2) shared2[threadIdx.x] = 0;
    __syncthreads();
    int n0 = 0, n1 = 0;
    for (int i = threadIdx.x; i <= S; i += blockDim.x) {
        const int o = offs[i];
        n0 += o <= t0;
        n1 += o <= t1;
    }
    if (n0) atomicAdd(&shared2[0], n0);
    if (n1) atomicAdd(&shared2[1], n1);
    __syncthreads();
    s0 = __builtin_amdgcn_readfirstlane(shared2[0]) - 1;
    s1 = max(s0, __builtin_amdgcn_readfirstlane(shared2[1]) - 1);
}

// LDS accesses of one wave stay in order; this keeps the compiler's order too.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

struct LossWs {
    float* psum;        // [pieces][EP] sums of probabilities
    int32_t* csum;      // [pieces][EP] kept slots
    int32_t* nsum;      // [pieces] valid tokens
    float* zsum;        // [pieces] sums of lse^2
    float* seq;         // [2][S] balance and z sums of each sequence
    int32_t* done;      // finished blocks of the second kernel
    int pieces, EP;
};

int loss_tokens_per_wave(int T) {
    // Four tokens at a time; a batch that fills the chip several times over takes
    // 16 a wave, so that a partial row is left for 64 tokens.
    return T >= 16384 ? 16 : T >= 4096 ? 8 : 4;
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

size_t loss_ws_layout(int T, int E, int S, void* base, LossWs* w) {
    const int per_wave = loss_tokens_per_wave(T);
    const int blocks = T > 0 ? (T - 1) / (per_wave * kLossWaves) + 1 : 0;
    const size_t pieces = static_cast<size_t>(blocks) * kLossWaves + S;
    const size_t EP = (E + 3) & ~3;
    size_t at = 0;
    char* p = static_cast<char*>(base);
    auto take = [&](size_t bytes) {
        char* q = p + at;
        at += up256(bytes);
        return q;
    };
    char* a = take(pieces * EP * 4);
    char* b = take(pieces * EP * 4);
    char* c = take(pieces * 4);
    char* d = take(pieces * 4);
    char* e = take(static_cast<size_t>(S) * 8);
    char* f = take(4);
    if (w) {
        w->psum = reinterpret_cast<float*>(a);
        w->csum = reinterpret_cast<int32_t*>(b);
        w->nsum = reinterpret_cast<int32_t*>(c);
        w->zsum = reinterpret_cast<float*>(d);
        w->seq = reinterpret_cast<float*>(e);
        w->done = reinterpret_cast<int32_t*>(f);
        w->pieces = static_cast<int>(pieces);
        w->EP = static_cast<int>(EP);
    }
    return at;
}

template <int NV, bool VEC>
__global__ __launch_bounds__(kLossThreads) void loss_pieces_kernel(
    int T, int k, int E, const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const uint8_t* __restrict__ keep, const uint8_t* __restrict__ mask, const int32_t* __restrict__ offs, int S,
    int per_wave, LossWs ws) {
    __shared__ int hist[kLossWaves][kMaxE];
    __shared__ float part[kLossWaves][kMaxE];
    __shared__ int part_n[kLossWaves];
    __shared__ float part_z[kLossWaves];
    __shared__ int found[2];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int g = lane / kRowLanes, j = lane % kRowLanes;
    if (blockIdx.x == 0 && threadIdx.x == 0) *ws.done = 0;
    const int block_t0 = blockIdx.x * per_wave * kLossWaves;
    const int block_t1 = min(T, block_t0 + per_wave * kLossWaves);
    int s0, s1;
    block_sequences(offs, S, block_t0, block_t1 - 1, found, s0, s1);
    for (int i = lane; i < kMaxE; i += kWave) hist[wave][i] = 0;
    wave_fence();

    const int wave_id = blockIdx.x * kLossWaves + wave;
    const int a = min(block_t1, block_t0 + wave * per_wave), b = min(block_t1, a + per_wave);
    float sum[NV][4];
    float zsum = 0.0f;
    int n = 0;

    auto tokens = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[c][i] = 0.0f;
        zsum = 0.0f;
        n = 0;
        for (int t4 = from; t4 < to; t4 += kTokPerStep) {
            const int t = t4 + g;
            const bool in = t < to;
            const size_t tc = in ? t : to - 1;
            float v[NV][4];
            load_row<NV, VEC>(logits + tc * E, E, j, v);
            int e = -1;
            if (in && j < k) {
                e = idx[tc * k + j];
                if (keep && !keep[tc * k + j]) e = -1;
            }
            float top, total;
            row_exp<NV>(v, top, total);
            const bool valid = in && !(top == -INFINITY) && (!mask || mask[tc] != 0);
            if (valid) {
                const float inv = 1.0f / total;
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[c][i] = __builtin_fmaf(v[c][i], inv, sum[c][i]);
                const float lse = top + logf(total);
                zsum = __builtin_fmaf(lse, lse, zsum);
                n += 1;
                if (static_cast<unsigned>(e) < static_cast<unsigned>(E)) atomicAdd(&hist[wave][e], 1);
            }
        }
        // over the wave's four rows
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                sum[c][i] += __shfl_xor(sum[c][i], 16);
                sum[c][i] += __shfl_xor(sum[c][i], 32);
            }
        zsum += __shfl_xor(zsum, 16);
        zsum += __shfl_xor(zsum, 32);
        n += __shfl_xor(n, 16);
        n += __shfl_xor(n, 32);
        wave_fence();
    };

    if (s0 == s1) {                                  // block-uniform: one piece
        if (s0 < 0 || s0 >= S) return;
        tokens(a, b);
        if (g == 0) {
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int i = 0; i < 4; ++i) part[wave][64 * c + 4 * j + i] = sum[c][i];
        }
        if (lane == 0) {
            part_n[wave] = n;
            part_z[wave] = zsum;
        }
        __syncthreads();
        const size_t slot = static_cast<size_t>(blockIdx.x) * kLossWaves + s0;
        const int e = threadIdx.x;
        if (e < ws.EP) {
            float p = 0.0f;
            int c = 0;
#pragma unroll
            for (int w = 0; w < kLossWaves; ++w) {
                p += part[w][e];
                c += hist[w][e];
            }
            ws.psum[slot * ws.EP + e] = p;
            ws.csum[slot * ws.EP + e] = c;
        }
        if (e == 0) {
            int m = 0;
            float z = 0.0f;
            for (int w = 0; w < kLossWaves; ++w) {
                m += part_n[w];
                z += part_z[w];
            }
            ws.nsum[slot] = m;
            ws.zsum[slot] = z;
        }
        return;
    }
    int at = a;
    int s = s0;
    while (at < b) {                                 // the wave's sequences
        s = s < 0 && at < offs[0] ? -1 : find_sequence(offs, at, max(s, 0), min(s1, S));
        const int end = s >= S ? b : min(b, max(at + 1, offs[s + 1]));
        if (s >= 0 && s < S) {
            tokens(at, end);
            const size_t slot = static_cast<size_t>(wave_id) + s;
            if (g == 0) {
#pragma unroll
                for (int c = 0; c < NV; ++c) {
                    const int col = 64 * c + 4 * j;
                    if (col < ws.EP)
                        *reinterpret_cast<f32x4*>(ws.psum + slot * ws.EP + col) =
                            f32x4{sum[c][0], sum[c][1], sum[c][2], sum[c][3]};
                }
            }
            for (int e = lane; e < ws.EP; e += kWave) {
                ws.csum[slot * ws.EP + e] = hist[wave][e];
                hist[wave][e] = 0;
            }
            wave_fence();
            if (lane == 0) {
                ws.nsum[slot] = n;
                ws.zsum[slot] = zsum;
            }
        }
        at = end;
    }
}

// Sum of v over the block's 1024 threads, in a fixed order; every thread gets it.
__device__ __forceinline__ float block_sum(float v, float* shared) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if (threadIdx.x % kWave == 0) shared[threadIdx.x / kWave] = v;
    __syncthreads();
    float r = 0.0f;
#pragma unroll
    for (int w = 0; w < kSumWaves; ++w) r += shared[w];
    return r;
}

// One block per sequence: wave w sums the pieces of token blocks w, w + 16, ..;
// lane l holds columns 4 l .. + 3.
__global__ __launch_bounds__(kSumThreads) void loss_sum_kernel(
    int T, int k, int E, const int32_t* __restrict__ offs, int S, int per_wave, float balance_coef, float z_coef,
    int32_t* __restrict__ counts, float* __restrict__ probs, int32_t* __restrict__ tokens, float* __restrict__ loss,
    LossWs ws) {
    __shared__ float psum[kSumWaves][kMaxE];
    __shared__ int csum[kSumWaves][kMaxE];
    __shared__ int nsum[kSumWaves];
    __shared__ float zsum[kSumWaves];
    __shared__ float red[kSumWaves];
    __shared__ int last;
    const int s = blockIdx.x;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int per_block = per_wave * kLossWaves;
    const int a = offs ? max(0, min(offs[s], T)) : 0;
    const int b = offs ? max(a, min(offs[s + 1], T)) : T;

    f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
    int c[4] = {0, 0, 0, 0};
    int n = 0;
    float z = 0.0f;
    auto add = [&](size_t slot) __attribute__((always_inline)) {
        if (4 * lane < ws.EP) {
            p += *reinterpret_cast<const f32x4*>(ws.psum + slot * ws.EP + 4 * lane);
            const u32x4 q = *reinterpret_cast<const u32x4*>(ws.csum + slot * ws.EP + 4 * lane);
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] += static_cast<int>(q[i]);
        }
        n += ws.nsum[slot];
        z += ws.zsum[slot];
    };
    if (a < b) {
        const int b0 = a / per_block, b1 = (b - 1) / per_block;
        // token blocks that lie in the sequence whole left one piece
        const int m0 = a == b0 * per_block ? b0 : b0 + 1;
        const int m1 = b == min(T, (b1 + 1) * per_block) ? b1 : b1 - 1;
#pragma unroll 4
        for (int i = m0 + wave; i <= m1; i += kSumWaves) add(static_cast<size_t>(i) * kLossWaves + s);
        // the waves of the others that have tokens of the sequence
        auto edge = [&](int block) {
            const int w0 = max(a / per_wave, block * kLossWaves);
            const int w1 = min((b - 1) / per_wave, block * kLossWaves + kLossWaves - 1);
            for (int v = w0; v <= w1; ++v) add(static_cast<size_t>(v) + s);
        };
        if (wave == 0 && m0 > b0) edge(b0);
        if (wave == 1 && m1 < b1 && (b1 > b0 || m0 == b0)) edge(b1);
    }
    *reinterpret_cast<f32x4*>(&psum[wave][4 * lane]) = p;
#pragma unroll
    for (int i = 0; i < 4; ++i) csum[wave][4 * lane + i] = c[i];
    if (lane == 0) {
        nsum[wave] = n;
        zsum[wave] = z;
    }
    __syncthreads();
    int nt = 0;
    float zt = 0.0f;
#pragma unroll
    for (int w = 0; w < kSumWaves; ++w) {
        nt += nsum[w];
        zt += zsum[w];
    }
    const float inv_n = nt > 0 ? 1.0f / static_cast<float>(nt) : 0.0f;
    float term = 0.0f;
    const int e = threadIdx.x;
    if (e < E) {
        float ps = 0.0f;
        int cs = 0;
#pragma unroll
        for (int w = 0; w < kSumWaves; ++w) {
            ps += psum[w][e];
            cs += csum[w][e];
        }
        ps = nt > 0 ? ps / static_cast<float>(nt) : 0.0f;
        const size_t at = static_cast<size_t>(s) * E + e;
        probs[at] = ps;
        counts[at] = cs;
        term = static_cast<float>(cs) * ps;
    }
    const float dot = block_sum(term, red);
    if (threadIdx.x == 0) {
        const float scale = static_cast<float>(E) / static_cast<float>(k) * inv_n;
        __hip_atomic_store(&ws.seq[s], dot * scale, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&ws.seq[S + s], zt, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __hip_atomic_store(&tokens[s], nt, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = __hip_atomic_fetch_add(ws.done, 1, __ATOMIC_ACQ_REL, __HIP_MEMORY_SCOPE_AGENT) == S - 1;
    }
    __syncthreads();
    if (!last) return;
    // the last block: sums over the sequences
    float bal = 0.0f, zz = 0.0f;
    int present = 0, total = 0;
    for (int i = threadIdx.x; i < S; i += kSumThreads) {
        bal += __hip_atomic_load(&ws.seq[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        zz += __hip_atomic_load(&ws.seq[S + i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        const int m = __hip_atomic_load(&tokens[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        present += m > 0;
        total += m;
    }
    bal = block_sum(bal, red);
    zz = block_sum(zz, red);
    // token totals as whole numbers
    __shared__ int ints[2];
    if (threadIdx.x < 2) ints[threadIdx.x] = 0;
    __syncthreads();
    if (present) atomicAdd(&ints[0], present);
    if (total) atomicAdd(&ints[1], total);
    __syncthreads();
    if (threadIdx.x == 0) {
        present = ints[0];
        total = ints[1];
        tokens[S] = present;
        tokens[S + 1] = total;
        bal = present > 0 ? bal / static_cast<float>(present) : 0.0f;
        zz = total > 0 ? zz / static_cast<float>(total) : 0.0f;
        // a loss that is switched off adds nothing, not 0 * inf (rows at the lowest value have an infinite lse^2)
        loss[0] = (balance_coef != 0.0f ? balance_coef * bal : 0.0f) + (z_coef != 0.0f ? z_coef * zz : 0.0f);
        loss[1] = bal;
        loss[2] = zz;
    }
}

// Gradient of the logits: each wave four tokens at a time, `steps` times.  The
// gates' part goes from the slots' lanes to the columns' lanes through a row of LDS.
template <int NV, bool VEC, bool BF16>
__global__ __launch_bounds__(kLossThreads) void router_grad_kernel(
    int T, int k, int E, const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const uint8_t* __restrict__ keep, const float* __restrict__ w, const float* __restrict__ d_w,
    const uint8_t* __restrict__ mask, const int32_t* __restrict__ offs, int S, const int32_t* __restrict__ counts,
    const int32_t* __restrict__ tokens, float balance_coef, float z_coef, const float* __restrict__ d_loss, int steps,
    void* __restrict__ out) {
    __shared__ __attribute__((aligned(16))) float gates[kLossThreads / kRowLanes][64 * NV];
    __shared__ int found[2];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int row = threadIdx.x / kRowLanes, g = lane / kRowLanes, j = lane % kRowLanes;
    const int per_block = kLossWaves * kTokPerStep * steps;
    const int block_t0 = blockIdx.x * per_block;
    int s0, s1;
    block_sequences(offs, S, block_t0, min(T, block_t0 + per_block) - 1, found, s0, s1);
#pragma unroll
    for (int c = 0; c < NV; ++c)
        *reinterpret_cast<f32x4*>(&gates[row][64 * c + 4 * j]) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    wave_fence();
    const float up = d_loss ? *d_loss : 1.0f;
    const int present = tokens[S], total_tokens = tokens[S + 1];
    const float bal = present > 0 ? up * balance_coef * static_cast<float>(E) / static_cast<float>(k) /
                                        static_cast<float>(present)
                                  : 0.0f;
    const float zed = total_tokens > 0 ? up * 2.0f * z_coef / static_cast<float>(total_tokens) : 0.0f;

    for (int i = 0; i < steps; ++i) {
        const int t = block_t0 + (i * kLossWaves + wave) * kTokPerStep + g;
        if (t >= T) continue;                            // whole 16-lane rows
        const size_t tt = t;
        float v[NV][4];
        load_row<NV, VEC>(logits + tt * E, E, j, v);
        int e = -1;
        float ws = 0.0f, dw = 0.0f;
        if (d_w && j < k) {
            e = idx[tt * k + j];
            if ((keep && !keep[tt * k + j]) || static_cast<unsigned>(e) >= static_cast<unsigned>(E)) e = -1;
            if (e >= 0) {
                ws = w[tt * k + j];
                dw = d_w[tt * k + j];
            }
        }
        const int s = s0 == s1 ? s0 : (offs[0] > t ? -1 : find_sequence(offs, t, max(s0, 0), min(s1, S)));
        const bool inside = s >= 0 && s < S;
        float top, total;
        row_exp<NV>(v, top, total);
        const bool valid = inside && !(top == -INFINITY) && (!mask || mask[t] != 0);
        const float inv = 1.0f / total;
        const float lse = top + logf(total);
        const int ns = inside ? tokens[s] : 0;
        const float cs = ns > 0 ? bal / static_cast<float>(ns) / static_cast<float>(ns) : 0.0f;
        float cc[NV][4];
        float dot = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = 64 * c + 4 * j;
            if constexpr (VEC) {
                u32x4 q = {0, 0, 0, 0};
                if (inside && col < E) q = *reinterpret_cast<const u32x4*>(counts + static_cast<size_t>(s) * E + col);
#pragma unroll
                for (int x = 0; x < 4; ++x) cc[c][x] = cs * static_cast<float>(static_cast<int>(q[x]));
            } else {
#pragma unroll
                for (int x = 0; x < 4; ++x)
                    cc[c][x] = inside && col + x < E
                                   ? cs * static_cast<float>(counts[static_cast<size_t>(s) * E + col + x])
                                   : 0.0f;
            }
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                v[c][x] *= inv;
                dot = __builtin_fmaf(v[c][x], cc[c][x], dot);
            }
        }
        const float shift = lse * zed - row_sum(dot);
        float gate[NV][4];
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int x = 0; x < 4; ++x) gate[c][x] = 0.0f;
        if (d_w) {
            const float mean = row_sum(ws * dw);
            if (e >= 0) atomicAdd(&gates[row][e], ws * (dw - mean));
            wave_fence();
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const f32x4 q = *reinterpret_cast<const f32x4*>(&gates[row][64 * c + 4 * j]);
#pragma unroll
                for (int x = 0; x < 4; ++x) gate[c][x] = q[x];
            }
            wave_fence();
            if (e >= 0) gates[row][e] = 0.0f;
            wave_fence();
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int col = 64 * c + 4 * j;
            float d[4];
#pragma unroll
            for (int x = 0; x < 4; ++x)
                d[x] = valid ? __builtin_fmaf(v[c][x], cc[c][x] + shift, gate[c][x]) : 0.0f;
            if constexpr (VEC) {
                if (col >= E) continue;
                if constexpr (BF16)
                    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(out) + tt * E + col) =
                        u32x2{pack_bf16x2_rne(d[0], d[1]), pack_bf16x2_rne(d[2], d[3])};
                else
                    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + tt * E + col) = f32x4{d[0], d[1], d[2], d[3]};
            } else {
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    if (col + x >= E) continue;
                    if constexpr (BF16)
                        static_cast<uint16_t*>(out)[tt * E + col + x] =
                            static_cast<uint16_t>(pack_bf16x2_rne(d[x], 0.0f));
                    else
                        static_cast<float*>(out)[tt * E + col + x] = d[x];
                }
            }
        }
    }
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

}  // namespace

size_t balance_workspace_bytes(int T, int E, int S) { return loss_ws_layout(T, E, S, nullptr, nullptr); }

cap_status balance_loss_launch(int T, int k, int E, const float* logits, const int32_t* idx, const uint8_t* keep,
                               const uint8_t* mask, const int32_t* offs, int S, float balance_coef, float z_coef,
                               int32_t* counts, float* probs, int32_t* tokens, float* loss, void* workspace,
                               hipStream_t stream) {
    LossWs ws;
    loss_ws_layout(T, E, S, workspace, &ws);
    const int per_wave = loss_tokens_per_wave(T);
    const int blocks = T > 0 ? (T - 1) / (per_wave * kLossWaves) + 1 : 1;
    const bool vec = E % 4 == 0 && aligned(logits, 16);
    auto launch = [&](auto NV) {
        constexpr int nv = decltype(NV)::value;
        if (vec)
            loss_pieces_kernel<nv, true><<<blocks, kLossThreads, 0, stream>>>(T, k, E, logits, idx, keep, mask, offs, S,
                                                                             per_wave, ws);
        else
            loss_pieces_kernel<nv, false><<<blocks, kLossThreads, 0, stream>>>(T, k, E, logits, idx, keep, mask, offs,
                                                                              S, per_wave, ws);
    };
    if (E <= 64) launch(std::integral_constant<int, 1>{});
    else if (E <= 128) launch(std::integral_constant<int, 2>{});
    else launch(std::integral_constant<int, 4>{});
    CAP_LAUNCH_CHECK();
    loss_sum_kernel<<<S, kSumThreads, 0, stream>>>(T, k, E, offs, S, per_wave, balance_coef, z_coef, counts, probs,
                                                   tokens, loss, ws);
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

cap_status router_grad_launch(int T, int k, int E, const float* logits, const int32_t* idx, const uint8_t* keep,
                              const float* w, const float* d_w, const uint8_t* mask, const int32_t* offs, int S,
                              const int32_t* counts, const int32_t* tokens, float balance_coef, float z_coef,
                              const float* d_loss, cap_dtype dtype, void* d_logits, hipStream_t stream) {
    const int steps = T >= 16384 ? 2 : 1;
    const int per_block = kLossWaves * kTokPerStep * steps;
    const int blocks = (T - 1) / per_block + 1;
    const bool bf16 = dtype == CAP_DTYPE_BF16;
    const bool vec = E % 4 == 0 && aligned(logits, 16) && aligned(counts, 16) && aligned(d_logits, bf16 ? 8 : 16);
    auto launch = [&](auto NV, auto VEC, auto BF) {
        router_grad_kernel<decltype(NV)::value, decltype(VEC)::value, decltype(BF)::value>
            <<<blocks, kLossThreads, 0, stream>>>(T, k, E, logits, idx, keep, w, d_w, mask, offs, S, counts, tokens,
                                                  balance_coef, z_coef, d_loss, steps, d_logits);
    };
    auto by_type = [&](auto NV) {
        if (vec && bf16) launch(NV, std::true_type{}, std::true_type{});
        else if (vec) launch(NV, std::true_type{}, std::false_type{});
        else if (bf16) launch(NV, std::false_type{}, std::true_type{});
        else launch(NV, std::false_type{}, std::false_type{});
    };
    if (E <= 64) by_type(std::integral_constant<int, 1>{});
    else if (E <= 128) by_type(std::integral_constant<int, 2>{});
    else by_type(std::integral_constant<int, 4>{});
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

}  // namespace cap
