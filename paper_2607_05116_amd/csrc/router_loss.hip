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
// LDS and leaves one piece.  A second kernel sums each sequence's pieces and a third the
// losses over the sequences; a small batch is one workgroup's in one launch.
//
// 32768 tokens, 256 experts, top 8, 8 sequences: the pieces 11.3 us for 35 MB (3.1 TB/s; the
// exponentials are not why, since the gradient takes them too; most likely the loads' latency,
// with two waves a SIMD and one step's rows on their way in each), their sums 5.4 and the losses 2.6 us;
// the gradient in fp32 15.1 us for 37 MB read and 34 MB written (4.7 TB/s).  8192 tokens, 64
// experts, 211 sequences: 5.9 + 5.7 + 2.5 and 4.8 us; 61 tokens: 4.1 and 3.5 us, a launch.
#include "cap_device.hpp"

#include <type_traits>

namespace cap {
namespace {

constexpr int kRowLanes = 16;                        // lanes that hold one token's row
constexpr int kTokPerStep = kWave / kRowLanes;       // tokens of a wave at a time
constexpr int kLossWaves = 8;                        // waves of a block of the loss, of the gradient
constexpr int kLossThreads = kLossWaves * kWave;
constexpr int kGradWaves = 4;
constexpr int kGradThreads = kGradWaves * kWave;
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

// The sequences that a block's tokens belong to: -1 before the first offset, S at or past
// the last.  Found by the whole block: the offsets <= a token are counted, in windows of
// one offset a thread; with more offsets than threads (T / 32 blocks that all counted all
// of them took 20 ms for 2^20 sequences) a window of samples first, and then the
// window between two of them.  The offsets from the first one's on are kept in LDS, so that
// a token's sequence is found there and not by a chain of loads.
constexpr int kSeqCache = 64;
struct Sequences {
    const int32_t* offs;
    const int32_t* cache;
    int S, first, last;

    __device__ __forceinline__ int offset(int i) const {
        const int c = i - first;
        return c < kSeqCache ? cache[max(c, 0)] : offs[i];
    }
    // sequence of token t, one of lo .. last: the last whose offset is <= t, so an empty
    // sequence never has a token
    __device__ __forceinline__ int of(int t, int lo) const {
        if (first == last) return first;
        lo = max(lo, first);
        if (lo < 0) {
            if (t < offs[0]) return -1;
            lo = 0;
        }
        int hi = min(last, S);
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (offset(mid) <= t) lo = mid; else hi = mid - 1;
        }
        return lo;
    }
};
struct SequencesLds {
    int found[2][2][16];                             // in turn; of two tokens, by wave
    int32_t cache[kSeqCache];
};
// A barrier for LDS alone: __syncthreads would wait for the rows on their way too.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Distance of a window's samples: 1 if every offset of it has a thread.
template <int THREADS>
__device__ __forceinline__ int sample_step(int size) { return max(1, (size + THREADS - 1) / THREADS); }

// This thread's first sample, to be asked for before the rows (loads return in order).
template <int THREADS>
__device__ __forceinline__ int first_offset(const int32_t* __restrict__ offs, int S) {
    const int at = (static_cast<int>(threadIdx.x) + 1) * sample_step<THREADS>(S + 1) - 1;
    return offs && at <= S ? offs[at] : INT32_MAX;
}

// Of tokens t0 and t1 and those between them.  Ends in a barrier.
template <int THREADS>
__device__ __forceinline__ Sequences block_sequences(const int32_t* __restrict__ offs, int S, int t0, int t1, int mine,
                                                     SequencesLds& lds) {
    Sequences q{offs, lds.cache, S, 0, 0};
    if (!offs) return q;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    // offsets below n0 are <= t0, those from end0 on are past it; n1, end1 of t1
    int n0 = 0, n1 = 0, end0 = S + 1, end1 = S + 1;
    for (int level = 0; n0 < end0 || n1 < end1; ++level) {
        const int step0 = sample_step<THREADS>(end0 - n0), step1 = sample_step<THREADS>(end1 - n1);
        const int at0 = n0 + (static_cast<int>(threadIdx.x) + 1) * step0 - 1, at1 = n1 + (static_cast<int>(threadIdx.x) + 1) * step1 - 1;
        const int o0 = at0 >= end0 ? INT32_MAX : level == 0 ? mine : offs[at0];
        const int o1 = at1 >= end1 ? INT32_MAX : level == 0 ? mine : offs[at1];
        // counted by ballots (LDS atomics on one word took 5 us for 211 sequences)
        const int c0 = __popcll(__ballot(at0 < end0 && o0 <= t0)), c1 = __popcll(__ballot(at1 < end1 && o1 <= t1));
        if (lane == 0) {
            lds.found[level & 1][0][wave] = c0;
            lds.found[level & 1][1][wave] = c1;
        }
        lds_barrier();
        int s0 = 0, s1 = 0;
#pragma unroll
        for (int w = 0; w < THREADS / kWave; ++w) {
            s0 += lds.found[level & 1][0][w];
            s1 += lds.found[level & 1][1][w];
        }
        s0 = __builtin_amdgcn_readfirstlane(s0);
        s1 = __builtin_amdgcn_readfirstlane(s1);
        n0 += s0 * step0;                            // s0 samples are <= t0, the next (or the end) is not
        n1 += s1 * step1;
        end0 = min(end0, n0 + step0 - 1);
        end1 = min(end1, n1 + step1 - 1);
    }
    q.first = __builtin_amdgcn_readfirstlane(n0) - 1;
    q.last = max(q.first, __builtin_amdgcn_readfirstlane(n1) - 1);
    if (q.first != q.last) {
        for (int i = threadIdx.x; i < kSeqCache; i += THREADS) lds.cache[i] = offs[min(max(q.first + i, 0), S)];
        lds_barrier();
    }
    return q;
}

// LDS accesses of one wave stay in order; this keeps the compiler's order too.
__device__ __forceinline__ void wave_fence() { __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront"); }

struct LossWs {
    float* psum;        // [pieces][EP] sums of probabilities
    int32_t* csum;      // [pieces][EP] kept slots
    int32_t* nsum;      // [pieces] valid tokens
    float* zsum;        // [pieces] sums of lse^2
    float* seq;         // [S][4] balance sums of each quarter of the experts, [S] z sums
    int EP;
};

// How a batch is cut: `per_wave` tokens a wave, `waves` waves a block.
struct LossPlan {
    int waves, per_wave, blocks;
    bool one_launch;
};
LossPlan loss_plan(int T, int S) {
    LossPlan p;
    // One workgroup and one launch while its waves take no more than 16 tokens each (61
    // tokens 5.9 us against 8.9 in three launches, 200 tokens 6.2 against 9.9) and no more
    // than one sequence at the end (60 tokens in 5 sequences 8.8 against 10.7, but in 30
    // 16.7 against 14.9).
    p.one_launch = S == 1 ? T <= 256 : T <= 64 && S <= kSumWaves;
    // Four tokens at a time; a batch that fills the chip several times over takes 16 a
    // wave, so that a piece is left for 128 tokens (32768 tokens of 256 experts 20 us
    // against 25 with four a wave; 8192 of 64 experts 16.5 against 13.8).
    p.waves = p.one_launch ? 16 : kLossWaves;
    // Past 2^29 tokens 64, for a launch of less than 2^32 threads.
    p.per_wave = p.one_launch ? (T <= 64 ? 4 : 16) : T > 1 << 29 ? 64 : T >= 16384 ? 16 : 4;
    p.blocks = T > 0 ? (T - 1) / (p.per_wave * p.waves) + 1 : 1;
    return p;
}

size_t up256(size_t v) { return (v + 255) & ~size_t(255); }

size_t loss_ws_layout(int T, int E, int S, void* base, LossWs* w) {
    const LossPlan plan = loss_plan(T, S);
    const size_t pieces = static_cast<size_t>(plan.blocks) * plan.waves + S;
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
    char* e = take(static_cast<size_t>(S) * 20);
    if (w) {
        w->psum = reinterpret_cast<float*>(a);
        w->csum = reinterpret_cast<int32_t*>(b);
        w->nsum = reinterpret_cast<int32_t*>(c);
        w->zsum = reinterpret_cast<float*>(d);
        w->seq = reinterpret_cast<float*>(e);
        w->EP = static_cast<int>(EP);
    }
    return at;
}

struct LossArgs {
    int T, k, E, S, per_wave;
    const float* logits;
    const int32_t* idx;
    const uint8_t *keep, *mask;
    const int32_t* offs;
    float balance_coef, z_coef;
    int32_t* counts;
    float* probs;
    int32_t* tokens;
    float* loss;
    LossWs ws;
};

// add(slot) for the pieces of sequence s (tokens a .. b - 1) that worker `me` of `of` takes.
// waves: of the blocks that left the pieces; 0: each piece is a wave's.
template <typename Add>
__device__ __forceinline__ void each_piece(const LossArgs& q, int waves, int s, int a, int b, int me, int of, Add&& add) {
    if (a >= b) return;
    if (waves == 0) {
        for (int v = a / q.per_wave + me; v <= (b - 1) / q.per_wave; v += of) add(static_cast<size_t>(v) + s);
        return;
    }
    const int per_block = q.per_wave * waves;
    const int b0 = a / per_block, b1 = (b - 1) / per_block;
    // token blocks that lie in the sequence whole left one piece
    const int m0 = a == b0 * per_block ? b0 : b0 + 1;
    const int m1 = b == min(q.T, (b1 + 1) * per_block) ? b1 : b1 - 1;
#pragma unroll 4
    for (int i = m0 + me; i <= m1; i += of) add(static_cast<size_t>(i) * waves + s);
    // the waves of the others that have tokens of the sequence
    auto edge = [&](int block) {
        const int w0 = max(a / q.per_wave, block * waves);
        const int w1 = min((b - 1) / q.per_wave, block * waves + waves - 1);
        for (int v = w0 + me; v <= w1; v += of) add(static_cast<size_t>(v) + s);
    };
    if (m0 > b0) edge(b0);
    if (m1 < b1 && (b1 > b0 || m0 == b0)) edge(b1);
}

__device__ __forceinline__ void sequence_range(const LossArgs& q, int s, int& a, int& b) {
    a = q.offs ? max(0, min(q.offs[s], q.T)) : 0;
    b = q.offs ? max(a, min(q.offs[s + 1], q.T)) : q.T;
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

// The losses from their sums over the sequences.
__device__ __forceinline__ void write_loss(const LossArgs& q, float bal, float zz, int present, int total) {
    q.tokens[q.S] = present;
    q.tokens[q.S + 1] = total;
    bal = present > 0 ? bal / static_cast<float>(present) : 0.0f;
    zz = total > 0 ? zz / static_cast<float>(total) : 0.0f;
    // a loss that is switched off adds nothing, not 0 * inf (rows at the lowest value have an infinite lse^2)
    q.loss[0] = (q.balance_coef != 0.0f ? q.balance_coef * bal : 0.0f) + (q.z_coef != 0.0f ? q.z_coef * zz : 0.0f);
    q.loss[1] = bal;
    q.loss[2] = zz;
}

// All sequences and the losses by one workgroup: a wave for every 16th sequence, lane l
// holds columns 4 l .. + 3.
__device__ __forceinline__ void sum_all(const LossArgs& q) {
    __shared__ float bal_w[kSumWaves], z_w[kSumWaves];
    __shared__ int present_w[kSumWaves], total_w[kSumWaves];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    float bal = 0.0f, zz = 0.0f;
    int present = 0, total = 0;
    for (int s = wave; s < q.S; s += kSumWaves) {
        int a, b;
        sequence_range(q, s, a, b);
        f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
        int c[4] = {0, 0, 0, 0};
        int n = 0;
        float z = 0.0f;
        each_piece(q, 0, s, a, b, 0, 1, [&](size_t slot) __attribute__((always_inline)) {
            if (4 * lane < q.ws.EP) {
                p += *reinterpret_cast<const f32x4*>(q.ws.psum + slot * q.ws.EP + 4 * lane);
                const u32x4 v = *reinterpret_cast<const u32x4*>(q.ws.csum + slot * q.ws.EP + 4 * lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) c[i] += static_cast<int>(v[i]);
            }
            n += q.ws.nsum[slot];
            z += q.ws.zsum[slot];
        });
        float term = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (4 * lane + i < q.E) {
                const float mean = n > 0 ? p[i] / static_cast<float>(n) : 0.0f;
                q.probs[static_cast<size_t>(s) * q.E + 4 * lane + i] = mean;
                q.counts[static_cast<size_t>(s) * q.E + 4 * lane + i] = c[i];
                term = __builtin_fmaf(static_cast<float>(c[i]), mean, term);
            }
        term = wave_sum(term);
        if (n > 0) bal += term * (static_cast<float>(q.E) / static_cast<float>(q.k) / static_cast<float>(n));
        zz += z;
        present += n > 0;
        total += n;
        if (lane == 0) q.tokens[s] = n;
    }
    if (lane == 0) {
        bal_w[wave] = bal;
        z_w[wave] = zz;
        present_w[wave] = present;
        total_w[wave] = total;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < kSumWaves; ++w) {
            bal += bal_w[w];
            zz += z_w[w];
            present += present_w[w];
            total += total_w[w];
        }
        write_loss(q, bal, zz, present, total);
    }
}

// WAVES == 16: the whole batch in one workgroup, which then sums its pieces too.
template <int NV, bool VEC, int WAVES>
__global__ __launch_bounds__(WAVES * kWave) void loss_pieces_kernel(LossArgs q) {
    constexpr bool ALL = WAVES == kSumWaves;
    __shared__ int hist[WAVES][64 * NV];
    __shared__ __attribute__((aligned(16))) float part[WAVES][64 * NV];
    __shared__ float term_w[WAVES];
    __shared__ int part_n[WAVES];
    __shared__ float part_z[WAVES];
    __shared__ SequencesLds found;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int g = lane / kRowLanes, j = lane % kRowLanes;
    const int T = q.T, k = q.k, E = q.E, S = q.S;
    const LossWs& ws = q.ws;
    const int block_t0 = blockIdx.x * q.per_wave * WAVES;
    const int block_t1 = min(T, block_t0 + q.per_wave * WAVES);
    for (int i = lane; i < 64 * NV; i += kWave) hist[wave][i] = 0;
    const int wave_id = blockIdx.x * WAVES + wave;
    const int a = min(block_t1, block_t0 + wave * q.per_wave), b = min(block_t1, a + q.per_wave);
    // four tokens: their logits, and the expert of lane j's slot (-1: none)
    struct Rows {
        float v[NV][4];
        int e;
        bool valid;
    };
    auto load = [&](Rows& x, int t4) __attribute__((always_inline)) {
        const int t = t4 + g;
        const size_t tc = min(t, b - 1);
        load_row<NV, VEC>(q.logits + tc * E, E, j, x.v);
        x.e = -1;
        if (j < k) {
            x.e = q.idx[tc * k + j];
            if (q.keep && !q.keep[tc * k + j]) x.e = -1;
        }
        x.valid = !q.mask || q.mask[tc] != 0;
    };
    // the first are on their way while the block finds its sequences
    const int mine = first_offset<WAVES * kWave>(q.offs, S);
    Rows next;
    if (a < b) load(next, a);
    const Sequences seq = block_sequences<WAVES * kWave>(q.offs, S, block_t0, block_t1 - 1, mine, found);
    wave_fence();
    float sum[NV][4];
    float zsum = 0.0f;
    int n = 0;

    auto over_rows = [&]() __attribute__((always_inline)) {
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
    auto tokens = [&](int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[c][i] = 0.0f;
        zsum = 0.0f;
        n = 0;
        if (from > a && from < to) load(next, from);
        for (int t4 = from; t4 < to; t4 += kTokPerStep) {
            Rows x = next;
            if (t4 + kTokPerStep < to) load(next, t4 + kTokPerStep);           // on their way during this step
            float top, total;
            row_exp<NV>(x.v, top, total);
            if (t4 + g < to && x.valid && !(top == -INFINITY)) {
                const float inv = 1.0f / total;
#pragma unroll
                for (int c = 0; c < NV; ++c)
#pragma unroll
                    for (int i = 0; i < 4; ++i) sum[c][i] = __builtin_fmaf(x.v[c][i], inv, sum[c][i]);
                const float lse = top + logf(total);
                zsum = __builtin_fmaf(lse, lse, zsum);
                n += 1;
                if (static_cast<unsigned>(x.e) < static_cast<unsigned>(E)) atomicAdd(&hist[wave][x.e], 1);
            }
        }
        over_rows();
    };
    // a wave of one step that holds several sequences: its rows once, then each sequence's
    // tokens among them
    auto step_once = [&](Rows& x, float& lse2) __attribute__((always_inline)) {
        float top, total;
        row_exp<NV>(x.v, top, total);
        x.valid = a + g < b && x.valid && !(top == -INFINITY);
        const float inv = 1.0f / total, lse = top + logf(total);
        lse2 = lse * lse;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) x.v[c][i] *= inv;
    };
    auto some = [&](const Rows& x, float lse2, int from, int to) __attribute__((always_inline)) {
        const bool mine = x.valid && a + g >= from && a + g < to;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[c][i] = mine ? x.v[c][i] : 0.0f;
        zsum = mine ? lse2 : 0.0f;
        n = mine;
        if (mine && static_cast<unsigned>(x.e) < static_cast<unsigned>(E)) atomicAdd(&hist[wave][x.e], 1);
        over_rows();
    };

    if (ALL ? S == 1 : seq.first == seq.last) {      // the block's tokens are of one sequence
        if (ALL) {
            // (of the sequence's own range: tokens may lie outside it)
            int lo = 0, hi = T;
            sequence_range(q, 0, lo, hi);
            tokens(max(a, lo), max(min(b, hi), max(a, lo)));
        } else {
            if (seq.first < 0 || seq.first >= S) return;
            tokens(a, b);
        }
        if (g == 0) {
#pragma unroll
            for (int c = 0; c < NV; ++c)
                *reinterpret_cast<f32x4*>(&part[wave][64 * c + 4 * j]) = f32x4{sum[c][0], sum[c][1], sum[c][2], sum[c][3]};
        }
        if (lane == 0) {
            part_n[wave] = n;
            part_z[wave] = zsum;
        }
        __syncthreads();
        const int e = threadIdx.x;
        float p = 0.0f, z = 0.0f;
        int c = 0, m = 0;
        if (e < 64 * NV) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                p += part[w][e];
                c += hist[w][e];
            }
        }
        if (ALL || e == 0) {
            for (int w = 0; w < WAVES; ++w) {
                m += part_n[w];
                z += part_z[w];
            }
        }
        if constexpr (!ALL) {                        // one piece
            const size_t slot = static_cast<size_t>(blockIdx.x) * WAVES + seq.first;
            if (e < ws.EP) {
                ws.psum[slot * ws.EP + e] = p;
                ws.csum[slot * ws.EP + e] = c;
            }
            if (e == 0) {
                ws.nsum[slot] = m;
                ws.zsum[slot] = z;
            }
        } else {                                     // the result
            float term = 0.0f;
            if (e < E) {
                p = m > 0 ? p / static_cast<float>(m) : 0.0f;
                q.probs[e] = p;
                q.counts[e] = c;
                term = static_cast<float>(c) * p;
            }
            term = wave_sum(term);
            if (lane == 0) term_w[wave] = term;
            __syncthreads();
            if (e == 0) {
                term = 0.0f;
                for (int w = 0; w < WAVES; ++w) term += term_w[w];
                q.tokens[0] = m;
                write_loss(q, m > 0 ? term * (static_cast<float>(E) / static_cast<float>(k) / static_cast<float>(m)) : 0.0f, z,
                           m > 0, m);
            }
        }
        return;
    }
    int at = a;
    int s = seq.first;
    const bool once = q.per_wave == kTokPerStep && seq.first != seq.last;
    float lse2 = 0.0f;
    if (once && a < b) step_once(next, lse2);
    while (at < b) {                                 // the wave's sequences
        s = seq.of(at, s);
        // (one sequence: its offsets are not kept)
        const int end = seq.first == seq.last || s >= S ? b : min(b, max(at + 1, seq.offset(s + 1)));
        if (s >= 0 && s < S) {
            if (once) some(next, lse2, at, end);
            else tokens(at, end);
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
    if constexpr (ALL) {
        __syncthreads();
        sum_all(q);
    }
}

// Sequences blockIdx.x, + gridDim.x, .., columns 64 blockIdx.y .. + 63: GROUPS groups of 16
// lanes share the pieces.  Latency: two loads after one another for every 4 x GROUPS pieces.
constexpr int kSumBlocks = 1 << 20;                  // at most, for a launch of less than 2^32 threads
template <int GROUPS>
__global__ __launch_bounds__(GROUPS * 16) void loss_sum_kernel(LossArgs q) {
    constexpr int WAVES = GROUPS / 4;
    __shared__ f32x4 psum[WAVES][16];
    __shared__ u32x4 csum[WAVES][16];
    __shared__ int nsum[WAVES];
    __shared__ float zsum[WAVES];
    const int quarter = blockIdx.y;
    const int group = threadIdx.x / 16, j = threadIdx.x % 16;
    const int col = 64 * quarter + 4 * j;
    for (int s = blockIdx.x; s < q.S; s += gridDim.x) {
        int a, b;
        sequence_range(q, s, a, b);
        f32x4 p = {0.0f, 0.0f, 0.0f, 0.0f};
        u32x4 c = {0, 0, 0, 0};
        int n = 0;
        float z = 0.0f;
        each_piece(q, kLossWaves, s, a, b, group, GROUPS, [&](size_t slot) __attribute__((always_inline)) {
            if (col < q.ws.EP) {
                p += *reinterpret_cast<const f32x4*>(q.ws.psum + slot * q.ws.EP + col);
                c += *reinterpret_cast<const u32x4*>(q.ws.csum + slot * q.ws.EP + col);
            }
            n += q.ws.nsum[slot];
            z += q.ws.zsum[slot];
        });
        // the four groups of a wave, then the waves through LDS
#pragma unroll
        for (int o = 16; o < kWave; o <<= 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] += __shfl_xor(p[i], o);
                c[i] += __shfl_xor(c[i], o);
            }
            n += __shfl_xor(n, o);
            z += __shfl_xor(z, o);
        }
        const int wave = threadIdx.x / kWave;
        if (threadIdx.x % kWave < 16) {
            psum[wave][j] = p;
            csum[wave][j] = c;
            if (j == 0) {
                nsum[wave] = n;
                zsum[wave] = z;
            }
        }
        __syncthreads();
        // thread e of the first wave: column 64 quarter + e
        float term = 0.0f;
        if (threadIdx.x < 64) {
            const int e = 64 * quarter + threadIdx.x;
            float ps = 0.0f, zt = 0.0f;
            int cs = 0, nt = 0;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                ps += psum[w][threadIdx.x / 4][threadIdx.x % 4];
                cs += static_cast<int>(csum[w][threadIdx.x / 4][threadIdx.x % 4]);
                nt += nsum[w];
                zt += zsum[w];
            }
            if (e < q.E) {
                ps = nt > 0 ? ps / static_cast<float>(nt) : 0.0f;
                q.probs[static_cast<size_t>(s) * q.E + e] = ps;
                q.counts[static_cast<size_t>(s) * q.E + e] = cs;
                term = static_cast<float>(cs) * ps;
            }
            term = wave_sum(term);
            if (threadIdx.x == 0) {
                q.ws.seq[4 * static_cast<size_t>(s) + quarter] =
                    nt > 0 ? term * (static_cast<float>(q.E) / static_cast<float>(q.k) / static_cast<float>(nt)) : 0.0f;
                if (quarter == 0) {
                    q.ws.seq[4 * static_cast<size_t>(q.S) + s] = zt;
                    q.tokens[s] = nt;
                }
            }
        }
        if (s + static_cast<int>(gridDim.x) < q.S) __syncthreads();          // the sums in LDS have been read
    }
}

// The losses: sums over the sequences.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void loss_final_kernel(LossArgs q, int quarters) {
    constexpr int WAVES = THREADS / kWave;
    __shared__ float bal_w[WAVES], z_w[WAVES];
    __shared__ int present_w[WAVES], total_w[WAVES];
    float bal = 0.0f, zz = 0.0f;
    int present = 0, total = 0;
#pragma unroll 4
    for (int s = threadIdx.x; s < q.S; s += THREADS) {
        for (int x = 0; x < quarters; ++x) bal += q.ws.seq[4 * static_cast<size_t>(s) + x];
        zz += q.ws.seq[4 * static_cast<size_t>(q.S) + s];
        const int m = q.tokens[s];
        present += m > 0;
        total += m;
    }
    bal = wave_sum(bal);
    zz = wave_sum(zz);
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        present += __shfl_xor(present, o);
        total += __shfl_xor(total, o);
    }
    if (threadIdx.x % kWave == 0) {
        bal_w[threadIdx.x / kWave] = bal;
        z_w[threadIdx.x / kWave] = zz;
        present_w[threadIdx.x / kWave] = present;
        total_w[threadIdx.x / kWave] = total;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            bal += bal_w[w];
            zz += z_w[w];
            present += present_w[w];
            total += total_w[w];
        }
        write_loss(q, bal, zz, present, total);
    }
}

// Gradient of the logits: each wave four tokens at a time, `steps` times.  The
// gates' part goes from the slots' lanes to the columns' lanes through a row of LDS.
template <int NV, bool VEC, bool BF16>
__global__ __launch_bounds__(kGradThreads) void router_grad_kernel(
    int T, int k, int E, const float* __restrict__ logits, const int32_t* __restrict__ idx,
    const uint8_t* __restrict__ keep, const float* __restrict__ w, const float* __restrict__ d_w,
    const uint8_t* __restrict__ mask, const int32_t* __restrict__ offs, int S, const int32_t* __restrict__ counts,
    const int32_t* __restrict__ tokens, float balance_coef, float z_coef, const float* __restrict__ d_loss, int steps,
    void* __restrict__ out) {
    __shared__ __attribute__((aligned(16))) float gates[kGradThreads / kRowLanes][64 * NV];
    __shared__ SequencesLds found;
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    const int row = threadIdx.x / kRowLanes, g = lane / kRowLanes, j = lane % kRowLanes;
    const int per_block = kGradWaves * kTokPerStep * steps;
    const int block_t0 = blockIdx.x * per_block;
    // four tokens: their logits and lane j's slot (expert -1: none)
    struct Rows {
        float v[NV][4];
        int e;
        float w, dw;
        bool masked;
    };
    auto load = [&](Rows& x, int t) __attribute__((always_inline)) {
        const size_t tt = t;
        load_row<NV, VEC>(logits + tt * E, E, j, x.v);
        x.e = -1;
        x.w = x.dw = 0.0f;
        if (d_w && j < k) {
            x.e = idx[tt * k + j];
            if ((keep && !keep[tt * k + j]) || static_cast<unsigned>(x.e) >= static_cast<unsigned>(E)) x.e = -1;
            const float a = w[tt * k + j], b = d_w[tt * k + j];
            if (x.e >= 0) {
                x.w = a;
                x.dw = b;
            }
        }
        x.masked = mask && mask[tt] == 0;
    };
    const int t_first = block_t0 + wave * kTokPerStep + g;
    const int mine = first_offset<kGradThreads>(offs, S);
    const float up = d_loss ? *d_loss : 1.0f;
    const int present = tokens[S], total_tokens = tokens[S + 1];
    Rows next;
    if (t_first < T) load(next, t_first);                // on their way while the block finds its sequences
    const Sequences seq = block_sequences<kGradThreads>(offs, S, block_t0, min(T, block_t0 + per_block) - 1, mine, found);
#pragma unroll
    for (int c = 0; c < NV; ++c)
        *reinterpret_cast<f32x4*>(&gates[row][64 * c + 4 * j]) = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    wave_fence();
    const float bal = present > 0 ? up * balance_coef * static_cast<float>(E) / static_cast<float>(k) /
                                        static_cast<float>(present)
                                  : 0.0f;
    const float zed = total_tokens > 0 ? up * 2.0f * z_coef / static_cast<float>(total_tokens) : 0.0f;

    for (int i = 0; i < steps; ++i) {
        const int t = t_first + i * kGradWaves * kTokPerStep;
        if (t >= T) break;                               // whole 16-lane rows
        const size_t tt = t;
        if (i > 0) load(next, t);
        Rows& x = next;
        float(&v)[NV][4] = x.v;
        const int e = x.e;
        const float ws = x.w, dw = x.dw;
        const int s = seq.of(t, seq.first);
        const bool inside = s >= 0 && s < S;
        float top, total;
        row_exp<NV>(v, top, total);
        const bool valid = inside && !(top == -INFINITY) && !x.masked;
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
                for (int i4 = 0; i4 < 4; ++i4) cc[c][i4] = cs * static_cast<float>(static_cast<int>(q[i4]));
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
    const LossPlan plan = loss_plan(T, S);
    LossArgs q{T, k, E, S, plan.per_wave, logits, idx, keep, mask, offs, balance_coef, z_coef, counts, probs, tokens, loss, {}};
    loss_ws_layout(T, E, S, workspace, &q.ws);
    const bool vec = E % 4 == 0 && aligned(logits, 16);
    auto launch = [&](auto NV) {
        constexpr int nv = decltype(NV)::value;
        constexpr int all = kSumWaves, few = kLossWaves;
        if (plan.one_launch && vec) loss_pieces_kernel<nv, true, all><<<1, kSumThreads, 0, stream>>>(q);
        else if (plan.one_launch) loss_pieces_kernel<nv, false, all><<<1, kSumThreads, 0, stream>>>(q);
        else if (vec) loss_pieces_kernel<nv, true, few><<<plan.blocks, kLossThreads, 0, stream>>>(q);
        else loss_pieces_kernel<nv, false, few><<<plan.blocks, kLossThreads, 0, stream>>>(q);
    };
    if (E <= 64) launch(std::integral_constant<int, 1>{});
    else if (E <= 128) launch(std::integral_constant<int, 2>{});
    else launch(std::integral_constant<int, 4>{});
    if (!plan.one_launch) {
        const int quarters = (E + 63) / 64;
        // more groups where a sequence has more pieces than 16 groups take soon (one sequence
        // of 8192 tokens 14 us against 20; 211 sequences of them 15 against 14)
        const dim3 grid(S < kSumBlocks ? S : kSumBlocks, quarters);
        if (plan.blocks / 8 > S) loss_sum_kernel<64><<<grid, 1024, 0, stream>>>(q);
        else loss_sum_kernel<16><<<grid, 256, 0, stream>>>(q);
        // sixteen waves past 1024 sequences (8192 tokens in 2000 18.3 us against 21.0 with four, 2^20
        // in 2^20 2349 against 3497; in 64 13.6 against 13.3)
        if (S <= 1024) loss_final_kernel<256><<<1, 256, 0, stream>>>(q, quarters);
        else loss_final_kernel<1024><<<1, 1024, 0, stream>>>(q, quarters);
    }
    CAP_LAUNCH_CHECK();
    return CAP_OK;
}

cap_status router_grad_launch(int T, int k, int E, const float* logits, const int32_t* idx, const uint8_t* keep,
                              const float* w, const float* d_w, const uint8_t* mask, const int32_t* offs, int S,
                              const int32_t* counts, const int32_t* tokens, float balance_coef, float z_coef,
                              const float* d_loss, cap_dtype dtype, void* d_logits, hipStream_t stream) {
    // two steps a wave once the chip is full (32768 tokens 15.2 us against 15.9; 8192 7.6 against
    // 6.4); past 2^28 tokens 16, for a launch of less than 2^32 threads
    const int steps = T > 1 << 28 ? 16 : T >= 16384 ? 2 : 1;
    const int per_block = kGradWaves * kTokPerStep * steps;
    const int blocks = (T - 1) / per_block + 1;
    const bool bf16 = dtype == CAP_DTYPE_BF16;
    const bool vec = E % 4 == 0 && aligned(logits, 16) && aligned(counts, 16) && aligned(d_logits, bf16 ? 8 : 16);
    auto launch = [&](auto NV, auto VEC, auto BF) {
        router_grad_kernel<decltype(NV)::value, decltype(VEC)::value, decltype(BF)::value>
            <<<blocks, kGradThreads, 0, stream>>>(T, k, E, logits, idx, keep, w, d_w, mask, offs, S, counts, tokens,
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
