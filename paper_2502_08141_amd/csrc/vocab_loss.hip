// Softmax cross entropy over a vocabulary and its gradient, without the logits in memory (the loss of the paper's fine-tuning runs, Sec. 2.1):
//   z = h W^T;   loss = log(sum_v exp z_v) - z_t;   dH = w (softmax(z) - e_t) W
//
// Two matrix products and two small passes.  The first product forms a tile of 256 words x 256 tokens of z in fp32 registers and leaves of it what
// does not depend on the other words: per token a whole number n not far from log2 e times the tile's largest z, the sum of 2^(z log2 e - n) over the words but
// the target, z_t where the tile has it, and, for the gradient, the exponentials themselves in bf16 (the target's as zero).  fp32 and bf16 reach from
// 2^-126 to 2^127, so n is zero where the largest is between 2^-32 and 2^64 (z from -22 to 44) and the multiple of 64 below elsewhere; what is less
// than 2^-94 of the largest may be lost.  A small pass over these numbers gives loss and lse.  The second product multiplies the exponentials with W and
// does not wait for that pass, whose workgroups stand behind its own.  Where n is not zero for every tile and every token with a target, it takes the tokens' largest n
// first and brings a tile's exponentials to that scale on the way into the matrix unit, a subtraction from their exponents and exact; else its loop is without
// (4096 x 32000 x 4096 by itself: 895 us with the subtraction, 818 without; a pass over the exponentials before it 90).  The token's factor
// weight / sum meets the fp32 sums.  So a probability is rounded once, to bf16; the factor also takes the rounded exponentials' sum back to that of the exact ones, so
// that a word's rounding counts by how far its row of W is from the others' mean, and not at all where one word has all that the target leaves (tokens sure of a wrong word,
// 32000 words, K 1024: dH 2.03e-3 off in the norm without, 1.68e-3 so, all of it the outputs' own rounding; 777 tokens of 50265 words take 217.5 us for 215.5).  The target's own term,
// weight (p_t - 1) W_t, is added in fp32: p_t is near one for most tokens of a trained model, and its rounding would be the gradient's error.  p_t - 1 and the loss come from
// the sum without the target, so that they keep their digits there.
// Tokens go in pieces whose exponentials fit kLossPiece bytes, so that neither the logits nor anything else of size M x V is ever there at once.
// (Pieces of the vocabulary would have to form z a second time for the gradient: 6 M V K operations in place of 4.)
// Graph replays: 4096 tokens of 32000 words, K 4096, 1636 to 1690 us by the card (1.27 to 1.31 PFLOP/s; the matrix unit busy for 76 % of the first product and 82 % of the
// second), 777 of 50265, K 1024, 217; 333 of 32000, K 4096, without the gradient 112, 90 with W in a cache; 16 of 32000, K 4096, 95 and without 53 (W at 5.6 and 5.0 TB/s); 19 of 1003, K 512, 15.1, three launches' latencies.
#include <algorithm>

#include "gemm_common.h"
#include "step.h"
#include "vocab_loss_plan.h"

namespace lowra {

namespace {

constexpr int THREADS = 512, WAVES = 8, DEPTH = kLossDepth;
typedef __bf16 v2bf16_t __attribute__((ext_vector_type(2)));
typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef short v8i16_t __attribute__((ext_vector_type(8)));
typedef unsigned short v2u16_t __attribute__((ext_vector_type(2)));
typedef unsigned short v8u16_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) v4i16_t* lds_v4i16_ptr;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -2e38f;                         // below every z that counts; times log2 e still finite, so that 2^(-inf - it) is zero

struct LossParams {
    const uint16_t *h, *W;
    const int32_t* targets;
    const float* weights;
    float *loss, *lse;
    uint16_t* dH;
    int M, V, K, VP, tiles, tile_shift;                  // this piece's tokens; VP: words in whole tiles of 2^tile_shift
    LossStat* stats;                                     // [tiles][M]
    float* rounded;                                      // [tiles][M]: the sum again, of the exponentials as they are in P
    float* zt;                                           // [M]
    uint32_t* apart;                                     // [M / apart_tokens][tiles]: a target's token of these has a shift that is not zero
    int apart_tokens;
    float2* rows;                                        // [M]: weight / sum (of rounded exponentials), weight (p_t - 1)
    uint16_t* P;                                         // [M][VP]
    float* part;                                         // [splits][M][K]
    int splits, words_per_split;
    bool rows_inside;                                    // the tokens' numbers come with the second product's launch
};

// The tile of a workgroup: `group` tiles of one operand against all of the other in turn, so that the workgroups of an L2 share both (4096 x 32768 x 4096 by
// itself: four or eight 884 us, one 955, with the loop as it was then).
__device__ __forceinline__ void tile_of(int tile, int major, int minor, int group, int& a, int& b) {
    const int g = tile / (group * minor), r = tile - g * group * minor, n = min(group, major - g * group);
    a = g * group + r % n;
    b = r / n;
}

template <int N>
__device__ __forceinline__ void wait_transfers() { asm volatile("s_waitcnt vmcnt(%0)" : : "n"(N) : "memory"); }

// The steps of a product.  A step's operands are two tiles in one of STAGES stages of LDS.  fetch(s, i) asks for transfer i of T of step s, of which some steps
// leave out all but the first WT; read(s, kk, i) for operand registers i of R of slice kk (16 deep) of step s; mul(kk, j) is matrix instruction j of N of a slice.
// The only barrier of a step stands before its last slice, when that slice's operands are in registers: from there on the stage is free for step s + STAGES, whose
// transfers are dealt over two slices, and step s + 1 is there, so that its first operands are read under the last slice's products.  4096 x 32768 x 4096 by
// itself: 838 us; a barrier and all transfers at the beginning of a step 1042, all transfers in one slice 862, in three 5 % more than in two, without the
// priority over the other wavefront while transfers are issued 2 % more; four wavefronts with 128 x 128 outputs each 846 to 950, and 900 with the transfers in
// one slice; two workgroups of 256 x 128 outputs a unit 1117.  The matrix units are busy for 76 % of the first product's time and 82 % of the second's.
template <int STAGES, int T, int WT, int R, int N, class Fetch, class Read, class Mul>
__device__ __forceinline__ void product_steps(int steps, Fetch fetch, Read read, Mul mul) {
    constexpr int H = (T + 1) / 2;                       // transfers in the first of the two slices
#pragma unroll
    for (int s = 0; s < STAGES; ++s)
        if (s < steps) {
#pragma unroll
            for (int i = 0; i < T; ++i) fetch(s, i);
        }
    if (steps >= STAGES) wait_transfers<WT * (STAGES - 1)>();
    else wait_transfers<0>();
    asm volatile("s_barrier" : : : "memory");
#pragma unroll
    for (int i = 0; i < R; ++i) read(0, 0, i);
    for (int s = 0; s < steps; ++s) {
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            if (kk == 3) {
                if (STAGES > 2 && s + STAGES - 1 < steps) wait_transfers<WT * (STAGES - 2)>();
                else wait_transfers<0>();
                asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory");
                __builtin_amdgcn_s_setprio(1);
            }
            if (kk == 1) __builtin_amdgcn_s_setprio(0);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                mul(kk, j);
#pragma unroll
                for (int i = j * R / N; i < (j + 1) * R / N; ++i) {
                    if (kk < 3) read(s, kk + 1, i);
                    else read(s + 1, 0, i);              // (past the last step: registers that nothing uses)
                }
                if (kk == 3 && s + STAGES < steps) {
#pragma unroll
                    for (int i = j * H / N; i < (j + 1) * H / N; ++i) fetch(s + STAGES, i);
                }
                if (kk == 0 && s > 0 && s + STAGES - 1 < steps) {
#pragma unroll
                    for (int i = j * (T - H) / N; i < (j + 1) * (T - H) / N; ++i) fetch(s + STAGES - 1, H + i);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    }
}

// sum + both halves
__device__ __forceinline__ float sum_bf16x2(uint32_t e, float sum) {
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(v2bf16_t, e), __builtin_bit_cast(v2bf16_t, 0x3f803f80u), sum, false);
}

// ---- first product.  Words are the matrix instruction's rows, tokens its columns, so that a token's words lie in one lane and its other half: WV x (8 / WV)
// wavefronts, each with AT x BT tiles of 32 words x 32 tokens.
template <int WV, int AT, int BT, int STAGES>
struct Logits {
    static constexpr int WORDS = WV * AT * 32, TOKENS = WAVES / WV * BT * 32, STAGE = (WORDS + TOKENS) * ROWB, SMEM = STAGES * STAGE;
    static_assert(TOKENS * WORDS * 2 <= SMEM, "the exponentials of a tile");
};
template <int WV, int AT, int BT, int STAGES>
__global__ __launch_bounds__(THREADS, 2) void loss_logits_kernel(LossParams p) {
    using S = Logits<WV, AT, BT, STAGES>;
    constexpr int WORDS = S::WORDS, TOKENS = S::TOKENS, TW = WORDS / 64, TT = TOKENS / 64;       // transfers of a wavefront: eight rows each
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float join[WV][TOKENS], join_rounded[WV][TOKENS];
    const uint32_t smem_lds = (uint32_t)(uintptr_t)(lptr_t)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int vt, mt;
    tile_of(xcd_tile(blockIdx.x, gridDim.x), p.tiles, (p.M + TOKENS - 1) / TOKENS, 8, vt, mt);
    const int m0 = mt * TOKENS, v0 = vt * WORDS, steps = (p.K + DEPTH - 1) / DEPTH;
    const bufdesc_t src_w = buffer_desc(p.W + (size_t)v0 * p.K), src_h = buffer_desc(p.h + (size_t)m0 * p.K);
    uint32_t off_w[TW], off_h[TT];                       // rows past the end: the last one again
    auto offset = [&](int r, int last) __attribute__((always_inline)) { return (uint32_t)min(r, last) * (uint32_t)p.K * 2u + (uint32_t)((lane & 7) ^ ((r >> 1) & 7)) * 16u; };
#pragma unroll
    for (int i = 0; i < TW; ++i) off_w[i] = offset(wave * (8 * TW) + 8 * i + (lane >> 3), p.V - v0 - 1);
#pragma unroll
    for (int i = 0; i < TT; ++i) off_h[i] = offset(wave * (8 * TT) + 8 * i + (lane >> 3), p.M - m0 - 1);
    // lanes of the last step whose features lie past K get zeros; a row's chunk order depends on bit 3 of its number
    uint32_t past[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) past[i] = (steps - 1) * DEPTH + 8 * ((lane & 7) ^ ((4 * i + (lane >> 4)) & 7)) < p.K ? 0u : 0x80000000u;
    // A tile of few tokens is the only one to read its rows of W, and workgroups that all read the same columns of rows that lie 2^n bytes apart meet in a part of the memory's
    // channels: each begins with another step (16 and 128 tokens of 128256 words, K 2048, 120 and 132 -> 103 and 104 us, 16 of 32000, K 4096, 61 -> 52; 16 steps level).
    // Where tiles share rows, they do so because they read them together: 4096 tokens 826 us, with this 840 to 890.
    int at = __builtin_amdgcn_readfirstlane(p.M <= TOKENS && steps >= 32 ? vt % steps : 0) - 1;
    auto fetch = [&](int s, int i) __attribute__((always_inline)) {
        if (i == 0) at = at + 1 == steps ? 0 : at + 1;   // (transfers are asked for in order)
        const uint32_t stage = smem_lds + (uint32_t)(s % STAGES) * S::STAGE, soff = (uint32_t)at * (DEPTH * 2u), end = at == steps - 1 ? ~0u : 0u;
        if (i < TW) dma16_b(src_w, off_w[i < TW ? i : 0] | (past[(wave * TW + i) & 1] & end), soff, stage + (uint32_t)(wave * TW + i) * 1024u);
        else dma16_b(src_h, off_h[i < TW ? 0 : i - TW] | (past[(wave * TT + i - TW) & 1] & end), soff, stage + WORDS * ROWB + (uint32_t)(wave * TT + i - TW) * 1024u);
    };
    const int wv = wave / (WAVES / WV), wt = wave % (WAVES / WV), fi = lane & 31, half = lane >> 5;
    int koff[4];
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) koff[kk] = ((2 * kk + half) ^ ((fi >> 1) & 7)) << 4;
    const int a0 = (wv * AT * 32 + fi) * ROWB, b0 = WORDS * ROWB + (wt * BT * 32 + fi) * ROWB;
    floatx16_t acc[AT][BT];
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int b = 0; b < BT; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    bf16x8_t fa[2][AT], fb[2][BT];
    product_steps<STAGES, TW + TT, TW + TT, AT + BT, AT * BT>(
        steps, fetch,
        [&](int s, int kk, int i) __attribute__((always_inline)) {
            const uint8_t* st = smem + (s % STAGES) * S::STAGE + koff[kk];
            if (i < AT) fa[kk & 1][i < AT ? i : 0] = *reinterpret_cast<const bf16x8_t*>(st + a0 + i * 32 * ROWB);
            else fb[kk & 1][i < AT ? 0 : i - AT] = *reinterpret_cast<const bf16x8_t*>(st + b0 + (i - AT) * 32 * ROWB);
        },
        [&](int kk, int j) __attribute__((always_inline)) {
            acc[j / BT][j % BT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[kk & 1][j / BT], fb[kk & 1][j % BT], acc[j / BT][j % BT], 0, 0, 0);
        });
    // accumulator v of tile (a, b): word wv 32 AT + 32 a + 8 (v / 4) + 4 half + v % 4, token wt 32 BT + 32 b + fi
    const int words = p.V - v0, w0 = wv * AT * 32 + 4 * half, t0 = wt * BT * 32 + fi;
    if (words < WORDS) {                                 // uniform: words past V
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                if (w0 + a * 32 + 8 * (v >> 2) + (v & 3) >= words) {
#pragma unroll
                    for (int b = 0; b < BT; ++b) acc[a][b][v] = -INFINITY;
                }
    }
    float shift[BT], sum[BT];
    bool there[BT];
#pragma unroll
    for (int b = 0; b < BT; ++b) {
        float most = kLeast;
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
            for (int v = 0; v < 16; ++v) most = fmaxf(most, acc[a][b][v]);
        most = fmaxf(most, __shfl_xor(most, 32));
        if (half == 0) join[wv][t0 + 32 * b] = most;
        // the target leaves the sum
        const int m = m0 + t0 + 32 * b;
        const uint32_t target = m < p.M ? (uint32_t)p.targets[m] : ~0u, mine = target < (uint32_t)p.V ? target - (uint32_t)(v0 + w0) : ~0u;
        there[b] = target < (uint32_t)p.V;
        if (__any(mine < AT * 32)) {
#pragma unroll
            for (int a = 0; a < AT; ++a)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (mine == (uint32_t)(a * 32 + 8 * (v >> 2) + (v & 3))) {
                        p.zt[m] = acc[a][b][v];
                        acc[a][b][v] = -INFINITY;
                    }
        }
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < BT; ++b) {
        float most = join[0][t0 + 32 * b];
#pragma unroll
        for (int w = 1; w < WV; ++w) most = fmaxf(most, join[w][t0 + 32 * b]);
        const float n = most * kLog2e;
        shift[b] = n >= -32.0f && n <= 64.0f ? 0.0f : 64.0f * floorf(n * (1.0f / 64.0f));
    }
    if (p.P && wv == 0) {                                // uniform
        bool apart = false;
#pragma unroll
        for (int b = 0; b < BT; ++b) apart |= there[b] && shift[b] != 0.0f;
        const int of = mt * (WAVES / WV) + wt;
        const bool any = __any(apart);
        if (lane == 0 && of * (BT * 32) < p.M) p.apart[(size_t)of * p.tiles + vt] = any;
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < BT; ++b) {
        sum[b] = 0.0f;
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                acc[a][b][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[a][b][v], kLog2e, -shift[b]));
                sum[b] += acc[a][b][v];
            }
        sum[b] += __shfl_xor(sum[b], 32);
        if (half == 0) join[wv][t0 + 32 * b] = sum[b];
    }
    if (p.P) {                                           // the exponentials to LDS: a row a token, 16-byte chunks in another order for each of 32 tokens
#pragma unroll
        for (int b = 0; b < BT; ++b) {
            float held = 0.0f, more = 0.0f;
#pragma unroll
            for (int a = 0; a < AT; ++a)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int c = wv * AT * 4 + a * 4 + q;
                    const uint2 e = make_uint2(pack_bf16x2(acc[a][b][4 * q], acc[a][b][4 * q + 1]), pack_bf16x2(acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]));
                    *reinterpret_cast<uint2*>(smem + (t0 + 32 * b) * (WORDS * 2) + ((c ^ (fi & (WORDS / 8 - 1))) << 4) + 8 * half) = e;
                    held = sum_bf16x2(e.x, held);
                    more = sum_bf16x2(e.y, more);
                }
            held += more;
            held += __shfl_xor(held, 32);
            if (half == 0) join_rounded[wv][t0 + 32 * b] = held;
        }
    }
    __syncthreads();
    if (wv == 0 && half == 0) {
#pragma unroll
        for (int b = 0; b < BT; ++b) {
            const int t = t0 + 32 * b;
            float s = join[0][t];
#pragma unroll
            for (int w = 1; w < WV; ++w) s += join[w][t];
            if (m0 + t < p.M) p.stats[(size_t)vt * p.M + m0 + t] = LossStat{shift[b], s};
            if (!p.P) continue;
            s = join_rounded[0][t];
#pragma unroll
            for (int w = 1; w < WV; ++w) s += join_rounded[w][t];
            if (m0 + t < p.M) p.rounded[(size_t)vt * p.M + m0 + t] = s;
        }
    }
    if (!p.P) return;                                    // uniform
    constexpr int CH = WORDS / 8;                        // chunks a row
#pragma unroll
    for (int i = 0; i < TOKENS * CH / THREADS; ++i) {
        const int t = i * (THREADS / CH) + tid / CH, c = tid % CH;
        if (m0 + t < p.M) *reinterpret_cast<uint4*>(p.P + (size_t)(m0 + t) * p.VP + v0 + 8 * c) = *reinterpret_cast<const uint4*>(smem + t * (WORDS * 2) + ((c ^ (t & 31 & (CH - 1))) << 4));
    }
}

// ---- loss, lse and what the gradient needs of a token, 16 tokens a workgroup, the tiles dealt to 64 groups of threads (16 groups and 64 tokens: 777 tokens of 197 tiles
// 9.8 us for 7.4).  N wavefronts: 16, or 8 that have two groups' sums each, so that the order is the same.
constexpr int ROWS_TOKENS = 16;
template <int N, bool GRAD>
__device__ __forceinline__ void loss_rows(const LossParams& p, int block, float (*join)[2][ROWS_TOKENS]) {
    constexpr int SETS = 16 / N, SUMS = GRAD ? 2 : 1;    // of the exponentials, and of those that the gradient has
    const int tok = threadIdx.x % ROWS_TOKENS, group = threadIdx.x / ROWS_TOKENS, wave = threadIdx.x >> 6, m = block * ROWS_TOKENS + tok, at = min(m, p.M - 1);
    const bool first = (threadIdx.x & 63) < ROWS_TOKENS;
    float most = kLeast * kLog2e;
#pragma unroll 4
    for (int i = group; i < p.tiles; i += 4 * N) most = fmaxf(most, p.stats[(size_t)i * p.M + at].shift);
    most = fmaxf(most, __shfl_xor(most, 16));
    most = fmaxf(most, __shfl_xor(most, 32));
    if (first) join[wave][0][tok] = most;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < N; ++w) most = fmaxf(most, join[w][0][tok]);
    __syncthreads();
    float sum[SUMS];
#pragma unroll
    for (int q = 0; q < SETS; ++q) {
#pragma unroll
        for (float& v : sum) v = 0.0f;
#pragma unroll 4
        for (int i = group + 4 * N * q; i < p.tiles; i += 64) {
            const LossStat st = p.stats[(size_t)i * p.M + at];
            const float of[2] = {st.sum, GRAD ? p.rounded[(size_t)i * p.M + at] : 0.0f};
            const int by = (int)fmaxf(st.shift - most, -1000.0f);                  // (2^-128 by itself is none in fp32)
#pragma unroll
            for (int k = 0; k < SUMS; ++k) sum[k] += ldexpf(of[k], by);
        }
#pragma unroll
        for (int k = 0; k < SUMS; ++k) {
            sum[k] += __shfl_xor(sum[k], 16);
            sum[k] += __shfl_xor(sum[k], 32);
            if (first) join[N * q + wave][k][tok] = sum[k];
        }
    }
    __syncthreads();
    if (threadIdx.x >= ROWS_TOKENS || m >= p.M) return;
#pragma unroll
    for (int k = 0; k < SUMS; ++k) {
        sum[k] = join[0][k][tok];
#pragma unroll
        for (int w = 1; w < 16; ++w) sum[k] += join[w][k][tok];
    }
    const float others = sum[0];
    const int t = p.targets[m];
    const bool there = t >= 0 && t < p.V;
    const float xt = there ? __builtin_fmaf(p.zt[m], kLog2e, -most) : -INFINITY, et = exp2f(xt), total = others + et, log_total = logf(total);
    if (p.lse) p.lse[m] = __builtin_fmaf(most, kLn2, log_total);
    // From 2^24 on the target is nothing in the total, and et may be too small to have all its digits (the others are 2^-32 at least, so below it has them).
    const float ratio = others / et;
    p.loss[m] = !there ? 0.0f : ratio < 0x1p24f ? log1pf(ratio) : log_total - xt * kLn2;
    if constexpr (GRAD) {
        const float w = !there ? 0.0f : p.weights ? p.weights[m] : 1.0f;
        p.rows[m] = make_float2(w / total * (sum[1] > 0.0f ? others / sum[1] : 1.0f), -w * (others / total));
    }
}
template <bool GRAD>
__global__ __launch_bounds__(1024) void loss_rows_kernel(LossParams p) {
    __shared__ float join[16][2][ROWS_TOKENS];
    loss_rows<16, GRAD>(p, blockIdx.x, join);
}

// ---- second product, over a run of words: tokens (the exponentials) are the matrix instruction's rows, features its columns, W's operand read across its rows
// (ds_read_b64_tr_b16).  2 x 4 wavefronts, each with AT x 2 tiles of 32 tokens x 32 features.
__device__ __forceinline__ int wswz(int row, int c) { return row * 512 + ((c ^ (((row & 3) << 2) | ((row >> 2) & 3))) << 4); }
template <int AT, int STAGES>
struct Grad {
    static constexpr int TOKENS = 2 * AT * 32, W0 = TOKENS * ROWB, D0 = W0 + DEPTH * 512, STAGE = D0 + TOKENS * 4, SMEM = STAGES * STAGE;      // tokens', words' rows, shifts
};
template <int AT, int STAGES>
__global__ __launch_bounds__(THREADS, 2) void loss_grad_kernel(LossParams p) {
    using S = Grad<AT, STAGES>;
    constexpr int TOKENS = S::TOKENS, TP = TOKENS / 64, TW = 4;
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t smem_lds = (uint32_t)(uintptr_t)(lptr_t)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles_k = (p.K + 255) / 256, tiles_m = (p.M + TOKENS - 1) / TOKENS;
    const int tiles = tiles_k * tiles_m * p.splits;
    if ((int)blockIdx.x >= tiles) { loss_rows<WAVES, true>(p, blockIdx.x - tiles, reinterpret_cast<float(*)[2][ROWS_TOKENS]>(smem)); return; }
    const int work = xcd_tile(blockIdx.x, tiles), split = __builtin_amdgcn_readfirstlane(work / (tiles_k * tiles_m));
    int mt, kt;
    tile_of(work - split * (tiles_k * tiles_m), tiles_m, tiles_k, 4, mt, kt);
    const int k0 = kt * 256, m0 = mt * TOKENS, w0 = split * p.words_per_split, steps = (min(w0 + p.words_per_split, p.VP) - w0) / DEPTH;
    const uint16_t* P = p.P + (size_t)m0 * p.VP + w0;
    const uint16_t* W = p.W + (size_t)w0 * p.K + k0;
    const bufdesc_t src_p = buffer_desc(P);
    uint32_t off_p[TP], off_w[TW];
#pragma unroll
    for (int i = 0; i < TP; ++i) {                       // token rows of 128 bytes, eight a transfer
        const int r = wave * (8 * TP) + 8 * i + (lane >> 3);
        off_p[i] = (uint32_t)min(r, p.M - 1 - m0) * (uint32_t)p.VP * 2u + (uint32_t)((lane & 7) ^ ((r >> 1) & 7)) * 16u;
    }
#pragma unroll
    for (int i = 0; i < TW; ++i) {                       // words' rows of 512 bytes, two a transfer; features past K come as zeros
        const int r = wave * 8 + 2 * i + (lane >> 5), c = (lane & 31) ^ (((r & 3) << 2) | ((r >> 2) & 3));
        off_w[i] = k0 + 8 * c < p.K ? (uint32_t)r * (uint32_t)p.K * 2u + (uint32_t)c * 16u : 0x80000000u;
    }
    const uint32_t off_d = (uint32_t)min(m0 + wave * 64 + lane, p.M - 1) * (uint32_t)sizeof(LossStat);
    const int per = (1 << p.tile_shift) / DEPTH - 1;     // of a tile's steps the first has none of these bits
    uint32_t apart = 0;
    {
        const int first = m0 / p.apart_tokens, n = ((min(m0 + TOKENS, p.M) - 1) / p.apart_tokens + 1 - first) * p.tiles;
        for (int i = tid; i < n; i += THREADS) apart |= p.apart[(size_t)first * p.tiles + i];
    }
    const bool scaled = __builtin_amdgcn_readfirstlane(__syncthreads_or((int)apart)) != 0;
    auto fetch = [&](int s, int i) __attribute__((always_inline)) {
        const uint32_t stage = smem_lds + (uint32_t)(s % STAGES) * S::STAGE;
        if (i == TP + TW) {                              // the shifts of a tile, with its first step
            if (scaled && wave < TP && (s & per) == 0)
                dma4_b(buffer_desc(p.stats + (size_t)((w0 + s * DEPTH) >> p.tile_shift) * p.M), off_d, stage + S::D0 + (uint32_t)wave * 256u);
        } else if (i < TP) dma16_b(src_p, off_p[i < TP ? i : 0], (uint32_t)s * (DEPTH * 2u), stage + (uint32_t)(wave * TP + i) * 1024u);
        else {                                           // words past V come as zeros, too
            const int r = wave * 8 + 2 * (i - TP) + (lane >> 5);
            dma16_b(buffer_desc(W + (size_t)s * DEPTH * p.K), r < p.V - w0 - s * DEPTH ? off_w[i < TP ? 0 : i - TP] : 0x80000000u, 0, stage + S::W0 + (uint32_t)(wave * TW + i - TP) * 1024u);
        }
    };
    const int wm = wave >> 2, wn = wave & 3, fi = lane & 31, half = lane >> 5;
    int koff[4], tr[2][2];                               // tr: lane -> (word 8 half + 4 e + L / 4, four features from 4 (L % 4))
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) koff[kk] = ((2 * kk + half) ^ ((fi >> 1) & 7)) << 4;
    {
        const int L = lane & 15, grp = (lane >> 4) & 1;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int b = 0; b < 2; ++b) tr[e][b] = S::W0 + wswz(8 * half + 4 * e + (L >> 2), wn * 8 + b * 4 + grp * 2 + ((L & 3) >> 1)) + (L & 1) * 8;
    }
    const int a0 = (wm * AT * 32 + fi) * ROWB;
    floatx16_t acc[AT][2];
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    bf16x8_t fa[2][AT];
    v4i16_t fb[2][2][2];
    float most[AT];                                      // the tokens' largest shifts, which their scale is
    uint32_t drop[AT];                                   // how far this step's tile is below: exponents of both halves
    if (scaled) {
        constexpr int PARTS = THREADS / TOKENS;
        float* join = reinterpret_cast<float*>(smem);
        if (tid < PARTS * TOKENS) {
            const LossStat* of = p.stats + min(m0 + tid % TOKENS, p.M - 1);
            float l = kLeast * kLog2e;
#pragma unroll 8
            for (int i = tid / TOKENS; i < p.tiles; i += PARTS) l = fmaxf(l, of[(size_t)i * p.M].shift);
            join[tid] = l;
        }
        __syncthreads();
#pragma unroll
        for (int a = 0; a < AT; ++a) {
            most[a] = kLeast * kLog2e;
#pragma unroll
            for (int r = 0; r < PARTS; ++r) most[a] = fmaxf(most[a], join[r * TOKENS + wm * AT * 32 + a * 32 + fi]);
        }
        __syncthreads();
    }
    auto run = [&](auto SCALED_) __attribute__((always_inline)) {
        constexpr bool SCALED = decltype(SCALED_)::value;
        product_steps<STAGES, TP + TW + SCALED, TP + TW, AT + 4 + (SCALED ? AT : 0), AT * 2>(
            steps, fetch,
            [&](int s, int kk, int i) __attribute__((always_inline)) {
                const uint32_t st = (uint32_t)(s % STAGES) * S::STAGE;
                if (i < AT) fa[kk & 1][i < AT ? i : 0] = *reinterpret_cast<const bf16x8_t*>(smem + st + koff[kk] + a0 + i * 32 * ROWB);
                else if (i >= AT + 4) {
                    const int a = i < AT + 4 ? 0 : i - AT - 4;
                    // an exponential times 2^-d: bf16 has its exponent from bit 7 on, and 255 leaves nothing of any
                    if (kk == 0 && (s & per) == 0)
                        drop[a] = ((uint32_t)fminf(most[a] - *reinterpret_cast<const float*>(smem + st + S::D0 + (wm * AT * 32 + a * 32 + fi) * 4), 255.0f) << 7) * 0x10001u;
                } else {
                    const int q = i < AT || i >= AT + 4 ? 0 : i - AT, b = q >> 1, e = q & 1;
                    fb[kk & 1][b][e] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(uintptr_t)(smem_lds + st + tr[e][b] + kk * 16 * 512));
                }
            },
            [&](int kk, int j) __attribute__((always_inline)) {
                const int a = j >> 1, b = j & 1;
                if (SCALED && b == 0) {                      // (an exponent that runs out leaves zero)
                    const v2u16_t d = __builtin_bit_cast(v2u16_t, drop[a]);
                    fa[kk & 1][a] = __builtin_bit_cast(bf16x8_t, __builtin_elementwise_sub_sat(__builtin_bit_cast(v8u16_t, fa[kk & 1][a]), v8u16_t{d[0], d[1], d[0], d[1], d[0], d[1], d[0], d[1]}));
                }
                const v4i16_t lo = fb[kk & 1][b][0], hi = fb[kk & 1][b][1];
                acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[kk & 1][a], __builtin_bit_cast(bf16x8_t, v8i16_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]}),
                                                                    acc[a][b], 0, 0, 0);
            });
    };
    if (scaled) run(std::true_type{});
    else run(std::false_type{});
    float* out = p.part + (size_t)split * p.M * p.K;
#pragma unroll
    for (int a = 0; a < AT; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int k = k0 + wn * 64 + b * 32 + fi;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int m = m0 + wm * AT * 32 + a * 32 + 8 * (v >> 2) + 4 * half + (v & 3);
                if (m < p.M && k < p.K) out[(size_t)m * p.K + k] = acc[a][b][v];
            }
        }
}

// ---- the splits' sums times the token's factor, and the target's term
__global__ __launch_bounds__(256) void loss_sum_kernel(LossParams p) {
    const int runs = p.K / 8;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < (long long)p.M * runs; id += (long long)gridDim.x * 256) {
        const int m = (int)(id / runs), c = (int)(id % runs), t = p.targets[m];
        const bool there = t >= 0 && t < p.V;
        const float2 f = p.rows[m];
        const uint4 q = reinterpret_cast<const uint4*>(p.W + (size_t)(there ? t : 0) * p.K)[c];
        float v[8] = {};
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            const float4* x = reinterpret_cast<const float4*>(p.part + ((size_t)s * p.M + m) * p.K + 8 * c);
            const float4 lo = x[0], hi = x[1];
            v[0] += lo.x; v[1] += lo.y; v[2] += lo.z; v[3] += lo.w; v[4] += hi.x; v[5] += hi.y; v[6] += hi.z; v[7] += hi.w;
        }
        const uint32_t u[4] = {q.x, q.y, q.z, q.w};
        uint4 o = zero4();
        if (there) {                                     // (nothing for a token without a target, whatever it holds)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __builtin_fmaf(f.y, bf16_bits_to_float(u[i] & 0xffffu), v[2 * i] * f.x);
                v[2 * i + 1] = __builtin_fmaf(f.y, __builtin_bit_cast(float, u[i] & 0xffff0000u), v[2 * i + 1] * f.x);
            }
            o = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        }
        reinterpret_cast<uint4*>(p.dH + (size_t)m * p.K)[c] = o;
    }
}

int loss_rows_blocks(int M) { return (M + ROWS_TOKENS - 1) / ROWS_TOKENS; }
template <class K>
hipError_t launch_tiles(K kernel, int smem, long long grid, const LossParams& p, hipStream_t st) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != hipSuccess) return e;
    kernel<<<dim3((unsigned)grid), dim3(THREADS), smem, st>>>(p);
    return hipGetLastError();
}
template <int WV, int AT, int BT, int STAGES>
hipError_t launch_logits(LossParams& p, hipStream_t st) {
    using S = Logits<WV, AT, BT, STAGES>;
    p.apart_tokens = BT * 32;
    return launch_tiles(loss_logits_kernel<WV, AT, BT, STAGES>, S::SMEM, (long long)((p.M + S::TOKENS - 1) / S::TOKENS) * p.tiles, p, st);
}
template <int AT, int STAGES>
hipError_t launch_grad(const LossParams& p, hipStream_t st) {
    using S = Grad<AT, STAGES>;
    return launch_tiles(loss_grad_kernel<AT, STAGES>, S::SMEM, (long long)((p.M + S::TOKENS - 1) / S::TOKENS) * ((p.K + 255) / 256) * p.splits + (p.rows_inside ? loss_rows_blocks(p.M) : 0), p, st);
}

}  // namespace

size_t vocab_loss_workspace_bytes(int M, int V, int K, bool grad) { return loss_plan(M, V, K, grad, device_compute_units()).bytes; }

hipError_t launch_vocab_loss(const VocabLossArgs& a, hipStream_t st) {
    const bool grad = a.dH != nullptr;
    const LossPlan l = loss_plan(a.M, a.V, a.K, grad, device_compute_units());
    uint8_t* ws = static_cast<uint8_t*>(a.workspace);
    for (int m0 = 0; m0 < a.M; m0 += l.rows) {
        LossParams p{};
        p.M = std::min(l.rows, a.M - m0); p.V = a.V; p.K = a.K; p.VP = l.VP; p.tiles = l.tiles; p.tile_shift = l.shift;
        p.h = a.h + (size_t)m0 * a.K; p.W = a.W; p.targets = a.targets + m0; p.weights = a.weights ? a.weights + m0 : nullptr;
        p.loss = a.loss + m0; p.lse = a.lse ? a.lse + m0 : nullptr; p.dH = grad ? a.dH + (size_t)m0 * a.K : nullptr;
        p.stats = reinterpret_cast<LossStat*>(ws + l.stats0); p.zt = reinterpret_cast<float*>(ws + l.zt0);
        if (grad) {
            p.rounded = reinterpret_cast<float*>(ws + l.rounded0); p.apart = reinterpret_cast<uint32_t*>(ws + l.apart0); p.rows = reinterpret_cast<float2*>(ws + l.rows0);
            p.part = reinterpret_cast<float*>(ws + l.part0); p.P = reinterpret_cast<uint16_t*>(ws + l.P0);
            p.splits = l.splits; p.words_per_split = l.words;
        }
        hipError_t e;
        // 64 tokens: two workgroups of three stages a unit where there are more tiles than units (K 640, 100000 words 42 -> 35 us), else one of six (K 8192, 16000 words 76 -> 71)
        if (l.shift == 7 && l.tokens == 128) e = launch_logits<4, 1, 2, 4>(p, st);
        else if (l.shift == 7 && l.tiles > device_compute_units()) e = launch_logits<4, 1, 1, 3>(p, st);
        else if (l.shift == 7) e = launch_logits<4, 1, 1, 6>(p, st);
        else if (l.tokens == 256) e = launch_logits<2, 4, 2, 2>(p, st);
        else if (l.tokens == 192) e = launch_logits<4, 2, 3, 2>(p, st);
        else if (l.tokens == 128) e = launch_logits<4, 2, 2, 3>(p, st);
        else e = launch_logits<4, 2, 1, 3>(p, st);
        if (e != hipSuccess) return e;
        // A launch less for few tokens (64 of 50265 words, K 1024, 64.0 -> 59.0 us, of 1003, K 512, 19.5 -> 16.0; 4096 of 1003 36.9 -> 35.2; 8192 level).  Beside the
        // second product's LDS a unit holds one such workgroup, so that many take longer (65536 tokens of 1003 words 257 us, in a launch of their own 251).
        p.rows_inside = grad && loss_rows_blocks(p.M) <= device_compute_units();
        if (!p.rows_inside) {
            if (grad) loss_rows_kernel<true><<<dim3((unsigned)loss_rows_blocks(p.M)), dim3(1024), 0, st>>>(p);
            else loss_rows_kernel<false><<<dim3((unsigned)loss_rows_blocks(p.M)), dim3(1024), 0, st>>>(p);
            if ((e = hipGetLastError()) != hipSuccess) return e;
        }
        if (!grad) continue;
        if (l.grad_tokens == 256) e = launch_grad<4, 2>(p, st);
        else if (l.grad_tokens == 192) e = launch_grad<3, 2>(p, st);
        else if (l.grad_tokens == 128) e = launch_grad<2, 3>(p, st);
        else e = launch_grad<1, 3>(p, st);
        if (e != hipSuccess) return e;
        loss_sum_kernel<<<dim3((unsigned)std::min<long long>(((long long)p.M * (a.K / 8) + 255) / 256, 16 * device_compute_units())), dim3(256), 0, st>>>(p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace lowra
