// Softmax cross entropy over a vocabulary and its gradient, without the logits in memory (the loss of the paper's fine-tuning runs, Sec. 2.1):
//   z = h W^T;   loss = log(sum_v exp z_v) - z_t;   dH = w (softmax(z) - e_t) W
//
// Two matrix products.  The first forms a tile of 256 words x 256 tokens of z in fp32 registers and leaves of it what does not depend on the
// other words: per token the tile's largest z, the sum of exp(z - largest) over the words but the target, z_t where the tile has it, and, for the gradient,
// the exponentials themselves in bf16 (the target's as zero).  A pass over these statistics gives loss and lse; another one
// turns the exponentials into probabilities times the token's weight, where they lie; the second product multiplies them with W.
// The target's own term, (p_t - 1) W_t, is added in fp32: p_t is near one for most tokens of a trained model, and its rounding would be the
// gradient's error.  p_t - 1 and the loss come from the sum without the target, so that they keep their digits there.
// Tokens go in pieces whose exponentials fit kLossPiece bytes, so that neither the logits nor anything else of size M x V is ever there at once.
// (Pieces of the vocabulary would have to form z a second time for the gradient: 6 M V K operations in place of 4.)
#include <algorithm>

#include "gemm_common.h"
#include "step.h"

namespace lowra {

namespace {

constexpr int TILE = 256, DEPTH = 64, THREADS = 512;
constexpr int OPB = TILE * DEPTH * 2;                    // one operand of a step: 32 KB
constexpr int SMEM = 4 * OPB;                            // two stages of both
typedef short v4i16_t __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) v4i16_t* lds_v4i16_ptr;

constexpr float kLeast = -2e38f;                         // below every z that counts; times log2 e still finite, so that exp(-inf - kLeast) is zero
struct LossStat { float most, sum; };                    // of a tile's words, the target aside in the sum

struct LossParams {
    const uint16_t *h, *W;
    const int32_t* targets;
    const float* weights;
    float *loss, *lse;
    uint16_t* dH;
    int M, V, K, VP, tiles;                              // this piece's tokens; VP: words in whole tiles
    LossStat* stats;                                     // [M][tiles]
    float* zt;                                           // [M]
    float2* rows;                                        // [M]: lse, weight (p_t - 1)
    uint16_t* P;                                         // [M][VP]
    float* part;                                         // [splits][M][K]
    int splits, words_per_split;
};

// ---- first product: 256 words (operand A) x 256 tokens (operand B) a workgroup; wavefront (wv, wt) has 128 words x 64 tokens
__global__ __launch_bounds__(THREADS) void loss_logits_kernel(LossParams p) {
    extern __shared__ __align__(16) uint8_t smem[];
    __shared__ float join[2][TILE];
    const uint32_t smem_lds = (uint32_t)(uintptr_t)(lptr_t)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = xcd_tile(blockIdx.x, gridDim.x), tiles_m = (p.M + TILE - 1) / TILE;
    const int mt = tile % tiles_m, vt = tile / tiles_m, m0 = mt * TILE, v0 = vt * TILE;      // workgroups of an L2 share words
    const int steps = (p.K + DEPTH - 1) / DEPTH;
    // transfers: wavefronts 0..3 bring the words' rows, 4..7 the tokens'; each 8 times 8 rows of 128 bytes
    const bool tok = wave >= 4;
    const int first_row = (wave & 3) * 64, last = (tok ? p.M - m0 : p.V - v0) - 1;
    const bufdesc_t src = buffer_desc(tok ? p.h + (size_t)m0 * p.K : p.W + (size_t)v0 * p.K);
    uint32_t voff[8];
    int chunk[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = first_row + 8 * i + (lane >> 3);
        chunk[i] = (lane & 7) ^ ((r >> 1) & 7);
        voff[i] = (uint32_t)min(r, last) * (uint32_t)p.K * 2u + (uint32_t)chunk[i] * 16u;
    }
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const uint32_t dst = smem_lds + (uint32_t)(s & 1) * (2 * OPB) + (tok ? OPB : 0) + (uint32_t)first_row * ROWB;
        if ((s + 1) * DEPTH <= p.K) {
#pragma unroll
            for (int i = 0; i < 8; ++i) dma16_b(src, voff[i], (uint32_t)s * (DEPTH * 2u), dst + i * 1024u);
        } else {                                         // the features past K come as zeros
#pragma unroll
            for (int i = 0; i < 8; ++i) dma16_b(src, s * DEPTH + 8 * chunk[i] < p.K ? voff[i] : 0x80000000u, (uint32_t)s * (DEPTH * 2u), dst + i * 1024u);
        }
    };
    const int wv = wave >> 2, wt = wave & 3, fi = lane & 31, half = lane >> 5, fsw = (fi >> 1) & 7;
    floatx16_t acc[4][2];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    fetch(0);
    for (int s = 0; s < steps; ++s) {
        dma_wait_all();
        __syncthreads();                                 // step s is there, and the last readers of the other stage are done
        if (s + 1 < steps) fetch(s + 1);
        const uint8_t* st = smem + (s & 1) * (2 * OPB);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            const int koff = ((2 * kk + half) ^ fsw) << 4;
            bf16x8_t fa[4], fb[2];
#pragma unroll
            for (int a = 0; a < 4; ++a) fa[a] = *reinterpret_cast<const bf16x8_t*>(st + (wv * 128 + a * 32 + fi) * ROWB + koff);
#pragma unroll
            for (int b = 0; b < 2; ++b) fb[b] = *reinterpret_cast<const bf16x8_t*>(st + OPB + (wt * 64 + b * 32 + fi) * ROWB + koff);
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 2; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[a], fb[b], acc[a][b], 0, 0, 0);
        }
    }
    // accumulator v of tile (a, b): word wv 128 + 32 a + 8 (v / 4) + 4 half + v % 4, token wt 64 + 32 b + fi
    const int words = p.V - v0;
    float most[2];
    int target[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int t = wt * 64 + b * 32 + fi;
        target[b] = m0 + t < p.M ? (int)((uint32_t)p.targets[m0 + t] - (uint32_t)v0) : -1;
        most[b] = kLeast;
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int word = wv * 128 + a * 32 + 8 * (v >> 2) + 4 * half + (v & 3);
                if (word < words) most[b] = fmaxf(most[b], acc[a][b][v]);
            }
        most[b] = fmaxf(most[b], __shfl_xor(most[b], 32));
        if (half == 0) join[wv][t] = most[b];
    }
    __syncthreads();
#pragma unroll
    for (int b = 0; b < 2; ++b) most[b] = fmaxf(join[0][wt * 64 + b * 32 + fi], join[1][wt * 64 + b * 32 + fi]);
    __syncthreads();
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int t = wt * 64 + b * 32 + fi;
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int word = wv * 128 + a * 32 + 8 * (v >> 2) + 4 * half + (v & 3);
                const float z = acc[a][b][v];
                float e = __builtin_amdgcn_exp2f((z - most[b]) * 1.4426950408889634f);      // (the difference first: its rounding does not grow with z)
                if (word >= words || word == target[b]) e = 0.0f;
                if (word == target[b] && word < words) p.zt[m0 + t] = z;
                sum[b] += e;
                acc[a][b][v] = e;
            }
        sum[b] += __shfl_xor(sum[b], 32);
        if (half == 0) join[wv][t] = sum[b];
    }
    __syncthreads();
    if (wv == 0 && half == 0) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int t = wt * 64 + b * 32 + fi;
            if (m0 + t < p.M) p.stats[(size_t)(m0 + t) * p.tiles + vt] = LossStat{most[b], join[0][t] + join[1][t]};
        }
    }
    if (!p.P) return;                                    // uniform
    // the exponentials through LDS: rows of 512 bytes a token, 16-byte chunks in another order for each of 32 tokens
#pragma unroll
    for (int b = 0; b < 2; ++b) {
        const int t = wt * 64 + b * 32 + fi;
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = (wv * 128 + a * 32 + 8 * q) >> 3;
                *reinterpret_cast<uint2*>(smem + t * 512 + ((c ^ fi) << 4) + 8 * half) =
                    make_uint2(pack_bf16x2(acc[a][b][4 * q], acc[a][b][4 * q + 1]), pack_bf16x2(acc[a][b][4 * q + 2], acc[a][b][4 * q + 3]));
            }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < TILE * 32 / THREADS; ++i) {
        const int t = i * (THREADS / 32) + (tid >> 5), c = tid & 31;
        if (m0 + t < p.M) *reinterpret_cast<uint4*>(p.P + (size_t)(m0 + t) * p.VP + v0 + 8 * c) = *reinterpret_cast<const uint4*>(smem + t * 512 + ((c ^ (t & 31)) << 4));
    }
}

// ---- a wavefront a token: loss, lse and the target's factor
__global__ __launch_bounds__(256) void loss_rows_kernel(LossParams p) {
    const int m = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (m >= p.M) return;
    const LossStat* st = p.stats + (size_t)m * p.tiles;
    const int t = p.targets[m];
    const bool there = t >= 0 && t < p.V;
    const float zt = there ? p.zt[m] : kLeast;
    float most = zt;
    for (int i = lane; i < p.tiles; i += 64) most = fmaxf(most, st[i].most);
    for (int s = 32; s; s >>= 1) most = fmaxf(most, __shfl_xor(most, s));
    float others = 0.0f;
    for (int i = lane; i < p.tiles; i += 64) others += st[i].sum * __builtin_amdgcn_exp2f((st[i].most - most) * 1.4426950408889634f);
    for (int s = 32; s; s >>= 1) others += __shfl_xor(others, s);
    if (lane != 0) return;
    const float et = there ? expf(zt - most) : 0.0f, total = others + et;
    const float log_total = zt == most ? log1pf(others) : logf(total);      // (e_t is one: by the others alone)
    const float lse = most + log_total;
    p.loss[m] = there ? (most - zt) + log_total : 0.0f;
    if (p.lse) p.lse[m] = lse;
    if (p.rows) {
        const float w = !there ? 0.0f : p.weights ? p.weights[m] : 1.0f;
        p.rows[m] = make_float2(lse, there ? -w * (others / total) : 0.0f);
    }
}

// ---- the exponentials of a tile become weight times probability, where they lie; nothing for a token without a target, whatever it holds
__global__ __launch_bounds__(256) void loss_scale_kernel(LossParams p) {
    const int parts = (p.VP / 8 + 1023) / 1024, m = blockIdx.x / parts;
    const int t = p.targets[m];
    const bool there = t >= 0 && t < p.V;
    const float w = !there ? 0.0f : p.weights ? p.weights[m] : 1.0f, lse = p.rows[m].x;
    uint4* row = reinterpret_cast<uint4*>(p.P + (size_t)m * p.VP);
    const int c0 = (blockIdx.x % parts) * 1024;
    for (int c = c0 + threadIdx.x; c < min(c0 + 1024, p.VP / 8); c += 256) {
        const float f = w * __builtin_amdgcn_exp2f((p.stats[(size_t)m * p.tiles + (c >> 5)].most - lse) * 1.4426950408889634f);
        uint4 q = there ? row[c] : zero4();
        uint32_t* u = reinterpret_cast<uint32_t*>(&q);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (there) u[i] = pack_bf16x2(bf16_bits_to_float(u[i] & 0xffffu) * f, __builtin_bit_cast(float, u[i] & 0xffff0000u) * f);
        row[c] = q;
    }
}

// ---- second product: 256 tokens (operand A: P) x 256 features (operand B: W, read across its rows) a workgroup, over a run of words
__device__ __forceinline__ int wswz(int row, int c) { return row * 512 + ((c ^ (((row & 3) << 2) | ((row >> 2) & 3))) << 4); }
__global__ __launch_bounds__(THREADS) void loss_grad_kernel(LossParams p) {
    extern __shared__ __align__(16) uint8_t smem[];
    const uint32_t smem_lds = (uint32_t)(uintptr_t)(lptr_t)smem;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tiles_k = (p.K + TILE - 1) / TILE, tiles_m = (p.M + TILE - 1) / TILE;
    const int work = xcd_tile(blockIdx.x, gridDim.x), split = work / (tiles_k * tiles_m), tile = work % (tiles_k * tiles_m);
    const int k0 = (tile % tiles_k) * TILE, m0 = (tile / tiles_k) * TILE;
    const int w0 = split * p.words_per_split, w1 = min(w0 + p.words_per_split, p.VP);
    const int steps = (w1 - w0) / DEPTH;
    const bool tok = wave >= 4;
    const int wq = wave & 3, last = p.M - 1 - m0;
    const size_t step_bytes = tok ? DEPTH * 2 : (size_t)DEPTH * p.K * 2;
    const uint8_t* base = tok ? reinterpret_cast<const uint8_t*>(p.P + (size_t)m0 * p.VP + w0) : reinterpret_cast<const uint8_t*>(p.W + (size_t)w0 * p.K + k0);
    uint32_t voff[8];
    int row[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (tok) {                                       // 64 token rows of 128 bytes
            row[i] = wq * 64 + 8 * i + (lane >> 3);
            voff[i] = (uint32_t)min(row[i], last) * (uint32_t)p.VP * 2u + (uint32_t)((lane & 7) ^ ((row[i] >> 1) & 7)) * 16u;
        } else {                                         // 16 words' rows of 512 bytes
            row[i] = wq * 16 + 2 * i + (lane >> 5);
            const int c = (lane & 31) ^ (((row[i] & 3) << 2) | ((row[i] >> 2) & 3));
            voff[i] = k0 + 8 * c < p.K ? (uint32_t)row[i] * (uint32_t)p.K * 2u + (uint32_t)c * 16u : 0x80000000u;
        }
    }
    auto fetch = [&](int s) __attribute__((always_inline)) {
        const uint32_t dst = smem_lds + (uint32_t)(s & 1) * (2 * OPB) + (tok ? 0 : OPB) + (uint32_t)wq * 8192u;
        const bufdesc_t src = buffer_desc(base + (size_t)s * step_bytes);
        if (tok || w0 + (s + 1) * DEPTH <= p.V) {
#pragma unroll
            for (int i = 0; i < 8; ++i) dma16_b(src, voff[i], 0, dst + i * 1024u);
        } else {                                         // the words past V come as zeros
#pragma unroll
            for (int i = 0; i < 8; ++i) dma16_b(src, w0 + s * DEPTH + row[i] < p.V ? voff[i] : 0x80000000u, 0, dst + i * 1024u);
        }
    };
    const int wm = wave >> 2, wn = wave & 3, fi = lane & 31, half = lane >> 5, fsw = (fi >> 1) & 7;
    int tr[2][2];                                        // lane -> (word 8 half + 4 e + L / 4, four features from 4 (L % 4))
    {
        const int L = lane & 15, grp = (lane >> 4) & 1;
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int b = 0; b < 2; ++b) tr[e][b] = OPB + wswz(8 * half + 4 * e + (L >> 2), wn * 8 + b * 4 + grp * 2 + ((L & 3) >> 1)) + (L & 1) * 8;
    }
    floatx16_t acc[4][2];
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[a][b][v] = 0.0f;
    if (steps > 0) fetch(0);
    for (int s = 0; s < steps; ++s) {
        dma_wait_all();
        __syncthreads();
        if (s + 1 < steps) fetch(s + 1);
        const uint8_t* st = smem + (s & 1) * (2 * OPB);
        const uint32_t sl = smem_lds + (uint32_t)(s & 1) * (2 * OPB);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            bf16x8_t fa[4], fb[2];
#pragma unroll
            for (int a = 0; a < 4; ++a) fa[a] = *reinterpret_cast<const bf16x8_t*>(st + (wm * 128 + a * 32 + fi) * ROWB + (((2 * kk + half) ^ fsw) << 4));
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const v4i16_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(uintptr_t)(sl + tr[0][b] + kk * 16 * 512));
                const v4i16_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4i16_ptr)(uintptr_t)(sl + tr[1][b] + kk * 16 * 512));
                typedef short v8i16_t __attribute__((ext_vector_type(8)));
                fb[b] = __builtin_bit_cast(bf16x8_t, v8i16_t{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
            }
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 2; ++b) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[a], fb[b], acc[a][b], 0, 0, 0);
        }
    }
    float* out = p.part + (size_t)split * p.M * p.K;
#pragma unroll
    for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const int k = k0 + wn * 64 + b * 32 + fi;
#pragma unroll
            for (int v = 0; v < 16; ++v) {
                const int m = m0 + wm * 128 + a * 32 + 8 * (v >> 2) + 4 * half + (v & 3);
                if (m < p.M && k < p.K) out[(size_t)m * p.K + k] = acc[a][b][v];
            }
        }
}

// ---- the splits' sums and the target's term
__global__ __launch_bounds__(256) void loss_sum_kernel(LossParams p) {
    const int runs = p.K / 8;
    for (long long id = blockIdx.x * 256 + threadIdx.x; id < (long long)p.M * runs; id += gridDim.x * 256) {
        const int m = (int)(id / runs), c = (int)(id % runs), t = p.targets[m];
        float v[8] = {};
        for (int s = 0; s < p.splits; ++s) {
            const float4* q = reinterpret_cast<const float4*>(p.part + ((size_t)s * p.M + m) * p.K + 8 * c);
            const float4 x = q[0], y = q[1];
            v[0] += x.x; v[1] += x.y; v[2] += x.z; v[3] += x.w; v[4] += y.x; v[5] += y.y; v[6] += y.z; v[7] += y.w;
        }
        uint4 o = zero4();
        if (t >= 0 && t < p.V) {
            const uint4 q = reinterpret_cast<const uint4*>(p.W + (size_t)t * p.K)[c];
            const float f = p.rows[m].y;
            const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __builtin_fmaf(f, bf16_bits_to_float(u[i] & 0xffffu), v[2 * i]);
                v[2 * i + 1] = __builtin_fmaf(f, __builtin_bit_cast(float, u[i] & 0xffff0000u), v[2 * i + 1]);
            }
            o = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        }
        reinterpret_cast<uint4*>(p.dH + (size_t)m * p.K)[c] = o;
    }
}

constexpr size_t kLossPiece = (size_t)256 << 20;         // bytes of a piece's exponentials
constexpr size_t kLossPart = (size_t)64 << 20;           // bytes of the second product's partial sums beyond one of each

struct LossPlan {
    int tiles, VP, rows, splits, words;                  // rows: tokens a piece
    size_t stats0, zt0, rows0, part0, P0, bytes;
};
LossPlan loss_plan(int M, int V, int K, bool grad) {
    LossPlan l{};
    l.tiles = (V + TILE - 1) / TILE;
    l.VP = l.tiles * TILE;
    const size_t fits = std::min(kLossPiece / ((size_t)l.VP * 2), kLossPiece / ((size_t)K * 4)) / TILE * TILE;
    l.rows = grad ? (int)std::min<size_t>(M, std::max<size_t>(fits, TILE)) : M;
    l.rows = std::min(l.rows, std::max((1 << 24) / l.tiles, TILE));      // (statistics of a piece: 128 MB)
    const long long out_tiles = (long long)((l.rows + TILE - 1) / TILE) * ((K + TILE - 1) / TILE);
    const size_t out_bytes = (size_t)l.rows * K * 4;
    const int steps = l.VP / DEPTH;
    long long splits = std::max<long long>(1, std::min<long long>(device_compute_units() / out_tiles, steps / 8));
    splits = std::max<long long>(1, std::min<long long>(splits, (long long)(kLossPart / out_bytes) + 1));
    l.words = (int)((steps + splits - 1) / splits) * DEPTH;
    l.splits = (l.VP + l.words - 1) / l.words;
    auto take = [&](size_t n) { const size_t at = l.bytes; l.bytes += (n + 255) / 256 * 256; return at; };
    l.stats0 = take((size_t)l.rows * l.tiles * sizeof(LossStat));
    l.zt0 = take((size_t)l.rows * 4);
    if (grad) {
        l.rows0 = take((size_t)l.rows * 8);
        l.part0 = take((size_t)l.splits * out_bytes);
        l.P0 = take((size_t)l.rows * l.VP * 2);
    }
    return l;
}

}  // namespace

size_t vocab_loss_workspace_bytes(int M, int V, int K, bool grad) { return loss_plan(M, V, K, grad).bytes; }

hipError_t launch_vocab_loss(const VocabLossArgs& a, hipStream_t st) {
    static const hipError_t attr[2] = {hipFuncSetAttribute(reinterpret_cast<const void*>(loss_logits_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, SMEM),
                                       hipFuncSetAttribute(reinterpret_cast<const void*>(loss_grad_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, SMEM)};
    if (attr[0] != hipSuccess) return attr[0];
    if (attr[1] != hipSuccess) return attr[1];
    const bool grad = a.dH != nullptr;
    const LossPlan l = loss_plan(a.M, a.V, a.K, grad);
    uint8_t* ws = static_cast<uint8_t*>(a.workspace);
    for (int m0 = 0; m0 < a.M; m0 += l.rows) {
        LossParams p{};
        p.M = std::min(l.rows, a.M - m0); p.V = a.V; p.K = a.K; p.VP = l.VP; p.tiles = l.tiles;
        p.h = a.h + (size_t)m0 * a.K; p.W = a.W; p.targets = a.targets + m0; p.weights = a.weights ? a.weights + m0 : nullptr;
        p.loss = a.loss + m0; p.lse = a.lse ? a.lse + m0 : nullptr; p.dH = grad ? a.dH + (size_t)m0 * a.K : nullptr;
        p.stats = reinterpret_cast<LossStat*>(ws + l.stats0); p.zt = reinterpret_cast<float*>(ws + l.zt0);
        if (grad) {
            p.rows = reinterpret_cast<float2*>(ws + l.rows0); p.part = reinterpret_cast<float*>(ws + l.part0); p.P = reinterpret_cast<uint16_t*>(ws + l.P0);
            p.splits = l.splits; p.words_per_split = l.words;
        }
        const int tiles_m = (p.M + TILE - 1) / TILE;
        loss_logits_kernel<<<dim3((unsigned)(tiles_m * l.tiles)), dim3(THREADS), SMEM, st>>>(p);
        loss_rows_kernel<<<dim3((unsigned)((p.M + 3) / 4)), dim3(256), 0, st>>>(p);
        hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (!grad) continue;
        loss_scale_kernel<<<dim3((unsigned)p.M * (unsigned)((l.VP / 8 + 1023) / 1024)), dim3(256), 0, st>>>(p);
        loss_grad_kernel<<<dim3((unsigned)(tiles_m * ((a.K + TILE - 1) / TILE) * l.splits)), dim3(THREADS), SMEM, st>>>(p);
        loss_sum_kernel<<<dim3((unsigned)std::min<long long>(((long long)p.M * (a.K / 8) + 255) / 256, 16 * device_compute_units())), dim3(256), 0, st>>>(p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace lowra
