// Layer and root-mean-square norm with their way back (the norms around a fine-tuned layer, Sec. 2.1):
//   forward    xh = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)  (rms: mean = 0);   y = xh weight + bias
//   backward   g = dY weight;   dX = rstd (g - mean(g) - xh mean(g xh)) + residual  (rms: without mean(g))
//              dweight[n] = sum over the tokens of dY xh;   dbias[n] = sum of dY
//
// Memory bound: every operand is read or written once, 16 bytes per lane.  A row stays in the registers of the threads that share it, so
// that the deviations are squared about the mean itself; the backward pass forms mean and rstd again from the x that it reads
// anyway, which costs it one reduction and saves the forward pass two arrays.  A thread keeps its columns from row to row and with them their
// sums; workgroups meet in the workspace, added in a fixed order.  Graph replays: 4096 x 4096 forward 13.1 us (5.1 TB/s), rms backward with residual and dweight
// 28.4 (4.7), dX alone 19.6; layer backward with both sums 30.4 and with residual 35.4; 777 x 1024 3.3 and 6.9, a launch each and one more for the sums.
#include <algorithm>

#include "gemm_common.h"
#include "step.h"

namespace lowra {

namespace {

__device__ __forceinline__ void unpack8(uint4 q, float (&v)[8]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = bf16_bits_to_float(w[i] & 0xffffu);
        v[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&v)[8]) {
    return make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
__device__ __forceinline__ float wave_sum_f32(float x) {
    auto add = [&](auto C_) __attribute__((always_inline)) {
        const int v = __builtin_bit_cast(int, x);
        x += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(v, v, decltype(C_)::value, 0xf, 0xf, true));
    };
    add(std::integral_constant<int, 0xB1>{});      // quad_perm [1,0,3,2]
    add(std::integral_constant<int, 0x4E>{});      // quad_perm [2,3,0,1]
    add(std::integral_constant<int, 0x124>{});     // row_ror:4
    add(std::integral_constant<int, 0x128>{});     // row_ror:8
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    return x;
}
// The sums of S values over the W wavefronts that share a row; every thread gets them.  `red` has two halves, taken in turn, so that one
// barrier a sum is enough.
template <int W, int S>
__device__ __forceinline__ void row_sums(float (&v)[S], float (*red)[W][4], int& turn) {
#pragma unroll
    for (int s = 0; s < S; ++s) v[s] = wave_sum_f32(v[s]);
    if constexpr (W > 1) {
        const int wave = (threadIdx.x >> 6) % W;                  // of the row
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int s = 0; s < S; ++s) red[turn][wave][s] = v[s];
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < S; ++s) {
            v[s] = red[turn][0][s];
#pragma unroll
            for (int w = 1; w < W; ++w) v[s] += red[turn][w][s];
        }
        turn ^= 1;
    }
}

constexpr int norm_threads(int W) { return W == 1 ? 256 : 64 * W; }      // W wavefronts share a row; one that has it alone: four rows

// C runs of eight columns a thread
template <int W, int C, bool RMS>
__global__ __launch_bounds__(norm_threads(W)) void norm_fwd_kernel(NormArgs a) {
    constexpr int ROWS = W == 1 ? 4 : 1;
    __shared__ float red[2][W][4];
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x, first = (int)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0), step = (int)gridDim.x * ROWS;
    const int runs = a.N >> 3;
    const float inv = 1.0f / (float)a.N;
    int turn = 0;
    for (int row = first; row < a.M; row += step) {               // (once, but for more rows than a launch has workgroups)
        const size_t at = (size_t)row * a.N;
        float v[C][8], sum[1] = {0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            unpack8(run < runs ? reinterpret_cast<const uint4*>(a.x + at)[run] : zero4(), v[c]);
        }
        float mean = 0.0f;
        if (!RMS) {
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] += v[c][i];
            row_sums<W>(sum, red, turn);
            mean = sum[0] * inv;
        }
        sum[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[c][i] -= mean;
                sum[0] += c * (64 * W) + t < runs ? v[c][i] * v[c][i] : 0.0f;
            }
        row_sums<W>(sum, red, turn);
        const float rstd = 1.0f / sqrtf(sum[0] * inv + a.eps);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= runs) continue;
            float w[8], b[8];
            if (a.weight) unpack8(reinterpret_cast<const uint4*>(a.weight)[run], w);
            if (a.bias) unpack8(reinterpret_cast<const uint4*>(a.bias)[run], b);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float y = v[c][i] * rstd;
                if (a.weight) y *= w[i];
                v[c][i] = a.bias ? y + b[i] : y;
            }
            reinterpret_cast<uint4*>(a.y + at)[run] = pack8(v[c]);
        }
    }
}

// A workgroup has G rows side by side, each W wavefronts', and takes rows in turn; sums: [dweight, dbias][workgroup][N], or null.  BIAS: dbias is asked for.  (At most
// 128 registers, so that two workgroups share a unit: with bias gradient 4096 x 4096 36 -> 31.7 us; a row's values stay unpacked, which saves 1 to 4 %.)
template <int W, int C, int G, bool RMS, bool BIAS>
__global__ __launch_bounds__(64 * W * G, C <= 2 ? 4 : 2) void norm_bwd_kernel(NormArgs a, float* sums) {
    __shared__ float red_of[G][2][W][4];
    extern __shared__ __align__(16) float join[];                 // [G][N]
    const int t = threadIdx.x % (64 * W), group = threadIdx.x / (64 * W), step = (int)gridDim.x * G;
    float(*red)[W][4] = red_of[group];
    const float inv = 1.0f / (float)a.N;
    int turn = 0;
    float dw[C][8], db[BIAS ? C : 1][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            dw[c][i] = 0.0f;
            if (BIAS) db[BIAS ? c : 0][i] = 0.0f;
        }
    for (int first = (int)blockIdx.x * G; first < a.M; first += step) {              // (uniform: the sums of a row of several wavefronts meet at barriers)
        const int runs = first + group < a.M ? a.N >> 3 : 0;
        const size_t at = (size_t)min(first + group, a.M - 1) * a.N;
        // (asking for the next row's operands here as well took longer: 16384 x 1024 26 -> 30 us, 4096 x 4096 31 -> 37 to 43)
        uint4 xq[C], gq[C], rq[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            xq[c] = run < runs ? reinterpret_cast<const uint4*>(a.x + at)[run] : zero4();
            gq[c] = run < runs ? reinterpret_cast<const uint4*>(a.dY + at)[run] : zero4();
        }
        if (a.residual) {
#pragma unroll
            for (int c = 0; c < C; ++c) rq[c] = c * (64 * W) + t < runs ? reinterpret_cast<const uint4*>(a.residual + at)[c * (64 * W) + t] : zero4();
        }
        float d[C][8], g[C][8], mean = 0.0f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            unpack8(xq[c], d[c]);
            unpack8(gq[c], g[c]);
        }
        if (!RMS) {
            float sum[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] += d[c][i];
            row_sums<W>(sum, red, turn);
            mean = sum[0] * inv;
        }
        // sums of d^2, g w d and g w, d = x - mean, g = dY
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= runs) continue;
            float w[8];
            if (a.weight) unpack8(reinterpret_cast<const uint4*>(a.weight)[run], w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[c][i] -= mean;
                const float gw = a.weight ? g[c][i] * w[i] : g[c][i];
                sum[0] = __builtin_fmaf(d[c][i], d[c][i], sum[0]);
                sum[1] = __builtin_fmaf(gw, d[c][i], sum[1]);
                if (!RMS) sum[2] += gw;
            }
        }
        row_sums<W>(sum, red, turn);
        // dX = rstd (g w - mean(g w)) - d rstd along
        const float rstd = 1.0f / sqrtf(sum[0] * inv + a.eps), along = sum[1] * inv * rstd * rstd * rstd, gmean = RMS ? 0.0f : sum[2] * inv;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= runs) continue;
            float w[8], r[8], out[8];
            if (a.weight) unpack8(reinterpret_cast<const uint4*>(a.weight)[run], w);
            if (a.residual) unpack8(rq[c], r);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float gw = a.weight ? g[c][i] * w[i] : g[c][i];
                dw[c][i] = __builtin_fmaf(g[c][i], d[c][i] * rstd, dw[c][i]);
                if (BIAS) db[BIAS ? c : 0][i] += g[c][i];
                out[i] = __builtin_fmaf(-along, d[c][i], rstd * (RMS ? gw : gw - gmean));
                if (a.residual) out[i] += r[i];
            }
            if (a.dX) reinterpret_cast<uint4*>(a.dX + at)[run] = pack8(out);
        }
    }
    if (!sums) return;                                            // uniform
#pragma unroll
    for (int half = 0; half < (BIAS ? 2 : 1); ++half) {
        float* out = sums + ((size_t)half * gridDim.x + blockIdx.x) * a.N;
        float* to = G > 1 ? join + group * a.N : out;
        if (G > 1 && half) __syncthreads();
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= a.N >> 3) continue;
            const float(&v)[8] = half ? db[BIAS ? c : 0] : dw[c];
            float4* p = reinterpret_cast<float4*>(to) + 2 * run;
            p[0] = make_float4(v[0], v[1], v[2], v[3]);
            p[1] = make_float4(v[4], v[5], v[6], v[7]);
        }
        if (G == 1) continue;
        __syncthreads();
        for (int q = threadIdx.x; q < a.N / 4; q += 64 * W * G) {
            float4 s = reinterpret_cast<const float4*>(join)[q];
#pragma unroll
            for (int r = 1; r < G; ++r) {
                const float4 u = reinterpret_cast<const float4*>(join + r * a.N)[q];
                s.x += u.x; s.y += u.y; s.z += u.z; s.w += u.w;
            }
            reinterpret_cast<float4*>(out)[q] = s;
        }
    }
}

// 32 columns a workgroup, a cache line of each chunk, the chunks dealt to 32 groups of threads, each with up to eight loads under way; blockIdx.y: dweight, dbias
// (4096 x 4096 rms with residual, both launches: 29.0 us; 16 columns 30.1, 64 29.6)
__global__ __launch_bounds__(1024) void norm_sum_kernel(const float* __restrict__ sums, int chunks, int N, float* dweight, float* dbias) {
    __shared__ float red[32][33];
    float* out = blockIdx.y ? dbias : dweight;
    if (!out) return;                                             // uniform
    const float* in = sums + (size_t)blockIdx.y * chunks * N;
    const int c = threadIdx.x & 31, grp = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float v = 0.0f;
    for (int k = grp; k < chunks; k += 256) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = in[(size_t)min(k + 32 * u, chunks - 1) * N + min(col, N - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) v += k + 32 * u < chunks ? x[u] : 0.0f;
    }
    red[grp][c] = v;
    __syncthreads();
    if (threadIdx.x >= 64) return;
    // a wavefront adds up the 32 groups, half of them a lane
    const int half = threadIdx.x >> 5;
    v = red[16 * half][c];
#pragma unroll
    for (int g = 1; g < 16; ++g) v += red[16 * half + g][c];
    v += __shfl_xor(v, 32);
    if (half == 0 && col < N) out[col] = v;
}

// Calls f with the wavefronts that share a row and the runs of eight columns a thread
template <class F>
hipError_t with_shape(int N, F f) {
    const int runs = N / 8;
    using std::integral_constant;
    if (runs <= 64) return f(integral_constant<int, 1>{}, integral_constant<int, 1>{});
    if (runs <= 128) return f(integral_constant<int, 1>{}, integral_constant<int, 2>{});
    if (runs <= 256) return f(integral_constant<int, 4>{}, integral_constant<int, 1>{});
    if (runs <= 512) return f(integral_constant<int, 4>{}, integral_constant<int, 2>{});
    if (runs <= 1024) return f(integral_constant<int, 8>{}, integral_constant<int, 2>{});
    return f(integral_constant<int, 16>{}, integral_constant<int, 2>{});
}
template <int W_, int C_, int G_> struct BwdShape { static constexpr int W = W_, C = C_, G = G_; };
// Two runs a thread and two workgroups of 512 threads a unit, so that few partial sums are left (4096 x 4096, rms, with residual: 44 us with one row to a workgroup
// and 1024 of those, 28.8 now; a wavefront to a row 35).  Up to 1024 columns few rows are done sooner with two wavefronts each (64 and 777 rows of 1024 7.1
// and 7.7 -> 6.2 and 7.2 us), many with one (16384: 28.8 -> 26.4).
template <class F>
auto with_bwd_shape(int M, int N, F f) {
    const int runs = N / 8;
    if (runs <= 64) return f(BwdShape<1, 1, 8>{});
    if (runs <= 128 && M > 8192) return f(BwdShape<1, 2, 8>{});
    if (runs <= 128) return f(BwdShape<2, 1, 4>{});
    if (runs <= 256) return f(BwdShape<2, 2, 4>{});
    if (runs <= 512) return f(BwdShape<4, 2, 2>{});
    if (runs <= 1024) return f(BwdShape<8, 2, 1>{});
    return f(BwdShape<8, 4, 1>{});
}
int norm_blocks(int M, int N) {
    return with_bwd_shape(M, N, [&](auto S_) {
        constexpr int G = decltype(S_)::G;
        return std::min((M + G - 1) / G, 2 * device_compute_units());
    });
}

}  // namespace

size_t norm_bwd_workspace_bytes(int M, int N) { return (size_t)norm_blocks(M, N) * 2 * N * sizeof(float); }

hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t st) {
    return with_shape(a.N, [&](auto W_, auto C_) {
        constexpr int W = decltype(W_)::value, C = decltype(C_)::value, ROWS = W == 1 ? 4 : 1;
        const dim3 grid((unsigned)std::min((a.M + ROWS - 1) / ROWS, 1 << 20)), block(norm_threads(W));
        if (a.rms) norm_fwd_kernel<W, C, true><<<grid, block, 0, st>>>(a);
        else norm_fwd_kernel<W, C, false><<<grid, block, 0, st>>>(a);
        return hipGetLastError();
    });
}

hipError_t launch_norm_bwd(const NormArgs& a, float* dweight, float* dbias, void* workspace, hipStream_t st) {
    const int blocks = norm_blocks(a.M, a.N);
    float* sums = dweight || dbias ? static_cast<float*>(workspace) : nullptr;
    const hipError_t e = with_bwd_shape(a.M, a.N, [&](auto S_) {
        constexpr int W = decltype(S_)::W, C = decltype(S_)::C, G = decltype(S_)::G;
        const int smem = G > 1 && sums ? G * a.N * (int)sizeof(float) : 0;          // (N G <= 8192 wherever G > 1: 32 KB at most)
        auto go = [&](auto kernel) {
            kernel<<<dim3((unsigned)blocks), dim3(64 * W * G), smem, st>>>(a, sums);
            return hipGetLastError();
        };
        if (dbias) return a.rms ? go(norm_bwd_kernel<W, C, G, true, true>) : go(norm_bwd_kernel<W, C, G, false, true>);
        return a.rms ? go(norm_bwd_kernel<W, C, G, true, false>) : go(norm_bwd_kernel<W, C, G, false, false>);
    });
    if (e != hipSuccess || !sums) return e;
    norm_sum_kernel<<<dim3((unsigned)((a.N + 31) / 32), dbias ? 2u : 1u), dim3(1024), 0, st>>>(sums, blocks, a.N, dweight, dbias);
    return hipGetLastError();
}

}  // namespace lowra
