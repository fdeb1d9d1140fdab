// Layer and root-mean-square norm with their way back (the norms around a fine-tuned layer, Sec. 2.1):
//   forward    xh = (x - mean) rstd,  rstd = 1 / sqrt(mean((x - mean)^2) + eps)  (rms: mean = 0);   y = xh weight + bias
//   backward   g = dY weight;   dX = rstd (g - mean(g) - xh mean(g xh)) + residual  (rms: without mean(g))
//              dweight[n] = sum over the tokens of dY xh;   dbias[n] = sum of dY
//
// Memory bound: every operand is read or written once, 16 bytes per lane.  A row stays in the registers of the threads that share it, so
// that the deviations are squared about the mean itself; the backward pass forms mean and rstd again from the x that it reads
// anyway, which costs it one reduction and saves the forward pass two arrays.  A thread keeps its columns from row to row and with them their
// sums; workgroups meet in the workspace, added in a fixed order.
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
        const int wave = threadIdx.x >> 6;
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

// Workgroups take rows in turn; sums: [workgroup][2][N] (dweight, dbias), or null
template <int W, int C, bool RMS>
__global__ __launch_bounds__(norm_threads(W)) void norm_bwd_kernel(NormArgs a, float* sums) {
    constexpr int ROWS = W == 1 ? 4 : 1;
    __shared__ float red[2][W][4];
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x, first = (int)blockIdx.x * ROWS + (W == 1 ? threadIdx.x >> 6 : 0), step = (int)gridDim.x * ROWS;
    const int runs = a.N >> 3;
    const float inv = 1.0f / (float)a.N;
    int turn = 0;
    float dw[C][8], db[C][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) dw[c][i] = db[c][i] = 0.0f;
    for (int row = first; row < a.M; row += step) {
        const size_t at = (size_t)row * a.N;
        uint4 xq[C], gq[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            xq[c] = run < runs ? reinterpret_cast<const uint4*>(a.x + at)[run] : zero4();
            gq[c] = run < runs ? reinterpret_cast<const uint4*>(a.dY + at)[run] : zero4();
        }
        float mean = 0.0f;
        if (!RMS) {
            float sum[1] = {0.0f};
#pragma unroll
            for (int c = 0; c < C; ++c) {
                float v[8];
                unpack8(xq[c], v);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum[0] += v[i];
            }
            row_sums<W>(sum, red, turn);
            mean = sum[0] * inv;
        }
        // sums of d^2, g d and g, d = x - mean, g = dY weight
        float sum[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= runs) continue;
            float d[8], g[8], w[8];
            unpack8(xq[c], d);
            unpack8(gq[c], g);
            if (a.weight) unpack8(reinterpret_cast<const uint4*>(a.weight)[run], w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] -= mean;
                if (a.weight) g[i] *= w[i];
                sum[0] += d[i] * d[i];
                sum[1] += g[i] * d[i];
                sum[2] += g[i];
            }
        }
        row_sums<W>(sum, red, turn);
        const float rstd = 1.0f / sqrtf(sum[0] * inv + a.eps), along = sum[1] * inv * rstd * rstd, gmean = RMS ? 0.0f : sum[2] * inv;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= runs) continue;
            float d[8], g[8], w[8], r[8];
            unpack8(xq[c], d);
            unpack8(gq[c], g);
            if (a.weight) unpack8(reinterpret_cast<const uint4*>(a.weight)[run], w);
            if (a.residual) unpack8(reinterpret_cast<const uint4*>(a.residual + at)[run], r);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[i] -= mean;
                dw[c][i] += g[i] * (d[i] * rstd);
                db[c][i] += g[i];
                if (a.weight) g[i] *= w[i];
                g[i] = rstd * (g[i] - gmean - d[i] * along);
                if (a.residual) g[i] += r[i];
            }
            if (a.dX) reinterpret_cast<uint4*>(a.dX + at)[run] = pack8(g);
        }
    }
    if (!sums) return;                                            // uniform
    float* out = sums + (size_t)blockIdx.x * 2 * a.N;
    if constexpr (W == 1) {
        __shared__ float join[4][64][8];
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                __syncthreads();
#pragma unroll
                for (int i = 0; i < 8; ++i) join[wave][t][i] = half ? db[c][i] : dw[c][i];
                __syncthreads();
                for (int o = threadIdx.x; o < 512; o += 256) {
                    const int col = c * 512 + o;
                    if (col < a.N) out[(size_t)half * a.N + col] = ((join[0][o >> 3][o & 7] + join[1][o >> 3][o & 7]) + join[2][o >> 3][o & 7]) + join[3][o >> 3][o & 7];
                }
            }
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int run = c * (64 * W) + t;
            if (run >= runs) continue;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                float4* p = reinterpret_cast<float4*>(out + (size_t)half * a.N) + 2 * run;
                const float(&v)[8] = half ? db[c] : dw[c];
                p[0] = make_float4(v[0], v[1], v[2], v[3]);
                p[1] = make_float4(v[4], v[5], v[6], v[7]);
            }
        }
    }
}

// 32 columns a workgroup, the chunks dealt to eight groups of threads, each with up to eight loads under way; blockIdx.y: dweight, dbias
__global__ __launch_bounds__(256) void norm_sum_kernel(const float* __restrict__ sums, int chunks, int N, float* dweight, float* dbias) {
    __shared__ float red[8][32];
    float* out = blockIdx.y ? dbias : dweight;
    if (!out) return;                                             // uniform
    const float* in = sums + (size_t)blockIdx.y * N;
    const int c = threadIdx.x & 31, grp = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float v = 0.0f;
    for (int k = grp; k < chunks; k += 64) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = in[(size_t)min(k + 8 * u, chunks - 1) * 2 * N + min(col, N - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) v += k + 8 * u < chunks ? x[u] : 0.0f;
    }
    red[grp][c] = v;
    __syncthreads();
    if (grp != 0 || col >= N) return;
    for (int g = 1; g < 8; ++g) v += red[g][c];
    out[col] = v;
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
int norm_blocks(int M, int N) {
    const int rows = N <= 1024 ? 4 : 1;
    return std::min((M + rows - 1) / rows, (N <= 4096 ? 4 : N <= 8192 ? 2 : 1) * device_compute_units());
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
    const hipError_t e = with_shape(a.N, [&](auto W_, auto C_) {
        constexpr int W = decltype(W_)::value, C = decltype(C_)::value;
        if (a.rms) norm_bwd_kernel<W, C, true><<<dim3((unsigned)blocks), dim3(norm_threads(W)), 0, st>>>(a, sums);
        else norm_bwd_kernel<W, C, false><<<dim3((unsigned)blocks), dim3(norm_threads(W)), 0, st>>>(a, sums);
        return hipGetLastError();
    });
    if (e != hipSuccess || !sums) return e;
    norm_sum_kernel<<<dim3((unsigned)((a.N + 31) / 32), 2), dim3(256), 0, st>>>(sums, blocks, a.N, dweight, dbias);
    return hipGetLastError();
}

}  // namespace lowra
