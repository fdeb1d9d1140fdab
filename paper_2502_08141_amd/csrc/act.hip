// Activation's backward pass with the bias gradient (a gradient that reaches a linear layer's output from outside, Sec. 2.1):
//   dZ = dY mul act'(z)      dmul = dY act(z)      db[n] = sum over the tokens of dZ[m,n], before it is rounded
//
// Memory bound: every operand is read or written once, 16 bytes per lane.  A thread keeps eight columns and walks down the
// tokens, so that their sums stay in registers; the wavefronts of a workgroup meet in LDS, workgroups in the workspace, both
// added in a fixed order.  Bias gradient alone of 4096 x 11008 (a read of 90 MB): 18.2 us, 4.9 TB/s; gelu of
// 4096 x 4096 (101 MB) 22.7 us, 4.4 TB/s; of 777 x 4096 (19 MB) 9.7 us, latency and the activations on half of the units.
#include <algorithm>

#include "epilogue.h"
#include "gemm_common.h"

namespace lowra {

namespace {

// Eight columns to a thread, LANES threads side by side; the rest of the workgroup has token rows of its own.  64 lanes read whole
// rows, and the tokens are cut between workgroups whose sums a second launch adds up.  8 and 4 lanes (64 and 32 columns, 1024
// threads) leave all tokens to one workgroup and need no second launch, but few units work.  Both ways, with bias gradient:
//   gelu, 4096 columns, 24, 400, 777, 1000 tokens     9.5, 9.6, 10.2, 10.7 us in chunks; 8 lanes 6.3, 7.2, 12.2, 14.8; 4 lanes 6.3, 6.7, 9.9, 11.5
//   gelu, 11008 columns, 160, 400, 777, 1200 tokens   9.7, 12.0, 15.0, 19.2 in chunks; 8 lanes 6.4, 9.8, 14.4, 19.1; 4 lanes 7.9, 13.2, 19.7, 27.6
//   the sums alone, 1200 tokens of 1024, 4096, 11008 columns  7.3, 7.2, 10.5 in chunks; 8 lanes 5.2, 5.5, 7.8; of 20000 13.3 and 15.3
//     (more strips than units); 3000 tokens 7.4, 10.2, 15.7; 7.7, 9.3, 14.0; 6000 tokens 8.8, 13.8, 29.7; 15.3, 15.8, 27.6
constexpr int act_threads(int LANES) { return LANES == 64 ? 256 : 1024; }
int act_lanes(int M, int N, bool sums_alone) {
    const int units = device_compute_units();
    const int most = N > 64 * units ? 400 : sums_alone ? 2048 + N / 4 : 800;
    if (M > most || N > 1 << 22) return 64;                         // (a launch has less than 2^32 threads)
    return !sums_alone && N <= 32 * units ? 4 : 8;
}

// Token rows per workgroup: enough workgroups to fill the chip several times, about sixteen rows each (777 x 4096, gelu: 9.5 us; eight
// 9.55, thirty-two 10.4).
int act_rows(int M, int N, int lanes) {
    if (lanes < 64) return M;
    const int strips = (N + 511) / 512, want = 8 * device_compute_units();
    const int chunks = std::max(1, std::min((M + 15) / 16, (want + strips - 1) / strips));
    return (M + chunks - 1) / chunks;
}

template <int LANES>
__global__ __launch_bounds__(act_threads(LANES)) void act_bwd_kernel(int M, int N, int rows, BwdEpi e, const uint16_t* dY, uint16_t* dZ, float* sums) {
    constexpr int THREADS = act_threads(LANES), WAVES = THREADS / 64, STEP = THREADS / LANES;
    __shared__ float red[WAVES][8][LANES];
    const int lane = threadIdx.x % LANES, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * (8 * LANES) + lane * 8;
    const int m0 = blockIdx.y * rows, m1 = min(m0 + rows, M);
    float total[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (col < N) {                                                  // N is a multiple of 8
        with_act(e.act, [&](auto A) {
            constexpr int ACT = decltype(A)::value;
            constexpr int U = 4;                                    // rows whose operands are asked for together
            for (int m = m0 + threadIdx.x / LANES; m < m1; m += U * STEP) {
                Bf16Run<8> g[U];
                EpiRun<BwdEpi, 8> r[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (m + u * STEP < m1) {
                        const size_t at = (size_t)(m + u * STEP) * N + col;
                        load_run<8>(dY + at, g[u]);
                        epi_load<8>(e, at, r[u]);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (m + u * STEP < m1) {
                        const size_t at = (size_t)(m + u * STEP) * N + col;
                        float v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = g[u][i];
                        epi_apply<ACT, 8>(e, v, v, r[u], [&](const float (&w)[8]) __attribute__((always_inline)) { store_run<8>(e.dmul + at, w); });
                        if (dZ) store_run<8>(dZ + at, v);
#pragma unroll
                        for (int i = 0; i < 8; ++i) total[i] += v[i];
                    }
            }
        });
    }
    if (!sums) return;                                              // uniform
#pragma unroll
    for (int s = LANES; s < 64; s *= 2)
#pragma unroll
        for (int i = 0; i < 8; ++i) total[i] += __shfl_xor(total[i], s);
    if ((threadIdx.x & 63) < LANES) {
#pragma unroll
        for (int i = 0; i < 8; ++i) red[wave][i][lane] = total[i];
    }
    __syncthreads();
    for (int o = threadIdx.x; o < 8 * LANES; o += THREADS) {
        const int c = blockIdx.x * (8 * LANES) + o;
        float v = red[0][o & 7][o >> 3];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += red[w][o & 7][o >> 3];
        if (c < N) sums[(size_t)blockIdx.y * N + c] = v;
    }
}

// 32 columns per workgroup, the chunks dealt to eight groups of threads, each with up to eight loads under way
__global__ __launch_bounds__(256) void act_sum_kernel(const float* __restrict__ sums, int chunks, int N, float* __restrict__ db) {
    __shared__ float red[8][32];
    const int c = threadIdx.x & 31, grp = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float v = 0.0f;
    for (int k = grp; k < chunks; k += 64) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = sums[(size_t)min(k + 8 * u, chunks - 1) * N + min(col, N - 1)];
#pragma unroll
        for (int u = 0; u < 8; ++u) v += k + 8 * u < chunks ? x[u] : 0.0f;
    }
    red[grp][c] = v;
    __syncthreads();
    if (grp != 0 || col >= N) return;
    for (int g = 1; g < 8; ++g) v += red[g][c];
    db[col] = v;
}

}  // namespace

size_t act_bwd_workspace_bytes(int M, int N) {
    size_t most = 0;
    for (const bool sums_alone : {false, true}) {
        const int rows = act_rows(M, N, act_lanes(M, N, sums_alone));
        if (rows < M) most = (size_t)((M + rows - 1) / rows) * N * sizeof(float);
    }
    return most;
}

hipError_t launch_act_bwd(int M, int N, const BwdEpi& e, const uint16_t* dY, uint16_t* dZ, float* db, void* workspace, hipStream_t st) {
    const int lanes = db ? act_lanes(M, N, !dZ && !e.dmul) : 64, rows = act_rows(M, N, lanes), chunks = (M + rows - 1) / rows;
    float* sums = !db ? nullptr : chunks > 1 ? static_cast<float*>(workspace) : db;
    const dim3 grid((unsigned)((N + 8 * lanes - 1) / (8 * lanes)), (unsigned)chunks), block(act_threads(lanes));
    if (lanes == 64) act_bwd_kernel<64><<<grid, block, 0, st>>>(M, N, rows, e, dY, dZ, sums);
    else if (lanes == 8) act_bwd_kernel<8><<<grid, block, 0, st>>>(M, N, rows, e, dY, dZ, sums);
    else act_bwd_kernel<4><<<grid, block, 0, st>>>(M, N, rows, e, dY, dZ, sums);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || !db || chunks == 1) return err;
    act_sum_kernel<<<dim3((unsigned)((N + 31) / 32)), dim3(256), 0, st>>>(sums, chunks, N, db);
    return hipGetLastError();
}

}  // namespace lowra
