// Activation's backward pass with the bias gradient (a gradient that reaches a linear layer's output from outside, Sec. 2.1):
//   dZ = dY mul act'(z)      dmul = dY act(z)      db[n] = sum over the tokens of dZ[m,n], before it is rounded
//
// Memory bound: every operand is read or written once, 16 bytes per lane.  A thread keeps eight columns and walks down the
// tokens, so that their sums stay in registers; the wavefronts of a workgroup meet in LDS, workgroups in the workspace, both
// added in a fixed order.  Bias gradient alone of 4096 x 11008 (a read of 90 MB): 17.2 us, 5.2 TB/s, and 2.3 to add up the
// chunks; gelu of 777 x 4096 (19 MB): 7.4 us and 2.3, between launch latency and bandwidth.
#include <algorithm>

#include "epilogue.h"
#include "gemm_common.h"

namespace lowra {

namespace {

constexpr int ACT_COLS = 512;            // columns per workgroup: 64 lanes x 8
constexpr int ACT_WAVES = 4;
static_assert(kActMaxSize <= 1 << 30, "rows and columns are rounded up in int");

// Token rows per workgroup: enough workgroups to fill the chip several times, about sixteen rows each (777 x 4096, gelu: 9.5 us; eight
// 9.55, thirty-two 10.4).  Few tokens are one workgroup's, which saves the launch that adds up the chunks: 24 x 4096, gelu, 9.4 -> 6.2;
// 64 are too many for it (9.1 -> 10.3).
int act_rows(int M, int N) {
    if (M <= 48) return M;
    const int strips = (N + ACT_COLS - 1) / ACT_COLS, want = 8 * device_compute_units();
    const int chunks = std::max(1, std::min((M + 15) / 16, (want + strips - 1) / strips));
    return (M + chunks - 1) / chunks;
}
int act_chunks(int M, int N) { const int rows = act_rows(M, N); return rows ? (M + rows - 1) / rows : 0; }

__global__ __launch_bounds__(ACT_WAVES * 64) void act_bwd_kernel(int M, int N, int rows, BwdEpi e, const uint16_t* dY, uint16_t* dZ, float* sums) {
    __shared__ float red[ACT_WAVES][8][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int col = blockIdx.x * ACT_COLS + lane * 8;
    const int m0 = blockIdx.y * rows, m1 = min(m0 + rows, M);
    float total[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
    if (col < N) {                                                  // N is a multiple of 8
        with_act(e.act, [&](auto A) {
            constexpr int ACT = decltype(A)::value;
            constexpr int U = 4;                                    // rows whose operands are asked for together
            for (int m = m0 + wave; m < m1; m += U * ACT_WAVES) {
                Bf16Run<8> g[U];
                EpiRun<BwdEpi, 8> r[U];
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (m + u * ACT_WAVES < m1) {
                        const size_t at = (size_t)(m + u * ACT_WAVES) * N + col;
                        load_run<8>(dY + at, g[u]);
                        epi_load<8>(e, at, r[u]);
                    }
#pragma unroll
                for (int u = 0; u < U; ++u)
                    if (m + u * ACT_WAVES < m1) {
                        const size_t at = (size_t)(m + u * ACT_WAVES) * N + col;
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
    for (int i = 0; i < 8; ++i) red[wave][i][lane] = total[i];
    __syncthreads();
    for (int o = threadIdx.x; o < ACT_COLS; o += ACT_WAVES * 64) {
        const int c = blockIdx.x * ACT_COLS + o;
        if (c < N) sums[(size_t)blockIdx.y * N + c] = ((red[0][o & 7][o >> 3] + red[1][o & 7][o >> 3]) + red[2][o & 7][o >> 3]) + red[3][o & 7][o >> 3];
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
    const int chunks = act_chunks(M, N);
    return chunks > 1 ? (size_t)chunks * N * sizeof(float) : 0;
}

hipError_t launch_act_bwd(int M, int N, const BwdEpi& e, const uint16_t* dY, uint16_t* dZ, float* db, void* workspace, hipStream_t st) {
    const int rows = act_rows(M, N), chunks = act_chunks(M, N);
    float* sums = !db ? nullptr : chunks > 1 ? static_cast<float*>(workspace) : db;
    act_bwd_kernel<<<dim3((unsigned)((N + ACT_COLS - 1) / ACT_COLS), (unsigned)chunks), dim3(ACT_WAVES * 64), 0, st>>>(M, N, rows, e, dY, dZ, sums);
    hipError_t err = hipGetLastError();
    if (err != hipSuccess || !db || chunks == 1) return err;
    act_sum_kernel<<<dim3((unsigned)((N + 31) / 32)), dim3(256), 0, st>>>(sums, chunks, N, db);
    return hipGetLastError();
}

}  // namespace lowra
