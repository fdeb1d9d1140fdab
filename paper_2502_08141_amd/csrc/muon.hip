// The optimiser step on the adapters (Sec. 2.1: only A and B are trained) with an orthogonalised update:
//   m' = beta m + g;  u = g + beta m' (Nesterov) or m';  X = u / (|u| + eps);  `steps` times X = a X + (b X X^T + c (X X^T)^2) X;
//   w' = w - lr (scale X + decay w)
//
// An adapter has one short side R <= 64 (its rank) and one long side L.  The products never touch the long side twice: with
// G = u u^T over the long side, R x R, every X is p(G) u for a polynomial p, and the Gram matrix of X is G p(G)^2.  So a step is
//   1. one pass over g and m that writes m' and adds up G,
//   2. the iteration on R x R matrices, one workgroup per adapter,
//   3. one pass that multiplies p(G) with u and updates the weights.
//
// Precision.  A direction of u that is small beside the largest grows by a = 3.4 in every step, 485 in five, and an error of G
// by a^2 in every step: in 32 bits X would be off by 1e-4 and more where the direct products are off by 1e-6 (R = 64, singular
// values over three decades).  G, its polynomial and the products are in 64 bits (off by 3e-13), on v_mfma_f64_16x16x4, at
// 68 TFLOP/s here, a library product's rate: per element the first pass takes 0.5 ps of
// them at R = 16 and 1.2 at R = 64 beside 2.4 ps of the memory (12 bytes), the last 0.5 and 1.9 beside 3.5 (18 bytes).
//
// Layouts of v_mfma_f64_16x16x4: A[i][k] and B[k][i] in lane i + 16 k; D[row][column] in lane column + 16 q, register v, with row = q + 4 v.
#include <algorithm>
#include <new>
#include <type_traits>

#include "gemm_common.h"
#include "muon.h"

namespace lowra {

namespace {

typedef double f64x4_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ f64x4_t mfma64(double a, double b, f64x4_t c) { return __builtin_amdgcn_mfma_f64_16x16x4f64(a, b, c, 0, 0, 0); }

constexpr int MU_SPAN = 256;             // long-side elements that a workgroup of either pass takes at a time
constexpr int MU_THREADS = 256;

// NT: 16-wide tiles of the short side (1, 2 or 4).  Gram matrices are symmetric: tiles (t1, t2), t1 <= t2.
constexpr int mu_tiles(int NT) { return NT * (NT + 1) / 2; }
constexpr int mu_tile(int NT, int t1, int t2) { return t1 * NT - t1 * (t1 - 1) / 2 + (t2 - t1); }
constexpr int mu_ld(int NT) { return 16 * NT + 2; }          // doubles per LDS row: 16 rows at one column lie 4 banks apart

// The matrices are accessed as buffers (lowra_dev.h): a quad that is not there has an offset past the end (with loads under masks the
// first pass took 1.3 times as long).
// A quad of fp32 from element e on.  VEC: quads are 16-byte aligned and whole or not there; else n of them are.
template <bool VEC>
__device__ __forceinline__ float4 load4(buffer_t r, bool ok, uint32_t e, int n) {
    if constexpr (VEC) {
        return __builtin_bit_cast(float4, __builtin_amdgcn_raw_buffer_load_b128(r, ok ? e * 4 : kNowhere, 0, 0));
    } else {
        float v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(r, ok && i < n ? (e + i) * 4 : kNowhere, 0, 0));
        return make_float4(v[0], v[1], v[2], v[3]);
    }
}
template <bool VEC>
__device__ __forceinline__ void store4(buffer_t r, bool ok, uint32_t e, int n, float4 v) {
    if constexpr (VEC) {
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(g_u32x4_t, v), r, ok ? e * 4 : kNowhere, 0, 0);
    } else {
        const float x[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(uint32_t, x[i]), r, ok && i < n ? (e + i) * 4 : kNowhere, 0, 0);
    }
}
template <bool VEC>
__device__ __forceinline__ void store4_bf16(buffer_t r, bool ok, uint32_t e, int n, float4 v) {
    const uint32_t lo = pack_bf16x2(v.x, v.y), hi = pack_bf16x2(v.z, v.w);
    if constexpr (VEC) {
        __builtin_amdgcn_raw_buffer_store_b64(g_u32x2_t{lo, hi}, r, ok ? e * 2 : kNowhere, 0, 0);
    } else {
        const uint32_t x[4] = {lo, lo >> 16, hi, hi >> 16};
#pragma unroll
        for (int i = 0; i < 4; ++i) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(x[i] & 0xffffu), r, ok && i < n ? (e + i) * 2 : kNowhere, 0, 0);
    }
}
__device__ __forceinline__ float at4(const float4& v, int e) { return e == 0 ? v.x : e == 1 ? v.y : e == 2 ? v.z : v.w; }

// calls f with the number of tiles that R ranks reach: NT, or three of four.  (One 7B layer at rank 48 88 us with four, 69 so.)
template <int NT, class F>
__device__ __forceinline__ void with_tiles(int R, F&& f) {
    if (NT == 4 && R <= 48) f(std::integral_constant<int, NT == 4 ? 3 : NT>{});
    else f(std::integral_constant<int, NT>{});
}

struct Momentum { float beta; int nesterov; };
// m' and u of one element
__device__ __forceinline__ float momentum_of(const Momentum& mo, float g, float m) { return __builtin_fmaf(mo.beta, m, g); }
__device__ __forceinline__ float update_of(const Momentum& mo, float g, float m1) { return mo.nesterov ? __builtin_fmaf(mo.beta, m1, g) : m1; }

// ---- 1. momentum and Gram matrix.  Products over four long-side elements at a time: lane (i, q) holds element 16 t + i of the
// short side, k = q.  A step of a wavefront is 64 / NT long-side elements, four quads to a lane whatever NT is, brought into the
// operands' order through a piece of LDS of the wavefront's own.
// Short side in rows (A): 16 / NT lanes side by side load a row's 256 / NT bytes of the step, 4 NT rows at a time (with 64 bytes of
// 16 rows per load the pass over A at rank 16 took 1.5 times as long).  LDS rows of 64 / NT + 4 values: the operands' reads, 16 rows at
// one column and three more, touch every bank once.
// Short side in columns (B): the step's rows are 64 R / NT values on end whatever R is, loaded, stored and kept in LDS as such.
// The loads of the next step are under way while this one is multiplied.
constexpr int mu_step(int NT) { return 64 / NT; }
constexpr int mu_stage(int NT) { return 16 * NT * (mu_step(NT) + 4); }     // floats: more than the 1024 of the other form
template <int NT> struct GramSums { f64x4_t acc[mu_tiles(NT)]; };
// N: tiles that R reaches (of 64 ranks' four, three up to 48); the others' sums stay zero.
template <int NT, int N, bool WIDE, bool VEC>
__device__ __forceinline__ void muon_gram(const MuonItem& it, int first, int last, const Momentum& mo, float* mine, GramSums<NT>& sums) {
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int R = it.R, L = it.L;
    const buffer_t grad = buffer_of(it.grad, (uint32_t)(R * L) * 4u), momentum = buffer_of(it.momentum, (uint32_t)(R * L) * 4u), momentum_out = buffer_of(it.momentum_out, (uint32_t)(R * L) * 4u);
    constexpr int STEP = mu_step(NT), LDW = STEP + 4, PER = STEP / 4;  // PER: lanes of a row
    // quad k of a lane in the step at c: its first element, whether it is there, and how many there are
    auto quad = [&](int c, int k, bool& ok, uint32_t& e) __attribute__((always_inline)) -> int {
        if (WIDE) {
            const int row = k * (64 / PER) + lane / PER, col = c + 4 * (lane % PER);
            ok = row < R && col < last;
            e = (uint32_t)row * (uint32_t)L + (uint32_t)col;               // (where nothing is, it may wrap)
            return last - col;
        }
        const int f = 4 * (k * 64 + lane), have = min(last - c, STEP) * R;
        ok = f < have;
        e = (uint32_t)(c * R + f);
        return have - f;
    };
    struct Step { float4 g[4], m[4]; };
    auto load = [&](int c, Step& s) __attribute__((always_inline)) {
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t e;
            bool ok;
            const int n = quad(c, k, ok, e);
            s.g[k] = load4<VEC>(grad, ok, e, n);
            s.m[k] = load4<VEC>(momentum, ok, e, n);
        }
    };
    // a wavefront's steps: 64 elements side by side, then the next 256
    auto after = [](int c, int j) { return c + ((j + 1) % NT == 0 ? MU_SPAN - (NT - 1) * STEP : STEP); };
    Step cur, nxt;
    int c = first + 64 * wave;
    if (c < last) load(c, cur);
    for (int j = 0; c < last; ++j) {                                  // uniform
        const int cn = after(c, j);
        if (cn < last) load(cn, nxt);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t e;
            bool ok;
            const int n = quad(c, k, ok, e);
            const float4 g = cur.g[k], o = cur.m[k];
            const float4 m1 = make_float4(momentum_of(mo, g.x, o.x), momentum_of(mo, g.y, o.y), momentum_of(mo, g.z, o.z), momentum_of(mo, g.w, o.w));
            store4<VEC>(momentum_out, ok, e, n, m1);
            // (what is not there has come as zeros)
            float* dst = mine + (WIDE ? (k * (64 / PER) + lane / PER) * LDW + 4 * (lane % PER) : 4 * (k * 64 + lane));
            *reinterpret_cast<float4*>(dst) = make_float4(update_of(mo, g.x, m1.x), update_of(mo, g.y, m1.y), update_of(mo, g.z, m1.z), update_of(mo, g.w, m1.w));
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
        for (int e = 0; e < STEP / 4; ++e) {
            double a[N];
#pragma unroll
            for (int t = 0; t < N; ++t) {
                if (WIDE) a[t] = (double)mine[(16 * t + i) * LDW + 4 * e + q];
                else a[t] = 16 * t + i < R ? (double)mine[(4 * e + q) * R + 16 * t + i] : 0.0;
            }
#pragma unroll
            for (int t1 = 0; t1 < N; ++t1)
#pragma unroll
                for (int t2 = t1; t2 < N; ++t2) sums.acc[mu_tile(NT, t1, t2)] = mfma64(a[t1], a[t2], sums.acc[mu_tile(NT, t1, t2)]);
        }
        cur = nxt;
        c = cn;
    }
}
// (two workgroups to a unit at least, or the accumulators are kept in the other half of the registers and copied in every step)
template <int NT>
__global__ __launch_bounds__(MU_THREADS, NT == 4 ? 2 : 4) void muon_gram_kernel(const MuonItem* __restrict__ items, const MuonChunk* __restrict__ chunks, Momentum mo,
                                                                                double* __restrict__ part) {
    constexpr int TILES = mu_tiles(NT);
    __shared__ __align__(16) union { double red[3][TILES][256]; float u[4][mu_stage(NT)]; } sh;
    const MuonItem it = items[chunks[blockIdx.x].item];
    const int first = chunks[blockIdx.x].first, last = chunks[blockIdx.x].last;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    GramSums<NT> s;
#pragma unroll
    for (int t = 0; t < TILES; ++t) s.acc[t] = f64x4_t{0.0, 0.0, 0.0, 0.0};
    const bool vec = ((it.wide ? it.L : it.R * it.L) & 3) == 0;
    with_tiles<NT>(it.R, [&](auto N_) __attribute__((always_inline)) {
        constexpr int N = decltype(N_)::value;
        if (it.wide) {
            if (vec) muon_gram<NT, N, true, true>(it, first, last, mo, sh.u[wave], s);
            else muon_gram<NT, N, true, false>(it, first, last, mo, sh.u[wave], s);
        } else {
            if (vec) muon_gram<NT, N, false, true>(it, first, last, mo, sh.u[wave], s);
            else muon_gram<NT, N, false, false>(it, first, last, mo, sh.u[wave], s);
        }
    });
    __syncthreads();
    // the wavefronts' sums, in order
    if (wave > 0) {
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) sh.red[wave - 1][t][v * 64 + lane] = s.acc[t][v];
    }
    __syncthreads();
    if (wave == 0) {
        double* dst = part + (size_t)blockIdx.x * (TILES * 256);
#pragma unroll
        for (int t = 0; t < TILES; ++t)
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int o = v * 64 + lane;
                dst[t * 256 + o] = ((s.acc[t][v] + sh.red[0][t][o]) + sh.red[1][t][o]) + sh.red[2][t][o];
            }
    }
}

// ---- 2. the iteration.  The polynomial is handed on as the operands of the third kernel: operand (to, t, k) of it, 64 values for the
// 64 lanes (x, q), row 16 to + x and column 16 t + 4 k + q; for B in another order of the short side, see there.
template <int NT>
__global__ __launch_bounds__(NT == 4 ? 1024 : NT == 2 ? 512 : 256) void muon_iterate_kernel(const MuonItem* __restrict__ items, const double* __restrict__ part,
                                                                                            double* __restrict__ poly, int steps, double ca, double cb,
                                                                                            double cc, double eps) {
    constexpr int TILES = mu_tiles(NT), LD = mu_ld(NT), RP = 16 * NT, WAVES = NT == 4 ? 16 : NT == 2 ? 8 : 4;
    static_assert(TILES <= WAVES, "a wavefront has one tile of a product at most");
    extern __shared__ __align__(16) uint8_t smem[];
    double* G = reinterpret_cast<double*>(smem);
    double *P = G + RP * LD, *Q = P + RP * LD, *T = Q + RP * LD;
    const MuonItem it = items[blockIdx.x];
    const int lane = threadIdx.x & 63, i = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // tile (t1, t2) of a symmetric matrix from its accumulators, both halves
    auto place = [&](double* M, int t1, int t2, int o, double x) __attribute__((always_inline)) {      // o: v * 64 + lane
        const int r = 16 * t1 + ((o >> 4) & 3) + 4 * (o >> 6), c = 16 * t2 + (o & 15);
        if (r <= c) { M[r * LD + c] = x; M[c * LD + r] = x; }        // (the two halves of a product differ by their rounding)
    };
    const double* src = part + (size_t)it.chunk0 * (TILES * 256);
    // the chunks' sums, in order; SLOTS of them for a thread, AT chunks' loads at a time (24 of one tile where there are many: one 7B layer
    // at rank 16 18.6 -> 17.7 us, 32 layers with their few chunks 253 -> 254.5)
    auto add_chunks = [&](auto AT_) __attribute__((always_inline)) {
        constexpr int AT = decltype(AT_)::value, SLOTS = (TILES * 256 + WAVES * 64 - 1) / (WAVES * 64);
        double x[SLOTS];
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) x[j] = 0.0;
        for (int k = 0; k < it.nchunks; k += AT) {
            double v[SLOTS][AT];
#pragma unroll
            for (int j = 0; j < SLOTS; ++j)
#pragma unroll
                for (int u = 0; u < AT; ++u)
                    v[j][u] = src[(size_t)min(k + u, it.nchunks - 1) * (TILES * 256) + min((int)threadIdx.x + j * WAVES * 64, TILES * 256 - 1)];
#pragma unroll
            for (int j = 0; j < SLOTS; ++j)
#pragma unroll
                for (int u = 0; u < AT; ++u) x[j] += k + u < it.nchunks ? v[j][u] : 0.0;
        }
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
            const int o = threadIdx.x + j * WAVES * 64;
            int t1 = 0, rest = o >> 8;
            while (rest >= NT - t1 && t1 < NT) { rest -= NT - t1; ++t1; }
            if (o < TILES * 256) place(G, t1, t1 + rest, o & 255, x[j]);
        }
    };
    if (NT == 1 && it.nchunks > 8) add_chunks(std::integral_constant<int, 24>{});
    else add_chunks(std::integral_constant<int, 8>{});
    __syncthreads();
    double trace = 0.0;
#pragma unroll
    for (int r = 0; r < RP; ++r) trace += G[r * LD + r];
    const double norm = 1.0 / (sqrt(trace) + eps);
    __syncthreads();
    if (NT == 4)                                                    // (tiles that the ranks do not reach are not computed)
        for (int o = threadIdx.x; o < RP * LD; o += WAVES * 64) P[o] = 0.0;
    for (int o = threadIdx.x; o < RP * RP; o += WAVES * 64) G[(o / RP) * LD + o % RP] *= norm * norm;
    __syncthreads();

    // One tile: a wavefront keeps the matrices in registers.  Register v of a result is row q + 4 v (or column, which is the same) at i, and
    // that is an operand for the four products k = q + 4 v: the sum over k may go in any order.  (A step 1.06 us in LDS, 0.57 so.)
    if constexpr (NT == 1) if (wave == 0) {
        f64x4_t g, p;
#pragma unroll
        for (int v = 0; v < 4; ++v) g[v] = G[(q + 4 * v) * LD + i];
        auto times = [&](f64x4_t x, f64x4_t y) __attribute__((always_inline)) {
            f64x4_t c = {0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int v = 0; v < 4; ++v) c = mfma64(x[v], y[v], c);
            return c;
        };
        for (int s = 0; s < steps; ++s) {
            f64x4_t w = times(g, g);
#pragma unroll
            for (int v = 0; v < 4; ++v) w[v] = cc * w[v] + cb * g[v] + (q + 4 * v == i ? ca : 0.0);
            p = s > 0 ? times(p, w) : w;
            if (s + 1 < steps) g = times(times(g, w), w);
        }
#pragma unroll
        for (int v = 0; v < 4; ++v) P[(q + 4 * v) * LD + i] = p[v];
    }
    if constexpr (NT == 1) __syncthreads();
    if constexpr (NT > 1) with_tiles<NT>(it.R, [&](auto N_) __attribute__((always_inline)) {
        constexpr int N = decltype(N_)::value, JOBS = mu_tiles(N);
        // tile (t1, t2) of the product of two symmetric matrices that commute
        auto product = [&](const double* X, const double* Y, int t1, int t2) __attribute__((always_inline)) {
            f64x4_t c = {0.0, 0.0, 0.0, 0.0};
            const double *x = X + (16 * t1 + i) * LD + q, *y = Y + (16 * t2 + i) * LD + q;
#pragma unroll
            for (int k = 0; k < 16 * N; k += 4) c = mfma64(x[k], y[k], c);
            return c;
        };
        auto tiles = [&](int job, int& t1, int& t2) __attribute__((always_inline)) {
            t1 = 0;
            while (job >= N - t1) { job -= N - t1; ++t1; }
            t2 = t1 + job;
        };
        for (int s = 0; s < steps; ++s) {
            const bool more = s + 1 < steps;
            for (int job = wave; job < JOBS; job += WAVES) {            // Q = a + b G + c G^2; P = Q in the first step
                int t1, t2;
                tiles(job, t1, t2);
                const f64x4_t g2 = product(G, G, t1, t2);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const int r = 16 * t1 + q + 4 * v, c = 16 * t2 + i;
                    const double x = cc * g2[v] + cb * G[r * LD + c] + (r == c ? ca : 0.0);
                    place(Q, t1, t2, v * 64 + lane, x);
                    if (s == 0) place(P, t1, t2, v * 64 + lane, x);
                }
            }
            __syncthreads();
            f64x4_t pn = {0.0, 0.0, 0.0, 0.0};                            // a tile of the new P: kept until everyone has read the old one
            int p1 = -1, p2 = 0;
            for (int job = wave; job < 2 * JOBS; job += WAVES) {        // T = G Q, and P Q (at most one tile of it for a wavefront)
                int t1, t2;
                if (job < JOBS) {
                    if (!more) continue;
                    tiles(job, t1, t2);
                    const f64x4_t x = product(G, Q, t1, t2);
#pragma unroll
                    for (int v = 0; v < 4; ++v) place(T, t1, t2, v * 64 + lane, x[v]);
                } else if (s > 0) {
                    tiles(job - JOBS, p1, p2);
                    pn = product(P, Q, p1, p2);
                }
            }
            __syncthreads();
            if (p1 >= 0) {
#pragma unroll
                for (int v = 0; v < 4; ++v) place(P, p1, p2, v * 64 + lane, pn[v]);
            }
            if (more) {
                for (int job = wave; job < JOBS; job += WAVES) {        // G = T Q
                    int t1, t2;
                    tiles(job, t1, t2);
                    const f64x4_t x = product(T, Q, t1, t2);
#pragma unroll
                    for (int v = 0; v < 4; ++v) place(G, t1, t2, v * 64 + lane, x[v]);
                }
            }
            __syncthreads();
        }
    });
    double* dst = poly + (size_t)blockIdx.x * (RP * RP);
    auto element = [&](int p) { return it.wide ? p : (p & ~15) | (4 * (p & 3) + ((p >> 2) & 3)); };
    for (int o = threadIdx.x; o < RP * RP; o += WAVES * 64) {
        const int l = o & 63, k = (o >> 6) & 3, t = (o >> 8) % NT, to = (o >> 8) / NT;
        dst[o] = P[element(16 * to + (l & 15)) * LD + element(16 * t + 4 * k + (l >> 4))] * norm;
    }
}

// ---- 3. X = p(G) u and the weights.  A wavefront takes 64 long-side elements: four operands o of 16, products k over the short side.
// Short side in rows: lane (x, q) holds rows 16 t + q + 4 v, columns 4 x .. + 3; operand o is column 4 x + o, k set (t, v) the rows
// 16 t + 4 v + q.  Results (row q + 4 v of a tile, column x) land where the lane's own elements are.
// Short side in columns: lane (x, q) holds row 16 o + x, columns 16 t + 4 q .. + 3; k set (t, e) the columns 16 t + 4 q + e.  With the
// short side in the order in which place p of a tile is element 4 (p % 4) + p / 4, that is place 4 e + q of the tile, and the results
// again land where the lane's own elements are.
// With 64 ranks two wavefronts share the four result tiles of their 64 elements (and load u twice, the second time from the cache): one
// layer's adapters are 1220 such pieces of 16400 matrix cycles on 1024 SIMDs, as halves they lie more evenly (a step of one 7B layer
// 100.8 -> 97.7 us; where all ranks are rows 91 -> 87, all columns, whose halves touch 64 bytes of a row at a time, 94.4 -> 95.5).
constexpr int mu_parts(int NT) { return NT == 4 ? 2 : 1; }
struct MuonScalars { float lr, decay; };
template <int NT, int N, bool WIDE, bool VEC>
__device__ __forceinline__ void muon_apply(const MuonItem& it, int first, int last, const Momentum& mo, const double* P, const MuonScalars& sc) {
    const int lane = threadIdx.x & 63, x = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int R = it.R, L = it.L, n_all = R * L;
    const buffer_t grad = buffer_of(it.grad, (uint32_t)(n_all) * 4u), momentum = buffer_of(it.momentum_out, (uint32_t)(n_all) * 4u), weight = buffer_of(it.weight, (uint32_t)(n_all) * 4u),
                 weight_out = buffer_of(it.weight_out, (uint32_t)(n_all) * 4u), update = buffer_of(it.update, (uint32_t)(n_all) * 4u), weight_bf16 = buffer_of(it.weight_bf16, (uint32_t)(n_all) * 2u);
    constexpr int PARTS = mu_parts(NT), SPAN = MU_SPAN / PARTS;       // wavefronts that share the result tiles of 64 elements
    const int part = wave % PARTS;
    for (int c = first + 64 * (wave / PARTS); c < last; c += SPAN) { // uniform
        // quad (t, j): wide: row 16 t + q + 4 j, columns c + 4 x; else row c + 16 j + x, columns 16 t + 4 q
        auto quad = [&](int t, int j, bool& ok, uint32_t& e) __attribute__((always_inline)) -> int {
            int y = q;
            if (!VEC) asm volatile("" : "+v"(y));                    // (taken afresh: the addresses of all elements at once do not fit)
            const int s = WIDE ? 16 * t + y + 4 * j : 16 * t + 4 * y;
            const int l = WIDE ? c + 4 * x : c + 16 * j + x;
            ok = s < R && l < last;
            e = WIDE ? (uint32_t)s * (uint32_t)L + (uint32_t)l : (uint32_t)l * (uint32_t)R + (uint32_t)s;
            return WIDE ? last - l : R - s;
        };
        float4 u[N][4];
        auto load = [&](buffer_t r, int t, int j) __attribute__((always_inline)) {
            uint32_t e;
            bool ok;
            const int n = quad(t, j, ok, e);
            return load4<VEC>(r, ok, e, n);
        };
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) u[t][j] = load(momentum, t, j);
        if (mo.nesterov) {
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float4 g = load(grad, t, j), m1 = u[t][j];
                    u[t][j] = make_float4(update_of(mo, g.x, m1.x), update_of(mo, g.y, m1.y), update_of(mo, g.z, m1.z), update_of(mo, g.w, m1.w));
                }
        }
#pragma unroll 1
        for (int to = part * (NT / PARTS); to < min((part + 1) * (NT / PARTS), N); ++to) {      // (one body: u in 64 bits takes half of the registers as it is)
            float4 w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = load(weight, to, j);
            f64x4_t acc[4];
#pragma unroll
            for (int o = 0; o < 4; ++o) acc[o] = f64x4_t{0.0, 0.0, 0.0, 0.0};
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const double p = P[((to * NT + t) * 4 + k) * 64 + lane];
#pragma unroll
                    for (int o = 0; o < 4; ++o) acc[o] = mfma64(p, (double)(WIDE ? at4(u[t][k], o) : at4(u[t][o], k)), acc[o]);
                }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t e;
                bool ok;
                const int n = quad(to, j, ok, e);
                float4 y;
                if (WIDE) y = make_float4((float)acc[0][j], (float)acc[1][j], (float)acc[2][j], (float)acc[3][j]);
                else y = make_float4((float)acc[j][0], (float)acc[j][1], (float)acc[j][2], (float)acc[j][3]);
                y.x *= it.scale; y.y *= it.scale; y.z *= it.scale; y.w *= it.scale;
                const float4 v = make_float4(w[j].x - sc.lr * __builtin_fmaf(sc.decay, w[j].x, y.x), w[j].y - sc.lr * __builtin_fmaf(sc.decay, w[j].y, y.y),
                                             w[j].z - sc.lr * __builtin_fmaf(sc.decay, w[j].z, y.z), w[j].w - sc.lr * __builtin_fmaf(sc.decay, w[j].w, y.w));
                if (it.update) store4<VEC>(update, ok, e, n, y);              // uniform
                store4<VEC>(weight_out, ok, e, n, v);
                store4_bf16<VEC>(weight_bf16, ok, e, n, v);
            }
        }
    }
}
template <int NT>
__global__ __launch_bounds__(MU_THREADS, NT == 1 ? 4 : NT == 2 ? 3 : 2) void muon_apply_kernel(const MuonItem* __restrict__ items, const MuonChunk* __restrict__ chunks,
                                                                                               Momentum mo, const double* __restrict__ poly, MuonScalars sc) {
    __shared__ double P[256 * NT * NT];
    const int item = chunks[blockIdx.x].item;
    const MuonItem it = items[item];
    const int first = chunks[blockIdx.x].first, last = chunks[blockIdx.x].last;
#pragma unroll
    for (int o = 0; o < NT * NT; ++o) P[o * 256 + threadIdx.x] = poly[((size_t)item * (NT * NT) + o) * 256 + threadIdx.x];
    __syncthreads();
    const bool vec = ((it.wide ? it.L : it.R) & 3) == 0;
    with_tiles<NT>(it.R, [&](auto N_) __attribute__((always_inline)) {
        constexpr int N = decltype(N_)::value;
        if (it.wide) {
            if (vec) muon_apply<NT, N, true, true>(it, first, last, mo, P, sc);
            else muon_apply<NT, N, true, false>(it, first, last, mo, P, sc);
        } else {
            if (vec) muon_apply<NT, N, false, true>(it, first, last, mo, P, sc);
            else muon_apply<NT, N, false, false>(it, first, last, mo, P, sc);
        }
    });
}

int mu_class(int R) { return R <= 16 ? 0 : R <= 32 ? 1 : 2; }
constexpr int kMuNT[3] = {1, 2, 4};

// Long-side elements per workgroup: enough workgroups to fill the chip several times, and no more than 2048.  The first pass takes at
// least 512 at 64 ranks, where a workgroup's partial Gram matrix is 20 KB and one unit adds up all of a matrix's: with 256, one layer at
// rank 64 spends 8 us more there, and a unit with two such workgroups is busy as long as one with one of 512.
int mu_chunk(long long total, int least) {
    const long long n = total / MU_SPAN / (4 * device_compute_units());
    return std::max(least, MU_SPAN * (int)std::max(1ll, std::min(n, 8ll)));
}

struct MuonPlan { int gram[3], apply[3]; size_t chunks[3], items[3], part0[3], poly0[3], bytes; };
MuonPlan mu_plan(int n, const MuonItem* items) {
    MuonPlan p{};
    long long total[3] = {0, 0, 0};
    for (int i = 0; i < n; ++i) total[mu_class(items[i].R)] += items[i].L;
    for (int c = 0; c < 3; ++c) { p.gram[c] = mu_chunk(total[c], c == 2 ? 512 : MU_SPAN); p.apply[c] = mu_chunk(total[c], MU_SPAN); }
    for (int i = 0; i < n; ++i) {
        const int c = mu_class(items[i].R);
        p.chunks[c] += (size_t)((items[i].L + p.gram[c] - 1) / p.gram[c]);
        ++p.items[c];
    }
    for (int c = 0; c < 3; ++c) {
        p.part0[c] = p.bytes; p.bytes += p.chunks[c] * mu_tiles(kMuNT[c]) * 256 * sizeof(double);
        p.poly0[c] = p.bytes; p.bytes += p.items[c] * (size_t)(256 * kMuNT[c] * kMuNT[c]) * sizeof(double);
    }
    return p;
}

template <class T>
hipError_t upload(const std::vector<T>& v, T*& d) {
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&d), v.size() * sizeof(T));
    return e != hipSuccess ? e : hipMemcpy(d, v.data(), v.size() * sizeof(T), hipMemcpyHostToDevice);
}

template <int NT>
hipError_t mu_run(const MuonGroup& g, const MuonStep& s, hipStream_t st) {
    constexpr int threads = NT == 4 ? 1024 : NT == 2 ? 512 : 256, sh = 4 * 16 * NT * mu_ld(NT) * (int)sizeof(double);
    static const hipError_t attr = hipFuncSetAttribute(reinterpret_cast<const void*>(muon_iterate_kernel<NT>), hipFuncAttributeMaxDynamicSharedMemorySize, sh);
    if (attr != hipSuccess) return attr;
    const Momentum mo{s.momentum, s.nesterov};
    hipError_t e;
    muon_gram_kernel<NT><<<dim3((unsigned)g.ngram), dim3(MU_THREADS), 0, st>>>(g.d_items, g.d_chunks, mo, g.part);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    muon_iterate_kernel<NT><<<dim3((unsigned)g.nitems), dim3(threads), sh, st>>>(g.d_items, g.part, g.poly, s.steps, (double)s.a, (double)s.b, (double)s.c,
                                                                                 (double)s.eps);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    muon_apply_kernel<NT><<<dim3((unsigned)g.napply), dim3(MU_THREADS), 0, st>>>(g.d_items, g.d_chunks + g.ngram, mo, g.poly, MuonScalars{s.lr, s.decay});
    return hipGetLastError();
}

}  // namespace

size_t muon_workspace_bytes(int n, const MuonItem* items) { return mu_plan(n, items).bytes; }

hipError_t muon_build(const std::vector<MuonItem>& all, void* workspace, MuonGroup (&groups)[3]) {
    const MuonPlan p = mu_plan((int)all.size(), all.data());
    for (int c = 0; c < 3; ++c) {
        std::vector<MuonItem> items;
        std::vector<MuonChunk> chunks, apply;
        auto cut = [](std::vector<MuonChunk>& to, int L, int by, int item) {
            for (int l = 0; l < L; l += std::min(by, L - l)) to.push_back(MuonChunk{l, l + std::min(by, L - l), item});
        };
        for (const MuonItem& a : all) {
            if (mu_class(a.R) != c) continue;
            MuonItem it = a;
            it.chunk0 = (int)chunks.size();
            cut(chunks, it.L, p.gram[c], (int)items.size());
            it.nchunks = (int)chunks.size() - it.chunk0;
            cut(apply, it.L, p.apply[c] / mu_parts(kMuNT[c]), (int)items.size());
            items.push_back(it);
        }
        MuonGroup& g = groups[c];
        g.nitems = (int)items.size(); g.ngram = (int)chunks.size(); g.napply = (int)apply.size();
        chunks.insert(chunks.end(), apply.begin(), apply.end());
        g.part = reinterpret_cast<double*>(static_cast<uint8_t*>(workspace) + p.part0[c]);
        g.poly = reinterpret_cast<double*>(static_cast<uint8_t*>(workspace) + p.poly0[c]);
        if (items.empty()) continue;
        hipError_t e;
        if ((e = upload(items, g.d_items)) != hipSuccess || (e = upload(chunks, g.d_chunks)) != hipSuccess) return e;
    }
    return hipSuccess;
}

hipError_t muon_run(const MuonGroup (&groups)[3], const MuonStep& s, hipStream_t st) {
    hipError_t e = hipSuccess;
    if (groups[0].nitems && (e = mu_run<1>(groups[0], s, st)) != hipSuccess) return e;
    if (groups[1].nitems && (e = mu_run<2>(groups[1], s, st)) != hipSuccess) return e;
    if (groups[2].nitems && (e = mu_run<4>(groups[2], s, st)) != hipSuccess) return e;
    return e;
}

void muon_free(MuonGroup (&groups)[3]) {
    for (MuonGroup& g : groups) {
        (void)hipFree(g.d_items); (void)hipFree(g.d_chunks);
        g = MuonGroup{};
    }
}

}  // namespace lowra
