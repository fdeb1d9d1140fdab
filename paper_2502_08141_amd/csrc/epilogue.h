// What the linear calls with an epilogue do to a result before it is stored, and the activation's backward pass.
//
//   forward         v = product + bias                 y = act(v) mul + residual     z = bf16(v), where it is kept
//   input gradient  g = product + residual             dX = g mul act'(z)            dmul = g act(z)
//
// All arithmetic is fp32 on the fp32 accumulators; every output is rounded to bf16 once.  z is kept as bf16, the type of the
// activations beside it: the gradient of an activation changes by its curvature times half a bf16 step of z, less than the
// gradient's own rounding for |z| up to about one, and fp32 would double what the backward pass reads.
//
// What bounds it: plain-ALU issue where a GEMM's workgroup is alone on its compute unit (nothing overlaps its epilogue), so
// the activations are a handful of instructions.  Quarter-rate instructions per value: 2 (exp2, reciprocal) in each.
#pragma once
#include <type_traits>

#include "lowra_host.h"

namespace lowra {

enum : int { kActNone = 0, kActRelu = 1, kActGelu = 2, kActGeluTanh = 3, kActSilu = 4 };

// log2(e)
constexpr float kLog2e = 1.44269504f;

// The normal distribution function at -|z|, and e = exp(-z^2 / 2): their quotient is smooth, a polynomial in 1 / (1 + 0.35 |z|) (our own
// minimax fit on [0, 13], relative error 3.1e-7; with the fp32 rounding 6e-7 up to |z| = 2, 8e-6 at 13).  In this form the small tail
// keeps its relative accuracy, which 1 + erf loses, and the slope has its density for one product.
__device__ __forceinline__ float normal_tail(float z, float& e) {
    e = __builtin_amdgcn_exp2f(z * z * (-0.5f * kLog2e));
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.35f, __builtin_fabsf(z), 1.0f));
    float q = 0x1.90efbep-5f;
    q = __builtin_fmaf(q, t, -0x1.9df0b8p-3f);
    q = __builtin_fmaf(q, t, 0x1.ecd51ap-3f);
    q = __builtin_fmaf(q, t, -0x1.16e98p-6f);
    q = __builtin_fmaf(q, t, 0x1.3f68bcp-3f);
    q = __builtin_fmaf(q, t, 0x1.111c7ap-3f);
    q = __builtin_fmaf(q, t, 0x1.1f460ep-3f);
    q = __builtin_fmaf(q, t, -0x1.ca4766p-16f);
    return e * q;
}

// act(z) and, with SLOPE, act'(z).  Infinite z give the limits (a factor that has become zero is not multiplied with one).
template <int ACT, bool SLOPE>
__device__ __forceinline__ void activation(float z, float& y, float& slope) {
    slope = 1.0f;
    if constexpr (ACT == kActNone) {
        y = z;
    } else if constexpr (ACT == kActRelu) {
        y = z < 0.0f ? 0.0f : z;                                   // (a NaN stays one)
        slope = z > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == kActGelu) {
        float e;
        const float tail = normal_tail(z, e), p = z > 0.0f ? 1.0f - tail : tail;
        y = p == 0.0f ? 0.0f : z * p;
        if constexpr (SLOPE) {
            const float d = e * 0.398942280f;                      // the density
            slope = d == 0.0f ? p : __builtin_fmaf(z, d, p);
        }
    } else {
        // z times the logistic function of w
        float w = z, dw = 1.0f;
        if constexpr (ACT == kActGeluTanh) {
            constexpr float c = 1.59576912f, d = 0.044715f;        // 2 sqrt(2 / pi)
            const float z2 = z * z;
            w = c * z * __builtin_fmaf(d, z2, 1.0f);
            dw = c * __builtin_fmaf(3.0f * d, z2, 1.0f);
        }
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(w * -kLog2e));
        y = s == 0.0f ? 0.0f : z * s;
        if constexpr (SLOPE) {
            const float t = s - s * s;                             // s (1 - s)
            slope = t == 0.0f ? s : __builtin_fmaf(z * dw, t, s);
        }
    }
}

// calls f(std::integral_constant<int, act>): a uniform branch around what follows
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case kActRelu: f(std::integral_constant<int, kActRelu>{}); break;
        case kActGelu: f(std::integral_constant<int, kActGelu>{}); break;
        case kActGeluTanh: f(std::integral_constant<int, kActGeluTanh>{}); break;
        case kActSilu: f(std::integral_constant<int, kActSilu>{}); break;
        default: f(std::integral_constant<int, kActNone>{}); break;
    }
}

// W (1, 4 or 8) neighbouring bf16 values in one access, kept as they are until they are used (a conversion beside the load would
// wait for it there)
template <int W> struct Bf16Run {
    uint32_t d[W == 1 ? 1 : W / 2];
    __device__ __forceinline__ float operator[](int i) const {
        return W == 1 || (i & 1) == 0 ? bf16_bits_to_float(d[i >> 1]) : __builtin_bit_cast(float, d[i >> 1] & 0xffff0000u);
    }
};
template <int W>
__device__ __forceinline__ void load_run(const uint16_t* p, Bf16Run<W>& r) {
    static_assert(W == 1 || W == 4 || W == 8, "one access");
    if constexpr (W == 8) { const uint4 t = *reinterpret_cast<const uint4*>(p); r.d[0] = t.x; r.d[1] = t.y; r.d[2] = t.z; r.d[3] = t.w; }
    if constexpr (W == 4) { const uint2 t = *reinterpret_cast<const uint2*>(p); r.d[0] = t.x; r.d[1] = t.y; }
    if constexpr (W == 1) r.d[0] = *p;
}
template <int W>
__device__ __forceinline__ void store_run(uint16_t* p, const float (&v)[W]) {
    if constexpr (W == 1) *p = (uint16_t)(pack_bf16x2(v[0], 0.0f) & 0xffffu);
    if constexpr (W == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    if constexpr (W == 8)
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}

// The operands of an epilogue; null: not there.  mul, residual, z, dmul: [M][columns] like the result.
struct FwdEpi {
    int act;
    const uint16_t* bias;        // [columns]
    const uint16_t* mul;
    const uint16_t* residual;    // may be the result's own buffer: an element is read before it is written, by the same thread
    uint16_t* z;                 // out
};
struct BwdEpi {
    int act;
    const uint16_t* z;
    const uint16_t* mul;
    const uint16_t* residual;    // as above
    uint16_t* dmul;              // out
};
struct NoEpi {};

// What an epilogue reads for W neighbouring results
template <class E, int W> struct EpiRun;
template <int W> struct EpiRun<FwdEpi, W> { Bf16Run<W> mul, residual; };
template <int W> struct EpiRun<BwdEpi, W> { Bf16Run<W> z, mul, residual; };
template <int W>
__device__ __forceinline__ void epi_load(const FwdEpi& e, size_t at, EpiRun<FwdEpi, W>& r) {
    if (e.mul) load_run<W>(e.mul + at, r.mul);
    if (e.residual) load_run<W>(e.residual + at, r.residual);
}
template <int W>
__device__ __forceinline__ void epi_load(const BwdEpi& e, size_t at, EpiRun<BwdEpi, W>& r) {
    if (e.z) load_run<W>(e.z + at, r.z);
    if (e.mul) load_run<W>(e.mul + at, r.mul);
    if (e.residual) load_run<W>(e.residual + at, r.residual);
}
// the bias of W neighbouring columns; none in the input gradient
template <int W>
__device__ __forceinline__ void epi_bias(const FwdEpi& e, int col, float (&b)[W]) {
    Bf16Run<W> r;
    if (e.bias) load_run<W>(e.bias + col, r);
#pragma unroll
    for (int i = 0; i < W; ++i) b[i] = e.bias ? r[i] : 0.0f;
}
template <int W>
__device__ __forceinline__ void epi_bias(const BwdEpi&, int, float (&)[W]) {}

// v: the products in, y out; keep(z) stores z
template <int ACT, int W, class Keep>
__device__ __forceinline__ void epi_apply(const FwdEpi& e, float (&v)[W], const float (&b)[W], const EpiRun<FwdEpi, W>& r, Keep&& keep) {
#pragma unroll
    for (int i = 0; i < W; ++i) v[i] += b[i];
    if (e.z) keep(v);
    float slope;
#pragma unroll
    for (int i = 0; i < W; ++i) activation<ACT, false>(v[i], v[i], slope);
    if (e.mul) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= r.mul[i];
    }
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += r.residual[i];
    }
}
// v: the products in, dX out; keep(dmul) stores dmul
template <int ACT, int W, class Keep>
__device__ __forceinline__ void epi_apply(const BwdEpi& e, float (&v)[W], const float (&)[W], const EpiRun<BwdEpi, W>& r, Keep&& keep) {
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] += r.residual[i];
    }
    float y[W], slope[W];
    if (ACT != kActNone || e.dmul) {
#pragma unroll
        for (int i = 0; i < W; ++i) activation<ACT, true>(r.z[i], y[i], slope[i]);
    }
    if (e.dmul) {
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] *= v[i];
        keep(y);
    }
    if (e.mul) {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] *= r.mul[i];
    }
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (ACT == kActRelu) v[i] = slope[i] != 0.0f ? v[i] : 0.0f;      // (an infinite gradient where nothing passes: zero)
        else if constexpr (ACT != kActNone) v[i] *= slope[i];
    }
}
// one run by itself: element `at` of the result
__device__ __forceinline__ uint16_t* epi_second(const FwdEpi& e) { return e.z; }
__device__ __forceinline__ uint16_t* epi_second(const BwdEpi& e) { return e.dmul; }
template <int W, class E>
__device__ __forceinline__ void epi_run(const E& e, size_t at, int col, float (&v)[W], uint16_t* out) {
    EpiRun<E, W> r;
    float b[W];
    epi_load<W>(e, at, r);
    epi_bias<W>(e, col, b);
    with_act(e.act, [&](auto A) __attribute__((always_inline)) {
        epi_apply<decltype(A)::value, W>(e, v, b, r, [&](const float (&w)[W]) __attribute__((always_inline)) { store_run<W>(epi_second(e) + at, w); });
    });
    store_run<W>(out + at, v);
}

// ---- the epilogue of a whole output tile: operands and results as buffers that start at the tile's first row (32-bit offsets; an
// operand that is not there is an empty buffer, a row past the last token has an offset past the end)
constexpr int kEpiMaxColumns = (1 << 22) - 8;          // 256 rows of a tile stay below 2^31 bytes
template <class E> struct EpiTile;
template <> struct EpiTile<FwdEpi> { buffer_t mul, residual, second, out; };
template <> struct EpiTile<BwdEpi> { buffer_t z, mul, residual, second, out; };
__device__ __forceinline__ buffer_t epi_buffer(const uint16_t* p, size_t at) { return buffer_of(p ? p + at : nullptr, 0x7fffffffu); }
__device__ __forceinline__ EpiTile<FwdEpi> epi_tile(const FwdEpi& e, uint16_t* out, size_t at) {
    return EpiTile<FwdEpi>{epi_buffer(e.mul, at), epi_buffer(e.residual, at), epi_buffer(e.z, at), epi_buffer(out, at)};
}
__device__ __forceinline__ EpiTile<BwdEpi> epi_tile(const BwdEpi& e, uint16_t* out, size_t at) {
    return EpiTile<BwdEpi>{epi_buffer(e.z, at), epi_buffer(e.mul, at), epi_buffer(e.residual, at), epi_buffer(e.dmul, at), epi_buffer(out, at)};
}
__device__ __forceinline__ void buffer_load8(buffer_t b, uint32_t off, Bf16Run<8>& r) {
    const uint4 t = __builtin_bit_cast(uint4, __builtin_amdgcn_raw_buffer_load_b128(b, off, 0, 0));
    r.d[0] = t.x; r.d[1] = t.y; r.d[2] = t.z; r.d[3] = t.w;
}
__device__ __forceinline__ void buffer_store8(buffer_t b, uint32_t off, const float (&v)[8]) {
    const u32x4_t t = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    __builtin_amdgcn_raw_buffer_store_b128(t, b, off, 0, 0);
}
__device__ __forceinline__ void epi_load(const EpiTile<FwdEpi>& t, uint32_t off, EpiRun<FwdEpi, 8>& r) {
    buffer_load8(t.mul, off, r.mul);
    buffer_load8(t.residual, off, r.residual);
}
__device__ __forceinline__ void epi_load(const EpiTile<BwdEpi>& t, uint32_t off, EpiRun<BwdEpi, 8>& r) {
    buffer_load8(t.z, off, r.z);
    buffer_load8(t.mul, off, r.mul);
    buffer_load8(t.residual, off, r.residual);
}
// Eight columns (from `col` on) of a thread's token rows, numbers FROM .. TO - 1 of TOTAL here: offset(j) is where the j-th one's are and
// read(j, v) gives its products.  run[j % U] holds its operands, asked for U rows ahead, over the passes through LDS: nothing else
// covers their way where a workgroup is alone on its unit.  (Input gradient of 4096 x 11008, 4096 tokens, through
// a silu gate: eight rows' loads together from pointers within a pass 519 us, so 401, with two rows ahead 417; without an epilogue 353.)
template <int U, class E, class Offset>
__device__ __forceinline__ void epi_fetch(const EpiTile<E>& t, EpiRun<E, 8> (&run)[U], Offset&& offset) {
#pragma unroll
    for (int u = 0; u < U; ++u) epi_load(t, offset(u), run[u]);
}
template <int FROM, int TO, int TOTAL, int U, class E, class Offset, class Read>
__device__ __forceinline__ void epi_rows(const E& e, const EpiTile<E>& t, const float (&b)[8], EpiRun<E, 8> (&run)[U], Offset&& offset, Read&& read) {
    static_assert((TO - FROM) % U == 0 && FROM % U == 0, "");
    with_act(e.act, [&](auto A) __attribute__((always_inline)) {
#pragma unroll 1
        for (int j = FROM; j < TO; j += U) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t off = offset(j + u);
                float v[8];
                read(j + u, v);
                epi_apply<decltype(A)::value, 8>(e, v, b, run[u], [&](const float (&w)[8]) __attribute__((always_inline)) { buffer_store8(t.second, off, w); });
                buffer_store8(t.out, off, v);
                if (j + U < TOTAL) epi_load(t, offset(j + u + U), run[u]);                       // uniform
            }
        }
    });
}
// The tile as fp32 in LDS, CHUNKS 16-byte chunks a row: chunk q (four columns) sits at half of the row by q's parity, place q / 2,
// xored with the row.  The accumulators' writes (one chunk of neighbouring rows) and the reads of eight columns (neighbouring
// even chunks, then odd ones, of one row) then both touch every bank.
template <int CHUNKS>
__device__ __forceinline__ int epi_chunk(int row, int q) { return row * (CHUNKS * 16) + ((((q >> 1) | ((q & 1) * (CHUNKS / 2))) ^ (row & (CHUNKS / 2 - 1))) << 4); }
template <int CHUNKS>
__device__ __forceinline__ void epi_read8(const uint8_t* smem, int row, int c8, float (&v)[8]) {
    const float4 a = *reinterpret_cast<const float4*>(smem + epi_chunk<CHUNKS>(row, 2 * c8)), b = *reinterpret_cast<const float4*>(smem + epi_chunk<CHUNKS>(row, 2 * c8 + 1));
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

// ---- act.hip
constexpr int kActMaxSize = 1 << 30;                   // of M and of N
size_t act_bwd_workspace_bytes(int M, int N);
// e.residual must be null; dZ null: only the sums (and dmul)
hipError_t launch_act_bwd(int M, int N, const BwdEpi& e, const uint16_t* dY, uint16_t* dZ, float* db, void* workspace, hipStream_t st);

}  // namespace lowra
