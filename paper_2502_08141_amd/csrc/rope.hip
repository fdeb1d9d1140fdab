// Rotary positions of queries and keys (what stands behind the projections of a fine-tuned layer, Sec. 2.1): the pair (a, b) of a head's columns
// j and j + rot/2 (or 2 j and 2 j + 1) becomes (a cos - b sin, a sin + b cos), the angle being the token's position times f_j; the inverse
// turns by the negative angle, which is the gradient's way back.
//
// Memory bound: 2 bytes in and 2 out per element.  The angle is position x turns mod 2^64 in whole numbers, 2^-64 of a full turn a unit, and then rounded to 2^-32 of a
// turn (2^-30 radians): no product loses digits at far positions, where fp32 is off by 0.03 at 2^20 and a table of cosines would be read beside the data.  What the plan's
// frequencies have lost (53 bits of each) grows with the position to 2^-32 at 2^20 and 2^-21 at 2^31.  What is left is at most an eighth of a turn, where
// the Taylor polynomials of degree 9 and 10 are exact to fp32 rounding (remainders pi/4^11 / 11! = 2e-9 and pi/4^12 / 12! = 1e-10).  A thread keeps
// the angles of its columns for several heads.  Graph replays: 4096 tokens of 32 + 32 heads of 128 columns 22.8 us (5.9 TB/s), 32 + 8 heads of neighbours 15.4,
// four tokens of 32 + 8 heads 3.2.
#include <algorithm>

#include "gemm_common.h"
#include "step.h"

namespace lowra {

namespace {

__device__ __forceinline__ void turn_of(uint64_t turns, int position, bool inverse, float magnitude, float& c, float& s) {
    const uint32_t hi = (uint32_t)((turns * (uint64_t)(int64_t)position + 0x80000000ull) >> 32);      // 2^-32 of a turn, to the nearest
    const uint32_t quarter = (hi + 0x20000000u) >> 30;
    const float a = (float)(int32_t)(hi - (quarter << 30)) * 1.4629180792671596e-09f;                 // 2 pi 2^-32
    const float q = a * a;
    float sn = __builtin_fmaf(q, 2.7557319223985893e-06f, -1.9841269841269841e-04f);
    sn = __builtin_fmaf(q, sn, 8.3333333333333332e-03f);
    sn = __builtin_fmaf(q, sn, -1.6666666666666666e-01f);
    sn = __builtin_fmaf(q * sn, a, a);
    float cs = __builtin_fmaf(q, -2.7557319223985888e-07f, 2.4801587301587302e-05f);
    cs = __builtin_fmaf(q, cs, -1.3888888888888889e-03f);
    cs = __builtin_fmaf(q, cs, 4.1666666666666664e-02f);
    cs = __builtin_fmaf(q, cs, -0.5f);
    cs = __builtin_fmaf(q, cs, 1.0f);
    const bool odd = quarter & 1u;
    const float x = odd ? sn : cs, y = odd ? cs : sn;
    c = ((quarter + 1u) & 2u ? -x : x) * magnitude;
    s = (((quarter & 2u) != 0) != inverse ? -y : y) * magnitude;
}

template <int V>
__device__ __forceinline__ void load_run16(const uint16_t* p, uint32_t (&w)[(V + 1) / 2]) {
    if constexpr (V == 8) {
        const uint4 q = *reinterpret_cast<const uint4*>(p);
        w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
    } else if constexpr (V == 4) {
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        w[0] = q.x; w[1] = q.y;
    } else if constexpr (V == 2) {
        w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        w[0] = *p;
    }
}
template <int V>
__device__ __forceinline__ void store_run16(uint16_t* p, const uint32_t (&w)[(V + 1) / 2]) {
    if constexpr (V == 8) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
    else if constexpr (V == 4) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    else if constexpr (V == 2) *reinterpret_cast<uint32_t*>(p) = w[0];
    else *p = (uint16_t)w[0];
}
__device__ __forceinline__ float lo16(uint32_t w) { return bf16_bits_to_float(w & 0xffffu); }
__device__ __forceinline__ float hi16(uint32_t w) { return __builtin_bit_cast(float, w & 0xffff0000u); }

// V columns to an access.  A unit is what a thread has of a head: V pairs of columns V apart from each other by rot / 2, or V neighbours that
// are V / 2 pairs (V = 1: a pair by itself), or V columns behind the rotated ones.  Threads: units fastest, then head slots, then tokens.
template <int V, bool INTER>
__global__ __launch_bounds__(256) void rope_kernel(RopeArgs a, int units, int rot_units, int slots, uint32_t total) {
    const uint32_t id = blockIdx.x * 256u + threadIdx.x;
    if (id >= total) return;
    const uint32_t rest = id / (uint32_t)units;
    const int unit = (int)(id - rest * (uint32_t)units);
    const int m = (int)(rest / (uint32_t)slots), slot = (int)(rest - (uint32_t)m * (uint32_t)slots);
    if (unit >= rot_units) {                                     // columns that stay
        const int col = a.rot + (unit - rot_units) * V;
        int h0 = 0;
        for (int i = 0; i < a.n; ++i) {
            const RopeTensor& t = a.t[i];
            if (t.x != t.y)
                for (int h = (slot + slots - h0 % slots) % slots; h < t.heads; h += slots) {
                    uint32_t w[(V + 1) / 2];
                    load_run16<V>(t.x + m * t.x_token + h * t.x_head + col, w);
                    store_run16<V>(t.y + m * t.y_token + h * t.y_head + col, w);
                }
            h0 += t.heads;
        }
        return;
    }
    constexpr int P = INTER ? (V + 1) / 2 : V;                   // pairs
    float c[P], s[P];
    const int position = a.positions[m];
#pragma unroll
    for (int p = 0; p < P; ++p) turn_of(a.turns[unit * P + p], position, a.inverse, a.magnitude, c[p], s[p]);
    int h0 = 0;
    for (int i = 0; i < a.n; ++i) {
        const RopeTensor& t = a.t[i];
        for (int h = (slot + slots - h0 % slots) % slots; h < t.heads; h += slots) {
            const uint16_t* x = t.x + m * t.x_token + h * t.x_head;
            uint16_t* y = t.y + m * t.y_token + h * t.y_head;
            if constexpr (INTER && V > 1) {
                uint32_t w[V / 2];
                load_run16<V>(x + unit * V, w);
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    const float u = lo16(w[p]), v = hi16(w[p]);
                    w[p] = pack_bf16x2(u * c[p] - v * s[p], u * s[p] + v * c[p]);
                }
                store_run16<V>(y + unit * V, w);
            } else {
                const int first = INTER ? 2 * unit : unit * V, second = INTER ? first + 1 : first + a.rot / 2;
                uint32_t f[(V + 1) / 2], g[(V + 1) / 2];
                load_run16<V>(x + first, f);
                load_run16<V>(x + second, g);
#pragma unroll
                for (int q = 0; q < (V + 1) / 2; ++q) {
                    const int p = 2 * q, r = V > 1 ? p + 1 : p;
                    const float u0 = lo16(f[q]), v0 = lo16(g[q]), u1 = hi16(f[q]), v1 = hi16(g[q]);
                    f[q] = pack_bf16x2(u0 * c[p] - v0 * s[p], u1 * c[r] - v1 * s[r]);
                    g[q] = pack_bf16x2(u0 * s[p] + v0 * c[p], u1 * s[r] + v1 * c[r]);
                }
                store_run16<V>(y + first, f);
                store_run16<V>(y + second, g);
            }
        }
        h0 += t.heads;
    }
}

// the widest access that pointers, strides and columns allow
bool rope_fits(const RopeArgs& a, int V) {
    if ((a.interleaved ? a.rot : a.rot / 2) % V != 0 || a.D % V != 0 || a.rot % V != 0) return false;
    for (int i = 0; i < a.n; ++i) {
        const RopeTensor& t = a.t[i];
        if ((t.x_token | t.x_head | t.y_token | t.y_head) % V != 0) return false;
        if (((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.y)) & (2 * V - 1)) != 0) return false;
    }
    return true;
}

template <int V, bool INTER>
hipError_t run(const RopeArgs& a, hipStream_t st) {
    int heads = 0;
    bool copies = false;
    for (int i = 0; i < a.n; ++i) { heads += a.t[i].heads; copies = copies || a.t[i].x != a.t[i].y; }
    const int rot_units = INTER && V > 1 ? a.rot / V : a.rot / 2 / V, units = rot_units + (copies ? (a.D - a.rot) / V : 0);
    // Heads a thread: the angles cost as much as four heads; few tokens take all the threads there are.
    const long long want = 4ll * 256 * device_compute_units();
    const int slots = (int)std::max<long long>(1, std::min<long long>(heads, std::max<long long>((heads + 7) / 8, want / std::max<long long>(1, (long long)a.M * units))));
    const long long total = (long long)a.M * slots * units;
    rope_kernel<V, INTER><<<dim3((unsigned)((total + 255) / 256)), dim3(256), 0, st>>>(a, units, rot_units, slots, (uint32_t)total);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t st) {
    if (rope_fits(a, 8)) return a.interleaved ? run<8, true>(a, st) : run<8, false>(a, st);
    if (rope_fits(a, 4)) return a.interleaved ? run<4, true>(a, st) : run<4, false>(a, st);
    if (rope_fits(a, 2)) return a.interleaved ? run<2, true>(a, st) : run<2, false>(a, st);
    return a.interleaved ? run<1, true>(a, st) : run<1, false>(a, st);
}

}  // namespace lowra
