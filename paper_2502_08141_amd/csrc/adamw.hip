// AdamW on the adapters of any number of layers at once (the optimiser of the paper's fine-tuning runs, App. H), states in 32 bits or in 8:
//   g = clip grad;   m' = b1 m + (1 - b1) g;   v' = b2 v + (1 - b2) g^2
//   w' = w - lr ((m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps) + decay w)
// States in 8 bits are groups of 64 with their largest magnitude A: a signed code q of m stands for sgn(q) (q / 127)^2 A, a code of v for (q / 255)^4 A,
// so that the quotient m / sqrt(v) is resolved alike on both sides, and a v above zero never becomes zero.  A code is the number of borders k + 1/2, on the
// scale of q, that lie below the magnitude; a step's own weights use m' and v' before they are coded.
//
// Memory bound: 28 bytes an element with 32-bit states (30 with the bf16 copy), 18.25 with 8-bit ones and the copy.  143 million elements in 8 bits: 481 us, 5.4 TB/s
// (without the coding it takes as long).  A lane has four consecutive elements, so that
// every access of a wavefront is contiguous, and sixteen lanes have a group.
#include <algorithm>

#include "gemm_common.h"
#include "step.h"

namespace lowra {

namespace {

constexpr int AW_THREADS = 256, AW_STEP = 4 * AW_THREADS;    // elements a workgroup takes at a time
constexpr int AW_MOST = 4;                                   // and how often, with all loads of these in flight together
constexpr int AW_AHEAD = 4;                                  // loads of codes in flight where they are only decoded

__device__ __forceinline__ float m_value(int q, float A) {
    const float u = (float)q * (float)(1.0 / 127.0);
    return u * __builtin_fabsf(u) * A;
}
__device__ __forceinline__ float v_value(uint32_t q, float A) {
    const float u = (float)q * (float)(1.0 / 255.0), s = u * u;
    return s * s * A;
}
// The group's largest magnitude, over sixteen lanes: as bit patterns, above which NaN lie, so that one is kept.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_umax(uint32_t x) { return max(x, (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)x, CTRL, 0xf, 0xf, true)); }
__device__ __forceinline__ float group_absmax(const float (&x)[4]) {
    uint32_t b = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) b = max(b, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffffu);
    b = dpp_umax<0xB1>(b);                                   // quad_perm [1,0,3,2]
    b = dpp_umax<0x4E>(b);                                   // quad_perm [2,3,0,1]
    b = dpp_umax<0x124>(b);                                  // row_ror:4
    b = dpp_umax<0x128>(b);                                  // row_ror:8
    return __builtin_bit_cast(float, b);
}
// The numbers of borders (k + 1/2)^P A below x MOST^P, P = 2 or 4.  In fp32 (quotient, roots and sum to one ulp) the count is right but next to a border:
// 255.5 roots are less than 2^-14 off.  There both sides are compared in 64 bits; a wavefront has such a place in one of eight times.
template <int P>
__device__ __forceinline__ void codes_of(const float (&x)[4], float A, float (&q)[4]) {
    constexpr float MOST = P == 2 ? 127.0f : 255.0f;
    const bool tiny = A < 0x1p-120f;                         // (the reciprocal would be none)
    float over = A > 0.0f ? __builtin_amdgcn_rcpf(tiny ? A * 0x1p30f : A) : 0.0f, worst = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float u = __builtin_fabsf(x[i]) * over;
        if (__any(tiny)) u = tiny ? __builtin_fabsf(x[i]) * 0x1p30f * over : u;
        u = __builtin_amdgcn_sqrtf(u);
        if (P == 4) u = __builtin_amdgcn_sqrtf(u);
        const float t = __builtin_fmaf(u, MOST, 0.5f), part = __builtin_amdgcn_fractf(t);
        q[i] = t - part;
        worst = fmaxf(worst, __builtin_fabsf(part - 0.5f));
    }
    if (worst > 0.5f - 0x1p-12f) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double full = (double)__builtin_fabsf(x[i]) * (double)(P == 2 ? 127ll * 127 : 255ll * 255 * 255 * 255);
            auto border = [&](double k) __attribute__((always_inline)) { return (P == 2 ? k * k : (k * k) * (k * k)) * (double)A; };
            if (q[i] > 0.0f && full <= border((double)q[i] - 0.5)) q[i] -= 1.0f;
            else if (q[i] < MOST && full > border((double)q[i] + 0.5)) q[i] += 1.0f;
        }
    }
}

// The root to one ulp, of subnormal numbers as well (v_sqrt_f32 takes those for zero); the IEEE one is fifteen instructions.
__device__ __forceinline__ float root_of(float x) {
    const bool tiny = x < 0x1p-96f;
    return __builtin_amdgcn_sqrtf(tiny ? x * 0x1p64f : x) * (tiny ? 0x1p-32f : 1.0f);
}

// STREAM: past the caches, for batches that none of them holds (below, at adamw_build)
template <bool FULL, bool STREAM>
__device__ __forceinline__ float4 get4(const float* p, long long left) {
    if (FULL) return STREAM ? load16_stream(reinterpret_cast<const float4*>(p)) : *reinterpret_cast<const float4*>(p);
    return make_float4(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, left > 3 ? p[3] : 0.0f);
}
template <bool FULL, bool STREAM>
__device__ __forceinline__ void put4(float* p, long long left, const float (&v)[4]) {
    if (FULL && STREAM) { store16_stream(p, make_float4(v[0], v[1], v[2], v[3])); return; }
    if (FULL) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (left > i) p[i] = v[i];
}

// Four elements of an item as they lie in memory
struct Quad { float4 g, w, m, v; uint32_t mq, vq; float mA, vA; };
template <bool EIGHT, bool FULL, bool STREAM>
__device__ __forceinline__ void adamw_load(const AdamwItem& it, long long at, Quad& q) {
    const long long left = it.count - at;
    q.g = get4<FULL, STREAM>(it.grad + at, left);
    q.w = get4<FULL, STREAM>(it.weight + at, left);
    if (!EIGHT) {
        q.m = get4<FULL, STREAM>(static_cast<const float*>(it.m) + at, left);
        q.v = get4<FULL, STREAM>(static_cast<const float*>(it.v) + at, left);
        return;
    }
    const uint8_t *m = static_cast<const uint8_t*>(it.m) + at, *v = static_cast<const uint8_t*>(it.v) + at;
    if (FULL) {
        q.mq = *reinterpret_cast<const uint32_t*>(m);
        q.vq = *reinterpret_cast<const uint32_t*>(v);
    } else {
        q.mq = q.vq = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (left > i) { q.mq |= (uint32_t)m[i] << (8 * i); q.vq |= (uint32_t)v[i] << (8 * i); }
    }
    q.mA = FULL || left > 0 ? it.m_absmax[at >> 6] : 0.0f;
    q.vA = FULL || left > 0 ? it.v_absmax[at >> 6] : 0.0f;
}

// All 16 lanes of a group come here together.
template <bool EIGHT, bool FULL, bool STREAM>
__device__ __forceinline__ void adamw_four(const AdamwItem& it, const AdamwStep& s, float clip, long long at, const Quad& r) {
    const long long left = it.count - at;
    float m[4], v[4];
    if (EIGHT) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m_value((int)(int8_t)(r.mq >> (8 * i)), r.mA);
            v[i] = v_value((r.vq >> (8 * i)) & 0xffu, r.vA);
        }
    } else {
        m[0] = r.m.x; m[1] = r.m.y; m[2] = r.m.z; m[3] = r.m.w;
        v[0] = r.v.x; v[1] = r.v.y; v[2] = r.v.z; v[3] = r.v.w;
    }
    const float g[4] = {r.g.x * clip, r.g.y * clip, r.g.z * clip, r.g.w * clip};
    float w[4] = {r.w.x, r.w.y, r.w.z, r.w.w};
    const float lr = s.lr * it.lr_scale, lr_m = lr * s.over_bias1, lr_w = lr * (s.decay * it.decay_scale);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = s.b1 * m[i] + s.c1 * g[i];
        v[i] = s.b2 * v[i] + s.c2 * (g[i] * g[i]);
        const float root = s.eps >= 1e-12f ? __builtin_amdgcn_sqrtf(v[i] * s.over_bias2) : root_of(v[i] * s.over_bias2);      // (uniform; the root of what is subnormal is below 1e-19)
        w[i] = __builtin_fmaf(-lr_w, w[i], w[i]) - lr_m * m[i] * __builtin_amdgcn_rcpf(root + s.eps);
    }
    put4<FULL, STREAM>(it.weight_out + at, left, w);
    if (it.weight_bf16) {                                    // uniform
        if (FULL) *reinterpret_cast<uint2*>(it.weight_bf16 + at) = make_uint2(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]));
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (left > i) it.weight_bf16[at + i] = (uint16_t)(pack_bf16x2(w[i], 0.0f) & 0xffffu);
        }
    }
    if (!EIGHT) {
        put4<FULL, STREAM>(static_cast<float*>(it.m_out) + at, left, m);
        put4<FULL, STREAM>(static_cast<float*>(it.v_out) + at, left, v);
        return;
    }
    if (!FULL) {                                             // lanes past the end have nothing in their group
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (left <= i) m[i] = v[i] = 0.0f;
    }
    const float mA = group_absmax(m), vA = group_absmax(v);
    float mc[4], vc[4];
    codes_of<2>(m, mA, mc);
    codes_of<4>(v, vA, vc);
    uint32_t mq = 0, vq = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        mq |= ((uint32_t)(int)(m[i] < 0.0f ? -mc[i] : mc[i]) & 0xffu) << (8 * i);
        vq |= ((uint32_t)(int)fmaxf(vc[i], v[i] > 0.0f ? 1.0f : 0.0f) & 0xffu) << (8 * i);
    }
    if (FULL) {
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(it.m_out) + at) = mq;
        *reinterpret_cast<uint32_t*>(static_cast<uint8_t*>(it.v_out) + at) = vq;
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (left > i) {
                static_cast<uint8_t*>(it.m_out)[at + i] = (uint8_t)(mq >> (8 * i));
                static_cast<uint8_t*>(it.v_out)[at + i] = (uint8_t)(vq >> (8 * i));
            }
    }
    if ((threadIdx.x & 15) == 0 && (FULL || left > 0)) {
        it.m_absmax_out[at >> 6] = mA;
        it.v_absmax_out[at >> 6] = vA;
    }
}

// STEPS: how often a workgroup takes AW_STEP elements
template <bool EIGHT, bool STREAM, int STEPS>
__global__ __launch_bounds__(AW_THREADS) void adamw_kernel(const AdamwItem* __restrict__ items, const AdamwChunk* __restrict__ chunks, AdamwStep s) {
    const AdamwChunk c = chunks[blockIdx.x];
    const AdamwItem it = items[c.item];
    const float clip = s.grad_scale ? *s.grad_scale : 1.0f;
    const long long first = (long long)c.first + 4 * threadIdx.x;
    if ((long long)c.first + STEPS * AW_STEP <= it.count) {  // uniform; all loads together
        Quad q[STEPS];
#pragma unroll
        for (int k = 0; k < STEPS; ++k) adamw_load<EIGHT, true, STREAM>(it, first + k * AW_STEP, q[k]);
#pragma unroll
        for (int k = 0; k < STEPS; ++k) adamw_four<EIGHT, true, STREAM>(it, s, clip, first + k * AW_STEP, q[k]);
        return;
    }
#pragma unroll 1
    for (int k = 0; k < STEPS && (long long)c.first + k * AW_STEP < it.count; ++k) {       // an item's end
        Quad q;
        adamw_load<EIGHT, false, STREAM>(it, first + k * AW_STEP, q);
        adamw_four<EIGHT, false, STREAM>(it, s, clip, first + k * AW_STEP, q);
    }
}

template <bool SIGNED>
__global__ __launch_bounds__(256) void adamw_state_kernel(long long count, const uint8_t* codes, const float* absmax, float* out) {
    const long long first = (long long)blockIdx.x * (1024 * AW_AHEAD) + 4 * threadIdx.x;
    auto value = [](uint32_t q, float A) __attribute__((always_inline)) { return SIGNED ? m_value((int)(int8_t)q, A) : v_value(q & 0xffu, A); };
    uint32_t q[AW_AHEAD];
    float A[AW_AHEAD];
#pragma unroll
    for (int k = 0; k < AW_AHEAD; ++k) {
        const long long at = first + 1024 * k;
        q[k] = at + 4 <= count ? *reinterpret_cast<const uint32_t*>(codes + at) : 0u;
        A[k] = at < count ? absmax[at >> 6] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < AW_AHEAD; ++k) {
        const long long at = first + 1024 * k;
        if (at + 4 <= count) store16_stream(out + at, make_float4(value(q[k], A[k]), value(q[k] >> 8, A[k]), value(q[k] >> 16, A[k]), value(q[k] >> 24, A[k])));
        else
            for (int i = 0; at + i < count; ++i) out[at + i] = value(codes[at + i], A[k]);
    }
}

template <class T>
hipError_t upload(const std::vector<T>& v, T*& d) {
    hipError_t e = hipMalloc(reinterpret_cast<void**>(&d), v.size() * sizeof(T));
    return e != hipSuccess ? e : hipMemcpy(d, v.data(), v.size() * sizeof(T), hipMemcpyHostToDevice);
}

}  // namespace

hipError_t adamw_build(const std::vector<AdamwItem>& items, bool eight, AdamwGroup& g) {
    if (items.empty()) return hipSuccess;
    long long total = 0;
    for (const AdamwItem& it : items) total += it.count;
    // A batch that reads and writes more than 128 MB, half of what the 256 MB behind the caches hold, goes past the caches, and a workgroup asks for AW_MOST rounds together: 32-bit
    // states of 201 MB 47 us through the caches and 43.5 in single rounds, 40.3 so; of 268 MB 57.6 in single rounds, 53.2 so; 8-bit states of 327 MB, two decodings with them, 98 and 91.
    // Below, workgroups of one round are as soon done or sooner (8-bit states of 82 MB 30.0 -> 27.4, 32-bit ones of 37 MB 8.4 -> 7.0).
    g.large = total * (eight ? 18 : 30) > (128ll << 20);
    const int chunk = (g.large ? AW_MOST : 1) * AW_STEP;
    std::vector<AdamwChunk> chunks;
    for (size_t i = 0; i < items.size(); ++i)
        for (long long at = 0; at < items[i].count; at += chunk) chunks.push_back(AdamwChunk{(int)i, (uint32_t)at});
    g.nchunks = (int)chunks.size();
    hipError_t e = upload(items, g.d_items);
    return e != hipSuccess ? e : upload(chunks, g.d_chunks);
}

template <bool EIGHT>
static hipError_t adamw_launch(const AdamwGroup& g, const AdamwStep& s, hipStream_t st) {
    if (!g.nchunks) return hipSuccess;
    const dim3 grid((unsigned)g.nchunks), block(AW_THREADS);
    if (g.large) adamw_kernel<EIGHT, true, AW_MOST><<<grid, block, 0, st>>>(g.d_items, g.d_chunks, s);
    else adamw_kernel<EIGHT, false, 1><<<grid, block, 0, st>>>(g.d_items, g.d_chunks, s);
    return hipGetLastError();
}
hipError_t adamw_run(const AdamwGroup (&groups)[2], const AdamwStep& s, hipStream_t st) {
    const hipError_t e = adamw_launch<false>(groups[0], s, st);
    return e != hipSuccess ? e : adamw_launch<true>(groups[1], s, st);
}

void adamw_free(AdamwGroup (&groups)[2]) {
    for (AdamwGroup& g : groups) {
        (void)hipFree(g.d_items); (void)hipFree(g.d_chunks);
        g = AdamwGroup{};
    }
}

hipError_t launch_adamw_state(long long count, bool is_signed, const void* codes, const float* absmax, float* out, hipStream_t st) {
    const dim3 grid((unsigned)((count + 1024 * AW_AHEAD - 1) / (1024 * AW_AHEAD))), block(256);
    if (is_signed) adamw_state_kernel<true><<<grid, block, 0, st>>>(count, static_cast<const uint8_t*>(codes), absmax, out);
    else adamw_state_kernel<false><<<grid, block, 0, st>>>(count, static_cast<const uint8_t*>(codes), absmax, out);
    return hipGetLastError();
}

}  // namespace lowra
