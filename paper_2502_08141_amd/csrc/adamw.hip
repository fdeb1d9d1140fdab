// AdamW on the adapters of any number of layers at once (the optimiser of the paper's fine-tuning runs, App. H), states in 32 bits or in 8:
//   g = clip grad;   m' = b1 m + (1 - b1) g;   v' = b2 v + (1 - b2) g^2
//   w' = w - lr ((m' / (1 - b1^t)) / (sqrt(v' / (1 - b2^t)) + eps) + decay w)
// States in 8 bits are groups of 64 with their largest magnitude A: a signed code q of m stands for sgn(q) (q / 127)^2 A, a code of v for (q / 255)^4 A,
// so that the quotient m / sqrt(v) is resolved alike on both sides, and a v above zero never becomes zero.  A code is the number of borders k + 1/2, on the
// scale of q, that lie below the magnitude; a step's own weights use m' and v' before they are coded.
//
// Memory bound: 22 to 26 bytes an element with 32-bit states (30 with the bf16 copy), 18 with 8-bit ones.  A lane has four consecutive elements, so that
// every access of a wavefront is contiguous, and sixteen lanes have a group.
#include <algorithm>

#include "gemm_common.h"
#include "step.h"

namespace lowra {

namespace {

constexpr int AW_THREADS = 256, AW_STEP = 4 * AW_THREADS;    // elements a workgroup takes at a time

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
// The number of borders (k + 1/2)^P A below x MOST^P, P = 2 or 4.  In fp32 the count is right but next to a border (the quotient and the roots are
// within 2^-22, so 255.5 of them within 2^-13.9); there both sides are compared in 64 bits.
template <int P>
__device__ __forceinline__ int code_of(float x, float A, float scale, float over) {
    constexpr int MOST = P == 2 ? 127 : 255;
    float u = sqrtf(x * scale * over);
    if (P == 4) u = sqrtf(u);
    const float t = u * (float)MOST + 0.5f;
    const float whole = floorf(t), part = t - whole;
    int q = (int)fminf(whole, (float)MOST);
    if (part < 0x1p-12f || part > 1.0f - 0x1p-12f) {
        const double full = (double)x * (double)(P == 2 ? 127ll * 127 : 255ll * 255 * 255 * 255);
        auto border = [&](double k) __attribute__((always_inline)) { return (P == 2 ? k * k : (k * k) * (k * k)) * (double)A; };
        if (q > 0 && full <= border(q - 0.5)) --q;
        else if (q < MOST && full > border(q + 0.5)) ++q;
    }
    return P == 4 && x > 0.0f ? max(q, 1) : q;
}

template <bool FULL>
__device__ __forceinline__ float4 get4(const float* p, long long left) {
    if (FULL) return *reinterpret_cast<const float4*>(p);
    return make_float4(left > 0 ? p[0] : 0.0f, left > 1 ? p[1] : 0.0f, left > 2 ? p[2] : 0.0f, left > 3 ? p[3] : 0.0f);
}
template <bool FULL>
__device__ __forceinline__ void put4(float* p, long long left, const float (&v)[4]) {
    if (FULL) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); return; }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (left > i) p[i] = v[i];
}

// Four elements of an item; all 16 lanes of a group come here together.
template <bool EIGHT, bool FULL>
__device__ __forceinline__ void adamw_four(const AdamwItem& it, const AdamwStep& s, float clip, long long at) {
    const long long left = it.count - at;
    const float4 g4 = get4<FULL>(it.grad + at, left), w4 = get4<FULL>(it.weight + at, left);
    float m[4], v[4];
    if (EIGHT) {
        uint32_t mq = 0, vq = 0;
        if (FULL) {
            mq = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(it.m) + at);
            vq = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(it.v) + at);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (left > i) {
                    mq |= (uint32_t)static_cast<const uint8_t*>(it.m)[at + i] << (8 * i);
                    vq |= (uint32_t)static_cast<const uint8_t*>(it.v)[at + i] << (8 * i);
                }
        }
        const float mA = FULL || left > 0 ? it.m_absmax[at >> 6] : 0.0f, vA = FULL || left > 0 ? it.v_absmax[at >> 6] : 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = m_value((int)(int8_t)(mq >> (8 * i)), mA);
            v[i] = v_value((vq >> (8 * i)) & 0xffu, vA);
        }
    } else {
        const float4 m4 = get4<FULL>(static_cast<const float*>(it.m) + at, left), v4 = get4<FULL>(static_cast<const float*>(it.v) + at, left);
        m[0] = m4.x; m[1] = m4.y; m[2] = m4.z; m[3] = m4.w;
        v[0] = v4.x; v[1] = v4.y; v[2] = v4.z; v[3] = v4.w;
    }
    const float g[4] = {g4.x * clip, g4.y * clip, g4.z * clip, g4.w * clip};
    float w[4] = {w4.x, w4.y, w4.z, w4.w};
    const float lr = s.lr * it.lr_scale, decay = s.decay * it.decay_scale;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = s.b1 * m[i] + s.c1 * g[i];
        v[i] = s.b2 * v[i] + s.c2 * (g[i] * g[i]);
        w[i] -= lr * (m[i] / s.bias1 / (sqrtf(v[i] / s.bias2) + s.eps) + decay * w[i]);
    }
    put4<FULL>(it.weight_out + at, left, w);
    if (it.weight_bf16) {                                    // uniform
        if (FULL) *reinterpret_cast<uint2*>(it.weight_bf16 + at) = make_uint2(pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]));
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (left > i) it.weight_bf16[at + i] = (uint16_t)(pack_bf16x2(w[i], 0.0f) & 0xffffu);
        }
    }
    if (!EIGHT) {
        put4<FULL>(static_cast<float*>(it.m_out) + at, left, m);
        put4<FULL>(static_cast<float*>(it.v_out) + at, left, v);
        return;
    }
    if (!FULL) {                                             // lanes past the end have nothing in their group
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (left <= i) m[i] = v[i] = 0.0f;
    }
    const float mA = group_absmax(m), vA = group_absmax(v);
    const float ms = mA < 0x1p-60f ? 0x1p64f : 1.0f, vs = vA < 0x1p-60f ? 0x1p64f : 1.0f;         // (the quotient of small numbers: both times a power of two)
    const float mo = mA > 0.0f ? 1.0f / (mA * ms) : 0.0f, vo = vA > 0.0f ? 1.0f / (vA * vs) : 0.0f;
    uint32_t mq = 0, vq = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int q = code_of<2>(__builtin_fabsf(m[i]), mA, ms, mo);
        mq |= (uint32_t)((m[i] < 0.0f ? -q : q) & 0xff) << (8 * i);
        vq |= (uint32_t)(code_of<4>(v[i], vA, vs, vo) & 0xff) << (8 * i);
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

template <bool EIGHT>
__global__ __launch_bounds__(AW_THREADS) void adamw_kernel(const AdamwItem* __restrict__ items, const AdamwChunk* __restrict__ chunks, int chunk, AdamwStep s) {
    const AdamwChunk c = chunks[blockIdx.x];
    const AdamwItem it = items[c.item];
    const float clip = s.grad_scale ? *s.grad_scale : 1.0f;
    const long long first = c.first, last = min(first + chunk, it.count);
    const long long whole = first + (last - first) / AW_STEP * AW_STEP;
    for (long long at = first; at < whole; at += AW_STEP) adamw_four<EIGHT, true>(it, s, clip, at + 4 * threadIdx.x);
    if (whole < last) adamw_four<EIGHT, false>(it, s, clip, whole + 4 * threadIdx.x);
}

template <bool SIGNED>
__global__ __launch_bounds__(256) void adamw_state_kernel(long long count, const uint8_t* codes, const float* absmax, float* out) {
    const long long at = ((long long)blockIdx.x * 256 + threadIdx.x) * 4;
    if (at >= count) return;
    const float A = absmax[at >> 6];
    auto value = [&](uint32_t q) __attribute__((always_inline)) { return SIGNED ? m_value((int)(int8_t)q, A) : v_value(q & 0xffu, A); };
    if (at + 4 <= count) {
        const uint32_t q = *reinterpret_cast<const uint32_t*>(codes + at);
        *reinterpret_cast<float4*>(out + at) = make_float4(value(q), value(q >> 8), value(q >> 16), value(q >> 24));
        return;
    }
    for (int i = 0; at + i < count; ++i) out[at + i] = value(codes[at + i]);
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
    // enough workgroups to fill the chip several times, and no more than 16 rounds each
    g.chunk = AW_STEP * (int)std::max(1ll, std::min(16ll, total / AW_STEP / (16 * device_compute_units())));
    std::vector<AdamwChunk> chunks;
    for (size_t i = 0; i < items.size(); ++i)
        for (long long at = 0; at < items[i].count; at += g.chunk) chunks.push_back(AdamwChunk{(int)i, (uint32_t)at});
    if (chunks.size() > 0x7fffffffu) return hipErrorInvalidValue;
    g.nchunks = (int)chunks.size();
    hipError_t e = upload(items, g.d_items);
    return e != hipSuccess ? e : upload(chunks, g.d_chunks);
}

hipError_t adamw_run(const AdamwGroup (&groups)[2], const AdamwStep& s, hipStream_t st) {
    if (groups[0].nchunks) adamw_kernel<false><<<dim3((unsigned)groups[0].nchunks), dim3(AW_THREADS), 0, st>>>(groups[0].d_items, groups[0].d_chunks, groups[0].chunk, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !groups[1].nchunks) return e;
    adamw_kernel<true><<<dim3((unsigned)groups[1].nchunks), dim3(AW_THREADS), 0, st>>>(groups[1].d_items, groups[1].d_chunks, groups[1].chunk, s);
    return hipGetLastError();
}

void adamw_free(AdamwGroup (&groups)[2]) {
    for (AdamwGroup& g : groups) {
        (void)hipFree(g.d_items); (void)hipFree(g.d_chunks);
        g = AdamwGroup{};
    }
}

hipError_t launch_adamw_state(long long count, bool is_signed, const void* codes, const float* absmax, float* out, hipStream_t st) {
    const dim3 grid((unsigned)((count + 1023) / 1024)), block(256);
    if (is_signed) adamw_state_kernel<true><<<grid, block, 0, st>>>(count, static_cast<const uint8_t*>(codes), absmax, out);
    else adamw_state_kernel<false><<<grid, block, 0, st>>>(count, static_cast<const uint8_t*>(codes), absmax, out);
    return hipGetLastError();
}

}  // namespace lowra
