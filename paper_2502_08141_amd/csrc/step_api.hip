// C ABI of the operators of a training step beside the linear: host-side validation and dispatch.
#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/lowra.h"
#include "api_util.h"
#include "step.h"

namespace {

lowra_status launched(hipError_t e) { return e == hipSuccess ? LOWRA_OK : LOWRA_HIP_ERROR; }
constexpr int kMaxSize = 1 << 30;

}  // namespace

extern "C" {

// ---- norms
static bool norm_sizes(int M, int N) { return N % 8 == 0 && M <= kMaxSize && N <= lowra::kNormMaxColumns; }
static bool norm_kind(int kind) { return kind == LOWRA_NORM_LAYER || kind == LOWRA_NORM_RMS; }

lowra_status lowra_norm_fwd(int M, int N, int kind, const uint16_t* x, const uint16_t* weight, const uint16_t* bias, float eps, uint16_t* y, void* stream) {
    if (M < 0 || N < 0 || !norm_kind(kind) || !(eps >= 0.0f)) return LOWRA_INVALID_ARG;
    if (!norm_sizes(M, N)) return LOWRA_UNSUPPORTED;
    if (M == 0 || N == 0) return LOWRA_OK;
    if (!x || !y) return LOWRA_INVALID_ARG;
    if (!aligned16(x) || !aligned16(weight) || !aligned16(bias) || !aligned16(y)) return LOWRA_MISALIGNED;
    const size_t size = (size_t)M * N * 2, row = (size_t)N * 2;
    if (outputs_overlap({Span{y, size}}, {Span{x, size}, Span{weight, row}, Span{bias, row}})) return LOWRA_INVALID_ARG;
    lowra::NormArgs a{};
    a.M = M; a.N = N; a.rms = kind == LOWRA_NORM_RMS; a.eps = eps; a.x = x; a.weight = weight; a.bias = bias; a.y = y;
    return launched(lowra::launch_norm_fwd(a, static_cast<hipStream_t>(stream)));
}

size_t lowra_norm_bwd_workspace_bytes(int M, int N) { return M > 0 && N > 0 && norm_sizes(M, N) ? lowra::norm_bwd_workspace_bytes(M, N) : 0; }

lowra_status lowra_norm_bwd(int M, int N, int kind, const uint16_t* dY, const uint16_t* x, const uint16_t* weight, float eps, const uint16_t* residual,
                            uint16_t* dX, float* dweight, float* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 0 || N < 0 || !norm_kind(kind) || !(eps >= 0.0f) || (!dX && !dweight && !dbias) || (residual && !dX)) return LOWRA_INVALID_ARG;
    if (!norm_sizes(M, N)) return LOWRA_UNSUPPORTED;
    if (N == 0) return LOWRA_OK;
    if (!aligned16(dweight) || !aligned16(dbias)) return LOWRA_MISALIGNED;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (M == 0) {                                                 // empty sums, written by a fill kernel (no memset node, so the call can be captured)
        for (float* out : {dweight, dbias})
            if (out && lowra::launch_zero_bf16(reinterpret_cast<uint16_t*>(out), (size_t)N * 2, st) != hipSuccess) return LOWRA_HIP_ERROR;
        return LOWRA_OK;
    }
    if (!dY || !x) return LOWRA_INVALID_ARG;
    if (!aligned16(dY) || !aligned16(x) || !aligned16(weight) || !aligned16(residual) || !aligned16(dX)) return LOWRA_MISALIGNED;
    const size_t need = dweight || dbias ? lowra::norm_bwd_workspace_bytes(M, N) : 0;
    if (need > 0) {
        if (!workspace) return LOWRA_INVALID_ARG;
        if (!aligned16(workspace)) return LOWRA_MISALIGNED;
        if (workspace_bytes < need) return LOWRA_WORKSPACE_TOO_SMALL;
    }
    const size_t size = (size_t)M * N * 2, row = (size_t)N * 2;
    if (outputs_overlap({Span{dX, size}, Span{dweight, 2 * row}, Span{dbias, 2 * row}, Span{workspace, need}},
                        {Span{residual, size}, Span{dY, size}, Span{x, size}, Span{weight, row}})) return LOWRA_INVALID_ARG;
    lowra::NormArgs a{};
    a.M = M; a.N = N; a.rms = kind == LOWRA_NORM_RMS; a.eps = eps; a.x = x; a.weight = weight; a.dY = dY; a.residual = residual; a.dX = dX;
    return launched(lowra::launch_norm_bwd(a, dweight, dbias, workspace, st));
}

// ---- rotary positions
lowra_status lowra_rope_frequencies(int rot, double base, int scaling, double factor, int original, double low, double high, uint64_t* turns_host) {
    if (!turns_host || rot <= 0 || !(base > 1.0) || !std::isfinite(base)) return LOWRA_INVALID_ARG;
    if (rot % 2 != 0 || rot > 1 << 20) return LOWRA_UNSUPPORTED;
    if (scaling < LOWRA_ROPE_SCALE_NONE || scaling > LOWRA_ROPE_SCALE_INDEX) return LOWRA_INVALID_ARG;
    if (scaling != LOWRA_ROPE_SCALE_NONE && !(factor >= 1.0 && std::isfinite(factor))) return LOWRA_INVALID_ARG;
    if (scaling >= LOWRA_ROPE_SCALE_TURNS && !(original > 0 && low > 0.0 && high > low && std::isfinite(high))) return LOWRA_INVALID_ARG;
    if (scaling == LOWRA_ROPE_SCALE_BASE) {
        if (rot == 2) return LOWRA_UNSUPPORTED;                   // one pair has no slower one to stretch towards
        base *= std::pow(factor, (double)rot / (rot - 2));
    }
    const double tau = 6.283185307179586476925;
    // the pair that turns `turns` times in the original context, as a place in the list of pairs
    auto place = [&](double turns) { return rot * std::log(original / (tau * turns)) / (2.0 * std::log(base)); };
    double first = 0.0, last = 0.0;
    if (scaling == LOWRA_ROPE_SCALE_INDEX) {
        first = std::max(std::floor(place(high)), 0.0);
        last = std::min(std::ceil(place(low)), rot - 1.0);
    }
    for (int j = 0; j < rot / 2; ++j) {
        double f = std::pow(base, -2.0 * j / rot);
        if (scaling == LOWRA_ROPE_SCALE_LINEAR) f /= factor;
        if (scaling >= LOWRA_ROPE_SCALE_TURNS) {
            double keep = scaling == LOWRA_ROPE_SCALE_TURNS ? (original * f / tau - low) / (high - low) : 1.0 - (j - first) / std::max(last - first, 1e-3);
            keep = std::min(std::max(keep, 0.0), 1.0);
            f *= keep + (1.0 - keep) / factor;
        }
        turns_host[j] = (uint64_t)std::llround(std::ldexp(f / tau, 64));   // f <= 1 radian: below a sixth of a turn
    }
    return LOWRA_OK;
}

// A tensor's elements: tokens one after another with their heads in between, or heads one after another with their tokens in between.
struct RopeSpan {
    uintptr_t p;
    uint64_t bytes, window, token;       // all of it; a token's heads; from token to token (0: heads one after another)
};
static bool rope_span(const void* p, int M, int heads, int D, int64_t token, int64_t head, bool out, RopeSpan& s) {
    const int64_t most = (int64_t)1 << 60;
    if (token < 0 || head < 0 || (M > 1 && token > most / M) || (heads > 1 && head > most / heads)) return false;
    const int64_t tokens = M > 1 ? token * (M - 1) : 0, row = heads > 1 ? head * (heads - 1) : 0;
    s.p = reinterpret_cast<uintptr_t>(p);
    s.bytes = 2 * (uint64_t)(tokens + row + D);
    s.window = 2 * (uint64_t)(row + D);
    const bool by_token = M == 1 || token >= row + D, heads_apart = heads == 1 || head >= D;
    const bool by_head = (M == 1 || token >= D) && (heads == 1 || head >= tokens + D);
    s.token = by_token && M > 1 ? 2 * (uint64_t)token : 0;
    return !out || (by_token && heads_apart) || by_head;
}
static bool rope_overlap(const RopeSpan& a, const RopeSpan& b) {
    if (a.p >= b.p + b.bytes || b.p >= a.p + a.bytes) return false;
    if (a.token == 0 || a.token != b.token) return true;         // interleaved in another way than row by row: not told apart
    const uint64_t d = b.p >= a.p ? (b.p - a.p) % a.token : (a.token - (a.p - b.p) % a.token) % a.token;       // b's rows behind a's
    return d < a.window || d + b.window > a.token;
}

lowra_status lowra_rope(int n, const lowra_rope_tensor* tensors, int M, int D, int rot, int layout, const int32_t* positions, const uint64_t* turns, float magnitude,
                        int inverse, void* stream) {
    if (n <= 0 || !tensors || M < 0 || D <= 0 || rot <= 0 || rot > D || (layout != LOWRA_ROPE_HALF && layout != LOWRA_ROPE_INTERLEAVED)) return LOWRA_INVALID_ARG;
    if (n > lowra::kRopeMaxTensors || rot % 2 != 0 || M > kMaxSize || D > 1 << 20) return LOWRA_UNSUPPORTED;
    lowra::RopeArgs a{};
    RopeSpan in[lowra::kRopeMaxTensors], out[lowra::kRopeMaxTensors];
    a.n = n; a.M = M; a.D = D; a.rot = rot; a.interleaved = layout == LOWRA_ROPE_INTERLEAVED; a.inverse = inverse != 0;
    a.positions = positions; a.turns = turns; a.magnitude = magnitude;
    long long heads = 0;
    for (int i = 0; i < n; ++i) {
        const lowra_rope_tensor& t = tensors[i];
        if (t.heads <= 0) return LOWRA_INVALID_ARG;
        heads += t.heads;
        a.t[i] = lowra::RopeTensor{t.x, t.y, t.heads, t.x_token_stride, t.x_head_stride, t.y_token_stride, t.y_head_stride};
    }
    if (heads > 1 << 20 || (long long)M * heads > (1ll << 32) / D) return LOWRA_UNSUPPORTED;       // (a launch has less than 2^32 threads, of two elements at least)
    if (M == 0) return LOWRA_OK;
    if (!positions || !turns) return LOWRA_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(positions) & 3u) || (reinterpret_cast<uintptr_t>(turns) & 7u)) return LOWRA_MISALIGNED;
    for (int i = 0; i < n; ++i) {
        const lowra_rope_tensor& t = tensors[i];
        if (!t.x || !t.y) return LOWRA_INVALID_ARG;
        if ((reinterpret_cast<uintptr_t>(t.x) | reinterpret_cast<uintptr_t>(t.y)) & 1u) return LOWRA_MISALIGNED;
        if (!rope_span(t.x, M, t.heads, D, t.x_token_stride, t.x_head_stride, false, in[i]) ||
            !rope_span(t.y, M, t.heads, D, t.y_token_stride, t.y_head_stride, true, out[i])) return LOWRA_INVALID_ARG;
    }
    const Span pos{positions, (size_t)M * 4}, freq{turns, (size_t)rot * 4};
    for (int i = 0; i < n; ++i) {
        const lowra_rope_tensor& t = tensors[i];
        const Span mine{t.y, (size_t)out[i].bytes};
        if (overlap(mine, pos) || overlap(mine, freq)) return LOWRA_INVALID_ARG;
        for (int k = 0; k < n; ++k) {
            const bool in_place = k == i && t.x == t.y && (t.x_token_stride == t.y_token_stride || M == 1) && (t.x_head_stride == t.y_head_stride || t.heads == 1);
            if (!in_place && rope_overlap(out[i], in[k])) return LOWRA_INVALID_ARG;
            if (k < i && rope_overlap(out[i], out[k])) return LOWRA_INVALID_ARG;
        }
    }
    return launched(lowra::launch_rope(a, static_cast<hipStream_t>(stream)));
}

// ---- AdamW
static bool adamw_overlaps(int n, const lowra_adamw_item* items) {
    struct Range { uintptr_t from, to; bool out; };
    std::vector<Range> v;
    for (int i = 0; i < n; ++i) {
        const lowra_adamw_item& it = items[i];
        const size_t count = (size_t)it.count, state = it.state_bits == 8 ? count : 4 * count, groups = it.state_bits == 8 ? (count + 63) / 64 * 4 : 0;
        auto add = [&](const void* p, size_t bytes, bool out) {
            if (p && bytes) v.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, out});
        };
        auto pair = [&](const void* in, const void* out, size_t bytes) {          // an output, and the input that it may replace
            if (in != out) add(in, bytes, false);
            add(out, bytes, true);
        };
        add(it.grad, 4 * count, false);
        pair(it.m, it.m_out, state); pair(it.v, it.v_out, state);
        pair(it.m_absmax, it.m_absmax_out, groups); pair(it.v_absmax, it.v_absmax_out, groups);
        pair(it.weight, it.weight_out, 4 * count);
        add(it.weight_bf16, 2 * count, true);
    }
    std::sort(v.begin(), v.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t any = 0, out = 0;                                   // how far what came before reaches
    for (const Range& r : v) {
        if (r.from < out || (r.out && r.from < any)) return true;
        any = std::max(any, r.to);
        if (r.out) out = std::max(out, r.to);
    }
    return false;
}

lowra_status lowra_adamw_batch_create(int n, const lowra_adamw_item* items, lowra_adamw_batch** out) {
    if (!out) return LOWRA_INVALID_ARG;
    *out = nullptr;
    if (n <= 0 || !items) return LOWRA_INVALID_ARG;
    for (int i = 0; i < n; ++i) {
        const lowra_adamw_item& it = items[i];
        if (it.count <= 0) return LOWRA_INVALID_ARG;
        if (it.count > (int64_t)1 << 31 || (it.state_bits != 8 && it.state_bits != 32)) return LOWRA_UNSUPPORTED;
        if (!it.grad || !it.m || !it.v || !it.weight || !it.m_out || !it.v_out || !it.weight_out) return LOWRA_INVALID_ARG;
        const void* scales[] = {it.m_absmax, it.v_absmax, it.m_absmax_out, it.v_absmax_out};
        for (const void* s : scales) {
            if ((s != nullptr) != (it.state_bits == 8)) return LOWRA_INVALID_ARG;
            if (reinterpret_cast<uintptr_t>(s) & 3u) return LOWRA_MISALIGNED;
        }
        if (!aligned16(it.grad) || !aligned16(it.m) || !aligned16(it.v) || !aligned16(it.weight) || !aligned16(it.m_out) || !aligned16(it.v_out) ||
            !aligned16(it.weight_out) || !aligned16(it.weight_bf16))
            return LOWRA_MISALIGNED;
    }
    long long pieces = 0;                                        // (a launch has less than 2^32 threads, 256 to a thousand elements at least)
    for (int i = 0; i < n; ++i) pieces += (items[i].count + 1023) / 1024;
    if (pieces >= 1 << 24) return LOWRA_UNSUPPORTED;
    lowra_adamw_batch* b = nullptr;
    lowra_status st = LOWRA_OK;
    try {
        if (adamw_overlaps(n, items)) return LOWRA_INVALID_ARG;
        std::vector<lowra::AdamwItem> by[2];
        for (int i = 0; i < n; ++i) {
            const lowra_adamw_item& it = items[i];
            by[it.state_bits == 8].push_back(lowra::AdamwItem{it.grad, it.m, it.v, it.m_absmax, it.v_absmax, it.weight, it.m_out, it.v_out, it.m_absmax_out,
                                                              it.v_absmax_out, it.weight_out, it.weight_bf16, it.count, it.lr_scale, it.decay_scale});
        }
        b = new lowra_adamw_batch;
        if (hipGetDevice(&b->device) != hipSuccess || lowra::adamw_build(by[0], false, b->groups[0]) != hipSuccess ||
            lowra::adamw_build(by[1], true, b->groups[1]) != hipSuccess)
            st = LOWRA_HIP_ERROR;
    } catch (const std::bad_alloc&) {
        st = LOWRA_OUT_OF_MEMORY;
    } catch (...) {
        st = LOWRA_INVALID_ARG;
    }
    if (st != LOWRA_OK) { (void)hipGetLastError(); lowra_adamw_batch_destroy(b); return st; }
    *out = b;
    return LOWRA_OK;
}

lowra_status lowra_adamw_batch_run(const lowra_adamw_batch* b, const lowra_adamw_step* s, const float* grad_scale, void* stream) {
    if (!b || !s || s->step < 1 || !(s->beta_one >= 0.0 && s->beta_one < 1.0) || !(s->beta_two >= 0.0 && s->beta_two < 1.0) || !(s->eps >= 0.0)) return LOWRA_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(grad_scale) & 3u) return LOWRA_MISALIGNED;
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) return LOWRA_HIP_ERROR;
    if (dev != b->device) return LOWRA_INVALID_ARG;
    // (1 - beta^t by expm1 and log: a beta next to one keeps its digits)
    auto over_bias = [&](double beta) { return beta > 0.0 ? (float)(-1.0 / std::expm1((double)s->step * std::log(beta))) : 1.0f; };
    // (an eps that the kernel's reciprocal takes for zero would make NaN of 0 / (0 + eps), and is nothing beside any other root)
    const float eps = s->eps > 0.0 ? std::max((float)s->eps, 0x1p-126f) : 0.0f;
    const lowra::AdamwStep a{(float)s->lr, (float)s->beta_one, (float)(1.0 - s->beta_one), (float)s->beta_two, (float)(1.0 - s->beta_two), over_bias(s->beta_one), over_bias(s->beta_two),
                             eps, (float)s->weight_decay, grad_scale};
    return launched(lowra::adamw_run(b->groups, a, static_cast<hipStream_t>(stream)));
}

void lowra_adamw_batch_destroy(lowra_adamw_batch* b) {
    if (!b) return;
    lowra::adamw_free(b->groups);
    delete b;
}

lowra_status lowra_adamw_state(int64_t count, int is_signed, const void* codes, const float* absmax, float* out, void* stream) {
    if (count < 0) return LOWRA_INVALID_ARG;
    if (count > (int64_t)1 << 33) return LOWRA_UNSUPPORTED;
    if (count == 0) return LOWRA_OK;
    if (!codes || !absmax || !out) return LOWRA_INVALID_ARG;
    if (!aligned16(codes) || !aligned16(out) || (reinterpret_cast<uintptr_t>(absmax) & 3u)) return LOWRA_MISALIGNED;
    const size_t size = (size_t)count;
    if (outputs_overlap({Span{nullptr, 0}, Span{out, 4 * size}}, {Span{codes, size}, Span{absmax, (size + 63) / 64 * 4}})) return LOWRA_INVALID_ARG;
    return launched(lowra::launch_adamw_state(count, is_signed != 0, codes, absmax, out, static_cast<hipStream_t>(stream)));
}

// ---- loss over the vocabulary
static bool loss_sizes(int M, int V, int K) { return K % 8 == 0 && M <= kMaxSize && V <= 1 << 21 && K <= 1 << 20; }

size_t lowra_vocab_loss_workspace_bytes(int M, int V, int K, int grad) {
    return M > 0 && V > 0 && K > 0 && loss_sizes(M, V, K) ? lowra::vocab_loss_workspace_bytes(M, V, K, grad != 0) : 0;
}

lowra_status lowra_vocab_loss(int M, int V, int K, const uint16_t* h, const uint16_t* W, const int32_t* targets, const float* weights, float* loss, float* lse, uint16_t* dH,
                              void* workspace, size_t workspace_bytes, void* stream) {
    if (M < 0 || V <= 0 || K <= 0) return LOWRA_INVALID_ARG;
    if (!loss_sizes(M, V, K)) return LOWRA_UNSUPPORTED;
    if (M == 0) return LOWRA_OK;
    if (!h || !W || !targets || !loss) return LOWRA_INVALID_ARG;
    if (!aligned16(h) || !aligned16(W) || !aligned16(targets) || !aligned16(weights) || !aligned16(loss) || !aligned16(lse) || !aligned16(dH)) return LOWRA_MISALIGNED;
    const size_t need = lowra::vocab_loss_workspace_bytes(M, V, K, dH != nullptr);
    if (!workspace) return LOWRA_INVALID_ARG;
    if (!aligned16(workspace)) return LOWRA_MISALIGNED;
    if (workspace_bytes < need) return LOWRA_WORKSPACE_TOO_SMALL;
    const size_t rows = (size_t)M * 4, hs = (size_t)M * K * 2;
    if (outputs_overlap({Span{nullptr, 0}, Span{loss, rows}, Span{lse, rows}, Span{dH, hs}, Span{workspace, need}},
                        {Span{h, hs}, Span{W, (size_t)V * K * 2}, Span{targets, rows}, Span{weights, rows}})) return LOWRA_INVALID_ARG;
    return launched(lowra::launch_vocab_loss(lowra::VocabLossArgs{M, V, K, h, W, targets, weights, loss, lse, dH, workspace}, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
