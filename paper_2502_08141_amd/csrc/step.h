// The operators of a training step beside the linear: norms, rotary positions, the loss over the vocabulary, AdamW.  Arguments and launchers;
// each launcher validates nothing (the C ABI did) and returns the launch status.
#pragma once
#include "lowra_host.h"

namespace lowra {

// ---- norms (norm.hip)
constexpr int kNormMaxColumns = 16384;          // a row's registers: sixteen wavefronts with two runs of eight columns a lane
struct NormArgs {
    int M, N, rms;
    float eps;
    const uint16_t *x, *weight, *bias, *dY, *residual;
    uint16_t *y, *dX;
};
size_t norm_bwd_workspace_bytes(int M, int N);
hipError_t launch_norm_fwd(const NormArgs& a, hipStream_t st);
hipError_t launch_norm_bwd(const NormArgs& a, float* dweight, float* dbias, void* workspace, hipStream_t st);

// ---- rotary positions (rope.hip)
constexpr int kRopeMaxTensors = 4;
struct RopeTensor {
    const uint16_t* x;
    uint16_t* y;
    int heads;
    int64_t x_token, x_head, y_token, y_head;   // strides in elements
};
struct RopeArgs {
    RopeTensor t[kRopeMaxTensors];
    int n, M, D, rot, interleaved, inverse;
    const int32_t* positions;
    const uint64_t* turns;                      // [rot / 2]: 2^-64 of a full turn a position
    float magnitude;
};
hipError_t launch_rope(const RopeArgs& a, hipStream_t st);

// ---- AdamW (adamw.hip)
struct AdamwItem {
    const float* grad; const void *m, *v; const float *m_absmax, *v_absmax, *weight;
    void *m_out, *v_out; float *m_absmax_out, *v_absmax_out, *weight_out; uint16_t* weight_bf16;
    long long count;
    float lr_scale, decay_scale;
};
struct AdamwChunk { int item; uint32_t first; };             // elements of an item from this one on, as many as a workgroup of the launch takes
struct AdamwGroup {                                          // the items whose states have the same width
    AdamwItem* d_items = nullptr; AdamwChunk* d_chunks = nullptr;
    int nchunks = 0; bool large = false;
};
struct AdamwStep { float lr, b1, c1, b2, c2, over_bias1, over_bias2, eps, decay; const float* grad_scale; };   // c = 1 - b; over_bias = 1 / (1 - b^t)
hipError_t adamw_build(const std::vector<AdamwItem>& items, bool eight, AdamwGroup& g);
hipError_t adamw_run(const AdamwGroup (&groups)[2], const AdamwStep& s, hipStream_t st);
void adamw_free(AdamwGroup (&groups)[2]);
hipError_t launch_adamw_state(long long count, bool is_signed, const void* codes, const float* absmax, float* out, hipStream_t st);

// ---- loss over the vocabulary (vocab_loss.hip)
struct VocabLossArgs {
    int M, V, K;
    const uint16_t *h, *W;
    const int32_t* targets;
    const float* weights;                       // null: one
    float *loss, *lse;                          // lse: or null
    uint16_t* dH;                               // or null
    void* workspace;
};
size_t vocab_loss_workspace_bytes(int M, int V, int K, bool grad);
hipError_t launch_vocab_loss(const VocabLossArgs& a, hipStream_t st);

}  // namespace lowra

struct lowra_adamw_batch {
    int device = -1;
    lowra::AdamwGroup groups[2];                // states in 32 bits, in 8
};
