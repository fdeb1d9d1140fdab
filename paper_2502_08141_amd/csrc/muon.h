// The orthogonalised adapter update (muon.hip): descriptors and launchers.
#pragma once
#include "lowra_host.h"

namespace lowra {

constexpr long long kMuonMaxElements = 1ll << 29;    // 32-bit byte offsets
constexpr int kMuonMaxShort = 64;        // the short side: the rank that the adapter gradients support

struct MuonItem {
    const float* grad; const float* momentum; const float* weight;        // weight null: the update only
    float* momentum_out; float* weight_out; float* update; uint16_t* weight_bf16;
    int L, R, wide;                      // the long side and the short one; wide: that counts the rows
    float scale;
    int chunk0, nchunks;                 // this matrix's chunks (muon_build)
};
struct MuonChunk { int first, last, item; };                              // long-side elements [first, last) of a matrix
struct MuonGroup {                       // the matrices of one short-side class
    MuonItem* d_items = nullptr; MuonChunk* d_chunks = nullptr;
    double *part = nullptr, *poly = nullptr;
    int nitems = 0, ngram = 0, napply = 0;                               // d_chunks: the first pass's, then the last's
};
struct MuonStep { float lr, momentum, decay, a, b, c, eps; int nesterov, steps; };

size_t muon_workspace_bytes(int n, const MuonItem* items);
hipError_t muon_build(const std::vector<MuonItem>& items, void* workspace, MuonGroup (&groups)[3]);
hipError_t muon_run(const MuonGroup (&groups)[3], const MuonStep& s, hipStream_t st);
void muon_free(MuonGroup (&groups)[3]);

}  // namespace lowra

struct lowra_muon_batch {
    int device = -1;
    lowra::MuonGroup groups[3];
};
