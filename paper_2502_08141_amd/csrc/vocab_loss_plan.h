// How the loss over a vocabulary goes through the card: pieces of tokens, tiles of both products, splits, and the workspace.  Host code only.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace lowra {

constexpr int kLossDepth = 64;                           // a step of either product: 64 features or words
struct LossStat { float shift, sum; };                   // of a tile's words: n, and the sum with the target aside

constexpr size_t kLossPiece = (size_t)256 << 20;         // bytes of a piece's exponentials
constexpr size_t kLossPart = (size_t)64 << 20;           // bytes of the second product's partial sums beyond one of each

// Microseconds of a round of tiles on all units: what does not depend on the steps, and a step (256 tiles of 1024 and 4096 features, or 2048 and 8192 words).
// Lower tiles cost more per token, but leave less of a round empty.
struct TileCost { int tokens; double fixed, step; };
constexpr TileCost kLogitsCost[] = {{256, 11.0, 1.48}, {192, 8.0, 1.20}, {128, 6.0, 0.93}, {64, 3.0, 0.62}};
constexpr TileCost kGradCost[] = {{256, 10.0, 1.55}, {192, 7.0, 1.23}, {128, 4.0, 1.08}, {64, 2.0, 0.78}};

struct LossPlan {
    int tokens, shift, tiles, VP, rows, grad_tokens, splits, words;      // rows: tokens a piece
    size_t stats0, zt0, rounded0, apart0, rows0, part0, P0, bytes;
};
// units: compute units
inline LossPlan loss_plan(int M, int V, int K, bool grad, int units) {
    LossPlan l{};
    const int V256 = (V + 255) / 256;
    size_t rows = (size_t)M;
    if (grad) rows = std::min(rows, std::max<size_t>(std::min(kLossPiece / ((size_t)V256 * 512), kLossPiece / 2 / ((size_t)K * 4)) / 256 * 256, 256));
    rows = std::min<size_t>(rows, std::max((1 << 24) / V256, 256));      // (statistics of a piece: 128 MB)
    l.rows = (int)rows;
    // Few tokens: tiles of 128 words, so that more units read W; up to 128 tokens only where a unit has no more than one of them (128 tokens, K 4096, 32000 words 71 -> 60 us,
    // K 8192, 16000 words 105 -> 82; K 1024, 50265 words would be 32 -> 41).
    l.shift = l.rows <= 64 || (l.rows <= 128 && (V + 127) / 128 <= units) ? 7 : 8;
    l.tiles = (V + (1 << l.shift) - 1) >> l.shift;
    l.VP = l.tiles << l.shift;
    auto rounds = [&](long long tiles) { return (double)((tiles + units - 1) / units); };
    double least = 1e300;
    for (const TileCost& c : kLogitsCost) {
        const double t = rounds((long long)((l.rows + c.tokens - 1) / c.tokens) * l.tiles) * (c.fixed + c.step * ((K + kLossDepth - 1) / kLossDepth));
        if (l.shift == 7 ? c.tokens == (l.rows <= 64 ? 64 : 128) : t < least) { least = t; l.tokens = c.tokens; }
    }
    // The second product has few tiles, so that its words are split between workgroups, whose sums are written and read once more (3.3 MB of them a microsecond).
    const size_t out_bytes = (size_t)l.rows * K * 4;
    const int most = (int)std::min<size_t>(std::min(l.tiles, 64), kLossPart / out_bytes + 1);
    least = 1e300;
    for (const TileCost& c : kGradCost) {
        const long long out_tiles = (long long)((l.rows + c.tokens - 1) / c.tokens) * ((K + 255) / 256);
        for (int splits = 1; splits <= most; ++splits) {
            const int words = ((l.tiles + splits - 1) / splits) << l.shift;
            const double t = rounds(out_tiles * splits) * (c.fixed + c.step * (words / kLossDepth)) + (double)splits * (double)out_bytes / 3.3e6;
            if (t < least) { least = t; l.grad_tokens = c.tokens; l.words = words; }
        }
    }
    l.splits = (l.VP + l.words - 1) / l.words;
    auto take = [&](size_t n) { const size_t at = l.bytes; l.bytes += (n + 255) / 256 * 256; return at; };
    l.stats0 = take((size_t)l.rows * l.tiles * sizeof(LossStat));
    l.zt0 = take((size_t)l.rows * 4);
    if (grad) {
        l.rounded0 = take((size_t)l.rows * l.tiles * sizeof(float));
        l.apart0 = take((size_t)((l.rows + 31) / 32) * l.tiles * 4);
        l.rows0 = take((size_t)l.rows * 8);
        l.part0 = take((size_t)l.splits * out_bytes);
        l.P0 = take((size_t)l.rows * l.VP * 2);
    }
    return l;
}

}  // namespace lowra
