// Which tile a product of two 4-bit matrices takes.  Plain C++: no device code.
#pragma once
#include <cstdint>

namespace llvq {

struct MxTile { int rows, tokens, stage, end; };         // rows of W by tokens; cycles that a stage of 256 columns takes, and the end of a tile, which writes it
constexpr MxTile kMxTiles[4] = {{256, 224, 1450, 4500}, {128, 256, 970, 1500}, {128, 128, 560, 1000}, {128, 64, 420, 700}};

// The tile whose rounds over the SMs take least.  us with the four: 28672 x 8192 x 2048 tokens 221, 226, 257, 423; 8192 x 8192 x 4096 142, 135, 156, 259;
// 4096 x 11008 x 512 36, 26, 20, 30; 4096 x 4096 x 237 18, 12, 9.0, 8.8.
inline int mx_tile_of(int64_t n_out, int64_t tokens, uint32_t k_stages, int sms)
{
    int pick = 0;
    uint64_t best = ~0ull;
    for (int i = 0; i < 4; ++i) {
        const MxTile& t = kMxTiles[i];
        const uint64_t tiles = (uint64_t)((n_out + t.rows - 1) / t.rows) * (uint64_t)((tokens + t.tokens - 1) / t.tokens);
        const uint64_t cost = (tiles + sms - 1) / sms * ((uint64_t)k_stages * t.stage + t.end);
        if (cost < best) { best = cost; pick = i; }
    }
    return pick;
}

}  // namespace llvq
