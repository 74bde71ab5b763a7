// Launch shapes of the gated linear recurrence, in plain C++ so that they can be checked over whole ranges of sizes on the
// CPU.
#pragma once
#include <initializer_list>

namespace lbscan {

// Tokens that a lane holds: 16 bytes of a row.
constexpr int gated_lane_tokens(int dtype) { return dtype == 0 ? 4 : 8; }
// Rows shorter than this are walked by one lane each.
constexpr int kGatedShort = 8;

struct GatedShape {
    // Tiles of lanes * waves * gated_lane_tokens tokens, one team of lanes a row
    int lanes, waves;
    int ntiles;
    // Rows cut into nseg segments of seg_tiles tiles, a team each
    int nseg, seg_tiles;
};

// Waves of a row's team, for a row of so many wave tiles (the tokens of 64 lanes).  As few idle lanes as possible
// first: a tile that the row does not fill costs as much as a full one.  Among equals a tile that holds the
// whole row (nothing is carried along: 86 registers instead of 112 in the backward kernel of 2-byte storage), then the order below.  Fewer
// waves than 8 a CU do not keep the memory busy, and sixteen to a team leave room for one
// team a CU with 2-byte storage (there they are for few rows only).  MI355X, us, forward / backward, by waves a
// team (calls in a loop, inputs partly in the caches):
//     8 x 768 x 4096 bf16     1: 39.7 / 78.9    4: 40.3 / 75.5    8: 37.1 / 68.7    16: 61.6 / 137.8
//     8 x 768 x 4096 fp32     1: 82.1 / 151.7   4: 78.8 / 141.4   8: 73.5 / 134.5   16: 71.6 / 132.2
//     1 x 768 x 8192 bf16     1: 16.0 / 30.6    4: 11.6 / 22.1    8: 11.9 / 23.0    16: 11.2 / 26.3
//     1 x 256 x 65536 fp32    1: 194.6 / 453.4  4: 59.4 / 130.5   8: 48.6 / 105.0   16: 49.5 / 98.2
//     1 x 384 x 20000 bf16    1: 35.9 / 64.1    4: 17.7 / 31.2    8: 15.5 / 28.9    16: 18.7 / 33.0
//     4 x 1000 x 3001 bf16    1: 21.6 / 35.6    4: 24.7 / 42.6    8: 23.9 / 49.9    16: 43.4 / 100.0
//     16 x 512 x 700 bf16     1: 13.3 / 23.9    2: 12.6 / 24.5    4: 20.2 / 37.7
//     8 x 200 x 2300 bf16     1: 9.4 / 17.4     2: 10.9 / 18.0    4: 12.3 / 20.2    8: 10.7 / 20.3
//     6 x 100 x 4400 bf16     2: 9.8 / 17.4     4: 9.1 / 15.5     8: 10.2 / 18.0    16: 9.4 / 20.1
//     1 x 300 x 4400 bf16     2: 9.2 / 16.9     4: 7.0 / 12.7     8: 7.5 / 13.8     16: 7.1 / 14.7
//     1 x 300 x 2300 fp32     2: 6.8 / 13.3     4: 5.7 / 11.2     8: 5.7 / 11.1     16: 5.6 / 11.2
// (For 257 to 512 rows of nine wave tiles in bf16 the rule gives eight waves, sixteen tiles' worth of lanes for nine, where
// four are 8% faster.)
inline int gated_team_waves(int wave_tiles, long rows, int dtype)
{
    int best = 0, padded = 0;
    for (const int w : {8, 4, 1, 2, 16}) {
        if (w > 1 && w >= 2 * wave_tiles) continue;                    // half of it would idle
        if (w < 16 && w < wave_tiles && rows * w <= 2048) continue;
        if (w == 16 && best && dtype != 0) continue;
        const int n = (wave_tiles + w - 1) / w * w;
        if (!best || n < padded || (n == padded && n == w)) { best = w; padded = n; }
    }
    return best;
}

// A row is cut where there are too few for the CUs and it is long; the maps of the pieces cost another pass over three
// of the tensors.  MI355X, us, forward / backward, whole and cut: 1 x 64 x 65536 bf16 21.1 / 35.7 and 16.1 / 21.2,
// 1 x 16 x 65536 fp32 22.4 / 39.8 and 9.6 / 14.2, 1 x 128 x 65536 fp32 29.7 / 56.0 and 40.1 / 60.7, and of three
// tiles 2 x 24 x 9000 fp32 6.4 / 12.1 and 7.8 / 11.6.  So few rows of several tiles have teams of sixteen waves by the rule
// above, and only kernels of such teams take cut rows.
constexpr int kGatedCutRows = 96, kGatedCutTiles = 4, kGatedCutWaves = 16;

inline GatedShape gated_shape_of(long rows, int seqlen, int dtype)
{
    GatedShape s{1, 1, 1, 1, 1};
    if (seqlen < kGatedShort) return s;
    const int v = gated_lane_tokens(dtype);
    s.lanes = 8;
    while (s.lanes < 64 && s.lanes * v < seqlen) s.lanes *= 2;
    const int wave_tiles = (seqlen + 64 * v - 1) / (64 * v);
    if (wave_tiles > 1) s.waves = gated_team_waves(wave_tiles, rows, dtype);
    const int tile = s.lanes * s.waves * v;
    s.ntiles = s.seg_tiles = (seqlen + tile - 1) / tile;
    if (rows <= kGatedCutRows && s.ntiles >= kGatedCutTiles) {
        int want = (int)((256 + rows - 1) / rows);
        want = want < 64 ? want : 64;                      // a lane folds a segment
        want = want < s.ntiles ? want : s.ntiles;
        s.seg_tiles = (s.ntiles + want - 1) / want;
        s.nseg = (s.ntiles + s.seg_tiles - 1) / s.seg_tiles;
    }
    return s;
}

}  // namespace lbscan
