// Sizes, pieces and scratch of a call of the loss.  No device code: the rules hold on the host alone.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace lbscan {

constexpr int kLossTile = 256;                // rows and columns of a block's product
constexpr int kLossFewTokens = 64, kLossFewVocab = 128;
constexpr int kLossUnits = 256;               // blocks under way at once

struct LossPlan {
    int dimp;                // dim in whole steps of the products (64 bytes)
    long rows;               // tokens in whole tiles
    int few;                 // tiles of 64 tokens
    int copy_weight;         // the table's rows are no whole steps, or not aligned
    int piece, pieces;       // columns of the vocabulary that G has room for
    int chunk, chunks;       // tiles of the vocabulary a block of the forward pass takes
    int splits_x, splits_w;
    // bytes from the start of the scratch
    size_t live, counts, rank, order, targets, lse2, down, both, own, part, x, w, g, acc, share, total;
};

inline long loss_ceil(long a, long b) { return (a + b - 1) / b; }

// Cuts the sum of a product of `tiles` blocks and `steps` steps so that the blocks are whole rounds of the machine, as
// far as the pieces' own cost (their sums are written and read once more, about `cost` steps each) allows.
inline int loss_splits(long tiles, long steps, long cost)
{
    int best = 1;
    long least = -1;
    for (int s = 1; s <= 16 && (s == 1 || s * 8 <= steps); ++s) {
        const long time = loss_ceil(tiles * s, kLossUnits) * (loss_ceil(steps, s) + cost);
        if (least < 0 || time < least) { least = time; best = s; }
    }
    return best;
}

inline LossPlan loss_plan_of(long tokens, int vocab, int dim, int element, bool aligned, bool backward, bool want_dx, bool want_dw)
{
    LossPlan p{};
    if (tokens == 0 || vocab == 0 || dim == 0) return p;        // (no kernel runs)
    const int step = 64 / element;
    p.dimp = (int)(loss_ceil(dim, step) * step);
    p.few = tokens <= kLossFewTokens;
    p.rows = loss_ceil(tokens, p.few ? kLossFewTokens : kLossTile) * (p.few ? kLossFewTokens : kLossTile);
    p.copy_weight = dim != p.dimp || !aligned;
    const long width = loss_ceil(vocab, kLossTile) * kLossTile;
    // G: at most a gigabyte of the vocabulary at a time, in pieces of one size
    const long most = ((long)1 << 30) / (p.rows * element) / kLossTile * kLossTile;
    p.pieces = (int)loss_ceil(width, most < kLossTile ? kLossTile : most);
    p.piece = (int)(loss_ceil(width / kLossTile, p.pieces) * kLossTile);
    p.pieces = (int)loss_ceil(width, p.piece);
    // blocks of several tiles of the vocabulary, where there are many
    const int vtile = p.few ? kLossFewVocab : kLossTile;
    const long vtiles = loss_ceil(vocab, vtile), ntiles = p.rows / (p.few ? kLossFewTokens : kLossTile);
    const long per = vtiles * ntiles / (8 * kLossUnits);
    p.chunk = (int)(per < 1 ? 1 : per > 8 ? 8 : per);
    p.chunks = (int)loss_ceil(vtiles, p.chunk);
    p.splits_x = p.splits_w = 1;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    p.live = take(4);
    p.counts = take(4 * (size_t)loss_ceil(tokens, 1024));
    p.rank = take(4 * (size_t)tokens);
    p.order = take(4 * (size_t)p.rows);
    p.targets = take(4 * (size_t)p.rows);
    p.x = take((size_t)p.rows * p.dimp * element);
    if (p.copy_weight) p.w = take((size_t)vocab * p.dimp * element);
    if (!backward) {
        p.own = take(4 * (size_t)p.rows);
        p.part = take(8 * (size_t)p.rows * p.chunks);
    } else {
        const long mtiles = loss_ceil(p.dimp, kLossTile);
        p.lse2 = take(4 * (size_t)p.rows);
        p.down = take(4 * (size_t)p.rows);
        p.both = take(4 * (size_t)p.rows);
        p.g = take((size_t)p.rows * p.piece * element);
        if (want_dx) {
            p.splits_x = loss_splits(mtiles * ntiles, p.piece / step, 8);
            p.acc = take(4 * (size_t)p.splits_x * p.rows * p.dimp);
        }
        if (want_dw) {
            p.splits_w = loss_splits(mtiles * (p.piece / kLossTile), loss_ceil(p.rows, step), 8);
            if (p.splits_w > 1) p.share = take(4 * (size_t)p.splits_w * p.piece * p.dimp);
        }
    }
    p.total = at;
    return p;
}

}  // namespace lbscan
