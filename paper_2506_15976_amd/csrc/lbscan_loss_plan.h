// Sizes, pieces and scratch of a call of the loss, and how its products are cut into the units that blocks take.  How many tokens
// are live is known on the device alone: the cuts are chosen there, by the same functions, within the room planned here.
#pragma once
#include <math.h>
#include <stddef.h>
#include <stdint.h>

#ifdef __HIPCC__
#define LBSCAN_BOTH __host__ __device__
#else
#define LBSCAN_BOTH
#endif

namespace lbscan {

constexpr int kLossTile = 256;                // rows of the table, or columns of x, of a block's product
constexpr int kLossLooseSteps = 4;            // steps under way of a product with loose rows, which has whole fours of them
constexpr int kLossFewTokens = 64;
// Rows of the table (columns of x) of few tokens' products.  fp32 with loose rows: half as many, as a compute unit with one block is bound by
// its matrix cores (MI355X, us, loss and gradients, 128 / 64: 35 x 11565 x 2753 fp32 377 / 279; 3 x 129028 x 2610 bf16 866 / 967).
LBSCAN_BOTH constexpr int loss_few_vocab(int loose, int element) { return loose && element == 4 ? 64 : 128; }
// Tokens (of dweight: rows of the table) of a block's product.  fp32: half as many and two blocks a compute unit, of which one
// alone keeps the matrix cores as busy: where the last round is not full a compute unit has one.  MI355X, us, logits of
// 1261 x 32003 x 385: 332 with one block of 256 x 256, 278 with two of 256 x 128; bf16 16384 x 50000 x 768: 1406, 1561.
LBSCAN_BOTH constexpr int loss_tokens(int few, int element) { return few ? kLossFewTokens : element == 4 ? 128 : 256; }
// Parts of a sum.  Loose rows are read by many blocks, or slowly: MI355X, us, dx of 2 x 86816 x 1103 fp32 and 60 x 50000 x 770 bf16 with
// 32 / 64 parts at most 283 / 191 and 66 / 42 (rows in place, 64 x 50000 x 768: 20 / 22.5).
LBSCAN_BOTH constexpr bool loss_loose_units(int units) { return units == 512 || units == 1024; }
LBSCAN_BOTH constexpr int loss_most_splits(int units) { return loss_loose_units(units) ? 64 : 32; }

// What the device chooses once the live tokens are counted (the start of the scratch).
struct LossChoice {
    int live, rows;                           // live tokens; in whole tiles
    int chunk_lse, chunk_slope[2];            // tiles of the vocabulary a unit: all of it; a piece, the last piece
    int splits_x, splits_w[2];                // parts of the sums; of dweight for a piece, the last piece
};

LBSCAN_BOTH inline long loss_ceil(long a, long b) { return (a + b - 1) / b; }
LBSCAN_BOTH inline int loss_ceil32(int a, int b) { return (a + b - 1) / b; }
// Compute units, whose rounds of units of the products are counted; of few tokens three blocks run on one at once, with loose rows two, in fp32 four.
LBSCAN_BOTH constexpr int loss_units(int few, int loose, int element) { return loose ? (element == 4 ? 1024 : 512) : few ? 768 : 256; }

// Time of the logits' products in steps, in units of `chunk` of `vtiles` tiles of the vocabulary for each of `ntiles` tiles of
// tokens: whole rounds of the machine.  A tile's exponentials take about as long as 6 steps, a unit's first loads 3.
LBSCAN_BOTH inline float loss_chunk_time(int ntiles, int vtiles, int chunk, int steps, int units)
{
    return ceilf((float)ntiles * (float)loss_ceil32(vtiles, chunk) / (float)units) * ((float)chunk * (float)(steps + 6) + 3.0f);
}
// The chunk that fills about `rounds` rounds.
LBSCAN_BOTH inline int loss_chunk_of(int ntiles, int vtiles, int rounds, int units)
{
    const int chunks = units * rounds / ntiles;
    return loss_ceil32(vtiles, chunks < 1 ? 1 : chunks > vtiles ? vtiles : chunks);
}
// Time of a sum over `steps` steps for `tiles` tiles, cut into `splits` parts, which are written and read once more (4 bytes a
// value at about 4.5 TB/s: 0.12 us a tile of 256 x 256, of 1.0 us a step in bf16, 0.06 us one of 256 x 128, of 1.8 us in fp32; steps of
// loose rows are those of memory, 0.4 us, of 0.015 us a tile).
LBSCAN_BOTH inline float loss_split_time(long tiles, int steps, int splits, int units, int element)
{
    const float all = (float)tiles * (float)splits;
    float rounds = ceilf(all / (float)units);
    // (fp32: a block alone on its compute unit takes about a quarter longer than half the time of two)
    if (element == 4 && !loss_loose_units(units) && ceilf(rounds / 2.0f) * 2.0f != rounds) rounds += 0.25f;
    return rounds * (float)(loss_ceil32(steps, splits) + 4) + (splits > 1 ? (element == 2 && !loss_loose_units(units) ? 0.12f : 0.035f) * all : 0.0f);
}
LBSCAN_BOTH inline bool loss_split_fits(int steps, int splits, long most) { return splits == 1 || (splits <= most && splits * 8 <= steps); }

struct LossPlan {
    int dimp;                // dim in whole steps of the products (64 bytes), loose: in fours of them
    long rows;               // tokens in whole tiles
    int few;                 // tiles of 64 tokens
    int loose;               // the table's rows are no whole steps, or not aligned: few tokens read them as they are,
    int copy_weight;         // others a copy
    int piece, pieces;       // columns of the vocabulary that G has room for
    long part_room;          // values of the forward pass's parts (rows x chunks)
    long acc_rows;           // rows of dx's sums (rows x splits)
    long share_rows;         // rows of dweight's, where it is cut (columns of a piece x splits)
    // bytes from the start of the scratch
    size_t choice, counts, rank, order, targets, lse2, down, both, own, part, x, w, g, acc, share;
    size_t hot, rest, rest_rows, list, slot, sort, total;              // bf16: what rounding the targets' slopes leaves
};

inline int loss_best_splits(long tiles, int steps, int units, int element)
{
    int best = 1;
    for (int s = 2; s <= loss_most_splits(units); ++s)
        if (loss_split_fits(steps, s, loss_most_splits(units)) &&
            loss_split_time(tiles, steps, s, units, element) < loss_split_time(tiles, steps, best, units, element))
            best = s;
    return best;
}

// sort_bytes: scratch of the list of sums by target.
inline LossPlan loss_plan_of(long tokens, int vocab, int dim, int element, bool aligned, bool backward, bool want_dx, bool want_dw, size_t sort_bytes)
{
    LossPlan p{};
    if (tokens == 0 || vocab == 0 || dim == 0) return p;        // (no kernel runs)
    const int step = 64 / element;
    p.few = tokens <= kLossFewTokens;
    const bool whole_rows = dim % step == 0 && aligned;
    p.loose = p.few && !whole_rows && dim * element >= 16;
    p.copy_weight = !whole_rows && !p.loose;
    const int whole = p.loose ? step * kLossLooseSteps : step;
    p.dimp = (int)(loss_ceil(dim, whole) * whole);
    const int ntile = loss_tokens(p.few, element), wtile = loss_tokens(0, element), units = loss_units(p.few, p.loose, element);
    p.rows = loss_ceil(tokens, ntile) * ntile;
    const long mtiles = loss_ceil(p.dimp, kLossTile), vtiles = loss_ceil(vocab, kLossTile);
    // G: a gigabyte of the vocabulary at a time, in pieces that are just a whole number of rounds of dweight's tiles; one tile of
    // 256 columns where that is more (from 2^21 tokens in bf16, 2^20 in fp32; 8 and 16 GiB of 2^24 tokens)
    long most = ((long)1 << 30) / (p.rows * element) / kLossTile;
    if (most < 1) most = 1;
    long tiles = vtiles;
    if (most < vtiles) {
        tiles = 256 * (most * mtiles / 256) / mtiles;
        if (tiles < 1) tiles = most;
    }
    p.piece = (int)(tiles * kLossTile);
    p.pieces = (int)loss_ceil(vtiles, tiles);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at += (bytes + 255) / 256 * 256; return here; };
    p.choice = take(sizeof(LossChoice));
    p.counts = take(4 * (size_t)loss_ceil(tokens, 1024));
    p.rank = take(4 * (size_t)tokens);
    p.order = take(4 * (size_t)p.rows);
    p.targets = take(4 * (size_t)p.rows);
    p.x = take((size_t)p.rows * p.dimp * element);
    if (p.copy_weight) p.w = take((size_t)vocab * p.dimp * element);
    if (!backward) {
        // chunks for up to 64 rounds of units
        const long all = p.rows * loss_ceil(vocab, p.few ? loss_few_vocab(p.loose, element) : kLossTile), room = 64L * units * ntile;
        p.part_room = all < room ? all : room < p.rows ? p.rows : room;
        p.own = take(4 * (size_t)p.rows);
        p.part = take(8 * (size_t)p.part_room);
    } else {
        p.lse2 = take(4 * (size_t)p.rows);
        p.down = take(4 * (size_t)p.rows);
        p.both = take(4 * (size_t)p.rows);
        p.g = take((size_t)p.rows * p.piece * element);
        if (element == 2) {
            p.hot = take(4 * (size_t)p.rows);
            p.rest = take(4 * (size_t)p.rows);
            if (want_dw) {
                p.rest_rows = take(2 * (size_t)p.rows * p.dimp);
                p.list = take(2 * (size_t)p.rows * p.dimp);
                p.slot = take(4 * (size_t)vocab);
                p.sort = take(sort_bytes);
            }
        }
        if (want_dx) {
            // as many parts as all tokens need, and more for fewer live ones: room for 8192 rows at the least (192 MiB of 6144 columns, 2 GiB
            // of 65536), 1024 of few tokens
            const long few_rows = p.few ? 1024 : 8192;
            p.acc_rows = p.rows * loss_best_splits(loss_ceil(p.dimp, p.few ? loss_few_vocab(p.loose, element) : kLossTile) * (p.rows / ntile), (int)loss_ceil(p.piece, step), units, element);
            if (p.acc_rows < few_rows) p.acc_rows = few_rows;
            p.acc = take(4 * (size_t)p.acc_rows * p.dimp);
        }
        if (want_dw) {
            const int steps = (int)loss_ceil(p.rows, step);
            const long last = loss_ceil(vocab - (p.pieces - 1L) * p.piece, wtile);
            const long whole = loss_best_splits(mtiles * (p.piece / wtile), steps, 256, element), end = loss_best_splits(mtiles * last, steps, 256, element);
            if (whole > 1 && p.pieces > 1) p.share_rows = whole * p.piece;
            if (end > 1 && end * last * wtile > p.share_rows) p.share_rows = end * last * wtile;
            if (p.share_rows) p.share = take(4 * (size_t)p.share_rows * p.dimp);
        }
    }
    p.total = at;
    return p;
}

}  // namespace lbscan
