// Token embedding and its gradient (formulas: lbscan_embed.h).  All of it is bound by memory: the lookup by
// the rows read and written, the gradient by the table written and dout read once (few tokens: by the latency of
// its three launches).  MI355X, three sets of inputs in turn, 32768 tokens of 50000 x 768 bf16: lookup 17.4 us (5.8 TB/s
// of rows, repeated ones from cache), gradient 47.2 (count 5.4, place and zeros 18.8, pieces 17.7, join 5.3); 256 tokens of
// 2000 x 256: 3.4 and 12.1 (sort 4.5, pieces 4.2, join 3.4).
#include "lbscan_device.h"
#include "lbscan_embed.h"
#include "lbscan_embed_plan.h"
#include "lbscan_internal.h"

#include <type_traits>

namespace lbscan {
namespace {

// E consecutive elements, at any element's address.
template <typename T, int E> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[E]; };

// The row's packs; the last one ends with the row: columns that the pack before it has too are written twice
// with the same value.
template <int E>
__device__ __forceinline__ int column_of(int pack, int dim) { return min(pack * E, dim - E); }

template <typename I>
__device__ __forceinline__ int row_of(I id, int vocab)
{
    return id >= 0 && id < (I)vocab ? (int)id : -1;
}

// ---- lookup ----------------------------------------------------------------------------------------
// A wave takes four tokens, so that four rows are in flight; a pack a lane at a time.
constexpr int kLookup = 4;
template <typename T, typename I, int E>
__global__ __launch_bounds__(256) void embed_fwd_kernel(const EmbedParams p)
{
    const int lane = threadIdx.x & 63;
    const long first = ((long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * kLookup;
    const int dim = p.dim, packs = (dim + E - 1) / E;
    const I* ids = static_cast<const I*>(p.ids);
    int row[kLookup];
#pragma unroll
    for (int k = 0; k < kLookup; ++k) row[k] = first + k < p.tokens ? row_of(ids[first + k], p.vocab) : -1;
    for (int c = lane + 64 * blockIdx.y; c < packs; c += 64 * gridDim.y) {
        const int col = column_of<E>(c, dim);
        Pack<T, E> q[kLookup];
#pragma unroll
        for (int k = 0; k < kLookup; ++k)
            q[k] = *reinterpret_cast<const Pack<T, E>*>(static_cast<const T*>(p.weight) + (long)max(row[k], 0) * dim + col);
#pragma unroll
        for (int k = 0; k < kLookup; ++k)
            if (first + k < p.tokens) {
                Pack<T, E> o;
#pragma unroll
                for (int e = 0; e < E; ++e) o.v[e] = from_f32<T>(row[k] < 0 ? 0.0f : p.scale * to_f32(q[k].v[e]));
                *reinterpret_cast<Pack<T, E>*>(static_cast<T*>(p.out) + (first + k) * dim + col) = o;
            }
    }
}

// ---- gradient: the tokens sorted by row ------------------------------------------------------------
// A stable counting sort.  Block (r, c) has the rows v = r mod R, R a power of two (so that rows that are used much and
// lie next to each other in a table ordered by frequency go to different blocks), and the c-th share of the
// tokens.  It looks at every id of its share and counts those of its rows, by row and by eighth of the share (a
// wave each).  Running sums of the counts over rows, shares and waves say where each wave puts its tokens; a wave takes
// them in order, so that the tokens of a row stay in theirs.  One share: one launch, in which a block also
// counts the tokens of the blocks before it.  Several: a launch that counts and one that places, since what
// takes the time is one wave walking through the tokens of a much used row.  More than eight lose by the counts of the
// other shares that every block reads.  MI355X, us, calls in a loop, the gradient of 32768 x 768 bf16 by Zipf's law over 50000 rows: one
// share 48.3, eight 44.6, sixteen 52.9; of 65536 x 512 bf16 over 300 rows 63.7, 43.2, 46.9.
constexpr int kSortWaves = 8;
constexpr int kSortThreads = 64 * kSortWaves;
constexpr int kSortRows = 2 * kSortThreads;   // most rows of a block: two to a thread, 32 KB of counts
constexpr int kSortShare = 4096;           // tokens of a share, where the grid allows
constexpr int kSortShares = 8;             // most shares: two blocks a CU where there are 64 of rows
constexpr int kSortAhead = 4;              // groups of 64 ids that a wave loads together at first

enum class Sort { all, count, place };

void sort_shape(EmbedParams& p)
{
    p.blocks_log2 = 6;
    while (((long)kSortRows << p.blocks_log2) < p.vocab) ++p.blocks_log2;
    const long most = (kSortShares << 6) >> p.blocks_log2, wanted = (p.tokens + kSortShare - 1) / kSortShare;
    p.shares = (int)(wanted < most ? wanted : most);
    if (p.shares < 1) p.shares = 1;
}
int sort_rows(const EmbedParams& p) { return (int)(((unsigned)p.vocab + (1u << p.blocks_log2) - 1) >> p.blocks_log2); }

// The row of an id, with the top bit set where it is none (vocab < 2^31).
template <typename I>
__device__ __forceinline__ unsigned sort_row(I id, unsigned vocab)
{
    using U = std::make_unsigned_t<I>;
    return (U)id < (U)vocab ? (unsigned)id : 0xffffffffu;
}

// Sum over the block's threads, the same in all of them.
__device__ __forceinline__ int block_sum(int v, int (&totals)[kSortWaves])
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) totals[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) v += totals[w];
    return v;
}

// Zeros to the rows of dweight that no token has: a wave looks at kZeroRows rows.  These blocks stand behind those that
// sort, in the same launch: the sort waits for memory and leaves its rate to them.  With one share the counts are
// not there yet, and every row is set to zero; the sums overwrite the few that have tokens.
constexpr int kZeroRows = 16;
constexpr int kZeroBlock = kZeroRows * kSortWaves;
struct __attribute__((packed, aligned(2))) Zeros { uint32_t w[4]; };

__device__ __forceinline__ void zero_rows(const EmbedParams& p, long v0, bool counted, unsigned blocks, int row_pitch)
{
    if (v0 >= p.vocab) return;
    const int lane = threadIdx.x & 63;
    const unsigned v = (unsigned)min(v0 + (lane & (kZeroRows - 1)), (long)p.vocab - 1);
    int tokens = 0;
    if (counted) {
        const int* of_row = p.share_count + (long)(v & (blocks - 1)) * row_pitch + (v >> p.blocks_log2);
#pragma unroll
        for (int c = 0; c < kSortShares; ++c) tokens += c < p.shares ? of_row[(long)c * blocks * row_pitch] : 0;
    }
    uint64_t empty = __ballot(lane < kZeroRows && v0 + lane < p.vocab && tokens == 0);
    const long bytes = (long)p.dim * (p.dtype == 0 ? 4 : 2);
    char* const table = static_cast<char*>(p.dweight);
    while (empty) {
        char* to = table + (v0 + __builtin_ctzll(empty)) * bytes;
        empty &= empty - 1;
        if (bytes >= 16) {
            for (long c = 16L * lane; c < bytes; c += 16 * 64) *reinterpret_cast<Zeros*>(to + min(c, bytes - 16)) = Zeros{};
        } else if (2 * lane < bytes) {
            reinterpret_cast<uint16_t*>(to)[lane] = 0;
        }
    }
}

template <typename I, Sort WHAT>
__global__ __launch_bounds__(kSortThreads) void embed_sort_kernel(const EmbedParams p)
{
    extern __shared__ int counts[];        // (waves, rows), and a place per lane for what does not count
    __shared__ int totals[kSortWaves];
    const int blocks_log2 = p.blocks_log2;
    if (WHAT != Sort::count && (int)blockIdx.y >= p.shares) {
        const long block = (long)(blockIdx.y - p.shares) * gridDim.x + blockIdx.x;
        zero_rows(p, block * kZeroBlock + (threadIdx.x >> 6) * kZeroRows, WHAT == Sort::place, gridDim.x,
                  (int)(((unsigned)p.vocab + (1u << blocks_log2) - 1) >> blocks_log2));
        return;
    }
    const unsigned shares = p.shares;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned mine = blockIdx.x, mask = (1u << blocks_log2) - 1;
    const unsigned mask_none = mask | 0x80000000u;
    const int rows = (int)(((unsigned)p.vocab + mask - mine) >> blocks_log2);   // v = mine + k * blocks < vocab
    const I* ids = static_cast<const I*>(p.ids);
    // the block's share of the tokens, and the wave's of that: whole groups of 64
    const long block_share = ((p.tokens + shares - 1) / shares + 63) / 64 * 64;
    const long block_begin = min(block_share * blockIdx.y, p.tokens), block_end = min(block_begin + block_share, p.tokens);
    const long share = ((block_end - block_begin + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const long begin = min(block_begin + share * wave, block_end), end = min(begin + share, block_end);
    // A bit of `hits` stands for 2^span_log2 groups of 64 ids and says whether one is the block's.
    const int span_log2 = sort_span_log2(share >> 6);
    uint64_t hits = 0;

    // What the launch before left is on its way meanwhile.  A thread has the rows threadIdx.x and, of many,
    // threadIdx.x + kSortThreads; `all`: their tokens in all shares, `before`: in those before this one.
    const int row_pitch = (int)(((unsigned)p.vocab + mask) >> blocks_log2);
    int all[2] = {0, 0}, before[2] = {0, 0}, below = 0;
    if constexpr (WHAT == Sort::place) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int row = threadIdx.x + k * kSortThreads;
            if (k && rows <= kSortThreads) break;
            const int* of_row = p.share_count + (long)mine * row_pitch + min(row, rows - 1);
#pragma unroll
            for (unsigned c = 0; c < kSortShares; ++c) {
                const int v = c < shares ? of_row[(long)c * gridDim.x * row_pitch] : 0;
                before[k] += c < blockIdx.y ? v : 0;
                all[k] += v;
            }
            if (row >= rows) all[k] = before[k] = 0;
        }
        for (unsigned k = threadIdx.x; k < gridDim.x * shares; k += kSortThreads) below += (k & mask) < mine ? p.share_total[k] : 0;
    }
    for (int k = threadIdx.x; k < rows * kSortWaves; k += kSortThreads) counts[k] = 0;
    __syncthreads();
    // Every block looks at every id: whole groups are loaded without a check, and no lane waits for a branch (ids of
    // other blocks are counted where nobody looks).
    const int nowhere = rows * kSortWaves + lane, base = wave * rows;
    auto count = [&](unsigned v, int group) {
        const unsigned block = v & mask_none;
        if (WHAT == Sort::all) below += block < mine;
        const bool match = block == mine;
        atomicAdd(&counts[match ? base + (int)(v >> blocks_log2) : nowhere], 1);
        hits |= (uint64_t)(__ballot(match) != 0) << (group >> span_log2);
    };
    int group = 0;
    long t = begin;
    for (; t + 64 * kSortAhead <= end; t += 64 * kSortAhead, group += kSortAhead) {
        const I* at = ids + t + lane;
        I id[kSortAhead];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) id[k] = at[64 * k];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) count(sort_row(id[k], p.vocab), group + k);
    }
    for (; t < end; t += 64, ++group) {
        const I id = ids[min(t + lane, end - 1)];
        count(t + lane < end ? sort_row(id, p.vocab) : 0xffffffffu, group);
    }
    __syncthreads();

    // running sums, rows first
    int n[2] = {0, 0};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int row = threadIdx.x + k * kSortThreads;
        if (row < rows) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) n[k] += counts[w * rows + row];
            if (WHAT == Sort::count) p.share_count[((long)blockIdx.y * gridDim.x + mine) * row_pitch + row] = n[k];
        }
    }
    if constexpr (WHAT == Sort::count) {
        const int own = block_sum(n[0] + n[1], totals);
        if (threadIdx.x == 0) p.share_total[blockIdx.y * gridDim.x + mine] = own;
        return;
    }
    int first = block_sum(below, totals);            // where the block's rows begin
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        if (k && rows <= kSortThreads) break;
        const int row = threadIdx.x + k * kSortThreads;
        if (WHAT == Sort::all) all[k] = n[k];
        if (row < rows && blockIdx.y == 0) p.count[mine + ((unsigned)row << blocks_log2)] = all[k];
        int sum = all[k];
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const int other = __shfl_up(sum, m);
            if (lane >= m) sum += other;
        }
        __syncthreads();
        if (lane == 63) totals[wave] = sum;
        __syncthreads();
        int at = first + sum - all[k] + before[k];
#pragma unroll
        for (int w = 0; w < kSortWaves; ++w) {
            if (w < wave) at += totals[w];
            first += totals[w];
        }
        if (row < rows) {
#pragma unroll
            for (int w = 0; w < kSortWaves; ++w) {
                const int c = counts[w * rows + row];
                counts[w * rows + row] = at;
                at += c;
            }
        }
    }
    if (mine == mask && blockIdx.y == 0 && threadIdx.x == 0) *p.valid = first;
    __syncthreads();

    // the groups that have some of the block's rows again, the next one's ids on their way
    volatile int* next = counts + base;              // of this wave alone
    auto id_of = [&](int g) { return ids[min(begin + 64L * g + lane, end - 1)]; };
    const int groups = (int)((end - begin + 63) >> 6);
    auto later = [&](int g) {                        // the first group from g on that may have some
        while (g < groups && !(hits >> (g >> span_log2) & 1)) g = ((g >> span_log2) + 1) << span_log2;
        return g;
    };
    int g = later(0);
    I ahead = g < groups ? id_of(g) : (I)0;
    while (g < groups) {
        const long t0 = begin + 64L * g;
        const unsigned v = t0 + lane < end ? sort_row(ahead, p.vocab) : 0xffffffffu;
        g = later(g + 1);
        if (g < groups) ahead = id_of(g);
        uint64_t left = __ballot((v & mask_none) == mine);
        while (left) {                                // the lanes of one row at a time
            const int leader = __builtin_ctzll(left);
            const unsigned r = __builtin_amdgcn_readlane(v, leader);
            const uint64_t same = __ballot(v == r);
            const int where = next[r >> blocks_log2];
            if (v == r) {
                const int o = where + __builtin_popcountll(same & ((1ull << lane) - 1));
                p.place[o] = (int)(t0 + lane);
                p.row[o] = (int)r;
            }
            if (lane == leader) next[r >> blocks_log2] = where + __builtin_popcountll(same);
            left &= ~same;
        }
    }
}

// ---- gradient: sums over the sorted tokens -----------------------------------------------------------
// A wave takes a piece of the sorted tokens and 64 packs of columns, and adds dout row by row.  A row of the
// table whose tokens all lie in the piece is written; of others the sum goes to scratch: [0] of a row that
// began in an earlier piece, [1] of one that begins here and goes on.
// Few tokens: short pieces, as what counts is how long a wave takes; many: long ones, as every piece costs a block that
// looks for rows to join.  MI355X, us, calls in a loop, the gradient with pieces of 8 / 16 / 32: 256 x 256 of 2000 rows 12.2 / 12.7 / 15.7,
// 4096 x 768 of 50000 24.5 / 25.1 / 28.6, 16384 x 2048 of 50000 68.4 / 62.7 / 60.4, 32768 x 768 48.9 / 43.7 / 43.2.
int piece_of(long tokens) { return tokens <= 4096 ? 8 : tokens <= 8192 ? 16 : 32; }
constexpr int kPieceAhead = 8;
constexpr int kJoinWaves = 8;

template <typename T, int E>
__device__ __forceinline__ void write_row(const EmbedParams& p, int row, int last, int col, const float acc[E])
{
    if (p.slot) {                                    // in a list: at the place of the row's last token
        p.slot[row] = last;                          // (every lane writes the same)
        row = last;
    }
    Pack<T, E> o;
#pragma unroll
    for (int e = 0; e < E; ++e) o.v[e] = from_f32<T>(p.scale * acc[e]);
    *reinterpret_cast<Pack<T, E>*>(static_cast<T*>(p.dweight) + (long)row * p.dim + col) = o;
}

template <typename T, int E>
__global__ __launch_bounds__(256) void embed_pieces_kernel(const EmbedParams p, unsigned pieces, unsigned tiles)
{
    const int lane = threadIdx.x & 63;
    const unsigned task = blockIdx.x * 4u + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int dim = p.dim, packs = (dim + E - 1) / E;
    if (task >= pieces * tiles) return;
    const int piece = (int)(task / tiles), c = (int)(task % tiles) * 64 + lane;
    const int valid = *p.valid, first = piece * p.piece, n = min(p.piece, valid - first);
    if (n <= 0) return;
    const bool there = c < packs;
    const int col = column_of<E>(min(c, packs - 1), dim);
    const int my_place = p.place[first + min(lane, n - 1)], my_row = p.row[first + min(lane, n - 1)];
    const int row_before = first > 0 ? p.row[first - 1] : -1, row_after = first + n < valid ? p.row[first + n] : -1;
    const T* dout = static_cast<const T*>(p.dout);

    // bit k: the k-th token is the last of its row in the piece
    const int my_next = __shfl_down(my_row, 1);
    const uint64_t last = __ballot(lane < n && (lane == n - 1 || my_next != my_row));
    const bool early = row_before == __builtin_amdgcn_readlane(my_row, 0);             // the first row began before
    const bool goes_on = row_after == __builtin_amdgcn_readlane(my_row, n - 1);        // the last one goes on behind
    const uint64_t first_row = last & -last;
    float acc[E] = {};
    for (int k0 = 0; k0 < n; k0 += kPieceAhead) {
        Pack<T, E> q[kPieceAhead];
#pragma unroll
        for (int k = 0; k < kPieceAhead; ++k) {
            const int token = __builtin_amdgcn_readlane(my_place, min(k0 + k, n - 1));
            q[k] = *reinterpret_cast<const Pack<T, E>*>(dout + (long)token * dim + col);
        }
#pragma unroll
        for (int k = 0; k < kPieceAhead; ++k) {
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] += to_f32(q[k].v[e]);
            const uint64_t bit = 1ull << (k0 + k);
            if (last & bit) {
                const bool in_part = (early && (bit & first_row)) || (goes_on && k0 + k == n - 1);
                if (there) {
                    if (!in_part) {
                        write_row<T, E>(p, __builtin_amdgcn_readlane(my_row, k0 + k), first + k0 + k, col, acc);
                    } else {
                        float* to = p.part + ((long)piece * 2 + (early && (bit & first_row) ? 0 : 1)) * dim + col;
                        Pack<float, E> o;
#pragma unroll
                        for (int e = 0; e < E; ++e) o.v[e] = acc[e];
                        *reinterpret_cast<Pack<float, E>*>(to) = o;
                    }
                }
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] = 0.0f;
            }
        }
    }
}

// The rows whose tokens lie in several pieces: the piece in which they begin finds them by its last token and
// adds the others' sums, eight waves a share each, in a fixed order.
template <typename T, int E>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(const EmbedParams p, int first_piece)
{
    __shared__ float sums[kJoinWaves - 1][64][E];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int dim = p.dim, packs = (dim + E - 1) / E;
    const int piece = first_piece + (int)blockIdx.x, begins = piece * p.piece, last = begins + p.piece - 1, valid = *p.valid;
    if (last + 1 >= valid) return;                                     // nothing behind this piece
    const int row = p.row[last];
    if (p.row[last + 1] != row) return;
    if (piece > 0 && p.row[begins - 1] == row) return;        // it began earlier
    // first token of the row: lanes compare the piece's rows
    const uint64_t same = __ballot(lane < p.piece && p.row[min(begins + lane, last)] == row);
    const int begin = begins + __builtin_ctzll(same);
    const int end_piece = (begin + p.count[row] - 1) / p.piece;        // the last piece that has some of it
    const int share = (end_piece - piece + kJoinWaves - 1) / kJoinWaves;
    const int from = piece + 1 + wave * share, to = min(from + share, end_piece + 1);
    const int c = blockIdx.y * 64 + lane;
    const int col = column_of<E>(min(c, packs - 1), dim);
    float acc[E] = {};
    if (wave == 0) {
        const float* tail = p.part + ((long)piece * 2 + 1) * dim + col;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = tail[e];
    }
#pragma unroll 8
    for (int q = from; q < to; ++q) {
        const Pack<float, E> part = *reinterpret_cast<const Pack<float, E>*>(p.part + (long)q * 2 * dim + col);
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += part.v[e];
    }
    if (wave) {
#pragma unroll
        for (int e = 0; e < E; ++e) sums[wave - 1][lane][e] = acc[e];
    }
    __syncthreads();
    if (wave || c >= packs) return;
    for (int w = 0; w < kJoinWaves - 1; ++w)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += sums[w][lane][e];
    write_row<T, E>(p, row, begin + p.count[row] - 1, col, acc);
}

int pieces_of(const EmbedParams& p)
{
    const int piece = piece_of(p.tokens);
    return (int)((p.tokens + piece - 1) / piece);
}

template <typename T, int E>
hipError_t launch_fwd(EmbedParams p, hipStream_t stream)
{
    const int packs = (p.dim + E - 1) / E, tiles = (packs + 63) / 64;
    constexpr int kTokens = 4 * kLookup;             // of a block
    constexpr long most = most_blocks(256) * kTokens;
    for (long left = p.tokens; left > 0; left -= most) {
        p.tokens = left < most ? left : most;
        const dim3 grid((unsigned)((p.tokens + kTokens - 1) / kTokens), tiles < 64 ? tiles : 64);
        if (p.wide_ids) embed_fwd_kernel<T, int64_t, E><<<grid, 256, 0, stream>>>(p);
        else embed_fwd_kernel<T, int32_t, E><<<grid, 256, 0, stream>>>(p);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        p.ids = static_cast<const char*>(p.ids) + p.tokens * (p.wide_ids ? 8 : 4);
        p.out = static_cast<T*>(p.out) + p.tokens * p.dim;
    }
    return hipSuccess;
}

template <typename T, int E>
hipError_t launch_sums(const EmbedParams& p, hipStream_t stream)
{
    const int pieces = pieces_of(p), packs = (p.dim + E - 1) / E, tiles = (packs + 63) / 64;
    const long tasks = (long)pieces * tiles;
    if (tasks == 0) return hipSuccess;
    if ((tasks + 3) / 4 > most_blocks(256)) return hipErrorInvalidConfiguration;      // (a dout of a terabyte)
    embed_pieces_kernel<T, E><<<(unsigned)((tasks + 3) / 4), 256, 0, stream>>>(p, pieces, tiles);
    hipError_t e = hipGetLastError();
    constexpr long most = most_blocks(64 * kJoinWaves);
    for (long first = 0; e == hipSuccess && first < pieces - 1; first += most) {
        const long n = pieces - 1 - first < most ? pieces - 1 - first : most;
        embed_join_kernel<T, E><<<dim3((unsigned)n, tiles), 64 * kJoinWaves, 0, stream>>>(p, (int)first);
        e = hipGetLastError();
    }
    return e;
}

}  // namespace

size_t embed_bwd_bytes(const EmbedParams& q)
{
    EmbedParams p = q;
    sort_shape(p);
    const size_t shares = p.shares > 1 ? ((size_t)p.shares << p.blocks_log2) * (1 + sort_rows(p)) : 0;
    return ((size_t)p.tokens * 2 + p.vocab + 1 + shares + (size_t)pieces_of(p) * 2 * p.dim) * 4;
}

template <typename I>
static hipError_t launch_sort(const EmbedParams& p, hipStream_t stream)
{
    const dim3 grid(1 << p.blocks_log2, p.shares), block(kSortThreads);
    const size_t lds = (size_t)(sort_rows(p) * kSortWaves + 64) * sizeof(int);
    const long zeros = ((long)p.vocab + kZeroBlock - 1) / kZeroBlock;
    const dim3 with_zeros(grid.x, (unsigned)(p.shares + (p.slot ? 0 : (zeros + grid.x - 1) / grid.x)));
    if (p.shares == 1) {
        embed_sort_kernel<I, Sort::all><<<with_zeros, block, lds, stream>>>(p);
        return hipGetLastError();
    }
    embed_sort_kernel<I, Sort::count><<<grid, block, lds, stream>>>(p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    embed_sort_kernel<I, Sort::place><<<with_zeros, block, lds, stream>>>(p);
    return hipGetLastError();
}

hipError_t launch_embed_fwd(const EmbedParams& p, hipStream_t stream)
{
    if (p.dtype == 0) return p.dim < 4 ? launch_fwd<float, 1>(p, stream) : launch_fwd<float, 4>(p, stream);
    return p.dim < 8 ? launch_fwd<bf16_t, 1>(p, stream) : launch_fwd<bf16_t, 8>(p, stream);
}

static void lay_out(EmbedParams& p, void* workspace)
{
    p.part = static_cast<float*>(workspace);
    p.piece = piece_of(p.tokens);
    p.place = reinterpret_cast<int*>(p.part + (size_t)pieces_of(p) * 2 * p.dim);
    p.row = p.place + p.tokens;
    p.count = p.row + p.tokens;
    p.valid = p.count + p.vocab;
    p.share_total = p.valid + 1;
    sort_shape(p);
    p.share_count = p.share_total + ((size_t)p.shares << p.blocks_log2);
}
const int* embed_counts(EmbedParams p, void* workspace)
{
    lay_out(p, workspace);
    return p.count;
}

hipError_t launch_embed_bwd(EmbedParams p, void* workspace, hipStream_t stream)
{
    lay_out(p, workspace);
    const hipError_t e = p.wide_ids ? launch_sort<int64_t>(p, stream) : launch_sort<int32_t>(p, stream);
    if (e != hipSuccess) return e;
    if (p.dtype == 0) return p.dim < 4 ? launch_sums<float, 1>(p, stream) : launch_sums<float, 4>(p, stream);
    return p.dim < 8 ? launch_sums<bf16_t, 1>(p, stream) : launch_sums<bf16_t, 8>(p, stream);
}

}  // namespace lbscan
