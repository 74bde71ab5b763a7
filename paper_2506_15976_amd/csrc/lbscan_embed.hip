// Token embedding and its gradient (formulas: lbscan_embed.h).  All of it is bound by memory: the lookup by
// the rows read and written, the gradient by the table written and dout read once.
#include "lbscan_device.h"
#include "lbscan_embed.h"
#include "lbscan_internal.h"

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
// One launch.  Block r of R (a power of two) has the rows v = r mod R, so that rows that are used much and lie
// next to each other in a table ordered by frequency go to different blocks.  Every block reads all ids:
// it counts those of blocks before it, which is where its own begin, and its own by row and by sixteenth
// of the tokens (a wave each).  The running sums of these counts are where each wave puts its tokens; a wave
// takes its tokens in order, so that those of a row stay in the order of the tokens.
constexpr int kSortWaves = 16;
constexpr int kSortRows = 512;             // most rows of a block: 32 KB of counts
constexpr int kSortAhead = 4;              // groups of 64 ids that a wave loads together

int sort_blocks_log2(int vocab)
{
    int log2 = 8;
    while (((long)kSortRows << log2) < vocab) ++log2;
    return log2;
}

template <typename I>
__global__ __launch_bounds__(64 * kSortWaves) void embed_sort_kernel(const EmbedParams p, int blocks_log2)
{
    extern __shared__ int counts[];        // (waves, rows)
    __shared__ int totals[kSortWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int mine = blockIdx.x, mask = (1 << blocks_log2) - 1;
    const int rows = (p.vocab - mine + mask) >> blocks_log2;          // v = mine + k * blocks < vocab
    const I* ids = static_cast<const I*>(p.ids);
    const long share = ((p.tokens + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
    const long begin = min(share * wave, p.tokens), end = min(begin + share, p.tokens);

    for (int k = threadIdx.x; k < rows * kSortWaves; k += 64 * kSortWaves) counts[k] = 0;
    __syncthreads();
    int below = 0;
    for (long t = begin; t < end; t += 64 * kSortAhead) {
        int v[kSortAhead];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            const long at = t + 64 * k + lane;
            v[k] = row_of(ids[min(at, p.tokens - 1)], p.vocab);
            if (at >= end) v[k] = -1;
        }
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            below += v[k] >= 0 && (v[k] & mask) < mine;
            if (v[k] >= 0 && (v[k] & mask) == mine) atomicAdd(&counts[wave * rows + (v[k] >> blocks_log2)], 1);
        }
    }
#pragma unroll
    for (int m = 1; m < 64; m *= 2) below += __shfl_xor(below, m);
    if (lane == 0) totals[wave] = below;
    __syncthreads();
    below = 0;
    for (int w = 0; w < kSortWaves; ++w) below += totals[w];
    __syncthreads();

    // running sums, rows first: a thread a row
    int n = 0;
    if ((int)threadIdx.x < rows) {
        for (int w = 0; w < kSortWaves; ++w) n += counts[w * rows + threadIdx.x];
        p.count[mine + ((int)threadIdx.x << blocks_log2)] = n;
    }
    int sum = n;
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int other = __shfl_up(sum, m);
        if (lane >= m) sum += other;
    }
    if (lane == 63) totals[wave] = sum;
    __syncthreads();
    int at = below + sum - n, own = 0;
    for (int w = 0; w < kSortWaves; ++w) {
        if (w < wave) at += totals[w];
        own += totals[w];
    }
    if ((int)threadIdx.x < rows)
        for (int w = 0; w < kSortWaves; ++w) {
            const int c = counts[w * rows + threadIdx.x];
            counts[w * rows + threadIdx.x] = at;
            at += c;
        }
    if (mine == mask && threadIdx.x == 0) *p.valid = below + own;
    __syncthreads();

    volatile int* next = counts + wave * rows;       // of this wave alone
    for (long t = begin; t < end; t += 64 * kSortAhead) {
        int v[kSortAhead];
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            const long i = t + 64 * k + lane;
            v[k] = row_of(ids[min(i, p.tokens - 1)], p.vocab);
            if (i >= end || (v[k] & mask) != mine) v[k] = -1;
        }
#pragma unroll
        for (int k = 0; k < kSortAhead; ++k) {
            uint64_t left = __ballot(v[k] >= 0);
            while (left) {                            // the lanes of one row at a time
                const int leader = __builtin_ctzll(left);
                const int r = __builtin_amdgcn_readlane(v[k], leader);
                const uint64_t same = __ballot(v[k] == r);
                const int where = next[r >> blocks_log2];
                if (v[k] == r) {
                    const int o = where + __builtin_popcountll(same & ((1ull << lane) - 1));
                    p.place[o] = (int)(t + 64 * k + lane);
                    p.row[o] = r;
                }
                if (lane == leader) next[r >> blocks_log2] = where + __builtin_popcountll(same);
                left &= ~same;
            }
        }
    }
}

// ---- gradient: sums over the sorted tokens -----------------------------------------------------------
// A wave takes a piece of kPiece sorted tokens and 64 packs of columns, and adds dout row by row.  A row of the
// table whose tokens all lie in the piece is written; of others the sum goes to scratch: [0] of a row that
// began in an earlier piece, [1] of one that begins here and goes on.  The waves behind the pieces write zeros to the
// rows that no token has.
constexpr int kPiece = 32;
constexpr int kPieceAhead = 8;
constexpr int kZeroRows = 16;              // rows that such a wave looks at

template <typename T, int E>
__device__ __forceinline__ void write_row(const EmbedParams& p, int row, int col, const float acc[E])
{
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
    if (task >= pieces * tiles) {
        const long v0 = (long)(task - pieces * tiles) * kZeroRows;
        if (v0 >= p.vocab) return;
        const int v = (int)v0 + (lane & (kZeroRows - 1));
        uint64_t empty = __ballot(lane < kZeroRows && v < p.vocab && p.count[min(v, p.vocab - 1)] == 0);
        const float zeros[E] = {};
        while (empty) {
            const int k = __builtin_ctzll(empty);
            empty &= empty - 1;
            for (int c = lane; c < packs; c += 64) write_row<T, E>(p, (int)v0 + k, column_of<E>(c, dim), zeros);
        }
        return;
    }
    const int piece = (int)(task / tiles), c = (int)(task % tiles) * 64 + lane;
    const int valid = *p.valid, first = piece * kPiece, n = min(kPiece, valid - first);
    if (n <= 0) return;
    const bool there = c < packs;
    const int col = column_of<E>(min(c, packs - 1), dim);
    const int my_place = p.place[first + min(lane, n - 1)], my_row = p.row[first + min(lane, n - 1)];
    const int row_before = first > 0 ? p.row[first - 1] : -1, row_after = first + n < valid ? p.row[first + n] : -1;
    const T* dout = static_cast<const T*>(p.dout);

    float acc[E] = {};
    int begun = 0;                          // where the present row's tokens begin in the piece
    for (int k0 = 0; k0 < n; k0 += kPieceAhead) {
        Pack<T, E> q[kPieceAhead];
#pragma unroll
        for (int k = 0; k < kPieceAhead; ++k) {
            const int token = __builtin_amdgcn_readlane(my_place, min(k0 + k, n - 1));
            q[k] = *reinterpret_cast<const Pack<T, E>*>(dout + (long)token * dim + col);
        }
#pragma unroll
        for (int k = 0; k < kPieceAhead; ++k) {
            const int at = k0 + k;
            if (at < n) {
                const int row = __builtin_amdgcn_readlane(my_row, at);
                const int follows = at + 1 < n ? __builtin_amdgcn_readlane(my_row, at + 1) : row_after;
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += to_f32(q[k].v[e]);
                if (row != follows || at + 1 == n) {
                    const bool early = begun == 0 && row_before == row, goes_on = row == follows;
                    if (there) {
                        if (!early && !goes_on) {
                            write_row<T, E>(p, row, col, acc);
                        } else {
                            float* to = p.part + ((long)piece * 2 + (early ? 0 : 1)) * dim + col;
#pragma unroll
                            for (int e = 0; e < E; ++e) to[e] = acc[e];
                        }
                    }
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[e] = 0.0f;
                    begun = at + 1;
                }
            }
        }
    }
}

// The rows whose tokens lie in several pieces: the piece in which they begin finds them by its last token and
// adds the others' sums, four waves a share each, in a fixed order.
template <typename T, int E>
__global__ __launch_bounds__(256) void embed_join_kernel(const EmbedParams p)
{
    __shared__ float sums[3][64][E];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int dim = p.dim, packs = (dim + E - 1) / E;
    const int piece = blockIdx.x, last = (piece + 1) * kPiece - 1, valid = *p.valid;
    if (last + 1 >= valid) return;                                     // nothing behind this piece
    const int row = p.row[last];
    if (p.row[last + 1] != row) return;
    if (piece > 0 && p.row[piece * kPiece - 1] == row) return;        // it began earlier
    // first token of the row: lanes compare the piece's rows
    const uint64_t same = __ballot(lane < kPiece && p.row[piece * kPiece + (lane & (kPiece - 1))] == row);
    const int begin = piece * kPiece + __builtin_ctzll(same);
    const int end_piece = (begin + p.count[row] - 1) / kPiece;        // the last piece that has some of it
    const int share = (end_piece - piece + 3) / 4;
    const int from = piece + 1 + wave * share, to = min(from + share, end_piece + 1);
    const int c = blockIdx.y * 64 + lane;
    const int col = column_of<E>(min(c, packs - 1), dim);
    float acc[E] = {};
    if (wave == 0) {
        const float* tail = p.part + ((long)piece * 2 + 1) * dim + col;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] = tail[e];
    }
#pragma unroll 4
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
    for (int w = 0; w < 3; ++w)
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] += sums[w][lane][e];
    write_row<T, E>(p, row, col, acc);
}

int pieces_of(const EmbedParams& p) { return (int)((p.tokens + kPiece - 1) / kPiece); }

template <typename T, int E>
hipError_t launch_fwd(const EmbedParams& p, hipStream_t stream)
{
    const long waves = (p.tokens + kLookup - 1) / kLookup;
    const int packs = (p.dim + E - 1) / E, tiles = (packs + 63) / 64;
    const dim3 grid((unsigned)((waves + 3) / 4), tiles < 64 ? tiles : 64);
    if (p.wide_ids) embed_fwd_kernel<T, int64_t, E><<<grid, 256, 0, stream>>>(p);
    else embed_fwd_kernel<T, int32_t, E><<<grid, 256, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T, int E>
hipError_t launch_sums(const EmbedParams& p, hipStream_t stream)
{
    const int pieces = pieces_of(p), packs = (p.dim + E - 1) / E, tiles = (packs + 63) / 64;
    const long tasks = (long)pieces * tiles + ((long)p.vocab + kZeroRows - 1) / kZeroRows;
    if (tasks > 0x7fffffffL) return hipErrorInvalidValue;
    embed_pieces_kernel<T, E><<<(unsigned)((tasks + 3) / 4), 256, 0, stream>>>(p, pieces, tiles);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || pieces < 2) return e;
    embed_join_kernel<T, E><<<dim3(pieces - 1, tiles), 256, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

size_t embed_bwd_bytes(const EmbedParams& p)
{
    return ((size_t)p.tokens * 2 + p.vocab + 1 + (size_t)pieces_of(p) * 2 * p.dim) * 4;
}

hipError_t launch_embed_fwd(const EmbedParams& p, hipStream_t stream)
{
    if (p.dtype == 0) return p.dim < 4 ? launch_fwd<float, 1>(p, stream) : launch_fwd<float, 4>(p, stream);
    return p.dim < 8 ? launch_fwd<bf16_t, 1>(p, stream) : launch_fwd<bf16_t, 8>(p, stream);
}

hipError_t launch_embed_bwd(EmbedParams p, void* workspace, hipStream_t stream)
{
    p.part = static_cast<float*>(workspace);
    p.place = reinterpret_cast<int*>(p.part + (size_t)pieces_of(p) * 2 * p.dim);
    p.row = p.place + p.tokens;
    p.count = p.row + p.tokens;
    p.valid = p.count + p.vocab;
    const int log2 = sort_blocks_log2(p.vocab);
    const size_t lds = (size_t)((p.vocab + (1 << log2) - 1) >> log2) * kSortWaves * sizeof(int);
    if (p.wide_ids) embed_sort_kernel<int64_t><<<1 << log2, 64 * kSortWaves, lds, stream>>>(p, log2);
    else embed_sort_kernel<int32_t><<<1 << log2, 64 * kSortWaves, lds, stream>>>(p, log2);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (p.dtype == 0) return p.dim < 4 ? launch_sums<float, 1>(p, stream) : launch_sums<float, 4>(p, stream);
    return p.dim < 8 ? launch_sums<bf16_t, 1>(p, stream) : launch_sums<bf16_t, 8>(p, stream);
}

}  // namespace lbscan
