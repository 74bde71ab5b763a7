// The loss around its products (formulas: lbscan_loss.h): live tokens packed together, sums of the blocks' parts, results put
// in their tokens' places.
#include "lbscan_device.h"
#include "lbscan_embed.h"
#include "lbscan_internal.h"
#include "lbscan_loss.h"

namespace lbscan {
namespace {

template <typename T, int E> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[E]; };

struct Sources {
    long tokens;
    int vocab, wide_ids;
    const void* targets;
};
__device__ __forceinline__ int target_of(const Sources& s, long t)
{
    const long id = s.wide_ids ? static_cast<const int64_t*>(s.targets)[t] : (long)static_cast<const int32_t*>(s.targets)[t];
    return id >= 0 && id < s.vocab ? (int)id : -1;
}

constexpr int kGroup = 1024;                    // tokens of a block that numbers them

__device__ __forceinline__ int block_sum(int v, int* slots)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m, 64);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    v = slots[0] + slots[1] + slots[2] + slots[3];
    __syncthreads();
    return v;
}

// Live tokens of each group.
__global__ __launch_bounds__(256) void loss_count_kernel(const Sources s, int* __restrict__ counts)
{
    __shared__ int slots[4];
    int n = 0;
    for (int i = 0; i < kGroup / 256; ++i) {
        const long t = (long)blockIdx.x * kGroup + i * 256 + threadIdx.x;
        if (t < s.tokens) n += target_of(s, t) >= 0;
    }
    n = block_sum(n, slots);
    if (threadIdx.x == 0) counts[blockIdx.x] = n;
}

// How the products are cut.
struct Cuts {
    int vocab, dimp, piece, few, loose, element;
    long part_room, acc_rows, share_rows;
};
// The lane's candidate of smallest time, found by a wave.
__device__ __forceinline__ int best_of(float time, int candidate)
{
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const float other = __shfl_xor(time, m, 64);
        const int theirs = __shfl_xor(candidate, m, 64);
        if (other < time || (other == time && theirs < candidate)) { time = other; candidate = theirs; }
    }
    return candidate;
}
__device__ int best_chunk(int ntiles, int vtiles, int steps, int units, int most_chunks)
{
    const int rounds = (threadIdx.x & 63) + 1;
    int chunk = loss_chunk_of(ntiles, vtiles, rounds, units);
    if (loss_ceil32(vtiles, chunk) > most_chunks) chunk = loss_ceil32(vtiles, most_chunks);
    return best_of(loss_chunk_time(ntiles, vtiles, chunk, steps, units), chunk);
}
__device__ int best_splits(long tiles, int steps, int units, int element, long most)
{
    const int splits = (threadIdx.x & 63) + 1;
    const bool fits = splits <= loss_most_splits(units) && loss_split_fits(steps, splits, most);
    return best_of(fits ? loss_split_time(tiles, steps, splits, units, element) : INFINITY, splits);
}
__device__ void choose(LossChoice* out, const Cuts& c, int live)
{
    const int ntile = loss_tokens(c.few, c.element), wtile = loss_tokens(0, c.element), vtile = c.few ? loss_few_vocab(c.loose, c.element) : kLossTile;
    const int units = loss_units(c.few, c.loose, c.element), step = 64 / c.element, ntiles = loss_ceil32(live, ntile);
    LossChoice r{};
    r.live = live;
    r.rows = ntiles * ntile;
    r.chunk_lse = r.chunk_slope[0] = r.chunk_slope[1] = r.splits_x = r.splits_w[0] = r.splits_w[1] = 1;
    if (live) {
        const int steps = c.dimp / step, last = c.vocab - (c.vocab - 1) / c.piece * c.piece;
        if (c.part_room) r.chunk_lse = best_chunk(ntiles, loss_ceil32(c.vocab, vtile), steps, units, (int)(c.part_room / r.rows));
        else {
            const long mx = (long)loss_ceil32(c.dimp, vtile) * ntiles, mw = loss_ceil32(c.dimp, kLossTile);
            const int tokens = loss_ceil32(live, step);
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int count = k ? last : c.piece, tiles = loss_ceil32(count, wtile);
                r.chunk_slope[k] = best_chunk(ntiles, loss_ceil32(count, vtile), steps, units, 1 << 30);
                r.splits_w[k] = c.share_rows ? best_splits(mw * tiles, tokens, 256, c.element, c.share_rows / ((long)tiles * wtile)) : 1;
            }
            // (one number of parts for all pieces: their sums are added to)
            r.splits_x = best_splits(mx, loss_ceil32(c.piece < c.vocab ? c.piece : c.vocab, step), units, c.element, c.acc_rows / r.rows);
        }
    }
    if ((threadIdx.x & 63) == 0) *out = r;
}

struct Numbering {
    int *rank, *order, *targets;
    LossChoice* choice;
    Cuts cuts;
    float *lse2, *down, *both;                  // backward
    const float *lse, *dloss, *dlse;
};
// The live tokens' numbers, in the order of the tokens, and what the products need of each.
__global__ __launch_bounds__(256) void loss_rank_kernel(const Sources s, const int* __restrict__ counts, const Numbering o)
{
    __shared__ int slots[4], waves[4];
    int before = 0;
    for (int g = threadIdx.x; g < (int)blockIdx.x; g += 256) before += counts[g];
    before = block_sum(before, slots);
    // four tokens a thread, side by side
    const long t0 = (long)blockIdx.x * kGroup + 4 * threadIdx.x;
    int id[4], mine = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        id[i] = t0 + i < s.tokens ? target_of(s, t0 + i) : -1;
        mine += id[i] >= 0;
    }
    int up = mine;                              // inclusive sum over the wave
#pragma unroll
    for (int m = 1; m < 64; m *= 2) {
        const int other = __shfl_up(up, m, 64);
        if ((int)(threadIdx.x & 63) >= m) up += other;
    }
    if ((threadIdx.x & 63) == 63) waves[threadIdx.x >> 6] = up;
    __syncthreads();
    int r = before + up - mine;
    for (int w = 0; w < (int)(threadIdx.x >> 6); ++w) r += waves[w];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const long t = t0 + i;
        if (t >= s.tokens) break;
        o.rank[t] = id[i] >= 0 ? r : -1;
        if (id[i] < 0) continue;
        o.order[r] = (int)t;
        o.targets[r] = id[i];
        if (o.lse2) {
            const float down = o.dloss ? o.dloss[t] : 0.0f;
            o.lse2[r] = o.lse[t] * kLog2e;
            o.down[r] = down;
            o.both[r] = down + (o.dlse ? o.dlse[t] : 0.0f);
        }
        ++r;
    }
    // (the last thread of the last block has counted them all)
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x >= 192) choose(o.choice, o.cuts, __builtin_amdgcn_readlane(r, 63));
}

// A wave a row: `dim` elements and zeros up to `dimp`.
template <typename T>
__device__ __forceinline__ void copy_row(T* __restrict__ to, const T* __restrict__ from, int dim, int dimp, int lane)
{
    constexpr int E = 16 / sizeof(T);
    for (int c = lane * E; c < dimp; c += 64 * E) {
        Pack<T, E> q;
        if (c + E <= dim) q = *reinterpret_cast<const Pack<T, E>*>(from + c);
        else {
#pragma unroll
            for (int k = 0; k < E; ++k) q.v[k] = c + k < dim ? from[c + k] : T{};
        }
        *reinterpret_cast<Pack<T, E>*>(to + c) = q;
    }
}
// The live rows one behind the other, then rows of zeros to a whole tile; no targets behind the live ones.
template <typename T>
__global__ __launch_bounds__(256) void loss_gather_kernel(const T* __restrict__ x, T* __restrict__ out, const int* __restrict__ order,
                                                          int* __restrict__ targets, const LossChoice* __restrict__ choice, long rows, int dim,
                                                          int dimp, int tile)
{
    const int live = choice->live;
    const long end = min(rows, ((long)live + tile - 1) / tile * tile);
    for (long r = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < rows; r += (long)gridDim.x * 4) {
        const bool there = r < live;
        if (!there && (threadIdx.x & 63) == 0) targets[r] = -1;
        if (r >= end) continue;
        copy_row<T>(out + r * dimp, there ? x + (long)order[r] * dim : x, there ? dim : 0, dimp, threadIdx.x & 63);
    }
}
// At most 64 tokens: all of that in one launch, a wave a row; each of them finds its token from the targets (two launches, one
// behind the other, were 9 of 30 us of the loss of 64 x 50000 x 768 in bf16).
template <typename T>
__global__ __launch_bounds__(256) void loss_few_kernel(const Sources s, const T* __restrict__ x, T* __restrict__ out, const Numbering o, int dim, int dimp)
{
    const int lane = threadIdx.x & 63, r = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int id = lane < s.tokens ? target_of(s, lane) : -1;
    const unsigned long long there = __ballot(id >= 0);
    const int live = __popcll(there), mine = __popcll(there & ((1ull << lane) - 1));
    if (r < 64) {
        const int token = __ffsll(__ballot(id >= 0 && mine == r)) - 1;
        copy_row<T>(out + (long)r * dimp, token < 0 ? x : x + (long)token * dim, token < 0 ? 0 : dim, dimp, lane);
        return;
    }
    if (r > 64) return;                        // one wave more
    if (lane < s.tokens) o.rank[lane] = id >= 0 ? mine : -1;
    if (lane >= live) o.targets[lane] = -1;
    if (id >= 0) {
        o.targets[mine] = id;
        if (o.lse2) {
            const float down = o.dloss ? o.dloss[lane] : 0.0f;
            o.lse2[mine] = o.lse[lane] * kLog2e;
            o.down[mine] = down;
            o.both[mine] = down + (o.dlse ? o.dlse[lane] : 0.0f);
        }
    }
    choose(o.choice, o.cuts, live);
}
template <typename T>
__global__ __launch_bounds__(256) void loss_rows_kernel(const T* __restrict__ from, T* __restrict__ to, long rows, int dim, int dimp)
{
    for (long r = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < rows; r += (long)gridDim.x * 4)
        copy_row<T>(to + r * dimp, from + r * dim, dim, dimp, threadIdx.x & 63);
}

// E elements of a row of `end` from c, zeros behind it.
template <int E, typename T>
__device__ __forceinline__ Pack<T, E> part_of(const T* __restrict__ row, int c, int end)
{
    if (c + E <= end) return *reinterpret_cast<const Pack<T, E>*>(row + c);
    Pack<T, E> q;
#pragma unroll
    for (int k = 0; k < E; ++k) q.v[k] = c + k < end ? row[c + k] : T{};
    return q;
}

// bf16: the slopes at the targets, rounded for G, and what is left of them; with rest_rows that times the tokens' rows.  A
// wave a token.
__global__ __launch_bounds__(256) void loss_target_kernel(const bf16_t* __restrict__ x, const bf16_t* __restrict__ w, const int* __restrict__ targets,
                                                          const float* __restrict__ lse2, const float* __restrict__ down,
                                                          const float* __restrict__ both, float* __restrict__ hot, float* __restrict__ rest,
                                                          bf16_t* __restrict__ rest_rows, const LossChoice* __restrict__ choice, int dimp,
                                                          int ldw, float scale)
{
    const int live = choice->live, lane = threadIdx.x & 63;
    for (long r = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < live; r += (long)gridDim.x * 4) {
        const bf16_t *mine = x + r * dimp, *row = w + (long)targets[r] * ldw;
        float dot = 0.0f;
#pragma unroll 2
        for (int c = lane * 8; c < dimp; c += 512) {
            const Pack<bf16_t, 8> a = *reinterpret_cast<const Pack<bf16_t, 8>*>(mine + c), b = part_of<8>(row, c, ldw);
#pragma unroll
            for (int k = 0; k < 8; ++k) dot = fmaf(to_f32(a.v[k]), to_f32(b.v[k]), dot);
        }
#pragma unroll
        for (int m = 1; m < 64; m *= 2) dot += __shfl_xor(dot, m, 64);
        const float slope = both[r] * fast_exp2(fmaf(dot, scale * kLog2e, -lse2[r])) - down[r];
        const float rounded = to_f32(from_f32<bf16_t>(slope)), left = slope - rounded;
        if (lane == 0) { hot[r] = rounded; rest[r] = left; }
        if (!rest_rows) continue;
        for (int c = lane * 8; c < dimp; c += 512) {
            const Pack<bf16_t, 8> a = *reinterpret_cast<const Pack<bf16_t, 8>*>(mine + c);
            Pack<bf16_t, 8> o;
#pragma unroll
            for (int k = 0; k < 8; ++k) o.v[k] = from_f32<bf16_t>(left * to_f32(a.v[k]));
            *reinterpret_cast<Pack<bf16_t, 8>*>(rest_rows + r * dimp + c) = o;
        }
    }
}

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2)
{
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
    s = s * fast_exp2(m - base) + s2 * fast_exp2(m2 - base);
    m = top;
}
// lse and loss of TOKENS tokens a block, 256 / TOKENS threads to each.  With m and s the maximum and sum to base 2 and e the target's
// exponent, computed as the sum's terms are (rounded once, in the difference with m), loss = log2(s 2^-e) ln2.  Near the maximum
// that is the logarithm of the ratio of the sum to the target's own term in it: at least one, and one where there is nothing
// else, so that a certain token's loss is zero or more and as exact as the sum is, whatever the logits' size (from lse - l it was off by
// some 2^-24 of |l|).  Farther away the term may vanish, and the difference of the logarithms is at least ln2.
template <int TOKENS>
__global__ __launch_bounds__(256) void loss_join_kernel(const float2* __restrict__ part, const float* __restrict__ own,
                                                        const int* __restrict__ rank, float* __restrict__ loss, float* __restrict__ lse,
                                                        long tokens, int vtiles, const LossChoice* __restrict__ choice, float scale2)
{
    constexpr int kPieces = 256 / TOKENS;
    const long rows = choice->rows, chunks = loss_ceil(vtiles, choice->chunk_lse);
    __shared__ float2 folds[kPieces][TOKENS + 1];
    const int at = threadIdx.x % TOKENS, piece = threadIdx.x / TOKENS;
    for (long first = (long)blockIdx.x * TOKENS; first < tokens; first += (long)gridDim.x * TOKENS) {
        const long t = first + at;
        const int r = t < tokens ? rank[t] : -1;
        float m = -INFINITY, s = 0.0f;
        if (r >= 0) {
#pragma unroll 4
            for (int c = piece; c < chunks; c += kPieces) {
                const float2 q = part[(long)c * rows + r];
                join(m, s, q.x, q.y);
            }
        }
        folds[piece][at] = float2{m, s};
        __syncthreads();
        for (int half = kPieces / 2; half >= 8; half /= 2) {
            if (piece < half) {
                join(m, s, folds[piece + half][at].x, folds[piece + half][at].y);
                folds[piece][at] = float2{m, s};
            }
            __syncthreads();
        }
        if (piece == 0 && t < tokens) {
            for (int k = 1; k < 8; ++k) join(m, s, folds[k][at].x, folds[k][at].y);
            float all = 0.0f, mine = 0.0f;
            if (r >= 0) {
                const float e = fmaf(own[r], scale2, -m);
                all = (m + fast_log2(s)) * kLn2;
                mine = (e > -1.0f ? fast_log2(s / fast_exp2(e)) : fast_log2(s) - e) * kLn2;
            }
            lse[t] = all;
            loss[t] = mine;
        }
        __syncthreads();
    }
}

// dx: the sums' parts added in their order, in their tokens' places; zeros for the others.  A wave has 256 columns of a token.
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_kernel(const float* __restrict__ acc, const int* __restrict__ rank, const float* __restrict__ rest,
                                                      const int* __restrict__ targets, const T* __restrict__ weight, T* __restrict__ dx, long tokens, int dim,
                                                      int dimp, int ldw, const LossChoice* __restrict__ choice, float scale)
{
    const long rows = choice->rows;
    const int splits = choice->splits_x, strips = (dim + 255) / 256;
    const long all = tokens * strips;
    for (long w = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); w < all; w += (long)gridDim.x * 4) {
        const long t = w / strips;
        const int r = rank[t], c = (int)(w - t * strips) * 256 + (threadIdx.x & 63) * 4;
        if (c >= dim) continue;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r >= 0) {
#pragma unroll 8
            for (int k = 0; k < splits; ++k) {
                const Pack<float, 4> q = *reinterpret_cast<const Pack<float, 4>*>(acc + ((long)k * rows + r) * dimp + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += q.v[i];
            }
            if constexpr (sizeof(T) == 2) {
                const Pack<T, 4> row = part_of<4>(weight + (long)targets[r] * ldw, c, ldw);
                const float left = rest[r];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = fmaf(left, to_f32(row.v[i]), v[i]);
            }
        }
        Pack<T, 4> o;
#pragma unroll
        for (int i = 0; i < 4; ++i) o.v[i] = from_f32<T>(v[i] * scale);
        T* to = dx + t * dim + c;
        if (c + 4 <= dim) *reinterpret_cast<Pack<T, 4>*>(to) = o;
        else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (c + i < dim) to[i] = o.v[i];
        }
    }
}
// dweight of a piece of the vocabulary, likewise.
template <typename T>
__global__ __launch_bounds__(256) void loss_dweight_kernel(const float* __restrict__ share, T* __restrict__ dweight, int count, int dim, int dimp,
                                                           const int* __restrict__ tokens_of, const int* __restrict__ slot, const T* __restrict__ list,
                                                           const LossChoice* __restrict__ choice, int last, float scale)
{
    constexpr int tile = loss_tokens(0, sizeof(T));
    const long columns = loss_ceil(count, tile) * tile;
    const int splits = choice->splits_w[last];
    if (splits == 1) return;                                    // (written by the products)
    for (long v = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); v < count; v += (long)gridDim.x * 4)
        for (int c = (threadIdx.x & 63) * 4; c < dim; c += 256) {
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < splits; ++k) {
                const Pack<float, 4> q = *reinterpret_cast<const Pack<float, 4>*>(share + (k * columns + v) * dimp + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += q.v[i];
            }
            if (sizeof(T) == 2 && tokens_of[v] > 0) {
                const Pack<T, 4> rest = *reinterpret_cast<const Pack<T, 4>*>(list + (long)slot[v] * dimp + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += to_f32(rest.v[i]);
            }
            Pack<T, 4> o;
#pragma unroll
            for (int i = 0; i < 4; ++i) o.v[i] = from_f32<T>(s[i] * scale);
            T* to = dweight + v * dim + c;
            if (c + 4 <= dim) *reinterpret_cast<Pack<T, 4>*>(to) = o;
            else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (c + i < dim) to[i] = o.v[i];
            }
        }
}
template <typename T>
__global__ __launch_bounds__(256) void loss_zero_kernel(T* __restrict__ out, long n)
{
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < n; i += (long)gridDim.x * 256) out[i] = T{};
}

unsigned some(long blocks) { return (unsigned)(blocks < 1 ? 1 : blocks < 8192 ? blocks : 8192); }

struct Scratch {
    char* base;
    template <typename P> P* at(size_t offset) const { return reinterpret_cast<P*>(base + offset); }
};

// Numbers of the live tokens, their rows, and the table in whole steps.
template <typename T>
hipError_t pack(const LossParams& p, const LossPlan& plan, const Scratch& s, bool backward, hipStream_t stream)
{
    const Sources src{p.tokens, p.vocab, p.wide_ids, p.targets};
    const long groups = (p.tokens + kGroup - 1) / kGroup;
    int* counts = s.at<int>(plan.counts);
    if (groups > 1) {                                          // (the first group needs no counts)
        loss_count_kernel<<<(unsigned)groups, 256, 0, stream>>>(src, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    Numbering o{s.at<int>(plan.rank), s.at<int>(plan.order), s.at<int>(plan.targets), s.at<LossChoice>(plan.choice),
                Cuts{p.vocab, plan.dimp, plan.piece, plan.few, plan.loose, (int)sizeof(T), plan.part_room, plan.acc_rows, plan.share_rows},
                nullptr, nullptr, nullptr, p.lse, p.dloss, p.dlse};
    if (backward) { o.lse2 = s.at<float>(plan.lse2); o.down = s.at<float>(plan.down); o.both = s.at<float>(plan.both); }
    const T* x = static_cast<const T*>(p.x);
    hipError_t e;
    if (plan.few) {
        loss_few_kernel<T><<<17, 256, 0, stream>>>(src, x, s.at<T>(plan.x), o, p.dim, plan.dimp);
        e = hipGetLastError();
    } else {
        loss_rank_kernel<<<(unsigned)groups, 256, 0, stream>>>(src, counts, o);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
        loss_gather_kernel<T><<<some(plan.rows / 4), 256, 0, stream>>>(x, s.at<T>(plan.x), o.order, o.targets, o.choice, plan.rows, p.dim,
                                                                     plan.dimp, loss_tokens(0, sizeof(T)));
        e = hipGetLastError();
    }
    if (e != hipSuccess || !plan.copy_weight) return e;
    loss_rows_kernel<T><<<some((p.vocab + 3L) / 4), 256, 0, stream>>>(static_cast<const T*>(p.weight), s.at<T>(plan.w), p.vocab, p.dim, plan.dimp);
    return hipGetLastError();
}

LossTiles tiles_of(const LossParams& p, const LossPlan& plan, const Scratch& s)
{
    LossTiles t{};
    t.choice = s.at<LossChoice>(plan.choice);
    t.w = plan.copy_weight ? s.at<void>(plan.w) : p.weight;
    t.x = s.at<void>(plan.x);
    t.targets = s.at<int>(plan.targets);
    t.vocab = p.vocab; t.dim = p.dim; t.dimp = plan.dimp; t.ldw = plan.loose ? p.dim : plan.dimp; t.piece = plan.piece;
    t.first = 0; t.count = p.vocab;
    t.last = 1;
    t.scale = p.scale;
    return t;
}

// The sums by target, as the gradient of an embedding kept as a list.
EmbedParams list_params(const LossParams& p, const LossPlan& plan)
{
    EmbedParams q{};
    q.tokens = plan.rows;
    q.vocab = p.vocab;
    q.dim = plan.dimp;
    q.dtype = p.dtype;
    q.scale = 1.0f;
    return q;
}

template <typename T>
hipError_t forward(const LossParams& p, const LossPlan& plan, const Scratch& s, hipStream_t stream)
{
    hipError_t e = pack<T>(p, plan, s, false, stream);
    if (e != hipSuccess) return e;
    LossTiles t = tiles_of(p, plan, s);
    t.own = s.at<float>(plan.own);
    t.part = s.at<float2>(plan.part);
    e = (sizeof(T) == 4 ? launch_loss_tiles_f32 : launch_loss_tiles_bf16)(LossKind::lse, t, plan.few, plan.loose, stream);
    if (e != hipSuccess) return e;
    const int vtiles = (int)loss_ceil(p.vocab, plan.few ? loss_few_vocab(plan.loose, sizeof(T)) : kLossTile);
    const float scale2 = p.scale * kLog2e;
    if (plan.few) loss_join_kernel<4><<<some((p.tokens + 3) / 4), 256, 0, stream>>>(t.part, t.own, s.at<int>(plan.rank), p.loss, p.lse, p.tokens,
                                                                                  vtiles, t.choice, scale2);
    else loss_join_kernel<16><<<some((p.tokens + 15) / 16), 256, 0, stream>>>(t.part, t.own, s.at<int>(plan.rank), p.loss, p.lse, p.tokens, vtiles,
                                                                            t.choice, scale2);
    return hipGetLastError();
}

template <typename T>
hipError_t backward(const LossParams& p, const LossPlan& plan, const Scratch& s, hipStream_t stream)
{
    const auto launch = sizeof(T) == 4 ? launch_loss_tiles_f32 : launch_loss_tiles_bf16;
    hipError_t e = pack<T>(p, plan, s, true, stream);
    LossTiles t = tiles_of(p, plan, s);
    t.lse2 = s.at<float>(plan.lse2); t.down = s.at<float>(plan.down); t.both = s.at<float>(plan.both);
    t.g = s.at<void>(plan.g);
    t.acc = s.at<float>(plan.acc);
    t.share = s.at<float>(plan.share);
    t.dweight = p.dweight;
    if constexpr (sizeof(T) == 2) {
        if (e != hipSuccess) return e;
        bf16_t* rows = p.dweight ? s.at<bf16_t>(plan.rest_rows) : nullptr;
        loss_target_kernel<<<some((p.tokens + 3) / 4), 256, 0, stream>>>(static_cast<const bf16_t*>(t.x), static_cast<const bf16_t*>(t.w), t.targets,
                                                                       t.lse2, t.down, t.both, s.at<float>(plan.hot), s.at<float>(plan.rest), rows,
                                                                       t.choice, plan.dimp, t.ldw, p.scale);
        e = hipGetLastError();
        if (e == hipSuccess && p.dweight) {
            EmbedParams q = list_params(p, plan);
            q.ids = t.targets;
            q.dout = rows;
            q.dweight = s.at<void>(plan.list);
            q.slot = s.at<int>(plan.slot);
            e = launch_embed_bwd(q, s.at<void>(plan.sort), stream);
            t.tokens_of = embed_counts(q, s.at<void>(plan.sort));
            t.slot = q.slot;
            t.list = q.dweight;
        }
        t.down = s.at<float>(plan.hot);
    }
    for (t.first = 0; t.first < p.vocab && e == hipSuccess; t.first += plan.piece) {
        t.count = p.vocab - t.first < plan.piece ? p.vocab - t.first : plan.piece;
        t.last = t.first + plan.piece >= p.vocab;
        e = launch(LossKind::slope, t, plan.few, plan.loose, stream);
        if (e == hipSuccess && p.dx) {
            t.add = t.first > 0;
            e = launch(LossKind::dx, t, plan.few, plan.loose, stream);
        }
        if (e == hipSuccess && p.dweight) {
            e = launch(LossKind::dweight, t, plan.few, plan.loose, stream);
            if (e == hipSuccess && plan.share_rows) {
                loss_dweight_kernel<T><<<some((t.count + 3L) / 4), 256, 0, stream>>>(t.share, static_cast<T*>(p.dweight) + (long)t.first * p.dim, t.count,
                                                                                   p.dim, plan.dimp, t.tokens_of + t.first, t.slot + t.first,
                                                                                   static_cast<const T*>(t.list), t.choice, t.last, p.scale);
                e = hipGetLastError();
            }
        }
    }
    if (e != hipSuccess || !p.dx) return e;
    loss_dx_kernel<T><<<some((p.tokens * ((p.dim + 255) / 256) + 3) / 4), 256, 0, stream>>>(t.acc, s.at<int>(plan.rank), s.at<float>(plan.rest),
                                                                  t.targets, static_cast<const T*>(t.w), static_cast<T*>(p.dx), p.tokens, p.dim, plan.dimp,
                                                                  t.ldw, t.choice, p.scale);
    return hipGetLastError();
}

template <typename T>
hipError_t zero(void* out, long n, hipStream_t stream)
{
    if (!out || n == 0) return hipSuccess;
    loss_zero_kernel<T><<<some((n + 255) / 256), 256, 0, stream>>>(static_cast<T*>(out), n);
    return hipGetLastError();
}

}  // namespace

LossPlan loss_plan(const LossParams& p, bool backward)
{
    auto plan = [&](size_t sort_bytes) {
        return loss_plan_of(p.tokens, p.vocab, p.dim, p.dtype == 0 ? 4 : 2, (reinterpret_cast<uintptr_t>(p.weight) & 15) == 0, backward,
                            p.dx != nullptr, p.dweight != nullptr, sort_bytes);
    };
    if (p.dtype == 0 || !backward || !p.dweight || p.tokens == 0 || p.vocab == 0) return plan(0);
    return plan(embed_bwd_bytes(list_params(p, plan(0))));
}

hipError_t launch_loss_fwd(const LossParams& p, const LossPlan& plan, void* workspace, hipStream_t stream)
{
    if (p.vocab == 0 || p.tokens == 0) {            // no token has a target
        const hipError_t e = zero<float>(p.loss, p.tokens, stream);
        return e == hipSuccess ? zero<float>(p.lse, p.tokens, stream) : e;
    }
    const Scratch s{static_cast<char*>(workspace)};
    return p.dtype == 0 ? forward<float>(p, plan, s, stream) : forward<bf16_t>(p, plan, s, stream);
}

hipError_t launch_loss_bwd(const LossParams& p, const LossPlan& plan, void* workspace, hipStream_t stream)
{
    if (p.vocab == 0 || p.tokens == 0) {
        const long nx = p.tokens * p.dim, nw = (long)p.vocab * p.dim;
        hipError_t e = p.dtype == 0 ? zero<float>(p.dx, nx, stream) : zero<bf16_t>(p.dx, nx, stream);
        if (e == hipSuccess) e = p.dtype == 0 ? zero<float>(p.dweight, nw, stream) : zero<bf16_t>(p.dweight, nw, stream);
        return e;
    }
    const Scratch s{static_cast<char*>(workspace)};
    return p.dtype == 0 ? backward<float>(p, plan, s, stream) : backward<bf16_t>(p, plan, s, stream);
}

}  // namespace lbscan
