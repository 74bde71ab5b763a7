// The loss around its products (formulas: lbscan_loss.h): live tokens packed together, sums of the blocks' parts, results put
// in their tokens' places.
#include "lbscan_device.h"
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

struct Numbering {
    int *rank, *order, *targets, *live;
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
    if (blockIdx.x == gridDim.x - 1 && threadIdx.x == 255) *o.live = r;
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
// The live rows one behind the other, then rows of zeros (of no target) to a whole tile.
template <typename T>
__global__ __launch_bounds__(256) void loss_gather_kernel(const T* __restrict__ x, T* __restrict__ out, const int* __restrict__ order,
                                                          int* __restrict__ targets, const int* __restrict__ live_tokens, long rows, int dim,
                                                          int dimp, int tile)
{
    const int live = *live_tokens;
    const long end = min(rows, ((long)live + tile - 1) / tile * tile);
    for (long r = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < end; r += (long)gridDim.x * 4) {
        const bool there = r < live;
        if (!there && (threadIdx.x & 63) == 0) targets[r] = -1;
        copy_row<T>(out + r * dimp, there ? x + (long)order[r] * dim : x, there ? dim : 0, dimp, threadIdx.x & 63);
    }
}
template <typename T>
__global__ __launch_bounds__(256) void loss_rows_kernel(const T* __restrict__ from, T* __restrict__ to, long rows, int dim, int dimp)
{
    for (long r = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); r < rows; r += (long)gridDim.x * 4)
        copy_row<T>(to + r * dimp, from + r * dim, dim, dimp, threadIdx.x & 63);
}

__device__ __forceinline__ void join(float& m, float& s, float m2, float s2)
{
    const float top = fmaxf(m, m2), base = top == -INFINITY ? 0.0f : top;
    s = s * fast_exp2(m - base) + s2 * fast_exp2(m2 - base);
    m = top;
}
// lse and loss of 16 tokens a block, 16 threads to each.
__global__ __launch_bounds__(256) void loss_join_kernel(const float2* __restrict__ part, const float* __restrict__ own,
                                                        const int* __restrict__ rank, float* __restrict__ loss, float* __restrict__ lse,
                                                        long tokens, long rows, int chunks)
{
    __shared__ float2 folds[16][17];
    const int at = threadIdx.x & 15, piece = threadIdx.x >> 4;
    for (long first = (long)blockIdx.x * 16; first < tokens; first += (long)gridDim.x * 16) {
        const long t = first + at;
        const int r = t < tokens ? rank[t] : -1;
        float m = -INFINITY, s = 0.0f;
        if (r >= 0) {
#pragma unroll 4
            for (int c = piece; c < chunks; c += 16) {
                const float2 q = part[(long)c * rows + r];
                join(m, s, q.x, q.y);
            }
        }
        folds[piece][at] = float2{m, s};
        __syncthreads();
        if (piece == 0 && t < tokens) {
            for (int k = 1; k < 16; ++k) join(m, s, folds[k][at].x, folds[k][at].y);
            const float v = r >= 0 ? (m + fast_log2(s)) * kLn2 : 0.0f;
            lse[t] = v;
            loss[t] = r >= 0 ? v - own[r] : 0.0f;
        }
        __syncthreads();
    }
}

// dx: the sums' pieces added in their order, in their tokens' places; zeros for the others.  A wave a token.
template <typename T>
__global__ __launch_bounds__(256) void loss_dx_kernel(const float* __restrict__ acc, const int* __restrict__ rank, T* __restrict__ dx,
                                                      long tokens, long rows, int dim, int dimp, int splits, float scale)
{
    for (long t = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); t < tokens; t += (long)gridDim.x * 4) {
        const int r = rank[t];
        for (int c = (threadIdx.x & 63) * 4; c < dim; c += 256) {
            float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (r >= 0)
                for (int k = 0; k < splits; ++k) {
                    const Pack<float, 4> q = *reinterpret_cast<const Pack<float, 4>*>(acc + ((long)k * rows + r) * dimp + c);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i] += q.v[i];
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
}
// dweight of a piece of the vocabulary, likewise.
template <typename T>
__global__ __launch_bounds__(256) void loss_dweight_kernel(const float* __restrict__ share, T* __restrict__ dweight, int count, long piece,
                                                           int dim, int dimp, int splits, float scale)
{
    for (long v = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); v < count; v += (long)gridDim.x * 4)
        for (int c = (threadIdx.x & 63) * 4; c < dim; c += 256) {
            float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            for (int k = 0; k < splits; ++k) {
                const Pack<float, 4> q = *reinterpret_cast<const Pack<float, 4>*>(share + (k * piece + v) * dimp + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[i] += q.v[i];
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
    if (groups > 1) {
        loss_count_kernel<<<(unsigned)groups, 256, 0, stream>>>(src, counts);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    Numbering o{s.at<int>(plan.rank), s.at<int>(plan.order), s.at<int>(plan.targets), s.at<int>(plan.live), nullptr, nullptr, nullptr,
                p.lse, p.dloss, p.dlse};
    if (backward) { o.lse2 = s.at<float>(plan.lse2); o.down = s.at<float>(plan.down); o.both = s.at<float>(plan.both); }
    loss_rank_kernel<<<(unsigned)groups, 256, 0, stream>>>(src, counts, o);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    loss_gather_kernel<T><<<some(plan.rows / 4), 256, 0, stream>>>(static_cast<const T*>(p.x), s.at<T>(plan.x), o.order, o.targets, o.live,
                                                                 plan.rows, p.dim, plan.dimp, plan.few ? kLossFewTokens : kLossTile);
    e = hipGetLastError();
    if (e != hipSuccess || !plan.copy_weight) return e;
    loss_rows_kernel<T><<<some((p.vocab + 3L) / 4), 256, 0, stream>>>(static_cast<const T*>(p.weight), s.at<T>(plan.w), p.vocab, p.dim, plan.dimp);
    return hipGetLastError();
}

LossTiles tiles_of(const LossParams& p, const LossPlan& plan, const Scratch& s)
{
    LossTiles t{};
    t.live = s.at<int>(plan.live);
    t.w = plan.copy_weight ? s.at<void>(plan.w) : p.weight;
    t.x = s.at<void>(plan.x);
    t.targets = s.at<int>(plan.targets);
    t.rows = plan.rows;
    t.vocab = p.vocab; t.dim = p.dim; t.dimp = plan.dimp; t.ldw = plan.dimp; t.piece = plan.piece;
    t.first = 0; t.count = p.vocab;
    t.chunk = plan.chunk;
    t.splits = 1;
    t.scale = p.scale;
    return t;
}

template <typename T>
hipError_t forward(const LossParams& p, const LossPlan& plan, const Scratch& s, hipStream_t stream)
{
    hipError_t e = pack<T>(p, plan, s, false, stream);
    if (e != hipSuccess) return e;
    LossTiles t = tiles_of(p, plan, s);
    t.own = s.at<float>(plan.own);
    t.part = s.at<float2>(plan.part);
    e = (sizeof(T) == 4 ? launch_loss_tiles_f32 : launch_loss_tiles_bf16)(LossKind::lse, t, plan.few, stream);
    if (e != hipSuccess) return e;
    loss_join_kernel<<<some((p.tokens + 15) / 16), 256, 0, stream>>>(t.part, t.own, s.at<int>(plan.rank), p.loss, p.lse, p.tokens, plan.rows,
                                                                   plan.chunks);
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
    for (t.first = 0; t.first < p.vocab && e == hipSuccess; t.first += plan.piece) {
        t.count = p.vocab - t.first < plan.piece ? p.vocab - t.first : plan.piece;
        e = launch(LossKind::slope, t, plan.few, stream);
        if (e == hipSuccess && p.dx) {
            t.splits = plan.splits_x;
            t.add = t.first > 0;
            e = launch(LossKind::dx, t, plan.few, stream);
        }
        if (e == hipSuccess && p.dweight) {
            t.splits = plan.splits_w;
            e = launch(LossKind::dweight, t, plan.few, stream);
            if (e == hipSuccess && plan.splits_w > 1) {
                loss_dweight_kernel<T><<<some((t.count + 3L) / 4), 256, 0, stream>>>(t.share, static_cast<T*>(p.dweight) + (long)t.first * p.dim, t.count,
                                                                                   plan.piece, p.dim, plan.dimp, plan.splits_w, p.scale);
                e = hipGetLastError();
            }
        }
    }
    if (e != hipSuccess || !p.dx) return e;
    loss_dx_kernel<T><<<some((p.tokens + 3) / 4), 256, 0, stream>>>(t.acc, s.at<int>(plan.rank), static_cast<T*>(p.dx), p.tokens, plan.rows, p.dim,
                                                                  plan.dimp, plan.splits_x, p.scale);
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
    return loss_plan_of(p.tokens, p.vocab, p.dim, p.dtype == 0 ? 4 : 2, (reinterpret_cast<uintptr_t>(p.weight) & 15) == 0, backward,
                        p.dx != nullptr, p.dweight != nullptr);
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
