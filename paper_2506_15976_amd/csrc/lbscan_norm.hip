// Layer norm and its gradient (formulas: lbscan_norm.h).
//
// A row is held in the registers of a team (16 lanes, a wave, or the waves of a block): it is read once, its
// mean and then the mean of the squared deviations are summed over the team (two passes over registers, so no
// difference of large numbers), and it is written once.  A team walks several rows with weight and bias (backward: the
// sums of their gradients) of its columns in registers, the next row's loads in flight.  Bound by memory: MI355X, three
// sets of inputs in turn, forward and gradients (with the launch that adds the blocks' shares), 32768 x 768 bf16 with a
// residual 55.1 us (5.5 TB/s) and 77.9 (5.2), 25216 x 384 fp32 15.2 (5.1) and 25.8 (4.5), 2048 x 8192 bf16 15.3 (4.4) and
// 33.3 (3.0: a block has eight rows and a share as large as four of them, which it stores element by element, 59.6 MB
// for the 50.3 that are needed).  A row of more columns is read three times, an element a lane at a time, its gradients'
// columns once more: 2048 x 16384 bf16 83 us (1.6 TB/s) and 120 (1.7).
#include "lbscan_device.h"
#include "lbscan_internal.h"
#include "lbscan_norm.h"

namespace lbscan {
namespace {

// E consecutive elements, at any element's address.
template <typename T, int E> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[E]; };

template <typename T, int E>
__device__ __forceinline__ void get(const T* __restrict__ p, float out[E])
{
    const Pack<T, E> q = *reinterpret_cast<const Pack<T, E>*>(p);
#pragma unroll
    for (int e = 0; e < E; ++e) out[e] = to_f32(q.v[e]);
}
template <typename T, int E>
__device__ __forceinline__ void put(T* __restrict__ p, const float in[E])
{
    Pack<T, E> q;
#pragma unroll
    for (int e = 0; e < E; ++e) q.v[e] = from_f32<T>(in[e]);
    *reinterpret_cast<Pack<T, E>*>(p) = q;
}

template <int CTRL>
__device__ __forceinline__ float turned(float v)
{
    return __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float lane_of(float v, int lane)
{
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane));
}
// Sum over 16 lanes (G = 16) or a wave (G = 64), the same in every lane.
template <int G>
__device__ __forceinline__ float lanes_sum(float v)
{
    v += turned<0x128>(v);                                        // row_ror 8, 4, 2, 1
    v += turned<0x124>(v);
    v += turned<0x122>(v);
    v += turned<0x121>(v);
    if constexpr (G == 64) v = (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
    return v;
}
// The same over the W waves of a block; `slot` is not used again before another barrier.
template <int G, int W>
__device__ __forceinline__ float team_sum(float v, float (*slot)[W])
{
    v = lanes_sum<G>(v);
    if constexpr (W > 1) {
        if ((threadIdx.x & 63) == 0) (*slot)[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int w = 0; w < W; ++w) v += (*slot)[w];
    }
    return v;
}

// Columns of a lane: NV packs of E.  The last pack of a row that E does not divide ends with the row; the
// columns that the pack before it holds too count once in the sums (`in`) and are written twice with the
// same value.
template <int E>
struct Columns {
    int col, own;           // first column loaded, first one that counts
    __device__ __forceinline__ Columns(int pack, int dim)
    {
        own = pack * E;
        col = min(own, dim - E);
    }
    __device__ __forceinline__ bool in(int e, int dim) const { return col + e >= own && own < dim; }
};

template <int G, int W, int P> struct NormTeam {          // P: elements of a lane
    static constexpr int kThreads = W == 1 ? 256 : 64 * W;
    static constexpr int kRows = W == 1 ? 4 * (64 / G) : 1;       // rows of a block at a time
    static constexpr int kLanes = G * W;
    // the next row is loaded before the present one is worked on, where there are registers for it
    static constexpr bool kAhead = P <= 16;
};

template <typename T, bool RES, int E, int G, int W, int NV>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void norm_fwd_kernel(const NormParams p)
{
    using Team = NormTeam<G, W, E * NV>;
    __shared__ float slots[4][W];
    const int dim = p.dim;
    const int member = W == 1 ? threadIdx.x & (G - 1) : threadIdx.x;
    const int team = W > 1 ? 0 : G == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / G;
    const float scale = 1.0f / (float)dim;
    // all packs are whole and inside the row
    const bool whole = dim == Team::kLanes * E * NV;

    float w[NV][E], b[NV][E];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const Columns<E> at(c * Team::kLanes + member, dim);
#pragma unroll
        for (int e = 0; e < E; ++e) { w[c][e] = 1.0f; b[c][e] = 0.0f; }
        if (p.weight) get<float, E>(p.weight + at.col, w[c]);
        if (p.bias) get<float, E>(p.bias + at.col, b[c]);
    }
    const long step = (long)gridDim.x * Team::kRows;
    long row = (long)blockIdx.x * Team::kRows + team;
    Pack<T, E> qx[NV];
    Pack<float, E> qr[NV];
    auto fetch = [&](long r) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
            qx[c] = *reinterpret_cast<const Pack<T, E>*>(static_cast<const T*>(p.x) + r * dim + at.col);
            if constexpr (RES) qr[c] = *reinterpret_cast<const Pack<float, E>*>(p.residual + r * dim + at.col);
        }
    };
    if (Team::kAhead && row < p.rows) fetch(row);
    for (int parity = 0; row < p.rows; row += step, parity ^= 2) {
        if (!Team::kAhead) fetch(row);
        float s[NV][E];
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                s[c][e] = to_f32(qx[c].v[e]);
                if constexpr (RES) s[c][e] += qr[c].v[e];
            }
        if (Team::kAhead && row + step < p.rows) fetch(row + step);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
#pragma unroll
            for (int e = 0; e < E; ++e) sum += whole || at.in(e, dim) ? s[c][e] : 0.0f;
        }
        const float mean = team_sum<G, W>(sum, &slots[parity]) / (float)dim;     // (exact for constant rows)
        float square = 0.0f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
            // (not before the team has met: in place, the columns of a last pack that others hold too would
            // be loaded by them with the sum already in them)
            if constexpr (RES) put<float, E>(p.sum + row * dim + at.col, s[c]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                s[c][e] -= mean;
                square += whole || at.in(e, dim) ? s[c][e] * s[c][e] : 0.0f;
            }
        }
        const float rstd = 1.0f / sqrtf(team_sum<G, W>(square, &slots[parity + 1]) * scale + p.eps);
        if (p.mean && member == 0) { p.mean[row] = mean; p.rstd[row] = rstd; }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
            float o[E];
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(s[c][e] * rstd, w[c][e], b[c][e]);
            put<T, E>(static_cast<T*>(p.y) + row * dim + at.col, o);
        }
    }
}

// Teams of a block: as many as four waves hold, so that few blocks (whose shares of dweight and dbias are written
// and read once more) keep many rows in flight.
template <int G, int W> constexpr int kBwdTeams = W == 1 ? 4 * (64 / G) : W == 2 ? 2 : 1;
template <int W> constexpr int kBwdThreads = W <= 4 ? 256 : 64 * W;

// Rows whose loads are under way beside the present one.  With two tensors of 2 bytes one row does not cover the
// latency of memory, two do; teams of two and four waves lose more by the registers.  MI355X, us, calls in a loop, gradients
// of 25 million values in bf16 by columns, one / two:
//     a wave        200: 67.7 / 58.7   768: 37.2 / 35.2    1000: 33.5 / 35.5
//     two waves     1025: 53.1 / 59.1  1500: 35.9 / 42.7   2000: 35.4 / 38.4
//     four waves    2100: 51.3 / 52.4  4000: 41.6 / 42.2   4096: 42.3 / 43.1
//     eight waves   4200: 56.5 / 44.9  6000: 47.2 / 39.6   8192: 46.8 / 41.5
template <typename T, bool RES, int W, int P>
constexpr int kBwdAhead = P > 16 ? 0 : sizeof(T) == 2 && !RES && (W == 1 || W == 8) ? 2 : 1;

template <typename T, bool RES, int E, int G, int W, int NV>
__global__ __launch_bounds__(kBwdThreads<W>) void norm_bwd_kernel(const NormParams p)
{
    using Team = NormTeam<G, W, E * NV>;
    constexpr int kTeams = kBwdTeams<G, W>;
    using S = std::conditional_t<RES, float, T>;
    __shared__ float slots[2][2][kTeams * W];
    __shared__ float fold[kTeams > 1 && G == 64 ? (kTeams - 1) * 64 * W * NV * E * 2 : 1];
    const int dim = p.dim;
    const int member = threadIdx.x & (G * W - 1), wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int team = G == 64 ? wave / W : threadIdx.x / G;
    const float scale = 1.0f / (float)dim;
    const bool whole = dim == Team::kLanes * E * NV;
    const S* s_in = RES ? reinterpret_cast<const S*>(p.sum) : static_cast<const S*>(p.x);

    float w[NV][E], dw[NV][E], db[NV][E];
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const Columns<E> at(c * Team::kLanes + member, dim);
#pragma unroll
        for (int e = 0; e < E; ++e) { w[c][e] = 1.0f; dw[c][e] = 0.0f; db[c][e] = 0.0f; }
        if (p.weight) get<float, E>(p.weight + at.col, w[c]);
    }
    const long step = (long)gridDim.x * kTeams;
    long row = (long)blockIdx.x * kTeams + team;
    // teams that meet at a barrier take the same number of rows, the last of them perhaps one that is not there
    constexpr bool kTogether = W > 1 && kTeams > 1;
    const long end = kTogether ? (p.rows + kTeams - 1) / kTeams * kTeams : p.rows;
    constexpr int kAhead = kBwdAhead<T, RES, W, E * NV>, kRows = kAhead > 1 ? 2 : 1;
    struct Row {
        Pack<S, E> s[NV];
        Pack<T, E> y[NV];
        float mean, rstd;
    };
    Row held[kRows];
    Pack<float, E> qd[NV];
    auto fetch = [&](long r, Row& q) {
        if (kTogether || kAhead > 1) r = min(r, p.rows - 1);
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
            q.s[c] = *reinterpret_cast<const Pack<S, E>*>(s_in + r * dim + at.col);
            q.y[c] = *reinterpret_cast<const Pack<T, E>*>(static_cast<const T*>(p.dy) + r * dim + at.col);
            if constexpr (RES && kAhead)
                if (p.dsum) qd[c] = *reinterpret_cast<const Pack<float, E>*>(p.dsum + r * dim + at.col);
        }
        q.mean = p.mean[r];
        q.rstd = p.rstd[r];
    };
    if (kAhead && row < end) fetch(row, held[0]);
    if (kAhead > 1 && row < end) fetch(row + step, held[kRows - 1]);
    for (int parity = 0; row < end; row += step, parity ^= 1) {
        if (!kAhead) fetch(row, held[0]);
        const bool there = !kTogether || row < p.rows;
        float hat[NV][E], g[NV][E], d[NV][E];
        float sum_g = 0.0f, sum_gh = 0.0f;
        const float rs = held[0].rstd, mean = held[0].mean;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool in = (whole || at.in(e, dim)) && there;
                const float dy = to_f32(held[0].y[c].v[e]);
                hat[c][e] = (to_f32(held[0].s[c].v[e]) - mean) * rs;
                g[c][e] = dy * w[c][e];
                if (kAhead) d[c][e] = RES && p.dsum ? qd[c].v[e] : 0.0f;
                sum_g += in ? g[c][e] : 0.0f;
                sum_gh += in ? g[c][e] * hat[c][e] : 0.0f;
                dw[c][e] += in ? dy * hat[c][e] : 0.0f;
                db[c][e] += in ? dy : 0.0f;
            }
        }
        if constexpr (kAhead > 1) {
            held[0] = held[1];
            if (row + step < end) fetch(row + 2 * step, held[1]);
        } else if (kAhead && row + step < end) {
            fetch(row + step, held[0]);
        }
        sum_g = lanes_sum<G>(sum_g);
        sum_gh = lanes_sum<G>(sum_gh);
        if constexpr (W > 1) {
            if ((threadIdx.x & 63) == 0) {
                slots[parity][0][wave] = sum_g;
                slots[parity][1][wave] = sum_gh;
            }
            __syncthreads();
            sum_g = sum_gh = 0.0f;
#pragma unroll
            for (int v = 0; v < W; ++v) { sum_g += slots[parity][0][team * W + v]; sum_gh += slots[parity][1][team * W + v]; }
        }
        sum_g *= scale;
        sum_gh *= scale;
        if (!there) continue;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const Columns<E> at(c * Team::kLanes + member, dim);
            if constexpr (!kAhead) {
#pragma unroll
                for (int e = 0; e < E; ++e) d[c][e] = 0.0f;
                if constexpr (RES)
                    if (p.dsum) get<float, E>(p.dsum + row * dim + at.col, d[c]);
            }
#pragma unroll
            for (int e = 0; e < E; ++e) d[c][e] += rs * (g[c][e] - sum_g - hat[c][e] * sum_gh);
            if (!RES || p.dx) put<T, E>(static_cast<T*>(p.dx) + row * dim + at.col, d[c]);
            if constexpr (RES)
                if (p.dresidual) put<float, E>(p.dresidual + row * dim + at.col, d[c]);
        }
    }

    // the block's share of dweight and dbias: its teams' sums, added in a fixed order
    float* part_w = p.part + (long)blockIdx.x * 2 * dim;
    float* part_b = part_w + dim;
    if constexpr (kTeams > 1 && G == 64) {
        constexpr int L = 64 * W;
        if (team > 0) {
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    fold[(((team - 1) * NV + c) * 2 * E + e) * L + member] = dw[c][e];
                    fold[(((team - 1) * NV + c) * 2 * E + E + e) * L + member] = db[c][e];
                }
        }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll 1
                for (int t = 0; t < kTeams - 1; ++t) {
                    dw[c][e] += fold[((t * NV + c) * 2 * E + e) * L + member];
                    db[c][e] += fold[((t * NV + c) * 2 * E + E + e) * L + member];
                }
    } else if constexpr (G == 16) {
        __shared__ float small[16 * 16 * NV * E * 2];
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                small[((c * 2 * E + e) * 16 + team) * 16 + member] = dw[c][e];
                small[((c * 2 * E + E + e) * 16 + team) * 16 + member] = db[c][e];
            }
        __syncthreads();
        if (team > 0) return;
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e)
#pragma unroll 1
                for (int t = 1; t < 16; ++t) {
                    dw[c][e] += small[((c * 2 * E + e) * 16 + t) * 16 + member];
                    db[c][e] += small[((c * 2 * E + E + e) * 16 + t) * 16 + member];
                }
    }
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const Columns<E> at(c * Team::kLanes + member, dim);
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (whole || at.in(e, dim)) {
                part_w[at.col + e] = dw[c][e];
                part_b[at.col + e] = db[c][e];
            }
    }
}

// Rows too long for registers: a block a row, which reads it once for each of mean, deviation and result.  `first`: of the
// launch, where the rows take several.
template <typename T, bool RES>
__global__ __launch_bounds__(1024) void norm_long_fwd_kernel(const NormParams p, long first)
{
    __shared__ float slots[2][16];
    const long row = first + blockIdx.x, at = row * p.dim;
    const T* x = static_cast<const T*>(p.x) + at;
    auto value = [&](int c) { return RES ? to_f32(x[c]) + p.residual[at + c] : to_f32(x[c]); };
    float sum = 0.0f;
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float s = value(c);
        if constexpr (RES) p.sum[at + c] = s;
        sum += s;
    }
    const float mean = team_sum<64, 16>(sum, &slots[0]) / (float)p.dim;
    float square = 0.0f;
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float s = (RES ? p.sum[at + c] : value(c)) - mean;
        square += s * s;
    }
    const float rstd = 1.0f / sqrtf(team_sum<64, 16>(square, &slots[1]) / (float)p.dim + p.eps);
    if (p.mean && threadIdx.x == 0) { p.mean[row] = mean; p.rstd[row] = rstd; }
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float s = (RES ? p.sum[at + c] : value(c)) - mean;
        static_cast<T*>(p.y)[at + c] = from_f32<T>(fmaf(s * rstd, p.weight ? p.weight[c] : 1.0f, p.bias ? p.bias[c] : 0.0f));
    }
}
template <typename T, bool RES>
__global__ __launch_bounds__(1024) void norm_long_bwd_kernel(const NormParams p, long first)
{
    using S = std::conditional_t<RES, float, T>;
    __shared__ float slots[2][16];
    const long row = first + blockIdx.x, at = row * p.dim;
    const S* s = (RES ? reinterpret_cast<const S*>(p.sum) : static_cast<const S*>(p.x)) + at;
    const T* dy = static_cast<const T*>(p.dy) + at;
    const float mean = p.mean[row], rstd = p.rstd[row];
    float sum_g = 0.0f, sum_gh = 0.0f;
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float g = to_f32(dy[c]) * (p.weight ? p.weight[c] : 1.0f);
        sum_g += g;
        sum_gh += g * (to_f32(s[c]) - mean) * rstd;
    }
    sum_g = team_sum<64, 16>(sum_g, &slots[0]) / (float)p.dim;
    sum_gh = team_sum<64, 16>(sum_gh, &slots[1]) / (float)p.dim;
    for (int c = threadIdx.x; c < p.dim; c += 1024) {
        const float g = to_f32(dy[c]) * (p.weight ? p.weight[c] : 1.0f);
        float d = rstd * (g - sum_g - (to_f32(s[c]) - mean) * rstd * sum_gh);
        if (RES && p.dsum) d += p.dsum[at + c];
        if (p.dx) static_cast<T*>(p.dx)[at + c] = from_f32<T>(d);
        if (RES && p.dresidual) p.dresidual[at + c] = d;
    }
}
// Their shares of dweight and dbias: a thread a column, a block's rows.
template <typename T, bool RES>
__global__ __launch_bounds__(256) void norm_long_columns_kernel(const NormParams p)
{
    using S = std::conditional_t<RES, float, T>;
    const int c = blockIdx.x * 256 + threadIdx.x;
    if (c >= p.dim) return;
    const S* s = RES ? reinterpret_cast<const S*>(p.sum) : static_cast<const S*>(p.x);
    float dw = 0.0f, db = 0.0f;
    for (long r = blockIdx.y; r < p.rows; r += gridDim.y) {
        const float dy = to_f32(static_cast<const T*>(p.dy)[r * p.dim + c]);
        dw += dy * (to_f32(s[r * p.dim + c]) - p.mean[r]) * p.rstd[r];
        db += dy;
    }
    p.part[(long)blockIdx.y * 2 * p.dim + c] = dw;
    p.part[((long)blockIdx.y * 2 + 1) * p.dim + c] = db;
}

// Adds the shares of the blocks, in a fixed order: 64 columns a block (a lane has two, and 2 dim is even), 32
// threads to a pair of columns, so that every load is under way at once (512 shares of 2 x 768: 10.7 -> 4.0 us against
// 16 threads to a column).
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ part, float* __restrict__ dweight,
                                                           float* __restrict__ dbias, int dim, int shares)
{
    __shared__ float sums[32][65];
    const int lane = threadIdx.x & 31, group = threadIdx.x >> 5;
    const long col = (long)blockIdx.x * 64 + 2 * lane, width = 2 * (long)dim;
    float s[2] = {0.0f, 0.0f};
    if (col < width) {
#pragma unroll 16
        for (int k = group; k < shares; k += 32) {
            const Pack<float, 2> q = *reinterpret_cast<const Pack<float, 2>*>(part + k * width + col);
            s[0] += q.v[0];
            s[1] += q.v[1];
        }
    }
    sums[group][2 * lane] = s[0];
    sums[group][2 * lane + 1] = s[1];
    __syncthreads();
    // 8 threads to a column, then 8 values
    const int c = threadIdx.x & 63, eighth = (threadIdx.x >> 6) & 7;
    float t = 0.0f;
    if (threadIdx.x < 512) {
#pragma unroll
        for (int g = 0; g < 4; ++g) t += sums[4 * eighth + g][c];
    }
    __syncthreads();
    if (threadIdx.x < 512) sums[eighth][c] = t;
    __syncthreads();
    const long out = (long)blockIdx.x * 64 + c;
    if (threadIdx.x >= 64 || out >= width) return;
#pragma unroll
    for (int g = 1; g < 8; ++g) t += sums[g][c];
    if (out < dim) { if (dweight) dweight[out] = t; }
    else if (dbias) dbias[out - dim] = t;
}

// ---- launch shapes ---------------------------------------------------------------------------------
// Elements of a pack: 16 bytes of the widest tensor of the row; rows of fewer elements go one by one.
template <typename T, bool RES> constexpr int kPack = RES || sizeof(T) == 4 ? 4 : 8;

struct NormShape { int pack, lanes, waves, packs; };              // packs == 0: the long kernels
NormShape norm_shape(const NormParams& p)
{
    const int full = p.with_residual || p.dtype == 0 ? 4 : 8;
    NormShape s{p.dim < full ? 1 : full, 64, 1, 1};
    const int n = (p.dim + s.pack - 1) / s.pack;
    if (n <= 16) { s.lanes = 16; return s; }
    // at most 16 elements a lane, 24 in the widest teams
    const int most = 16 / s.pack;
    for (s.waves = 1; s.waves <= 8; s.waves *= 2) {
        s.packs = (n + 64 * s.waves - 1) / (64 * s.waves);
        if (s.packs <= most) return s;
    }
    s.waves = 8;
    if (s.packs <= most * 3 / 2) { s.packs = most * 3 / 2; return s; }
    s.packs = 0;
    return s;
}
// Teams of a block, forward.
int norm_block_rows(const NormShape& s) { return s.packs == 0 || s.waves > 1 ? 1 : 4 * (64 / s.lanes); }

template <typename T, bool RES, int E, int G, int W, int NV>
hipError_t launch_shape(const NormParams& p, bool backward, unsigned blocks, hipStream_t stream)
{
    if (backward) norm_bwd_kernel<T, RES, E, G, W, NV><<<blocks, kBwdThreads<W>, 0, stream>>>(p);
    else norm_fwd_kernel<T, RES, E, G, W, NV><<<blocks, W == 1 ? 256 : 64 * W, 0, stream>>>(p);
    return hipGetLastError();
}
template <typename T, bool RES, int W>
hipError_t launch_packs(const NormParams& p, int packs, bool backward, unsigned blocks, hipStream_t stream)
{
    constexpr int E = kPack<T, RES>, kMost = 16 / E;
    if (packs == kMost) return launch_shape<T, RES, E, 64, W, kMost>(p, backward, blocks, stream);
    // (several waves: the row was too long for half of them, so more than half of their packs are needed)
    if constexpr (kMost == 4) if (packs == 3) return launch_shape<T, RES, E, 64, W, 3>(p, backward, blocks, stream);
    if constexpr (W == 1) {
        if (packs == 1) return launch_shape<T, RES, E, 64, W, 1>(p, backward, blocks, stream);
        if constexpr (kMost == 4) if (packs == 2) return launch_shape<T, RES, E, 64, W, 2>(p, backward, blocks, stream);
    }
    if constexpr (W == 8)
        if (packs == kMost * 3 / 2) return launch_shape<T, RES, E, 64, W, kMost * 3 / 2>(p, backward, blocks, stream);
    return hipErrorInvalidValue;
}
template <typename T, bool RES>
hipError_t launch_typed(const NormParams& p, bool backward, hipStream_t stream)
{
    const NormShape s = norm_shape(p);
    if (s.packs == 0) {
        constexpr long most = most_blocks(1024);
        for (long first = 0; first < p.rows; first += most) {
            const unsigned n = (unsigned)(p.rows - first < most ? p.rows - first : most);
            if (backward) norm_long_bwd_kernel<T, RES><<<n, 1024, 0, stream>>>(p, first);
            else norm_long_fwd_kernel<T, RES><<<n, 1024, 0, stream>>>(p, first);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        if (!backward || (!p.dweight && !p.dbias)) return hipSuccess;
        norm_long_columns_kernel<T, RES><<<dim3((p.dim + 255) / 256, p.shares), 256, 0, stream>>>(p);
        return hipGetLastError();
    }
    const int per = norm_block_rows(s);
    const long whole = (p.rows + per - 1) / per;
    const unsigned blocks = backward ? p.shares : (unsigned)(whole < 2048 ? whole : 2048);
    if (s.lanes == 16)
        return s.pack == 1 ? launch_shape<T, RES, 1, 16, 1, 1>(p, backward, blocks, stream)
                           : launch_shape<T, RES, kPack<T, RES>, 16, 1, 1>(p, backward, blocks, stream);
    if (s.waves == 1) return launch_packs<T, RES, 1>(p, s.packs, backward, blocks, stream);
    if (s.waves == 2) return launch_packs<T, RES, 2>(p, s.packs, backward, blocks, stream);
    if (s.waves == 4) return launch_packs<T, RES, 4>(p, s.packs, backward, blocks, stream);
    return launch_packs<T, RES, 8>(p, s.packs, backward, blocks, stream);
}
hipError_t launch(const NormParams& p, bool backward, hipStream_t stream)
{
    if (p.dtype == 0)
        return p.with_residual ? launch_typed<float, true>(p, backward, stream) : launch_typed<float, false>(p, backward, stream);
    return p.with_residual ? launch_typed<bf16_t, true>(p, backward, stream) : launch_typed<bf16_t, false>(p, backward, stream);
}
// Blocks of the backward kernel, each with a share of dweight and dbias.  MI355X, us, calls in a loop,
// blocks 256 / 512 / 768 / 1024:
// 32768 x 768 bf16 with a residual 99.4 / 80.1 / 92.5 / 86.2, 25216 x 384 fp32 31.3 / 25.5 / 28.0 / 27.9,
// 8000 x 1025 bf16 27.7 / 22.5 / 24.6 / 25.8, 4096 x 4096 bf16 37.9 / 33.9 / 39.4 / 47.6.  Teams of eight waves: one
// a CU.
int norm_shares(const NormParams& p)
{
    const NormShape s = norm_shape(p);
    const int per = s.packs == 0 ? 1 : s.waves == 1 ? 4 * (64 / s.lanes) : s.waves == 2 ? 2 : 1;
    const long whole = (p.rows + per - 1) / per;
    const long most = s.waves == 8 || s.packs == 0 ? 256 : 512;
    return (int)(whole < most ? whole : most);
}

}  // namespace

size_t norm_bwd_floats(const NormParams& p) { return p.rows > 0 ? (size_t)norm_shares(p) * 2 * p.dim : 0; }

hipError_t launch_norm_fwd(const NormParams& p, hipStream_t stream) { return launch(p, false, stream); }

hipError_t launch_norm_bwd(NormParams p, float* workspace, hipStream_t stream)
{
    p.part = workspace;
    p.shares = norm_shares(p);
    hipError_t e = launch(p, true, stream);
    if (e != hipSuccess || (!p.dweight && !p.dbias)) return e;
    norm_reduce_kernel<<<(unsigned)((2 * (long)p.dim + 63) / 64), 1024, 0, stream>>>(workspace, p.dweight, p.dbias, p.dim, p.shares);
    return hipGetLastError();
}

}  // namespace lbscan
