// Single tokens through the selective scan (with the convolution in front of it in the same launch), and prompts through
// the convolution with its state (formulas: lbscan_step.h).
#include "lbscan_device.h"
#include "lbscan_internal.h"
#include "lbscan_step.h"

#include <type_traits>

namespace lbscan {
namespace {

// E consecutive elements, at any element's address.
template <typename T, int E> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[E]; };

// Rows of the batch that stand along y of a grid; a block takes several of more.
constexpr int kMostRows = 65535;

// Whether an earlier row has the slot, too.  (Looked up by whole waves: a row of 1024 has 16 loads to make, all under way at
// once.)  All 64 lanes take part, with the same b.
__device__ __forceinline__ bool taken(const int32_t* __restrict__ slots, int b, int slot)
{
    bool found = false;
    for (int j = threadIdx.x & 63; j < b; j += 64) found |= slots[j] == slot;
    return __any(found);
}

__device__ __forceinline__ float silu_f32(float v) { return v * sigmoid_f32(v); }

// ---- one token -------------------------------------------------------------------------------------------
// A channel's states are four to a lane, Q lanes to a channel.  WIDE: a wave has 64 channels of one row of the batch, and a lane two
// parts: what a channel has one of (x through the convolution, dt, the gate, y) for channel `lane`, and states of Q channels,
// to which dt and dt x come from the channels' lanes and from which the sums go back.  Otherwise a wave has U times 64 / Q channels,
// whose lanes all compute what a channel has one of.  Everything is loaded before the search for an earlier row with the same slot
// ends: only what is stored waits for it.  Loads of the optional inputs stand in branches, where a sum or a conversion would wait for
// all loads before it: those come later (256 x 4096 without the convolution 34.2 -> 25.3 us).  Bound by memory, read and written in
// the same places: MI355X, three sets of inputs in turn, 256 x 4096 x 16 bf16 with the convolution, states in a pool (155.6 MB) 41.2 us
// (3.8 TB/s; two sets, part of which the last cache keeps, 36.9), without it 25.1 (5.7 TB/s).
template <typename T, int Q, int K, int U, bool WIDE>
__global__ __launch_bounds__(256) void step_kernel(const StepParams p)
{
    constexpr int kGroup = 64 / Q, S = WIDE ? 1 : U;              // channels whose states are updated at once; channels of a lane
    static_assert(!WIDE || U == Q, "a channel a lane");
    const int lane = threadIdx.x & 63, N = p.dstate, n0 = 4 * (lane % Q);
    const int first = (int)(blockIdx.x * (blockDim.x >> 6) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * (kGroup * U);
    if (first >= p.dim) return;
    const bool whole = n0 + 4 <= N;
    int d[S];
    bool channel[S], writer[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
        d[s] = first + (WIDE ? lane : s * kGroup + lane / Q);
        channel[s] = d[s] < p.dim;
        writer[s] = channel[s] && (WIDE || lane % Q == 0);
    }
    auto four = [&](const auto* from, float to[4]) {           // the lane's four of N, zeros behind them
        using V = std::remove_cv_t<std::remove_reference_t<decltype(*from)>>;
        if (whole) {
            const Pack<V, 4> v = *reinterpret_cast<const Pack<V, 4>*>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = to_f32(v.v[i]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) to[i] = n0 + i < N ? to_f32(from[i]) : 0.0f;
        }
    };
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        T* y = static_cast<T*>(p.y) + (long)b * p.dim;
        auto padding = [&] {
#pragma unroll
            for (int s = 0; s < S; ++s)
                if (writer[s]) y[d[s]] = from_f32<T>(0.0f);
        };
        const int slot = p.slots ? p.slots[b] : b;
        if ((unsigned)slot >= (unsigned)p.pool) {
            padding();
            continue;
        }
        const long row = (long)slot * p.dim;                      // of the pools
        float h[U][4], a[U][4], bm[4], cm[4];
        four(static_cast<const T*>(p.Bm) + b * p.b_stride + n0, bm);
        four(static_cast<const T*>(p.Cm) + b * p.c_stride + n0, cm);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int of = first + u * kGroup + lane / Q;
            if (of >= p.dim) continue;
            four(p.state + (row + of) * N + n0, h[u]);
            four(p.A + (long)of * N + n0, a[u]);
        }
        float x[S], dt[S], skip[S], bias[S], pre[S], in[S], total[S];
        Pack<float, (K > 0 ? K : 1)> w[S];
        Pack<T, (K > 1 ? K - 1 : 1)> old[S];
        T raw[S], delta[S], gate[S];                              // (converted later: here that would wait for the loads)
#pragma unroll
        for (int s = 0; s < S; ++s) {
            skip[s] = bias[s] = pre[s] = total[s] = 0.0f;
            raw[s] = delta[s] = gate[s] = T{};
            w[s] = {};
            old[s] = {};
            if (!channel[s]) continue;
            raw[s] = static_cast<const T*>(p.x)[b * p.x_stride + d[s]];
            delta[s] = static_cast<const T*>(p.delta)[b * p.delta_stride + d[s]];
            if (p.delta_bias) bias[s] = p.delta_bias[d[s]];
            if (p.z) gate[s] = static_cast<const T*>(p.z)[b * p.z_stride + d[s]];
            if (p.Dskip) skip[s] = p.Dskip[d[s]];
            if constexpr (K > 0) {
                if (p.conv_bias) pre[s] = p.conv_bias[d[s]];
                w[s] = *reinterpret_cast<const Pack<float, K>*>(p.conv_weight + (long)d[s] * K);
            }
            if constexpr (K > 1)
                old[s] = *reinterpret_cast<const Pack<T, K - 1>*>(static_cast<const T*>(p.conv_state) + (row + d[s]) * (K - 1));
        }
        if (p.slots && taken(p.slots, b, slot)) {
            padding();
            continue;
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            x[s] = to_f32(raw[s]);
            if constexpr (K > 0) {
                if constexpr (K > 1) {
                    Pack<T, K - 1> next;
#pragma unroll
                    for (int k = 0; k < K - 1; ++k) {
                        pre[s] = fmaf(w[s].v[k], to_f32(old[s].v[k]), pre[s]);
                        next.v[k] = k < K - 2 ? old[s].v[k < K - 2 ? k + 1 : k] : raw[s];
                    }
                    if (writer[s]) *reinterpret_cast<Pack<T, K - 1>*>(static_cast<T*>(p.conv_state) + (row + d[s]) * (K - 1)) = next;
                }
                pre[s] = fmaf(w[s].v[K - 1], x[s], pre[s]);
                x[s] = p.activation ? silu_f32(pre[s]) : pre[s];
            }
            dt[s] = to_f32(delta[s]) + bias[s];
            if (p.softplus) dt[s] = softplus_f32(dt[s]);
            in[s] = dt[s] * x[s];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int from = u * kGroup + lane / Q, of = first + from;
            const float dtu = WIDE ? __shfl(dt[0], from, 64) : dt[WIDE ? 0 : u], inu = WIDE ? __shfl(in[0], from, 64) : in[WIDE ? 0 : u];
            float sum = 0.0f;
            if (of < p.dim) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    h[u][i] = fmaf(fast_exp2(dtu * a[u][i] * kLog2e), h[u][i], inu * bm[i]);
                    // (a lane's places behind N add nothing, also where the input is not finite)
                    sum = n0 + i < N ? fmaf(cm[i], h[u][i], sum) : sum;
                }
                float* state = p.state + (row + of) * N + n0;
                if (whole) {
                    Pack<float, 4> v;
#pragma unroll
                    for (int i = 0; i < 4; ++i) v.v[i] = h[u][i];
                    *reinterpret_cast<Pack<float, 4>*>(state) = v;
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (n0 + i < N) state[i] = h[u][i];
                }
            }
#pragma unroll
            for (int m = 1; m < Q; m *= 2) sum += __shfl_xor(sum, m, 64);
            if constexpr (WIDE) {
                const float own = __shfl(sum, lane % kGroup * Q, 64);
                if (lane / kGroup == u) total[0] = own;
            } else {
                total[u] = sum;
            }
        }
#pragma unroll
        for (int s = 0; s < S; ++s) {
            if (!writer[s]) continue;
            if (p.Dskip) total[s] = fmaf(skip[s], x[s], total[s]);
            y[d[s]] = from_f32<T>(p.z ? total[s] * silu_f32(to_f32(gate[s])) : total[s]);
        }
    }
}

template <typename T, int Q, int U, bool WIDE>
hipError_t launch_step_conv(const StepParams& p, const dim3 grid, hipStream_t stream)
{
    switch (p.width) {
        case 1: step_kernel<T, Q, 1, U, WIDE><<<grid, 256, 0, stream>>>(p); break;
        case 2: step_kernel<T, Q, 2, U, WIDE><<<grid, 256, 0, stream>>>(p); break;
        case 3: step_kernel<T, Q, 3, U, WIDE><<<grid, 256, 0, stream>>>(p); break;
        case 4: step_kernel<T, Q, 4, U, WIDE><<<grid, 256, 0, stream>>>(p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
// MI355X, us, bf16, N = 16.  With the convolution, three sets of inputs in turn, in a graph, wide where that has two waves for every SIMD, wide /
// not: 256 x 4096 41.3 / 47.0, 64 x 4096 11.7 / 13.6, 64 x 1536 6.5 / 5.7, 64 x 768 5.0 / 4.3.  Without it, U = 2 where there are eight blocks for every compute unit,
// U = 2 / 1: 256 x 4096 25.7 / 27.7, 128 x 1536 8.0 / 8.5, 64 x 1536 4.9 / 5.1, 64 x 768 4.0 / 3.8.
template <typename T, int Q>
hipError_t launch_step_lanes(const StepParams& p, hipStream_t stream)
{
    auto grid = [&](int waves) { return dim3((p.dim + 256 / Q * waves - 1) / (256 / Q * waves), min(p.batch, kMostRows)); };
    if (p.width == 0) {
        if ((long)p.batch * grid(1).x >= 2048) step_kernel<T, Q, 0, 2, false><<<grid(2), 256, 0, stream>>>(p);
        else step_kernel<T, Q, 0, 1, false><<<grid(1), 256, 0, stream>>>(p);
        return hipGetLastError();
    }
    if constexpr (Q == 4)
        if ((long)p.batch * ((p.dim + 63) / 64) >= 2048) return launch_step_conv<T, Q, Q, true>(p, grid(Q), stream);
    return launch_step_conv<T, Q, 1, false>(p, grid(1), stream);
}
template <typename T>
hipError_t launch_step_typed(const StepParams& p, hipStream_t stream)
{
    return p.dstate <= 4 ? launch_step_lanes<T, 1>(p, stream)
         : p.dstate <= 8 ? launch_step_lanes<T, 2>(p, stream) : launch_step_lanes<T, 4>(p, stream);
}

// ---- prompts through the convolution ---------------------------------------------------------------------
// A thread has E tokens of one row (b, d); the one with a row's first tokens has its state, too: it alone reads the old one and
// writes the new one, whose tokens are the row's last.  The K - 1 tokens before a thread's are the last of the lane before.
// LONG: a block has tokens of one row, whose weights are scalars then.
template <int CTRL>
__device__ __forceinline__ unsigned shifted(unsigned v) { return __builtin_amdgcn_update_dpp(0u, v, CTRL, 0xF, 0xF, false); }
// The last N elements of the lane before (N at most E).
template <int N, typename T, int E>
__device__ __forceinline__ void lane_before(const Pack<T, E>& q, T out[N])
{
    constexpr int kWords = E * (int)sizeof(T) / 4;
    unsigned words[kWords];
    __builtin_memcpy(words, &q, sizeof(words));
    constexpr int kFirst = (E - N) * (int)sizeof(T) / 4;
#pragma unroll
    for (int w = kFirst; w < kWords; ++w) words[w] = shifted<0x138>(words[w]);           // wave_shr 1
    Pack<T, E> r;
    __builtin_memcpy(&r, words, sizeof(words));
#pragma unroll
    for (int k = 0; k < N; ++k) out[k] = r.v[E - N + k];
}

template <typename T, int E, int K, bool LONG>
__global__ __launch_bounds__(256) void prompt_kernel(const PromptParams p, unsigned chunks, unsigned tiles)
{
    const int L = p.seqlen;
    int d, t0;
    if constexpr (LONG) {
        d = blockIdx.x / tiles;
        t0 = ((blockIdx.x - d * tiles) * 256 + threadIdx.x) * E;
    } else {
        const unsigned at = blockIdx.x * 256 + threadIdx.x;
        d = (int)(at / chunks);
        t0 = (int)(at - d * chunks) * E;
    }
    const bool there = d < p.dim && t0 < L;
    Pack<float, K> w{};
    if (d < p.dim) w = *reinterpret_cast<const Pack<float, K>*>(p.weight + (long)d * K);
    const float bias = p.bias && d < p.dim ? p.bias[d] : 0.0f;
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        int slot = p.slots ? p.slots[b] : b;
        if ((unsigned)slot >= (unsigned)p.pool || (p.slots && taken(p.slots, b, slot))) slot = -1;
        const int n = slot < 0 ? 0 : p.lengths ? min(max(p.lengths[b], 0), L) : L;
        const T* x = static_cast<const T*>(p.x) + b * p.x_stride + (long)d * L;
        const bool whole = there && t0 <= n - E;              // all tokens are there
        Pack<T, E> own{};
        if (whole) own = *reinterpret_cast<const Pack<T, E>*>(x + t0);
        else if (there && t0 < n) {
#pragma unroll
            for (int e = 0; e < E; ++e) own.v[e] = t0 + e < n ? x[t0 + e] : T{};
        }
        T* state = K > 1 && slot >= 0 ? static_cast<T*>(p.state) + ((long)slot * p.dim + d) * (K - 1) : nullptr;
        T v[E + K - 1], old[K];
#pragma unroll
        for (int e = 0; e < E; ++e) v[K - 1 + e] = own.v[e];
        if constexpr (K > 1) {
            // (a chunk of one is a row of one token, which has them from the state)
            if constexpr (E > 1) lane_before<K - 1>(own, v);
            if (there && t0 == 0) {
#pragma unroll
                for (int k = 0; k < K - 1; ++k) v[k] = old[k] = state ? state[k] : T{};
            } else if (there && (threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < K - 1; ++k) {
                    const int t = t0 - (K - 1) + k;               // (not negative: t0 is E at the least)
                    v[k] = t < n ? x[t] : T{};
                }
            }
        }
        if (!there) continue;
        if (t0 == 0 && state && n > 0) {
#pragma unroll
            for (int k = 0; k < K - 1; ++k) {
                const int t = n - (K - 1) + k;                // the new state's token; before the row: of the old state
                T s = T{};
                if (t >= 0) s = x[t];
                else {
#pragma unroll
                    for (int j = 0; j < K - 1; ++j) s = t + K - 1 == j ? old[j] : s;
                }
                state[k] = s;
            }
        }
        T* y = static_cast<T*>(p.y) + ((long)b * p.dim + d) * L + t0;
        auto value = [&](int e) {
            float pre = bias;
#pragma unroll
            for (int k = 0; k < K; ++k) pre = fmaf(w.v[k], to_f32(v[e + k]), pre);
            return from_f32<T>(p.activation ? silu_f32(pre) : pre);
        };
        // (three ways of their own: with one that chooses, 8 x 768 x 4096 bf16 took 29.3 us instead of 26.3)
        Pack<T, E> out;
        if (whole) {
#pragma unroll
            for (int e = 0; e < E; ++e) out.v[e] = value(e);
            *reinterpret_cast<Pack<T, E>*>(y) = out;
        } else if (t0 >= n && t0 <= L - E) {
            *reinterpret_cast<Pack<T, E>*>(y) = Pack<T, E>{};
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (t0 + e < L) y[e] = t0 + e < n ? value(e) : T{};
        }
    }
}

template <typename T, int E, bool LONG>
hipError_t launch_prompt_width(const PromptParams& p, hipStream_t stream)
{
    const unsigned chunks = (p.seqlen + E - 1) / E, tiles = (chunks + 255) / 256;
    const dim3 grid(LONG ? p.dim * tiles : (unsigned)(((long)p.dim * chunks + 255) / 256), min(p.batch, kMostRows));
    switch (p.width) {
        case 1: prompt_kernel<T, E, 1, LONG><<<grid, 256, 0, stream>>>(p, chunks, tiles); break;
        case 2: prompt_kernel<T, E, 2, LONG><<<grid, 256, 0, stream>>>(p, chunks, tiles); break;
        case 3: prompt_kernel<T, E, 3, LONG><<<grid, 256, 0, stream>>>(p, chunks, tiles); break;
        case 4: prompt_kernel<T, E, 4, LONG><<<grid, 256, 0, stream>>>(p, chunks, tiles); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
// 32 bytes a thread: MI355X, us, 8 x 768 x 4096 bf16, 16 bytes / 32: 28.3 / 25.3 (half the divisions and addresses; logistic
// functions and products are 15 of it, copying the tensors would take 19), 64 x 384 x 197 9.9 / 8.9.
template <typename T>
hipError_t launch_prompt_typed(const PromptParams& p, hipStream_t stream)
{
    constexpr int E = 32 / sizeof(T);
    if (p.seqlen == 1) return launch_prompt_width<T, 1, false>(p, stream);
    // blocks of one row where three quarters of their threads have tokens (2 x 1024 x 5000 fp32 15.9 -> 15.2)
    const long chunks = (p.seqlen + E - 1) / E, places = (chunks + 255) / 256 * 256;
    return 4 * chunks >= 3 * places ? launch_prompt_width<T, E, true>(p, stream) : launch_prompt_width<T, E, false>(p, stream);
}

}  // namespace

hipError_t launch_step(const StepParams& p, hipStream_t stream)
{
    return p.dtype == 0 ? launch_step_typed<float>(p, stream) : launch_step_typed<bf16_t>(p, stream);
}

hipError_t launch_prompt(const PromptParams& p, hipStream_t stream)
{
    return p.dtype == 0 ? launch_prompt_typed<float>(p, stream) : launch_prompt_typed<bf16_t>(p, stream);
}

}  // namespace lbscan
