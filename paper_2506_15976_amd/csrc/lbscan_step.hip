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
// A channel's states are four to a lane, Q lanes to a channel; a block has one row of the batch and 256 / Q channels, U times, so
// that it reads and writes whole kilobytes of the pool.  Everything is loaded before the search for an earlier row with the same
// slot ends: only what is stored waits for it.  Bound by memory, read and written in the same places: MI355X, us, 256 rows of
// 4096 x 16 in bf16 with the convolution, states in a pool (155.6 MB), U = 1 / 2 / 3: 43.9 / 43.4 / 45.2 (3.6 TB/s);
// with two rows of the batch to a block, whose constants stay in registers, 48.9.  64 rows of 768: 4.1, of which the call is 3.8.
template <typename T, int Q, int U, int K>
__global__ __launch_bounds__(256) void step_kernel(const StepParams p)
{
    constexpr int kChannels = 256 / Q;
    const int q = threadIdx.x & (Q - 1), N = p.dstate, n0 = 4 * q;
    const bool whole = n0 + 4 <= N;
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
        const int slot = p.slots ? p.slots[b] : b;
        const bool inside = (unsigned)slot < (unsigned)p.pool;
        float h[U][4], a[U][4], bm[4], cm[4], delta[U], z[U], pre[U];
        Pack<float, (K > 0 ? K : 1)> w[U];
        Pack<T, (K > 1 ? K - 1 : 1)> old[U];
        T raw[U];
        int d[U];
        bool there[U];
        four(static_cast<const T*>(p.Bm) + b * p.b_stride + n0, bm);
        four(static_cast<const T*>(p.Cm) + b * p.c_stride + n0, cm);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            d[u] = (blockIdx.x * U + u) * kChannels + threadIdx.x / Q;
            there[u] = inside && d[u] < p.dim;
            if (!there[u]) continue;
            const long at = (long)slot * p.dim + d[u];
            four(p.state + at * N + n0, h[u]);
            four(p.A + (long)d[u] * N + n0, a[u]);
            raw[u] = static_cast<const T*>(p.x)[b * p.x_stride + d[u]];
            delta[u] = to_f32(static_cast<const T*>(p.delta)[b * p.delta_stride + d[u]]);
            z[u] = p.z ? to_f32(static_cast<const T*>(p.z)[b * p.z_stride + d[u]]) : 0.0f;
            if constexpr (K > 0) {
                pre[u] = p.conv_bias ? p.conv_bias[d[u]] : 0.0f;
                w[u] = *reinterpret_cast<const Pack<float, K>*>(p.conv_weight + (long)d[u] * K);
            }
            if constexpr (K > 1) old[u] = *reinterpret_cast<const Pack<T, K - 1>*>(static_cast<const T*>(p.conv_state) + at * (K - 1));
        }
        const bool mine = !p.slots || !taken(p.slots, b, slot);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (d[u] >= p.dim) continue;
            T* y = static_cast<T*>(p.y) + (long)b * p.dim + d[u];
            if (!there[u] || !mine) {
                if (q == 0) *y = from_f32<T>(0.0f);
                continue;
            }
            const long at = (long)slot * p.dim + d[u];
            float x = to_f32(raw[u]);
            if constexpr (K > 0) {
                if constexpr (K > 1) {
#pragma unroll
                    for (int k = 0; k < K - 1; ++k) pre[u] = fmaf(w[u].v[k], to_f32(old[u].v[k]), pre[u]);
                    if (q == 0) {
                        Pack<T, K - 1> next;
#pragma unroll
                        for (int k = 0; k < K - 1; ++k) next.v[k] = k < K - 2 ? old[u].v[k < K - 2 ? k + 1 : k] : raw[u];
                        *reinterpret_cast<Pack<T, K - 1>*>(static_cast<T*>(p.conv_state) + at * (K - 1)) = next;
                    }
                }
                pre[u] = fmaf(w[u].v[K - 1], x, pre[u]);
                x = p.activation ? silu_f32(pre[u]) : pre[u];
            }
            float dt = delta[u] + (p.delta_bias ? p.delta_bias[d[u]] : 0.0f);
            if (p.softplus) dt = softplus_f32(dt);
            const float in = dt * x;
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[u][i] = fmaf(fast_exp2(dt * a[u][i] * kLog2e), h[u][i], in * bm[i]);
                // (a lane's places behind N add nothing, also where the input is not finite)
                sum = n0 + i < N ? fmaf(cm[i], h[u][i], sum) : sum;
            }
            float* state = p.state + at * N + n0;
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
#pragma unroll
            for (int m = 1; m < Q; m *= 2) sum += __shfl_xor(sum, m, 64);
            if (q == 0) {
                if (p.Dskip) sum = fmaf(p.Dskip[d[u]], x, sum);
                *y = from_f32<T>(p.z ? sum * silu_f32(z[u]) : sum);
            }
        }
    }
}

template <typename T, int Q, int U>
hipError_t launch_step_tiles(const StepParams& p, hipStream_t stream)
{
    constexpr int kChannels = 256 / Q * U;
    const dim3 grid((p.dim + kChannels - 1) / kChannels, min(p.batch, kMostRows));
    switch (p.width) {
        case 0: step_kernel<T, Q, U, 0><<<grid, 256, 0, stream>>>(p); break;
        case 1: step_kernel<T, Q, U, 1><<<grid, 256, 0, stream>>>(p); break;
        case 2: step_kernel<T, Q, U, 2><<<grid, 256, 0, stream>>>(p); break;
        case 3: step_kernel<T, Q, U, 3><<<grid, 256, 0, stream>>>(p); break;
        case 4: step_kernel<T, Q, U, 4><<<grid, 256, 0, stream>>>(p); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
// Blocks of twice the channels where there are several for each place on the machine.
template <typename T, int Q>
hipError_t launch_step_lanes(const StepParams& p, hipStream_t stream)
{
    const long blocks = (long)p.batch * ((p.dim + 256 / Q - 1) / (256 / Q));
    return blocks >= 4096 ? launch_step_tiles<T, Q, 2>(p, stream) : launch_step_tiles<T, Q, 1>(p, stream);
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
