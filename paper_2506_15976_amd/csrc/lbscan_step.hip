// Single tokens through the selective scan (with the convolution in front of it in the same launch), and prompts through
// the convolution with its state (formulas: lbscan_step.h).
#include "lbscan_device.h"
#include "lbscan_internal.h"
#include "lbscan_step.h"

namespace lbscan {
namespace {

// E consecutive elements, at any element's address.
template <typename T, int E> struct __attribute__((packed, aligned(sizeof(T)))) Pack { T v[E]; };

// Rows of the batch that stand along y of a grid; a block takes several of more.
constexpr int kMostRows = 65535;

// The row's place in the pools, -1 for padding.  All 64 lanes take part, with the same b.
__device__ __forceinline__ int slot_of(const int32_t* __restrict__ slots, int b, int pool)
{
    if (!slots) return b;
    const int mine = slots[b];
    // (looked up by whole waves: a row of 1024 has 16 loads to make, all under way at once)
    bool taken = false;
    for (int j = threadIdx.x & 63; j < b; j += 64) taken |= slots[j] == mine;
    return (unsigned)mine < (unsigned)pool && !__any(taken) ? mine : -1;
}

__device__ __forceinline__ float silu_f32(float v) { return v * sigmoid_f32(v); }

// ---- one token -------------------------------------------------------------------------------------------
// A channel's states are four to a lane, Q lanes to a channel, 256 / Q channels to a block, which has one row of the batch.
template <typename T, int Q>
__global__ __launch_bounds__(256) void step_kernel(const StepParams p)
{
    const int q = threadIdx.x & (Q - 1);
    const int d = blockIdx.x * (256 / Q) + threadIdx.x / Q;
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        const int slot = slot_of(p.slots, b, p.pool);
        if (d >= p.dim) continue;
        T* y = static_cast<T*>(p.y) + (long)b * p.dim + d;
        if (slot < 0) {
            if (q == 0) *y = from_f32<T>(0.0f);
            continue;
        }
        const int N = p.dstate, n0 = 4 * q;
        float* state = p.state + ((long)slot * p.dim + d) * N + n0;
        const float* A = p.A + (long)d * N + n0;
        const T* Bm = static_cast<const T*>(p.Bm) + b * p.b_stride + n0;
        const T* Cm = static_cast<const T*>(p.Cm) + b * p.c_stride + n0;
        float h[4], a[4], bm[4], cm[4];
        if (n0 + 4 <= N) {
            const auto vh = *reinterpret_cast<const Pack<float, 4>*>(state);
            const auto va = *reinterpret_cast<const Pack<float, 4>*>(A);
            const auto vb = *reinterpret_cast<const Pack<T, 4>*>(Bm);
            const auto vc = *reinterpret_cast<const Pack<T, 4>*>(Cm);
#pragma unroll
            for (int i = 0; i < 4; ++i) { h[i] = vh.v[i]; a[i] = va.v[i]; bm[i] = to_f32(vb.v[i]); cm[i] = to_f32(vc.v[i]); }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const bool in = n0 + i < N;
                h[i] = in ? state[i] : 0.0f;
                a[i] = in ? A[i] : 0.0f;
                bm[i] = in ? to_f32(Bm[i]) : 0.0f;
                cm[i] = in ? to_f32(Cm[i]) : 0.0f;
            }
        }
        const T raw = static_cast<const T*>(p.x)[b * p.x_stride + d];
        float x = to_f32(raw);
        const float delta = to_f32(static_cast<const T*>(p.delta)[b * p.delta_stride + d]);
        const float z = p.z ? to_f32(static_cast<const T*>(p.z)[b * p.z_stride + d]) : 0.0f;
        if (p.width) {
            const int K = p.width;
            T* before = static_cast<T*>(p.conv_state) + ((long)slot * p.dim + d) * (K - 1);
            const float* w = p.conv_weight + (long)d * K;
            float pre = p.conv_bias ? p.conv_bias[d] : 0.0f;
            T old[3];
#pragma unroll
            for (int k = 0; k < 3; ++k)
                if (k < K - 1) { old[k] = before[k]; pre = fmaf(w[k], to_f32(old[k]), pre); }
            pre = fmaf(w[K - 1], x, pre);
            x = p.activation ? silu_f32(pre) : pre;
            if (q == 0) {
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (k < K - 2) before[k] = old[k + 1];
                if (K > 1) before[K - 2] = raw;
            }
        }
        float dt = delta + (p.delta_bias ? p.delta_bias[d] : 0.0f);
        if (p.softplus) dt = softplus_f32(dt);
        const float u = dt * x;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            h[i] = fmaf(fast_exp2(dt * a[i] * kLog2e), h[i], u * bm[i]);
            // (a lane's places behind N stand still at zero, also where u is not finite)
            sum = n0 + i < N ? fmaf(cm[i], h[i], sum) : sum;
        }
#pragma unroll
        for (int m = 1; m < Q; m *= 2) sum += __shfl_xor(sum, m, 64);
        if (n0 + 4 <= N) {
            Pack<float, 4> v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v.v[i] = h[i];
            *reinterpret_cast<Pack<float, 4>*>(state) = v;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n0 + i < N) state[i] = h[i];
        }
        if (q == 0) {
            if (p.Dskip) sum = fmaf(p.Dskip[d], x, sum);
            *y = from_f32<T>(p.z ? sum * silu_f32(z) : sum);
        }
    }
}

template <typename T, int Q>
hipError_t launch_step_lanes(const StepParams& p, hipStream_t stream)
{
    step_kernel<T, Q><<<dim3((p.dim + 256 / Q - 1) / (256 / Q), min(p.batch, kMostRows)), 256, 0, stream>>>(p);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_step_typed(const StepParams& p, hipStream_t stream)
{
    return p.dstate <= 4 ? launch_step_lanes<T, 1>(p, stream)
         : p.dstate <= 8 ? launch_step_lanes<T, 2>(p, stream) : launch_step_lanes<T, 4>(p, stream);
}

// ---- prompts through the convolution ---------------------------------------------------------------------
// A thread has E tokens of one row (b, d); the one with a row's first tokens has its state, too: it alone reads the old
// one and writes the new one, whose tokens are the row's last.
template <typename T, int E, int K>
__global__ __launch_bounds__(256) void prompt_kernel(const PromptParams p, unsigned chunks)
{
    const unsigned at = blockIdx.x * 256 + threadIdx.x;
    const int d = (int)(at / chunks), t0 = (int)(at - d * chunks) * E, L = p.seqlen;
    for (int b = blockIdx.y; b < p.batch; b += gridDim.y) {
        const int slot = slot_of(p.slots, b, p.pool);
        if (d >= p.dim) continue;
        int n = p.lengths ? min(max(p.lengths[b], 0), L) : L;
        if (slot < 0) n = 0;
        const T* x = static_cast<const T*>(p.x) + b * p.x_stride + (long)d * L;
        T* y = static_cast<T*>(p.y) + ((long)b * p.dim + d) * L + t0;
        const int here = min(E, L - t0);                      // tokens of this thread
        T* state = K > 1 && slot >= 0 ? static_cast<T*>(p.state) + ((long)slot * p.dim + d) * (K - 1) : nullptr;
        T old[K];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) old[k] = t0 == 0 && state ? state[k] : T{};
        T v[E + K - 1];
#pragma unroll
        for (int k = 0; k < K - 1; ++k) {
            // (a row of one token has the rest of the window in its state)
            const int t = t0 - (K - 1) + k;
            v[k] = t < 0 ? old[k] : t < n ? x[t] : T{};
        }
        if (t0 + E <= n) {
            const auto q = *reinterpret_cast<const Pack<T, E>*>(x + t0);
#pragma unroll
            for (int e = 0; e < E; ++e) v[K - 1 + e] = q.v[e];
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[K - 1 + e] = t0 + e < n ? x[t0 + e] : T{};
        }
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
        float w[K];
#pragma unroll
        for (int k = 0; k < K; ++k) w[k] = p.weight[(long)d * K + k];
        const float bias = p.bias ? p.bias[d] : 0.0f;
        Pack<T, E> out;
#pragma unroll
        for (int e = 0; e < E; ++e) {
            float pre = bias;
#pragma unroll
            for (int k = 0; k < K; ++k) pre = fmaf(w[k], to_f32(v[e + k]), pre);
            if (p.activation) pre = silu_f32(pre);
            out.v[e] = from_f32<T>(t0 + e < n ? pre : 0.0f);
        }
        if (here == E) *reinterpret_cast<Pack<T, E>*>(y) = out;
        else {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (e < here) y[e] = out.v[e];
        }
    }
}

template <typename T, int E>
hipError_t launch_prompt_width(const PromptParams& p, hipStream_t stream)
{
    const unsigned chunks = (p.seqlen + E - 1) / E;
    const dim3 grid((unsigned)(((long)p.dim * chunks + 255) / 256), min(p.batch, kMostRows));
    switch (p.width) {
        case 1: prompt_kernel<T, E, 1><<<grid, 256, 0, stream>>>(p, chunks); break;
        case 2: prompt_kernel<T, E, 2><<<grid, 256, 0, stream>>>(p, chunks); break;
        case 3: prompt_kernel<T, E, 3><<<grid, 256, 0, stream>>>(p, chunks); break;
        case 4: prompt_kernel<T, E, 4><<<grid, 256, 0, stream>>>(p, chunks); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
// 16 bytes a thread; a single token is a thread of its own.
template <typename T>
hipError_t launch_prompt_typed(const PromptParams& p, hipStream_t stream)
{
    return p.seqlen == 1 ? launch_prompt_width<T, 1>(p, stream) : launch_prompt_width<T, 16 / sizeof(T)>(p, stream);
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
