// ssm.cu -- selective state space scan: N states a channel that decay at rates
// their input sets.  With delta = softplus(dt + dt_bias),
//   h_t[c][n] = exp(delta A[c][n]) h_{t-1}[c][n] + delta B_t[n] u_t[c],
//   y_t[c] = (sum_n C_t[n] h_t[c][n] + D[c] u_t[c]) silu(z_t[c]),
// over a sequence, and one token on a cache of states.
#include "lm_common.cuh"

namespace isam {

namespace {

constexpr float kLog2e = 1.4426950408889634f;

// log(1 + exp(x)) to a few units in its own last place: with e = exp(-|x|) it is
// max(x, 0) + log(1 + e), and log(1 + e) = 2 atanh(e / (2 + e)), whose series in
// s = e / (2 + e) <= 1/3 ends after eight terms (s^17 / 17 < 1e-8 of the sum).
__device__ __forceinline__ float softplus(float x) {
    const float e = __expf(-fabsf(x));
    const float s = __fdividef(e, 2.0f + e);
    const float q = s * s;
    float p = 1.0f / 15.0f;
    p = fmaf(p, q, 1.0f / 13.0f);
    p = fmaf(p, q, 1.0f / 11.0f);
    p = fmaf(p, q, 1.0f / 9.0f);
    p = fmaf(p, q, 1.0f / 7.0f);
    p = fmaf(p, q, 1.0f / 5.0f);
    p = fmaf(p, q, 1.0f / 3.0f);
    p = fmaf(p, q, 1.0f);
    return fmaf(2.0f * s, p, fmaxf(x, 0.0f));
}

__device__ __forceinline__ float silu(float v) {
    const Gate s = gate(v);
    return v * s.keep;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr int kThreads = 128;

// G lanes a channel, S states a lane (n = lane's part * S + i).
template <typename U, typename P, int S, int G>
__global__ void __launch_bounds__(kThreads)
    ssm_forward_kernel(int T, int batch, int C, int N, const U *u, const P *dt, const float *dt_bias, const float *A,
                       const P *B, const P *Cm, int64_t bc_stride, const float *D, const P *z, int64_t z_stride,
                       const float *h0, const int32_t *lengths, U *y, float *h_last) {
    dependent_start();
    const int b = blockIdx.y;
    const int c0 = (blockIdx.x * kThreads + threadIdx.x) / G, part = threadIdx.x % G;
    const bool on = c0 < C;
    const int c = on ? c0 : C - 1;
    const int len = lengths ? min(max(lengths[b], 0), T) : T;
    float a[S], h[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        const int n = part * S + i;
        const int64_t at = static_cast<int64_t>(c) * N + n;
        a[i] = n < N ? A[at] * kLog2e : 0.0f;
        h[i] = n < N && h0 ? h0[static_cast<int64_t>(b) * C * N + at] : 0.0f;
    }
    const float bias = dt_bias ? dt_bias[c] : 0.0f, skip = D ? D[c] : 0.0f;
    for (int t = 0; t < len; ++t) {
        const int64_t row = static_cast<int64_t>(t) * batch + b;
        const float uv = to_f32(u[row * C + c]);
        const float delta = softplus(to_f32(dt[row * C + c]) + bias);
        const float in = delta * uv;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int n = part * S + i;
            if (n < N) {
                h[i] = fmaf(exp2_fast(delta * a[i]), h[i], in * to_f32(B[row * bc_stride + n]));
                sum = fmaf(to_f32(Cm[row * bc_stride + n]), h[i], sum);
            }
        }
#pragma unroll
        for (int d = 1; d < G; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
        sum = fmaf(skip, uv, sum);
        if (z) sum *= silu(to_f32(z[row * z_stride + c]));
        if (on && part == 0) y[row * C + c] = from_f32<U>(sum);
    }
    if (on && part == 0)
        for (int t = len; t < T; ++t) y[(static_cast<int64_t>(t) * batch + b) * C + c] = from_f32<U>(0.0f);
    if (h_last && on)
#pragma unroll
        for (int i = 0; i < S; ++i) {
            const int n = part * S + i;
            if (n < N) h_last[(static_cast<int64_t>(b) * C + c) * N + n] = h[i];
        }
}

// One token: G lanes a channel, S words of V states a lane, neighbouring lanes on neighbouring words.
template <typename U, typename P, int V, int S, int G>
__global__ void __launch_bounds__(kThreads)
    ssm_step_kernel(int64_t channels, int C, int N, int slots, const U *u, const P *dt, const float *dt_bias,
                    const float *A, const P *B, const P *Cm, int64_t bc_stride, const float *D, const P *z,
                    int64_t z_stride, const int32_t *slot_ids, const float *state, float *new_state, U *y) {
    dependent_start();
    const int64_t i0 = (static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x) / G;
    const int part = threadIdx.x % G;
    const bool on = i0 < channels;
    const int64_t i = on ? i0 : channels - 1;
    const int64_t b = i / C;
    const int c = static_cast<int>(i - b * C);
    const int slot = slot_ids ? slot_ids[b] : static_cast<int>(b);
    const bool used = slot >= 0 && slot < slots;
    float sum = 0.0f, out = 0.0f;
    if (used) {
        const float uv = to_f32(u[i]);
        const float delta = softplus(to_f32(dt[i]) + (dt_bias ? dt_bias[c] : 0.0f));
        const float in = delta * uv;
        const int64_t at = (static_cast<int64_t>(slot) * C + c) * N;
#pragma unroll
        for (int j = 0; j < S; ++j) {
            const int n = (j * G + part) * V;
            if (n < N) {
                float h[V], a[V];
                if constexpr (V == 4) {
                    const float4 hv = *reinterpret_cast<const float4 *>(state + at + n);
                    const float4 av = *reinterpret_cast<const float4 *>(A + static_cast<int64_t>(c) * N + n);
                    h[0] = hv.x, h[1] = hv.y, h[2] = hv.z, h[3] = hv.w;
                    a[0] = av.x, a[1] = av.y, a[2] = av.z, a[3] = av.w;
                } else {
                    h[0] = state[at + n];
                    a[0] = A[static_cast<int64_t>(c) * N + n];
                }
#pragma unroll
                for (int k = 0; k < V; ++k) {
                    h[k] = fmaf(exp2_fast(delta * (a[k] * kLog2e)), h[k], in * to_f32(B[b * bc_stride + n + k]));
                    sum = fmaf(to_f32(Cm[b * bc_stride + n + k]), h[k], sum);
                }
                if (on) {
                    if constexpr (V == 4)
                        *reinterpret_cast<float4 *>(new_state + at + n) = make_float4(h[0], h[1], h[2], h[3]);
                    else
                        new_state[at + n] = h[0];
                }
            }
        }
        out = fmaf(D ? D[c] : 0.0f, uv, 0.0f);
    }
#pragma unroll
    for (int d = 1; d < G; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
    if (on && part == 0) {
        out += sum;
        if (used && z) out *= silu(to_f32(z[b * z_stride + c]));
        y[i] = from_f32<U>(used ? out : 0.0f);
    }
}

template <typename F>
int by_type(int type, F &&f) {
    return type == ISAM_F32 ? f(float()) : f(bf16());
}

template <typename U, typename P, int S, int G>
int forward(const SsmDesc &p, cudaStream_t s) {
    const unsigned across = static_cast<unsigned>((static_cast<int64_t>(p.C) * G + kThreads - 1) / kThreads);
    if (p.batch > 65535) return set_error(ISAM_ERR_UNSUPPORTED, "isam_ssm_forward: batch (%d) above 65535", p.batch);
    return launch_dependent(ssm_forward_kernel<U, P, S, G>, dim3(across, p.batch), kThreads, 0, s, 1,
                            "launch ssm_forward_kernel", p.T, p.batch, p.C, p.N, static_cast<const U *>(p.u),
                            static_cast<const P *>(p.dt), p.dt_bias, p.A, static_cast<const P *>(p.B),
                            static_cast<const P *>(p.Cm), p.bc_stride, p.D, static_cast<const P *>(p.z), p.z_stride,
                            p.state, p.lengths, static_cast<U *>(p.y), p.new_state);
}

template <typename U, typename P, int V, int S, int G>
int step(const SsmDesc &p, cudaStream_t s) {
    const int64_t channels = static_cast<int64_t>(p.batch) * p.C;
    const int64_t blocks = (channels * G + kThreads - 1) / kThreads;
    if (blocks > 0x7fffffff) return set_error(ISAM_ERR_UNSUPPORTED, "isam_ssm_step: batch x C too large");
    return launch_dependent(ssm_step_kernel<U, P, V, S, G>, dim3(static_cast<unsigned>(blocks)), kThreads, 0, s, 1,
                            "launch ssm_step_kernel", channels, p.C, p.N, p.slots, static_cast<const U *>(p.u),
                            static_cast<const P *>(p.dt), p.dt_bias, p.A, static_cast<const P *>(p.B),
                            static_cast<const P *>(p.Cm), p.bc_stride, p.D, static_cast<const P *>(p.z), p.z_stride,
                            p.slot_ids, p.state, p.new_state, static_cast<U *>(p.y));
}

}  // namespace

int ssm_forward_launch(const SsmDesc &p, DeviceState &, cudaStream_t s) {
    return by_type(p.u_type, [&](auto u) {
        return by_type(p.p_type, [&](auto q) {
            using U = decltype(u);
            using P = decltype(q);
            if (p.N <= 8) return forward<U, P, 8, 1>(p, s);
            if (p.N <= 16) return forward<U, P, 16, 1>(p, s);
            if (p.N <= 32) return forward<U, P, 16, 2>(p, s);
            if (p.N <= 64) return forward<U, P, 16, 4>(p, s);
            return forward<U, P, 16, 8>(p, s);
        });
    });
}

int ssm_step_launch(const SsmDesc &p, cudaStream_t s) {
    const bool four = p.N % 4 == 0 && reinterpret_cast<uintptr_t>(p.state) % 16 == 0 &&
                      reinterpret_cast<uintptr_t>(p.new_state) % 16 == 0 && reinterpret_cast<uintptr_t>(p.A) % 16 == 0;
    return by_type(p.u_type, [&](auto u) {
        return by_type(p.p_type, [&](auto q) {
            using U = decltype(u);
            using P = decltype(q);
            if (!four) return p.N <= 16 ? step<U, P, 1, 1, 16>(p, s) : step<U, P, 1, 4, 32>(p, s);
            if (p.N <= 8) return step<U, P, 4, 1, 2>(p, s);
            if (p.N <= 16) return step<U, P, 4, 1, 4>(p, s);
            if (p.N <= 32) return step<U, P, 4, 1, 8>(p, s);
            return step<U, P, 4, 2, 16>(p, s);
        });
    });
}

}  // namespace isam
