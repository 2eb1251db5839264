// glr.cu -- gated linear recurrence over time: the GRU's update
// (Section 5.1.2) with gates that do not read the state,
//   z_t = sigmoid(g_z), n_t = g_n,  h_t = z_t h_{t-1} + (1 - z_t) n_t,
// forward over a sequence, its backward pass, and one token on a state cache.
#include "internal.h"
#include "lm_common.cuh"

namespace isam {

namespace {

constexpr int kSimpleThreads = 128;

// One thread per (sequence, channel), walking time.
template <typename G, typename Hy>
__global__ void __launch_bounds__(kSimpleThreads)
    glr_forward_kernel(int T, int batch, int hidden, const G *g, const float *h0, const int32_t *lengths, Hy *h_out,
                       float *h_last) {
    const int c = blockIdx.x * kSimpleThreads + threadIdx.x;
    const int b = blockIdx.y;
    if (c >= hidden) return;
    const int64_t chain = static_cast<int64_t>(b) * hidden + c;
    const int64_t step = static_cast<int64_t>(batch) * hidden;
    int len = T;
    if (lengths) len = min(max(lengths[b], 0), T);
    float h = h0 ? h0[chain] : 0.0f;
    const G *gp = g + static_cast<int64_t>(b) * 2 * hidden + c;
    Hy *hp = h_out + chain;
    for (int t = 0; t < T; ++t, gp += 2 * step, hp += step) {
        if (t < len) {
            const Gate z = gate(to_f32(gp[0]));
            h = z.keep * h + z.take * to_f32(gp[hidden]);
        }
        *hp = from_f32<Hy>(t < len ? h : 0.0f);
    }
    if (h_last) h_last[chain] = h;
}

template <typename G, typename Hy>
__global__ void __launch_bounds__(kSimpleThreads)
    glr_backward_kernel(int T, int batch, int hidden, const G *g, const float *h0, const int32_t *lengths,
                        const Hy *h_out, const Hy *dh_out, const float *dh_last, G *dg, float *dh0) {
    const int c = blockIdx.x * kSimpleThreads + threadIdx.x;
    const int b = blockIdx.y;
    if (c >= hidden) return;
    const int64_t chain = static_cast<int64_t>(b) * hidden + c;
    const int64_t step = static_cast<int64_t>(batch) * hidden;
    int len = T;
    if (lengths) len = min(max(lengths[b], 0), T);
    float e = dh_last ? dh_last[chain] : 0.0f;
    const int64_t goff = static_cast<int64_t>(b) * 2 * hidden + c;
    for (int t = T - 1; t >= 0; --t) {
        const int64_t at = goff + 2 * step * t;
        float dz = 0.0f, dn = 0.0f;
        if (t < len) {
            const Gate z = gate(to_f32(g[at]));
            const float n = to_f32(g[at + hidden]);
            const float before = t ? to_f32(h_out[chain + step * (t - 1)]) : (h0 ? h0[chain] : 0.0f);
            const float d = (dh_out ? to_f32(dh_out[chain + step * t]) : 0.0f) + e;
            dz = d * (before - n) * (z.keep * z.take);
            dn = d * z.take;
            e = z.keep * d;
        }
        dg[at] = from_f32<G>(dz);
        dg[at + hidden] = from_f32<G>(dn);
    }
    if (dh0) dh0[chain] = e;
}

template <typename G, typename Hy>
__global__ void __launch_bounds__(kSimpleThreads)
    glr_step_kernel(int hidden, int slots, const G *g, const int32_t *slot_ids, const float *state, float *new_state,
                    Hy *h) {
    const int c = blockIdx.x * kSimpleThreads + threadIdx.x;
    const int b = blockIdx.y;
    if (c >= hidden) return;
    const int slot = slot_ids ? slot_ids[b] : b;
    float v = 0.0f;
    if (slot >= 0 && slot < slots) {
        const int64_t at = static_cast<int64_t>(slot) * hidden + c;
        const int64_t go = static_cast<int64_t>(b) * 2 * hidden + c;
        const Gate z = gate(to_f32(g[go]));
        v = z.keep * state[at] + z.take * to_f32(g[go + hidden]);
        new_state[at] = v;
    }
    h[static_cast<int64_t>(b) * hidden + c] = from_f32<Hy>(v);
}

template <typename F>
int by_types(int g_type, int h_type, F &&f) {
    if (g_type == ISAM_F32) return h_type == ISAM_F32 ? f(float(), float()) : f(float(), bf16());
    return h_type == ISAM_F32 ? f(bf16(), float()) : f(bf16(), bf16());
}

}  // namespace

int glr_forward_launch(const GlrDesc &p, DeviceState &ds, cudaStream_t s) {
    return by_types(p.g_type, p.h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        const dim3 grid((p.hidden + kSimpleThreads - 1) / kSimpleThreads, p.batch);
        glr_forward_kernel<G, Hy><<<grid, kSimpleThreads, 0, s>>>(p.T, p.batch, p.hidden, static_cast<const G *>(p.g),
                                                                  p.h0, p.lengths, static_cast<Hy *>(p.h_out),
                                                                  p.h_last);
        return launch_status("launch glr_forward_kernel");
    });
}

int glr_backward_launch(const GlrDesc &p, DeviceState &ds, cudaStream_t s) {
    return by_types(p.g_type, p.h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        const dim3 grid((p.hidden + kSimpleThreads - 1) / kSimpleThreads, p.batch);
        glr_backward_kernel<G, Hy><<<grid, kSimpleThreads, 0, s>>>(
            p.T, p.batch, p.hidden, static_cast<const G *>(p.g), p.h0, p.lengths, static_cast<const Hy *>(p.h_in),
            static_cast<const Hy *>(p.dh_out), p.dh_last, static_cast<G *>(p.dg), p.dh0);
        return launch_status("launch glr_backward_kernel");
    });
}

int glr_step_launch(int batch, int hidden, int slots, int g_type, const void *g, const int32_t *slot_ids,
                    const float *state, float *new_state, int h_type, void *h, cudaStream_t s) {
    return by_types(g_type, h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        const dim3 grid((hidden + kSimpleThreads - 1) / kSimpleThreads, batch);
        glr_step_kernel<G, Hy><<<grid, kSimpleThreads, 0, s>>>(hidden, slots, static_cast<const G *>(g), slot_ids,
                                                               state, new_state, static_cast<Hy *>(h));
        return launch_status("launch glr_step_kernel");
    });
}

}  // namespace isam
