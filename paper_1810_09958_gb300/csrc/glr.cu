// glr.cu -- gated linear recurrence over time: the GRU's update
// (Section 5.1.2) with gates that do not read the state,
//   z_t = sigmoid(g_z), n_t = g_n,  h_t = z_t h_{t-1} + (1 - z_t) n_t,
// forward over a sequence, its backward pass, and one token on a state cache.
//
// A step is the affine map h -> z h + b, b = (1 - z) n, and a run of steps is
// one affine map (A, B): A the product of the z, B the state the run ends in
// from zero.  So time is split: a warp owns L consecutive steps of 32 V
// neighbouring channels (lane = V channels; a row of a warp is 128 bytes of
// gates), folds them to (A, B) while keeping z and b of each step in
// registers, learns the state before its first step from the folds of the
// warps before it, and runs its steps again from registers.  Every gate is
// read once and every state written once; that is the bound (HBM).
//
// The warps of a CTA follow each other in time, the CTAs of a cluster too, and
// a cluster walks its channels' time axis in rounds of (CTAs x warps x L)
// steps, the next round's gates in flight while a round is folded.  Folds pass
// between warps through shared memory, between CTAs through distributed shared
// memory (one cluster barrier per round, buffers alternate); every warp
// carries the state at the end of the round itself, from the same folds in
// the same order, so nothing depends on timing.  The cluster size (1 to 8) is
// picked so that one long sequence fills the GPU as a batch does.
//
// The backward pass is the same scan from the last step to the first with
// e_t = z_t (dh_t + e_{t+1}), d_t = dh_t + e_{t+1}.
#include <algorithm>

#include "internal.h"
#include "lm_common.cuh"
#include "ptx.cuh"

namespace isam {

namespace {

constexpr int kMaxWarps = 8;
constexpr int kMaxCluster = 8;
constexpr int kCtasPerSm = 2;  // launch bounds: at most 128 registers a thread
constexpr int kStepThreads = 128;

// V neighbouring elements, moved as one word; data used once, so loads and
// stores are marked streaming.
template <int BYTES>
struct Word;
template <>
struct Word<2> {
    using T = unsigned short;
};
template <>
struct Word<4> {
    using T = unsigned int;
};
template <>
struct Word<8> {
    using T = uint2;
};
template <>
struct Word<16> {
    using T = uint4;
};

template <typename T, int V>
union Pack {
    using W = typename Word<sizeof(T) * V>::T;
    W w;
    T v[V];
    __device__ Pack() {}
};

template <typename T, int V>
__device__ __forceinline__ void load(Pack<T, V> &p, const T *at) {
    p.w = __ldcs(reinterpret_cast<const typename Pack<T, V>::W *>(at));
}

template <typename T, int V>
__device__ __forceinline__ void store(T *at, const float (&x)[V]) {
    Pack<T, V> p;
#pragma unroll
    for (int i = 0; i < V; ++i) p.v[i] = from_f32<T>(x[i]);
    __stcs(reinterpret_cast<typename Pack<T, V>::W *>(at), p.w);
}

// sigmoid(x) and 1 - sigmoid(x) without a branch on the sign: with
// e = exp(-x) they are 1 / (1 + e) and e / (1 + e), each accurate to its own
// size; e stops at 2^126 so that e / (1 + e) stays 1 (a NaN passes).
__device__ __forceinline__ Gate scan_gate(float x) {
    float t = x * -1.4426950408889634f, e;
    asm("min.NaN.f32 %0, %0, 0f42FC0000;" : "+f"(t));
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(t));
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
    return Gate{r, e * r};
}

// One affine map per channel of a lane.  A product of many gates may underflow;
// it is kept at 2^-126 (no gate is zero), so that an infinite state stays
// infinite as it does step by step, instead of 0 * inf.  A finite state h is
// changed by at most 2^-126 h.
template <int V>
struct Fold {
    float a[V], b[V];
};
__device__ __forceinline__ float positive(float a) { return fmaxf(a, 1.17549435e-38f); }

// Folds of one round: of the CTA's warps, and of the cluster's CTAs.
template <int V>
struct FoldBuffers {
    Fold<V> warp[2][kMaxWarps][32];
    Fold<V> cta[2][kMaxCluster][32];
};

// What a warp needs from the others' folds: `in` becomes the state before its
// first step of this round, `carry` the state after the round.
template <int V>
__device__ __forceinline__ void exchange(FoldBuffers<V> &s, int parity, Fold<V> &own, int warp, int warps, int lane,
                                         uint32_t rank, uint32_t cluster, float (&carry)[V], float (&in)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) own.a[i] = positive(own.a[i]);
    s.warp[parity][warp][lane] = own;
    __syncthreads();
    if (cluster == 1) {
        for (int w = 0; w < warps; ++w) {
            const Fold<V> f = s.warp[parity][w][lane];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                if (w == warp) in[i] = carry[i];
                carry[i] = f.a[i] * carry[i] + f.b[i];
            }
        }
        return;
    }
    Fold<V> before;
#pragma unroll
    for (int i = 0; i < V; ++i) before.a[i] = 1.0f, before.b[i] = 0.0f;
    for (int w = 0; w < warp; ++w) {
        const Fold<V> f = s.warp[parity][w][lane];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            before.b[i] = f.a[i] * before.b[i] + f.b[i];
            before.a[i] = positive(before.a[i] * f.a[i]);
        }
    }
    if (warp == warps - 1) {
        Fold<V> all;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            all.a[i] = positive(own.a[i] * before.a[i]);
            all.b[i] = own.a[i] * before.b[i] + own.b[i];
        }
        const uint32_t at = smem_u32(&s.cta[parity][rank][lane]);
        for (uint32_t q = 0; q < cluster; ++q) {
            const uint32_t to = mapa_shared(at, q);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4 * i), "f"(all.a[i]) : "memory");
                asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(to + 4 * (V + i)), "f"(all.b[i]) : "memory");
            }
        }
    }
    __syncwarp();
    cluster_sync_all();
    for (uint32_t q = 0; q < cluster; ++q) {
        const Fold<V> f = s.cta[parity][q][lane];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            if (q == rank) in[i] = before.a[i] * carry[i] + before.b[i];
            carry[i] = f.a[i] * carry[i] + f.b[i];
        }
    }
}

struct ScanParams {
    GlrDesc d;
    int tiles;  // channel tiles of 32 V per sequence
    uint32_t cluster;
    uint32_t *err;
};

// Where this thread works.
template <int V>
struct Place {
    int lane, warp, warps, b, c;
    uint32_t rank;
    bool on;        // the lane's channels exist (idle lanes read the last ones)
    int len;        // steps of this sequence
    int64_t chain;  // b * hidden + c
    __device__ Place(const ScanParams &p) {
        lane = threadIdx.x & 31;
        warp = threadIdx.x >> 5;
        warps = blockDim.x >> 5;
        rank = blockIdx.x % p.cluster;
        const uint32_t group = blockIdx.x / p.cluster;
        b = group / p.tiles;
        c = (static_cast<int>(group) - b * p.tiles) * 32 * V + lane * V;
        on = c < p.d.hidden;
        c = min(c, p.d.hidden - V);
        len = p.d.T;
        if (p.d.lengths) len = min(max(p.d.lengths[b], 0), p.d.T);
        chain = static_cast<int64_t>(b) * p.d.hidden + c;
    }
};

template <typename G, typename Hy, int V, int L>
__global__ void __launch_bounds__(32 * kMaxWarps, kCtasPerSm) glr_forward_kernel(const ScanParams p) {
    if (p.cluster > 1 && !launch_shape_ok(p.err, p.cluster, gridDim.x, 0x601u)) return;
    __shared__ FoldBuffers<V> folds;
    const Place<V> at(p);
    const int hidden = p.d.hidden;
    const int64_t step = static_cast<int64_t>(p.d.batch) * hidden;
    const int span = at.warps * L, round = span * p.cluster;
    const int rounds = (at.len + round - 1) / round;
    const int first = at.rank * span + at.warp * L;
    const G *g = static_cast<const G *>(p.d.g) + at.chain + static_cast<int64_t>(at.b) * hidden;  // rows of 2 hidden
    Hy *out = static_cast<Hy *>(p.d.h_out) + at.chain;

    float carry[V];
#pragma unroll
    for (int i = 0; i < V; ++i) carry[i] = p.d.h0 ? p.d.h0[at.chain + i] : 0.0f;

    Pack<G, V> gz[L], gn[L];
    const auto fetch = [&](int t) {
        const int n = min(at.len - t, L);
        const G *q = g + 2 * step * t;
        if (n == L) {
#pragma unroll
            for (int i = 0; i < L; ++i, q += 2 * step) {
                load<G, V>(gz[i], q);
                load<G, V>(gn[i], q + hidden);
            }
        } else {
#pragma unroll
            for (int i = 0; i < L; ++i, q += 2 * step)
                if (i < n) {
                    load<G, V>(gz[i], q);
                    load<G, V>(gn[i], q + hidden);
                }
        }
    };
    if (rounds > 0) fetch(first);
    for (int r = 0; r < rounds; ++r) {
        const int t = r * round + first;
        const int n = min(at.len - t, L);  // steps of this warp, below 1 past the end
        float z[L][V], b[L][V];
        Fold<V> own;
#pragma unroll
        for (int i = 0; i < V; ++i) own.a[i] = 1.0f, own.b[i] = 0.0f;
        if (n == L) {
#pragma unroll
            for (int k = 0; k < L; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const Gate s = scan_gate(to_f32(gz[k].v[i]));
                    z[k][i] = s.keep;
                    b[k][i] = s.take * to_f32(gn[k].v[i]);
                }
        } else {
#pragma unroll
            for (int k = 0; k < L; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    z[k][i] = 1.0f, b[k][i] = 0.0f;
                    if (k < n) {
                        const Gate s = scan_gate(to_f32(gz[k].v[i]));
                        z[k][i] = s.keep;
                        b[k][i] = s.take * to_f32(gn[k].v[i]);
                    }
                }
        }
#pragma unroll
        for (int k = 0; k < L; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                own.a[i] *= z[k][i];
                own.b[i] = z[k][i] * own.b[i] + b[k][i];
            }
        if (r + 1 < rounds) fetch(t + round);
        float h[V];
        exchange<V>(folds, r & 1, own, at.warp, at.warps, at.lane, at.rank, p.cluster, carry, h);
        if (at.on) {
            Hy *q = out + step * t;
            const int left = p.d.T - t;
#pragma unroll
            for (int k = 0; k < L; ++k, q += step) {
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    h[i] = z[k][i] * h[i] + b[k][i];
                    v[i] = k < n ? h[i] : 0.0f;
                }
                if (k < left) store<Hy, V>(q, v);
            }
        }
    }
    if (at.on) {
        const float zero[V] = {};
        for (int t = rounds * round + at.rank * at.warps + at.warp; t < p.d.T; t += at.warps * p.cluster)
            store<Hy, V>(out + step * t, zero);
        if (p.d.h_last && at.rank == 0 && at.warp == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) p.d.h_last[at.chain + i] = carry[i];
        }
    }
    if (p.cluster > 1) cluster_sync_all();  // no CTA leaves while another may still write its folds
}

template <typename G, typename Hy, int V, int L>
__global__ void __launch_bounds__(32 * kMaxWarps, kCtasPerSm) glr_backward_kernel(const ScanParams p) {
    if (p.cluster > 1 && !launch_shape_ok(p.err, p.cluster, gridDim.x, 0x602u)) return;
    __shared__ FoldBuffers<V> folds;
    const Place<V> at(p);
    const int hidden = p.d.hidden;
    const int64_t step = static_cast<int64_t>(p.d.batch) * hidden;
    const int span = at.warps * L, round = span * p.cluster;
    const int rounds = (at.len + round - 1) / round;
    const int first = at.rank * span + at.warp * L;  // counted back from the last step
    const int64_t goff = at.chain + static_cast<int64_t>(at.b) * hidden;
    const G *g = static_cast<const G *>(p.d.g) + goff;
    G *dg = static_cast<G *>(p.d.dg) + goff;
    const Hy *hs = static_cast<const Hy *>(p.d.h_in) + at.chain;
    const Hy *dh = static_cast<const Hy *>(p.d.dh_out) + at.chain;
    const bool has_dh = p.d.dh_out != nullptr;

    float carry[V], h0[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        carry[i] = p.d.dh_last ? p.d.dh_last[at.chain + i] : 0.0f;
        h0[i] = p.d.h0 ? p.d.h0[at.chain + i] : 0.0f;
    }

    Pack<G, V> gz[L], gn[L];
    Pack<Hy, V> hb[L], gh[L];
    const auto fetch = [&](int t) {  // steps t, t - 1, ... (the first n exist)
        const int n = min(t + 1, L);
        const G *q = g + 2 * step * t;
        const Hy *qh = hs + step * (t - 1);
        const Hy *qd = dh + step * t;
        if (t >= L && has_dh) {
#pragma unroll
            for (int k = 0; k < L; ++k, q -= 2 * step, qh -= step, qd -= step) {
                load<G, V>(gz[k], q);
                load<G, V>(gn[k], q + hidden);
                load<Hy, V>(hb[k], qh);
                load<Hy, V>(gh[k], qd);
            }
        } else {
#pragma unroll
            for (int k = 0; k < L; ++k, q -= 2 * step, qh -= step, qd -= step)
                if (k < n) {
                    load<G, V>(gz[k], q);
                    load<G, V>(gn[k], q + hidden);
                    if (k < t) load<Hy, V>(hb[k], qh);
                    if (has_dh) load<Hy, V>(gh[k], qd);
                }
        }
    };
    if (rounds > 0) fetch(at.len - 1 - first);
    for (int r = 0; r < rounds; ++r) {
        const int t = at.len - 1 - (r * round + first);
        const int n = min(t + 1, L);
        // z, 1 - z, (h_{t-1} - n) z (1 - z) and dh of each step.
        float z[L][V], take[L][V], q[L][V], d[L][V];
        Fold<V> own;
#pragma unroll
        for (int i = 0; i < V; ++i) own.a[i] = 1.0f, own.b[i] = 0.0f;
#pragma unroll
        for (int k = 0; k < L; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const bool live = k < n;
                const Gate s = scan_gate(to_f32(gz[k].v[i]));
                const float before = k == t ? h0[i] : to_f32(hb[k].v[i]);
                z[k][i] = live ? s.keep : 1.0f;
                take[k][i] = s.take;
                q[k][i] = (before - to_f32(gn[k].v[i])) * (s.keep * s.take);
                d[k][i] = live && has_dh ? to_f32(gh[k].v[i]) : 0.0f;
                own.a[i] *= z[k][i];
                own.b[i] = z[k][i] * (own.b[i] + d[k][i]);
            }
        if (r + 1 < rounds) fetch(t - round);
        float e[V];
        exchange<V>(folds, r & 1, own, at.warp, at.warps, at.lane, at.rank, p.cluster, carry, e);
        if (at.on) {
            G *o = dg + 2 * step * t;
#pragma unroll
            for (int k = 0; k < L; ++k, o -= 2 * step) {
                float dz[V], dn[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float whole = d[k][i] + e[i];
                    dz[i] = whole * q[k][i];
                    dn[i] = whole * take[k][i];
                    e[i] = z[k][i] * whole;
                }
                if (k < n) {
                    store<G, V>(o, dz);
                    store<G, V>(o + hidden, dn);
                }
            }
        }
    }
    if (at.on) {
        const float zero[V] = {};
        for (int t = at.len + at.rank * at.warps + at.warp; t < p.d.T; t += at.warps * p.cluster) {
            store<G, V>(dg + 2 * step * t, zero);
            store<G, V>(dg + 2 * step * t + hidden, zero);
        }
        if (p.d.dh0 && at.rank == 0 && at.warp == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i) p.d.dh0[at.chain + i] = carry[i];
        }
    }
    if (p.cluster > 1) cluster_sync_all();
}

// One token a sequence: one thread per V channels.
template <typename G, typename Hy, int V>
__global__ void __launch_bounds__(kStepThreads)
    glr_step_kernel(int64_t threads, int hidden, int slots, const G *g, const int32_t *slot_ids, const float *state,
                    float *new_state, Hy *h) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x;
    if (i >= threads) return;
    const int per = hidden / V;
    const int64_t b = i / per;
    const int c = static_cast<int>(i - b * per) * V;
    const int slot = slot_ids ? slot_ids[b] : static_cast<int>(b);
    float v[V] = {};
    if (slot >= 0 && slot < slots) {
        const int64_t at = static_cast<int64_t>(slot) * hidden + c;
        Pack<G, V> gz, gn;
        Pack<float, V> s;
        load<G, V>(gz, g + b * 2 * hidden + c);
        load<G, V>(gn, g + b * 2 * hidden + hidden + c);
        s.w = *reinterpret_cast<const typename Pack<float, V>::W *>(state + at);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Gate z = scan_gate(to_f32(gz.v[k]));
            s.v[k] = v[k] = z.keep * s.v[k] + z.take * to_f32(gn.v[k]);
        }
        *reinterpret_cast<typename Pack<float, V>::W *>(new_state + at) = s.w;
    }
    store<Hy, V>(h + b * hidden + c, v);
}

template <typename F>
int by_types(int g_type, int h_type, F &&f) {
    if (g_type == ISAM_F32) return h_type == ISAM_F32 ? f(float(), float()) : f(float(), bf16());
    return h_type == ISAM_F32 ? f(bf16(), float()) : f(bf16(), bf16());
}

// Whether rows of `hidden` elements and p allow V elements in one word.
bool vector_ok(int hidden, int V, int type, const void *p) {
    return hidden % V == 0 && reinterpret_cast<uintptr_t>(p) % ((type == ISAM_F32 ? 4 : 2) * V) == 0;
}

int scan_launch(void (*fn)(const ScanParams), const GlrDesc &d, int V, int L, const DeviceState &ds, cudaStream_t s,
                const char *what) {
    ScanParams p{};
    p.d = d;
    p.err = ds.err_word;
    p.tiles = (d.hidden + 32 * V - 1) / (32 * V);
    const int64_t groups = static_cast<int64_t>(p.tiles) * d.batch;
    const int warps = std::min(kMaxWarps, (d.T + L - 1) / L);
    // The cluster size with the fewest rounds times waves of CTAs: enough CTAs
    // for the GPU where the channels alone are too few, no more than one wave
    // of them where time is split.
    const int64_t slots = static_cast<int64_t>(ds.num_sms) * kCtasPerSm;
    int64_t best = 0;
    for (int c = 1; c <= kMaxCluster; ++c) {
        const int64_t rounds = (d.T + static_cast<int64_t>(c) * warps * L - 1) / (static_cast<int64_t>(c) * warps * L);
        const int64_t cost = rounds * ((groups * c + slots - 1) / slots);
        if (c == 1 || cost < best) {
            best = cost;
            p.cluster = static_cast<uint32_t>(c);
        }
    }
    if (groups * p.cluster > 0x7fffffffLL)
        return set_error(ISAM_ERR_UNSUPPORTED, "batch * hidden is too large for one launch");
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = dim3(static_cast<unsigned>(groups * p.cluster));
    cfg.blockDim = dim3(32 * warps);
    cfg.stream = s;
    if (p.cluster > 1) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = p.cluster;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, static_cast<const ScanParams>(p));
    return e == cudaSuccess ? ISAM_OK : cuda_error(e, what);
}

}  // namespace

// V and L keep a row of a warp at 128 bytes of gates and a thread's z, b and
// prefetched gates within 128 registers.
int glr_forward_launch(const GlrDesc &d, DeviceState &ds, cudaStream_t s) {
    return by_types(d.g_type, d.h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        const char *what = "launch glr_forward_kernel";
        if constexpr (sizeof(G) == 2) {
            if (vector_ok(d.hidden, 2, d.g_type, d.g) && vector_ok(d.hidden, 2, d.h_type, d.h_out))
                return scan_launch(glr_forward_kernel<G, Hy, 2, 16>, d, 2, 16, ds, s, what);
        }
        return scan_launch(glr_forward_kernel<G, Hy, 1, 16>, d, 1, 16, ds, s, what);
    });
}

int glr_backward_launch(const GlrDesc &d, DeviceState &ds, cudaStream_t s) {
    return by_types(d.g_type, d.h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        const char *what = "launch glr_backward_kernel";
        if constexpr (sizeof(G) == 2) {
            if (vector_ok(d.hidden, 2, d.g_type, d.g) && vector_ok(d.hidden, 2, d.g_type, d.dg) &&
                vector_ok(d.hidden, 2, d.h_type, d.h_in) && vector_ok(d.hidden, 2, d.h_type, d.dh_out))
                return scan_launch(glr_backward_kernel<G, Hy, 2, 8>, d, 2, 8, ds, s, what);
        }
        return scan_launch(glr_backward_kernel<G, Hy, 1, 8>, d, 1, 8, ds, s, what);
    });
}

int glr_step_launch(int batch, int hidden, int slots, int g_type, const void *g, const int32_t *slot_ids,
                    const float *state, float *new_state, int h_type, void *h, cudaStream_t s) {
    return by_types(g_type, h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        const bool four = vector_ok(hidden, 4, g_type, g) && vector_ok(hidden, 4, h_type, h) &&
                          vector_ok(hidden, 4, ISAM_F32, state) && vector_ok(hidden, 4, ISAM_F32, new_state);
        const int64_t threads = static_cast<int64_t>(batch) * (four ? hidden / 4 : hidden);
        const unsigned blocks = static_cast<unsigned>((threads + kStepThreads - 1) / kStepThreads);
        const auto fn = four ? glr_step_kernel<G, Hy, 4> : glr_step_kernel<G, Hy, 1>;
        fn<<<blocks, kStepThreads, 0, s>>>(threads, hidden, slots, static_cast<const G *>(g), slot_ids, state,
                                           new_state, static_cast<Hy *>(h));
        return launch_status("launch glr_step_kernel");
    });
}

}  // namespace isam
