// norm.cu -- root-mean-square norm of the rows of a residual stream, with the
// addition before it and an output in bf16, fp32 or block-scaled E4M3, and its
// backward pass:
//   r = x + res,  k = 1 / sqrt(mean(r^2) + eps),  y = r k w;
//   d = w dy, n = r k:  dx = k (d - n mean(d n)) + dres,  dw = sum over rows of dy n.
//
// A row is held in the registers of one team of warps from its only reading to
// its only writing, so the bound is HBM: every operand moves once.  A team has
// as many warps as its row needs with NV vectors of V elements a thread; rows
// that start on 16-byte boundaries take V = 8, others V = 1, neighbouring
// threads on neighbouring elements either way.
#include "lm_common.cuh"

namespace isam {

namespace {

constexpr int kMaxThreads = 1024;

template <typename T, int V>
struct alignas(V == 8 ? 16 : sizeof(T)) Vec {
    T v[V];
};

// V elements at p as fp32.
template <int V, typename T>
__device__ __forceinline__ void load(const T *p, float (&f)[V]) {
    const Vec<T, V> a = *reinterpret_cast<const Vec<T, V> *>(p);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = to_f32(a.v[i]);
}

template <int V, typename T>
__device__ __forceinline__ void store(T *p, const float (&f)[V]) {
    Vec<T, V> a;
#pragma unroll
    for (int i = 0; i < V; ++i) a.v[i] = from_f32<T>(f[i]);
    *reinterpret_cast<Vec<T, V> *>(p) = a;
}

__device__ __forceinline__ float warp_sum(float s) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(~0u, s, d);
    return s;
}

// The team's sum in every thread of it: `part` holds a word for each warp of the
// CTA; all its threads call this.  Two buffers in turn need one barrier a sum.
__device__ __forceinline__ float team_sum(float s, int warps, float *part) {
    s = warp_sum(s);
    if (warps == 1) return s;
    const int warp = threadIdx.x / 32, first = warp / warps * warps;
    if (threadIdx.x % 32 == 0) part[warp] = s;
    __syncthreads();
    float t = 0.0f;
    for (int i = 0; i < warps; ++i) t += part[first + i];
    return t;
}

struct Mx {};  // output in E4M3 with a scale for each 32

// The scale byte of a block whose largest magnitude has these bits, and the
// factor that brings its values to E4M3's range: the least 2^e with
// amax <= 448 2^e = 1.75 2^(e + 8).  The mantissa is compared with 1.75 by a carry.
__device__ __forceinline__ uint32_t mx_scale(uint32_t amax_bits, float &inv) {
    if (amax_bits >= 0x7f800000u) {
        inv = __uint_as_float(0x7fc00000u);
        return 255u;
    }
    const int e = static_cast<int>((amax_bits + 0x1fffffu) >> 23) - 8;
    const uint32_t byte = e < 0 ? 0u : static_cast<uint32_t>(e);
    inv = __uint_as_float((254u - byte) << 23);  // 2^(127 - byte); byte <= 247
    return byte;
}

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}

template <typename X, typename R, typename Y, int V, int NV>
__global__ void __launch_bounds__(kMaxThreads)
    norm_forward_kernel(int T, int D, int team_warps, int teams, const X *x, const R *res, R *res_out, const float *w,
                        float eps, Y *y, uint8_t *y8, uint8_t *y8_scales) {
    __shared__ float part[32];
    dependent_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int team = warp / team_warps, tid = (warp - team * team_warps) * 32 + lane;
    const int64_t row = static_cast<int64_t>(blockIdx.x) * teams + team;
    const bool on = row < T;
    const int step = team_warps * 32 * V;
    const int64_t base = row * D;

    float r[NV][V], sum = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = j * step + tid * V;
#pragma unroll
        for (int i = 0; i < V; ++i) r[j][i] = 0.0f;
        if (on && c < D) load<V>(x + base + c, r[j]);
    }
    if (res)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = j * step + tid * V;
            if (on && c < D) {
                float a[V];
                load<V>(res + base + c, a);
#pragma unroll
                for (int i = 0; i < V; ++i) r[j][i] += a[i];
            }
        }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = j * step + tid * V;
        if (res_out && on && c < D) store<V>(res_out + base + c, r[j]);
#pragma unroll
        for (int i = 0; i < V; ++i) sum = fmaf(r[j][i], r[j][i], sum);
    }
    sum = team_sum(sum, team_warps, part);
    const float k = rsqrtf(sum / static_cast<float>(D) + eps);
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const int c = j * step + tid * V;
        float o[V];
#pragma unroll
        for (int i = 0; i < V; ++i) o[i] = 0.0f;
        if (c < D) {
            load<V>(w + c, o);
#pragma unroll
            for (int i = 0; i < V; ++i) o[i] *= r[j][i] * k;
        }
        if constexpr (!std::is_same<Y, Mx>::value) {
            if (on && c < D) store<V>(y + base + c, o);
        } else {
            // A block of 32 is 4 lanes of 8 elements, or 32 lanes of one; infinities and NaN have the largest bits.
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(o[i]) & 0x7fffffffu);
#pragma unroll
            for (int d = 1; d < 32 / V; d <<= 1) top = max(top, __shfl_xor_sync(~0u, top, d));
            float inv;
            uint32_t scale = mx_scale(top, inv);
            const int atom = c / 128, atoms = (D + 127) / 128;
            if constexpr (V == 8) {
                uint2 q;
                q.x = e4m3x2(o[0] * inv, o[1] * inv) | e4m3x2(o[2] * inv, o[3] * inv) << 16;
                q.y = e4m3x2(o[4] * inv, o[5] * inv) | e4m3x2(o[6] * inv, o[7] * inv) << 16;
                if (on && c < D) *reinterpret_cast<uint2 *>(y8 + base + c) = q;
                // The four blocks of an atom lie in 16 lanes: one word.
                scale |= __shfl_down_sync(~0u, scale, 4) << 8;
                scale |= __shfl_down_sync(~0u, scale, 8) << 16;
                if (on && lane % 16 == 0 && atom < atoms)
                    *reinterpret_cast<uint32_t *>(y8_scales + (static_cast<int64_t>(atom) * T + row) * 4) = scale;
            } else {
                if (on && c < D) y8[base + c] = static_cast<uint8_t>(e4m3x2(o[0] * inv, 0.0f));
                if (on && lane == 0 && atom < atoms)
                    y8_scales[(static_cast<int64_t>(atom) * T + row) * 4 + c / 32 % 4] = static_cast<uint8_t>(scale);
            }
        }
    }
}

// Rows are walked by persistent CTAs, whose threads keep their columns' sums of
// dw; the CTA's sum goes to a row of `part` in the workspace.  KEEP: r and dy
// stay in registers between the sums and dx; else they are read again (wide rows).
template <typename R, typename G, int V, int NV, bool KEEP>
__global__ void __launch_bounds__(kMaxThreads)
    norm_backward_kernel(int T, int D, int team_warps, int teams, const R *r, const float *w, float eps, const G *dy,
                         const G *dres, G *dx, float *part) {
    extern __shared__ float smem[];  // [teams - 1][D] behind the loop
    __shared__ float2 sums[2][32];
    dependent_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    const int team = warp / team_warps, tid = (warp - team * team_warps) * 32 + lane;
    const int step = team_warps * 32 * V;
    float acc[NV][V];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[j][i] = 0.0f;

    int turn = 0;
    for (int64_t first = static_cast<int64_t>(blockIdx.x) * teams; first < T;
         first += static_cast<int64_t>(gridDim.x) * teams, turn ^= 1) {
        const int64_t row = first + team;
        const bool on = row < T;
        const int64_t base = row * D;
        Vec<R, V> rv[KEEP ? NV : 1];
        Vec<G, V> gv[KEEP ? NV : 1];
        float s2 = 0.0f, sd = 0.0f;
        if constexpr (KEEP) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int c = j * step + tid * V;
                if (on && c < D) {
                    rv[j] = *reinterpret_cast<const Vec<R, V> *>(r + base + c);
                    gv[j] = *reinterpret_cast<const Vec<G, V> *>(dy + base + c);
                }
            }
        }
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = j * step + tid * V;
            if (on && c < D) {
                float a[V], g[V], ww[V];
                if constexpr (KEEP) {
#pragma unroll
                    for (int i = 0; i < V; ++i) a[i] = to_f32(rv[j].v[i]), g[i] = to_f32(gv[j].v[i]);
                } else {
                    load<V>(r + base + c, a);
                    load<V>(dy + base + c, g);
                }
                load<V>(w + c, ww);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    s2 = fmaf(a[i], a[i], s2);
                    sd = fmaf(a[i] * ww[i], g[i], sd);
                }
            }
        }
        s2 = warp_sum(s2);
        sd = warp_sum(sd);
        if (team_warps > 1) {
            if (lane == 0) sums[turn][warp] = make_float2(s2, sd);
            __syncthreads();
            s2 = sd = 0.0f;
            for (int i = 0; i < team_warps; ++i) {
                const float2 p = sums[turn][team * team_warps + i];
                s2 += p.x;
                sd += p.y;
            }
        }
        const float k = rsqrtf(s2 / static_cast<float>(D) + eps);
        const float m = sd * k / static_cast<float>(D);  // mean(d n)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = j * step + tid * V;
            if (on && c < D) {
                float a[V], g[V], ww[V], o[V];
                if constexpr (KEEP) {
#pragma unroll
                    for (int i = 0; i < V; ++i) a[i] = to_f32(rv[j].v[i]), g[i] = to_f32(gv[j].v[i]);
                } else {
                    load<V>(r + base + c, a);
                    load<V>(dy + base + c, g);
                }
                load<V>(w + c, ww);
#pragma unroll
                for (int i = 0; i < V; ++i) o[i] = 0.0f;
                if (dx && dres) load<V>(dres + base + c, o);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float n = a[i] * k;
                    acc[j][i] = fmaf(g[i], n, acc[j][i]);
                    o[i] = fmaf(k, fmaf(-n, m, ww[i] * g[i]), o[i]);
                }
                if (dx) store<V>(dx + base + c, o);
            }
        }
    }
    if (!part) return;
    // The teams' sums, in the teams' order.
    if (team > 0)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = j * step + tid * V;
            if (c < D)
#pragma unroll
                for (int i = 0; i < V; ++i) smem[(team - 1) * D + c + i] = acc[j][i];
        }
    __syncthreads();
    if (team == 0)
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int c = j * step + tid * V;
            if (c < D) {
                for (int t = 1; t < teams; ++t)
#pragma unroll
                    for (int i = 0; i < V; ++i) acc[j][i] += smem[(t - 1) * D + c + i];
#pragma unroll
                for (int i = 0; i < V; ++i) part[static_cast<int64_t>(blockIdx.x) * D + c + i] = acc[j][i];
            }
        }
}

constexpr int kSumRows = 32;

// dw from the CTAs' rows: 32 columns a CTA, its 32 warps share the rows.
__global__ void __launch_bounds__(32 * kSumRows) norm_sum_kernel(int D, int rows, const float *part, float *dw) {
    __shared__ float sums[kSumRows][33];
    dependent_start();
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, c = blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (c < D)
        for (int i = warp; i < rows; i += kSumRows) s += part[static_cast<int64_t>(i) * D + c];
    sums[warp][lane] = s;
    __syncthreads();
    s = warp_sum(sums[lane][warp]);
    if (lane == 0 && blockIdx.x * 32 + warp < D) dw[blockIdx.x * 32 + warp] = s;
}

bool rows16(int D, int type, const void *p) {
    const int size = type == ISAM_F32 ? 4 : 2;
    return static_cast<int64_t>(D) * size % 16 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

template <typename F>
int by_type(int type, F &&f) {
    return type == ISAM_F32 ? f(float()) : f(bf16());
}

// Warps of a team for rows of D elements, NV vectors of V a thread.
int team_warps(int D, int V, int NV) { return (D + 32 * V * NV - 1) / (32 * V * NV); }

template <typename X, typename R, typename Y, int V, int NV>
int forward(const NormDesc &p, cudaStream_t s) {
    const int tw = team_warps(p.D, V, NV);
    const int teams = tw >= 4 ? 1 : 4 / tw;
    const unsigned blocks = static_cast<unsigned>((p.T + static_cast<int64_t>(teams) - 1) / teams);
    return launch_dependent(norm_forward_kernel<X, R, Y, V, NV>, dim3(blocks), teams * tw * 32, 0, s, 1,
                            "launch norm_forward_kernel", p.T, p.D, tw, teams, static_cast<const X *>(p.x),
                            static_cast<const R *>(p.res), static_cast<R *>(p.res_out), p.w, p.eps,
                            static_cast<Y *>(p.y), p.y8, p.y8_scales);
}

constexpr int kBackCtas = 152;  // the workspace has a row for each

template <typename R, typename G, int V, int NV, bool KEEP>
int backward(const NormBackDesc &p, cudaStream_t s) {
    const int tw = team_warps(p.D, V, NV);
    const int teams = tw >= 16 ? 1 : 16 / tw;
    const int64_t most = (p.T + static_cast<int64_t>(teams) - 1) / teams;
    const int blocks = static_cast<int>(most < kBackCtas ? most : kBackCtas);
    const size_t smem = static_cast<size_t>(teams - 1) * p.D * 4;
    const auto fn = norm_backward_kernel<R, G, V, NV, KEEP>;
    int rc = launch_dependent(fn, dim3(blocks), teams * tw * 32, smem, s, 1, "launch norm_backward_kernel", p.T, p.D,
                              tw, teams, static_cast<const R *>(p.r), p.w, p.eps, static_cast<const G *>(p.dy),
                              static_cast<const G *>(p.dres), static_cast<G *>(p.dx), p.dw ? p.workspace : nullptr);
    if (rc || !p.dw) return rc;
    return launch_dependent(norm_sum_kernel, dim3((p.D + 31) / 32), 32 * kSumRows, 0, s, 1, "launch norm_sum_kernel",
                            p.D, blocks, p.workspace, p.dw);
}

}  // namespace

int norm_forward_launch(const NormDesc &p, DeviceState &, cudaStream_t s) {
    const bool wide = rows16(p.D, p.x_type, p.x) && rows16(p.D, p.r_type, p.res) && rows16(p.D, p.r_type, p.res_out) &&
                      reinterpret_cast<uintptr_t>(p.w) % 16 == 0 && p.D % 8 == 0 &&
                      (p.y ? rows16(p.D, p.y_type, p.y) : reinterpret_cast<uintptr_t>(p.y8) % 8 == 0);
    return by_type(p.x_type, [&](auto x) {
        return by_type(p.r_type, [&](auto r) {
            using X = decltype(x);
            using R = decltype(r);
            const auto as = [&](auto y) {
                using Y = decltype(y);
                if (!wide) return p.D <= 8192 ? forward<X, R, Y, 1, 8>(p, s) : forward<X, R, Y, 1, 32>(p, s);
                if (p.D <= 8192) return forward<X, R, Y, 8, 1>(p, s);
                return forward<X, R, Y, 8, 4>(p, s);
            };
            return p.y_type < 0 ? as(Mx()) : by_type(p.y_type, as);
        });
    });
}

size_t norm_backward_workspace(int, int D) { return static_cast<size_t>(kBackCtas) * D * 4; }

int norm_backward_launch(const NormBackDesc &p, DeviceState &, cudaStream_t s) {
    if (!p.dx && !p.dw) return ISAM_OK;
    const bool wide = rows16(p.D, p.r_type, p.r) && rows16(p.D, p.g_type, p.dy) && rows16(p.D, p.g_type, p.dres) &&
                      rows16(p.D, p.g_type, p.dx) && reinterpret_cast<uintptr_t>(p.w) % 16 == 0 && p.D % 8 == 0;
    return by_type(p.r_type, [&](auto r) {
        return by_type(p.g_type, [&](auto g) {
            using R = decltype(r);
            using G = decltype(g);
            if (!wide) return p.D <= 8192 ? backward<R, G, 1, 8, true>(p, s) : backward<R, G, 1, 32, false>(p, s);
            if (p.D <= 8192) return backward<R, G, 8, 1, true>(p, s);
            return backward<R, G, 8, 4, false>(p, s);
        });
    });
}

}  // namespace isam
