// glu.cu -- gated feed-forward product h = act(x Wg^T) * (x Wu^T), with
// W = [Wg; Wu] one [2F][D] matrix, and its backward pass.
#include "internal.h"
#include "lm_common.cuh"

namespace isam {

namespace {

constexpr int kTile = 16;

// Gate and up sums of one (token, feature) by one thread, 16 x 16 a block;
// BACK: writes d[t][f] = dh u act'(g) and d[t][F + f] = dh act(g).
template <int ACT, bool BACK>
__global__ void __launch_bounds__(kTile *kTile)
    glu_kernel(int T, int D, int F, const bf16 *x, const bf16 *W, const bf16 *dh, bf16 *out) {
    __shared__ float sx[kTile][kTile + 1], sg[kTile][kTile + 1], su[kTile][kTile + 1];
    const int tx = threadIdx.x % kTile, ty = threadIdx.x / kTile;
    const int64_t f = static_cast<int64_t>(blockIdx.x) * kTile + tx, t = static_cast<int64_t>(blockIdx.y) * kTile + ty;
    const int64_t wf = static_cast<int64_t>(blockIdx.x) * kTile + ty;
    float g = 0.0f, u = 0.0f;
    for (int k0 = 0; k0 < D; k0 += kTile) {
        const int k = k0 + tx;
        sx[ty][tx] = t < T && k < D ? to_f32(x[t * D + k]) : 0.0f;
        sg[ty][tx] = wf < F && k < D ? to_f32(W[wf * D + k]) : 0.0f;
        su[ty][tx] = wf < F && k < D ? to_f32(W[(wf + F) * D + k]) : 0.0f;
        __syncthreads();
        for (int i = 0; i < kTile; ++i) {
            g += sx[ty][i] * sg[tx][i];
            u += sx[ty][i] * su[tx][i];
        }
        __syncthreads();
    }
    if (t >= T || f >= F) return;
    float a, da;
    activation<ACT>(g, a, da);
    if (BACK) {
        const float d = to_f32(dh[t * F + f]);
        out[t * 2 * F + f] = from_f32<bf16>(d * u * da);
        out[t * 2 * F + F + f] = from_f32<bf16>(d * a);
    } else {
        out[t * F + f] = from_f32<bf16>(a * u);
    }
}

// C (M x N, bf16) = op(A) B, B K x N; A_T: A stored K x M.
template <bool A_T>
__global__ void __launch_bounds__(kTile *kTile)
    glu_product_kernel(int64_t M, int64_t N, int64_t K, const bf16 *A, const bf16 *B, bf16 *C) {
    __shared__ float sa[kTile][kTile + 1], sb[kTile][kTile + 1];
    const int tx = threadIdx.x % kTile, ty = threadIdx.x / kTile;
    const int64_t m0 = static_cast<int64_t>(blockIdx.y) * kTile, n = static_cast<int64_t>(blockIdx.x) * kTile + tx;
    float sum = 0.0f;
    for (int64_t k0 = 0; k0 < K; k0 += kTile) {
        if (A_T)
            sa[tx][ty] = m0 + tx < M && k0 + ty < K ? to_f32(A[(k0 + ty) * M + m0 + tx]) : 0.0f;
        else
            sa[ty][tx] = m0 + ty < M && k0 + tx < K ? to_f32(A[(m0 + ty) * K + k0 + tx]) : 0.0f;
        sb[ty][tx] = n < N && k0 + ty < K ? to_f32(B[(k0 + ty) * N + n]) : 0.0f;
        __syncthreads();
        for (int i = 0; i < kTile; ++i) sum += sa[ty][i] * sb[i][tx];
        __syncthreads();
    }
    if (m0 + ty < M && n < N) C[(m0 + ty) * N + n] = from_f32<bf16>(sum);
}

dim3 tiles(int64_t n, int64_t m) {
    return dim3(static_cast<unsigned>((n + kTile - 1) / kTile), static_cast<unsigned>((m + kTile - 1) / kTile));
}

template <bool BACK>
int glu_run(int T, int D, int F, int act, const uint16_t *x, const uint16_t *W, const uint16_t *dh, uint16_t *out,
            cudaStream_t s) {
    const auto fn = act == ISAM_ACT_SILU   ? glu_kernel<ISAM_ACT_SILU, BACK>
                    : act == ISAM_ACT_GELU ? glu_kernel<ISAM_ACT_GELU, BACK>
                    : act == ISAM_ACT_RELU ? glu_kernel<ISAM_ACT_RELU, BACK>
                                           : glu_kernel<ISAM_ACT_SIGMOID, BACK>;
    fn<<<tiles(F, T), kTile * kTile, 0, s>>>(T, D, F, reinterpret_cast<const bf16 *>(x),
                                             reinterpret_cast<const bf16 *>(W), reinterpret_cast<const bf16 *>(dh),
                                             reinterpret_cast<bf16 *>(out));
    return launch_status("launch glu_kernel");
}

}  // namespace

int glu_forward_launch(const GluDesc &p, DeviceState &ds, cudaStream_t s) {
    return glu_run<false>(p.T, p.D, p.F, p.act, p.x, p.W, nullptr, p.h, s);
}

size_t glu_backward_workspace(int T, int D, int F) { return static_cast<size_t>(T) * F * 4; }

int glu_backward_launch(const GluDesc &p, DeviceState &ds, cudaStream_t s) {
    uint16_t *d = static_cast<uint16_t *>(p.workspace);
    int rc = glu_run<true>(p.T, p.D, p.F, p.act, p.x, p.W, p.dh, d, s);
    if (rc) return rc;
    const int64_t F2 = 2 * static_cast<int64_t>(p.F);
    if (p.dx) {
        glu_product_kernel<false><<<tiles(p.D, p.T), kTile * kTile, 0, s>>>(
            p.T, p.D, F2, reinterpret_cast<const bf16 *>(d), reinterpret_cast<const bf16 *>(p.W),
            reinterpret_cast<bf16 *>(p.dx));
        if ((rc = launch_status("launch glu_product_kernel"))) return rc;
    }
    if (p.dW) {
        glu_product_kernel<true><<<tiles(p.D, F2), kTile * kTile, 0, s>>>(
            F2, p.D, p.T, reinterpret_cast<const bf16 *>(d), reinterpret_cast<const bf16 *>(p.x),
            reinterpret_cast<bf16 *>(p.dW));
        if ((rc = launch_status("launch glu_product_kernel"))) return rc;
    }
    return ISAM_OK;
}

}  // namespace isam
