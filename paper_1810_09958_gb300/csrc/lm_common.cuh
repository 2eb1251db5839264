// lm_common.cuh -- element types, the gate and the activations shared by the
// gated linear recurrence and the gated feed-forward kernels.
#pragma once
#include <cuda_bf16.h>

#include "internal.h"
#include "ptx.cuh"

namespace isam {

using bf16 = __nv_bfloat16;

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(bf16 v) { return __bfloat162float(v); }
template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) {
    return v;
}
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float v) {
    return __float2bfloat16_rn(v);
}

// sigmoid(x) and 1 - sigmoid(x), each to a few units in the last place of
// its own size (the smaller of the two is not a difference from 1): with
// e = exp(-|x|) they are 1 / (1 + e) and e / (1 + e), in the order of x's sign.
struct Gate {
    float keep;  // sigmoid(x)
    float take;  // 1 - sigmoid(x)
};
__device__ __forceinline__ Gate gate(float x) {
    const float e = __expf(-fabsf(x));
    const float r = __fdividef(1.0f, 1.0f + e);
    const float s = e * r;
    return x >= 0.0f ? Gate{r, s} : Gate{s, r};
}

// P(-x), x >= 0, of the normal distribution, given e = exp(-x^2 / 2), to 4e-7 of itself
// (x from 0 to 14, beside e's own error): (1 + erf(-x / sqrt 2)) / 2 comes in steps of
// 3e-8, which is all of P from x = 5.4 on.  P(-x) / e falls from 1/2 like 1 / x, so it
// is t (c0 + c1 t + ... + c7 t^7) with t = 1 / (1 + 0.305 x); the coefficients minimise
// the largest relative error (least squares, reweighted), and 0.305 is the best of
// the poles tried.  200 x 1760 x 4096 with GELU takes 11.5 us, with erfcf 13.5.
__device__ __forceinline__ float normal_tail(float x, float e) {
    const float t = __fdividef(1.0f, fmaf(0.305000007f, x, 1.0f));
    float p = 0.0366991833f;
    p = fmaf(p, t, -0.152988285f);
    p = fmaf(p, t, 0.185716853f);
    p = fmaf(p, t, -0.0379767828f);
    p = fmaf(p, t, 0.121021651f);
    p = fmaf(p, t, 0.103420876f);
    p = fmaf(p, t, 0.122466817f);
    p = fmaf(p, t, 0.121639736f);
    return p * t * e;
}

// act(a) and its derivative.
template <int ACT>
__device__ __forceinline__ void activation(float a, float &v, float &dv) {
    if (ACT == ISAM_ACT_RELU) {
        v = a > 0.0f ? a : (a != a ? a : 0.0f);
        dv = a > 0.0f ? 1.0f : 0.0f;
    } else if (ACT == ISAM_ACT_GELU) {
        // a P(a) with P the normal distribution function.
        const float e = __expf(-0.5f * a * a);
        const float q = normal_tail(fabsf(a), e);
        const float p = a < 0.0f ? q : 1.0f - q;
        v = a * p;
        dv = p + a * (0.39894228040143268f * e);
    } else {
        const Gate s = gate(a);
        if (ACT == ISAM_ACT_SIGMOID) {
            v = s.keep;
            dv = s.keep * s.take;
        } else {
            v = a * s.keep;
            dv = s.keep * (1.0f + a * s.take);
        }
    }
}

// Launches a kernel that begins with dependent_start(): its CTAs may be set up
// while the stream's previous kernel drains (programmatic dependent launch).
// `cluster` CTAs a cluster where above 1.
template <typename... Params, typename... Args>
int launch_dependent(void (*fn)(Params...), dim3 grid, int threads, size_t smem, cudaStream_t s, unsigned cluster,
                     const char *what, Args &&...args) {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.numAttrs = 1;
    if (cluster > 1) {
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.numAttrs = 2;
    }
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, static_cast<Params>(args)...);
    return e == cudaSuccess ? ISAM_OK : cuda_error(e, what);
}

// Before a kernel's first access to global memory: the next kernel may be set
// up from here, and everything the previous ones wrote is visible after.
__device__ __forceinline__ void dependent_start() {
    griddep_launch_dependents();
    griddep_wait();
}

inline int launch_status(const char *what) {
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? ISAM_OK : cuda_error(e, what);
}

}  // namespace isam
