// two.cuh -- packed pairs of fp32 (half the issue slots of single ones; the same
// rate on the multiply-add pipe) and the exponential unit's instruction.
#pragma once
#include <cstdint>

namespace isam {

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Two fp32 values in one 64-bit register pair.
struct Two {
    uint64_t x;
};
__device__ __forceinline__ Two two(float lo, float hi) {
    Two d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d.x) : "f"(lo), "f"(hi));
    return d;
}
__device__ __forceinline__ float2 apart(Two a) {
    float2 f;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(f.x), "=f"(f.y) : "l"(a.x));
    return f;
}
__device__ __forceinline__ Two mul(Two a, Two b) {
    Two d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.x) : "l"(a.x), "l"(b.x));
    return d;
}
__device__ __forceinline__ Two fma(Two a, Two b, Two c) {
    Two d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.x) : "l"(a.x), "l"(b.x), "l"(c.x));
    return d;
}
__device__ __forceinline__ Two add2(Two a, Two b) {
    Two d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.x) : "l"(a.x), "l"(b.x));
    return d;
}
__device__ __forceinline__ Two exp2_fast(Two a) {
    const float2 f = apart(a);
    return two(exp2_fast(f.x), exp2_fast(f.y));
}

}  // namespace isam
