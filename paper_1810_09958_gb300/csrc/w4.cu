// w4.cu -- products of a few tokens with 4-bit weights and group scales:
//   y[m][n] = sum_k x[m][k] s[n][k / group] (q[n][k] - 8).
#include "internal.h"
#include "lm_common.cuh"

namespace isam {

namespace {

constexpr int kThreads = 256;

// Nibble i of a code word holds k offset nibble_k(i): a mask of 0x000F000F on
// the word shifted right by 4 i leaves the neighbours 2 i and 2 i + 1.
__host__ __device__ constexpr int nibble_k(int i) { return i < 4 ? 2 * i : 2 * (i - 4) + 1; }

// One thread per 32-bit word of tiled codes.
__global__ void __launch_bounds__(kThreads)
    w4_pack_codes_kernel(int N, int K, int kt, int64_t words, const uint8_t *codes, uint32_t *tiled) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= words) return;
    const int w = static_cast<int>(i & 255);
    const int64_t tile = i >> 8;
    const int half = w >> 7, lane = (w >> 2) & 31, j = w & 3;
    const int64_t n = tile / kt * 16 + half * 8 + (lane >> 2);
    const int64_t k0 = tile % kt * 128 + 32 * j + 8 * (lane & 3);
    uint32_t v = 0;
    for (int b = 0; b < 8; ++b) {
        const int64_t k = k0 + nibble_k(b);
        uint32_t q = 8;  // padding: weight 0
        if (n < N && k < K) q = (codes[n * (K / 2) + k / 2] >> (4 * (k & 1))) & 15u;
        v |= q << (4 * b);
    }
    tiled[i] = v;
}

__global__ void __launch_bounds__(kThreads)
    w4_pack_scales_kernel(int N, int groups, int kt, int per, int64_t count, const uint16_t *scales, uint16_t *tiled) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= count) return;
    const int p = static_cast<int>(i % per);
    const int row = static_cast<int>(i / per % 16);
    const int64_t tile = i / (per * 16);
    const int64_t n = tile / kt * 16 + row;
    const int64_t gr = tile % kt * per + p;
    tiled[i] = n < N && gr < groups ? scales[n * groups + gr] : static_cast<uint16_t>(0);
}

// One warp per output row and token.
__global__ void __launch_bounds__(kThreads)
    gemv_w4_kernel(int M, int N, int K, int group, int kt, const bf16 *x, const uint32_t *tiled, const bf16 *scales,
                   float *y) {
    const int64_t n = static_cast<int64_t>(blockIdx.x) * (kThreads / 32) + (threadIdx.x >> 5);
    const int m = blockIdx.y, lane = threadIdx.x & 31;
    if (n >= N) return;
    const int per = 128 / group, row = static_cast<int>(n & 15);
    float sum = 0.0f;
    for (int k = lane; k < K; k += 32) {
        const int64_t tile = (n >> 4) * kt + (k >> 7);
        const int in = k & 127, j = in >> 5, t = (in >> 3) & 3, e = in & 7;
        const int nib = (e >> 1) + 4 * (e & 1);
        const uint32_t w = tiled[tile * 256 + (row >> 3) * 128 + ((row & 7) * 4 + t) * 4 + j];
        const float q = static_cast<float>((w >> (4 * nib)) & 15u) - 8.0f;
        sum += to_f32(x[static_cast<int64_t>(m) * K + k]) * q * to_f32(scales[(tile * 16 + row) * per + in / group]);
    }
    for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == 0) y[static_cast<int64_t>(m) * N + n] = sum;
}

}  // namespace

int w4_pack_launch(int N, int K, int group, const uint8_t *codes, const uint16_t *scales, uint8_t *tiled,
                   uint16_t *tiled_scales, cudaStream_t s) {
    const int nb = (N + 15) / 16, kt = (K + 127) / 128, per = 128 / group;
    const int64_t words = static_cast<int64_t>(nb) * kt * 256, count = static_cast<int64_t>(nb) * kt * 16 * per;
    w4_pack_codes_kernel<<<static_cast<unsigned>((words + kThreads - 1) / kThreads), kThreads, 0, s>>>(
        N, K, kt, words, codes, reinterpret_cast<uint32_t *>(tiled));
    const int rc = launch_status("launch w4_pack_codes_kernel");
    if (rc) return rc;
    w4_pack_scales_kernel<<<static_cast<unsigned>((count + kThreads - 1) / kThreads), kThreads, 0, s>>>(
        N, (K + group - 1) / group, kt, per, count, scales, tiled_scales);
    return launch_status("launch w4_pack_scales_kernel");
}

int gemv_w4_launch(int M, int N, int K, int group, const uint16_t *x, const uint8_t *tiled, const uint16_t *scales,
                   float *y, DeviceState &ds, cudaStream_t s) {
    const dim3 grid((N + kThreads / 32 - 1) / (kThreads / 32), M);
    gemv_w4_kernel<<<grid, kThreads, 0, s>>>(M, N, K, group, (K + 127) / 128, reinterpret_cast<const bf16 *>(x),
                                             reinterpret_cast<const uint32_t *>(tiled),
                                             reinterpret_cast<const bf16 *>(scales), y);
    return launch_status("launch gemv_w4_kernel");
}

}  // namespace isam
