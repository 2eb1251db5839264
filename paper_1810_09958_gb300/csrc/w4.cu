// w4.cu -- products of a few tokens with 4-bit weights and group scales:
//   y[m][n] = sum_k x[m][k] s[n][k / group] (q[n][k] - 8).
#include <algorithm>

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

constexpr int kMaxWarps = 16;
constexpr int kTileWords = 256;  // 32-bit words of a 16 x 128 tile

__device__ __forceinline__ void mma_16x8x16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
        "{%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// Codes 2 i and 2 i + 1 (in k) of a word as bf16 q - 8: the codes become the low
// mantissa bits of 128 + q, and 136 is subtracted, all exact.
__device__ __forceinline__ uint32_t dequant(uint32_t w, int i) {
    uint32_t v;
    asm("lop3.b32 %0, %1, 0x000F000F, 0x43004300, 0xEA;" : "=r"(v) : "r"(w >> (4 * i)));
    asm("fma.rn.bf16x2 %0, %0, %1, %2;" : "+r"(v) : "r"(0x3F803F80u), "r"(0xC308C308u));
    return v;
}

// The scales of a row in one tile: 128 / GROUP bf16.
template <int GROUP>
struct RowScales {
    static constexpr int kPer = 128 / GROUP;
    uint32_t w[(kPer + 1) / 2];
    __device__ __forceinline__ void load(const uint16_t *at) {
        if constexpr (kPer == 4) {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(at));
            w[0] = v.x, w[1] = v.y;
        } else if constexpr (kPer == 2) {
            w[0] = __ldg(reinterpret_cast<const uint32_t *>(at));
        } else {
            w[0] = __ldg(at);
        }
    }
    __device__ __forceinline__ float get(int j) const {
        return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
};

// RB blocks of 16 rows by 8 NT tokens a CTA; its warps share K's tiles in turn
// and their sums meet in shared memory, in the order of the warps.
//
// A tile is one k range of 128; lane 4 r + t holds rows r and 8 + r, in word j the
// k of group t of 8 in 32-block j.  The order of k inside a product does not
// matter, so the words' codes are operands of m16n8k16 as they lie, with the
// token's same eight k, 16 bytes of x, beside them, and 16 of one 32-block's k in
// each instruction: a scale applies to whole sums.
template <int NT, int GROUP, int RB>
__global__ void __launch_bounds__(32 * kMaxWarps)
    gemv_w4_kernel(int M, int N, int K, int kt, const uint16_t *x, const uint4 *tiled, const uint16_t *scales,
                   float *y) {
    constexpr int kPer = 128 / GROUP;
    extern __shared__ float part[];  // [warps][8 NT tokens][16 RB rows]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const int r = lane >> 2, t = lane & 3;
    const int nb = (N + 15) / 16, nb0 = blockIdx.x * RB;
    float sum[RB][NT][4] = {};
    uint4 code[RB][2];
    RowScales<GROUP> sc[RB][2];
    const auto load = [&](int k) {
#pragma unroll
        for (int b = 0; b < RB; ++b) {
            const int64_t tile = static_cast<int64_t>(min(nb0 + b, nb - 1)) * kt + k;
            const uint4 *at = tiled + tile * (kTileWords / 4) + lane;
            code[b][0] = __ldcs(at);
            code[b][1] = __ldcs(at + 32);
            sc[b][0].load(scales + (tile * 16 + r) * kPer);
            sc[b][1].load(scales + (tile * 16 + 8 + r) * kPer);
        }
    };
    if (warp < kt) load(warp);
    for (int k = warp; k < kt; k += warps) {
        uint32_t w[RB][2][4];
        RowScales<GROUP> s[RB][2];
#pragma unroll
        for (int b = 0; b < RB; ++b)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                w[b][h][0] = code[b][h].x, w[b][h][1] = code[b][h].y;
                w[b][h][2] = code[b][h].z, w[b][h][3] = code[b][h].w;
                s[b][h] = sc[b][h];
            }
        if (k + warps < kt) load(k + warps);
        float acc[RB][NT][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint4 xv[NT];
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const int m = 8 * n + r, at = 128 * k + 32 * j + 8 * t;
                xv[n] = make_uint4(0, 0, 0, 0);
                if (m < M && at < K) xv[n] = __ldg(reinterpret_cast<const uint4 *>(x + static_cast<int64_t>(m) * K + at));
            }
#pragma unroll
            for (int b = 0; b < RB; ++b) {
                if (j % (GROUP / 32) == 0) {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) acc[b][n][i] = 0.0f;
                }
                uint32_t a[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    a[0] = dequant(w[b][0][j], 2 * h);
                    a[1] = dequant(w[b][1][j], 2 * h);
                    a[2] = dequant(w[b][0][j], 2 * h + 1);
                    a[3] = dequant(w[b][1][j], 2 * h + 1);
#pragma unroll
                    for (int n = 0; n < NT; ++n)
                        mma_16x8x16(acc[b][n], a, h ? xv[n].z : xv[n].x, h ? xv[n].w : xv[n].y);
                }
                if ((j + 1) % (GROUP / 32) == 0) {
                    const float lo = s[b][0].get(j / (GROUP / 32)), hi = s[b][1].get(j / (GROUP / 32));
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        sum[b][n][0] += lo * acc[b][n][0];
                        sum[b][n][1] += lo * acc[b][n][1];
                        sum[b][n][2] += hi * acc[b][n][2];
                        sum[b][n][3] += hi * acc[b][n][3];
                    }
                }
            }
        }
    }
    constexpr int kRows = 16 * RB, kSize = kRows * 8 * NT;
#pragma unroll
    for (int b = 0; b < RB; ++b)
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                part[warp * kSize + (8 * n + 2 * t + (i & 1)) * kRows + 16 * b + r + 8 * (i >> 1)] = sum[b][n][i];
    __syncthreads();
    for (int i = threadIdx.x; i < kSize; i += blockDim.x) {
        const int m = i / kRows, n = nb0 * 16 + i % kRows;
        if (m >= M || n >= N) continue;
        float v = 0.0f;
        for (int q = 0; q < warps; ++q) v += part[q * kSize + i];
        y[static_cast<int64_t>(m) * N + n] = v;
    }
}

template <int NT, int GROUP, int RB>
int gemv_launch(int M, int N, int K, const uint16_t *x, const uint8_t *tiled, const uint16_t *scales, float *y,
                int warps, cudaStream_t s) {
    const int nb = (N + 15) / 16, kt = (K + 127) / 128;
    const size_t smem = static_cast<size_t>(warps) * 16 * RB * 8 * NT * sizeof(float);
    gemv_w4_kernel<NT, GROUP, RB><<<(nb + RB - 1) / RB, 32 * warps, smem, s>>>(
        M, N, K, kt, x, reinterpret_cast<const uint4 *>(tiled), scales, y);
    return launch_status("launch gemv_w4_kernel");
}

template <int NT, int GROUP>
int gemv_rows(int M, int N, int K, const uint16_t *x, const uint8_t *tiled, const uint16_t *scales, float *y,
              const DeviceState &ds, cudaStream_t s) {
    const int nb = (N + 15) / 16, kt = (K + 127) / 128;
    const int warps = std::min(8, kt);
    if (nb >= 8 * ds.num_sms) return gemv_launch<NT, GROUP, 2>(M, N, K, x, tiled, scales, y, warps, s);
    return gemv_launch<NT, GROUP, 1>(M, N, K, x, tiled, scales, y, warps, s);
}

template <int NT>
int gemv_group(int M, int N, int K, int group, const uint16_t *x, const uint8_t *tiled, const uint16_t *scales,
               float *y, const DeviceState &ds, cudaStream_t s) {
    if (group == 32) return gemv_rows<NT, 32>(M, N, K, x, tiled, scales, y, ds, s);
    if (group == 64) return gemv_rows<NT, 64>(M, N, K, x, tiled, scales, y, ds, s);
    return gemv_rows<NT, 128>(M, N, K, x, tiled, scales, y, ds, s);
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
    if (M <= 8) return gemv_group<1>(M, N, K, group, x, tiled, scales, y, ds, s);
    if (M <= 16) return gemv_group<2>(M, N, K, group, x, tiled, scales, y, ds, s);
    return gemv_group<4>(M, N, K, group, x, tiled, scales, y, ds, s);
}

}  // namespace isam
