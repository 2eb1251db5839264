// w4.cu -- products of a few tokens with 4-bit weights and group scales:
//   y[m][n] = sum_k x[m][k] s[n][k / group] (q[n][k] - 8).
#include <algorithm>

#include "internal.h"
#include "lm_common.cuh"
#include "mma_few.cuh"
#include "ptx.cuh"

namespace isam {

namespace {

constexpr int kThreads = 256;

// Nibble i of a code word holds k offset nibble_k(i): a mask of 0x000F000F on
// the word shifted right by 4 i leaves the neighbours 2 i and 2 i + 1.
__host__ __device__ constexpr int nibble_k(int i) { return i < 4 ? 2 * i : 2 * (i - 4) + 1; }

// One thread per 32-bit word of tiled codes.  Run once per matrix: 32001 x 8192
// with its scales 238 us, 1.2 TB/s, bound by byte loads of a row's neighbours.
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

constexpr int kTileBytes = 1024;  // codes of 16 rows x 128 k
constexpr int kMaxStages = 4;     // of a warp's ring
constexpr int kMaxSmem = 224 * 1024;
constexpr int kMostPer = 4;       // tiles of a warp in a stage

// Bulk copy of global memory into shared memory, counted on a barrier.
__device__ __forceinline__ void copy(uint32_t to, const void *from, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(to),
                 "l"(from), "r"(bytes), "r"(bar)
                 : "memory");
}

// The word's eight codes as four pairs of bf16 (q - 8) / 8, exactly, in the
// order of k.  A code in the low four bits of a half is or-ed into the mantissa
// of 16, where it counts eighths, and 17 is subtracted.  One in the next four
// bits needs no shift: read as a bf16 it is q 2^-129 (eight and above reach the
// lowest exponent, which has the spacing of the subnormals below it), and one
// fused multiply-add makes that q / 8 - 1.
__device__ __forceinline__ void dequant(uint32_t w, uint32_t (&v)[4]) {
#pragma unroll
    for (int i = 0; i < 4; i += 2, w >>= 8) {
        asm("lop3.b32 %0, %1, 0x000F000F, 0x41804180, 0xEA;" : "=r"(v[i]) : "r"(w));
        asm("fma.rn.bf16x2 %0, %0, %1, %2;" : "+r"(v[i]) : "r"(0x3F803F80u), "r"(0xC188C188u));
        asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(v[i + 1]) : "r"(w & 0x00F000F0u), "r"(0x7E807E80u), "r"(0xBF80BF80u));
    }
}

// The scales of a row in one tile: 128 / GROUP bf16.
template <int GROUP>
struct RowScales {
    static constexpr int kPer = 128 / GROUP;
    uint32_t w[(kPer + 1) / 2];
    __device__ __forceinline__ void load(uint32_t at) {
        if constexpr (kPer == 4) {
            asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at));
        } else if constexpr (kPer == 2) {
            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at));
        } else {
            uint16_t h;
            asm volatile("ld.shared.u16 %0, [%1];" : "=h"(h) : "r"(at));
            w[0] = h;
        }
    }
    __device__ __forceinline__ float get(int j) const {
        return __uint_as_float(j & 1 ? w[j / 2] & 0xffff0000u : w[j / 2] << 16);
    }
};

struct W4Params {
    int M, N, K;
    int kt;         // k tiles
    int groups;     // of 16 RB rows
    int team;       // warps that share the K of a group
    int per;        // k tiles of a warp in a stage
    int stages;     // of a team's ring
    int copies;     // of a team's sums: two save a barrier a group, one leaves more to the ring
    int x_stride;   // bytes of a token's row of x in shared memory
    const uint16_t *x;
    const uint8_t *tiled;
    const uint16_t *scales;
    float *y;
    unsigned long long timeout_ns;
    uint32_t *err;
};

template <int GROUP, int RB>
constexpr int tile_bytes() {
    return RB * (kTileBytes + 32 * (128 / GROUP));
}
// Words between tokens of a warp's sums: four more than rows, and a store touches
// every bank once.  (Two blocks of rows: their memory is better left to the L1 cache.)
template <int RB>
constexpr int part_step() {
    return RB == 1 ? 20 : 32;
}
template <int NT, int RB>
constexpr int part_bytes() {  // a warp's sums
    return 8 * NT * part_step<RB>() * 4;
}

// One CTA an SM.  A team of its warps takes 16 RB rows by 8 NT tokens at a time;
// its warps share K's tiles, `per` neighbours each in a stage, and their sums meet
// in shared memory, in the order of the warps.  A thread of a warp of its own
// brings a team's stage, the codes of team * per neighbouring tiles and their
// scales, by two bulk copies a block of rows, across groups of rows.  (Copies by
// each warp for itself took 130 instructions a stage beside a tile's 107.)  x is
// in shared memory as a whole where it fits (XS), rows 64 bytes off a multiple of
// 128 so that eight lanes' 16 bytes touch every bank once.
//
// Lane 4 r + t holds rows r and 8 + r of a tile, in word j the k of eight t of
// 32-block j.  The order of k inside a product does not matter, so the words'
// codes are operands of m16n8k16 as they lie, with the token's same eight k, 16
// bytes of x, beside them, and 16 k of one 32-block in each instruction: a scale
// applies to whole sums.
//
// Bound: reading the codes, and beside it the instructions that make them bf16
// (nine for eight codes) and scale sums.  32001 x 8192, groups of 32: one token
// 27.4 us, 5.4 TB/s, 0.79 of the copy bandwidth, eight 33.5 us, 0.65 (issue slots
// 60% full); 4096 x 4096, groups of 128, one token 4.4 us, a launch and one
// stage's latency.  More tokens leave less memory to the ring, and wait for shared
// memory and their sums: 16 x 57344 x 4096 39 us, 0.48; 32 x 57344 x 2048 43, 0.24.
template <int NT, int GROUP, int RB, bool XS, int WARPS>
__global__ void __launch_bounds__(32 * (WARPS + 1), 1) gemv_w4_kernel(const __grid_constant__ W4Params p) {
    constexpr int kPer = 128 / GROUP, kRows = 16 * RB, kStep = part_step<RB>(), kSize = part_bytes<NT, RB>() / 4;
    // Word blocks of one scale summed before it applies (all of a tile's would cost
    // registers where rows and tokens are many).
    constexpr int kSpan = RB * NT > 2 ? 1 : GROUP / 32;
    constexpr int kBlock = kTileBytes + 32 * kPer;  // codes and scales of one tile
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ uint64_t full[WARPS][kMaxStages], empty[WARPS][kMaxStages];  // of each team
    __shared__ int abort_flag;
    const int stages = XS ? p.stages : 2, copies = XS ? p.copies : 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int teams = WARPS / p.team, tiles = p.team * p.per;  // of a stage
    const int stage_bytes = tiles * RB * kBlock;
    uint8_t *xs = smem + WARPS * copies * part_bytes<NT, RB>() + teams * stages * stage_bytes;
    if (threadIdx.x < teams)
        for (int i = 0; i < stages; ++i) {
            mbar_init(&full[threadIdx.x][i], 1);
            mbar_init(&empty[threadIdx.x][i], p.team);
        }
    if (threadIdx.x == 0) abort_flag = 0;
    fence_mbar_init();
    __syncthreads();
    dependent_start();
    const WaitCtx wait{p.timeout_ns, p.err, &abort_flag};
    const int blocks = (p.N - 1) / 16 + 1;
    const int stride = teams * gridDim.x;  // groups: team t's are t * gridDim.x + blockIdx.x and every stride-th

    if (warp == WARPS) {
        // A stage: for each block of rows its tiles' codes, then their scales.
        if (lane == 0) {
            const uint32_t ring = smem_u32(smem + WARPS * copies * part_bytes<NT, RB>());
            int stage = 0;
            uint32_t phase = 1;
            bool ok = true;
            for (int g0 = blockIdx.x; ok && g0 < p.groups; g0 += stride)
                for (int k = 0; ok && k < p.kt; k += tiles) {
                    const uint32_t n = min(tiles, p.kt - k);
                    for (int team = 0; team < teams; ++team) {
                        const int g = g0 + team * gridDim.x;
                        if (g >= p.groups) break;
                        if (!bounded_wait(&empty[team][stage], phase, wait, 0x802u)) {
                            ok = false;
                            break;
                        }
                        const uint32_t bar = smem_u32(&full[team][stage]);
                        uint32_t to = ring + (team * stages + stage) * stage_bytes;
                        const int rows = RB == 1 ? 1 : min(RB, blocks - g * RB);
                        mbar_arrive_expect_tx(&full[team][stage], rows * n * kBlock);
                        for (int b = 0; b < rows; ++b) {
                            const int64_t tile = static_cast<int64_t>(g * RB + b) * p.kt + k;
                            copy(to, p.tiled + tile * kTileBytes, n * kTileBytes, bar);
                            copy(to + tiles * kTileBytes, p.scales + tile * 16 * kPer, n * 32 * kPer, bar);
                            to += tiles * kBlock;
                        }
                    }
                    if (++stage == stages) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
        }
        __syncwarp();
    } else {
        const int team = warp / p.team, member = warp - team * p.team;
        const uint32_t ring = smem_u32(smem + WARPS * copies * part_bytes<NT, RB>()) + team * stages * stage_bytes;
        float *part = reinterpret_cast<float *>(smem) + team * p.team * copies * kSize;
        const int r = lane >> 2, t = lane & 3;
        if (XS) {
            // x, and zeros behind K up to whole tiles.
            const int chunks = 16 * p.kt;  // of 16 bytes
            for (int i = threadIdx.x; i < p.M * chunks; i += 32 * WARPS) {
                const int m = i / chunks, c = i - m * chunks;
                uint8_t *to = xs + m * p.x_stride + 16 * c;
                if (8 * c < p.K)
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)),
                                 "l"(p.x + static_cast<int64_t>(m) * p.K + 8 * c)
                                 : "memory");
                else
                    *reinterpret_cast<uint4 *>(to) = make_uint4(0, 0, 0, 0);
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            named_bar(15, 32 * WARPS);
        }
        // A token's k of this lane (lanes behind the last token read it again).
        const uint16_t *xg[NT];
        uint32_t xa[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int m = min(8 * n + r, p.M - 1);
            xg[n] = p.x + static_cast<int64_t>(m) * p.K + 8 * t;
            xa[n] = smem_u32(xs) + m * p.x_stride + 16 * t;
        }
        int stage = 0, half = 0;
        uint32_t phase = 0;
        for (int g = team * gridDim.x + blockIdx.x; g < p.groups; g += stride, half ^= 1) {
            float sum[RB][NT][4] = {};
            for (int k0 = 0; k0 < p.kt; k0 += tiles) {
                const int k = member * p.per, n_tiles = min(p.per, p.kt - k0 - k);  // of the stage; below 1: none
                bounded_wait(&full[team][stage], phase, wait, 0x801u);
                uint32_t code_at = ring + stage * stage_bytes + k * kTileBytes + 16 * lane;
                uint32_t scale_at = ring + stage * stage_bytes + tiles * kTileBytes + k * 32 * kPer + 2 * kPer * r;
                const uint32_t code_end = code_at + max(n_tiles, 0) * kTileBytes;
                uint32_t x_at = 256u * static_cast<uint32_t>(k0 + k);  // bytes into a token's row, below 2^32
#pragma unroll 1
                for (; code_at != code_end; code_at += kTileBytes, scale_at += 32 * kPer, x_at += 256) {
                    uint4 code[RB][2];
                    RowScales<GROUP> scale[RB][2];
#pragma unroll
                    for (int b = 0; b < RB; ++b)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            code[b][h] = lds16(code_at + b * tiles * kBlock + 512 * h);
                            scale[b][h].load(scale_at + b * tiles * kBlock + 16 * kPer * h);
                        }
                    float acc[RB][NT][4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint4 xv[NT];
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            if (XS) {
                                xv[n] = lds16(xa[n] + x_at + 64 * j);
                            } else {
                                xv[n] = make_uint4(0, 0, 0, 0);
                                if (static_cast<int>(x_at / 2) + 32 * j + 8 * t < p.K)
                                    xv[n] = *reinterpret_cast<const uint4 *>(xg[n] + x_at / 2 + 32 * j);
                            }
                        }
#pragma unroll
                        for (int b = 0; b < RB; ++b) {
                            const auto word = [&](const uint4 &c) { return j == 0 ? c.x : j == 1 ? c.y : j == 2 ? c.z : c.w; };
                            uint32_t v[2][4];
                            dequant(word(code[b][0]), v[0]);
                            dequant(word(code[b][1]), v[1]);
                            const uint32_t a0[4] = {v[0][0], v[1][0], v[0][1], v[1][1]};
                            const uint32_t a1[4] = {v[0][2], v[1][2], v[0][3], v[1][3]};
#pragma unroll
                            for (int n = 0; n < NT; ++n) {
                                if (j % kSpan == 0)
                                    mma_16x8x16<true>(acc[b][n], a0, xv[n].x, xv[n].y);
                                else
                                    mma_16x8x16<false>(acc[b][n], a0, xv[n].x, xv[n].y);
                                mma_16x8x16<false>(acc[b][n], a1, xv[n].z, xv[n].w);
                            }
                            if ((j + 1) % kSpan == 0) {
                                const float lo = scale[b][0].get(j * 32 / GROUP), hi = scale[b][1].get(j * 32 / GROUP);
#pragma unroll
                                for (int n = 0; n < NT; ++n) {
                                    sum[b][n][0] = fmaf(lo, acc[b][n][0], sum[b][n][0]);
                                    sum[b][n][1] = fmaf(lo, acc[b][n][1], sum[b][n][1]);
                                    sum[b][n][2] = fmaf(hi, acc[b][n][2], sum[b][n][2]);
                                    sum[b][n][3] = fmaf(hi, acc[b][n][3], sum[b][n][3]);
                                }
                            }
                        }
                    }
                }
                __syncwarp();  // every lane has read the stage
                if (lane == 0) mbar_arrive(&empty[team][stage]);
                if (++stage == stages) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
            float *mine = part + (copies == 2 ? half * p.team * kSize : 0);
#pragma unroll
            for (int b = 0; b < RB; ++b)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        mine[member * kSize + (8 * n + 2 * t + (i & 1)) * kStep + 16 * b + r + 8 * (i >> 1)] = sum[b][n][i];
            const auto team_bar = [&]() {
                if (p.team == 1)
                    __syncwarp();
                else
                    named_bar(1 + team, 32 * p.team);
            };
            team_bar();
            for (int i = 32 * member + lane; i < kRows * 8 * NT; i += 32 * p.team) {
                const int m = i / kRows, row = i % kRows, n = g * kRows + row;
                if (m >= p.M || n >= p.N) continue;
                float v = 0.0f;
                for (int q = 0; q < p.team; ++q) v += mine[q * kSize + m * kStep + row];
                p.y[static_cast<int64_t>(m) * p.N + n] = 8.0f * v;  // (weights counted in eighths)
            }
            if (copies == 1) team_bar();  // the sums have been read
        }
    }
    if (*static_cast<volatile int *>(&abort_flag)) {  // copies in flight get time to land
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 50000ull) {
        }
    }
}

template <int NT, int GROUP, int RB, bool XS, int WARPS>
int gemv_launch(W4Params p, DeviceState &ds, cudaStream_t s) {
    static_assert(WARPS % 8 == 0, "teams of 8, 4, 2 and 1 warps share out a CTA's warps without rest");
    const auto fn = gemv_w4_kernel<NT, GROUP, RB, XS, WARPS>;
    const int rc = ensure_smem_optin(reinterpret_cast<const void *>(fn), kMaxSmem, ds.device,
                                     "cudaFuncSetAttribute(4-bit product)");
    if (rc) return rc;
    p.groups = (p.N - 1) / (16 * RB) + 1;
    const int grid = std::min(p.groups, ds.num_sms);
    // The whole CTA on one group where there are no more groups than SMs, else
    // teams of up to eight; no more warps than tiles.
    p.team = p.groups <= ds.num_sms ? WARPS : 8;
    while (p.team > p.kt) p.team = p.team > 8 ? 8 : p.team / 2;
    // Tiles of a warp in a stage: up to four, in at least two stages a group and two of
    // the ring, which has up to four (x from global memory: one, in two stages, as the
    // rest of the SM's memory caches x).  1, 2, 3, 4 at most, us: 1 x 32001 x 8192 40.3,
    // 28.3, 30.2, 27.5; 8 x 14336 x 4096 10.7, 10.0, 10.0, 10.0.  A group in one stage of
    // four took 8.9 for 8.4 on 1 x 14336 x 4096.
    const int x = XS ? p.x_stride * p.M : 0;
    const auto tiles = [&](int copies) {  // of a warp's ring
        return (kMaxSmem - x - WARPS * copies * part_bytes<NT, RB>()) / (WARPS * tile_bytes<GROUP, RB>());
    };
    p.copies = !XS || tiles(2) >= 4 ? 2 : 1;
    const int fit = tiles(p.copies);
    const int own = (p.kt + p.team - 1) / p.team;  // tiles of a warp in a group
    const int most = XS ? std::max(1, std::min({kMostPer, (own + 1) / 2, fit / 2})) : 1;
    const int visits = (p.kt + p.team * most - 1) / (p.team * most);
    p.per = (p.kt + p.team * visits - 1) / (p.team * visits);
    p.stages = XS ? std::min(kMaxStages, fit / p.per) : 2;
    const size_t smem = WARPS * (p.copies * part_bytes<NT, RB>() + p.stages * p.per * tile_bytes<GROUP, RB>()) + x;
    return launch_dependent(fn, dim3(grid), 32 * (WARPS + 1), smem, s, 1, "launch gemv_w4_kernel", p);
}

// x goes to shared memory where it leaves room for two tiles a warp, with 16 warps
// or (17 to 32 tokens) 8; else it is read through the L1 cache by a kernel whose
// two blocks of rows share what is read.
template <int NT, int GROUP, int WARPS>
bool x_fits(W4Params &p) {
    const int64_t stride = p.kt * int64_t{256} + 64;  // (above 32 bits from K = 2^30 on)
    const int64_t rest = WARPS * (2 * tile_bytes<GROUP, 1>() + part_bytes<NT, 1>());
    if (stride * p.M + rest > kMaxSmem) return false;
    p.x_stride = static_cast<int>(stride);
    return true;
}

// Measured, us, with (RB, warps): 16 x 14336 x 4096 (x fits) (1, 16) 13.0, (2, 8) 15.8;
// 16 x 8192 x 8192 (it does not) 25.9, 20.4; 32 x 14336 x 2048 (fits) (1, 16) 13.7, (1, 8)
// 15.5; 20 x 16384 x 4096 (fits 8 warps) (1, 8) 23.7, (2, 8) 37; 32 x 8192 x 8192 (does
// not) (1, 8) 43, (2, 8) 35.7, (2, 16) 52.
template <int NT, int GROUP>
int gemv_rows(W4Params p, DeviceState &ds, cudaStream_t s) {
    if (x_fits<NT, GROUP, 16>(p)) return gemv_launch<NT, GROUP, 1, true, 16>(p, ds, s);
    if constexpr (NT == 1) {
        return gemv_launch<NT, GROUP, 1, false, 16>(p, ds, s);
    } else {
        if constexpr (NT == 4)
            if (x_fits<NT, GROUP, 8>(p)) return gemv_launch<NT, GROUP, 1, true, 8>(p, ds, s);
        return gemv_launch<NT, GROUP, 2, false, 8>(p, ds, s);
    }
}

template <int NT>
int gemv_group(const W4Params &p, int group, DeviceState &ds, cudaStream_t s) {
    if (group == 32) return gemv_rows<NT, 32>(p, ds, s);
    if (group == 64) return gemv_rows<NT, 64>(p, ds, s);
    return gemv_rows<NT, 128>(p, ds, s);
}

}  // namespace

int w4_pack_launch(int N, int K, int group, const uint8_t *codes, const uint16_t *scales, uint8_t *tiled,
                   uint16_t *tiled_scales, cudaStream_t s) {
    const int nb = (N - 1) / 16 + 1, kt = (K - 1) / 128 + 1, per = 128 / group;
    const int64_t words = static_cast<int64_t>(nb) * kt * 256, count = static_cast<int64_t>(nb) * kt * 16 * per;
    w4_pack_codes_kernel<<<static_cast<unsigned>((words + kThreads - 1) / kThreads), kThreads, 0, s>>>(
        N, K, kt, words, codes, reinterpret_cast<uint32_t *>(tiled));
    const int rc = launch_status("launch w4_pack_codes_kernel");
    if (rc) return rc;
    w4_pack_scales_kernel<<<static_cast<unsigned>((count + kThreads - 1) / kThreads), kThreads, 0, s>>>(
        N, (K - 1) / group + 1, kt, per, count, scales, tiled_scales);
    return launch_status("launch w4_pack_scales_kernel");
}

int gemv_w4_launch(int M, int N, int K, int group, const uint16_t *x, const uint8_t *tiled, const uint16_t *scales,
                   float *y, DeviceState &ds, cudaStream_t s) {
    const W4Params p{M, N, K, (K - 1) / 128 + 1, 0, 0, 0, 0, 0, 0, x, tiled, scales, y, wait_timeout_ns(), ds.err_word};
    if (M <= 8) return gemv_group<1>(p, group, ds, s);
    if (M <= 16) return gemv_group<2>(p, group, ds, s);
    return gemv_group<4>(p, group, ds, s);
}

}  // namespace isam
