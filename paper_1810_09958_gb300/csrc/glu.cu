// glu.cu -- gated feed-forward product h = act(x Wg^T) * (x Wu^T), with
// W = [Wg; Wu] one [2F][D] matrix, and its backward pass.
//
// One kernel on pairs of SMs (tcgen05 cta_group::2) computes 256 x BN tiles in
// four roles.  PROJECT: A = x (256 tokens), B = BN/2 gate rows of W in the first
// CTA's shared memory and the same features' up rows in the second's, so one
// MMA gives both projections of a feature in one TMEM lane, BN/2 columns
// apart, and the epilogue forms act(g) u without either reaching memory.
// PROJECT_BACK: the same product, but the epilogue reads dh and writes
// d = [dh u act'(g) | dh act(g)] (g and u fp32; d is rounded to bf16 once, as an
// operand of the next products).  PRODUCT: dx = d W and dW = d^T x, bf16 out,
// A K-major or MN-major, B MN-major; the tiles that a last round would leave most
// pairs without are split over K, and a second kernel adds their fp32 parts in
// order (4096 x 2560 x 15360, 160 tiles on 76 pairs).  PRODUCT_FEW: dx for up to 128
// tokens with the roles changed, (W^T d^T), so that a stage is W and not empty
// token rows.
//
// Up to 32 tokens are a reading of W: glu_few_kernel streams 8 gate and 8 up rows
// at a time through m16n8k16, as long as x fits shared memory beside the rings: a D of
// up to 8832 at 8 tokens, 3904 at 16, 2240 at 20, 1408 at 32.  Beyond that the pair
// kernel runs with most of its 256 rows empty.
#include <algorithm>

#include "gemm_common.cuh"
#include "internal.h"
#include "lm_common.cuh"
#include "mma_few.cuh"
#include "ptx.cuh"

namespace isam {

namespace {

enum Role { PROJECT, PROJECT_BACK, PRODUCT, PRODUCT_FEW };

constexpr int kPM = 256;   // tile rows of a pair
constexpr int kHalf = 128; // rows of A in each CTA
constexpr int kBK = 64;
constexpr int kThreads = 192;
constexpr int kAStage = kHalf * kBK * 2;
constexpr int kStage = 4096;                  // 32 rows x 64 bf16 of a result, 128-byte swizzled
constexpr int kEpiBytes = 4 * 2 * kStage;     // two a warp
constexpr uint32_t kTmemCols = 512;           // two accumulators of up to 256 columns
constexpr uint16_t kBoth = 0x3;
constexpr int kGroupM = 8;  // tiles of a rasterisation group

enum : uint32_t {
    SITE_U_EMPTY = 0x701,
    SITE_U_FULL = 0x702,
    SITE_U_TEMPTY = 0x703,
    SITE_U_TFULL = 0x704,
    SITE_U_DONE = 0x705,
};

// B's columns in each CTA (BN / 2), padded to what MN-major loads bring.
constexpr int b_stage(int BN, bool B_MN) { return (B_MN ? (BN / 2 + 63) / 64 * 64 : BN / 2) * kBK * 2; }

struct GluParams {
    int T, F, N;       // tokens and features of a projection; N: columns of a product
    int64_t M;         // rows of the result
    int m_tiles, n_tiles, kb_total;
    int stages, group_m;
    int act;
    int tma_out;       // the result's rows are on 16-byte boundaries
    // Products: tiles from main_tiles on are computed in `splits` parts of kb_split
    // 64-wide blocks of K, to parts[part][tile - main_tiles][256][BN]; transposed
    // ones all are, to parts[part][N][M].
    int main_tiles, splits, kb_split;
    float *parts;
    uint16_t *out;     // h, or d
    const uint16_t *dh;
    unsigned long long timeout_ns;
    uint32_t *err;
};

__device__ __forceinline__ void tile_coords(int tile, const GluParams &p, int &mt, int &nt) {
    const int per_group = p.group_m * p.n_tiles;
    const int g = tile / per_group;
    const int first_m = g * p.group_m;
    const int gm = min(p.group_m, p.m_tiles - first_m);
    const int local = tile - g * per_group;
    mt = first_m + local % gm;
    nt = local / gm;
}

// ---- issue of the pair's MMAs.  A whole warp runs the loop and one elected lane
// issues, so that addresses stay in uniform registers, and a matrix descriptor is
// two words of which only the lower one changes: with 64-bit descriptors built by
// one lane, the issuing thread took 640 cycles a 64-deep block whatever the
// tile's width, more than the 512 of the MMAs of the widest.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "elect.sync _|q, 0xffffffff;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(p));
    return p != 0;
}

// The words of sdesc_sw128 (ptx.cuh): K-major operands 16 and MN-major ones 8192
// bytes between their chunks, 1024 between groups of eight rows or k.
constexpr uint32_t kDescHigh = (1024u >> 4) | (1u << 14) | (2u << 29);
__device__ __forceinline__ uint32_t desc_low(uint32_t saddr, bool mn) {
    return (saddr >> 4) | ((mn ? 8192u >> 4 : 16u >> 4) << 16);
}
__device__ __forceinline__ void umma_pair_words(uint32_t d_tmem, uint32_t a_low, uint32_t b_low, uint32_t idesc,
                                                uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .b64 a, b;\n\t"
        "setp.ne.b32 p, %5, 0;\n\t"
        "mov.b64 a, {%1, %4};\n\t"
        "mov.b64 b, {%2, %4};\n\t"
        "tcgen05.mma.cta_group::2.kind::f16 [%0], a, b, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_low), "r"(b_low), "r"(idesc), "r"(kDescHigh), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

// 32 gate and up sums of one token to packed bf16: h, or dg and du.
template <int ACT, bool BACK>
__device__ __forceinline__ void gate32(const uint32_t (&g)[32], const uint32_t (&u)[32], const uint32_t (&dh)[16],
                                       uint32_t (&a)[16], uint32_t (&b)[16]) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        float x[2], y[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float v, dv;
            const float up = __uint_as_float(u[2 * i + k]);
            activation<ACT>(__uint_as_float(g[2 * i + k]), v, dv);
            if (BACK) {
                const float d = __uint_as_float(k ? dh[i] & 0xffff0000u : dh[i] << 16);
                x[k] = d * up * dv;
                y[k] = d * v;
            } else {
                x[k] = v * up;
            }
        }
        a[i] = pack2(x[0], x[1]);
        if (BACK) b[i] = pack2(y[0], y[1]);
    }
}

template <bool BACK>
__device__ __forceinline__ void gate32(int act, const uint32_t (&g)[32], const uint32_t (&u)[32],
                                       const uint32_t (&dh)[16], uint32_t (&a)[16], uint32_t (&b)[16]) {
    if (act == ISAM_ACT_SILU)
        gate32<ISAM_ACT_SILU, BACK>(g, u, dh, a, b);
    else if (act == ISAM_ACT_GELU)
        gate32<ISAM_ACT_GELU, BACK>(g, u, dh, a, b);
    else if (act == ISAM_ACT_RELU)
        gate32<ISAM_ACT_RELU, BACK>(g, u, dh, a, b);
    else
        gate32<ISAM_ACT_SIGMOID, BACK>(g, u, dh, a, b);
}

// 32 packed values (64 bytes) of this lane's row into half `half` of a
// 32-row, 128-byte-swizzled staging tile.
__device__ __forceinline__ void stage32(uint8_t *tile, int lane, int half, const uint32_t (&a)[16]) {
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const int pos = (half * 4 + c) ^ (lane & 7);
        *reinterpret_cast<uint4 *>(tile + lane * 128 + pos * 16) =
            make_uint4(a[4 * c], a[4 * c + 1], a[4 * c + 2], a[4 * c + 3]);
    }
}

// One warp of each CTA issues TMA, one of the pair the MMAs, four read the
// accumulators (two of them, so that a tile's epilogue runs beside the next one's
// MMAs).  Both issuing warps stay whole and elect a lane at each instruction, with
// descriptors advanced as 32-bit words: from a single diverged thread a 64-deep
// block took 644 cycles at every width, more than its MMAs (8192 x 4096 x 8192
// 558 us, 200 x 1760 x 4096 13.8).  Bound by the tensor cores where tiles fill the
// GPU.  In short bursts 8192 x 4096 x 8192 forward 518 to 542 us, 1.03 to 1.07 of the
// measured bf16 burst, and 4096 x 2560 x 7680 backward, three launches of this kernel
// and one sum, 496 to 524 us (box to box), 0.93 to 0.99; in a stream of calls, under
// the power cap, 612 us and 580 to 590, 1.03 and 0.94 to 0.95 of the measured sustained rate
// (0.91 and 0.83 of the burst).  By the chain of first loads, one round of
// blocks and the epilogue where they do not: 200 x 1760 x 4096 11.5 us, 0.40 of
// reading its bytes.
template <Role ROLE, int BN, bool A_MN, bool B_MN>
__global__ void __launch_bounds__(kThreads, 1)
    glu_pair_kernel(const __grid_constant__ CUtensorMap tmA, const __grid_constant__ CUtensorMap tmB,
                    const __grid_constant__ CUtensorMap tmC, const __grid_constant__ CUtensorMap tmC2,
                    const __grid_constant__ GluParams p) {
    if (!launch_shape_ok(p.err, 2u, gridDim.x, 0x7F0u)) return;
    constexpr int kBHalf = BN / 2;
    constexpr int kBStage = b_stage(BN, B_MN);
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                                ~static_cast<uintptr_t>(1023));
    const int ST = p.stages;
    uint8_t *sA = smem;
    uint8_t *sB = smem + static_cast<size_t>(ST) * kAStage;
    uint8_t *ebuf = sB + static_cast<size_t>(ST) * kBStage;
    uint64_t *bars = reinterpret_cast<uint64_t *>(ebuf + kEpiBytes);
    uint64_t *full = bars;         // [ST] first CTA: both CTAs' copies of a stage landed
    uint64_t *empty = full + ST;   // [ST] both: the pair's MMAs have read the stage
    uint64_t *tfull = empty + ST;  // [2] both: accumulator complete
    uint64_t *tempty = tfull + 2;  // [2] first CTA: 8 epilogue warps released it
    uint64_t *done = tempty + 2;   // local epilogue warps finished with TMEM
    uint64_t *mq = done + 1;       // first CTA: all its MMAs complete
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(mq + 1);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 1);

    const int warp = threadIdx.x >> 5;
    const int lane = threadIdx.x & 31;
    const uint32_t rank = cluster_ctarank();
    const bool leader = rank == 0;
    const int pair = blockIdx.x >> 1;
    const int num_pairs = gridDim.x >> 1;
    const int split_tiles = p.m_tiles * p.n_tiles - p.main_tiles;
    const int num_tiles = p.main_tiles + split_tiles * p.splits;
    // Tile i of the list: its place, its blocks of K, and its part (-1: the whole).
    struct Item {
        int mt, nt, kb0, kb1, part, local;
    };
    const auto item = [&](int i) {
        Item t;
        t.part = -1, t.local = 0, t.kb0 = 0, t.kb1 = p.kb_total;
        int tile = i;
        if ((ROLE == PRODUCT || ROLE == PRODUCT_FEW) && i >= p.main_tiles) {
            t.part = (i - p.main_tiles) / split_tiles;
            t.local = (i - p.main_tiles) - t.part * split_tiles;
            t.kb0 = t.part * p.kb_split;
            t.kb1 = min(t.kb0 + p.kb_split, p.kb_total);
            tile = p.main_tiles + t.local;
        }
        tile_coords(tile, p, t.mt, t.nt);
        return t;
    };

    if (threadIdx.x == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(&full[i], 1);
            mbar_init(&empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&tfull[i], 1);
            mbar_init(&tempty[i], 8);
        }
        mbar_init(done, 4);
        mbar_init(mq, 1);
        *abort_flag = 0;
        fence_mbar_init();
        tma_prefetch_desc(&tmA);
        tma_prefetch_desc(&tmB);
    }
    __syncwarp();
    if (warp == 1) {
        tmem_alloc_pair(tmem_slot, kTmemCols);
        tmem_relinquish_pair();
    }
    tc_fence_before();
    __syncthreads();
    cluster_sync_all();  // both CTAs' barriers and TMEM exist before any cross-CTA traffic
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    const WaitCtx w{p.timeout_ns, p.err, abort_flag};

    griddep_launch_dependents();
    griddep_wait();

    bool aborted = false;
    if (warp == 0) {
        // ------------------------------------------------ TMA producer (both CTAs)
        const bool one = elect_one();
        int stage = 0;
        uint32_t phase = 0;
        bool ok = true;
        const uint32_t full_at = mapa_shared(smem_u32(full), 0u);
        for (int tile = pair; ok && tile < num_tiles; tile += num_pairs) {
            const Item it = item(tile);
            const int nt = it.nt;
            const int arow = it.mt * kPM + static_cast<int>(rank) * kHalf;
            // Projections: this CTA's rows of W are the tile's gate rows or its up rows.
            const int bcol = ROLE == PRODUCT || ROLE == PRODUCT_FEW ? nt * BN + static_cast<int>(rank) * kBHalf
                                                                    : nt * kBHalf + (leader ? 0 : p.F);
            for (int kb = it.kb0; kb < it.kb1; ++kb) {
                if (!warp_wait<true>(&empty[stage], phase ^ 1u, w, SITE_U_EMPTY)) {
                    ok = false;
                    break;
                }
                if (one) {
                    if (leader) mbar_arrive_expect_tx(&full[stage], 2u * (kAStage + kBStage));
                    const uint32_t fb = full_at + 8 * stage;
                    uint8_t *a = sA + stage * kAStage;
                    uint8_t *b = sB + stage * kBStage;
                    const int k0 = kb * kBK;
                    if (A_MN) {
                        tma_load_2d_pair(&tmA, fb, a, arow, k0);
                        tma_load_2d_pair(&tmA, fb, a + 8192, arow + 64, k0);
                    } else {
                        tma_load_2d_pair(&tmA, fb, a, k0, arow);
                    }
                    if (B_MN) {
#pragma unroll
                        for (int c = 0; c < kBHalf; c += 64) tma_load_2d_pair(&tmB, fb, b + c * 128, bcol + c, k0);
                    } else {
                        tma_load_2d_pair(&tmB, fb, b, k0, bcol);
                    }
                }
                if (++stage == ST) {
                    stage = 0;
                    phase ^= 1u;
                }
            }
        }
        aborted = !ok;
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------ MMA issuer (first CTA)
        if (leader) {
            const uint32_t idesc = idesc_bf16_f32(kPM, BN, A_MN, B_MN);
            const bool one = elect_one();
            constexpr uint32_t kStepA = (A_MN ? 2048 : 32) >> 4, kStepB = (B_MN ? 2048 : 32) >> 4;
            const uint32_t a_first = desc_low(smem_u32(sA), A_MN), b_first = desc_low(smem_u32(sB), B_MN);
            int stage = 0, acc = 0;
            uint32_t phase = 0, acc_phase = 0;
            bool ok = true, issued = false;
            for (int tile = pair; ok && tile < num_tiles; tile += num_pairs) {
                if (!warp_wait<true>(&tempty[acc], acc_phase ^ 1u, w, SITE_U_TEMPTY)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const uint32_t d = tmem_base + static_cast<uint32_t>(acc * 256);
                const Item it = item(tile);
                const int kbs = it.kb1 - it.kb0;
                for (int kb = 0; kb < kbs; ++kb) {
                    if (!warp_wait<true>(&full[stage], phase, w, SITE_U_FULL)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t a = a_first + stage * (kAStage >> 4), b = b_first + stage * (kBStage >> 4);
                    if (one) {
#pragma unroll
                        for (int k = 0; k < kBK / 16; ++k)
                            umma_pair_words(d, a + k * kStepA, b + k * kStepB, idesc, (kb > 0 || k > 0) ? 1u : 0u);
                        umma_commit_pair(&empty[stage], kBoth);
                    }
                    issued = true;
                    if (++stage == ST) {
                        stage = 0;
                        phase ^= 1u;
                    }
                }
                if (!ok) break;
                if (one) umma_commit_pair(&tfull[acc], kBoth);
                if (++acc == 2) {
                    acc = 0;
                    acc_phase ^= 1u;
                }
            }
            // Every MMA of this thread has completed before TMEM can be freed.
            if (issued && one) {
                umma_commit_pair(mq, 0x1);
                drain_wait(mq, 0, p.timeout_ns);
            }
            aborted = !ok;
        }
        __syncwarp();
    } else {
        // ------------------------------------------------ epilogue (warps 2-5, both CTAs)
        const int q = warp & 3;  // TMEM lane quadrant this warp may read
        uint8_t *stg = ebuf + (warp - 2) * 2 * kStage;
        int acc = 0, buf = 0;
        uint32_t acc_phase = 0;
        bool ok = true;
        for (int tile = pair; tile < num_tiles; tile += num_pairs) {
            const Item it = item(tile);
            const int nt = it.nt;
            const int row0 = it.mt * kPM + static_cast<int>(rank) * kHalf + q * 32;
            const int64_t row = row0 + lane;
            const uint32_t tb =
                tmem_base + (static_cast<uint32_t>(q * 32) << 16) + static_cast<uint32_t>(acc * 256);
            if constexpr (ROLE == PRODUCT_FEW) {
                if (!warp_wait<true>(&tfull[acc], acc_phase, w, SITE_U_TFULL)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                // Lanes are columns of dx, TMEM columns its tokens: 128 bytes a token and warp.
                float *at = p.parts + static_cast<int64_t>(it.part) * p.N * p.M + row;
#pragma unroll 1
                for (int j = 0; j < BN / 32; ++j) {
                    const int t0 = nt * BN + 32 * j;
                    if (row0 >= p.M || t0 >= p.N) break;
                    uint32_t r[32];
                    tmem_ld32(tb + j * 32, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int c = 0; c < 32; ++c)
                        if (row < p.M && t0 + c < p.N) at[(t0 + c) * p.M] = __uint_as_float(r[c]);
                }
            } else if constexpr (ROLE == PRODUCT) {
                if (!warp_wait<true>(&tfull[acc], acc_phase, w, SITE_U_TFULL)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
                const int col0 = nt * BN;
                if (it.part >= 0) {
                    // This part's sums, from registers (N is a multiple of 8).
                    float *at = p.parts + (static_cast<int64_t>(it.part) * split_tiles + it.local) * kPM * BN +
                                (row - it.mt * kPM) * BN;
#pragma unroll 1
                    for (int j = 0; j < BN / 32; ++j) {
                        if (row0 >= p.M || col0 + 32 * j >= p.N) break;
                        uint32_t r[32];
                        tmem_ld32(tb + j * 32, r);
                        tmem_ld_wait(r);
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            if (row < p.M && col0 + 32 * j + 4 * c < p.N)
                                *reinterpret_cast<uint4 *>(at + 32 * j + 4 * c) =
                                    make_uint4(r[4 * c], r[4 * c + 1], r[4 * c + 2], r[4 * c + 3]);
                    }
                } else
#pragma unroll 1
                for (int j = 0; j < BN / 64; ++j, buf ^= 1) {
                    if (lane == 0) bulk_wait_read<1>();  // the store of two chunks ago has left the tile
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        uint32_t r[32], a[16];
                        tmem_ld32(tb + j * 64 + h * 32, r);
                        tmem_ld_wait(r);
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            a[i] = pack2(__uint_as_float(r[2 * i]), __uint_as_float(r[2 * i + 1]));
                        stage32(stg + buf * kStage, lane, h, a);
                    }
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) {
                        if (row0 < p.M && col0 + j * 64 < p.N) tma_store_2d(&tmC, stg + buf * kStage, col0 + j * 64, row0);
                        bulk_commit();
                    }
                }
            } else {
                constexpr bool BACK = ROLE == PROJECT_BACK;
                const int f0 = nt * kBHalf;
                uint32_t dh[16] = {}, next[16] = {};
                const auto fetch = [&](int f) {  // 32 gradients of this lane's token (F is a multiple of 8)
                    if (!BACK) return;
                    const uint4 *at = reinterpret_cast<const uint4 *>(p.dh + row * p.F + f);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (row < p.T && f + 8 * c < p.F) v = __ldcs(at + c);
                        next[4 * c] = v.x, next[4 * c + 1] = v.y, next[4 * c + 2] = v.z, next[4 * c + 3] = v.w;
                    }
                };
                fetch(f0);
                if (!warp_wait<true>(&tfull[acc], acc_phase, w, SITE_U_TFULL)) {
                    ok = false;
                    break;
                }
                tc_fence_after();
#pragma unroll 1
                for (int j = 0; j < kBHalf / 32; ++j) {
                    const int f = f0 + j * 32;
                    uint32_t g[32], u[32], a[16], b[16];
                    tmem_ld32(tb + j * 32, g);
                    tmem_ld32(tb + kBHalf + j * 32, u);
#pragma unroll
                    for (int i = 0; i < 16; ++i) dh[i] = next[i];
                    if (j + 1 < kBHalf / 32) fetch(f + 32);
                    tmem_ld_wait(g);
                    tmem_ld_wait(u);
                    gate32<BACK>(p.act, g, u, dh, a, b);
                    if (kBHalf % 64 != 0 && p.tma_out) {
                        // A tile of 32 features: a row's 64 bytes go out by themselves.
                        if (row < p.T) {
                            uint16_t *at = p.out + row * (BACK ? 2 * static_cast<int64_t>(p.F) : p.F) + f;
#pragma unroll
                            for (int c = 0; c < 4; ++c)
                                if (f + 8 * c < p.F) {
                                    *reinterpret_cast<uint4 *>(at + 8 * c) =
                                        make_uint4(a[4 * c], a[4 * c + 1], a[4 * c + 2], a[4 * c + 3]);
                                    if (BACK)
                                        *reinterpret_cast<uint4 *>(at + p.F + 8 * c) =
                                            make_uint4(b[4 * c], b[4 * c + 1], b[4 * c + 2], b[4 * c + 3]);
                                }
                        }
                    } else if (p.tma_out) {
                        // PROJECT: two 64-column tiles in turn; PROJECT_BACK: dg in one, du in the other.
                        uint8_t *to = stg + (BACK ? 0 : buf * kStage);
                        if ((j & 1) == 0) {
                            if (lane == 0) {
                                if (BACK)
                                    bulk_wait_read<0>();
                                else
                                    bulk_wait_read<1>();
                            }
                            __syncwarp();
                        }
                        stage32(to, lane, j & 1, a);
                        if (BACK) stage32(to + kStage, lane, j & 1, b);
                        if (j & 1) {
                            fence_proxy_async_smem();
                            __syncwarp();
                            if (lane == 0) {
                                const int c = f - 32;
                                if (row0 < p.T && c < p.F) {
                                    tma_store_2d(&tmC, to, c, row0);
                                    if (BACK) tma_store_2d(&tmC2, to + kStage, c, row0);
                                }
                                bulk_commit();
                            }
                            buf ^= 1;
                        }
                    } else if (row < p.T) {
                        uint16_t *at = p.out + row * p.F + f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (f + 2 * i < p.F) at[2 * i] = static_cast<uint16_t>(a[i]);
                            if (f + 2 * i + 1 < p.F) at[2 * i + 1] = static_cast<uint16_t>(a[i] >> 16);
                        }
                    }
                }
            }
            // Release this accumulator on the first CTA's barrier.
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive_remote(&tempty[acc], 0u);
            __syncwarp();
            if (++acc == 2) {
                acc = 0;
                acc_phase ^= 1u;
            }
        }
        if (lane == 0) bulk_wait_all<0>();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(done);
        __syncwarp();
        aborted = !ok;
    }

    // ---- teardown.  After an abort, copies this CTA issued may still be in
    // flight towards its shared memory and complete on the first CTA's
    // barriers: give them time to land (bounded, only on that path).
    if (__syncthreads_or(aborted ? 1 : 0) && threadIdx.x == 0) {
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 50000ull) {
        }
    }
    if (warp == 1) bounded_wait(done, 0, w, SITE_U_DONE);
    __syncwarp();
    tc_fence_before();
    __syncthreads();
    // Both CTAs' epilogues are done reading TMEM and the first CTA's MMAs have
    // completed before the pair releases its TMEM together.
    cluster_sync_all();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc_pair(tmem_base, kTmemCols);
    }
}

size_t pair_smem(int stages, int bstage) {
    return 1024 + static_cast<size_t>(stages) * (kAStage + bstage) + kEpiBytes + (2 * stages + 6) * 8 + 16;
}

template <Role ROLE, int BN, bool A_MN, bool B_MN>
int pair_launch(GluParams p, const CUtensorMap &a, const CUtensorMap &b, const CUtensorMap &c, const CUtensorMap &c2,
                DeviceState &ds, cudaStream_t s) {
    const auto fn = glu_pair_kernel<ROLE, BN, A_MN, B_MN>;
    constexpr int bstage = b_stage(BN, B_MN);
    const int pairs = gemm_cluster_capacity(ds, 2);
    if (pairs < 1) return set_error(ISAM_ERR_UNSUPPORTED, "no pair of SMs is free for the gated feed-forward kernel");
    int st = 8;
    while (st > 2 && pair_smem(st, bstage) > static_cast<size_t>(ds.max_smem_optin)) --st;
    p.stages = st;
    p.group_m = kGroupM;
    p.timeout_ns = wait_timeout_ns();
    p.err = ds.err_word;
    const int64_t whole = static_cast<int64_t>(p.m_tiles) * p.n_tiles;
    const int64_t tiles = p.main_tiles + (whole - p.main_tiles) * p.splits;
    if (whole > 0x3fffffffLL || tiles > 0x7fffffffLL) return set_error(ISAM_ERR_UNSUPPORTED, "too many tiles for one launch");
    const int rc = ensure_smem_optin(reinterpret_cast<const void *>(fn), ds.max_smem_optin, ds.device,
                                     "cudaFuncSetAttribute(gated feed-forward)");
    if (rc) return rc;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = dim3(static_cast<unsigned>(2 * std::min<int64_t>(tiles, pairs)));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = pair_smem(st, bstage);
    cfg.stream = s;
    cfg.attrs = attr;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = 2;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, fn, a, b, c, c2, p);
    return e == cudaSuccess ? ISAM_OK : cuda_error(e, "launch glu_pair_kernel");
}

int tiles_of(int64_t n, int tile) { return static_cast<int>((n + tile - 1) / tile); }

template <Role ROLE, int BN>
int project_launch(const GluDesc &d, DeviceState &ds, cudaStream_t s) {
    GluParams p{};
    p.T = d.T, p.F = d.F, p.M = d.T, p.N = d.F, p.act = d.act, p.out = d.h, p.dh = d.dh;
    p.m_tiles = tiles_of(d.T, kPM);
    p.n_tiles = tiles_of(d.F, BN / 2);
    p.kb_total = tiles_of(d.D, kBK);
    p.splits = 1, p.kb_split = p.kb_total, p.main_tiles = p.m_tiles * p.n_tiles;
    CUtensorMap a{}, b{}, c{}, c2{};
    const uint64_t pitch = static_cast<uint64_t>(d.D) * 2, F = d.F;
    int rc;
    if ((rc = make_tmap_2d_bf16(&a, d.x, d.D, d.T, pitch, 64, kHalf))) return rc;
    if ((rc = make_tmap_2d_bf16(&b, d.W, d.D, 2 * F, pitch, 64, BN / 2))) return rc;
    if (ROLE == PROJECT_BACK) {
        uint16_t *ws = static_cast<uint16_t *>(d.workspace);
        p.tma_out = 1;
        p.out = ws;
        if ((rc = make_tmap_2d_bf16(&c, ws, F, d.T, 4 * F, 64, 32))) return rc;
        if ((rc = make_tmap_2d_bf16(&c2, ws + F, F, d.T, 4 * F, 64, 32))) return rc;
    } else if (F % 8 == 0 && reinterpret_cast<uintptr_t>(d.h) % 16 == 0) {
        p.tma_out = 1;
        if ((rc = make_tmap_2d_bf16(&c, d.h, F, d.T, 2 * F, 64, 32))) return rc;
    }
    return pair_launch<ROLE, BN, false, false>(p, a, b, c, c2, ds, s);
}

// 256 tokens x 128, 64 or 32 features a tile: a round of narrow tiles takes less
// time than one of wide ones, but not in proportion (a block's loads and issue
// cost the same), so they are taken where all of them are one round.  Measured,
// us at 32 / 64 / 128 features: 100 x 4096 x 1024 14.6 / 15.6 / 22.6, 200 x 1760 x
// 4096 14.6 / 11.2 / 14.1, 700 x 2560 x 3000 32 / 21 / 19, 2000 x 2560 x 7680 184 /
// 102 / 87.
template <Role ROLE>
int project(const GluDesc &d, DeviceState &ds, cudaStream_t s) {
    const int pairs = std::max(1, gemm_cluster_capacity(ds, 2));
    const int64_t mt = tiles_of(d.T, kPM);
    if (mt * tiles_of(d.F, 32) <= pairs) return project_launch<ROLE, 64>(d, ds, s);
    if (mt * tiles_of(d.F, 64) <= pairs) return project_launch<ROLE, 128>(d, ds, s);
    return project_launch<ROLE, 256>(d, ds, s);
}

// ---------------------------------------------------------------- few tokens
constexpr int kFewTokens = 32;
constexpr int kFewWarps = 16;
constexpr int kTeam = 8;          // warps that share the depth of a group of features
constexpr int kFewBlock = 2048;   // 64 deep: 8 gate and 8 up rows of 128 bytes
constexpr int kFewSmem = 220 * 1024;

struct FewParams {
    int T, D, F;
    int kb;        // 64-deep blocks of D
    int groups;    // of 8 features
    int stages, x_stride, act;
    const uint16_t *x;
    const uint16_t *dh;
    uint16_t *out;  // h [T][F], or d [T][2F]
    unsigned long long timeout_ns;
    uint32_t *err;
};

template <int NT>
constexpr int few_part() {  // a warp's sums, twice
    return 2 * 16 * 8 * NT * 4;
}

__device__ __forceinline__ float act_of(int act, float a, float &da) {
    float v;
    if (act == ISAM_ACT_SILU)
        activation<ISAM_ACT_SILU>(a, v, da);
    else if (act == ISAM_ACT_GELU)
        activation<ISAM_ACT_GELU>(a, v, da);
    else if (act == ISAM_ACT_RELU)
        activation<ISAM_ACT_RELU>(a, v, da);
    else
        activation<ISAM_ACT_SIGMOID>(a, v, da);
    return v;
}

// Both projections of 8 features at a time by a team of eight warps, two teams a
// CTA, one CTA an SM: rows 0-7 of an m16n8k16's A are gate rows, 8-15 the same
// features' up rows.  W arrives by TMA (boxes of 8 rows x 64, 128-byte swizzled)
// into a ring a warp, across groups; a warp's blocks are every eighth of D's, and
// the team's sums meet in shared memory in the order of the warps.  x is in
// shared memory as a whole, rows 64 bytes off a multiple of 128.  The order of k
// inside a product does not matter: lane 4 r + t holds eight consecutive k of rows
// r and 8 + r, and of token r, sixteen bytes each, which are two instructions'
// operands.  Bound by reading W: 1 x 2560 x 7680 16.0 us, 4.9 TB/s, 0.72 of the copy
// bandwidth (960 groups on 304 teams leave a part round), 1 x 5120 x 13824 44.4 us,
// 0.94; 16 tokens 2560 x 7680 17.4 us.
template <int NT, bool BACK>
__global__ void __launch_bounds__(32 * kFewWarps, 1)
    glu_few_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ FewParams p) {
    constexpr int kSize = 16 * 8 * NT;
    extern __shared__ uint8_t smem_raw[];
    __shared__ uint64_t full_all[kFewWarps][8];
    __shared__ int abort_flag;
    uint8_t *smem =
        reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int team = warp / kTeam, member = warp % kTeam;
    uint8_t *ring = smem + warp * p.stages * kFewBlock;
    float *part = reinterpret_cast<float *>(smem + kFewWarps * p.stages * kFewBlock) + team * kTeam * 2 * kSize;
    uint8_t *xs = smem + kFewWarps * (p.stages * kFewBlock + few_part<NT>());
    uint64_t *full = full_all[warp];
    if (lane == 0)
        for (int i = 0; i < p.stages; ++i) mbar_init(&full[i], 1);
    if (threadIdx.x == 0) {
        abort_flag = 0;
        tma_prefetch_desc(&tmW);
    }
    fence_mbar_init();
    __syncthreads();
    dependent_start();
    const WaitCtx wait{p.timeout_ns, p.err, &abort_flag};
    const int r = lane >> 2, t = lane & 3;
    constexpr int kTeams = kFewWarps / kTeam;
    const int first = team * gridDim.x + blockIdx.x, stride = kTeams * gridDim.x;

    int load_group = first, load_k = member, load_stage = 0;
    const auto fetch = [&]() {  // lane 0
        if (load_k >= p.kb) {
            load_k = member;
            load_group += stride;
        }
        if (load_group >= p.groups || load_k >= p.kb) return;
        uint64_t *bar = &full[load_stage];
        uint8_t *to = ring + load_stage * kFewBlock;
        mbar_arrive_expect_tx(bar, kFewBlock);
        tma_load_2d(&tmW, bar, to, load_k * 64, load_group * 8);
        tma_load_2d(&tmW, bar, to + kFewBlock / 2, load_k * 64, p.F + load_group * 8);
        load_k += kTeam;
        load_stage = load_stage + 1 == p.stages ? 0 : load_stage + 1;
    };
    if (lane == 0)
        for (int i = 0; i < p.stages; ++i) fetch();
    {
        // x, and zeros behind D up to whole blocks.
        const int chunks = 8 * p.kb;  // of 16 bytes
        for (int i = threadIdx.x; i < p.T * chunks; i += 32 * kFewWarps) {
            const int m = i / chunks, c = i - m * chunks;
            uint8_t *to = xs + m * p.x_stride + 16 * c;
            if (8 * c < p.D)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(to)),
                             "l"(p.x + static_cast<int64_t>(m) * p.D + 8 * c)
                             : "memory");
            else
                *reinterpret_cast<uint4 *>(to) = make_uint4(0, 0, 0, 0);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
    }
    uint32_t xa[NT];  // (lanes behind the last token read it again)
#pragma unroll
    for (int n = 0; n < NT; ++n) xa[n] = smem_u32(xs) + min(8 * n + r, p.T - 1) * p.x_stride + 16 * t;
    const uint32_t ring_at = smem_u32(ring) + 128 * r;
    int stage = 0, half = 0;
    uint32_t phase = 0;
    for (int g = first; g < p.groups; g += stride, half ^= 1) {
        float sum[NT][4] = {};
        for (int k = member; k < p.kb; k += kTeam) {
            bounded_wait(&full[stage], phase, wait, 0x711u);
            const uint32_t at = ring_at + stage * kFewBlock;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t chunk = 16 * ((4 * j + t) ^ r);
                const uint4 gate = lds16(at + chunk), up = lds16(at + kFewBlock / 2 + chunk);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    const uint4 xv = lds16(xa[n] + 128 * k + 64 * j);
                    const uint32_t a0[4] = {gate.x, up.x, gate.y, up.y}, a1[4] = {gate.z, up.z, gate.w, up.w};
                    mma_16x8x16<false>(sum[n], a0, xv.x, xv.y);
                    mma_16x8x16<false>(sum[n], a1, xv.z, xv.w);
                }
            }
            __syncwarp();  // every lane has read the stage
            if (lane == 0) fetch();
            if (++stage == p.stages) {
                stage = 0;
                phase ^= 1u;
            }
        }
        float *mine = part + half * kTeam * kSize;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                mine[member * kSize + (8 * n + 2 * t + (i & 1)) * 16 + r + 8 * (i >> 1)] = sum[n][i];
        named_bar(1 + team, 32 * kTeam);
        for (int i = 32 * member + lane; i < 8 * 8 * NT; i += 32 * kTeam) {
            const int m = i >> 3, f = g * 8 + (i & 7);
            if (m >= p.T || f >= p.F) continue;
            float a = 0.0f, u = 0.0f, da;
            for (int q = 0; q < kTeam; ++q) {
                a += mine[q * kSize + 16 * m + (i & 7)];
                u += mine[q * kSize + 16 * m + 8 + (i & 7)];
            }
            const float v = act_of(p.act, a, da);
            bf16 *out = reinterpret_cast<bf16 *>(p.out);
            if (BACK) {
                const float d = __uint_as_float(static_cast<uint32_t>(p.dh[static_cast<int64_t>(m) * p.F + f]) << 16);
                bf16 *row = out + static_cast<int64_t>(m) * 2 * p.F + f;
                row[0] = from_f32<bf16>(d * u * da);
                row[p.F] = from_f32<bf16>(d * v);
            } else {
                out[static_cast<int64_t>(m) * p.F + f] = from_f32<bf16>(v * u);
            }
        }
    }
    if (*static_cast<volatile int *>(&abort_flag)) {  // copies in flight get time to land
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 50000ull) {
        }
    }
}

// Stages of a warp's ring beside x, 0 where x does not fit.  Three already hold
// 96 KB an SM in flight, and more spread the reads over more of memory at once:
// 2 / 3 / 4 stages 17.2 / 16.1 / 16.3 us (1 x 2560 x 7680), 46.7 / 44.4 / 53.9
// (1 x 5120 x 13824).
template <int NT>
int few_stages(int T, int D) {
    const int64_t x = (tiles_of(D, kBK) * int64_t{128} + 64) * T;
    const int64_t left = kFewSmem - 1024 - x - kFewWarps * few_part<NT>();
    const int64_t st = left / (kFewWarps * kFewBlock);
    return st < 2 ? 0 : static_cast<int>(std::min<int64_t>(st, 3));
}

template <int NT, bool BACK>
int few_launch(const GluDesc &d, int stages, DeviceState &ds, cudaStream_t s) {
    const auto fn = glu_few_kernel<NT, BACK>;
    FewParams p{};
    p.T = d.T, p.D = d.D, p.F = d.F, p.act = d.act;
    p.kb = tiles_of(d.D, kBK);
    p.groups = tiles_of(d.F, 8);
    p.stages = stages;
    p.x_stride = p.kb * 128 + 64;
    p.x = d.x, p.dh = d.dh, p.out = BACK ? static_cast<uint16_t *>(d.workspace) : d.h;
    p.timeout_ns = wait_timeout_ns();
    p.err = ds.err_word;
    CUtensorMap w;
    int rc = make_tmap_2d_bf16(&w, d.W, d.D, 2 * static_cast<uint64_t>(d.F), static_cast<uint64_t>(d.D) * 2, 64, 8);
    if (rc) return rc;
    if ((rc = ensure_smem_optin(reinterpret_cast<const void *>(fn), kFewSmem, ds.device,
                                "cudaFuncSetAttribute(gated feed-forward, few tokens)")))
        return rc;
    const size_t smem = 1024 + kFewWarps * (stages * kFewBlock + few_part<NT>()) + static_cast<size_t>(p.x_stride) * d.T;
    return launch_dependent(fn, dim3(std::min(p.groups, ds.num_sms)), 32 * kFewWarps, smem, s, 1,
                            "launch glu_few_kernel", w, p);
}

// The projections and their gate: h, or d into the workspace.
template <Role ROLE>
int gated(const GluDesc &d, DeviceState &ds, cudaStream_t s) {
    constexpr bool BACK = ROLE == PROJECT_BACK;
    int st;
    if (d.T <= 8 && (st = few_stages<1>(d.T, d.D))) return few_launch<1, BACK>(d, st, ds, s);
    if (d.T > 8 && d.T <= 16 && (st = few_stages<2>(d.T, d.D))) return few_launch<2, BACK>(d, st, ds, s);
    if (d.T > 16 && d.T <= kFewTokens && (st = few_stages<4>(d.T, d.D))) return few_launch<4, BACK>(d, st, ds, s);
    return project<ROLE>(d, ds, s);
}

// ---------------------------------------------------------------- products
constexpr int kPairs = 76;  // of a GB300; the workspace's size does not ask the device
constexpr int kMaxSplits = 16;
constexpr int kFewColumns = 128;  // tokens of dx's transposed product
constexpr int kOneTokens = 4, kOuterTokens = 32;  // most tokens of dW as sums of outer products
constexpr int kSumThreads = 256;

// How a product M x N over K is cut: tile width, whole tiles, parts of the others.
struct Cut {
    int width, main_tiles, tail_tiles, splits, kb_split;
    size_t part_bytes() const {
        return splits > 1 ? static_cast<size_t>(splits) * tail_tiles * kPM * width * sizeof(float) : 0;
    }
};

// Estimated time, ns: a 64-wide block of K takes a pair 270, 215 or 165 at widths
// 256, 192 and 128 (the wide one is the tensor cores' rate, the narrow ones the
// issuing threads'), a round of tiles 800 beside its blocks, and parts 4500 (their
// sums are a kernel of their own).  A last round with less than half the pairs
// busy may be split over K.  Measured against this choice, dx with its
// projections, us at 128 / 192 / 256 whole and as chosen: 360 x 920 x 1744 17.6 /
// 19.8 / 20.2 and 17.6; 200 x 1760 x 8192 37 / 41 / 50 and 30; 4096 x 2560 x 15360
// 395 / 358 / 386 and 345.
Cut cut_product(int64_t M, int N, int64_t K) {
    const int kb = tiles_of(K, kBK);
    constexpr int64_t kRound = 800, kParts = 4500;
    Cut best{};
    int64_t best_cost = 0;
    const int64_t block_ns[3] = {270, 215, 165};
    for (int i = 0; i < 3; ++i) {
        const int width = 256 - 64 * i;
        const int64_t tiles = static_cast<int64_t>(tiles_of(M, kPM)) * tiles_of(N, width);
        const int64_t rest = tiles % kPairs, whole = kb * block_ns[i] + kRound;
        Cut c{width, static_cast<int>(std::min<int64_t>(tiles, 0x3fffffff)), 0, 1, kb};
        int64_t cost = (tiles + kPairs - 1) / kPairs * whole;
        const int splits = rest ? static_cast<int>(std::min<int64_t>({kPairs / rest, kMaxSplits, kb / 8})) : 1;
        if (splits > 1) {
            const int kb_split = tiles_of(kb, splits);
            const int64_t split_cost = tiles / kPairs * whole + kb_split * block_ns[i] + kRound + kParts;
            if (split_cost < cost) {
                cost = split_cost;
                c = Cut{width, static_cast<int>(tiles - rest), static_cast<int>(rest), tiles_of(kb, kb_split), kb_split};
            }
        }
        if (best.width == 0 || cost < best_cost) {
            best = c;
            best_cost = cost;
        }
    }
    return best;
}

__device__ __forceinline__ float4 sum_parts(const float4 *at, int64_t step, int splits) {
    float4 v = *at;
#pragma unroll 4
    for (int q = 1; q < splits; ++q) {
        const float4 w = at[q * step];
        v.x += w.x, v.y += w.y, v.z += w.z, v.w += w.w;
    }
    return v;
}

// The split tiles' parts added in order, to bf16: four columns a thread.  Bound by
// reading the parts from L2 (2048 x 2560 of K 15360: 8.7 us under a profiler).
__global__ void __launch_bounds__(kSumThreads)
    glu_sum_tiles_kernel(const __grid_constant__ GluParams p, int width, uint16_t *out) {
    dependent_start();
    const int tiles = p.m_tiles * p.n_tiles - p.main_tiles, per_row = width / 4;
    const int i = blockIdx.x * kSumThreads + threadIdx.x;
    const int local = i / (kPM * per_row), in = i - local * (kPM * per_row);
    const int r = in / per_row, c = 4 * (in - r * per_row);
    if (local >= tiles) return;
    int mt, nt;
    tile_coords(p.main_tiles + local, p, mt, nt);
    const int64_t row = static_cast<int64_t>(mt) * kPM + r;
    const int col = nt * width + c;
    if (row >= p.M || col >= p.N) return;  // (N is a multiple of 8)
    const float4 v = sum_parts(reinterpret_cast<const float4 *>(p.parts) + i, static_cast<int64_t>(tiles) * kPM * per_row,
                               p.splits);
    *reinterpret_cast<uint2 *>(out + row * p.N + col) = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}

// parts [splits][quads * 4] added in order, to bf16 (bound by its launch: at most
// 128 rows).
__global__ void __launch_bounds__(kSumThreads) glu_sum_kernel(int64_t quads, int splits, const float4 *parts, uint2 *out) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kSumThreads + threadIdx.x;
    if (i >= quads) return;
    dependent_start();
    const float4 v = sum_parts(parts + i, quads, splits);
    out[i] = make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
}

// C (M x N, bf16) = op(A) B with B K x N; A_MN: A stored K x M.
template <bool A_MN, int BN>
int product_launch(int64_t M, int N, int64_t K, const uint16_t *A, const uint16_t *B, uint16_t *C, const Cut &cut,
                   float *parts, DeviceState &ds, cudaStream_t s) {
    GluParams p{};
    p.M = M, p.N = N;
    p.m_tiles = tiles_of(M, kPM);
    p.n_tiles = tiles_of(N, BN);
    p.kb_total = tiles_of(K, kBK);
    p.main_tiles = cut.main_tiles, p.splits = cut.splits, p.kb_split = cut.kb_split;
    p.parts = parts;
    CUtensorMap a{}, b{}, c{};
    int rc;
    rc = A_MN ? make_tmap_2d_bf16(&a, A, M, K, M * 2, 64, kBK) : make_tmap_2d_bf16(&a, A, K, M, K * 2, 64, kHalf);
    if (rc) return rc;
    if ((rc = make_tmap_2d_bf16(&b, B, N, K, static_cast<uint64_t>(N) * 2, 64, kBK))) return rc;
    if ((rc = make_tmap_2d_bf16(&c, C, N, M, static_cast<uint64_t>(N) * 2, 64, 32))) return rc;
    if ((rc = pair_launch<PRODUCT, BN, A_MN, true>(p, a, b, c, c, ds, s))) return rc;
    if (p.splits == 1) return ISAM_OK;
    p.group_m = kGroupM;
    const int quads = cut.tail_tiles * kPM * BN / 4;  // below 76 tiles
    return launch_dependent(glu_sum_tiles_kernel, dim3(tiles_of(quads, kSumThreads)), kSumThreads, 0, s, 1,
                            "launch glu_sum_tiles_kernel", p, BN, C);
}

template <bool A_MN>
int product(int64_t M, int N, int64_t K, const uint16_t *A, const uint16_t *B, uint16_t *C, float *parts,
            DeviceState &ds, cudaStream_t s) {
    const Cut cut = cut_product(M, N, K);
    if (cut.width == 128) return product_launch<A_MN, 128>(M, N, K, A, B, C, cut, parts, ds, s);
    if (cut.width == 192) return product_launch<A_MN, 192>(M, N, K, A, B, C, cut, parts, ds, s);
    return product_launch<A_MN, 256>(M, N, K, A, B, C, cut, parts, ds, s);
}

// dx^T = W^T d^T for few tokens: parts of K for every pair of SMs.
int few_splits(int D, int64_t K) {
    const int tiles = tiles_of(D, kPM);
    return static_cast<int>(std::max<int64_t>(1, std::min<int64_t>({kPairs / tiles, kMaxSplits, tiles_of(K, kBK) / 8})));
}

template <int BN>
int few_product_launch(const GluDesc &d, const uint16_t *dg, float *parts, DeviceState &ds, cudaStream_t s) {
    const int64_t K = 2 * static_cast<int64_t>(d.F);
    GluParams p{};
    p.M = d.D, p.N = d.T;
    p.m_tiles = tiles_of(d.D, kPM);
    p.n_tiles = 1;
    p.kb_total = tiles_of(K, kBK);
    p.main_tiles = 0;
    p.kb_split = tiles_of(p.kb_total, few_splits(d.D, K));
    p.splits = tiles_of(p.kb_total, p.kb_split);
    p.parts = parts;
    CUtensorMap a{}, b{};
    int rc;
    if ((rc = make_tmap_2d_bf16(&a, d.W, d.D, K, static_cast<uint64_t>(d.D) * 2, 64, kBK))) return rc;
    if ((rc = make_tmap_2d_bf16(&b, dg, K, d.T, K * 2, 64, BN / 2))) return rc;
    if ((rc = pair_launch<PRODUCT_FEW, BN, true, false>(p, a, b, b, b, ds, s))) return rc;
    const int64_t quads = static_cast<int64_t>(d.T) * d.D / 4;
    return launch_dependent(glu_sum_kernel, dim3(tiles_of(quads, kSumThreads)), kSumThreads, 0, s, 1,
                            "launch glu_sum_kernel", quads, p.splits, reinterpret_cast<const float4 *>(parts),
                            reinterpret_cast<uint2 *>(d.dx));
}

// dW for up to four tokens, bound by writing dW: a sum of T outer products in
// registers.  A thread has eight columns of eight rows; a token's eight x and its
// eight d (the same for the whole block) make 64 products, two a packed
// instruction.  1 x 2560 x 7680: 18.2 us, what filling 79 MB takes (20).
constexpr int kOneThreads = 128, kOneRows = 8;
__global__ void __launch_bounds__(kOneThreads)
    glu_outer_few_kernel(int T, int D, int64_t F2, const uint16_t *d, const uint16_t *x, uint16_t *dW) {
    const int64_t row0 = static_cast<int64_t>(blockIdx.x) * kOneRows;
    const int col = static_cast<int>((blockIdx.z * gridDim.y + blockIdx.y) * kOneThreads + threadIdx.x) * 8;
    if (col >= D) return;
    dependent_start();
    unsigned long long sum[kOneRows][4] = {};
#pragma unroll 4
    for (int t = 0; t < T; ++t) {
        const uint4 xv = *reinterpret_cast<const uint4 *>(x + static_cast<int64_t>(t) * D + col);
        const uint4 dv = *reinterpret_cast<const uint4 *>(d + t * F2 + row0);  // 2F is a multiple of 16
        const uint32_t xw[4] = {xv.x, xv.y, xv.z, xv.w}, dw[4] = {dv.x, dv.y, dv.z, dv.w};
        unsigned long long xp[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            asm("mov.b64 %0, {%1, %2};" : "=l"(xp[i]) : "r"(xw[i] << 16), "r"(xw[i] & 0xffff0000u));
#pragma unroll
        for (int r = 0; r < kOneRows; ++r) {
            const uint32_t v = r & 1 ? dw[r / 2] & 0xffff0000u : dw[r / 2] << 16;
            unsigned long long dd;
            asm("mov.b64 %0, {%1, %1};" : "=l"(dd) : "r"(v));
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(sum[r][i]) : "l"(dd), "l"(xp[i]));
        }
    }
#pragma unroll
    for (int r = 0; r < kOneRows; ++r) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float lo, hi;
            asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(sum[r][i]));
            w[i] = pack2(lo, hi);
        }
        __stcs(reinterpret_cast<uint4 *>(dW + (row0 + r) * D + col), make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// dW for 5 to 32 tokens, bound by writing dW: m16n8k16 on tiles of 16 features x 512
// columns, whose tokens are all in shared memory (four CTAs an SM write while
// others load).  Both operands have tokens outside, so their fragments are
// transposed loads; a token's chunks of 16 bytes are rotated by its number, so that
// eight tokens' touch every bank once.  Rounded to bf16 once, results leave through
// shared memory, half a kilobyte of a row an instruction.  2560 x 7680, us, here /
// sums in registers / SM pairs: 4 tokens 25.0 / 21.5 / 27.7, 8 tokens 24.6 / 27.8 /
// 27.7, 16 tokens 24.6 / 42 / 27.7, 32 tokens 29.7 / - / 27.2; 512 x 1024 1.8 / 1.6 /
// 3.6, 1.8 / 2.5 / 3.5, 2.3 / 4.2 / 3.9, 3.4 / - / 3.7.
constexpr int kOuterThreads = 256, kOuterF = 16, kOuterCols = 512;
constexpr int outer_smem(int T) { return (T + 15) / 16 * 16 * 2 * (kOuterF + kOuterCols) + 8 * kOuterF * 128; }
__global__ void __launch_bounds__(kOuterThreads, 4)
    glu_outer_kernel(int T, int D, int64_t F2, int tile_cols, const uint16_t *d, const uint16_t *x, uint16_t *dW) {
    extern __shared__ __align__(128) uint8_t outer_raw[];
    constexpr int kX = 2 * kOuterCols, kD = 2 * kOuterF;  // bytes of a token
    const int tokens = (T + 15) & ~15;
    const uint32_t xs = smem_u32(outer_raw), ds = xs + tokens * kX;
    const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
    uint8_t *results = outer_raw + tokens * (kX + kD);  // [8 warps][16 features][64 columns]
    const uint32_t ft = blockIdx.x / tile_cols;
    const int64_t f0 = static_cast<int64_t>(ft) * kOuterF;
    const int c0 = static_cast<int>(blockIdx.x - ft * tile_cols) * kOuterCols;
    const auto bring = [&](uint32_t to, const uint16_t *from, bool in) {
        if (in)
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
        else
            asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(to), "r"(0u) : "memory");
    };
    dependent_start();
    for (int i = threadIdx.x; i < tokens * (kX / 16); i += kOuterThreads) {
        const int t = i / (kX / 16), c = i % (kX / 16);
        bring(xs + t * kX + 16 * (c ^ (t & 7)), x + static_cast<int64_t>(t) * D + c0 + 8 * c, t < T && c0 + 8 * c < D);
    }
    for (int i = threadIdx.x; i < tokens * (kD / 16); i += kOuterThreads) {  // (2F is a multiple of 16)
        const int t = i / (kD / 16), c = i % (kD / 16);
        bring(ds + t * kD + 16 * (c ^ (t / 4 & 1)), d + t * F2 + f0 + 8 * c, t < T);
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    const int at = lane & 7, hi = lane >> 4, lo = (lane >> 3) & 1;
    float sum[8][4] = {};
    for (int t = 0; t < tokens; t += 16) {
        uint32_t a[4], b[4];
        // Blocks: features lo, tokens hi; tokens lo, columns hi.
        ldmatrix4_trans(a, ds + (t + 8 * hi + at) * kD + 16 * (lo ^ (at / 4)));
#pragma unroll
        for (int n = 0; n < 8; n += 2) {
            ldmatrix4_trans(b, xs + (t + 8 * lo + at) * kX + 16 * ((8 * warp + n + hi) ^ at));
            mma_16x8x16<false>(sum[n], a, b[0], b[1]);
            mma_16x8x16<false>(sum[n + 1], a, b[2], b[3]);
        }
    }
    const int r = lane / 4, q = lane % 4;
#pragma unroll
    for (int n = 0; n < 8; ++n)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            *reinterpret_cast<uint32_t *>(results + (warp * kOuterF + 8 * h + r) * 128 + 16 * (n ^ r) + 4 * q) =
                pack2(sum[n][2 * h], sum[n][2 * h + 1]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOuterF / 4; ++i) {
        const int row = i / 2 * 8 + warp, w = i % 2 * 4 + lane / 8, c = c0 + 64 * w + 8 * (lane % 8);
        const uint4 v = *reinterpret_cast<const uint4 *>(results + (w * kOuterF + row) * 128 + 16 * ((lane % 8) ^ (row & 7)));
        if (c < D) __stcs(reinterpret_cast<uint4 *>(dW + (f0 + row) * D + c), v);
    }
}

// Bytes of d in the workspace, up to where the products' parts follow.
size_t d_bytes(int T, int F) { return (static_cast<size_t>(T) * F * 4 + 255) / 256 * 256; }

}  // namespace

int glu_forward_launch(const GluDesc &d, DeviceState &ds, cudaStream_t s) { return gated<PROJECT>(d, ds, s); }

size_t glu_backward_workspace(int T, int D, int F) {
    const int64_t F2 = 2 * static_cast<int64_t>(F);
    const size_t dx = T <= kFewColumns ? static_cast<size_t>(few_splits(D, F2)) * T * D * sizeof(float)
                                       : cut_product(T, D, F2).part_bytes();
    const size_t dW = T <= kOuterTokens ? 0 : cut_product(F2, D, T).part_bytes();
    return d_bytes(T, F) + std::max(dx, dW);
}

int glu_backward_launch(const GluDesc &d, DeviceState &ds, cudaStream_t s) {
    if (!d.dx && !d.dW) return ISAM_OK;
    int rc = gated<PROJECT_BACK>(d, ds, s);
    if (rc) return rc;
    const uint16_t *dg = static_cast<const uint16_t *>(d.workspace);
    float *parts = reinterpret_cast<float *>(static_cast<uint8_t *>(d.workspace) + d_bytes(d.T, d.F));
    const int64_t F2 = 2 * static_cast<int64_t>(d.F);
    if (d.dx) {
        rc = d.T <= 32            ? few_product_launch<32>(d, dg, parts, ds, s)
             : d.T <= 64          ? few_product_launch<64>(d, dg, parts, ds, s)
             : d.T <= kFewColumns ? few_product_launch<128>(d, dg, parts, ds, s)
                                  : product<false>(d.T, d.D, F2, dg, d.W, d.dx, parts, ds, s);
        if (rc) return rc;
    }
    if (d.dW && d.T <= kOneTokens) {
        // Columns by y and, beyond a grid's 65535, by z too: a few blocks at the end may have none.
        const int cols = tiles_of(d.D, 8 * kOneThreads), layers = tiles_of(cols, 65535);
        const dim3 grid(static_cast<unsigned>(F2 / kOneRows), static_cast<unsigned>(tiles_of(cols, layers)),
                        static_cast<unsigned>(layers));
        return launch_dependent(glu_outer_few_kernel, grid, kOneThreads, 0, s, 1, "launch glu_outer_few_kernel", d.T, d.D,
                                F2, dg, d.x, d.dW);
    }
    if (d.dW && d.T <= kOuterTokens) {
        const int cols = tiles_of(d.D, kOuterCols);
        const int64_t tiles = F2 / kOuterF * cols;
        if (tiles > 0x7fffffffLL) return set_error(ISAM_ERR_UNSUPPORTED, "isam_glu_backward: dW is too large");
        rc = ensure_smem_optin(reinterpret_cast<const void *>(glu_outer_kernel), outer_smem(kOuterTokens), ds.device,
                               "cudaFuncSetAttribute(feed-forward dW)");
        if (rc) return rc;
        return launch_dependent(glu_outer_kernel, dim3(static_cast<unsigned>(tiles)), kOuterThreads, outer_smem(d.T), s, 1,
                                "launch glu_outer_kernel", d.T, d.D, F2, cols, dg, d.x, d.dW);
    }
    if (d.dW) return product<true>(F2, d.D, d.T, dg, d.x, d.dW, parts, ds, s);
    return ISAM_OK;
}

}  // namespace isam
