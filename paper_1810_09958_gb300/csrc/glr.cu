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
// steps, then takes the next channels (the grid is no larger than what is
// resident).  Each warp has its own ring of tiles in shared memory, filled by
// TMA (where rows are not on 16-byte boundaries: by asynchronous copies), so the
// loads of later rounds stay in flight while a round is folded; states leave
// through shared memory and TMA as well.  With gates loaded straight into registers the forward kernel spent 34
// instructions an element, half of them addresses, and stopped at 55% of the
// copy bandwidth.  Folds pass between warps through shared memory, between
// CTAs through distributed shared memory (asynchronous stores counted on an
// mbarrier, buffers alternate; a cluster barrier per round, whose release waits
// for the states' stores, took 529 us where this took 243 us on
// 65536 x 1 x 2560); every warp carries the state at the end of the round
// itself, from the same folds in the same order, so nothing depends on timing.
// The cluster size (1 to 8) is picked so that one long sequence fills the GPU
// as a batch does.
//
// The backward pass is the same scan from the last step to the first with
// e_t = z_t (dh_t + e_{t+1}), d_t = dh_t + e_{t+1}.
#include <algorithm>
#include <type_traits>

#include "gemm_common.cuh"
#include "internal.h"
#include "known.h"
#include "lm_common.cuh"
#include "ptx.cuh"

namespace isam {

namespace {

constexpr int kMaxCluster = 8;
constexpr int kStages = 2;  // tiles of each input in a warp's ring

// Warps of a CTA, CTAs of an SM (launch bounds) and steps of a warp per round
// (L).  A round costs a warp about 350 instructions beside its steps', so the
// steps are as many as registers hold z and b (backward: four values) of.
// Measured, us (65536 x 1 x 2560 bf16 forward, 4096 x 8 x 1024 bf16 backward):
// 8 warps of 16 / 8 steps 207, 72; 4 warps of 32 / 16 steps 168, 62.  With
// one fp32 channel a lane (128 x 32 x 1024 forward, 20001 x 2 x 1760 backward):
// 8 warps of 16 / 8 steps 10.5, 189; 4 warps, 4 CTAs an SM 9.5, 224; 8 warps of
// 32 / 16 steps 10.4, 201.
// Rows that TMA does not bring cost the warps more instructions a step, and more
// warps hide them: 4 warps of 32 / 16 steps and 8 of 16 / 8, 7791 x 3 x 2042
// backward 202, 121; 3104 x 1 x 1757 forward 29, 24; 4096 x 8 x 1022 backward
// 108, 112.  With one fp32 channel a lane forward it goes by length, and this form
// is the one for few rounds: 4 warps, 4 CTAs an SM and 8 warps, 2 CTAs, 777 x 6 x 1001
// 18.0, 20.9 (ragged 15.3, 17.1), but 3104 x 1 x 1757 22.7, 20.1 and 20000 x 1 x 1001
// 87, 69.
template <int V, bool BACK, bool TMA>
struct Shape;
template <>
struct Shape<2, false, true> {
    static constexpr int kWarps = 4, kCtas = 2, kSteps = 32;
};
template <>
struct Shape<2, true, true> {
    static constexpr int kWarps = 4, kCtas = 2, kSteps = 16;
};
template <>
struct Shape<2, false, false> {
    static constexpr int kWarps = 8, kCtas = 2, kSteps = 16;
};
template <>
struct Shape<2, true, false> {
    static constexpr int kWarps = 8, kCtas = 2, kSteps = 8;
};
template <bool TMA>
struct Shape<1, false, TMA> {
    static constexpr int kWarps = 4, kCtas = 4, kSteps = 16;
};
template <bool TMA>
struct Shape<1, true, TMA> {
    static constexpr int kWarps = 8, kCtas = 2, kSteps = 8;
};
constexpr int kStepThreads = 128;
constexpr int kWalkBlock = 8, kWalkBack = 4;  // steps of a block, forward and backward

// V neighbouring elements, moved as one word.
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

// The V channels of a lane in fp32.  Two of them share one instruction for
// products and sums (f32x2), which halves the issue slots of the scan.
template <int V>
struct Lane;
template <>
struct Lane<1> {
    float x;
    __device__ __forceinline__ Lane() {}
    __device__ __forceinline__ explicit Lane(float v) : x(v) {}
    __device__ __forceinline__ Lane(const float (&v)[1]) : x(v[0]) {}
    __device__ __forceinline__ void get(float (&v)[1]) const { v[0] = x; }
};
template <>
struct Lane<2> {
    unsigned long long x;
    __device__ __forceinline__ Lane() {}
    __device__ __forceinline__ Lane(float lo, float hi) { asm("mov.b64 %0, {%1, %2};" : "=l"(x) : "f"(lo), "f"(hi)); }
    __device__ __forceinline__ explicit Lane(float v) : Lane(v, v) {}
    __device__ __forceinline__ Lane(const float (&v)[2]) : Lane(v[0], v[1]) {}
    __device__ __forceinline__ void get(float (&v)[2]) const {
        asm("mov.b64 {%0, %1}, %2;" : "=f"(v[0]), "=f"(v[1]) : "l"(x));
    }
};
__device__ __forceinline__ Lane<1> mul(Lane<1> a, Lane<1> b) { return Lane<1>(a.x * b.x); }
__device__ __forceinline__ Lane<1> add(Lane<1> a, Lane<1> b) { return Lane<1>(a.x + b.x); }
__device__ __forceinline__ Lane<1> fma(Lane<1> a, Lane<1> b, Lane<1> c) { return Lane<1>(fmaf(a.x, b.x, c.x)); }
__device__ __forceinline__ Lane<2> mul(Lane<2> a, Lane<2> b) {
    Lane<2> d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.x) : "l"(a.x), "l"(b.x));
    return d;
}
__device__ __forceinline__ Lane<2> add(Lane<2> a, Lane<2> b) {
    Lane<2> d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.x) : "l"(a.x), "l"(b.x));
    return d;
}
__device__ __forceinline__ Lane<2> fma(Lane<2> a, Lane<2> b, Lane<2> c) {
    Lane<2> d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.x) : "l"(a.x), "l"(b.x), "l"(c.x));
    return d;
}

// Elements to fp32 and back, a lane's word at a time.
template <typename T, int V>
__device__ __forceinline__ Lane<V> widen(const Pack<T, V> &p) {
    if constexpr (sizeof(T) == 2 && V == 2) {
        return Lane<2>(__uint_as_float(p.w << 16), __uint_as_float(p.w & 0xffff0000u));
    } else {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = to_f32(p.v[i]);
        return Lane<V>(v);
    }
}
template <typename T, int V>
__device__ __forceinline__ void narrow(Pack<T, V> &p, const Lane<V> &x) {
    float v[V];
    x.get(v);
    if constexpr (sizeof(T) == 2 && V == 2) {
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(p.w) : "f"(v[1]), "f"(v[0]));
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) p.v[i] = from_f32<T>(v[i]);
    }
}
// max(x, -87), a NaN staying one.
template <typename T, int V>
__device__ __forceinline__ Lane<V> widen_from_minus_87(Pack<T, V> p) {
    if constexpr (sizeof(T) == 2 && V == 2) {
        asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(p.w) : "r"(0xC2AEC2AEu));
        return widen<T, V>(p);
    } else {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v[i] = to_f32(p.v[i]);
            asm("max.NaN.f32 %0, %0, 0fC2AE0000;" : "+f"(v[i]));
        }
        return Lane<V>(v);
    }
}

// sigmoid(x) and 1 - sigmoid(x) without a branch on the sign: with
// e = exp(-x) they are 1 / (1 + e) and e / (1 + e), each accurate to its own
// size.  x >= -87, where the first is 2e-38, keeps e finite.
template <int V>
struct Gates {
    Lane<V> keep, take;
    __device__ __forceinline__ explicit Gates(const Lane<V> &x) {
        float t[V];
        mul(x, Lane<V>(-1.4426950408889634f)).get(t);
#pragma unroll
        for (int i = 0; i < V; ++i) asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(t[i]));
        const Lane<V> e(t);
        add(e, Lane<V>(1.0f)).get(t);
#pragma unroll
        for (int i = 0; i < V; ++i) asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(t[i]));
        keep = Lane<V>(t);
        take = mul(e, keep);
    }
};

// One affine map per channel of a lane.  A product of many gates may underflow;
// it is kept at 2^-126 (no gate is zero), so that an infinite state stays
// infinite as it does step by step, instead of 0 * inf.  A finite state h is
// changed by at most 2^-126 h.
template <int V>
struct __align__(8 * V) Fold {
    Lane<V> a, b;
    __device__ __forceinline__ Fold() {}
    __device__ __forceinline__ Fold(float av, float bv) : a(av), b(bv) {}
    // This map after `first`.
    __device__ __forceinline__ Fold after(const Fold &first) const {
        Fold f;
        f.a = positive(mul(a, first.a));
        f.b = fma(a, first.b, b);
        return f;
    }
    __device__ __forceinline__ Lane<V> of(const Lane<V> &h) const { return fma(a, h, b); }
    static __device__ __forceinline__ Lane<V> positive(const Lane<V> &a) {
        float v[V];
        a.get(v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = fmaxf(v[i], 1.17549435e-38f);
        return Lane<V>(v);
    }
};

// Folds of one round: of the CTA's warps, and of the cluster's CTAs (written
// by them, their bytes counted on `landed`).
template <int V, int WARPS>
struct FoldBuffers {
    Fold<V> warp[2][WARPS][32];
    Fold<V> cta[2][kMaxCluster][32];
    uint64_t landed[2];
    int abort;
};

// Buffers of round r are written again in round r + 2.  A CTA sends its fold of
// round r + 1 after all its warps are done with round r (their barrier in
// exchange), and a fold of round r + 2 is sent by a warp that holds every
// CTA's fold of round r + 1: nothing still reads, or waits for, round r.
template <int V, int WARPS>
__device__ __forceinline__ void exchange_init(FoldBuffers<V, WARPS> &s, uint32_t cluster) {
    if (threadIdx.x == 0) {
        mbar_init(&s.landed[0], 1);
        mbar_init(&s.landed[1], 1);
        s.abort = 0;
        fence_mbar_init();
    }
    if (cluster == 1)
        __syncthreads();
    else
        cluster_sync_all();
}

// The end of a kernel: stores have left shared memory; after a wait that ran
// out, copies into this CTA's shared memory get time to land; and no CTA leaves
// while another may still send it folds.
template <int V, int WARPS>
__device__ __forceinline__ void exchange_end(FoldBuffers<V, WARPS> &s, uint32_t cluster) {
    if ((threadIdx.x & 31) == 0) bulk_wait_all<0>();
    if (*static_cast<volatile int *>(&s.abort)) {
        const unsigned long long t0 = globaltimer();
        while (globaltimer() - t0 < 50000ull) {
        }
    }
    __syncwarp();
    if (cluster > 1) cluster_sync_all();
}

// Eight or sixteen bytes into a CTA of this cluster, counted on its barrier.
// Asynchronous: unlike a release, it does not wait for this thread's stores of
// states to reach L2.
__device__ __forceinline__ void send(uint32_t to, const Fold<2> &f, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(to),
                 "l"(f.a.x), "l"(f.b.x), "r"(bar)
                 : "memory");
}
__device__ __forceinline__ void send(uint32_t to, const Fold<1> &f, uint32_t bar) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.f32 [%0], {%1, %2}, [%3];" ::"r"(to),
                 "f"(f.a.x), "f"(f.b.x), "r"(bar)
                 : "memory");
}

// What a warp needs from the others' folds: returns the state before its first
// step of this round; `carry` becomes the state after the round.
template <int V, int WARPS>
__device__ __forceinline__ Lane<V> exchange(FoldBuffers<V, WARPS> &s, int r, Fold<V> &own, int warp, int warps, int lane,
                                            uint32_t rank, uint32_t cluster, const WaitCtx &wait, Lane<V> &carry) {
    const int parity = r & 1;
    own.a = Fold<V>::positive(own.a);
    s.warp[parity][warp][lane] = own;
    __syncthreads();
    Lane<V> in;
    if (cluster == 1) {
        for (int w = 0; w < warps; ++w) {
            if (w == warp) in = carry;
            carry = s.warp[parity][w][lane].of(carry);
        }
        return in;
    }
    Fold<V> before(1.0f, 0.0f);
    for (int w = 0; w < warp; ++w) before = s.warp[parity][w][lane].after(before);
    if (warp == warps - 1) {
        const Fold<V> all = own.after(before);
        if (lane == 0)
            mbar_arrive_expect_tx(&s.landed[parity], cluster * 32u * static_cast<uint32_t>(sizeof(Fold<V>)));
        const uint32_t at = smem_u32(&s.cta[parity][rank][lane]), bar = smem_u32(&s.landed[parity]);
        for (uint32_t q = 0; q < cluster; ++q) send(mapa_shared(at, q), all, mapa_shared(bar, q));
    }
    __syncwarp();
    bounded_wait<true>(&s.landed[parity], (r >> 1) & 1, wait, 0x603u);
    for (uint32_t q = 0; q < cluster; ++q) {
        if (q == rank) in = before.of(carry);
        carry = s.cta[parity][q][lane].of(carry);
    }
    return in;
}

struct ScanParams {
    GlrDesc d;
    uint32_t tiles;   // channel tiles of 32 V per sequence
    uint32_t groups;  // tiles * batch: the units a cluster takes one after another
    uint32_t cluster;
    uint32_t *err;
    unsigned long long timeout_ns;
};

__device__ __forceinline__ void lane_copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void lane_copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// How rows reach shared memory and leave the kernel: by TMA (16-byte
// boundaries), by asynchronous copies of each lane's own word (rows on
// boundaries of V elements), or as the 4-byte words that cover a row.
enum Rows { kTma, kLaneWords, kCover };

// A tile: L rows of a warp's 32 V channels.  Covering words: rows carry one
// more word, and a bf16 row may start in the upper half of its first word:
// `odd` is 1 then.  (Copies of two bytes a lane, or of covering words with
// bounds checked word by word, ran at 15% of the copy bandwidth.)
template <typename T, int V, int L, Rows ROWS>
struct Tile {
    static constexpr int kRow = 32 * V * static_cast<int>(sizeof(T)) + (ROWS == kCover ? 4 : 0);
    uint8_t bytes[L * kRow];
    __device__ __forceinline__ Pack<T, V> get(int k, int lane, uint32_t odd) const {
        Pack<T, V> p;
        const uint8_t *row = bytes + k * kRow;
        if constexpr (ROWS == kCover && sizeof(T) == 2 && V == 2) {
            const uint32_t *w = reinterpret_cast<const uint32_t *>(row) + lane;
            p.w = __funnelshift_r(w[0], w[1], 16 * odd);
        } else if constexpr (ROWS == kCover && sizeof(T) == 2) {
            p.w = reinterpret_cast<const unsigned short *>(row)[lane + odd];
        } else if constexpr (ROWS == kCover && V == 2) {
            p.w.x = reinterpret_cast<const uint32_t *>(row)[2 * lane];
            p.w.y = reinterpret_cast<const uint32_t *>(row)[2 * lane + 1];
        } else {
            p.w = reinterpret_cast<const typename Pack<T, V>::W *>(row)[lane];
        }
        return p;
    }
    __device__ __forceinline__ void put(int k, int lane, const Lane<V> &x) {
        Pack<T, V> p;
        narrow<T, V>(p, x);
        reinterpret_cast<typename Pack<T, V>::W *>(bytes + k * kRow)[lane] = p.w;
    }
    // Rows k = from .. n - 1 of `width` elements at src + k * pitch, by the
    // whole warp; [begin, end) is the array they lie in.
    __device__ __forceinline__ void copy(int lane, const T *src, int64_t pitch, int width, int from, int n,
                                         const T *begin, const T *end) {
        src += from * pitch;
        if constexpr (ROWS == kLaneWords) {
            if (lane * V >= width) return;
            constexpr int kWord = static_cast<int>(sizeof(T)) * V;
            src += lane * V;
            uint32_t at = smem_u32(bytes + from * kRow + lane * kWord);
#pragma unroll 4
            for (int k = from; k < n; ++k, src += pitch, at += kRow)
                asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(at), "l"(src), "n"(kWord < 4 ? 4 : kWord)
                             : "memory");
        } else if (sizeof(T) == 2 && (pitch & 1)) {  // rows start odd and even in turn
            copy_alike(lane, src, 2 * pitch, width, from, 2, n, begin, end);
            copy_alike(lane, src + pitch, 2 * pitch, width, from + 1, 2, n, begin, end);
        } else {
            copy_alike(lane, src, pitch, width, from, 1, n, begin, end);
        }
    }
    // Rows from, from + every, ... that all start in the same half of a word.
    __device__ __forceinline__ void copy_alike(int lane, const T *src, int64_t pitch, int width, int from, int every,
                                               int n, const T *begin, const T *end) {
        if (from >= n) return;
        const uint8_t *word = reinterpret_cast<const uint8_t *>(reinterpret_cast<uintptr_t>(src) & ~uintptr_t{3});
        const uint8_t *lo = reinterpret_cast<const uint8_t *>(begin), *hi = reinterpret_cast<const uint8_t *>(end);
        const int covered = (width * static_cast<int>(sizeof(T)) + 2 * static_cast<int>(odd_of(src)) + 3) & ~3;
        pitch *= sizeof(T);
        // A word that covers the array's first or last element may reach past it.
        const bool inside = word >= lo && word + (n - 1 - from) / every * pitch + covered <= hi;
        const bool one = lane * 4 < covered, more = lane * 4 + 128 < covered;
        word += lane * 4;
        uint8_t *to = bytes + from * kRow + lane * 4;
        if (inside) {
            uint32_t at = smem_u32(to);
#pragma unroll 4
            for (int k = from; k < n; k += every, word += pitch, at += every * kRow) {
                if (one) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at), "l"(word) : "memory");
                if (V == 2 && more)
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(at + 128), "l"(word + 128) : "memory");
            }
        } else {
            for (int k = from; k < n; k += every, word += pitch, to += every * kRow)
                for (int w = 0; lane * 4 + w < covered; w += 128)
#pragma unroll
                    for (int i = 0; i < 4; i += 2)
                        if (word + w + i >= lo && word + w + i < hi)
                            *reinterpret_cast<unsigned short *>(to + w + i) =
                                *reinterpret_cast<const unsigned short *>(word + w + i);
        }
    }
    static __device__ __forceinline__ uint32_t odd_of(const T *src) {
        return sizeof(T) == 2 ? (reinterpret_cast<uintptr_t>(src) >> 1) & 1u : 0u;
    }
};

// A row of a warp's states or gradients without TMA; at: the lane's first
// element, of which `left` exist from there to the row's end (by all lanes).
template <typename T, int V, Rows ROWS>
__device__ __forceinline__ void store_row(T *at, int lane, int left, const Lane<V> &x) {
    Pack<T, V> p;
    narrow<T, V>(p, x);
    if constexpr (V == 1 || ROWS != kCover) {
        if (left > 0) __stcs(reinterpret_cast<typename Pack<T, V>::W *>(at), p.w);
    } else if constexpr (sizeof(T) == 4) {
        if (left > 0) __stcs(reinterpret_cast<uint32_t *>(at), p.w.x);
        if (left > 1) __stcs(reinterpret_cast<uint32_t *>(at) + 1, p.w.y);
    } else if ((reinterpret_cast<uintptr_t>(at) & 2) == 0) {  // the same for every lane
        if (left > 1)
            __stcs(reinterpret_cast<uint32_t *>(at), p.w);
        else if (left > 0)
            __stcs(reinterpret_cast<unsigned short *>(at), static_cast<unsigned short>(p.w));
    } else {
        // Aligned words hold the neighbour's second element and this lane's first.
        const uint32_t below = __shfl_up_sync(0xffffffffu, p.w, 1);
        unsigned short *h = reinterpret_cast<unsigned short *>(at);
        if (lane == 0) {
            if (left > 0) __stcs(h, static_cast<unsigned short>(p.w));
        } else if (left > 0) {
            __stcs(reinterpret_cast<uint32_t *>(h - 1), __funnelshift_r(below, p.w, 16));
        } else if (left == 0) {  // the row ends with the neighbour's second element
            __stcs(h - 1, static_cast<unsigned short>(below >> 16));
        }
        if (lane == 31 && left > 1) __stcs(h + 1, static_cast<unsigned short>(p.w >> 16));
    }
}

// Shared memory of a warp (tiles start 128-byte aligned: every size is a
// multiple of 128).
struct Nothing {};
template <typename G, typename Hy, int V, int L, Rows ROWS>
struct __align__(128) ForwardTiles {
    struct In {
        Tile<G, V, L, ROWS> z, n;
    } in[kStages];
    std::conditional_t<ROWS == kTma, Tile<Hy, V, L, ROWS>, Nothing> out;
};
template <typename G, typename Hy, int V, int L, Rows ROWS>
struct __align__(128) BackwardTiles {
    struct In {
        Tile<G, V, L, ROWS> z, n;
        Tile<Hy, V, L, ROWS> before, dh;
    } in[kStages];
    std::conditional_t<ROWS == kTma, Tile<G, V, L, ROWS>, Nothing> dz, dn;
};

// A warp's place in its cluster, and one group of channels.
struct Warp {
    int lane, warp, warps;
    uint32_t rank, cluster;
    int chunk, span;  // this warp's L steps in a round of span warps, in time order
    uint32_t id, ids;  // this cluster, clusters of the grid
    __device__ Warp(const ScanParams &p) {
        lane = threadIdx.x & 31;
        warp = threadIdx.x >> 5;
        warps = blockDim.x >> 5;
        cluster = p.cluster;
        rank = blockIdx.x % cluster;
        id = blockIdx.x / cluster;
        ids = gridDim.x / cluster;
        chunk = rank * warps + warp;
        span = warps * cluster;
    }
};
template <int V>
struct Group {
    int b, c;       // sequence, first channel of the tile
    int len;        // steps of this sequence
    int own;        // this lane's first channel
    int left;       // channels from there to the row's end (below 1: none)
    int64_t chain;  // b * hidden + own
    int rounds;     // of this sequence
    __device__ __forceinline__ Group(const ScanParams &p, uint32_t g, int lane, int round) {
        g = min(g, p.groups - 1);  // behind the last one: not used
        b = static_cast<int>(g / p.tiles);
        c = static_cast<int>(g - static_cast<uint32_t>(b) * p.tiles) * 32 * V;
        own = c + lane * V;
        left = p.d.hidden - own;
        len = p.d.T;
        if (p.d.lengths) len = min(max(p.d.lengths[b], 0), p.d.T);
        rounds = static_cast<int>((static_cast<uint32_t>(len) + round - 1) / static_cast<uint32_t>(round));
        chain = static_cast<int64_t>(b) * p.d.hidden + own;
    }
};

// One value per channel of a lane from a [batch][hidden] array (or zero).
template <int V>
__device__ __forceinline__ Lane<V> edge(const float *from, const Group<V> &g) {
    float x[V];
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = from && i < g.left ? from[g.chain + i] : 0.0f;
    return Lane<V>(x);
}
template <int V>
__device__ __forceinline__ void put_edge(float *to, const Group<V> &g, const Lane<V> &x) {
    float v[V];
    x.get(v);
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < g.left) to[g.chain + i] = v[i];
}

// Forward.  Bound by HBM where sequences are long (65536 x 1 x 2560 bf16 169 us,
// 5.9 TB/s, 0.87 of the copy bandwidth); where they are short by a launch, first
// loads and few rounds that follow each other (128 x 32 x 1024, fp32 gates, 9.8 us,
// 0.64: 1024 groups on 608 CTAs, two turns of two rounds, no clusters; clusters of two
// would have four turns of one); without TMA by the instructions that copy and
// store words (777 x 6 x 1001, fp32, 18.0 us, 0.46) and, ragged, by the longest
// sequences, as turns are dealt out as if all had T steps (13.8 us, 0.33).
template <typename G, typename Hy, int V, int L, Rows ROWS>
__global__ void __launch_bounds__(32 * Shape<V, false, ROWS == kTma>::kWarps, (Shape<V, false, ROWS == kTma>::kCtas))
    glr_forward_kernel(const __grid_constant__ CUtensorMap tm_g, const __grid_constant__ CUtensorMap tm_h,
                       const __grid_constant__ ScanParams p) {
    if (p.cluster > 1 && !launch_shape_ok(p.err, p.cluster, gridDim.x, 0x601u)) return;
    constexpr bool TMA = ROWS == kTma;
    using Tiles = ForwardTiles<G, Hy, V, L, ROWS>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ FoldBuffers<V, Shape<V, false, ROWS == kTma>::kWarps> folds;
    __shared__ uint64_t full_all[Shape<V, false, ROWS == kTma>::kWarps][kStages];
    const WaitCtx wait{p.timeout_ns, p.err, &folds.abort};
    const Warp w(p);
    Tiles &mine = reinterpret_cast<Tiles *>(smem)[w.warp];
    uint64_t *full = full_all[w.warp];
    if (TMA && w.lane == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(&full[i], 1);
        fence_mbar_init();
    }
    exchange_init(folds, p.cluster);
    dependent_start();
    const int hidden = p.d.hidden;
    const int64_t step = static_cast<int64_t>(p.d.batch) * hidden;
    const int round = w.span * L, first = w.chunk * L;

    // Loads run kStages rounds ahead of their use, across groups.
    uint32_t load_group = w.id;
    Group<V> ahead(p, load_group, w.lane, round);
    int load_round = 0, load_stage = 0;
    const auto fetch = [&]() {
        while (load_group < p.groups && load_round >= ahead.rounds) {
            load_group += w.ids;
            load_round = 0;
            ahead = Group<V>(p, load_group, w.lane, round);
        }
        if (load_group < p.groups) {
            const Group<V> &g = ahead;
            const int t = load_round * round + first;
            typename Tiles::In &to = mine.in[load_stage];
            if (t < g.len) {
                if (TMA) {
                    if (w.lane == 0) {
                        mbar_arrive_expect_tx(&full[load_stage], sizeof(to));
                        tma_load_3d(&tm_g, &full[load_stage], &to.z, g.c, 2 * g.b, t);
                        tma_load_3d(&tm_g, &full[load_stage], &to.n, g.c, 2 * g.b + 1, t);
                    }
                } else {
                    const G *all = static_cast<const G *>(p.d.g), *end = all + 2 * step * p.d.T;
                    const G *q = all + 2 * step * t + static_cast<int64_t>(g.b) * 2 * hidden + g.c;
                    const int n = min(g.len - t, L), width = min(32 * V, hidden - g.c);
                    to.z.copy(w.lane, q, 2 * step, width, 0, n, all, end);
                    to.n.copy(w.lane, q + hidden, 2 * step, width, 0, n, all, end);
                }
            }
            ++load_round;
        }
        if (!TMA) lane_copies_commit();
        load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
    };
    Lane<V> next = edge<V>(p.d.h0, ahead);
    for (int i = 0; i < kStages; ++i) fetch();
    int it = 0, stage = 0;
    uint32_t phases = 0;
    for (uint32_t gi = w.id; gi < p.groups; gi += w.ids) {
        const Group<V> g(p, gi, w.lane, round);
        const int rounds = g.rounds;
        Hy *out = static_cast<Hy *>(p.d.h_out) + g.chain;
        Lane<V> carry = next;
        if (gi + w.ids < p.groups) next = edge<V>(p.d.h0, Group<V>(p, gi + w.ids, w.lane, round));
        for (int r = 0; r < rounds; ++r, ++it) {
            const int t = r * round + first;
            const int n = min(g.len - t, L);  // steps of this warp, below 1 past the end
            if (TMA) {
                if (n > 0) {
                    bounded_wait(&full[stage], (phases >> stage) & 1u, wait, 0x604u);
                    phases ^= 1u << stage;
                }
            } else {
                lane_copies_wait<kStages - 1>();
                __syncwarp();
            }
            Lane<V> z[L], b[L];
            const typename Tiles::In &in = mine.in[stage];
            // Rows of gates are an even number of elements apart: one parity for all.
            const G *row = static_cast<const G *>(p.d.g) + g.c;
            const uint32_t odd_z = Tile<G, V, L, ROWS>::odd_of(row), odd_n = Tile<G, V, L, ROWS>::odd_of(row + hidden);
#pragma unroll
            for (int k = 0; k < L; ++k) {
                const Gates<V> s(widen_from_minus_87<G, V>(in.z.get(k, w.lane, odd_z)));
                z[k] = s.keep;
                b[k] = mul(s.take, widen<G, V>(in.n.get(k, w.lane, odd_n)));
            }
            if (n < L) {
#pragma unroll
                for (int k = 0; k < L; ++k)
                    if (k >= n) z[k] = Lane<V>(1.0f), b[k] = Lane<V>(0.0f);
            }
            __syncwarp();  // every lane has read the tile
            fetch();
            stage = stage + 1 == kStages ? 0 : stage + 1;
            Fold<V> own(1.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < L; ++k) {
                own.a = mul(own.a, z[k]);
                own.b = fma(z[k], own.b, b[k]);
            }
            Lane<V> h = exchange(folds, it, own, w.warp, w.warps, w.lane, w.rank, w.cluster, wait, carry);
            if (TMA) {
                if (w.lane == 0) bulk_wait_read<0>();  // the last round's states have left the tile
                __syncwarp();
            }
            const auto emit = [&](bool whole) {
                Hy *q = out + step * t;
#pragma unroll
                for (int k = 0; k < L; ++k, q += step) {
                    h = fma(z[k], h, b[k]);
                    const Lane<V> v = whole || k < n ? h : Lane<V>(0.0f);
                    if constexpr (TMA) {
                        mine.out.put(k, w.lane, v);
                    } else {
                        if (whole || t + k < p.d.T) store_row<Hy, V, ROWS>(q, w.lane, g.left, v);
                    }
                }
            };
            if (n == L)
                emit(true);
            else
                emit(false);
            if (TMA) {
                fence_proxy_async_smem();
                __syncwarp();
                if (w.lane == 0 && t < p.d.T) {
                    tma_store_3d(&tm_h, &mine.out, g.c, g.b, t);
                    bulk_commit();
                }
            }
        }
        for (int t = rounds * round + w.chunk; t < p.d.T; t += w.span)
            store_row<Hy, V, ROWS>(out + step * t, w.lane, g.left, Lane<V>(0.0f));
        if (p.d.h_last && w.chunk == 0) put_edge<V>(p.d.h_last, g, carry);
    }
    exchange_end(folds, p.cluster);
}

// Backward: four values a step in, two out.  Bound by HBM: 4096 x 8 x 1024 bf16
// 63 us (6.4 TB/s, 0.94 of the copy bandwidth), 20001 x 2 x 1760 with fp32 gates,
// ragged, 194 us (0.91).
template <typename G, typename Hy, int V, int L, Rows ROWS>
__global__ void __launch_bounds__(32 * Shape<V, true, ROWS == kTma>::kWarps, (Shape<V, true, ROWS == kTma>::kCtas))
    glr_backward_kernel(const __grid_constant__ CUtensorMap tm_g, const __grid_constant__ CUtensorMap tm_h,
                        const __grid_constant__ CUtensorMap tm_dh, const __grid_constant__ CUtensorMap tm_dg,
                        const __grid_constant__ ScanParams p) {
    if (p.cluster > 1 && !launch_shape_ok(p.err, p.cluster, gridDim.x, 0x602u)) return;
    constexpr bool TMA = ROWS == kTma;
    using Tiles = BackwardTiles<G, Hy, V, L, ROWS>;
    extern __shared__ __align__(128) uint8_t smem[];
    __shared__ FoldBuffers<V, Shape<V, true, ROWS == kTma>::kWarps> folds;
    __shared__ uint64_t full_all[Shape<V, true, ROWS == kTma>::kWarps][kStages];
    const WaitCtx wait{p.timeout_ns, p.err, &folds.abort};
    const Warp w(p);
    Tiles &mine = reinterpret_cast<Tiles *>(smem)[w.warp];
    uint64_t *full = full_all[w.warp];
    if (TMA && w.lane == 0) {
        for (int i = 0; i < kStages; ++i) mbar_init(&full[i], 1);
        fence_mbar_init();
    }
    exchange_init(folds, p.cluster);
    dependent_start();
    const int hidden = p.d.hidden;
    const int64_t step = static_cast<int64_t>(p.d.batch) * hidden;
    const bool has_dh = p.d.dh_out != nullptr;
    // Rounds and their chunks start at multiples of L from step 0 and are taken
    // from the last to the first: the folds' order is the reverse of time.
    const int round = w.span * L, first = (w.span - 1 - w.chunk) * L;

    uint32_t load_group = w.id;
    Group<V> ahead(p, load_group, w.lane, round);
    int load_round = 0, load_stage = 0;  // rounds counted from the last
    const auto fetch = [&]() {
        while (load_group < p.groups && load_round >= ahead.rounds) {
            load_group += w.ids;
            load_round = 0;
            ahead = Group<V>(p, load_group, w.lane, round);
        }
        if (load_group < p.groups) {
            const Group<V> &g = ahead;
            const int t = (g.rounds - 1 - load_round) * round + first;
            typename Tiles::In &to = mine.in[load_stage];
            if (t < g.len) {
                if (TMA) {
                    if (w.lane == 0) {
                        uint64_t *bar = &full[load_stage];
                        mbar_arrive_expect_tx(bar, sizeof(to) - (has_dh ? 0 : sizeof(to.dh)));
                        tma_load_3d(&tm_g, bar, &to.z, g.c, 2 * g.b, t);
                        tma_load_3d(&tm_g, bar, &to.n, g.c, 2 * g.b + 1, t);
                        tma_load_3d(&tm_h, bar, &to.before, g.c, g.b, t - 1);  // row -1 reads zeros
                        if (has_dh) tma_load_3d(&tm_dh, bar, &to.dh, g.c, g.b, t);
                    }
                } else {
                    const G *all = static_cast<const G *>(p.d.g), *end = all + 2 * step * p.d.T;
                    const G *q = all + 2 * step * t + static_cast<int64_t>(g.b) * 2 * hidden + g.c;
                    const int64_t row = static_cast<int64_t>(g.b) * hidden + g.c;
                    const Hy *hs = static_cast<const Hy *>(p.d.h_in), *dh = static_cast<const Hy *>(p.d.dh_out);
                    const int n = min(g.len - t, L), width = min(32 * V, hidden - g.c);
                    to.z.copy(w.lane, q, 2 * step, width, 0, n, all, end);
                    to.n.copy(w.lane, q + hidden, 2 * step, width, 0, n, all, end);
                    to.before.copy(w.lane, hs + step * (t - 1) + row, step, width, t == 0, n, hs, hs + step * p.d.T);
                    if (has_dh) to.dh.copy(w.lane, dh + step * t + row, step, width, 0, n, dh, dh + step * p.d.T);
                }
            }
            ++load_round;
        }
        if (!TMA) lane_copies_commit();
        load_stage = load_stage + 1 == kStages ? 0 : load_stage + 1;
    };
    Lane<V> next = edge<V>(p.d.dh_last, ahead);
    for (int i = 0; i < kStages; ++i) fetch();
    int it = 0, stage = 0;
    uint32_t phases = 0;
    for (uint32_t gi = w.id; gi < p.groups; gi += w.ids) {
        const Group<V> g(p, gi, w.lane, round);
        const int rounds = g.rounds;
        G *dg = static_cast<G *>(p.d.dg) + g.chain + static_cast<int64_t>(g.b) * hidden;
        const Lane<V> h0 = edge<V>(p.d.h0, g);
        Lane<V> carry = next;
        if (gi + w.ids < p.groups) next = edge<V>(p.d.dh_last, Group<V>(p, gi + w.ids, w.lane, round));
        for (int r = rounds - 1; r >= 0; --r, ++it) {
            const int t = r * round + first;
            const int n = min(g.len - t, L);
            if (TMA) {
                if (n > 0) {
                    bounded_wait(&full[stage], (phases >> stage) & 1u, wait, 0x605u);
                    phases ^= 1u << stage;
                }
            } else {
                lane_copies_wait<kStages - 1>();
                __syncwarp();
            }
            // z, 1 - z, (h_{t-1} - n) z (1 - z) and dh of each step.
            Lane<V> z[L], take[L], q[L], d[L];
            const typename Tiles::In &in = mine.in[stage];
            // Rows of gates are an even number of elements apart, rows of states may
            // alternate.
            using TileG = Tile<G, V, L, ROWS>;
            using TileH = Tile<Hy, V, L, ROWS>;
            const G *row = static_cast<const G *>(p.d.g) + g.c;
            const uint32_t odd_z = TileG::odd_of(row), odd_n = TileG::odd_of(row + hidden);
            const int64_t first_h = static_cast<int64_t>(g.b) * hidden + g.c + step * t;
            const uint32_t odd_h = TileH::odd_of(static_cast<const Hy *>(p.d.h_in) + first_h - step);
            const uint32_t odd_d = TileH::odd_of(static_cast<const Hy *>(p.d.dh_out) + first_h);
            const uint32_t turn = static_cast<uint32_t>(step) & 1u;
#pragma unroll
            for (int k = 0; k < L; ++k) {
                const Gates<V> s(widen_from_minus_87<G, V>(in.z.get(k, w.lane, odd_z)));
                Lane<V> before = widen<Hy, V>(in.before.get(k, w.lane, odd_h ^ (turn & k)));
                if (k == 0 && t == 0) before = h0;
                z[k] = s.keep;
                take[k] = s.take;
                q[k] = mul(fma(widen<G, V>(in.n.get(k, w.lane, odd_n)), Lane<V>(-1.0f), before), mul(s.keep, s.take));
                d[k] = widen<Hy, V>(in.dh.get(k, w.lane, odd_d ^ (turn & k)));
            }
            if (n < L || !has_dh) {
#pragma unroll
                for (int k = 0; k < L; ++k) {
                    if (k >= n) z[k] = Lane<V>(1.0f);
                    if (k >= n || !has_dh) d[k] = Lane<V>(0.0f);
                }
            }
            __syncwarp();
            fetch();
            stage = stage + 1 == kStages ? 0 : stage + 1;
            Fold<V> own(1.0f, 0.0f);
#pragma unroll
            for (int k = L - 1; k >= 0; --k) {
                own.a = mul(own.a, z[k]);
                own.b = mul(z[k], add(own.b, d[k]));
            }
            Lane<V> e = exchange(folds, it, own, w.warp, w.warps, w.lane, w.rank, w.cluster, wait, carry);
            if (TMA) {
                if (w.lane == 0) bulk_wait_read<0>();
                __syncwarp();
            }
            const auto emit = [&](bool whole) {
                G *o = dg + 2 * step * (t + L - 1);
#pragma unroll
                for (int k = L - 1; k >= 0; --k, o -= 2 * step) {
                    const Lane<V> all = add(d[k], e);
                    const bool live = whole || k < n;
                    const Lane<V> dz = live ? mul(all, q[k]) : Lane<V>(0.0f);
                    const Lane<V> dn = live ? mul(all, take[k]) : Lane<V>(0.0f);
                    e = mul(z[k], all);
                    if constexpr (TMA) {
                        mine.dz.put(k, w.lane, dz);
                        mine.dn.put(k, w.lane, dn);
                    } else {
                        if (whole || t + k < p.d.T) {
                            store_row<G, V, ROWS>(o, w.lane, g.left, dz);
                            store_row<G, V, ROWS>(o + hidden, w.lane, g.left, dn);
                        }
                    }
                }
            };
            if (n == L)
                emit(true);
            else
                emit(false);
            if (TMA) {
                fence_proxy_async_smem();
                __syncwarp();
                if (w.lane == 0 && t < p.d.T) {
                    tma_store_3d(&tm_dg, &mine.dz, g.c, 2 * g.b, t);
                    tma_store_3d(&tm_dg, &mine.dn, g.c, 2 * g.b + 1, t);
                    bulk_commit();
                }
            }
        }
        for (int t = rounds * round + w.chunk; t < p.d.T; t += w.span) {
            store_row<G, V, ROWS>(dg + 2 * step * t, w.lane, g.left, Lane<V>(0.0f));
            store_row<G, V, ROWS>(dg + 2 * step * t + hidden, w.lane, g.left, Lane<V>(0.0f));
        }
        if (p.d.dh0 && w.chunk == 0) put_edge<V>(p.d.dh0, g, carry);
    }
    exchange_end(folds, p.cluster);
}

// Few steps, or channels enough to fill the GPU by themselves: one thread walks
// the time of its V channels, a block of steps' loads in flight.  Bound by HBM
// where the gates are fp32, by the instructions of an element in bf16: 8 x 2000 x
// 2048 bf16 forward 43 us (0.79 of the copy bandwidth), backward 80 us (0.82);
// 96 x 2000 x 1024 188 us (0.94) and 371 us (0.95), with fp32 gates 278 us (1.05)
// and 574 us (1.01).  Blocks of eight steps backward, whose four values a step
// leave a third fewer threads in the registers, took 8 x 2000 x 2048 91 us.
struct Walker {
    int64_t b, chain;  // sequence, first channel of it all
    int len;
    __device__ __forceinline__ Walker(const GlrDesc &d, int64_t i, int V) {
        const int per = d.hidden / V;  // (a row of `per` threads is one of `hidden` channels)
        b = i >> 32 ? i / per : static_cast<uint32_t>(i) / static_cast<uint32_t>(per);
        chain = i * V;
        len = d.lengths ? min(max(d.lengths[b], 0), d.T) : d.T;
    }
};
template <int V>
__device__ __forceinline__ Lane<V> walk_edge(const float *from, int64_t chain) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = from ? from[chain + i] : 0.0f;
    return Lane<V>(v);
}
template <int V>
__device__ __forceinline__ void walk_edge(float *to, int64_t chain, const Lane<V> &x) {
    float v[V];
    x.get(v);
#pragma unroll
    for (int i = 0; i < V; ++i) to[chain + i] = v[i];
}
template <typename T, int V>
__device__ __forceinline__ Pack<T, V> load_pack(const T *p) {
    Pack<T, V> v;
    v.w = *reinterpret_cast<const typename Pack<T, V>::W *>(p);
    return v;
}
template <typename T, int V>
__device__ __forceinline__ void store_pack(T *p, const Lane<V> &x) {
    Pack<T, V> v;
    narrow<T, V>(v, x);
    *reinterpret_cast<typename Pack<T, V>::W *>(p) = v.w;
}

template <typename G, typename Hy, int V>
__global__ void __launch_bounds__(kStepThreads, V == 1 ? 8 : 6)
    glr_walk_forward_kernel(const __grid_constant__ GlrDesc d, int64_t threads) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x;
    if (i >= threads) return;
    dependent_start();
    const Walker w(d, i, V);
    const int hidden = d.hidden;
    const int64_t step = static_cast<int64_t>(d.batch) * hidden;
    Lane<V> h = walk_edge<V>(d.h0, w.chain);
    const G *g = static_cast<const G *>(d.g) + w.chain + w.b * hidden;
    Hy *out = static_cast<Hy *>(d.h_out) + w.chain;
    const auto block = [&](int t, bool whole) {
        Pack<G, V> z[kWalkBlock], n[kWalkBlock];
#pragma unroll
        for (int k = 0; k < kWalkBlock; ++k, g += 2 * step)
            if (whole || t + k < w.len) {
                z[k] = load_pack<G, V>(g);
                n[k] = load_pack<G, V>(g + hidden);
            }
#pragma unroll
        for (int k = 0; k < kWalkBlock; ++k, out += step) {
            if (!whole && t + k >= d.T) break;
            if (whole || t + k < w.len) {
                const Gates<V> s(widen_from_minus_87<G, V>(z[k]));
                h = fma(s.keep, h, mul(s.take, widen<G, V>(n[k])));
                store_pack<Hy, V>(out, h);
            } else {
                store_pack<Hy, V>(out, Lane<V>(0.0f));
            }
        }
    };
    int t = 0;
#pragma unroll 1
    for (; t + kWalkBlock <= w.len; t += kWalkBlock) block(t, true);
#pragma unroll 1
    for (; t < d.T; t += kWalkBlock) block(t, false);
    if (d.h_last) walk_edge<V>(d.h_last, w.chain, h);
}

template <typename G, typename Hy, int V>
__global__ void __launch_bounds__(kStepThreads, V == 1 ? 8 : 6)
    glr_walk_backward_kernel(const __grid_constant__ GlrDesc d, int64_t threads) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x;
    if (i >= threads) return;
    dependent_start();
    const Walker w(d, i, V);
    const int hidden = d.hidden;
    const int64_t step = static_cast<int64_t>(d.batch) * hidden;
    Lane<V> e = walk_edge<V>(d.dh_last, w.chain);
    const Lane<V> h0 = walk_edge<V>(d.h0, w.chain);
    const bool has_dh = d.dh_out != nullptr;
    const int64_t at_g = w.chain + w.b * hidden;
    const auto block = [&](int t, bool whole) {  // steps t, t - 1, ...
        Pack<G, V> z[kWalkBack], n[kWalkBack];
        Pack<Hy, V> before[kWalkBack], own[kWalkBack];
        const G *g = static_cast<const G *>(d.g) + at_g + 2 * step * t;
        const Hy *hs = static_cast<const Hy *>(d.h_in) + w.chain + step * (t - 1);
        const Hy *dh = static_cast<const Hy *>(d.dh_out) + w.chain + step * t;
#pragma unroll
        for (int k = 0; k < kWalkBack; ++k, g -= 2 * step, hs -= step, dh -= step)
            if (whole || (t - k >= 0 && t - k < w.len)) {
                z[k] = load_pack<G, V>(g);
                n[k] = load_pack<G, V>(g + hidden);
                if (whole || t - k > 0) before[k] = load_pack<Hy, V>(hs);
                if (has_dh) own[k] = load_pack<Hy, V>(dh);
            }
        G *dg = static_cast<G *>(d.dg) + at_g + 2 * step * t;
#pragma unroll
        for (int k = 0; k < kWalkBack; ++k, dg -= 2 * step) {
            if (!whole && t - k < 0) break;
            Lane<V> dz(0.0f), dn(0.0f);
            if (whole || t - k < w.len) {
                const Gates<V> s(widen_from_minus_87<G, V>(z[k]));
                const Lane<V> prior = whole || t - k > 0 ? widen<Hy, V>(before[k]) : h0;
                const Lane<V> all = has_dh ? add(widen<Hy, V>(own[k]), e) : e;
                dz = mul(all, mul(fma(widen<G, V>(n[k]), Lane<V>(-1.0f), prior), mul(s.keep, s.take)));
                dn = mul(all, s.take);
                e = mul(s.keep, all);
            }
            store_pack<G, V>(dg, dz);
            store_pack<G, V>(dg + hidden, dn);
        }
    };
#pragma unroll 1
    for (int t = d.T - 1; t >= 0; t -= kWalkBack) {
        if (t < w.len && t >= kWalkBack)
            block(t, true);
        else
            block(t, false);
    }
    if (d.dh0) walk_edge<V>(d.dh0, w.chain, e);
}

// One token a sequence: one thread per V channels.  Bound by HBM, a few sequences
// by the launch: 4096 sequences of 2048 bf16 19.9 us (5.9 TB/s, 0.87 of the copy
// bandwidth), 32 of 1024 1.3 us.
template <typename G, typename Hy, int V>
__global__ void __launch_bounds__(kStepThreads)
    glr_step_kernel(int64_t threads, int hidden, int slots, const G *g, const int32_t *slot_ids, const float *state,
                    float *new_state, Hy *h) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kStepThreads + threadIdx.x;
    if (i >= threads) return;
    dependent_start();
    const int per = hidden / V;
    const int64_t b = i / per;
    const int c = static_cast<int>(i - b * per) * V;
    const int slot = slot_ids ? slot_ids[b] : static_cast<int>(b);
    float v[V] = {};
    if (slot >= 0 && slot < slots) {
        const int64_t at = static_cast<int64_t>(slot) * hidden + c;
        Pack<G, V> gz, gn;
        Pack<float, V> s;
        gz.w = *reinterpret_cast<const typename Pack<G, V>::W *>(g + b * 2 * hidden + c);
        gn.w = *reinterpret_cast<const typename Pack<G, V>::W *>(g + b * 2 * hidden + hidden + c);
        s.w = *reinterpret_cast<const typename Pack<float, V>::W *>(state + at);
#pragma unroll
        for (int k = 0; k < V; ++k) {
            const Gate z = gate(to_f32(gz.v[k]));
            s.v[k] = v[k] = z.keep * s.v[k] + z.take * to_f32(gn.v[k]);
        }
        *reinterpret_cast<typename Pack<float, V>::W *>(new_state + at) = s.w;
    }
    Pack<Hy, V> o;
#pragma unroll
    for (int k = 0; k < V; ++k) o.v[k] = from_f32<Hy>(v[k]);
    *reinterpret_cast<typename Pack<Hy, V>::W *>(h + b * hidden + c) = o.w;
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

// Rows of `hidden` elements on 16-byte boundaries: what TMA addresses.
bool rows16(int hidden, int type, const void *p) {
    const int size = type == ISAM_F32 ? 4 : 2;
    return static_cast<int64_t>(hidden) * size % 16 == 0 && reinterpret_cast<uintptr_t>(p) % 16 == 0;
}

int rows_tmap(CUtensorMap *out, const void *p, int type, int hidden, int64_t rows, int T, int width, int L) {
    const uint64_t size = type == ISAM_F32 ? 4 : 2;
    const uint64_t dims[3] = {static_cast<uint64_t>(hidden), static_cast<uint64_t>(rows), static_cast<uint64_t>(T)};
    const uint64_t strides[2] = {hidden * size, hidden * size * rows};
    const uint32_t box[3] = {static_cast<uint32_t>(width), 1, static_cast<uint32_t>(L)};
    return make_tmap_3d_plain(out, p, type == ISAM_F32, dims, strides, box);
}

// Clusters of `c` CTAs of this kernel resident at once, asked once per device,
// kernel and shape.
int resident_clusters(const void *fn, int c, int threads, int smem, const DeviceState &ds, int *n) {
    struct Key {
        int device;
        const void *fn;
        int c, threads;
        bool operator==(const Key &o) const {
            return device == o.device && fn == o.fn && c == o.c && threads == o.threads;
        }
    };
    static Known<Key, 512> known;
    return known.get(Key{ds.device, fn, c, threads}, n, [&](int *clusters) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        cfg.gridDim = dim3(static_cast<unsigned>(c * ds.num_sms));
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = c;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(clusters, fn, &cfg);
        if (e == cudaSuccess) return static_cast<int>(ISAM_OK);
        cudaGetLastError();
        return cuda_error(e, "cudaOccupancyMaxActiveClusters(gated linear recurrence)");
    });
}

// Fills in the launch shape: `smem` bytes a warp.  The cluster size is the one
// with the fewest rounds in all (rounds of a sequence times turns of a
// cluster): several CTAs share a sequence's time where the channels alone would
// leave SMs idle.
template <typename S, int V>
int scan_shape(const void *fn, const GlrDesc &d, int smem, const DeviceState &ds, ScanParams &p,
               cudaLaunchConfig_t &cfg) {
    constexpr int L = S::kSteps;
    p.d = d;
    p.err = ds.err_word;
    p.timeout_ns = wait_timeout_ns();
    p.tiles = static_cast<uint32_t>((d.hidden + 32LL * V - 1) / (32 * V));
    const int64_t groups = static_cast<int64_t>(p.tiles) * d.batch;
    if (groups > (1LL << 31)) return set_error(ISAM_ERR_UNSUPPORTED, "batch * hidden is too large for one launch");
    p.groups = static_cast<uint32_t>(groups);
    const int warps = std::min(S::kWarps, (d.T + L - 1) / L);
    const int bytes = smem * warps;
    int rc = ensure_smem_optin(fn, smem * S::kWarps, ds.device, "cudaFuncSetAttribute(gated linear recurrence)");
    if (rc) return rc;
    int64_t best = 0, grid = 0;
    for (int c = 1; c <= kMaxCluster; ++c) {
        const int64_t span = static_cast<int64_t>(c) * warps * L;
        if (c > 1 && span - warps * L >= d.T) break;  // CTAs without steps
        int resident = 0;
        const int failed = resident_clusters(fn, c, 32 * warps, bytes, ds, &resident);
        if (failed) rc = failed;  // matters where every size fails
        if (failed || resident < 1) continue;
        const int64_t ids = std::min<int64_t>(resident, groups);
        const int64_t cost = (d.T + span - 1) / span * ((groups + ids - 1) / ids);
        if (grid == 0 || cost < best) {
            best = cost;
            grid = ids * c;
            p.cluster = static_cast<uint32_t>(c);
        }
    }
    if (grid == 0 && rc) return rc;
    if (grid == 0) return set_error(ISAM_ERR_UNSUPPORTED, "the gated linear recurrence's kernel fits no SM");
    cfg.gridDim = dim3(static_cast<unsigned>(grid));
    cfg.blockDim = dim3(32 * warps);
    cfg.dynamicSmemBytes = bytes;
    return ISAM_OK;
}

template <typename G, typename Hy, int V, Rows ROWS>
int forward_launch(const GlrDesc &d, DeviceState &ds, cudaStream_t s) {
    using S = Shape<V, false, ROWS == kTma>;
    constexpr int L = S::kSteps;
    const auto fn = glr_forward_kernel<G, Hy, V, L, ROWS>;
    ScanParams p{};
    cudaLaunchConfig_t cfg = {};
    int rc = scan_shape<S, V>(reinterpret_cast<const void *>(fn), d, sizeof(ForwardTiles<G, Hy, V, L, ROWS>), ds, p, cfg);
    if (rc) return rc;
    CUtensorMap tg{}, th{};
    if (ROWS == kTma) {
        if ((rc = rows_tmap(&tg, d.g, d.g_type, d.hidden, 2LL * d.batch, d.T, 32 * V, L))) return rc;
        if ((rc = rows_tmap(&th, d.h_out, d.h_type, d.hidden, d.batch, d.T, 32 * V, L))) return rc;
    }
    return launch_dependent(fn, cfg.gridDim, static_cast<int>(cfg.blockDim.x), cfg.dynamicSmemBytes, s, p.cluster,
                            "launch glr_forward_kernel", tg, th, p);
}

template <typename G, typename Hy, int V, Rows ROWS>
int backward_launch(const GlrDesc &d, DeviceState &ds, cudaStream_t s) {
    using S = Shape<V, true, ROWS == kTma>;
    constexpr int L = S::kSteps;
    const auto fn = glr_backward_kernel<G, Hy, V, L, ROWS>;
    ScanParams p{};
    cudaLaunchConfig_t cfg = {};
    int rc = scan_shape<S, V>(reinterpret_cast<const void *>(fn), d, sizeof(BackwardTiles<G, Hy, V, L, ROWS>), ds, p, cfg);
    if (rc) return rc;
    CUtensorMap tg{}, th{}, tdh{}, tdg{};
    if (ROWS == kTma) {
        if ((rc = rows_tmap(&tg, d.g, d.g_type, d.hidden, 2LL * d.batch, d.T, 32 * V, L))) return rc;
        if ((rc = rows_tmap(&th, d.h_in, d.h_type, d.hidden, d.batch, d.T, 32 * V, L))) return rc;
        if (d.dh_out && (rc = rows_tmap(&tdh, d.dh_out, d.h_type, d.hidden, d.batch, d.T, 32 * V, L))) return rc;
        if ((rc = rows_tmap(&tdg, d.dg, d.g_type, d.hidden, 2LL * d.batch, d.T, 32 * V, L))) return rc;
    }
    return launch_dependent(fn, cfg.gridDim, static_cast<int>(cfg.blockDim.x), cfg.dynamicSmemBytes, s, p.cluster,
                            "launch glr_backward_kernel", tg, th, tdh, tdg, p);
}

// Whether walking beats the scan.  Measured, us, walk against scan, bf16 with rows
// of 1024 channels, forward and backward: 12 steps of 64 sequences 3.3 / 5.1 and
// 4.4 / 5.2; 32 steps of 64 6.2 / 5.9 and 11 / 8, of 128 7.7 / 9.2 and 13.4 / 12.9;
// 96 steps of 300 36 / 36 and 69 / 66, of 600 61 / 67 and 118 / 126.  Without TMA the
// scan is slower, rows of 1022: 96 steps of 16 sequences 8.5 / 4.5 and 23 / 8.9, of
// 64 15.1 / 15.4 and 28 / 32; 300 steps of 64 42 / 48 and 78 / 85.
bool walk(const GlrDesc &d, bool tma) {
    const int64_t channels = static_cast<int64_t>(d.batch) * d.hidden;
    if (d.T <= 16) return true;
    if (!tma) return channels >= 3 << 14;
    return channels >= 1 << 19 || (d.T <= 32 && channels >= 1 << 17);
}

int walk_launch(void (*fn)(const GlrDesc, int64_t), const GlrDesc &d, int V, cudaStream_t s, const char *what) {
    const int64_t threads = static_cast<int64_t>(d.batch) * (d.hidden / V);
    const int64_t blocks = (threads + kStepThreads - 1) / kStepThreads;
    if (blocks > 0x7fffffffLL) return set_error(ISAM_ERR_UNSUPPORTED, "batch * hidden is too large for one launch");
    return launch_dependent(fn, dim3(static_cast<unsigned>(blocks)), kStepThreads, 0, s, 1, what, d, threads);
}

}  // namespace

// V keeps a row of a warp at 128 bytes of gates, L its z and b (backward: four
// values a step) within the registers that Shape's CTAs an SM leave.
int glr_forward_launch(const GlrDesc &d, DeviceState &ds, cudaStream_t s) {
    return by_types(d.g_type, d.h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        constexpr int V = sizeof(G) == 2 ? 2 : 1;
        const bool tma = rows16(d.hidden, d.g_type, d.g) && rows16(d.hidden, d.h_type, d.h_out);
        if (walk(d, tma)) {
            const bool two = vector_ok(d.hidden, 2, d.g_type, d.g) && vector_ok(d.hidden, 2, d.h_type, d.h_out);
            return walk_launch(two ? glr_walk_forward_kernel<G, Hy, 2> : glr_walk_forward_kernel<G, Hy, 1>, d,
                               two ? 2 : 1, s, "launch glr_walk_forward_kernel");
        }
        if (tma) return forward_launch<G, Hy, V, kTma>(d, ds, s);
        if constexpr (V == 2) {
            if (vector_ok(d.hidden, V, d.g_type, d.g) && vector_ok(d.hidden, V, d.h_type, d.h_out))
                return forward_launch<G, Hy, V, kLaneWords>(d, ds, s);
        }
        return forward_launch<G, Hy, V, kCover>(d, ds, s);
    });
}

int glr_backward_launch(const GlrDesc &d, DeviceState &ds, cudaStream_t s) {
    return by_types(d.g_type, d.h_type, [&](auto gt, auto ht) {
        using G = decltype(gt);
        using Hy = decltype(ht);
        constexpr int V = sizeof(G) == 2 ? 2 : 1;
        const bool tma = rows16(d.hidden, d.g_type, d.g) && rows16(d.hidden, d.h_type, d.h_in) &&
                         rows16(d.hidden, d.h_type, d.dh_out) && rows16(d.hidden, d.g_type, d.dg);
        if (walk(d, tma)) {
            const bool two = vector_ok(d.hidden, 2, d.g_type, d.g) && vector_ok(d.hidden, 2, d.g_type, d.dg) &&
                             vector_ok(d.hidden, 2, d.h_type, d.h_in) && vector_ok(d.hidden, 2, d.h_type, d.dh_out);
            return walk_launch(two ? glr_walk_backward_kernel<G, Hy, 2> : glr_walk_backward_kernel<G, Hy, 1>, d,
                               two ? 2 : 1, s, "launch glr_walk_backward_kernel");
        }
        if (tma) return backward_launch<G, Hy, V, kTma>(d, ds, s);
        if constexpr (V == 2) {
            if (vector_ok(d.hidden, V, d.g_type, d.g) && vector_ok(d.hidden, V, d.g_type, d.dg) &&
                vector_ok(d.hidden, V, d.h_type, d.h_in) && vector_ok(d.hidden, V, d.h_type, d.dh_out))
                return backward_launch<G, Hy, V, kLaneWords>(d, ds, s);
        }
        return backward_launch<G, Hy, V, kCover>(d, ds, s);
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
        return launch_dependent(fn, dim3(blocks), kStepThreads, 0, s, 1, "launch glr_step_kernel", threads, hidden, slots,
                                static_cast<const G *>(g), slot_ids, state, new_state, static_cast<Hy *>(h));
    });
}

}  // namespace isam
