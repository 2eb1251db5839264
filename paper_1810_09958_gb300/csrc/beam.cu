// beam.cu -- beam search's selection over beams and vocabulary, and the
// reordering of state caches after it.
//
// Selection.  The best `count` of a sequence are among the best `count` of each
// of its rows, and a row's own order does not depend on its score and
// log-sum-exp.  So the rows kernel reads the logits once, in pieces that fill the
// GPU: a CTA keeps its piece's largest logit, the sum of exponentials over it and
// its best `count` entries.  The merge kernel, one CTA a sequence, adds the
// pieces' sums, forms scores in 64 bits and picks the best.  The bound is reading
// the logits (HBM).
//
// An entry is one 64-bit number: the logit's bits in the order of their values,
// then the token's complement; no two are equal, so "the best" is one set whatever
// order entries were found in.
#include <math_constants.h>

#include "lm_common.cuh"

namespace isam {

namespace {

constexpr int kThreads = 256;
constexpr int kPer = 16;                       // logits a thread and tile
constexpr int kTile = kThreads * kPer;
constexpr int kList = kTile + 1024;            // entries a CTA holds

using Key = unsigned long long;

__device__ __forceinline__ uint32_t ordered(float v) {
    const uint32_t u = __float_as_uint(v);
    return u ^ (static_cast<uint32_t>(static_cast<int32_t>(u) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t o) {
    return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// The best min(n, count) of list[0, n), best first, into best[]; all threads of
// the CTA call it, and list may be written again after it.
__device__ void take_best(Key *list, int n, int count, Key *best, Key *warp_best) {
    if (n <= 2 * kThreads) {
        // Each entry's place is the number of those above it.
        for (int i = threadIdx.x; i < n; i += kThreads) {
            const Key k = list[i];
            int above = 0;
            for (int j = 0; j < n; ++j) above += list[j] > k;
            if (above < count) best[above] = k;
        }
        __syncthreads();
        return;
    }
    for (int r = 0; r < count; ++r) {
        Key m = 0;
        for (int i = threadIdx.x; i < n; i += kThreads) m = max(m, list[i]);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) m = max(m, __shfl_xor_sync(~0u, m, d));
        if (threadIdx.x % 32 == 0) warp_best[threadIdx.x / 32] = m;
        __syncthreads();
        m = 0;
        for (int i = 0; i < kThreads / 32; ++i) m = max(m, warp_best[i]);
        if (threadIdx.x == 0) best[r] = m;
        for (int i = threadIdx.x; i < n; i += kThreads)
            if (list[i] == m) list[i] = 0;
        __syncthreads();
    }
}

struct Piece {
    float top;  // largest logit (-inf: none)
    float sum;  // sum of exp(logit - top)
};

template <typename L>
__global__ void __launch_bounds__(kThreads)
    beam_rows_kernel(int V, int count, int pieces, int piece, const L *logits, const float *scores,
                     const uint8_t *finished, Piece *out, Key *out_best) {
    __shared__ Key list[kList];
    __shared__ Key best[64];
    __shared__ Key warp_best[kThreads / 32];
    __shared__ float group_top[64];
    __shared__ int listed;
    __shared__ Piece warp_piece[kThreads / 32];
    dependent_start();
    const int row = blockIdx.x / pieces, part = blockIdx.x % pieces;
    Key *row_best = out_best + static_cast<int64_t>(blockIdx.x) * count;
    const float score = scores[row];
    if ((finished && finished[row]) || !(fabsf(score) < CUDART_INF_F)) return;  // the merge does not look at it
    const int lo = part * piece, hi = min(V, lo + piece);
    const L *l = logits + static_cast<int64_t>(row) * V;
    const int groups = count <= 8 ? 8 : count <= 16 ? 16 : count <= 32 ? 32 : 64, lanes = kThreads / groups;
    float top = -CUDART_INF_F, sum = 0.0f, floor = -CUDART_INF_F;
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
    for (int at = lo; at < hi; at += kTile) {
        float v[kPer], m = -CUDART_INF_F;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int t = at + i * kThreads + threadIdx.x;
            // (the larger of NaN and -inf is -inf; -0 becomes 0)
            v[i] = t < hi ? fmaxf(to_f32(l[t]), -CUDART_INF_F) + 0.0f : -CUDART_INF_F;
            m = fmaxf(m, v[i]);
        }
        if (m > top) {
            sum *= exp2f((top - m) * 1.4426950408889634f);
            top = m;
        }
        if (top > -CUDART_INF_F)
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum += exp2f((v[i] - top) * 1.4426950408889634f);
        if (at == lo) {
            // At least `count` entries are no lower than the lowest of `count` groups' largest.
            float g = m;
            for (int d = 1; d < lanes; d <<= 1) g = fmaxf(g, __shfl_xor_sync(~0u, g, d));
            if (threadIdx.x % lanes == 0) group_top[threadIdx.x / lanes] = g;
            __syncthreads();
            floor = group_top[0];
            for (int i = 1; i < groups; ++i) floor = fminf(floor, group_top[i]);
        }
        if (m >= floor && m > -CUDART_INF_F)
#pragma unroll
            for (int i = 0; i < kPer; ++i)
                if (v[i] >= floor && v[i] > -CUDART_INF_F)
                    list[atomicAdd(&listed, 1)] =
                        static_cast<Key>(ordered(v[i])) << 32 | static_cast<uint32_t>(~(at + i * kThreads + threadIdx.x));
        __syncthreads();
        const int n = listed;
        if (n > kList - kTile) {
            take_best(list, n, count, best, warp_best);
            if (threadIdx.x < count) list[threadIdx.x] = best[threadIdx.x];
            floor = unordered(static_cast<uint32_t>(best[count - 1] >> 32));
            if (threadIdx.x == 0) listed = count;
        }
        __syncthreads();
    }
    const int n = listed;
    take_best(list, n, count, best, warp_best);
    if (threadIdx.x < count) row_best[threadIdx.x] = threadIdx.x < n ? best[threadIdx.x] : 0;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
        const float t2 = __shfl_xor_sync(~0u, top, d), s2 = __shfl_xor_sync(~0u, sum, d);
        const float m = fmaxf(top, t2);
        if (m > -CUDART_INF_F)
            sum = sum * exp2f((top - m) * 1.4426950408889634f) + s2 * exp2f((t2 - m) * 1.4426950408889634f);
        top = m;
    }
    if (threadIdx.x % 32 == 0) warp_piece[threadIdx.x / 32] = Piece{top, sum};
    __syncthreads();
    if (threadIdx.x == 0) {
        Piece p = warp_piece[0];
        for (int i = 1; i < kThreads / 32; ++i) {
            const Piece q = warp_piece[i];
            const float m = fmaxf(p.top, q.top);
            if (m > -CUDART_INF_F)
                p.sum = p.sum * exp2f((p.top - m) * 1.4426950408889634f) + q.sum * exp2f((q.top - m) * 1.4426950408889634f);
            p.top = m;
        }
        out[blockIdx.x] = p;
    }
}

// A candidate of the merge: by score, then by its place (beam, logit, token).
__global__ void __launch_bounds__(kThreads)
    beam_merge_kernel(int beams, int count, int pieces, const float *scores, int eos, const uint8_t *finished,
                      const Piece *part, const Key *part_best, float *new_scores, int32_t *parents, int32_t *tokens,
                      uint8_t *new_finished) {
    __shared__ double base[64];  // score - log-sum-exp
    __shared__ int kind[64];     // 0 none, 1 open, 2 ended
    __shared__ double best_score[kThreads / 32];
    __shared__ long long best_place[kThreads / 32];
    dependent_start();
    const int64_t seq = blockIdx.x, first = seq * beams;
    if (threadIdx.x < beams) {
        const int64_t row = first + threadIdx.x;
        const double score = scores[row];
        int what = 0;
        double at = 0.0;
        if (fabs(score) < CUDART_INF) {
            if (finished && finished[row]) {
                what = 2;
                at = score;
            } else {
                float top = -CUDART_INF_F;
                for (int i = 0; i < pieces; ++i) top = fmaxf(top, part[row * pieces + i].top);
                if (fabsf(top) < CUDART_INF_F) {
                    double sum = 0.0;
                    for (int i = 0; i < pieces; ++i) {
                        const Piece p = part[row * pieces + i];
                        if (p.top > -CUDART_INF_F)
                            sum += p.sum * exp(static_cast<double>(p.top) - static_cast<double>(top));
                    }
                    what = 1;
                    at = score - (static_cast<double>(top) + log(sum));
                }
            }
        }
        base[threadIdx.x] = at;
        kind[threadIdx.x] = what;
    }
    __syncthreads();
    // Round r takes the best candidate below round r - 1's.  Place: beam, then the key from the largest down.
    const int each = pieces * count;
    double last_score = CUDART_INF;
    int last_beam = -1;
    Key last_key = ~0ull;
    for (int r = 0; r < count; ++r) {
        double s = -CUDART_INF;
        int beam = 64;
        Key key = 0;
        for (int i = threadIdx.x; i < beams * each; i += kThreads) {
            const int k = i / each;
            if (kind[k] == 0 || (kind[k] == 2 && i % each != 0)) continue;
            Key e = 1;
            double v = base[k];
            if (kind[k] == 1) {
                e = part_best[(first + k) * each + i % each];
                if (e == 0) continue;
                v += unordered(static_cast<uint32_t>(e >> 32));
            }
            const bool left = v < last_score || (v == last_score && (k > last_beam || (k == last_beam && e < last_key)));
            if (left && (v > s || (v == s && (k < beam || (k == beam && e > key))))) s = v, beam = k, key = e;
        }
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) {
            const double s2 = __shfl_xor_sync(~0u, s, d);
            const int b2 = __shfl_xor_sync(~0u, beam, d);
            const Key k2 = __shfl_xor_sync(~0u, key, d);
            if (s2 > s || (s2 == s && (b2 < beam || (b2 == beam && k2 > key)))) s = s2, beam = b2, key = k2;
        }
        __shared__ Key best_key[kThreads / 32];
        if (threadIdx.x % 32 == 0) {
            best_score[threadIdx.x / 32] = s;
            best_place[threadIdx.x / 32] = beam;
            best_key[threadIdx.x / 32] = key;
        }
        __syncthreads();
        for (int i = 0; i < kThreads / 32; ++i) {
            const double s2 = best_score[i];
            const int b2 = static_cast<int>(best_place[i]);
            const Key k2 = best_key[i];
            if (s2 > s || (s2 == s && (b2 < beam || (b2 == beam && k2 > key)))) s = s2, beam = b2, key = k2;
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            const bool found = beam < 64;
            const int token = !found ? 0 : kind[beam] == 2 ? eos : static_cast<int>(~static_cast<uint32_t>(key));
            const int64_t at = seq * count + r;
            new_scores[at] = found ? static_cast<float>(s) : -CUDART_INF_F;
            parents[at] = found ? beam : 0;
            tokens[at] = token;
            if (new_finished) new_finished[at] = found && (kind[beam] == 2 || token == eos);
        }
        last_score = s;
        last_beam = beam;
        last_key = key;
    }
}

constexpr int kChunk = 512;  // bytes of a row a CTA moves

// A CTA moves one chunk of the rows of one layer's sequence: all of its beams'
// chunks into shared memory, then each from its parent's.
template <typename W>
__global__ void __launch_bounds__(kThreads)
    beam_reorder_kernel(int batch, int beams, int slots, size_t row_bytes, int chunks, const int32_t *parents,
                        const int32_t *slot_ids, const char *state, char *new_state) {
    extern __shared__ uint4 raw[];
    W *held = reinterpret_cast<W *>(raw);
    dependent_start();
    constexpr int words = kChunk / sizeof(W);
    const int chunk = blockIdx.x % chunks;
    const int64_t group = blockIdx.x / chunks;
    const int b = static_cast<int>(group % batch);
    const int64_t layer = group / batch;
    const size_t at = static_cast<size_t>(chunk) * kChunk;
    const int live = static_cast<int>((min(row_bytes - at, static_cast<size_t>(kChunk))) / sizeof(W));
    const auto slot = [&](int k) { return slot_ids ? slot_ids[b * beams + k] : b * beams + k; };
    for (int i = threadIdx.x; i < beams * words; i += kThreads) {
        const int k = i / words, j = i % words, sl = slot(k);
        if (j < live && sl >= 0 && sl < slots)
            held[i] = reinterpret_cast<const W *>(state + (layer * slots + sl) * row_bytes + at)[j];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < beams * words; i += kThreads) {
        const int k = i / words, j = i % words, sl = slot(k), from = parents[b * beams + k];
        if (j >= live || sl < 0 || sl >= slots || from < 0 || from >= beams) continue;
        const int fs = slot(from);
        if (fs < 0 || fs >= slots) continue;
        reinterpret_cast<W *>(new_state + (layer * slots + sl) * row_bytes + at)[j] = held[from * words + j];
    }
}

// Pieces a row is cut into, and their length: enough CTAs to fill the GPU, no more
// than 64 pieces, and none shorter than a tile.
void cut(int rows, int V, int *pieces, int *piece) {
    int n = (152 * 4 + rows - 1) / rows;
    const int most = (V + kTile - 1) / kTile;
    n = n > most ? most : n;
    n = n > 64 ? 64 : n;
    *piece = (V + n - 1) / n;
    *pieces = (V + *piece - 1) / *piece;
}

}  // namespace

size_t beam_select_workspace(int batch, int beams, int V, int count) {
    int pieces, piece;
    cut(batch * beams, V, &pieces, &piece);
    return static_cast<size_t>(batch) * beams * pieces * (count * sizeof(Key) + sizeof(Piece));
}

int beam_select_launch(const BeamDesc &p, cudaStream_t s) {
    int pieces, piece;
    const int rows = p.batch * p.beams;
    cut(rows, p.V, &pieces, &piece);
    Key *best = static_cast<Key *>(p.workspace);
    Piece *part = reinterpret_cast<Piece *>(best + static_cast<size_t>(rows) * pieces * p.count);
    const dim3 grid(static_cast<unsigned>(rows) * pieces);
    int rc;
    if (p.l_type == ISAM_F32)
        rc = launch_dependent(beam_rows_kernel<float>, grid, kThreads, 0, s, 1, "launch beam_rows_kernel", p.V, p.count,
                              pieces, piece, static_cast<const float *>(p.logits), p.scores, p.finished, part, best);
    else
        rc = launch_dependent(beam_rows_kernel<bf16>, grid, kThreads, 0, s, 1, "launch beam_rows_kernel", p.V, p.count,
                              pieces, piece, static_cast<const bf16 *>(p.logits), p.scores, p.finished, part, best);
    if (rc) return rc;
    return launch_dependent(beam_merge_kernel, dim3(p.batch), kThreads, 0, s, 1, "launch beam_merge_kernel", p.beams,
                            p.count, pieces, p.scores, p.eos, p.finished, part, best, p.new_scores, p.parents, p.tokens,
                            p.new_finished);
}

int beam_reorder_launch(int layers, int batch, int beams, int slots, size_t row_bytes, const int32_t *parents,
                        const int32_t *slot_ids, const void *state, void *new_state, cudaStream_t s) {
    const int64_t chunks = static_cast<int64_t>((row_bytes + kChunk - 1) / kChunk);
    const int64_t blocks = chunks * layers * batch;
    if (blocks > 0x7fffffff) return set_error(ISAM_ERR_UNSUPPORTED, "isam_beam_reorder: too many bytes");
    const uintptr_t odd = reinterpret_cast<uintptr_t>(state) | reinterpret_cast<uintptr_t>(new_state) | row_bytes;
    const auto fn = odd % 16 == 0  ? beam_reorder_kernel<uint4>
                    : odd % 4 == 0 ? beam_reorder_kernel<uint32_t>
                    : odd % 2 == 0 ? beam_reorder_kernel<uint16_t>
                                   : beam_reorder_kernel<uint8_t>;
    return launch_dependent(fn, dim3(static_cast<unsigned>(blocks)), kThreads, static_cast<size_t>(beams) * kChunk, s, 1,
                            "launch beam_reorder_kernel", batch, beams, slots, row_bytes, static_cast<int>(chunks),
                            parents, slot_ids, static_cast<const char *>(state), static_cast<char *>(new_state));
}

}  // namespace isam
