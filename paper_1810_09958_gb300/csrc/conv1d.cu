// conv1d.cu -- short causal convolution over time, each channel by itself,
//   y_t[c] = act(bias[c] + sum_j w[j][c] x_{t - width + 1 + j}[c]),
// over a sequence, and one token on a cache of the last inputs.
//
// A thread has V neighbouring channels and walks a run of steps with the last
// width - 1 inputs in registers, so every input is read once (and width - 1
// more at the start of a run); the bound is HBM.
#include "lm_common.cuh"

namespace isam {

namespace {

constexpr int kThreads = 128;

template <typename T, int V>
struct alignas(sizeof(T) * V) Vec {
    T v[V];
};

template <int V, typename T>
__device__ __forceinline__ Vec<T, V> load(const T *p) {
    return *reinterpret_cast<const Vec<T, V> *>(p);
}

template <int V, typename T>
__device__ __forceinline__ void zero(Vec<T, V> &a) {
#pragma unroll
    for (int i = 0; i < V; ++i) a.v[i] = from_f32<T>(0.0f);
}

__device__ __forceinline__ float silu(float v) {
    const Gate s = gate(v);
    return v * s.keep;
}

template <typename X, typename Y, int V, int W>
__global__ void __launch_bounds__(kThreads)
    conv1d_forward_kernel(int T, int batch, int C, int run, int silu_on, const X *x, int64_t x_stride, const float *w,
                          const float *bias, const X *state, const int32_t *lengths, Y *y, X *new_state) {
    const int c = (blockIdx.x * kThreads + threadIdx.x) * V;
    if (c >= C) return;
    dependent_start();
    const int b = blockIdx.z % batch;
    const int64_t first = (static_cast<int64_t>(blockIdx.y) + static_cast<int64_t>(blockIdx.z / batch) * gridDim.y) * run;
    if (first >= T) return;
    const int len = lengths ? min(max(lengths[b], 0), T) : T;
    const int64_t pitch = static_cast<int64_t>(batch) * x_stride;
    const X *xb = x + b * x_stride + c;

    // What lies `back` steps before the sequence's first.
    const auto before = [&](int back) {
        Vec<X, V> a;
        zero(a);
        if (state) a = load<V>(state + (static_cast<int64_t>(b) * (W - 1) + (W - 1 - back)) * C + c);
        return a;
    };
    Vec<X, V> past[W];  // past[W - 1]: this step's input
    Vec<X, V> last[W - 1];
    // Run 0 reads the states and, with the same threads, writes the new ones.
    const bool ends = first == 0 && new_state;
    if (ends)
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int t = len - (W - 1) + j;
            last[j] = t >= 0 ? load<V>(xb + t * pitch) : before(-t);
        }
    float tap[W][V], add[V];
#pragma unroll
    for (int j = 0; j < W; ++j)
#pragma unroll
        for (int i = 0; i < V; ++i) tap[j][i] = w[static_cast<int64_t>(j) * C + c + i];
#pragma unroll
    for (int i = 0; i < V; ++i) add[i] = bias ? bias[c + i] : 0.0f;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        const int64_t t = first - (W - 1) + j;
        zero(past[j + 1]);
        if (t < 0) past[j + 1] = before(static_cast<int>(-t));
        else if (t < len) past[j + 1] = load<V>(xb + t * pitch);
    }
    const int64_t stop = min(first + run, static_cast<int64_t>(T));
    Y *out = y + (first * batch + b) * C + c;
    for (int64_t t = first; t < stop; ++t, out += static_cast<int64_t>(batch) * C) {
        Vec<Y, V> o;
        zero(o);
        if (t < len) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j) past[j] = past[j + 1];
            past[W - 1] = load<V>(xb + t * pitch);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float v = add[i];
#pragma unroll
                for (int j = 0; j < W; ++j) v = fmaf(to_f32(past[j].v[i]), tap[j][i], v);
                o.v[i] = from_f32<Y>(silu_on ? silu(v) : v);
            }
        }
        *reinterpret_cast<Vec<Y, V> *>(out) = o;
    }
    if (ends)
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            *reinterpret_cast<Vec<X, V> *>(new_state + (static_cast<int64_t>(b) * (W - 1) + j) * C + c) = last[j];
}

template <typename X, typename Y, int V, int W>
__global__ void __launch_bounds__(kThreads)
    conv1d_step_kernel(int64_t threads, int C, int slots, int silu_on, const X *x, int64_t x_stride, const float *w,
                       const float *bias, const int32_t *slot_ids, const X *state, X *new_state, Y *y) {
    const int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
    if (i >= threads) return;
    dependent_start();
    const int per = C / V;
    const int64_t b = i / per;
    const int c = static_cast<int>(i - b * per) * V;
    const int slot = slot_ids ? slot_ids[b] : static_cast<int>(b);
    Vec<Y, V> o;
    zero(o);
    if (slot >= 0 && slot < slots) {
        const int64_t at = static_cast<int64_t>(slot) * (W - 1) * C + c;
        Vec<X, V> past[W];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) past[j] = load<V>(state + at + static_cast<int64_t>(j) * C);
        past[W - 1] = load<V>(x + b * x_stride + c);
        float v[V];
#pragma unroll
        for (int k = 0; k < V; ++k) v[k] = bias ? bias[c + k] : 0.0f;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const Vec<float, V> tap = load<V>(w + static_cast<int64_t>(j) * C + c);
#pragma unroll
            for (int k = 0; k < V; ++k) v[k] = fmaf(to_f32(past[j].v[k]), tap.v[k], v[k]);
        }
#pragma unroll
        for (int k = 0; k < V; ++k) o.v[k] = from_f32<Y>(silu_on ? silu(v[k]) : v[k]);
#pragma unroll
        for (int j = 0; j < W - 1; ++j)
            *reinterpret_cast<Vec<X, V> *>(new_state + at + static_cast<int64_t>(j) * C) = past[j + 1];
    }
    *reinterpret_cast<Vec<Y, V> *>(y + b * C + c) = o;
}

// Whether p and rows `stride` elements apart allow V elements in one word.
bool words(const void *p, int type, int64_t stride, int V) {
    const int size = type == ISAM_F32 ? 4 : 2;
    return stride % V == 0 && reinterpret_cast<uintptr_t>(p) % (size * V) == 0;
}

bool words_ok(const ConvDesc &p, int V) {
    return p.C % V == 0 && words(p.x, p.x_type, p.x_stride, V) && words(p.state, p.x_type, p.C, V) &&
           words(p.new_state, p.x_type, p.C, V) && words(p.y, p.y_type, p.C, V) && words(p.w, ISAM_F32, p.C, V) &&
           words(p.bias, ISAM_F32, p.C, V);
}

template <typename F>
int by_type(int type, F &&f) {
    return type == ISAM_F32 ? f(float()) : f(bf16());
}

template <int W>
struct Width {
    static constexpr int value = W;
};

template <typename F>
int by_width(int width, F &&f) {
    switch (width) {
        case 2: return f(Width<2>());
        case 3: return f(Width<3>());
        case 4: return f(Width<4>());
        case 5: return f(Width<5>());
        case 6: return f(Width<6>());
        case 7: return f(Width<7>());
        default: return f(Width<8>());
    }
}

template <typename F>
int by_all(const ConvDesc &p, F &&f) {
    const bool four = words_ok(p, 4);
    return by_type(p.x_type, [&](auto x) {
        return by_type(p.y_type, [&](auto y) {
            return by_width(p.width, [&](auto w) { return four ? f(x, y, w, Width<4>()) : f(x, y, w, Width<1>()); });
        });
    });
}

}  // namespace

int conv1d_forward_launch(const ConvDesc &p, DeviceState &ds, cudaStream_t s) {
    return by_all(p, [&](auto x, auto y, auto w, auto v) {
        using X = decltype(x);
        using Y = decltype(y);
        constexpr int W = decltype(w)::value, V = decltype(v)::value;
        const unsigned across = static_cast<unsigned>((p.C / V + kThreads - 1) / kThreads);
        // Runs long enough that the inputs read twice are few, short enough to fill the GPU.
        int run = 32;
        while (run > 4 && static_cast<int64_t>(across) * p.batch * ((p.T + run - 1) / run) < ds.num_sms * 8) run /= 2;
        const int64_t runs = (p.T + static_cast<int64_t>(run) - 1) / run;
        const unsigned gy = static_cast<unsigned>(runs < 32768 ? runs : 32768);
        const int64_t gz = (runs + gy - 1) / gy * p.batch;
        if (gz > 65535) return set_error(ISAM_ERR_UNSUPPORTED, "isam_conv1d_forward: batch x steps too large");
        return launch_dependent(conv1d_forward_kernel<X, Y, V, W>, dim3(across, gy, static_cast<unsigned>(gz)), kThreads,
                                0, s, 1, "launch conv1d_forward_kernel", p.T, p.batch, p.C, run, p.silu,
                                static_cast<const X *>(p.x), p.x_stride, p.w, p.bias, static_cast<const X *>(p.state),
                                p.lengths, static_cast<Y *>(p.y), static_cast<X *>(p.new_state));
    });
}

int conv1d_step_launch(const ConvDesc &p, cudaStream_t s) {
    return by_all(p, [&](auto x, auto y, auto w, auto v) {
        using X = decltype(x);
        using Y = decltype(y);
        constexpr int W = decltype(w)::value, V = decltype(v)::value;
        const int64_t threads = static_cast<int64_t>(p.batch) * (p.C / V);
        const int64_t blocks = (threads + kThreads - 1) / kThreads;
        if (blocks > 0x7fffffff) return set_error(ISAM_ERR_UNSUPPORTED, "isam_conv1d_step: batch x C too large");
        return launch_dependent(conv1d_step_kernel<X, Y, V, W>, dim3(static_cast<unsigned>(blocks)), kThreads, 0, s, 1,
                                "launch conv1d_step_kernel", threads, p.C, p.slots, p.silu,
                                static_cast<const X *>(p.x), p.x_stride, p.w, p.bias, p.slot_ids,
                                static_cast<const X *>(p.state), static_cast<X *>(p.new_state), static_cast<Y *>(p.y));
    });
}

}  // namespace isam
