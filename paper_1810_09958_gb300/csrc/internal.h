// internal.h -- host-side declarations shared by the library's translation
// units.  Not part of the public ABI (that is include/isam.h).
#pragma once
#include <cstddef>
#include <cstdint>
#include <cuda.h>
#include <cuda_runtime.h>

#include "../../include/isam.h"

namespace isam {

// Device error word layout (uint32 x 4), written by kernels and read by
// isam_sync: [0] flags, [1] site of the first error, [2] blockIdx.x of that
// CTA, [3] detail (the cluster size a kernel found, for a launch-shape error).
enum : uint32_t { DEV_ERR_TIMEOUT = 1u, DEV_ERR_LAUNCH_SHAPE = 2u };

// Per-device state, created on first use with that device current.
struct DeviceState {
    int device = -1;
    int num_sms = 0;
    int max_smem_optin = 0;
    // Clusters of 2, 4 and 8 CTAs resident at once; 0 = ask the device (a
    // host-side plan for given limits fills them in).
    int cluster_cap[3] = {0, 0, 0};
    uint32_t *err_word = nullptr;  // 4 x uint32 on the device
    // GRU workspaces (grown on demand).
    float *gru_gx = nullptr;       // [T*batch][3H] fp32 input projection
    size_t gru_gx_bytes = 0;
    uint16_t *gru_hx = nullptr;    // 2 x [32][H] bf16 hidden-state exchange
    size_t gru_hx_bytes = 0;
    uint32_t *gru_counter = nullptr;  // step counter (1 x uint32, padded)
    float *gru_gxp = nullptr;      // 2 x [ks][T*batch][3H] fp32 stacked layers' projections
    size_t gru_gxp_bytes = 0;
    uint16_t *gru_xb = nullptr;    // [T*batch][H] bf16 states of a layer (next pair's input)
    size_t gru_xb_bytes = 0;
};

DeviceState *device_state(int *status);  // current device; null + status on failure
cudaStream_t current_stream();
unsigned long long wait_timeout_ns();

int set_error(int code, const char *fmt, ...);
int cuda_error(cudaError_t e, const char *what);

// Raises kernel fn's dynamic shared-memory limit to at least `bytes` on the
// current device, whose ordinal is `device`.  The attribute belongs to each
// device's context, so the record of what was set is kept per (device, kernel).
int ensure_smem_optin(const void *fn, int bytes, int device, const char *what);

// cuTensorMapEncodeTiled through the runtime's driver entry point, with a
// small cache keyed on every encoded field.
int make_tmap_2d_bf16(CUtensorMap *out, const void *base, uint64_t inner, uint64_t outer,
                      uint64_t row_pitch_bytes, uint32_t box_inner, uint32_t box_outer);
int make_tmap_2d_f32(CUtensorMap *out, const void *base, uint64_t inner, uint64_t outer,
                     uint64_t row_pitch_bytes, uint32_t box_inner, uint32_t box_outer);
// Same for 8-bit elements (E4M3 operands), 128-byte swizzle.
int make_tmap_2d_u8(CUtensorMap *out, const void *base, uint64_t inner, uint64_t outer,
                    uint64_t row_pitch_bytes, uint32_t box_inner, uint32_t box_outer);
int make_tmap_3d_bf16(CUtensorMap *out, const void *base, const uint64_t dims[3],
                      const uint64_t strides_bytes[2], const uint32_t box[3]);

// 3-D map of bf16 or fp32 elements without swizzle (boxes read row by row).
int make_tmap_3d_plain(CUtensorMap *out, const void *base, bool f32, const uint64_t dims[3],
                       const uint64_t strides_bytes[2], const uint32_t box[3]);

// GEMM C = alpha op(A) op(B) + beta C (+ bias[n] per column when bias != null).
struct GemmDesc {
    int M, N, K;
    int transA, transB;
    float alpha, beta;
    const uint16_t *A;
    const uint16_t *B;
    float *C;
    const float *bias_n;
    int fp8 = 0;  // A and B are E4M3 bytes (A: M x K, B: N x K, both K-major)
};

// Tile plan chosen by the cost model (or forced through ISAM_FORCE_TILE).
struct GemmPlan {
    int BN;       // tile width (tile height is always 128)
    int ka;       // 64-wide K atoms per pipeline stage
    int split;    // CTAs of one cluster sharing a tile along K (1, 2, 4 or 8)
    int stages;   // shared-memory ring depth
    int group_m;  // rasterisation group height (tiles)
    int grid;     // CTAs launched (persistent)
    size_t smem;  // dynamic shared memory bytes
    double est_us;
    int pair = 0; // 1: 256 x 256 tiles on CTA pairs (cta_group::2), see gemm_pair.cu
};

int gemm_validate(const GemmDesc &g);
int gemm_plan(const GemmDesc &g, const DeviceState &ds, GemmPlan *plan);
int gemm_launch(const GemmDesc &g, const GemmPlan &plan, DeviceState &ds, cudaStream_t s);
// The CTA-pair kernel: fills *plan and returns 1 when the problem suits it
// (K-major A, bf16, N % 4 == 0, at least one 256 x 256 tile per SM pair).
int gemm_pair_plan(const GemmDesc &g, const DeviceState &ds, GemmPlan *plan);
// Clusters of `size` CTAs (one per SM) resident at once on this device.
int gemm_cluster_capacity(const DeviceState &ds, int size);
int gemm_pair_launch(const GemmDesc &g, const GemmPlan &plan, DeviceState &ds, cudaStream_t s);

// Independent GEMMs in one persistent launch (1 <= count <= 64).
int gemm_grouped_launch(int count, const GemmDesc *g, DeviceState &ds, cudaStream_t s);

// Block-scaled E4M3 GEMM (OCP MX): C = alpha (SA o A)(SB o B)^T + beta C with
// A M x K and B N x K E4M3 bytes (K-major) and one E8M0 scale byte per 32 K
// elements of each row, atom-major: SA [ceil(K/128)][M][4], SB
// [ceil(K/128)][N][4] (4-byte aligned).
struct MxDesc {
    int M, N, K;
    float alpha, beta;
    const uint8_t *A;
    const uint8_t *SA;
    const uint8_t *B;
    const uint8_t *SB;
    float *C;
};
int gemm_mx_validate(const MxDesc &g);
// One persistent launch over the tiles of 1 <= count <= 64 problems.
int gemm_mx_launch(int count, const MxDesc *g, DeviceState &ds, cudaStream_t s);

// reset_before: the candidate's recurrent input is U_n (r * h) (two rounds per step).
int gru_launch(int T, int batch, int hidden, const uint16_t *x, const uint16_t *W,
               const uint16_t *U, const float *b, const float *h0, float *h_out, DeviceState &ds,
               cudaStream_t s, int reset_before = 0);
// Two stacked layers in one persistent kernel (reset gate after the
// product, hidden a multiple of 256): layer a's projection gx_a is given,
// layer b's comes from W_b and layer a's states inside the kernel.
bool gru_wave_supported(int H, int batch, const DeviceState &ds);
bool gru_wave_fits(int H, int batch, int num_sms, int smem_optin);
size_t gru_wave_smem_bytes(int H);

// How a GRU call runs on a device with num_sms SMs and smem_optin bytes of
// shared memory per CTA (host arithmetic only, no CUDA call).
struct GruPlan {
    int ks = 0;       // K splits per group of 32 units (cluster size)
    int ka = 0;       // 64-wide K atoms per CTA
    int bp = 0;       // padded batch (the MMA's N)
    int n_cta = 0;    // CTAs of the recurrence
    int smem = 0;     // shared memory of one recurrence CTA (the largest launched)
    int path = 0;     // 0 one layer, 1 layer pairs in one kernel, 2 per-layer chain, 3 layer by layer in batch chunks
    int chunks = 0;   // recurrence launches per layer
};
int gru_plan(int layers, int batch, int hidden, int reset_before, int num_sms, int smem_optin, GruPlan *g);
int gru_wave_launch(int T, int batch, int H, const float *gx_a, const uint16_t *U_a, const uint16_t *W_b,
                    const uint16_t *U_b, const float *b_a, const float *b_b, const float *h0_a,
                    const float *h0_b, float *out_a, float *out_b, uint16_t *hx_a, uint16_t *hx_b,
                    uint32_t *counter, DeviceState &ds, cudaStream_t stream);
int gru_stack_launch(int layers, int T, int batch, int hidden, int reset_before, const uint16_t *x,
                     const uint16_t *W, const uint16_t *U, const float *b, const float *h0, float *h_out,
                     DeviceState &ds, cudaStream_t stream);

int dwsep_launch(int N, int H, int W, int Cin, int Cout, const uint16_t *x, const uint16_t *dw,
                 const uint16_t *pw, float *out, DeviceState &ds, cudaStream_t s);
// The 3x3 depthwise stage alone: y (NHWC bf16) from x (NHWC bf16) and dw
// [3][3][C]; C a multiple of 8, pointers 16-byte aligned (checked by the caller).
int depthwise_launch(int N, int H, int W, int C, const uint16_t *x, const uint16_t *dw, uint16_t *y,
                     const DeviceState &ds, cudaStream_t s);
// out[4]: kernel (0 row ring, 1 per-pixel), image rows per tile, channel blocks, block width.
int dwsep_plan(int W, int Cin, int Cout, int smem_optin, int *out);

// Gated linear recurrence (forward uses h_out and h_last; backward h_in,
// dh_out, dh_last, dg and dh0).  Null pointers as in include/isam.h.
struct GlrDesc {
    int T, batch, hidden;
    int g_type, h_type;
    const void *g;
    const float *h0;
    const int32_t *lengths;
    void *h_out;
    float *h_last;
    const void *h_in;
    const void *dh_out;
    const float *dh_last;
    void *dg;
    float *dh0;
};
int glr_forward_launch(const GlrDesc &p, DeviceState &ds, cudaStream_t s);
int glr_backward_launch(const GlrDesc &p, DeviceState &ds, cudaStream_t s);
int glr_step_launch(int batch, int hidden, int slots, int g_type, const void *g, const int32_t *slot_ids,
                    const float *state, float *new_state, int h_type, void *h, cudaStream_t s);

// Gated feed-forward product (forward: h; backward: dh, workspace, dx, dW).
struct GluDesc {
    int T, D, F;
    int act;
    const uint16_t *x;
    const uint16_t *W;
    uint16_t *h;
    const uint16_t *dh;
    void *workspace;
    uint16_t *dx;
    uint16_t *dW;
};
int glu_forward_launch(const GluDesc &p, DeviceState &ds, cudaStream_t s);
size_t glu_backward_workspace(int T, int D, int F);
int glu_backward_launch(const GluDesc &p, DeviceState &ds, cudaStream_t s);

int w4_pack_launch(int N, int K, int group, const uint8_t *codes, const uint16_t *scales, uint8_t *tiled,
                   uint16_t *tiled_scales, cudaStream_t s);
int gemv_w4_launch(int M, int N, int K, int group, const uint16_t *x, const uint8_t *tiled, const uint16_t *scales,
                   float *y, DeviceState &ds, cudaStream_t s);

// Root-mean-square norm (y_type -1: y8 and y8_scales).
struct NormDesc {
    int T, D;
    int x_type, r_type, y_type;
    const void *x;
    const void *res;
    void *res_out;
    const float *w;
    float eps;
    void *y;
    uint8_t *y8;
    uint8_t *y8_scales;
};
int norm_forward_launch(const NormDesc &p, DeviceState &ds, cudaStream_t s);
struct NormBackDesc {
    int T, D;
    int r_type, g_type;
    const void *r;
    const float *w;
    float eps;
    const void *dy;
    const void *dres;
    float *workspace;
    void *dx;
    float *dw;
};
size_t norm_backward_workspace(int T, int D);
int norm_backward_launch(const NormBackDesc &p, DeviceState &ds, cudaStream_t s);

// Causal convolution (forward: lengths; one token: slots and slot_ids).
struct ConvDesc {
    int T, batch, C, width, slots;
    int x_type, y_type, silu;
    const void *x;
    int64_t x_stride;
    const float *w;
    const float *bias;
    const void *state;
    const int32_t *lengths;
    const int32_t *slot_ids;
    void *y;
    void *new_state;
};
int conv1d_forward_launch(const ConvDesc &p, DeviceState &ds, cudaStream_t s);
int conv1d_step_launch(const ConvDesc &p, cudaStream_t s);

// Selective scan (forward: state is h0, new_state h_last; one token: slots and slot_ids).
struct SsmDesc {
    int T, batch, C, N, slots;
    int u_type, p_type;
    const void *u;
    const void *dt;
    const float *dt_bias;
    const float *A;
    const void *B;
    const void *Cm;
    int64_t bc_stride;
    const float *D;
    const void *z;
    int64_t z_stride;
    const int32_t *lengths;
    const int32_t *slot_ids;
    const float *state;
    float *new_state;
    void *y;
};
int ssm_forward_launch(const SsmDesc &p, DeviceState &ds, cudaStream_t s);
int ssm_step_launch(const SsmDesc &p, cudaStream_t s);

struct BeamDesc {
    int batch, beams, V, count, l_type, eos;
    const void *logits;
    const float *scores;
    const uint8_t *finished;
    void *workspace;
    float *new_scores;
    int32_t *parents;
    int32_t *tokens;
    uint8_t *new_finished;
};
size_t beam_select_workspace(int batch, int beams, int V, int count);
int beam_select_launch(const BeamDesc &p, DeviceState &ds, cudaStream_t s);
int beam_reorder_launch(int layers, int batch, int beams, int slots, size_t row_bytes, const int32_t *parents,
                        const int32_t *slot_ids, const void *state, void *new_state, cudaStream_t s);

}  // namespace isam
