// Internal interface between the C-ABI layer (teal_api.cpp: argument checks,
// launch-shape choice) and the gfx950 kernels (*.hip).  Not installed.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mlp_schedule.h"

namespace teal {

constexpr int kMaxSplits = 128;     // most split-K blocks a caller may ask for (longer inputs force more)
constexpr int kMaxSlice = 4096;     // most input channels one block compacts (LDS list capacity)
constexpr int kMaxLongSlice = 8192; // the same for the launches that run without split-K on
                                    // padded rows (the list then takes 64 KiB of LDS)
constexpr int kMaxDim = 1 << 24;    // largest m or n accepted
constexpr int kMaxMatrices = 4;     // matrices per fused launch
constexpr int kMinTile = 64;        // narrowest output tile of any kernel variant
constexpr int kMaxNormInput = 16384; // longest hidden state the fused normalisation takes
constexpr int kMaxBatch = 8;        // rows of a small batch (Section 5.4.4)
constexpr int kMaxSliceBatch = 2048;  // most input channels one block compacts for a batch
constexpr int kMaxLongSliceBatch = 4096;   // the same where that runs without split-K in one round of blocks
// Head of the workspace: the column words of a launch, or one arrival counter per output tile (zero between calls).
constexpr size_t kCounterBytes = (size_t)(kMaxDim / kMinTile) * sizeof(int);
constexpr int kCounterLineInts = 32;    // counters 128 bytes apart while the area has room
constexpr int kMaxSpacedTiles = (int)(kCounterBytes / (kCounterLineInts * sizeof(int)));
// The survivor report follows the counters: kReportHeaderInts ints that start with one
// total per matrix of the call, then kMaxMatrices rows of per-split counts.
constexpr int kReportHeaderInts = 64;

// How one sparse GEMV is laid over the chip.
struct GemvShape {
    int lanes_per_row;   // 64, 32, 16 or 8 lanes read one weight row per load (16 bytes each)
    int splits;          // blocks along the input dimension
    int tile_cols;       // output columns per block; 0 = lanes_per_row * elements per lane
    int waves;           // wavefronts per block (4, 8 or 16)
    int unroll;          // row loads per batch, two batches in flight per wavefront (4 or 8; 4 with 16 waves)
};

bool gemv_shape_supported(const GemvShape &s);

// Each returns the HIP status of its launches; all are asynchronous on `stream`.
hipError_t launch_sparsify(const void *x_f16, int m, float t, uint8_t *mask,
                           int32_t *idx, int32_t *count, hipStream_t stream);

hipError_t launch_gemv_bf16(const void *Wt, const void *x_f16, float t, float *y,
                            int m, int n, float *partial, int *counters,
                            const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_bf16_swiglu(const void *Wt, const float *gate, const float *up, float t,
                                   float *y, int m, int n, float *partial, int *counters,
                                   const GemvShape &shape, hipStream_t stream);

// The grouped bf16 launch with its shared input formed from the hidden state h before the
// normalisation layer and the layer's weights gamma.  8 <= m <= 16384, m % 8 == 0; shapes
// with 8 wavefronts, 4 loads per batch and 16, 32 or 64 lanes per row.
hipError_t launch_gemv_bf16_rmsnorm_multi(int count, const void *const *Wt, const int *row_pitch,
                                          const float *t, float *const *y, const int *n,
                                          const float *h, const float *gamma, float eps, int m,
                                          float *partial, int *counters, const GemvShape &sh,
                                          hipStream_t stream);
hipError_t launch_rmsnorm_f16(const float *h, const float *gamma, float eps, void *x_f16, int m,
                              hipStream_t stream);
hipError_t launch_swiglu_f16(const float *gate, const float *up, void *h_f16, int m,
                             hipStream_t stream);

hipError_t launch_gemv_bf16_multi(int count, const void *const *Wt, const int *row_pitch,
                                  const float *t, float *const *y, const int *n,
                                  const void *x_f16, int m, float *partial, int *counters,
                                  const GemvShape &sh, hipStream_t stream);

// Up to kMaxStackGroups grouped calls of one weight format that do not depend on each other,
// in one launch.  Shapes with 8 wavefronts, 4 loads per batch and the format's lanes per row.
constexpr int kMaxStackGroups = 16;
struct StackGroupDesc {
    int count;                 // matrices of the group, 1..kMaxMatrices
    const void *const *Wt;
    const void *const *scale;  // quantised formats; NULL for bf16
    const float *t;
    float *const *y;
    const int *n;
    const void *x_f16;
    int m;
    float *partial;            // the group's own partial rows and counters
    int *counters;
    GemvShape shape;
};
hipError_t launch_gemv_bf16_stack(int groups, const StackGroupDesc *g, hipStream_t stream);
hipError_t launch_gemv_w8_stack(int groups, const StackGroupDesc *g, hipStream_t stream);
hipError_t launch_gemv_w4_stack(int groups, const StackGroupDesc *g, hipStream_t stream);

// Small batch (Section 5.4.4).  The slice of a block, ceil(m / splits) rounded up to 64,
// must not exceed kMaxLongSliceBatch.
bool gemv_batch_shape_supported(int batch, const GemvShape &s);

hipError_t launch_gemv_bf16_batch(const void *Wt, const void *X_f16, int batch, float t, float *Y,
                                  int m, int n, float *partial, int *counters,
                                  const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_bf16_batch_multi(int count, const void *const *Wt, const float *t,
                                        float *const *Y, const int *n, const void *X_f16,
                                        int batch, int m, float *partial, int *counters,
                                        const GemvShape &shape, hipStream_t stream);

hipError_t launch_sparsify_batch(const void *X_f16, int batch, int m, float t, uint8_t *mask,
                                 int32_t *idx, int32_t *count, hipStream_t stream);

hipError_t launch_gemv_w8(const int8_t *Wq, const void *scale_f16, const void *x_f16,
                          float t, float *y, int m, int n, float *partial, int *counters,
                          const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_w8_multi(int count, const int8_t *const *Wq, const int *row_pitch,
                                const void *const *scale_f16, const float *t, float *const *y,
                                const int *n, const void *x_f16, int m, float *partial,
                                int *counters, const GemvShape &sh, hipStream_t stream);

hipError_t launch_gemv_w8_swiglu(const int8_t *Wq, const void *scale_f16, const float *gate,
                                 const float *up, float t, float *y, int m, int n, float *partial,
                                 int *counters, const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_w8_rmsnorm_multi(int count, const int8_t *const *Wq, const int *row_pitch,
                                        const void *const *scale_f16, const float *t,
                                        float *const *y, const int *n, const float *h,
                                        const float *gamma, float eps, int m, float *partial,
                                        int *counters, const GemvShape &sh, hipStream_t stream);

hipError_t launch_gemv_w4(const uint8_t *Wq, const void *scale_f16, const void *x_f16,
                          float t, float *y, int m, int n, float *partial, int *counters,
                          const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_w4_swiglu(const uint8_t *Wq, const void *scale_f16, const float *gate,
                                 const float *up, float t, float *y, int m, int n, float *partial,
                                 int *counters, const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_w4_rmsnorm_multi(int count, const uint8_t *const *Wq,
                                        const void *const *scale_f16, const float *t,
                                        float *const *y, const int *n, const float *h,
                                        const float *gamma, float eps, int m, float *partial,
                                        int *counters, const GemvShape &shape, hipStream_t stream);

hipError_t launch_gemv_w4_multi(int count, const uint8_t *const *Wq, const void *const *scale_f16,
                                const float *t, float *const *y, const int *n, const void *x_f16,
                                int m, float *partial, int *counters, const GemvShape &shape,
                                hipStream_t stream);

// Microscaled 4-bit weights: [m][n / 2] bytes of codes, a scale byte per channel and block of 32 outputs in tiles
// of 8 channels by 16 blocks (gemv_mx4.hip).  Shapes with 16 lanes per row, 8 wavefronts, 4 loads per batch.
constexpr int kMx4TileBytes = 128;
__host__ __device__ constexpr int mx4_scale_tiles(int n) { return (n + 511) / 512; }
__host__ __device__ constexpr size_t mx4_scale_bytes(int m, int n)
{
    return (size_t)((m + 7) / 8) * mx4_scale_tiles(n) * kMx4TileBytes;
}
hipError_t launch_pack_mx4(const void *W_rowmajor, uint8_t *Wq, uint8_t *scale, int m, int n, hipStream_t stream);
hipError_t launch_unpack_mx4(const uint8_t *Wq, const uint8_t *scale, void *W_rowmajor, int m, int n,
                             hipStream_t stream);
hipError_t launch_gemv_mx4(const uint8_t *Wq, const uint8_t *scale, const void *x_f16, float t, float *y, int m,
                           int n, float *partial, int *counters, const GemvShape &shape, hipStream_t stream);
hipError_t launch_gemv_mx4_swiglu(const uint8_t *Wq, const uint8_t *scale, const float *gate, const float *up,
                                  float t, float *y, int m, int n, float *partial, int *counters,
                                  const GemvShape &shape, hipStream_t stream);
hipError_t launch_gemv_mx4_multi(int count, const uint8_t *const *Wq, const uint8_t *const *scale, const float *t,
                                 float *const *y, const int *n, const void *x_f16, int m, float *partial,
                                 int *counters, const GemvShape &shape, hipStream_t stream);
hipError_t launch_gemv_mx4_rmsnorm_multi(int count, const uint8_t *const *Wq, const uint8_t *const *scale,
                                         const float *t, float *const *y, const int *n, const float *h,
                                         const float *gamma, float eps, int m, float *partial, int *counters,
                                         const GemvShape &shape, hipStream_t stream);

// The experts a router chose, for a small batch of tokens (gemv_experts.h).  With `weight` the W_down step of the
// experts (gate and up in, one matrix, y[tokens][n]), else count matrices on x (y_k[tokens][top_k][n_k]).
struct ExpertHostArgs {
    int count;
    const void *const *W;          // of expert 0 each
    const void *const *scale;      // microscaled weights, else NULL
    const float *const *t;         // device arrays [experts]
    float *const *y;
    const int *n;
    int experts, tokens, top_k;
    const int *idx;                // device, [tokens][top_k]
    const void *x_f16;
    const float *weight, *gate, *up;
    int m;
    float *partial;
    int *counters;
};
hipError_t launch_experts_bf16(const ExpertHostArgs &h, const GemvShape &sh, hipStream_t stream);
hipError_t launch_experts_mx4(const ExpertHostArgs &h, const GemvShape &sh, hipStream_t stream);

constexpr int kMaxExperts = 1024;      // of a router
constexpr int kMaxExpertGroups = 64;
constexpr int kMaxTopK = 32;           // experts per token
struct RouteHostArgs {
    const float *logits, *bias;
    bool sigmoid, renormalise;
    int tokens, experts, groups, top_groups, group_top, top_k;
    float scaling;
    int *idx;
    float *weight;
};
hipError_t launch_route_experts(const RouteHostArgs &h, hipStream_t stream);

// Products of many rows (gemm_w8.hip, grouped_experts.hip).
constexpr int kMaxRowSum = 1 << 17;    // channels whose sum of products of 8-bit integers fits int32
constexpr int kMaxPairs = 1 << 24;     // (token, expert) pairs of a grouped call
__host__ __device__ constexpr int quantized_pitch(int m) { return (m + 127) / 128 * 128; }
struct GemmShape {
    int bm, bn;          // rows and columns of a block's tile
    int splits;          // blocks along the sum
};
constexpr int kMaxSlicedRows = 128;    // of a tile whose sum is cut into slices
struct GemmW8HostArgs {
    int count;
    const int8_t *const *W;
    const void *const *scale;
    float *const *y;
    const int *n;
    const int8_t *Q;
    const float *row_scale;
    int rows, m;
    int *counters, *partial;
};
hipError_t launch_quantize_rows(const void *X, bool bf16, int rows, int m, float t, int8_t *Q, float *scale,
                                hipStream_t stream);
hipError_t launch_quantize_rows_swiglu(const float *gate, const float *up, int rows, int m, float t, int8_t *Q,
                                       float *scale, hipStream_t stream);
hipError_t launch_gemm_w8(const GemmW8HostArgs &h, const GemmShape &sh, hipStream_t stream);

struct GroupedHostArgs {
    const void *W[2];              // of expert 0: gate and up, or W_down
    const uint8_t *scale[2];       // microscaled weights, else NULL
    int experts, tokens, top_k;
    const int *order, *start;      // device: pairs in the experts' order, first place of each expert's
    const int *idx;                // device [tokens][top_k]
    const float *weight;
    const void *rows;              // X [tokens][m] (gate and up) or H [tokens * top_k][m] (W_down), bf16
    void *out;                     // H or y
    int m, n;
    float *partial;                // W_down: a row per pair
    int slab_cols;                 // columns that it has room for
};
hipError_t launch_arrange_experts(const int *idx, int tokens, int top_k, int experts, int *order, int *start,
                                  int *counts, hipStream_t stream);
constexpr int kMaxArrangeChunks = 128;
hipError_t launch_grouped_gate_up(const GroupedHostArgs &h, hipStream_t stream);
hipError_t launch_grouped_down(const GroupedHostArgs &h, hipStream_t stream);

// The MLP of a block in one launch (Appendix A.3): gate and up from x, then W_down on
// SiLU(gate) . up, the blocks of W_down waiting for the gate / up tiles they read.
struct MlpLaunch {
    GemvShape gu, down;          // 8 wavefronts, 4 loads per batch
    int phase_tiles;             // gate / up tiles per phase of the grid order; 0 = one phase
    int extra_lds;               // dynamic LDS requested beyond need (fewer blocks per unit)
    unsigned spin_limit;         // polls before a waiting block gives up
};
struct MlpHostArgs {
    const void *W_gate, *W_up, *W_down;
    const void *scale_gate, *scale_up, *scale_down;   // quantised formats, else NULL
    const void *x_f16;
    float t_gate, t_up, t_down;
    float *gate, *up, *y;
    int m, f, d;                 // model width in, MLP width, model width out
    int gu_pitch, down_pitch;    // elements between rows of W_gate / W_up and of W_down; 0 = f, d
    float *partial_gu;
    int *counters_gu;            // head of the gate / up region of the workspace
    float *partial_d;
    int *counters_d;             // head of the W_down region
    int *control;                // kMlpControlBytes: status word, one readiness counter per W_down block
};
constexpr int kMlpMaxConsumers = 4096;       // most thread blocks of the W_down product
constexpr size_t kMlpControlBytes = 128 * (size_t)(1 + kMlpMaxConsumers);
// The grid of such a launch for a weight format (16, 8 or 4 bits); false if the shapes do
// not give a launchable grid.
bool mlp_grid_of(int weight_bits, const MlpLaunch &L, int m, int f, int d, MlpGrid &grid);
hipError_t launch_mlp_bf16(const MlpHostArgs &h, const MlpLaunch &L, hipStream_t stream);
hipError_t launch_mlp_w8(const MlpHostArgs &h, const MlpLaunch &L, hipStream_t stream);
hipError_t launch_mlp_w4(const MlpHostArgs &h, const MlpLaunch &L, hipStream_t stream);

hipError_t launch_abs_histogram(const void *x_f16, size_t count, unsigned long long *hist,
                                hipStream_t stream);

hipError_t launch_histogram_thresholds(const unsigned long long *hist, const double *p, int np,
                                       float *t_out, hipStream_t stream);

hipError_t launch_stream_read(const void *buf, size_t bytes, int blocks, uint32_t match,
                              uint32_t *sink, hipStream_t stream);

hipError_t launch_pack_bf16(const void *W_rowmajor, void *Wt, int m, int n, int pitch,
                            hipStream_t stream);

}  // namespace teal
