// The products of a mixture of experts: every token of a small batch goes through the top_k experts that its
// router chose, and their numbers are on the device.  A block reads the number of its expert and takes that
// expert's matrix and threshold; it is otherwise a block of the products of one matrix (Body::run, gemv_mlp.h), so a
// token's product with one expert is, up to the order of the sums, what the plain call gives on its matrix.
// What bounds it is memory (us at 50 %: one token's two of eight 4096 -> 2 x 14336 bf16 experts 39.5 to 41.5, 5.7 to 6.0
// TB/s), and for small experts the fullest unit and what a block does before its first row: the number is there 0.5 us after
// its start, the threshold 0.35 later (56 pairs of 2048 -> 2 x 768 mx4 in 13.9, 9.3 of them from the first row to the last,
// 46.8 MB at 5.0 TB/s: blocks of 512 columns beside blocks of 256, which end before them).  Asking for all
// thresholds at once, and for the activations before the number, took 0.3 to 1 us longer.
// Pairs are products of their own, in the tokens' order: an expert that several tokens chose is read for each of them
// (8 tokens, 8 of 8 bf16 experts of 4096 -> 2 x 14336: 7.57 GB fetched in 1155, where the union of the rows is 1.87 GB).
#pragma once

#include "gemv_common.h"
#include "gemv_mlp.h"

namespace teal {

template <class F>
struct ExpertArgs {
    typename F::Args a[kMaxMulti];     // of expert 0; the other experts' matrices follow each other
    const float *t[kMaxMulti];         // a threshold per expert
    float *y[kMaxMulti];
    int n[kMaxMulti];
    int tile_begin[kMaxMulti + 1];     // of one (token, expert) pair
    int count;
    const int *idx;                    // [tokens][top_k]
    int experts, top_k;
    int m, ks, tile_cols, splits;
    float *partial;
    Meeting meet;
};

// A threshold in device memory has not been checked: a negative one or a NaN counts as zero.  (A negative one would keep
// the zeros past the end of a slice, more than the list has room for.)  An infinite one stays: nothing is above it.
__device__ __forceinline__ float expert_threshold(const float *t, int e) { return fmaxf(t[e], 0.f); }

// Gate and up: y_k[pair] = s_{t_k[e]}(x[token]) W_k[e]^T, e = idx[pair], pair = token * top_k + slot.  A pair
// without an expert (a number out of range) gets zeros.  Grid: tiles of a pair, slices, pairs.
template <class Body, int LPR>
__global__ __launch_bounds__(8 * 64) void sparse_experts_kernel(ExpertArgs<typename Body::Format> ea,
                                                                const __half *__restrict__ X)
{
    typedef typename Body::Format F;
    trace_mark(0);
    const int pair = blockIdx.z, gtile = blockIdx.x, s = blockIdx.y;
    const int e = ea.idx[pair];
    int first = 0, n = ea.n[0], n_before = 0, n_total = ea.n[0];
    typename F::Args a = ea.a[0];
    float *y = ea.y[0];
    const float *t = ea.t[0];
#pragma unroll
    for (int j = 1; j < kMaxMulti; ++j) {
        const bool here = j < ea.count && gtile >= ea.tile_begin[j];
        n_before += here ? ea.n[j - 1] : 0;
        n_total += ea.n[j];                                       // 0 past the last matrix
        first = here ? ea.tile_begin[j] : first;
        n = here ? ea.n[j] : n;
        y = here ? ea.y[j] : y;
        t = here ? ea.t[j] : t;
        F::select(a, ea.a[j], here);
    }
    const int tile = gtile - first;
    y += (size_t)pair * n;
    if ((unsigned)e >= (unsigned)ea.experts) {
        if (s == 0)
            for (int c = threadIdx.x; c < ea.tile_cols; c += 8 * 64)
                if (tile * ea.tile_cols + c < n) store_coherent(y + tile * ea.tile_cols + c, 0.f);
        return;
    }
    F::expert(a, e, ea.m, n);
    Body::template run<LPR>(a, HalfSource{X + (size_t)(pair / ea.top_k) * ea.m}, expert_threshold(t, e),
                            ea.partial + ((size_t)pair * n_total + n_before) * ea.splits, ea.meet,
                            pair * ea.tile_begin[kMaxMulti] + gtile, y, ea.m, n, ea.ks, tile, s, ea.tile_cols,
                            ea.splits, NoReport{});
    trace_mark(6);
}

// What meets in a token's output: the slices of all its experts, each counted with the router's weight.
struct ExpertSum {
    int slot, splits, top_k;
    float weight;
    float t;                      // of one of the token's experts: what is on the grid has to be the same for all
    __device__ __forceinline__ int slice(int s) const { return slot * splits + s; }
    __device__ __forceinline__ int slices(int) const { return top_k * splits; }
    __device__ __forceinline__ float grid_threshold(float) const { return t; }
    __device__ __forceinline__ float sum(float v) const { return weight * v; }
};

// W_down: y[token] = sum over its experts of weight[pair] * s_{t[e]}(h[pair]) W[e]^T, h = fp16(SiLU(gate) * up) formed
// in the kernel.  A pair without an expert adds nothing.  Grid: tiles, slices of a pair, pairs.
template <class Body, int LPR>
__global__ __launch_bounds__(8 * 64) void sparse_experts_down_kernel(ExpertArgs<typename Body::Format> ea,
                                                                     const float *__restrict__ gate,
                                                                     const float *__restrict__ up,
                                                                     const float *__restrict__ weight)
{
    typedef typename Body::Format F;
    trace_mark(0);
    const int pair = blockIdx.z, tile = blockIdx.x;
    const int token = pair / ea.top_k, slot = pair - token * ea.top_k;
    const int e = ea.idx[pair], e0 = ea.idx[pair - slot], n = ea.n[0];
    const bool has = (unsigned)e < (unsigned)ea.experts;
    typename F::Args a = ea.a[0];
    F::expert(a, has ? e : 0, ea.m, n);
    // without an expert nothing survives
    const float t = has ? expert_threshold(ea.t[0], e) : __builtin_inff();
    const ExpertSum join{slot, ea.splits, ea.top_k, has ? weight[pair] : 0.f,
                         (unsigned)e0 < (unsigned)ea.experts ? expert_threshold(ea.t[0], e0) : 0.f};
    const SwigluSource h{gate + (size_t)pair * ea.m, up + (size_t)pair * ea.m};
    Body::template run<LPR>(a, h, t, ea.partial + (size_t)token * n * ea.top_k * ea.splits, ea.meet,
                            token * (int)gridDim.x + tile, ea.y[0] + (size_t)token * n, ea.m, n, ea.ks, tile,
                            (int)blockIdx.y, ea.tile_cols, ea.splits, NoReport{}, join);
    trace_mark(6);
}

// Host side, for shapes with 8 wavefronts and 4 loads per batch.
template <class Body, class SetArgs>
hipError_t launch_experts(const ExpertHostArgs &h, const GemvShape &sh, hipStream_t stream, SetArgs set_args)
{
    typedef typename Body::Format F;
    const GemvGeometry g = gemv_geometry(h.m, h.n[0], sh, F::kElemsPerLane, 64);
    ExpertArgs<F> ea{};
    for (int k = 0; k < kMaxMulti; ++k) {
        ea.tile_begin[k + 1] = ea.tile_begin[k];
        if (k >= h.count) continue;
        set_args(ea.a[k], h.W[k], h.scale ? h.scale[k] : nullptr);
        ea.t[k] = h.t[k];
        ea.y[k] = h.y[k];
        ea.n[k] = h.n[k];
        ea.tile_begin[k + 1] += (h.n[k] + g.tile_cols - 1) / g.tile_cols;
    }
    ea.count = h.count;
    ea.idx = h.idx;
    ea.experts = h.experts;
    ea.top_k = h.top_k;
    ea.m = h.m;
    ea.ks = g.ks;
    ea.tile_cols = g.tile_cols;
    ea.splits = g.splits;
    ea.partial = h.partial;
    const int tiles = ea.tile_begin[kMaxMulti], pairs = h.tokens * h.top_k;
    const dim3 grid(tiles, g.splits, pairs), block(8 * 64);
    if (h.weight) {
        ea.meet = meeting_of(h.counters, h.tokens * tiles, g.tile_cols, h.top_k * g.splits);
#define TEAL_LAUNCH_E(LPR)                                                                     \
    hipLaunchKernelGGL((sparse_experts_down_kernel<Body, LPR>), grid, block, g.lds, stream, ea, h.gate, h.up, h.weight)
        if constexpr (F::kElemsPerLane == 32) TEAL_LAUNCH_E(16);
        else if (sh.lanes_per_row == 64) TEAL_LAUNCH_E(64);
        else if (sh.lanes_per_row == 32) TEAL_LAUNCH_E(32);
        else TEAL_LAUNCH_E(16);
#undef TEAL_LAUNCH_E
        return hipGetLastError();
    }
    ea.meet = meeting_of(h.counters, pairs * tiles, g.tile_cols, g.splits);
#define TEAL_LAUNCH_E(LPR)                                                                     \
    hipLaunchKernelGGL((sparse_experts_kernel<Body, LPR>), grid, block, g.lds, stream, ea,     \
                       static_cast<const __half *>(h.x_f16))
    if constexpr (F::kElemsPerLane == 32) TEAL_LAUNCH_E(16);
    else if (sh.lanes_per_row == 64) TEAL_LAUNCH_E(64);
    else if (sh.lanes_per_row == 32) TEAL_LAUNCH_E(32);
    else TEAL_LAUNCH_E(16);
#undef TEAL_LAUNCH_E
    return hipGetLastError();
}

}  // namespace teal
