// A mixture of experts for many tokens: the pairs of a token and an expert that a router chose, sorted by expert, and the
// products of every expert with the rows that are its own.
#include "gemm_tile.h"
#include "grouped_shape.h"
#include "teal_internal.h"

namespace teal {

namespace {

// ---- the pairs in the experts' order ----
//
// A counting sort that keeps the pairs of an expert in their order: how many of each expert every chunk of pairs has, then
// places.  A wavefront takes a contiguous part of a chunk, 64 pairs at a time; the lanes with the same expert find each
// other by a ballot per bit of its number.

constexpr int kArrangeWaves = 16;
constexpr int kArrangeThreads = kArrangeWaves * 64;

struct ArrangeArgs {
    const int *idx;
    int pairs, experts;
    int chunk;               // pairs of a block, a multiple of kArrangeThreads
    int *order, *start;
    int *counts;             // [chunks][experts + 1]; the last one of those without an expert
};

// The expert of pair p; `experts` for none.
__device__ __forceinline__ int key_of(const ArrangeArgs &a, int p)
{
    const unsigned e = (unsigned)a.idx[p];
    return e < (unsigned)a.experts ? (int)e : a.experts;
}

// Lanes of the wavefront whose key is this lane's, among those of `live`.
__device__ __forceinline__ unsigned long long lanes_alike(int key, int bits, unsigned long long live)
{
    unsigned long long same = live;
    for (int b = 0; b < bits; ++b) {
        const unsigned long long set = __ballot(key >> b & 1);
        same &= (key >> b & 1) ? set : ~set;
    }
    return same;
}

// 64 pairs a step, kSteps steps of a wavefront's pairs [begin, end) at a time: their keys, `experts` past the end.
constexpr int kSteps = 4;
__device__ __forceinline__ void load_keys(const ArrangeArgs &a, int begin, int end, int (&key)[kSteps])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int s = 0; s < kSteps; ++s) key[s] = key_of(a, max(min(begin + 64 * s + lane, end - 1), 0));
}

__global__ __launch_bounds__(kArrangeThreads) void count_experts_kernel(ArrangeArgs a)
{
    __shared__ int counted[kMaxExperts + 1];
    const int keys = a.experts + 1;
    for (int e = threadIdx.x; e < keys; e += kArrangeThreads) counted[e] = 0;
    __syncthreads();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int begin = blockIdx.x * a.chunk, end = min(a.pairs, begin + a.chunk);
    for (int p = begin + w * 64 * kSteps; p < end; p += kArrangeThreads * kSteps) {
        int key[kSteps];
        load_keys(a, p, end, key);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            if (p + 64 * s + lane < end) atomicAdd(&counted[key[s]], 1);
    }
    __syncthreads();
    for (int e = threadIdx.x; e < keys; e += kArrangeThreads) a.counts[blockIdx.x * keys + e] = counted[e];
}

// One block a chunk.  ALONE: there is one chunk, which the block counts itself.
template <bool ALONE>
__global__ __launch_bounds__(kArrangeThreads) void place_pairs_kernel(ArrangeArgs a)
{
    // of each expert: the pairs of the wavefronts before, then the next place of the wavefront's own
    __shared__ int at[kArrangeWaves][kMaxExperts + 1];
    __shared__ int sums[kArrangeWaves];
    const int keys = a.experts + 1;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int begin = blockIdx.x * a.chunk, end = min(a.pairs, begin + a.chunk);
    const int share = a.chunk / kArrangeThreads * 64;
    const int p0 = begin + w * share, p1 = min(end, p0 + share);
    int key[kSteps];
    if (p0 < p1) load_keys(a, p0, p1, key);

    // Thread e has expert e (and the last one the key of no expert, where there are as many experts as threads).
    static_assert(kMaxExperts == kArrangeThreads, "an expert a thread, and one more key");
    int total = 0, before = 0;           // of all chunks, of the chunks before this one
    const int e = threadIdx.x;
    if constexpr (!ALONE) {
        if (e < keys) {
            // several on their way together: one after the other each would take a trip to memory
            const int chunks = gridDim.x;
            for (int c0 = 0; c0 < chunks; c0 += 32) {
                int n[32];
#pragma unroll
                for (int c = 0; c < 32; ++c) n[c] = a.counts[min(c0 + c, chunks - 1) * keys + e];
#pragma unroll
                for (int c = 0; c < 32; ++c) {
                    total += c0 + c < chunks ? n[c] : 0;
                    before += c0 + c < (int)blockIdx.x ? n[c] : 0;
                }
            }
        }
    }
    for (int k = lane; k < keys; k += 64) at[w][k] = 0;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    for (int p = p0; p < p1; p += 64 * kSteps) {
        if (p > p0) load_keys(a, p, p1, key);
#pragma unroll
        for (int s = 0; s < kSteps; ++s)
            if (p + 64 * s + lane < p1) atomicAdd(&at[w][key[s]], 1);
    }
    __syncthreads();
    if (ALONE && e < keys)
        for (int v = 0; v < kArrangeWaves; ++v) total += at[v][e];
    const int upto = wave_inclusive_scan(total);
    if (lane == 63) sums[w] = upto;
    __syncthreads();
    int base = 0;
    for (int v = 0; v < kArrangeWaves; ++v) base += v < w ? sums[v] : 0;
    const int first = base + upto - total;
    if (blockIdx.x == 0 && e < keys) a.start[e] = first;           // (of no expert: where the experts' pairs end)
    if (e < keys) {
        int next = first + before;
        for (int v = 0; v < kArrangeWaves; ++v) {
            const int n = at[v][e];
            at[v][e] = next;
            next += n;
        }
    }
    if (keys > kArrangeThreads && e == kArrangeThreads - 1) {      // the pairs without an expert, behind all others
        const int none = kArrangeThreads;
        int next = first + total;
        if (blockIdx.x == 0) a.start[none] = next;
        if constexpr (!ALONE)
            for (int c = 0; c < (int)blockIdx.x; ++c) next += a.counts[c * keys + none];
        for (int v = 0; v < kArrangeWaves; ++v) {
            const int n = at[v][none];
            at[v][none] = next;
            next += n;
        }
    }
    __syncthreads();

    const int bits = 32 - __builtin_clz(a.experts);
    for (int p = p0; p < p1; p += 64 * kSteps) {                   // wavefront-uniform
        if (share > 64 * kSteps) load_keys(a, p, p1, key);         // (else they are still there)
#pragma unroll
        for (int s = 0; s < kSteps; ++s) {
            const bool live = p + 64 * s + lane < p1;
            const unsigned long long same = lanes_alike(key[s], bits, __ballot(live));
            const int rank = lanes_below(same);
            if (live) {
                const int place = at[w][key[s]] + rank;
                // (idx may not change meanwhile; if it does, nothing outside `order` is written)
                if ((unsigned)place < (unsigned)a.pairs) a.order[place] = p + 64 * s + lane;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (live && rank == 0) at[w][key[s]] += __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
    }
}

// ---- the products ----

struct GroupedArgs {
    const unsigned char *W[2];         // of expert 0
    const unsigned char *scale[2];
    int experts, pairs, top_k;
    const int *order, *start;
    const unsigned char *rows;         // X or H
    void *out;                         // H, or a row of partial sums per pair
    int m, n;
    int col_begin, col_tiles;          // of this launch
    int out_pitch;                     // of the partial rows
};

// The tile of a block: an expert, its pairs' places and a part of its columns.  The tiles of an expert follow each other,
// those of all experts are spread evenly over the XCDs.  What `start` holds is not checked: places are cut to what there is.
struct GroupTile {
    int expert, row0, row_end, col_tile;
};
template <int BM>
__device__ __forceinline__ bool find_tile(const GroupedArgs &a, GroupTile &t)
{
    const int lane = threadIdx.x & 63;
    const int each = (a.experts + 63) / 64;
    const int e0 = lane * each, e1 = min(a.experts, e0 + each);
    auto place = [&](int e) { return min(max(a.start[e], 0), a.pairs); };
    int mine = 0;
    for (int e = e0; e < e1; ++e) mine += (max(place(e + 1) - place(e), 0) + BM - 1) / BM;
    const int upto = wave_inclusive_scan(mine);
    const int row_tiles = __builtin_amdgcn_readlane(upto, 63);
    const long long tiles = (long long)row_tiles * a.col_tiles;
    const int each_xcd = (int)((tiles + kXcds - 1) / kXcds);
    const int xcd = blockIdx.x % kXcds, in_xcd = blockIdx.x / kXcds;
    const long long at = (long long)xcd * each_xcd + in_xcd;
    if (in_xcd >= each_xcd || at >= tiles) return false;
    // the expert whose row tiles, times the column tiles, have place `at`
    const int row_at = (int)(at / a.col_tiles);
    const unsigned long long past = __ballot(upto > row_at);
    const int owner = __builtin_ctzll(past);                // there is one: row_at < row_tiles
    int before = upto - mine, e = e0, begin = 0, end = 0, count = 0;
    for (; e < e1; ++e) {
        begin = place(e);
        end = max(place(e + 1), begin);
        count = (end - begin + BM - 1) / BM;
        if (before + count > row_at) break;
        before += count;
    }
    t.expert = __builtin_amdgcn_readlane(e, owner);
    begin = __builtin_amdgcn_readlane(begin, owner);
    t.row_end = __builtin_amdgcn_readlane(end, owner);
    before = __builtin_amdgcn_readlane(before, owner);
    count = __builtin_amdgcn_readlane(count, owner);
    const int2 tile = tile_at((int)(at - (long long)before * a.col_tiles), count, a.col_tiles);
    t.row0 = begin + tile.x * BM;
    t.col_tile = tile.y;
    return true;
}

// The pair at place p of the experts' order; `order` is not checked either.
__device__ __forceinline__ int pair_at(const GroupedArgs &a, int p)
{
    const unsigned pair = (unsigned)a.order[p];
    return pair < (unsigned)a.pairs ? (int)pair : 0;
}

template <class F>
__device__ __forceinline__ size_t expert_bytes(int m, int n)
{
    return F::kMx4 ? (size_t)m * (n / 2) : (size_t)m * n * 2;
}

// SiLU(g) * u for a result of 8 bits, by the hardware's exponential and reciprocal: g / (1 + 2^(-g log2 e)) * u.  The product
// -g log2 e is off by 2^-24 of itself and its constant by 2^-26.1, so for g >= -87 the power by 87 (2^-24 + 2^-26.1) < 2^-17.2;
// the rest adds five steps of 2^-23: less than 2^-16 together.  Below that the reciprocal is no normal number (e^-87.3 is
// 2^-126) and the result may be zero.  (A tile of 256 x 256 has 64 values a thread: 9 us of 66 with a polynomial and a
// correctly rounded division.)
__device__ __forceinline__ float swiglu_fast(float g, float u)
{
    return g * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(g * -1.44269504f)) * u;
}

// H = bf16(SiLU(X W_gate[e]^T) * (X W_up[e]^T)), a row per place of the experts' order.
template <class F, class S>
__global__ __launch_bounds__(S::kThreads) void grouped_gate_up_kernel(GroupedArgs a)
{
    typedef TileProduct<F, S, 2> Product;
    __shared__ __align__(1024) unsigned char smem[Product::kLds];
    GroupTile t;
    if (!find_tile<S::BM>(a, t)) return;
    const int col0 = a.col_begin + t.col_tile * (S::BN / 2);
    Product p;
    p.begin(smem);
    if (p.multiplies()) p.begin_multiplying(col0, a.n);
    if (S::LOADERS == 0 || !p.multiplies())
        p.begin_loading(
            [&](int r) {
                return a.rows + (size_t)(pair_at(a, min(t.row0 + r, t.row_end - 1)) / a.top_k) * (2 * (size_t)a.m);
            },
            [&](int half) { return a.W[half] + t.expert * expert_bytes<F>(a.m, a.n); },
            [&](int half) { return a.scale[half] + t.expert * mx4_scale_bytes(a.m, a.n); }, col0, a.n);
    p.run(0, (a.m + F::kSlabRows - 1) / F::kSlabRows, a.m, t.row_end - t.row0);
    if (!p.multiplies()) return;
#pragma unroll
    for (int f = 0; f < S::NF / 2; ++f) {
        const int col = col0 + p.col_of(f);
        if (col >= a.n) continue;                     // n is a multiple of 8
#pragma unroll
        for (int i = 0; i < S::MF; ++i) {
            const int row = t.row0 + p.row_of(i);
            if (row < t.row_end) {
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                bf16x4 h;
#pragma unroll
                for (int r = 0; r < 4; ++r) h[r] = (__bf16)swiglu_fast(p.acc[i][f][r], p.acc[i][f + S::NF / 2][r]);
                *reinterpret_cast<bf16x4 *>(static_cast<__bf16 *>(a.out) + (size_t)row * a.n + col) = h;
            }
        }
    }
}

// H W_down[e]^T of every pair, in the pair's own row.
template <class F, class S>
__global__ __launch_bounds__(S::kThreads) void grouped_down_kernel(GroupedArgs a)
{
    typedef TileProduct<F, S, 1> Product;
    __shared__ __align__(1024) unsigned char smem[Product::kLds];
    GroupTile t;
    if (!find_tile<S::BM>(a, t)) return;
    const int col0 = a.col_begin + t.col_tile * S::BN;
    Product p;
    p.begin(smem);
    if (p.multiplies()) p.begin_multiplying(col0, a.n);
    if (S::LOADERS == 0 || !p.multiplies())
        p.begin_loading([&](int r) { return a.rows + (size_t)min(t.row0 + r, t.row_end - 1) * (2 * (size_t)a.m); },
                        [&](int) { return a.W[0] + t.expert * expert_bytes<F>(a.m, a.n); },
                        [&](int) { return a.scale[0] + t.expert * mx4_scale_bytes(a.m, a.n); }, col0, a.n);
    p.run(0, (a.m + F::kSlabRows - 1) / F::kSlabRows, a.m, t.row_end - t.row0);
    if (!p.multiplies()) return;
#pragma unroll
    for (int i = 0; i < S::MF; ++i) {
        const int row = t.row0 + p.row_of(i);
        if (row >= t.row_end) continue;
        float *const out = static_cast<float *>(a.out) + (size_t)pair_at(a, row) * a.out_pitch - a.col_begin;
#pragma unroll
        for (int f = 0; f < S::NF; ++f) {
            const int col = col0 + p.col_of(f);
            if (col < min(a.n, a.col_begin + a.out_pitch)) *reinterpret_cast<f32x4 *>(out + col) = p.acc[i][f];
        }
    }
}

// y[b] = sum over j of weight[b][j] * (row of pair (b, j)), j ascending, for those with an expert.
__global__ __launch_bounds__(256) void join_pairs_kernel(const float *partial, const int *idx, const float *weight,
                                                         int tokens, int top_k, int experts, int quads, int pitch,
                                                         float *y, int n, int col_begin)
{
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int token = (int)(at / quads), col = 4 * (int)(at % quads);
    if (token >= tokens) return;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int j = 0; j < top_k; ++j) {
        const int pair = token * top_k + j;
        if ((unsigned)idx[pair] >= (unsigned)experts) continue;
        const f32x4 v = *reinterpret_cast<const f32x4 *>(partial + (size_t)pair * pitch + col);
        const float w = weight[pair];
#pragma unroll
        for (int r = 0; r < 4; ++r) sum[r] = fmaf(w, v[r], sum[r]);
    }
    float *const to = y + (size_t)token * n + col_begin + col;
#pragma unroll
    for (int r = 0; r < 4; ++r) to[r] = sum[r];
}

// Blocks for all row tiles that the experts' pairs can make, times the column tiles.
unsigned grid_of(const GroupedArgs &a, int bm)
{
    const long long row_tiles = a.pairs / bm + (a.experts < a.pairs ? a.experts : a.pairs);
    const long long tiles = row_tiles * a.col_tiles;
    return (unsigned)((tiles + kXcds - 1) / kXcds * kXcds);
}

GroupedArgs grouped_args(const GroupedHostArgs &h)
{
    GroupedArgs a{};
    for (int k = 0; k < 2; ++k) {
        a.W[k] = static_cast<const unsigned char *>(h.W[k]);
        a.scale[k] = h.scale[k];
    }
    a.experts = h.experts;
    a.pairs = h.tokens * h.top_k;
    a.top_k = h.top_k;
    a.order = h.order;
    a.start = h.start;
    a.rows = static_cast<const unsigned char *>(h.rows);
    a.m = h.m;
    a.n = h.n;
    return a;
}

template <class F, class S>
struct GateUp {
    static hipError_t run(const GroupedHostArgs &h, hipStream_t stream)
    {
        GroupedArgs a = grouped_args(h);
        a.out = h.out;
        a.col_tiles = (h.n + S::BN / 2 - 1) / (S::BN / 2);
        hipLaunchKernelGGL((grouped_gate_up_kernel<F, S>), dim3(grid_of(a, S::BM)), dim3(S::kThreads), 0, stream, a);
        return hipGetLastError();
    }
};

template <class F, class S>
struct Down {
    static hipError_t run(const GroupedHostArgs &h, hipStream_t stream)
    {
        GroupedArgs a = grouped_args(h);
        a.out = h.partial;
        for (int col = 0; col < h.n; col += h.slab_cols) {
            const int cols = h.n - col < h.slab_cols ? h.n - col : h.slab_cols;
            a.col_begin = col;
            a.out_pitch = cols;
            a.col_tiles = (cols + S::BN - 1) / S::BN;
            hipLaunchKernelGGL((grouped_down_kernel<F, S>), dim3(grid_of(a, S::BM)), dim3(S::kThreads), 0, stream, a);
            const long long threads = (long long)h.tokens * (cols / 4);
            hipLaunchKernelGGL(join_pairs_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, stream, h.partial,
                               h.idx, h.weight, h.tokens, h.top_k, h.experts, cols / 4, cols, static_cast<float *>(h.out),
                               h.n, col);
        }
        return hipGetLastError();
    }
};

}  // namespace

hipError_t launch_arrange_experts(const int *idx, int tokens, int top_k, int experts, int *order, int *start,
                                  int *counts, hipStream_t stream)
{
    ArrangeArgs a{idx, tokens * top_k, experts, 0, order, start, counts};
    constexpr int kAlone = 8192;
    if (a.pairs <= kAlone) {
        a.chunk = (a.pairs + kArrangeThreads - 1) / kArrangeThreads * kArrangeThreads;
        hipLaunchKernelGGL(place_pairs_kernel<true>, dim3(1), dim3(kArrangeThreads), 0, stream, a);
        return hipGetLastError();
    }
    int chunks = (a.pairs + 4095) / 4096;
    if (chunks > kMaxArrangeChunks) chunks = kMaxArrangeChunks;
    a.chunk = ((a.pairs + chunks - 1) / chunks + kArrangeThreads - 1) / kArrangeThreads * kArrangeThreads;
    chunks = (a.pairs + a.chunk - 1) / a.chunk;
    hipLaunchKernelGGL(count_experts_kernel, dim3(chunks), dim3(kArrangeThreads), 0, stream, a);
    hipLaunchKernelGGL(place_pairs_kernel<false>, dim3(chunks), dim3(kArrangeThreads), 0, stream, a);
    return hipGetLastError();
}

namespace {

GroupedShape shape_of(const GroupedHostArgs &h, int cols)
{
    return grouped_shape(h.scale[0] != nullptr, (long long)h.tokens * h.top_k, h.experts, cols);
}

template <template <class, class> class Call>
hipError_t run_grouped(const GroupedHostArgs &h, GroupedShape s, hipStream_t stream)
{
    if (h.scale[0]) {
        if (s.bm == 32) return Call<WeightsMx4, TileShape<32, 128, 1, 4, 4, 4>>::run(h, stream);
        if (s.bm == 64) return Call<WeightsMx4, TileShape<64, 128, 1, 4, 3, 4>>::run(h, stream);
        // (with wavefronts that load beside them those of 256 x 256 would have 168 registers each, and be 6 % slower)
        return s.bn == 128 ? Call<WeightsMx4, TileShape<256, 128, 4, 1, 3, 4>>::run(h, stream)
                           : Call<WeightsMx4, TileShape<256, 256, 2, 4, 2>>::run(h, stream);
    }
    if (s.bm == 32) return Call<WeightsBf16, TileShape<32, 128, 1, 4, 3, 4>>::run(h, stream);
    if (s.bm == 64) return Call<WeightsBf16, TileShape<64, 128, 1, 4, 3, 4>>::run(h, stream);
    if (s.bm == 256) return Call<WeightsBf16, TileShape<256, 256, 2, 4, 2>>::run(h, stream);
    return s.bn == 128 ? Call<WeightsBf16, TileShape<128, 128, 2, 4, 4, 4>>::run(h, stream)
                       : Call<WeightsBf16, TileShape<128, 256, 2, 4, 3, 4>>::run(h, stream);
}

}  // namespace

hipError_t launch_grouped_gate_up(const GroupedHostArgs &h, hipStream_t stream)
{
    return run_grouped<GateUp>(h, shape_of(h, 2 * h.n), stream);
}

hipError_t launch_grouped_down(const GroupedHostArgs &h, hipStream_t stream)
{
    return run_grouped<Down>(h, shape_of(h, h.n), stream);
}

}  // namespace teal
