// y = s_t(x) W^T for microscaled 4-bit weights: blocks of 32 neighbouring outputs of one input channel share a
// power of two, W[j][i] = level(code(i, j)) * 2^(scale(i, j / 32) - 127), level one of 0, 0.5, 1, 1.5, 2, 3, 4, 6
// and a sign.  The blocks lie along the outputs, not along the sum: a channel that is dropped takes its scales
// with it, and a lane's 16 bytes are one block with one scale.
//
// Scales are stored in tiles of 8 channels by 16 blocks, 128 bytes: what an output tile of 512 columns reads of
// a channel's scales are 16 bytes, and a row of them would be a line that the tiles beside it, on other XCDs,
// fetch too; of a tile of scales the line's other bytes belong to the next channels of the same block.
#include "gemv_common.h"
#include "gemv_experts.h"
#include "gemv_mlp.h"

namespace teal {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

struct FmtMx4 {
    static constexpr int kElemsPerLane = 32;   // 16 bytes = 32 codes, one block
    static constexpr int kBitsPerElem = 4;
    // scales of any size, as bf16 weights
    static __device__ __forceinline__ int grid_unit(float t) { return grid_unit_bf16(t); }
    struct Args {
        const void *W;
        const unsigned char *scale;
    };
    static __device__ __forceinline__ void select(Args &a, const Args &b, bool take)
    {
        a.W = take ? b.W : a.W;
        a.scale = take ? b.scale : a.scale;
    }
    // The same matrix of expert e, [m][n] matrices one behind the other.
    static __device__ __forceinline__ void expert(Args &a, int e, int m, int n)
    {
        a.W = static_cast<const unsigned char *>(a.W) + (size_t)e * m * (n / 2);
        a.scale += (size_t)e * mx4_scale_bytes(m, n);
    }
    static __device__ __forceinline__ void read_now(const Args (&a)[4])
    {
        asm volatile("" ::"s"(a[0].scale), "s"(a[1].scale), "s"(a[2].scale), "s"(a[3].scale));
    }
    struct ColumnScale {};
    static __device__ __forceinline__ ColumnScale column_scale(const Args &, int) { return {}; }
    static __device__ __forceinline__ float finish(float sum, ColumnScale) { return sum; }
};

constexpr int kMx4Waves = 8;
constexpr int kMx4Unroll = 4;
constexpr int kMx4Lanes = 16;

// The products run on the matrix cores.  v_mfma_f32_16x16x32_bf16: a lane's 8 values of A are 8 of the 32 places of
// the sum, its lane % 16 the row, lane / 16 the quarter.  A lane's 16 bytes are one block: 4 instructions per word
// turn its 8 codes into 8 bf16 numbers, exact and already scaled by the block's power of two, and they go in as
// they come, 16 blocks (rows of A) by 4 channels (quarters).  B separates the columns again: it is zero except
// where the place in the word equals the column, B[8 g + j][j] = the activation of quarter g's channel.  Columns j and
// j + 8 of B take two parts of it: an fp16 number has 11 significant bits, 8 of them in the first bf16 number and
// the rest in the second, so the products are exact; they are added in fp32, four channels at a time (against
// binary64 as near as a chain of FMAs, for sizes 2^24 apart too).  Of the instruction for 4-bit floats
// itself, which would need no conversion, the sums lose bits: products far below the largest one of an
// instruction are cut to 17 bits or so, 5e-5 of the result where 2e-7 is what fp32 gives.
// What bounds it is memory, and the ends of a launch where there is little to read: 42 vector and 4 matrix instructions
// per 16-byte load issue in 31 and 12 % of the time of 2 x 28672 x 8192 at 50 % (24.4 us, 125 MB, 7 TB/s between the
// first row and the last; 26.7 us with 16 conversions and 32 FMAs per load).
struct Bf16Parts {
    static constexpr bool kMagnitude = false;
    // Channel of the slice, and the two parts of x; of an infinity the second is zero.
    static __device__ __forceinline__ int2 entry(int, int offset, float x)
    {
        const unsigned first = __float_as_uint(x) & 0xFFFF0000u;
        const float rest = x == __uint_as_float(first) ? 0.f : x - __uint_as_float(first);
        return make_int2(offset, (int)__builtin_amdgcn_perm(__float_as_uint(rest), first, 0x07060302u));
    }
};

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

template <int U>
struct Mx4Batch {
    u32x4 v[U];
    unsigned sc[U];
    unsigned x[U];
};

// Work of one block: output tile `tile` (tile_cols columns, at most 512) x K-slice `s` (ks channels).  16 lanes share a
// row, four rows per wavefront load; the wavefronts take equal contiguous shares of the compacted list, two
// batches of loads in flight (as stream_rows).  Returns how many of the tile's outputs this thread wrote.
template <int LPR, int WAVES, int U, class XS, class Report = SurvivorReport, class Join = OneProduct>
__device__ __forceinline__ int mx4_block(const FmtMx4::Args &a, const XS &x, float t, float *partial,
                                          const Meeting &meet, int gtile, float *y, int m, int n, int ks, int tile,
                                          int s, int tile_cols, int splits, const Report &report,
                                          const Join &join = Join{})
{
    using F = FmtMx4;
    constexpr int EPL = F::kElemsPerLane;
    static_assert(LPR == 16, "the rows of the matrix instruction");
    constexpr int R = 4;                          // rows per wavefront load
    extern __shared__ __align__(16) unsigned char smem[];
    int2 *list = reinterpret_cast<int2 *>(smem);
    float *red = reinterpret_cast<float *>(smem + (size_t)ks * sizeof(int2));
    __shared__ int counts[kCompactInts];

    asm volatile("" ::"s"(a.W), "s"(a.scale), "s"(partial), "s"(meet.counters), "s"(y));   // as in gemv_block
    const int k0 = s * ks;                       // a multiple of 64, so of the 8 channels of a tile of scales
    const int k1 = min(m, k0 + ks);
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int group_excl;
    int cnt = 0;
    bool compacted = false;
    if constexpr (XS::kPlainHalf) {
        if (k1 - k0 <= kPrivateSlice) {         // block-uniform: short slices need no barrier
            cnt = compact_slice_private<Bf16Parts>(x.x, t, k0, k1, w, WAVES, list, group_excl);
            compacted = true;
        }
    }
    if (!compacted) cnt = compact_slice<WAVES, XS, Bf16Parts>(x, t, k0, k1, list, counts, group_excl);

    trace_mark(2);
    if constexpr (Report::kOn) {
        if (tile == 0 && !meet.word_step && threadIdx.x == (WAVES - 1) * 64) report_slice(report, s, splits, cnt);
    }
    const int lane = threadIdx.x & 63;
    const int l = lane & 15, g = lane >> 4;
    const int col0 = tile * tile_cols;
    const int col = lane_column<EPL>(col0, tile_cols, n, l);
    // A channel's codes in units of 16 bytes, 8 channels' scales in bytes: with the channel of a slice both are products
    // of less than 24 bits each, below 2^32 (n below 2^24, slices of at most 4096 channels).
    static_assert(kMaxSlice <= 4096, "offsets inside a slice fit 32 bits");
    const unsigned row_units = (unsigned)(n / 32);
    const unsigned tiles_bytes = (unsigned)mx4_scale_tiles(n) * kMx4TileBytes;
    const unsigned char *lane_base =
        static_cast<const unsigned char *>(a.W) + (size_t)k0 * (unsigned)(n / 2) + col / 2;
    const unsigned char *scale_base =
        a.scale + (size_t)(k0 / 8) * tiles_bytes + col / 512 * kMx4TileBytes + col / 32 % 16;
    // B: this lane's column takes place l % 8 of a word's 8, the first (l < 8) or second part of the activation
    unsigned pick[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const unsigned part = l < 8 ? 0x0100u : 0x0302u;
        pick[q] = l % 8 / 2 != q ? 0x0C0C0C0Cu : l % 2 ? part << 16 | 0x0C0Cu : 0x0C0C0000u | part;
    }

    f32x4 acc[4];                                 // [word]: blocks 4 g + r, output 8 * word + l % 8, part l / 8
#pragma unroll
    for (int q = 0; q < 4; ++q) acc[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    cnt = __builtin_amdgcn_readfirstlane(cnt);
    int start, mine;
    wave_share(cnt, w, WAVES, start, mine);
    if (mine > 0) {
        const int last = mine - 1;
        const int batches = (mine + U * R - 1) / (U * R);
        // slots past the end of the share repeat the last row with a zero multiplier
        auto issue = [&](Mx4Batch<U> &b, int batch) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int e = (batch * U + u) * R + g;
                const int2 ent = list[start + min(e, last)];
                const unsigned i = (unsigned)ent.x;
                b.x[u] = e <= last ? (unsigned)ent.y : 0u;
                b.v[u] = load_stream16(lane_base + ((size_t)__umul24(i, row_units) << 4));
                b.sc[u] = scale_base[__umul24(i >> 3, tiles_bytes) + (i << 4 & 0x70u)];
            }
        };
        auto consume = [&](const Mx4Batch<U> &b) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float sc = __uint_as_float(b.sc[u] << 23);
                u32x4 B;
#pragma unroll
                for (int q = 0; q < 4; ++q) B[q] = __builtin_amdgcn_perm(b.x[u], b.x[u], pick[q]);
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    u32x4 A;
                    A[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[u][q], sc, 0));
                    A[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[u][q], sc, 1));
                    A[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[u][q], sc, 2));
                    A[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(b.v[u][q], sc, 3));
                    acc[q] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, A),
                                                                     __builtin_bit_cast(bf16x8, B), acc[q], 0, 0, 0);
                }
            }
        };
        Mx4Batch<U> b0, b1;
        issue(b0, 0);
        int it = 0;
        for (; it + 2 < batches; it += 2) {
            issue(b1, it + 1);
            consume(b0);
            issue(b0, it + 2);
            consume(b1);
        }
        if (it + 1 < batches) {
            issue(b1, it + 1);
            consume(b0);
            consume(b1);
        } else {
            consume(b0);
        }
    }
    trace_mark(3);
    trace_mark_thread(1, (WAVES - 1) * 64);
    // The lanes l < 8 take the first two words of a block and give the other two to the lane 8 further, which holds
    // the other part.
    float *row = red + w * combine_row<EPL, LPR> + (l < 8 ? 0 : 16) + l % 8;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const float own = l < 8 ? acc[q][r] : acc[q + 2][r], give = l < 8 ? acc[q + 2][r] : acc[q][r];
            const float got = __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(
                0, (int)__float_as_uint(give), 0x128 /* row_ror:8 */, 0xF, 0xF, false));
            row[EPL * (4 * g + r) + 8 * q] = own + got;
        }
    return block_finish<F, LPR, WAVES>(red, partial, meet, gtile, y, tile, col0, tile_cols, join.slice(s),
                                       join.slices(splits), n, a, report, cnt, join.grid_threshold(t), join);
}

struct Mx4Body {
    typedef FmtMx4 Format;
    template <int LPR, class XS, class Report, class Join = OneProduct>
    static __device__ __forceinline__ int run(const FmtMx4::Args &a, const XS &x, float t, float *partial,
                                               const Meeting &meet, int gtile, float *y, int m, int n, int ks,
                                               int tile, int s, int tile_cols, int splits, const Report &report,
                                               const Join &join = Join{})
    {
        return mx4_block<LPR, kMx4Waves, kMx4Unroll>(a, x, t, partial, meet, gtile, y, m, n, ks, tile, s, tile_cols,
                                                     splits, report, join);
    }
};

__global__ __launch_bounds__(kMx4Waves * 64) void sparse_gemv_mx4_kernel(
    FmtMx4::Args a, const __half *__restrict__ x, float t, float *partial, Meeting meet, float *y, int m, int n,
    int ks, int tile_cols, int splits)
{
    trace_mark(0);
    const int tile = blockIdx.x;
    Mx4Body::run<kMx4Lanes>(a, HalfSource{x}, t, partial, meet, tile, y, m, n, ks, tile, blockIdx.y, tile_cols, splits,
                            survivor_report(meet.counters, 0, splits));
    trace_mark(6);
}

// The input formed from the two products that precede W_down, as in sparse_gemv_swiglu_kernel.
__global__ __launch_bounds__(kMx4Waves * 64) void sparse_gemv_mx4_swiglu_kernel(
    FmtMx4::Args a, const float *__restrict__ gate, const float *__restrict__ up, float t, float *partial,
    Meeting meet, float *y, int m, int n, int ks, int tile_cols, int splits)
{
    trace_mark(0);
    const int tile = blockIdx.x;
    Mx4Body::run<kMx4Lanes>(a, SwigluSource{gate, up}, t, partial, meet, tile, y, m, n, ks, tile, blockIdx.y, tile_cols,
                            splits, survivor_report(meet.counters, 0, splits));
}

// Several matrices that read the same state; the block finds its matrix as in multi_block.
template <class XS>
__device__ __forceinline__ void mx4_multi_block(const MultiArgs<FmtMx4> &ma, const XS &x, float *partial,
                                                const Meeting &meet, int m, int ks, int tile_cols, int splits,
                                                int gtile, int s)
{
    trace_mark(0);
    int k = 0, first = 0, n = ma.n[0];
    size_t partial_off = 0;
    FmtMx4::Args a = ma.a[0];
    float *y = ma.y[0];
    float t = ma.t[0];
    asm volatile("" ::"s"(ma.y[0]), "s"(ma.y[1]), "s"(ma.y[2]), "s"(ma.y[3]), "s"(ma.n[0]), "s"(ma.n[1]),
                 "s"(ma.n[2]), "s"(ma.n[3]), "s"(ma.t[0]), "s"(ma.t[1]), "s"(ma.t[2]), "s"(ma.t[3]),
                 "s"(ma.a[0].W), "s"(ma.a[1].W), "s"(ma.a[2].W), "s"(ma.a[3].W), "s"(ma.tile_begin[4]),
                 "s"(partial), "s"(meet.counters), "s"(splits));
    FmtMx4::read_now(ma.a);
#pragma unroll
    for (int j = 1; j < kMaxMulti; ++j) {
        const bool here = j < ma.count && gtile >= ma.tile_begin[j];
        partial_off += here ? (size_t)splits * ma.n[j - 1] : 0;
        k = here ? j : k;
        first = here ? ma.tile_begin[j] : first;
        n = here ? ma.n[j] : n;
        y = here ? ma.y[j] : y;
        t = here ? ma.t[j] : t;
        FmtMx4::select(a, ma.a[j], here);
    }
    Mx4Body::run<kMx4Lanes>(a, x, t, partial + partial_off, meet, gtile, y, m, n, ks, gtile - first, s, tile_cols,
                            splits, survivor_report(meet.counters, k, splits));
    trace_mark(6);
}

__global__ __launch_bounds__(kMx4Waves * 64) void sparse_gemv_mx4_multi_kernel(
    MultiArgs<FmtMx4> ma, const __half *__restrict__ x, float *partial, Meeting meet, int m, int ks, int tile_cols,
    int splits)
{
    asm volatile("" ::"s"(x));                 // as in multi_block
    mx4_multi_block(ma, HalfSource{x}, partial, meet, m, ks, tile_cols, splits, (int)blockIdx.x, (int)blockIdx.y);
}

__global__ __launch_bounds__(kNormWaves * 64) void sparse_gemv_mx4_rmsnorm_multi_kernel(
    MultiArgs<FmtMx4> ma, const float *__restrict__ h, const float *__restrict__ gamma, float eps, double inv_m,
    float *partial, Meeting meet, int m, int ks, int tile_cols, int splits)
{
    static_assert(kMx4Waves == kNormWaves, "the normalisation's scale is formed by a block of kNormWaves");
    __shared__ double wave_sums[kMaxNormChunks * kNormWaves];
    asm volatile("" ::"s"(h), "s"(gamma), "s"(eps), "s"(inv_m));      // as in multi_block
    mx4_multi_block(ma, RmsnormSource{h, gamma, m, inv_m, eps, wave_sums}, partial, meet, m, ks, tile_cols, splits,
                    (int)blockIdx.x, (int)blockIdx.y);
}

static bool mx4_shape_ok(const GemvShape &sh)
{
    return sh.lanes_per_row == kMx4Lanes && sh.waves == kMx4Waves && sh.unroll == kMx4Unroll && sh.splits >= 1 &&
           sh.tile_cols > 0 && sh.tile_cols % FmtMx4::kElemsPerLane == 0 &&
           sh.tile_cols <= kMx4Lanes * FmtMx4::kElemsPerLane;
}

hipError_t launch_gemv_mx4(const uint8_t *Wq, const uint8_t *scale, const void *x_f16, float t, float *y, int m,
                           int n, float *partial, int *counters, const GemvShape &sh, hipStream_t stream)
{
    if (!mx4_shape_ok(sh)) return hipErrorInvalidValue;
    const GemvGeometry g = gemv_geometry(m, n, sh, FmtMx4::kElemsPerLane, 64);
    const Meeting meet = meeting_of(counters, g.tiles, g.tile_cols, g.splits);
    hipLaunchKernelGGL(sparse_gemv_mx4_kernel, dim3(g.tiles, g.splits), dim3(kMx4Waves * 64), g.lds, stream,
                       (FmtMx4::Args{Wq, scale}), static_cast<const __half *>(x_f16), t, partial, meet, y, m, n, g.ks,
                       g.tile_cols, g.splits);
    return hipGetLastError();
}

hipError_t launch_gemv_mx4_swiglu(const uint8_t *Wq, const uint8_t *scale, const float *gate, const float *up,
                                  float t, float *y, int m, int n, float *partial, int *counters,
                                  const GemvShape &sh, hipStream_t stream)
{
    if (!mx4_shape_ok(sh)) return hipErrorInvalidValue;
    const GemvGeometry g = gemv_geometry(m, n, sh, FmtMx4::kElemsPerLane, 64);
    const Meeting meet = meeting_of(counters, g.tiles, g.tile_cols, g.splits);
    hipLaunchKernelGGL(sparse_gemv_mx4_swiglu_kernel, dim3(g.tiles, g.splits), dim3(kMx4Waves * 64), g.lds, stream,
                       (FmtMx4::Args{Wq, scale}), gate, up, t, partial, meet, y, m, n, g.ks, g.tile_cols, g.splits);
    return hipGetLastError();
}

static MultiArgs<FmtMx4> mx4_multi_args(int count, const uint8_t *const *Wq, const uint8_t *const *scale,
                                        const float *t, float *const *y, const int *n, int tile_cols)
{
    MultiArgs<FmtMx4> ma{};
    ma.count = count;
    for (int k = 0; k < count; ++k) {
        ma.a[k] = FmtMx4::Args{Wq[k], scale[k]};
        ma.y[k] = y[k];
        ma.t[k] = t[k];
        ma.n[k] = n[k];
        ma.tile_begin[k + 1] = ma.tile_begin[k] + (n[k] + tile_cols - 1) / tile_cols;
    }
    return ma;
}

hipError_t launch_gemv_mx4_multi(int count, const uint8_t *const *Wq, const uint8_t *const *scale, const float *t,
                                 float *const *y, const int *n, const void *x_f16, int m, float *partial,
                                 int *counters, const GemvShape &sh, hipStream_t stream)
{
    if (!mx4_shape_ok(sh)) return hipErrorInvalidValue;
    const GemvGeometry g = gemv_geometry(m, n[0], sh, FmtMx4::kElemsPerLane, 64);
    const MultiArgs<FmtMx4> ma = mx4_multi_args(count, Wq, scale, t, y, n, g.tile_cols);
    const int tiles = ma.tile_begin[count];
    const Meeting meet = meeting_of(counters, tiles, g.tile_cols, g.splits);
    hipLaunchKernelGGL(sparse_gemv_mx4_multi_kernel, dim3(tiles, g.splits), dim3(kMx4Waves * 64), g.lds, stream, ma,
                       static_cast<const __half *>(x_f16), partial, meet, m, g.ks, g.tile_cols, g.splits);
    return hipGetLastError();
}

hipError_t launch_gemv_mx4_rmsnorm_multi(int count, const uint8_t *const *Wq, const uint8_t *const *scale,
                                         const float *t, float *const *y, const int *n, const float *h,
                                         const float *gamma, float eps, int m, float *partial, int *counters,
                                         const GemvShape &sh, hipStream_t stream)
{
    if (m < 8 || m > kMaxNormDim || m % 8 != 0 || !mx4_shape_ok(sh)) return hipErrorInvalidValue;
    const GemvGeometry g = gemv_geometry(m, n[0], sh, FmtMx4::kElemsPerLane, 64);
    const MultiArgs<FmtMx4> ma = mx4_multi_args(count, Wq, scale, t, y, n, g.tile_cols);
    const int tiles = ma.tile_begin[count];
    const Meeting meet = meeting_of(counters, tiles, g.tile_cols, g.splits);
    hipLaunchKernelGGL(sparse_gemv_mx4_rmsnorm_multi_kernel, dim3(tiles, g.splits), dim3(kNormWaves * 64), g.lds,
                       stream, ma, h, gamma, eps, 1.0 / m, partial, meet, m, g.ks, g.tile_cols, g.splits);
    return hipGetLastError();
}

hipError_t launch_experts_mx4(const ExpertHostArgs &h, const GemvShape &sh, hipStream_t stream)
{
    if (!mx4_shape_ok(sh)) return hipErrorInvalidValue;
    return launch_experts<Mx4Body>(h, sh, stream, [](FmtMx4::Args &a, const void *W, const void *scale) {
        a.W = W;
        a.scale = static_cast<const unsigned char *>(scale);
    });
}

// ---- the format itself: bf16 weights in and out ----
//
// A thread block has 128 channels by 128 outputs, a wavefront one block of 32 outputs of all of them, a lane two
// neighbouring channels: the 32 rows of W[n][m] are read (written) 256 bytes at a time, a block's 32 weights are in
// one lane's registers, and the conversions of the hardware take and give two outputs at once.  (8192 x 28672:
// 105 us to mx4, 5.7 TB/s, and 85 us back, 7.0; turned through LDS two bytes at a time both together took 715.)  Codes
// and scales pass through LDS so that a channel's 64 bytes of codes and 4 scales travel together: 16 bytes and one byte
// per lane and wavefront were four times the requests.  Large weights are read with four channels to a lane, 512 bytes
// of a row (8192 x 28672 111 -> 105 us; 4096 x 1024 would be 64 blocks instead of 256).
constexpr int kMx4PackRows = 128, kMx4PackWaves = 4;

// Two bf16 values of neighbouring channels; a row of W begins on an even address only.
typedef unsigned Mx4Pair __attribute__((aligned(2)));

// W past the caches, where that pays.  Written, if rows begin on cache lines, so that a wavefront writes whole ones
// (unpack of 8192 x 28672 123 -> 89 us, 4096 x 14336 23.7 -> 22.6; where they do not, 5001 x 3424, it would be 10.6 ->
// 17.8).  Read, if moreover W is larger than the last cache and so cannot come from it (pack of 8192 x 28672
// 126 -> 111 us; 4096 x 14336 just written 22 -> 29).
constexpr size_t kLastCache = (size_t)256 << 20;
inline bool mx4_whole_lines(const void *W, int m) { return m % 64 == 0 && (reinterpret_cast<uintptr_t>(W) & 127) == 0; }

template <int ROWS>
struct Mx4PackTile {
    u32x4 codes[ROWS][kMx4PackWaves + 1];             // one of padding: lanes two channels apart do not meet in a bank
    unsigned char scale[ROWS][kMx4PackWaves];
};

// The channel of the tile whose codes thread `t` moves between LDS and memory in pass k: 64 channels a pass, four threads to
// a channel, a block each.  (Two passes for tiles of 128 channels, four for the wide ones of pack_mx4_kernel.)
__device__ __forceinline__ int mx4_tile_channel(int t, int k) { return k * 64 + t / kMx4PackWaves; }

__device__ __forceinline__ size_t mx4_scale_place(int i, int b, int n)
{
    return ((size_t)(i / 8) * mx4_scale_tiles(n) + b / 16) * kMx4TileBytes + i % 8 * 16 + b % 16;
}

template <bool PAST, int PAIRS>
__global__ __launch_bounds__(kMx4PackWaves * 64) void pack_mx4_kernel(const uint16_t *__restrict__ W,
                                                                      uint8_t *__restrict__ Wq,
                                                                      uint8_t *__restrict__ scale, int m, int n,
                                                                      int tiles_m)
{
    constexpr int CH = 2 * PAIRS, ROWS = 64 * CH;
    typedef unsigned Load __attribute__((ext_vector_type(PAIRS), aligned(2)));
    __shared__ Mx4PackTile<ROWS> tile;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i0 = blockIdx.x % tiles_m * ROWS, b0 = blockIdx.x / tiles_m * kMx4PackWaves;
    const int i = i0 + CH * lane, blocks = n / 32;
    if (b0 + w < blocks) {                                  // wavefront-uniform
        unsigned v[32][PAIRS];                              // the first channel of a pair in the lower half
        const uint16_t *first = W + (size_t)(b0 + w) * 32 * m;
        if (i0 + ROWS <= m) {
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                const Load *p = reinterpret_cast<const Load *>(first + (size_t)r * m + i);
                const Load x = PAST ? __builtin_nontemporal_load(p) : *p;
#pragma unroll
                for (int c = 0; c < PAIRS; ++c) v[r][c] = x[c];
            }
        } else {
#pragma unroll
            for (int r = 0; r < 32; ++r)
#pragma unroll
                for (int c = 0; c < PAIRS; ++c) {
                    const uint16_t *p = first + (size_t)r * m + i + 2 * c;
                    const int at = i + 2 * c;
                    v[r][c] = at + 1 < m ? *reinterpret_cast<const Mx4Pair *>(p) : at < m ? *p : 0u;
                }
        }
        typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
        u16x2 largest[PAIRS] = {};
#pragma unroll
        for (int r = 0; r < 32; ++r)
#pragma unroll
            for (int c = 0; c < PAIRS; ++c)
                largest[c] = __builtin_elementwise_max(largest[c], __builtin_bit_cast(u16x2, v[r][c] & 0x7FFF7FFFu));
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            // floor(log2) of the largest magnitude; below 2^-125 the scale is the smallest one anyway
            const unsigned most = largest[c / 2][c % 2];
            const int s = most >= 0x7F80u ? 255 : max((int)(most >> 7) - 2, 0);
            const float x = __uint_as_float((unsigned)s << 23);
            u32x4 codes = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                unsigned word = 0;
#define TEAL_PAIR(B)                                                                           \
    do {                                                                                       \
        const unsigned two = __builtin_amdgcn_perm(v[8 * q + 2 * B + 1][c / 2], v[8 * q + 2 * B][c / 2], \
                                                   c % 2 ? 0x07060302u : 0x05040100u);         \
        word = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(word, __builtin_bit_cast(bf16x2, two), x, B); \
    } while (0)
                TEAL_PAIR(0);
                TEAL_PAIR(1);
                TEAL_PAIR(2);
                TEAL_PAIR(3);
#undef TEAL_PAIR
                codes[q] = s == 255 ? 0u : word;
            }
            tile.codes[CH * lane + c][w] = codes;
            tile.scale[CH * lane + c][w] = i + c < m ? (unsigned char)s : 0;
        }
    } else {
#pragma unroll
        for (int c = 0; c < CH; ++c) tile.scale[CH * lane + c][w] = 0;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < CH; ++k) {
        const int c = mx4_tile_channel(threadIdx.x, k), b = b0 + (int)threadIdx.x % kMx4PackWaves;
        if (i0 + c < m && b < blocks)
            *reinterpret_cast<u32x4 *>(Wq + ((size_t)(i0 + c) * blocks + b) * 16) =
                tile.codes[c][threadIdx.x % kMx4PackWaves];
    }
    // zeros past the last channel and block of a tile of scales
    static_assert(ROWS <= kMx4PackWaves * 64, "a thread per channel");
    const int c = threadIdx.x;
    if (c < ROWS && i0 + c < (m + 7) / 8 * 8)
        for (int b = b0; b < (b0 + kMx4PackWaves < blocks ? b0 + kMx4PackWaves : mx4_scale_tiles(n) * 16);
             b += kMx4PackWaves)
            *reinterpret_cast<unsigned *>(scale + mx4_scale_place(i0 + c, b, n)) =
                b == b0 ? *reinterpret_cast<const unsigned *>(tile.scale[c]) : 0u;
}

template <bool PAST>
__global__ __launch_bounds__(kMx4PackWaves * 64) void unpack_mx4_kernel(const uint8_t *__restrict__ Wq,
                                                                        const uint8_t *__restrict__ scale,
                                                                        uint16_t *__restrict__ W, int m, int n,
                                                                        int tiles_m)
{
    __shared__ Mx4PackTile<kMx4PackRows> tile;
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i0 = blockIdx.x % tiles_m * kMx4PackRows, b0 = blockIdx.x / tiles_m * kMx4PackWaves;
    const int blocks = n / 32;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int c = mx4_tile_channel(threadIdx.x, k), b = b0 + (int)threadIdx.x % kMx4PackWaves;
        if (i0 + c < m && b < blocks)
            tile.codes[c][threadIdx.x % kMx4PackWaves] =
                *reinterpret_cast<const u32x4 *>(Wq + ((size_t)(i0 + c) * blocks + b) * 16);
    }
    if (threadIdx.x < kMx4PackRows && i0 + (int)threadIdx.x < m)
        *reinterpret_cast<unsigned *>(tile.scale[threadIdx.x]) =
            *reinterpret_cast<const unsigned *>(scale + mx4_scale_place(i0 + (int)threadIdx.x, b0, n));
    __syncthreads();
    if (b0 + w >= blocks) return;
    const int i = i0 + 2 * lane;
    if (i >= m) return;
    // two outputs of one channel each, by channel
    unsigned two[2][16];
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const u32x4 codes = tile.codes[2 * lane + c][w];
        const float x = __uint_as_float((unsigned)tile.scale[2 * lane + c][w] << 23);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
#define TEAL_PAIR(B)                                                                           \
    two[c][4 * q + B] =                                                                        \
        __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[q], x, B))
            TEAL_PAIR(0);
            TEAL_PAIR(1);
            TEAL_PAIR(2);
            TEAL_PAIR(3);
#undef TEAL_PAIR
        }
    }
    uint16_t *first = W + (size_t)(b0 + w) * 32 * m + i;
    const bool both = i + 1 < m;
#pragma unroll
    for (int r = 0; r < 32; ++r) {
        const unsigned v = __builtin_amdgcn_perm(two[1][r / 2], two[0][r / 2], r % 2 ? 0x07060302u : 0x05040100u);
        Mx4Pair *p = reinterpret_cast<Mx4Pair *>(first + (size_t)r * m);
        if (PAST) __builtin_nontemporal_store(v, p);                  // an even number of channels
        else if (both) *p = v;
        else first[(size_t)r * m] = (uint16_t)v;
    }
}

// Tiles of the channels, fastest in the grid, and all tiles.
struct Mx4LayoutGrid {
    int tiles_m;
    long long tiles;
    Mx4LayoutGrid(int m, int n, int rows)
        : tiles_m((m + rows - 1) / rows),
          tiles((long long)tiles_m * ((n / 32 + kMx4PackWaves - 1) / kMx4PackWaves))
    {
    }
};

hipError_t launch_pack_mx4(const void *W, uint8_t *Wq, uint8_t *scale, int m, int n, hipStream_t stream)
{
    const bool past = mx4_whole_lines(W, m) && (size_t)m * n * sizeof(uint16_t) > kLastCache;
    const Mx4LayoutGrid g(m, n, past ? 2 * kMx4PackRows : kMx4PackRows);
    if (g.tiles > 0x7fffffffLL) return hipErrorInvalidValue;      // more weights than a GPU has bytes
    hipLaunchKernelGGL((past ? pack_mx4_kernel<true, 2> : pack_mx4_kernel<false, 1>), dim3((unsigned)g.tiles),
                       dim3(kMx4PackWaves * 64), 0, stream, static_cast<const uint16_t *>(W), Wq, scale, m, n, g.tiles_m);
    return hipGetLastError();
}

hipError_t launch_unpack_mx4(const uint8_t *Wq, const uint8_t *scale, void *W, int m, int n, hipStream_t stream)
{
    const Mx4LayoutGrid g(m, n, kMx4PackRows);
    if (g.tiles > 0x7fffffffLL) return hipErrorInvalidValue;
    hipLaunchKernelGGL(mx4_whole_lines(W, m) ? unpack_mx4_kernel<true> : unpack_mx4_kernel<false>,
                       dim3((unsigned)g.tiles), dim3(kMx4PackWaves * 64), 0, stream, Wq, scale,
                       static_cast<uint16_t *>(W), m, n, g.tiles_m);
    return hipGetLastError();
}

}  // namespace teal

#ifdef TEAL_TRACE_BLOCKS
extern "C" int teal_trace_read_mx4(unsigned long long *host, size_t count) { return teal::read_trace(host, count); }
#endif
