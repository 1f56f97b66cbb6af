// Products of many rows with 8-bit channel-wise quantised weights (Section 5.3 for the weights; a row of X is one token of
// a prompt or of a batch, thresholded like any input): rows to 8-bit integers with a scale each, and the product of
// integers, exact in int32 and scaled once per row and once per output channel.
#include "gemm_tile.h"
#include "teal_internal.h"

namespace teal {

namespace {

// ---- rows to 8-bit integers ----
//
// v = s_t(x), a = max |v| of the row, scale = a / 127, q = rint(127 v / a).  The quotient decides an integer, so it has to be
// the real one's rounding.  a = unit * 2^e with unit in [1/2, 1); p = 127 * 2^-e * v is exact, v has at most 11 significant bits
// and 127 seven.  y = fl(p / unit) by a rounded reciprocal and one correction (rem = p - y * unit exactly, y + rem / unit)
// is off by less than 2^-23 of itself.  A quotient of 0.49 or more is at least 2^-21 of itself away from the middle k + 1/2 of two
// integers, or there: it differs by (254 v - (2k + 1) a) / 2a, whose numerator is a whole multiple of the last place of v and
// whose denominator is below 2^12 last places of a.  Where it is there, rem / unit completes y to the quotient itself, which is
// representable.  Either way the rounding sees the side that the real quotient is on.  (Rows whose 2^-e is no
// binary32 number, and those with an infinity, go another way.)
// Memory bounds it, with few instructions a value: maxima of magnitudes as 16-bit integers, two at a time, and the rounding
// by the addition of 1.5 * 2^23, which leaves the integer in the low bits.  (4096 rows of 8192 bf16 in 30 us with
// maxima in binary32, a select for infinities and conversions to integers.)  A row stays in registers between its maximum
// and its integers.

struct RowsF16 {
    const unsigned short *x;
    static constexpr bool kBf16 = false;
};
struct RowsBf16 {
    const unsigned short *x;
    static constexpr bool kBf16 = true;
};
struct RowsSwiglu {                 // fp16(SiLU(gate) * up)
    const float *gate, *up;
    static constexpr bool kBf16 = false;
};

template <bool Bf16>
__device__ __forceinline__ float value_of(unsigned half_word)
{
    if constexpr (Bf16) return __uint_as_float(half_word << 16);
    else return __half2float(__ushort_as_half((unsigned short)half_word));
}

// 8 values from channel i on as 16-bit words, zeros from m on.
template <bool Wide, class Rows>
__device__ __forceinline__ u32x4 load_values(const Rows &r, size_t row, int i, int m)
{
    u32x4 v = {0u, 0u, 0u, 0u};
    if (i >= m) return v;
    const unsigned short *x = r.x + row * m + i;
    if constexpr (Wide) {
        v = *reinterpret_cast<const u32x4 *>(x);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const unsigned h = x[min(e, m - 1 - i)];
            v[e / 2] |= (i + e < m ? h : 0u) << 16 * (e % 2);
        }
    }
    return v;
}
template <bool Wide>
__device__ __forceinline__ u32x4 load_values(const RowsSwiglu &r, size_t row, int i, int m)
{
    u32x4 v = {0u, 0u, 0u, 0u};
    if (i >= m) return v;
    const float *gate = r.gate + row * m + i, *up = r.up + row * m + i;
    float g[8], u[8];
    if constexpr (Wide) {
#pragma unroll
        for (int e = 0; e < 8; e += 4) {
            *reinterpret_cast<f32x4 *>(g + e) = *reinterpret_cast<const f32x4 *>(gate + e);
            *reinterpret_cast<f32x4 *>(u + e) = *reinterpret_cast<const f32x4 *>(up + e);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            g[e] = gate[min(e, m - 1 - i)];
            u[e] = up[min(e, m - 1 - i)];
        }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const unsigned h = __half_as_ushort(__float2half_rn(swiglu_value(g[e], u[e])));
        v[e / 2] |= (i + e < m ? h : 0u) << 16 * (e % 2);
    }
    return v;
}

// One row per block: CHUNKS loads of 8 values per thread.
template <int THREADS, int CHUNKS, bool Wide, class Rows>
__global__ __launch_bounds__(THREADS) void quantize_rows_kernel(Rows rows, int m, int pitch, float t, int8_t *Q,
                                                                float *scale)
{
    const size_t row = blockIdx.x;
    u32x4 v[CHUNKS];
    if constexpr (std::is_same<Rows, RowsSwiglu>::value) {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) v[c] = load_values<Wide>(rows, row, (c * THREADS + (int)threadIdx.x) * 8, m);
    } else {
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c) v[c] = load_values<Wide, Rows>(rows, row, (c * THREADS + (int)threadIdx.x) * 8, m);
    }
    // the largest magnitude as a 16-bit pattern; beyond that of infinity there is a NaN, which does not count
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    constexpr unsigned kInfinity = Rows::kBf16 ? 0x7F80u : 0x7C00u;
    u16x2 most2 = {0, 0};
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
        for (int q = 0; q < 4; ++q)
            most2 = __builtin_elementwise_max(most2, __builtin_bit_cast(u16x2, v[c][q] & 0x7FFF7FFFu));
    unsigned top = max(most2[0], most2[1]);
    if (__ballot(top > kInfinity)) {                             // wavefront-uniform, and hardly ever
        top = 0;
#pragma unroll
        for (int c = 0; c < CHUNKS; ++c)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const unsigned h = v[c][e / 2] >> 16 * (e % 2) & 0x7FFFu;
                top = max(top, h > kInfinity ? 0u : h);
            }
    }
    for (int d = 32; d; d >>= 1) top = max(top, (unsigned)__shfl_xor((int)top, d));
    if constexpr (THREADS > 64) {
        __shared__ unsigned most[THREADS / 64];
        if ((threadIdx.x & 63) == 0) most[threadIdx.x / 64] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) top = max(top, most[w]);
    }
    float a = value_of<Rows::kBf16>(top);
    if (!(a > t)) a = 0.f;                         // nothing is kept
    if (threadIdx.x == 0) scale[row] = a / 127.f;
    const bool infinite = a == __builtin_inff();
    int exponent;
    const float unit = frexpf(infinite || a == 0.f ? 1.f : a, &exponent);
    const float inverse = 1.f / unit;
    const float factor = ldexpf(127.f, -exponent);               // of ordinary rows
    constexpr float kRound = 12582912.f;
    const bool ordinary = !infinite && exponent > -100 && exponent < 100;        // block-uniform
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c) {
        const int i = (c * THREADS + (int)threadIdx.x) * 8;
        unsigned q[8];
        if (ordinary) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = value_of<Rows::kBf16>(v[c][e / 2] >> 16 * (e % 2) & 0xFFFFu);
                const float p = (fabsf(x) > t ? x : 0.f) * factor;
                const float y = p * inverse;
                q[e] = __float_as_uint(fmaf(fmaf(-y, unit, p), inverse, y) + kRound);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = value_of<Rows::kBf16>(v[c][e / 2] >> 16 * (e % 2) & 0xFFFFu);
                const float z = fabsf(x) > t ? x : 0.f;
                const float p = ldexpf(z, -exponent) * 127.f;
                const float y = p * inverse;
                float r = fmaf(fmaf(-y, unit, p), inverse, y);
                if (infinite) r = fabsf(z) == __builtin_inff() ? copysignf(127.f, z) : 0.f;
                q[e] = __float_as_uint(r + kRound);
            }
        }
        // the low bytes of four
        uint2 out;
        out.x = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0C0C0400u),
                                      __builtin_amdgcn_perm(q[1], q[0], 0x0C0C0400u), 0x05040100u);
        out.y = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[7], q[6], 0x0C0C0400u),
                                      __builtin_amdgcn_perm(q[5], q[4], 0x0C0C0400u), 0x05040100u);
        if (i < pitch) *reinterpret_cast<uint2 *>(Q + row * pitch + i) = out;
    }
}

template <bool Wide, class Rows>
void quantize(const Rows &r, int rows, int m, float t, int8_t *Q, float *scale, hipStream_t stream)
{
    const int pitch = quantized_pitch(m);
    const dim3 grid((unsigned)rows);
#define TEAL_QUANTIZE(THREADS, CHUNKS)                                                                              \
    hipLaunchKernelGGL((quantize_rows_kernel<THREADS, CHUNKS, Wide, Rows>), grid, dim3(THREADS), 0, stream, r, m,   \
                       pitch, t, Q, scale)
    if (pitch <= 64 * 8) TEAL_QUANTIZE(64, 1);
    else if (pitch <= 64 * 8 * 2) TEAL_QUANTIZE(64, 2);
    else if (pitch <= 256 * 8) TEAL_QUANTIZE(256, 1);
    else if (pitch <= 256 * 8 * 2) TEAL_QUANTIZE(256, 2);
    else if (pitch <= 256 * 8 * 4) TEAL_QUANTIZE(256, 4);
    else if (pitch <= 256 * 8 * 8) TEAL_QUANTIZE(256, 8);
    else if (pitch <= 1024 * 8 * 4) TEAL_QUANTIZE(1024, 4);
    else TEAL_QUANTIZE(1024, 16);
#undef TEAL_QUANTIZE
}

// ---- the product ----

struct GemmW8Args {
    const int8_t *W[kMaxMatrices];
    const __half *scale[kMaxMatrices];
    float *y[kMaxMatrices];
    int n[kMaxMatrices];
    int tile_begin[kMaxMatrices + 1];     // first column tile of each matrix; of those past the last one, their number
    const int8_t *Q;
    const float *row_scale;
    int rows, m, pitch;
    int row_tiles, splits, slabs_per_split;
    int *counters, *partial;
};

__device__ __forceinline__ int block_order(int block, int blocks)
{
    const int xcd = block % kXcds, each = blocks / kXcds, more = blocks % kXcds;
    return xcd * each + min(xcd, more) + block / kXcds;
}

// y = (S * row scale) * column scale, S the sum of the integers, exact: m <= 2^17 and |q| <= 127, |W| <= 128.
template <class S>
__global__ __launch_bounds__(S::kThreads) void gemm_w8_kernel(GemmW8Args a)
{
    typedef TileProduct<WeightsInt8, S, 1> Product;
    __shared__ __align__(1024) unsigned char smem[Product::kLds];
    __shared__ int arrived;
    const int tiles = a.tile_begin[kMaxMatrices];
    const int at = block_order(blockIdx.x, gridDim.x);
    const int split = at % a.splits, place = at / a.splits;
    const int2 tile = tile_at(place, a.row_tiles, tiles);
    const int gtile = tile.y, row0 = tile.x * S::BM;

    const int8_t *W = a.W[0];
    const __half *col_scale = a.scale[0];
    float *y = a.y[0];
    int n = a.n[0], first = 0;
#pragma unroll
    for (int k = 1; k < kMaxMatrices; ++k) {
        const bool here = gtile >= a.tile_begin[k];
        W = here ? a.W[k] : W;
        col_scale = here ? a.scale[k] : col_scale;
        y = here ? a.y[k] : y;
        n = here ? a.n[k] : n;
        first = here ? a.tile_begin[k] : first;
    }
    const int col0 = (gtile - first) * S::BN;

    Product p;
    p.begin(smem);
    if (p.multiplies()) p.begin_multiplying(col0, n);
    if (S::LOADERS == 0 || !p.multiplies())
        p.begin_loading(
            [&](int r) {
                return reinterpret_cast<const unsigned char *>(a.Q) + (size_t)min(row0 + r, a.rows - 1) * a.pitch;
            },
            [&](int) { return reinterpret_cast<const unsigned char *>(W); }, [](int) { return nullptr; }, col0, n);
    const int slabs = a.pitch / kSlabBytes;
    const int slab0 = split * a.slabs_per_split;
    p.run(slab0, min(slabs, slab0 + a.slabs_per_split), a.m, a.rows - row0);

    // (tiles of more rows are not sliced)
    if (S::BM <= kMaxSlicedRows && a.splits > 1) {
        // Every slice leaves its sums, and the last one of a tile to arrive adds the others' to its own: whole numbers, in any
        // order the same.
        constexpr int kPieces = S::MF * S::NF, kOwners = 64 * S::kWaves;
        const Buffer sums = buffer_of(a.partial + (size_t)place * a.splits * (S::BM * S::BN),
                                      4u * a.splits * (S::BM * S::BN));
        if (p.multiplies()) {
#pragma unroll
            for (int i = 0; i < S::MF; ++i)
#pragma unroll
                for (int f = 0; f < S::NF; ++f)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, p.acc[i][f]), sums,
                                                           16 * (int)threadIdx.x,
                                                           16 * kOwners * (split * kPieces + i * S::NF + f), kAgentScope);
            wait_vector_memory();
        }
        __syncthreads();
        if (threadIdx.x == 0)
            arrived = __hip_atomic_fetch_add(a.counters + place, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (arrived != a.splits - 1 || !p.multiplies()) return;
        if (threadIdx.x == 0) store_coherent(a.counters + place, 0);
        // 16 loads on their way together: one after the other each would take a trip to memory
        constexpr int kBatch = kPieces < 16 ? kPieces : 16, kTogether = 16 / kBatch;
        for (int s0 = 0; s0 < a.splits; s0 += kTogether) {
#pragma unroll
            for (int q0 = 0; q0 < kPieces; q0 += kBatch) {
                u32x4 other[kTogether][kBatch];
#pragma unroll
                for (int t = 0; t < kTogether; ++t)
#pragma unroll
                    for (int q = 0; q < kBatch; ++q)
                        other[t][q] = __builtin_amdgcn_raw_buffer_load_b128(
                            sums, 16 * (int)threadIdx.x,
                            16 * kOwners * (min(s0 + t, a.splits - 1) * kPieces + q0 + q), kAgentScope);
#pragma unroll
                for (int t = 0; t < kTogether; ++t) {
                    const int take = s0 + t < a.splits && s0 + t != split ? -1 : 0;
#pragma unroll
                    for (int q = 0; q < kBatch; ++q)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            p.acc[(q0 + q) / S::NF][(q0 + q) % S::NF][r] += (int)other[t][q][r] & take;
                }
            }
        }
    }

    if (!p.multiplies()) return;
#pragma unroll
    for (int f = 0; f < S::NF; ++f) {
        const int col = col0 + p.col_of(f);
        if (col >= n) continue;                       // n is a multiple of 16
        float sc[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[r] = __half2float(col_scale[col + r]);
#pragma unroll
        for (int i = 0; i < S::MF; ++i) {
            const int row = row0 + p.row_of(i);
            if (row < a.rows) {
                const float sx = a.row_scale[row];
                float out[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) out[r] = (float)p.acc[i][f][r] * sx * sc[r];
                float *to = y + (size_t)row * n + col;
#pragma unroll
                for (int r = 0; r < 4; ++r) to[r] = out[r];
            }
        }
    }
}

template <class S>
hipError_t launch(const GemmW8Args &a, hipStream_t stream)
{
    const unsigned blocks = (unsigned)(a.tile_begin[kMaxMatrices] * a.row_tiles * a.splits);
    hipLaunchKernelGGL(gemm_w8_kernel<S>, dim3(blocks), dim3(S::kThreads), 0, stream, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_quantize_rows(const void *X, bool bf16, int rows, int m, float t, int8_t *Q, float *scale,
                                hipStream_t stream)
{
    const bool wide = m % 8 == 0 && (reinterpret_cast<uintptr_t>(X) & 15) == 0;
    const unsigned short *x = static_cast<const unsigned short *>(X);
    if (bf16) {
        if (wide) quantize<true>(RowsBf16{x}, rows, m, t, Q, scale, stream);
        else quantize<false>(RowsBf16{x}, rows, m, t, Q, scale, stream);
    } else {
        if (wide) quantize<true>(RowsF16{x}, rows, m, t, Q, scale, stream);
        else quantize<false>(RowsF16{x}, rows, m, t, Q, scale, stream);
    }
    return hipGetLastError();
}

hipError_t launch_quantize_rows_swiglu(const float *gate, const float *up, int rows, int m, float t, int8_t *Q,
                                       float *scale, hipStream_t stream)
{
    const RowsSwiglu r{gate, up};
    if (m % 8 == 0 && ((reinterpret_cast<uintptr_t>(gate) | reinterpret_cast<uintptr_t>(up)) & 15) == 0)
        quantize<true>(r, rows, m, t, Q, scale, stream);
    else
        quantize<false>(r, rows, m, t, Q, scale, stream);
    return hipGetLastError();
}

hipError_t launch_gemm_w8(const GemmW8HostArgs &h, const GemmShape &sh, hipStream_t stream)
{
    GemmW8Args a{};
    int tiles = 0;
    for (int k = 0; k < kMaxMatrices; ++k) {
        a.tile_begin[k] = tiles;
        if (k >= h.count) {
            a.tile_begin[k] = INT32_MAX;               // no tile is in it
            continue;
        }
        a.W[k] = h.W[k];
        a.scale[k] = static_cast<const __half *>(h.scale[k]);
        a.y[k] = h.y[k];
        a.n[k] = h.n[k];
        tiles += (h.n[k] + sh.bn - 1) / sh.bn;
    }
    a.tile_begin[kMaxMatrices] = tiles;
    a.Q = h.Q;
    a.row_scale = h.row_scale;
    a.rows = h.rows;
    a.m = h.m;
    a.pitch = quantized_pitch(h.m);
    a.row_tiles = (h.rows + sh.bm - 1) / sh.bm;
    const int slabs = a.pitch / kSlabBytes;
    a.slabs_per_split = (slabs + sh.splits - 1) / sh.splits;
    a.splits = (slabs + a.slabs_per_split - 1) / a.slabs_per_split;      // none of them empty
    a.counters = h.counters;
    a.partial = h.partial;
    switch (sh.bm) {
    case 16: return launch<TileShape<16, 128, 1, 4, 4, 2>>(a, stream);
    case 32: return launch<TileShape<32, 128, 1, 4, 3, 4>>(a, stream);
    case 64: return launch<TileShape<64, 128, 1, 4, 3, 4>>(a, stream);
    case 128: return launch<TileShape<128, 128, 2, 4, 4, 4>>(a, stream);
    default:
        // (256 x 256: 168 registers a lane, and 13 more that are stored before the loop over the slabs and read behind it,
        // once a tile; nothing is spilled in the loop)
        return sh.bn == 128 ? launch<TileShape<256, 128, 4, 2, 3, 4>>(a, stream)
                            : launch<TileShape<256, 256, 2, 4, 2, 4>>(a, stream);
    }
}

}  // namespace teal
