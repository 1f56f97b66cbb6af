// Products of many rows on the matrix cores: a thread block's tile of Y = X W, X rows contiguous along the sum, W
// input-channel-major as the one-row products store it (Wt[m][n], n contiguous).
//
// A block takes BM rows by BN columns and walks the sum in slabs of 128 bytes of a row of X: 64 channels of bf16, 128 of
// int8.  X and W travel from memory into LDS without registers (global_load_lds), in a ring of STAGES slabs: one barrier a
// slab, the loads of the slab STAGES - 1 further in flight while a slab is multiplied.  The matrix instructions (16 x 16,
// K = 32 for bf16, 64 for int8) want both operands contiguous along the sum in a lane; X is, and W comes through the
// transposing LDS reads (ds_read_b64_tr_b16: 16 lanes read a 4 x 16 block of 16-bit values and get a column each;
// ds_read_b64_tr_b8: an 8 x 16 block of bytes).  W is the first operand and X the second, so a lane ends up with four
// neighbouring columns of one row, 16 bytes of y.
//
// LDS banks.  A row of X in LDS is 128 bytes, 8 chunks of 16: chunk c of row r is at place c ^ (r & 7), so 8 lanes that
// read one chunk of 8 rows touch all banks.  A row of W has 32-byte units (bf16) or 16-byte units (int8), what one row
// gives to a transposing read: unit u of channel k is at place u ^ swizzle(k), so that the 4 (8) rows of a group of 16
// lanes, and the groups of two halves of a wavefront, touch different banks.  The direct loads fill LDS linearly; the
// permutation is in the lanes' global addresses, within one row's bytes.
//
// What bounds it.  Tiles up to 256 x 128: the way from the L2 caches into LDS, which gives all compute units together about
// 12 TB/s whatever the tile (int8, 700 rows of 11008 -> 4096, the weights in the last cache: 43 us; with every wavefront
// loading its part 55, since the address arithmetic and the waits of the loads then stand between its matrix instructions;
// 59 with weights from memory).  256 x 256 loads least for what
// it multiplies (9 TB/s) and has the matrix cores busy; there their rate, which falls with the power that the operands'
// bits take (7 to 20 % between zeros and random numbers), bounds it with the LDS reads: 4096 x 8192 -> 28672 int8 at
// 2.3 POPS.  Tiles of few rows: memory, once for W.
#pragma once

#include "gemv_common.h"

namespace teal {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr int kSlabBytes = 128;            // of a row of X

// Source of the zeros for channels past the last one.
static __device__ const u32x4 zero_chunk = {0u, 0u, 0u, 0u};

// 16 bytes per lane from `from` to LDS at `to` (wavefront-uniform) + 16 * lane.  The wait is the caller's.  In assembly,
// because the compiler, which cannot know which part of LDS a load fills, waits for all of them before any LDS read
// that follows.  m0 is written right before it is read, and nothing else in these kernels uses it.
__device__ __forceinline__ void load_to_lds(const unsigned char *from, unsigned to)
{
    asm volatile("s_mov_b32 m0, %1\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dwordx4 %0, off" ::"v"(from), "s"(to));
}
// Waits until at most `left` of this wavefront's vector-memory operations are under way and all its LDS operations are
// done, then for the block.  Afterwards what every wavefront loaded before is in LDS, and nobody reads what it read.
template <int left>
__device__ __forceinline__ void wait_and_meet()
{
    static_assert(left >= 0 && left < 64, "six bits");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(left) : "memory");
}
// The same for wavefronts that load nothing.
__device__ __forceinline__ void finish_lds_and_meet() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned lds_address(const void *p)
{
    typedef const __attribute__((address_space(3))) unsigned char *lds_ptr;
    return (unsigned)(uintptr_t)(lds_ptr)p;
}

// How W is stored.
struct WeightsBf16 {
    static constexpr int kBytes = 2;               // of a value in LDS
    static constexpr int kSlabRows = 64;           // channels of a slab
    static constexpr bool kMx4 = false;
    typedef f32x4 Acc;
};
struct WeightsInt8 {
    static constexpr int kBytes = 1;
    static constexpr int kSlabRows = 128;
    static constexpr bool kMx4 = false;
    typedef i32x4 Acc;
};
// Microscaled 4-bit numbers, made bf16 numbers (exactly, by the hardware's conversion with a scale) on their way: codes
// and scales come into the ring, every thread converts one block of 32 a slab, one slab ahead of its use, and a second
// pair of buffers has the bf16 tile.
struct WeightsMx4 {
    static constexpr int kBytes = 2;
    static constexpr int kSlabRows = 64;
    static constexpr bool kMx4 = true;
    typedef f32x4 Acc;
};

// LOADERS wavefronts beside those that multiply do nothing but load (0: every wavefront loads its part).
template <int BM_, int BN_, int WM_, int WN_, int STAGES_, int LOADERS_ = 0>
struct TileShape {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, STAGES = STAGES_, LOADERS = LOADERS_;
    static constexpr int kWaves = WM * WN, kThreads = 64 * (kWaves + LOADERS);
    static constexpr int kLoadWaves = LOADERS > 0 ? LOADERS : kWaves;
    static constexpr int MF = BM / WM / 16, NF = BN / WN / 16;       // 16 x 16 pieces of a wavefront
};

// The product of one tile.  HALVES = 1: the tile's BN columns are neighbours in one matrix; 2: BN / 2 columns of each of
// two matrices, and piece f of a wavefront and piece f + NF / 2 are the same columns of the two.
template <class F, class S, int HALVES>
struct TileProduct {
    static constexpr int BM = S::BM, BN = S::BN, MF = S::MF, NF = S::NF, STAGES = S::STAGES;
    static constexpr int kRowBytes = BN * F::kBytes;                   // of W in LDS
    static constexpr int kSlabX = BM * kSlabBytes, kSlabW = F::kSlabRows * kRowBytes;
    static constexpr int kCodes = F::kSlabRows * BN / 2, kScales = HALVES * F::kSlabRows * 16;     // of mx4, in a slab
    static constexpr int kStage = kSlabX + (F::kMx4 ? kCodes + kScales : kSlabW);
    static constexpr int kRing = STAGES * kStage;
    static constexpr int kLds = kRing + (F::kMx4 ? 2 * kSlabW : 0);
    static constexpr int kLoadWaves = S::kLoadWaves;
    static constexpr int kLoadsX = (BM / 8 + kLoadWaves - 1) / kLoadWaves;     // of 64 lanes x 16 bytes, a wavefront's
    static constexpr int kLoadsC = kCodes / 1024 / kLoadWaves;                 // mx4: of codes
    static constexpr int kLoadsW = F::kMx4 ? kLoadsC + 1 : kSlabW / 1024 / kLoadWaves;
    static constexpr int kRowsPerLoad = F::kMx4 ? 2048 / BN : 1024 / kRowBytes;     // rows of W that a load covers
    static constexpr int kRowStep = kRowsPerLoad * kLoadWaves;
    static constexpr int kUnit = F::kBytes == 2 ? 32 : 16;             // bytes that a permutation keeps together
    static constexpr int kHalfUnits = kRowBytes / HALVES / kUnit;      // of one matrix in a row
    static constexpr int kUnitMask = kRowBytes / kUnit < 16 ? kRowBytes / kUnit - 1 : 15;
    // A lane's permutation in its loads of W repeats with the bits of the row that it depends on.
    static constexpr int kPeriod = F::kBytes == 2 ? 16 : 32;
    static constexpr int kWLanes = F::kMx4 || kRowStep % kPeriod == 0 ? 1 : 2;
    static_assert(BM % (16 * S::WM) == 0 && BN % (16 * S::WN) == 0 && kSlabW % (1024 * kLoadWaves) == 0, "");
    static_assert(F::kMx4 || kWLanes * kRowStep % kPeriod == 0, "");
    static_assert(!F::kMx4 || (kCodes == 16 * 64 * S::kWaves && kCodes % (1024 * kLoadWaves) == 0 && kLoadWaves >= HALVES),
                  "a block of 32 codes per multiplying thread");
    static_assert(HALVES == 1 || NF % 2 == 0, "both matrices in every wavefront");
    static_assert(kLds <= 160 * 1024, "");

    typedef typename F::Acc Acc;
    Acc acc[MF][NF];

    static __device__ __forceinline__ int swizzle(int k)
    {
        // Rows of 128 bytes have half of the banks each: four of every eight rows that are read together lie in the same half.
        if (F::kBytes == 1 && kRowBytes == 128) return (k >> 1 & 3) | (k >> 4 & 1) << 2;
        return (F::kBytes == 2 ? (k & 3) | (k >> 3 & 1) << 2 : (k & 7) | (k >> 4 & 1) << 3) & kUnitMask;
    }

    // Place of a unit of channel k in its row.  (Where the permutation stays within a matrix's units, its part is a constant.)
    static __device__ __forceinline__ int unit_at(int half, int unit, int k)
    {
        if (kHalfUnits >= (F::kBytes == 2 ? 8 : 16)) return half * (kRowBytes / HALVES) + (unit ^ swizzle(k)) * kUnit;
        return ((half * kHalfUnits + unit) ^ swizzle(k)) * kUnit;
    }

    unsigned lds;                                // of the ring
    int wave, lane, wm, wn;
    int load_wave;                               // among those that load
    const unsigned char *x_lane[kLoadsX];        // this lane's chunk of its rows, first channel
    const unsigned char *w_lane[kWLanes];        // this lane's columns, its row of the first loads, first channel of the sum
    int w_pitch;                                 // bytes
    int x_chunk, w_row;                          // chunk of the row and row of the slab that the lane loads
    // mx4: this lane's 16 bytes of scales, which come in tiles of 8 channels by 16 blocks; the row of the block that this
    // thread converts, where its scale is and where its numbers go
    const unsigned char *s_lane;
    int s_pitch;                                 // bytes between tiles of one block row
    int block_row;
    unsigned scale_at, value_at[4];
    int other_first;                             // whether it writes the second of a unit's two chunks before the first

    __device__ __forceinline__ void begin(void *smem)
    {
        lds = lds_address(smem);
        lane = threadIdx.x & 63;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        wm = wave / S::WN;
        wn = wave % S::WN;
        load_wave = S::LOADERS > 0 ? wave - S::kWaves : wave;
    }
    // Whether this wavefront multiplies and has a part of the result.
    __device__ __forceinline__ bool multiplies() const { return S::LOADERS == 0 || wave < S::kWaves; }

    __device__ __forceinline__ void begin_multiplying(int col0, int n)
    {
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int f = 0; f < NF; ++f) acc[i][f] = Acc{};
        if constexpr (F::kMx4) {
            constexpr int kBlocks = BN / 32 / HALVES;                  // of a row of one matrix
            block_row = threadIdx.x / (BN / 32);
            const int half = threadIdx.x % (BN / 32) / kBlocks, in_half = threadIdx.x % kBlocks;
            const int col = min(col0 + 32 * in_half, n - 32);
            scale_at = kSlabX + kCodes + half * (kScales / HALVES) + (block_row / 8) * kMx4TileBytes + block_row % 8 * 16 +
                       col / 32 % 16;
            // Eight lanes write together.  They have a row of 512 bytes, every second unit of 32: half of them begin with
            // their units' other chunks, or four would meet four in the same banks.
            other_first = kRowBytes == 512 ? threadIdx.x >> 2 & 1 : 0;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                value_at[q] = block_row * kRowBytes + unit_at(half, 2 * in_half + q / 2, block_row) +
                              (q ^ other_first) % 2 * 16;
        }
    }

    // `row_of(r)`: the address of the tile's row r of X (of any valid row where the tile has none).  `w_of(half)`: of the
    // matrix; `scale_of(half)`: of its scales (mx4).  Columns from n on repeat the last ones (n a multiple of a chunk): they
    // are not stored.
    template <class RowOf, class WOf, class ScaleOf>
    __device__ __forceinline__ void begin_loading(const RowOf &row_of, const WOf &w_of, const ScaleOf &scale_of, int col0,
                                                  int n)
    {
        x_chunk = (lane & 7) ^ (lane >> 3);
#pragma unroll
        for (int j = 0; j < kLoadsX; ++j) x_lane[j] = row_of(x_load(j) * 8 + (lane >> 3)) + 16 * x_chunk;
        const int chunk = load_wave * 64 + lane;                       // of 16 bytes, in a slab of W
        if constexpr (F::kMx4) {
            constexpr int kBlocks = BN / 32 / HALVES;
            w_row = chunk / (BN / 32);
            const int half = chunk % (BN / 32) / kBlocks, in_half = chunk % kBlocks;
            w_pitch = n / 2;
            w_lane[0] = w_of(half) + (long long)w_row * w_pitch + min(col0 + 32 * in_half, n - 32) / 2;
            // a wavefront loads the slab's scales of one matrix: lane / 8 the tile, lane % 8 the channel in it
            s_pitch = mx4_scale_tiles(n) * kMx4TileBytes;
            s_lane = scale_of(load_wave % HALVES) + (long long)(lane >> 3) * s_pitch + col0 / 512 * kMx4TileBytes +
                     (lane & 7) * 16;
            return;
        }
        const int at = chunk * 16;
        w_row = at / kRowBytes;
        w_pitch = n * F::kBytes;
#pragma unroll
        for (int v = 0; v < kWLanes; ++v) {
            const int row = w_row + v * kRowStep;
            const int unit = at % kRowBytes / kUnit ^ swizzle(row);
            const int col = min(col0 + (unit % kHalfUnits * kUnit + at % kUnit) / F::kBytes, n - 16 / F::kBytes);
            w_lane[v] = w_of(unit / kHalfUnits) + (long long)row * w_pitch + (long long)col * F::kBytes;
        }
    }
    // Which 8 rows of X the wavefront's load j takes: where there are fewer loads than wavefronts some load the same.
    __device__ __forceinline__ int x_load(int j) const { return (load_wave + j * kLoadWaves) % (BM / 8); }

    // Slab `slab` of a sum of m channels into place `stage` of the ring: X, and W.  Channels from m on are zeros.
    template <int LOADS>
    __device__ __forceinline__ void load_x(int slab, int stage, int m)
    {
        const unsigned to = lds + stage * kStage;
        const long long x_at = (long long)slab * kSlabBytes;
        const int k0 = slab * F::kSlabRows;
        // (rows of 8-bit integers have zeros behind their end)
        if (F::kBytes == 1 || k0 + F::kSlabRows <= m) {
#pragma unroll
            for (int j = 0; j < LOADS; ++j) load_to_lds(x_lane[j] + x_at, to + x_load(j) * 1024);
        } else {
            const unsigned char *const zero = reinterpret_cast<const unsigned char *>(&zero_chunk);
            const bool in_row = k0 + x_chunk * (16 / F::kBytes) < m;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) load_to_lds(in_row ? x_lane[j] + x_at : zero, to + x_load(j) * 1024);
        }
    }
    __device__ __forceinline__ void load_w(int slab, int stage, int m)
    {
        const unsigned to = lds + stage * kStage + kSlabX + load_wave * 1024;
        const unsigned scales_to = lds + stage * kStage + kSlabX + kCodes + load_wave % HALVES * 1024;
        constexpr int kLoads = F::kMx4 ? kLoadsC : kLoadsW;            // beside that of the scales
        const int k0 = slab * F::kSlabRows;
        const unsigned char *const s_at = F::kMx4 ? s_lane + (long long)(k0 / 8) * s_pitch : nullptr;
        if (k0 + F::kSlabRows <= m) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) load_to_lds(w_at(k0, j), to + j * kLoadWaves * 1024);
            if constexpr (F::kMx4) load_to_lds(s_at, scales_to);
        } else {
            const unsigned char *const zero = reinterpret_cast<const unsigned char *>(&zero_chunk);
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                load_to_lds(k0 + w_row + j * kRowStep < m ? w_at(k0, j) : zero, to + j * kLoadWaves * 1024);
            if constexpr (F::kMx4) load_to_lds(k0 + (lane & ~7) < m ? s_at : zero, scales_to);
        }
    }
    // This lane's 16 bytes of load j of W, the slab from channel k0 on.
    __device__ __forceinline__ const unsigned char *w_at(int k0, int j) const
    {
        return w_lane[j % kWLanes] + (long long)(k0 + j / kWLanes * kWLanes * kRowStep) * w_pitch;
    }

    // mx4: this thread's block of 32 codes at `stage` of the ring and its scale, and those as bf16 numbers into buffer `to`.
    struct Block {
        u32x4 codes;
        unsigned scale;
    };
    __device__ __forceinline__ Block read_block(int stage) const
    {
        typedef const __attribute__((address_space(3))) unsigned char *lds_ptr;
        typedef const __attribute__((address_space(3))) u32x4 *lds_u32x4;
        const lds_ptr from = (lds_ptr)(uintptr_t)(lds + stage * kStage);
        return {*(lds_u32x4)(from + kSlabX + threadIdx.x * 16), from[scale_at]};
    }
    __device__ __forceinline__ void convert(const Block &b, int slab, int to, int m)
    {
        typedef __attribute__((address_space(3))) u32x4 *lds_out;
        // what lies behind the last channel of a tile of scales has no meaning
        const float sc = slab * F::kSlabRows + block_row < m ? __uint_as_float(b.scale << 23) : 0.f;
        const unsigned buffer = lds + kRing + to * kSlabW;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const unsigned codes = other_first ? b.codes[q ^ 1] : b.codes[q];
            u32x4 v;
            v[0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 0));
            v[1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 1));
            v[2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 2));
            v[3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, sc, 3));
            *(lds_out)(uintptr_t)(buffer + value_at[q]) = v;
        }
    }

    // Multiplies in a slab whose X is at `x_at` and whose W is at `w_at` in LDS; the first LIVE pieces of rows.
    template <int LIVE>
    __device__ __forceinline__ void multiply(unsigned x_at, unsigned w_at)
    {
        typedef const __attribute__((address_space(3))) unsigned char *lds_ptr;
        typedef const __attribute__((address_space(3))) u32x4 *lds_u32x4;
        const lds_ptr x = (lds_ptr)(uintptr_t)x_at, w = (lds_ptr)(uintptr_t)w_at;
        const int l = lane & 15, g = lane >> 4;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            u32x4 W[NF];
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                const int half = HALVES == 1 ? 0 : f / (NF / 2);
                const int piece = HALVES == 1 ? wn * NF + f : wn * (NF / 2) + f % (NF / 2);
                if constexpr (F::kBytes == 2) {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    typedef __attribute__((address_space(3))) s16x4 *lds_s16x4;
                    const int k = 32 * ks + 8 * g + l / 4;             // and 4 further
                    const lds_ptr p = w + k * kRowBytes + unit_at(half, piece, k) + l % 4 * 8;
                    const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)p));
                    const uint2 b = __builtin_bit_cast(
                        uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(p + 4 * kRowBytes)));
                    W[f] = u32x4{a.x, a.y, b.x, b.y};
                } else {
                    typedef int i32x2 __attribute__((ext_vector_type(2)));
                    typedef __attribute__((address_space(3))) i32x2 *lds_i32x2;
                    const int k = 64 * ks + 16 * g + l / 2;            // and 8 further
                    const lds_ptr p = w + k * kRowBytes + unit_at(half, piece, k) + l % 2 * 8;
                    const uint2 a = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)p));
                    const uint2 b = __builtin_bit_cast(
                        uint2, __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2)(p + 8 * kRowBytes)));
                    W[f] = u32x4{a.x, a.y, b.x, b.y};
                }
            }
#pragma unroll
            for (int i = 0; i < LIVE; ++i) {
                const int row = (i * S::WM + wm) * 16 + l;
                const u32x4 X = *(lds_u32x4)(x + row * kSlabBytes + ((4 * ks + g) ^ (l & 7)) * 16);
#pragma unroll
                for (int f = 0; f < NF; ++f) {
                    if constexpr (F::kBytes == 2)
                        acc[i][f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                            __builtin_bit_cast(bf16x8, W[f]), __builtin_bit_cast(bf16x8, X), acc[i][f], 0, 0, 0);
                    else
                        acc[i][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(
                            __builtin_bit_cast(i32x4, W[f]), __builtin_bit_cast(i32x4, X), acc[i][f], 0, 0, 0);
                }
            }
        }
    }

    // Slabs [first, last) of a sum of m channels, for the first `rows` rows of the tile: a tile that is a
    // quarter, half or three quarters empty multiplies (and loads) only the others of its pieces.
    __device__ __forceinline__ void run(int first, int last, int m, int rows)
    {
        if constexpr (MF >= 4) {
            if (rows <= BM / 4) return run_pieces<MF / 4>(first, last, m);
            if (rows <= BM / 2) return run_pieces<MF / 2>(first, last, m);
            if constexpr (MF >= 8)
                if (rows <= BM / 4 * 3) return run_pieces<MF / 4 * 3>(first, last, m);
        }
        run_pieces<MF>(first, last, m);
    }
    template <int LIVE>
    __device__ __forceinline__ void run_pieces(int first, int last, int m)
    {
        constexpr int kPieceLoads = LIVE * S::WM * 2 / kLoadWaves;
        constexpr int kLiveX = kPieceLoads < 1 ? 1 : kPieceLoads;
        constexpr int kLoads = kLiveX + kLoadsW;
        constexpr int kAhead = F::kMx4 ? 1 : 0;          // by how many slabs W is ahead of X
        if constexpr (S::LOADERS > 0 && !F::kMx4) {
            // Two loops that have only the barriers in common (int8, 2048 rows of 14336 -> 4096: 110 us; both in one 115).
            if (multiplies())
                multiply_slabs<LIVE>(last - first);
            else
                load_slabs<kLiveX>(first, last, m);
            return;
        }
        const bool loads = S::LOADERS == 0 || !multiplies();
        if constexpr (F::kMx4) {
            if (loads) load_w(first, STAGES - 1, m);
            wait_and_meet<0>();
            if (multiplies()) convert(read_block(STAGES - 1), first, 0, m);      // (filled again after the next meeting)
        }
        // Place s of the ring: X of slab first + s, and W of the same slab (mx4: of the next one).
        if (loads) {
#pragma unroll
            for (int s = 0; s < STAGES - 1; ++s) {
                if (first + s < last) load_x<kLiveX>(first + s, s, m);
                if (first + s + kAhead < last) load_w(first + s + kAhead, s, m);
            }
        }
        // Before slab `slab`: what later slabs loaded may still be under way.
        auto meet = [&](int slab) {
            if (slab + STAGES - 2 + kAhead < last)
                wait_and_meet<(STAGES - 2) * kLoads>();
            else
                wait_and_meet<0>();
        };
        auto load_next = [&](int slab, int stage) {
            const int next = slab + STAGES - 1, to = stage == 0 ? STAGES - 1 : stage - 1;
            if (next < last) load_x<kLiveX>(next, to, m);
            if (next + kAhead < last) load_w(next + kAhead, to, m);
        };
        int stage = 0, buffer = 0;
        if (S::LOADERS > 0 && !multiplies()) {
            for (int slab = first; slab < last; ++slab) {
                meet(slab);
                load_next(slab, stage);
                stage = stage == STAGES - 1 ? 0 : stage + 1;
            }
            return;
        }
        for (int slab = first; slab < last; ++slab) {
            if constexpr (S::LOADERS > 0) {
                finish_lds_and_meet();
            } else {
                meet(slab);
                load_next(slab, stage);
            }
            const unsigned x_at = lds + stage * kStage;
            if constexpr (F::kMx4) {
                const Block block = read_block(stage);         // (past the last slab: what is there)
                multiply<LIVE>(x_at, lds + kRing + buffer * kSlabW);
                buffer ^= 1;
                // Past the last slab into a buffer that nobody reads: without a branch the instructions go between those of
                // the product (1100 us where 1163, r = 512; tiles of few rows are the faster for the branch).
                if (MF >= 4 || slab + 1 < last) convert(block, slab + 1, buffer, m);
            } else {
                multiply<LIVE>(x_at, x_at + kSlabX);
            }
            stage = stage == STAGES - 1 ? 0 : stage + 1;
        }
    }

    template <int LIVE>
    __device__ __forceinline__ void multiply_slabs(int slabs)
    {
        int stage = 0;
        for (int s = 0; s < slabs; ++s) {
            finish_lds_and_meet();
            const unsigned x_at = lds + stage * kStage;
            multiply<LIVE>(x_at, x_at + kSlabX);
            stage = stage == STAGES - 1 ? 0 : stage + 1;
        }
    }
    template <int LOADS>
    __device__ __forceinline__ void load_slabs(int first, int last, int m)
    {
        auto load = [&](int slab, int stage) {
            if (slab >= last) return;
            load_x<LOADS>(slab, stage, m);
            load_w(slab, stage, m);
        };
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) load(first + s, s);
        int stage = 0;
        for (int slab = first; slab < last; ++slab) {
            // what later slabs loaded may still be under way
            if (slab + STAGES - 2 < last)
                wait_and_meet<(STAGES - 2) * (LOADS + kLoadsW)>();
            else
                wait_and_meet<0>();
            load(slab + STAGES - 1, stage == 0 ? STAGES - 1 : stage - 1);
            stage = stage == STAGES - 1 ? 0 : stage + 1;
        }
    }

    // Row of the tile and first of four neighbouring columns (of a half) that acc[i][f] holds.
    __device__ __forceinline__ int row_of(int i) const { return (i * S::WM + wm) * 16 + (lane & 15); }
    __device__ __forceinline__ int col_of(int f) const
    {
        const int piece = HALVES == 1 ? wn * NF + f : wn * (NF / 2) + f % (NF / 2);
        return piece * 16 + 4 * (lane >> 4);
    }
};

// Order of the tiles: neighbours in it share an XCD (its blocks are every eighth of the grid), and the blocks that run there
// together are 8 row tiles by as many column tiles, so that what they read of X and of W is read once into its L2.
constexpr int kXcds = 8;
constexpr int kRowTileGroup = 8;
// Place `at` among row_tiles x col_tiles of them: row tile and column tile.
__device__ __forceinline__ int2 tile_at(int at, int row_tiles, int col_tiles)
{
    const int group = at / (kRowTileGroup * col_tiles), in_group = at - group * kRowTileGroup * col_tiles;
    const int rows = min(kRowTileGroup, row_tiles - group * kRowTileGroup);
    return make_int2(group * kRowTileGroup + in_group % rows, in_group / rows);
}

}  // namespace teal
