// Routing to experts: scores from a router's logits, the top_k experts of each token and their weights.
//
// The result is defined in binary64, but hardly a token needs all of its scores there.  fp32 values (the score and a
// bias, or the logit), cut to the upper bits of a word above the expert's number, find top_k + 1 candidates, and
// their binary64 scores, which are the weights, put those in order.  What the words left out matters only if a
// third value lies within their error of the last one chosen: then the row goes on to 16 candidates, and tokens of more
// equals than that take a wavefront each, by binary64 values throughout.  So do calls with more than 512 places for experts
// (a group has a power of two), with more than 15 experts chosen or with more than 16 groups.  Groups whose fp32 values are
// too near each other are valued again by the binary64 scores of their largest.
//
// What bounds it is instruction issue, 880 vector instructions of the four wavefronts a SIMD has, and the memory's and a
// launch's latency.  (us for 16384 tokens of 256 experts in 8 groups, 4 groups and 8 experts taken, sigmoid scores and a
// bias; reading the logits takes 4: a wavefront per token in binary64 46; the selection on fp32 scores, the place of each
// maximum found by ballots, 28; a row of lanes per token on words, with all scores in binary64, 24; fp32 scores and keys
// in sorted fours 16, 1270 instructions; without branches and double work 12.4; all of a near group's scores in binary64,
// for one or two wavefronts of a launch, cost all the others' wait: the two largest 11.)
#include <hip/hip_runtime.h>

#include "teal_internal.h"

namespace teal {

namespace {

constexpr int kRouteWaves = 4;
constexpr int kNone = 0x7fffffff;

// The other lanes of a row of 16 in turn; after four of these with the same operation all lanes have it of all.
template <int N>
__device__ __forceinline__ unsigned row_rotate(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + N /* row_ror */, 0xF, 0xF, false);
}
template <int N>
__device__ __forceinline__ float row_rotate(float v)
{
    return __uint_as_float(row_rotate<N>(__float_as_uint(v)));
}
__device__ __forceinline__ unsigned row_max(unsigned v)
{
    v = max(v, row_rotate<1>(v));
    v = max(v, row_rotate<2>(v));
    v = max(v, row_rotate<4>(v));
    return max(v, row_rotate<8>(v));
}
__device__ __forceinline__ float row_max(float v)
{
    v = fmaxf(v, row_rotate<1>(v));
    v = fmaxf(v, row_rotate<2>(v));
    v = fmaxf(v, row_rotate<4>(v));
    return fmaxf(v, row_rotate<8>(v));
}
template <int CTRL>
__device__ __forceinline__ double lane_of(double v)
{
    const int lo = __builtin_amdgcn_update_dpp(0, __double2loint(v), CTRL, 0xF, 0xF, false);
    const int hi = __builtin_amdgcn_update_dpp(0, __double2hiint(v), CTRL, 0xF, 0xF, false);
    return __hiloint2double(hi, lo);
}
template <int CTRL>
__device__ __forceinline__ float lane_of(float v)
{
    return __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, 0xF, 0xF, false));
}
// lane ^ 1, lane ^ 2, the other quad of 8 lanes, the other half of a row
constexpr int kSwap1 = 0xB1, kSwap2 = 0x4E, kSwap4 = 0x141, kSwap8 = 0x140;
__device__ __forceinline__ double row_sum(double v)
{
    v += lane_of<kSwap1>(v);
    v += lane_of<kSwap2>(v);
    v += lane_of<kSwap4>(v);
    return v + lane_of<kSwap8>(v);
}
__device__ __forceinline__ double wave_max(double v)
{
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ double wave_sum(double v)
{
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// Order of numbers as that of unsigned ones, none of them zero; -0 comes before 0.
__device__ __forceinline__ unsigned order_key(float v)
{
    const unsigned u = __float_as_uint(v);
    return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned key)
{
    return __uint_as_float(key ^ ((int)key < 0 ? 0x80000000u : 0xFFFFFFFFu));
}

// A logit as it counts: NaN as -infinity, +infinity as the largest finite number; and -0 as 0.
__device__ __forceinline__ float clean_logit(float l)
{
    return fminf(fmaxf(l + 0.f, -__builtin_inff()), 3.402823466e38f);
}

// exp(x) for x of at most 709.7827 to a last place or two: x = k ln 2 + r, the Taylor polynomial of degree 12 at
// |r| <= 0.347 (the next term is below 2^-52), times 2^k.
__device__ __forceinline__ double exponential(double x)
{
    x = fmax(x, -1000.0);
    const double k = rint(x * 1.4426950408889634);
    double r = fma(k, -0x1.62e42fefa0000p-1, x);        // 41 bits of ln 2: k times them is exact
    r = fma(k, -0x1.cf79abc9e3b3ap-40, r);              // the rest
    double p = 1.0 / 479001600.0;
    p = fma(p, r, 1.0 / 39916800.0);
    p = fma(p, r, 1.0 / 3628800.0);
    p = fma(p, r, 1.0 / 362880.0);
    p = fma(p, r, 1.0 / 40320.0);
    p = fma(p, r, 1.0 / 5040.0);
    p = fma(p, r, 1.0 / 720.0);
    p = fma(p, r, 1.0 / 120.0);
    p = fma(p, r, 1.0 / 24.0);
    p = fma(p, r, 1.0 / 6.0);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    return ldexp(p, (int)k);
}
// 1 / d for d of at least 1, by Newton's iteration from the hardware's estimate.
__device__ __forceinline__ double reciprocal(double d)
{
    double r = __builtin_amdgcn_rcp(d);
    r = fma(r, fma(-d, r, 1.0), r);
    return fma(r, fma(-d, r, 1.0), r);
}
// (-709.7827 lies between the last fp32 number whose exponential binary64 holds and the next.)
__device__ __forceinline__ double sigmoid_score(double z)
{
    return z < -709.7827 ? 0.0 : reciprocal(1.0 + exponential(-fmax(z, -709.7827)));
}
__device__ __forceinline__ double softmax_part(double z, double top)
{
    return z == -__builtin_inf() ? 0.0 : exponential(z - top);
}

// fp32 sigmoid from the hardware's exponential and reciprocal, 1 / (1 + e), wrong by at most kScoreError.  Wrong last places of
// the argument (of at most 88 log2 e where it matters), of e (2^-23 relative), of the sum and of the reciprocal do
// s (1 - s) |l| 2^-23 < 2^-25, s (1 - s) 2^-23 <= 2^-25, 2^-24 and 2^-23 to s: together less than 2^-22.
__device__ __forceinline__ float rough_sigmoid(float l)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * l));
}
constexpr float kScoreError = 0x1p-22f;

// One token by one wavefront, in binary64 throughout; lane l has experts l, l + 64, ...  `values`: LDS for E * 64.
template <int E>
__device__ void route_exactly(const RouteHostArgs &h, int token, double *values)
{
    const int lane = threadIdx.x & 63;
    const float *logits = h.logits + (size_t)token * h.experts;
    double z[E], score[E], order[E];
    unsigned available = 0;
    double top = -__builtin_inf();
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int e = lane + 64 * j;
        available |= (unsigned)(e < h.experts) << j;
        z[j] = e < h.experts ? clean_logit(logits[e]) : -__builtin_inff();
        top = fmax(top, z[j]);
    }
    if (h.sigmoid) {
#pragma unroll
        for (int j = 0; j < E; ++j) score[j] = sigmoid_score(z[j]);
    } else {
        top = wave_max(top);
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < E; ++j) sum += score[j] = softmax_part(z[j], top);
        sum = wave_sum(sum);
#pragma unroll
        for (int j = 0; j < E; ++j) score[j] = sum > 0.0 ? score[j] / sum : 0.0;
    }
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int e = lane + 64 * j;
        double v = z[j];
        if (h.bias && e < h.experts) v = score[j] + (double)h.bias[e];
        order[j] = v != v ? -__builtin_inf() : v;
    }
    if (h.groups > 1) {
        const int size = h.experts / h.groups;
#pragma unroll
        for (int j = 0; j < E; ++j)          // two experts' logits say nothing about the sum of their scores
            values[lane + 64 * j] = h.group_top == 2 && !h.bias ? score[j] : order[j];
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        double first = -__builtin_inf(), second = -__builtin_inf();
        if (lane < h.groups)
            for (int k = 0; k < size; ++k) {
                const double v = values[lane * size + k];
                second = fmax(second, fmin(first, v));
                first = fmax(first, v);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        double value = h.group_top == 2 && size > 1 ? first + second : first;
        value = value != value ? -__builtin_inf() : value;
        int before = 0;
        for (int k = 0; k < h.groups; ++k) {
            const double v = __shfl(value, k);
            before += v > value || (v == value && k < lane);
        }
        const unsigned long long taken = __ballot(lane < h.groups && before < h.top_groups);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int e = lane + 64 * j;
            if (!(taken >> min(e / size, 63) & 1)) available &= ~(1u << j);
        }
    }
    double chosen_score = 0.0, total = 0.0;        // of slot `lane`
    int chosen = 0;
    for (int k = 0; k < h.top_k; ++k) {
        double best = -__builtin_inf();
        int at = kNone;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const bool free = available >> j & 1;
            if (free && (at == kNone || order[j] > best)) {
                best = order[j];
                at = lane + 64 * j;
            }
        }
        for (int d = 32; d; d >>= 1) {
            const double v = __shfl_xor(best, d);
            const int o = __shfl_xor(at, d);
            const bool take = o != kNone && (at == kNone || v > best || (v == best && o < at));
            best = take ? v : best;
            at = take ? o : at;
        }
        double s = 0.0;
#pragma unroll
        for (int j = 0; j < E; ++j)
            if (at == lane + 64 * j) {
                s = score[j];
                available &= ~(1u << j);
            }
        s = __shfl(s, at & 63);
        total += s;
        chosen = lane == k ? at : chosen;
        chosen_score = lane == k ? s : chosen_score;
    }
    if (lane < h.top_k) {
        double v = chosen_score;
        if (h.renormalise) v = total > 0.0 ? v / total : 0.0;
        h.idx[(size_t)token * h.top_k + lane] = chosen;
        h.weight[(size_t)token * h.top_k + lane] = (float)(v * (double)h.scaling);
    }
}

// The two largest values of a lane's experts.
template <int E>
__device__ __forceinline__ void largest_two(const float (&v)[E], float &first, float &second)
{
    first = v[0];
    second = -__builtin_inff();
#pragma unroll
    for (int j = 1; j < E; ++j) {
        second = __builtin_amdgcn_fmed3f(first, second, v[j]);
        first = fmaxf(first, v[j]);
    }
}
// From the two largest of each lane those of a group in its `lanes` lanes (a power of two up to 16).
template <class V>
__device__ __forceinline__ void largest_two_of_group(int lanes, V &first, V &second)
{
    const auto larger = [](V a, V b) { return a > b ? a : b; };
    const auto smaller = [](V a, V b) { return a > b ? b : a; };
    const auto merge = [&](V a, V b) {
        second = larger(smaller(first, a), larger(second, b));
        first = larger(first, a);
    };
    if (lanes > 1) merge(lane_of<kSwap1>(first), lane_of<kSwap1>(second));
    if (lanes > 2) merge(lane_of<kSwap2>(first), lane_of<kSwap2>(second));
    if (lanes > 4) merge(lane_of<kSwap4>(first), lane_of<kSwap4>(second));
    if (lanes > 8) merge(lane_of<kSwap8>(first), lane_of<kSwap8>(second));
}

// How many groups of the token come before this lane's, by value and of equal ones by number.  Lanes of a row that
// belong to no group have -infinity.
template <class V>
__device__ __forceinline__ int groups_before(V value, int groups, int group_lanes)
{
    const int lane = threadIdx.x & 63, row = lane & 48, group = (lane & 15) >> __builtin_ctz((unsigned)group_lanes);
    int before = 0;
#pragma unroll 1
    for (int g = 0; g < groups; g += 4) {
        V x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = __shfl(value, row + min((g + u) * group_lanes, 15));
#pragma unroll
        for (int u = 0; u < 4; ++u)          // (not && and ||, which become branches)
            before += (int)((g + u < groups) & ((x[u] > value) | ((x[u] == value) & (g + u < group))));
    }
    return before;
}

// Keys of a lane in descending fours (of fewer: as they are), so that a maximum is looked for among their heads.
template <int E>
__device__ __forceinline__ void sort_fours(unsigned (&key)[E])
{
    if constexpr (E >= 4) {
        const auto order = [&](int a, int b) {
            const unsigned x = key[a], y = key[b];
            key[a] = max(x, y);
            key[b] = min(x, y);
        };
#pragma unroll
        for (int q = 0; q < E; q += 4) {
            order(q, q + 1);
            order(q + 2, q + 3);
            order(q, q + 2);
            order(q + 1, q + 3);
            order(q + 1, q + 2);
        }
    }
}
template <int E>
__device__ __forceinline__ unsigned largest_key(const unsigned (&key)[E])
{
    constexpr int STEP = E >= 4 ? 4 : 1;
    unsigned best = key[0];
#pragma unroll
    for (int j = STEP; j < E; j += STEP) best = max(best, key[j]);
    return best;
}
template <int E>
__device__ __forceinline__ void remove_key(unsigned (&key)[E], unsigned taken)
{
    constexpr int STEP = E >= 4 ? 4 : 1;
#pragma unroll
    for (int q = 0; q < E; q += STEP) {
        const bool here = key[q] == taken;
#pragma unroll
        for (int j = q; j < q + STEP - 1; ++j) key[j] = here ? key[j + 1] : key[j];
        key[q + STEP - 1] = here ? 0u : key[q + STEP - 1];
    }
}

// The `count` values from p on, zeros past them.  quads: by 16 bytes; full: E of them in all lanes.
template <int E>
__device__ __forceinline__ void lane_values(float (&v)[E], const float *p, int count, bool quads, bool full)
{
    if (E % 4 == 0 && quads && full) {
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const float4 q = *reinterpret_cast<const float4 *>(p + j);
            v[j] = q.x;
            v[j + 1] = q.y;
            v[j + 2] = q.z;
            v[j + 3] = q.w;
        }
    } else if (E % 4 == 0 && quads) {
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const float4 q = j < count ? *reinterpret_cast<const float4 *>(p + j) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[j] = q.x;
            v[j + 1] = q.y;
            v[j + 2] = q.z;
            v[j + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = j < count ? p[j] : 0.f;
    }
}

// A row of 16 lanes has a token: place E l + j of a row is experts' value j of lane l, and after the selection lane l has
// candidate l.  A group has group_lanes lanes, a power of two up to 16, the last of which may have fewer than E experts or
// none; places increase with the experts' numbers.  quads: the logits and the bias of all lanes begin on 16 bytes, and
// their numbers are multiples of four.
template <int E>
__global__ __launch_bounds__(kRouteWaves * 64) void route_rows_kernel(RouteHostArgs h, int group_lanes, bool quads)
{
    __shared__ double values[kRouteWaves][E < 4 ? 64 : 16 * E];
    constexpr unsigned kIndex = 16 * E - 1;    // the lower bits of a key: kIndex - place, so that of equal values
                                               // the lower number is the larger key
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token0 = ((int)blockIdx.x * kRouteWaves + w) * 4;
    if (token0 >= h.tokens) return;            // no barrier below: a wavefront has its tokens to itself
    const int l16 = lane & 15, row = lane - l16, token = min(token0 + lane / 16, h.tokens - 1);
    const bool biased = h.bias != nullptr, full = h.experts == 16 * E;
    const int group_shift = __builtin_ctz((unsigned)group_lanes), size = h.groups > 1 ? h.experts / h.groups : h.experts;
    const int group = l16 >> group_shift, at = (l16 & (group_lanes - 1)) * E, first_expert = group * size + at;
    const int count = group < h.groups ? min(max(size - at, 0), E) : 0;                  // of this lane
    const bool two = h.groups > 1 && h.group_top == 2;
    const bool scored = biased || two;                                  // all of them, not the candidates alone
    const bool all_sums = !h.sigmoid && (scored || !h.renormalise);
    const float *logits = h.logits + (size_t)token * h.experts;
    float l[E];
    lane_values(l, logits + first_expert, count, quads, full);
    float bias[E], error = 0.f;                          // of a bias that is infinite or NaN: not finite, nothing is sure
    if (biased) {
        unsigned largest = 0;
        lane_values(bias, h.bias + first_expert, count, quads, full);
#pragma unroll
        for (int j = 0; j < E; ++j) largest = max(largest, __float_as_uint(bias[j]) & 0x7FFFFFFFu);
        error = 0x1p-23f * __uint_as_float(row_max(largest));
    }
    if (scored) error += kScoreError + 0x1p-23f;         // of any value, twice what rounding a sum does
#pragma unroll
    for (int j = 0; j < E; ++j) l[j] = clean_logit(l[j]);
    if (!full) {
#pragma unroll
        for (int j = 0; j < E; ++j) l[j] = j < count ? l[j] : -__builtin_inff();
    }

    double top = 0.0, scale = 1.0;
    float v[E];
    if (!h.sigmoid) {
        float m = l[0];
#pragma unroll
        for (int j = 1; j < E; ++j) m = fmaxf(m, l[j]);
        top = (double)row_max(m);
        if (all_sums) {
            double part[E], sum = 0.0;
#pragma unroll
            for (int j = 0; j < E; ++j) sum += part[j] = softmax_part((double)l[j], top);
            sum = row_sum(sum);
            scale = sum > 0.0 ? 1.0 / sum : 0.0;
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = (float)(part[j] * scale);
        }
    } else if (scored) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = rough_sigmoid(l[j]);
    }
    if (biased) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] += bias[j];                   // (no sum is -0: no score is)
    } else if (!two) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = l[j];
    }
    if (!full) {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = j < count ? v[j] : -__builtin_inff();
    }
    bool taken = true, sure = error < __builtin_inff();
    if (h.groups > 1) {
        const bool sum_two = h.group_top == 2 && h.experts > h.groups;
        float first, second;
        largest_two(v, first, second);
        const float lane_first = first, lane_second = second;
        largest_two_of_group(group_lanes, first, second);
        const float value = sum_two ? first + second : first;
        // The largest value again and again.  It takes equal groups all at once, which their number tells.
        unsigned left = order_key(value), in = 0;
        taken = false;
#pragma unroll 1
        for (int g = 0; g < h.top_groups; ++g) {
            in = row_max(left);
            const bool here = left == in;
            taken |= here;
            left = here ? 0u : left;
        }
        // (row-uniform; two values of two scores each)
        const bool equal = (int)__popc((unsigned)(__ballot(taken) >> row) & 0xFFFFu) != h.top_groups * group_lanes;
        const bool near = equal || (scored && !(key_value(in) - key_value(row_max(left)) > 5.f * error));
        if (__ballot(near)) {
            bool before;
            if (scored) {
                // In binary64 those of a lane's scores that count, if it is certain which: none of another value
                // within its error.
                const float last = sum_two && lane_second > -__builtin_inff() ? lane_second : lane_first;
                const float least = last - 2.f * error;
                float l1 = 0.f, l2 = 0.f, b1 = 0.f, b2 = 0.f;
                int most = 0;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    l1 = v[j] == lane_first ? l[j] : l1;
                    l2 = v[j] == lane_second ? l[j] : l2;
                    most += v[j] >= least;
                }
                if (biased) {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        b1 = v[j] == lane_first ? bias[j] : b1;
                        b2 = v[j] == lane_second ? bias[j] : b2;
                    }
                }
                const auto score = [&](float l) {
                    return h.sigmoid ? sigmoid_score((double)l) : softmax_part((double)l, top) * scale;
                };
                const bool none = lane_first == -__builtin_inff();             // a lane of no group
                double a = none ? -__builtin_inf() : score(l1) + (double)b1;
                double b = lane_second == -__builtin_inff() ? -__builtin_inf() : score(l2) + (double)b2;
                if (b > a) {
                    const double c = a;
                    a = b;
                    b = c;
                }
                const bool certain = none || (most <= (sum_two ? 2 : 1) && !(sum_two && lane_first == lane_second));
                sure &= !(near && (unsigned)(__ballot(!certain) >> row) & 0xFFFFu);
                largest_two_of_group(group_lanes, a, b);
                before = groups_before(sum_two ? a + b : a, h.groups, group_lanes) < h.top_groups;
            } else {
                before = groups_before(value, h.groups, group_lanes) < h.top_groups;
            }
            taken = near ? before : taken;
        }
        if (two && !biased) {                                          // the experts' order is that of the logits
#pragma unroll
            for (int j = 0; j < E; ++j) v[j] = l[j];
        }
    }
    unsigned key[E];                                                   // never 0 but for what takes no part
#pragma unroll
    for (int j = 0; j < E; ++j) {
        key[j] = (order_key(v[j]) & ~kIndex) | (kIndex - (unsigned)(l16 * E + j));
        key[j] = taken ? key[j] : 0u;
    }
    if (!full) {
#pragma unroll
        for (int j = 0; j < E; ++j) key[j] = j < count ? key[j] : 0u;
    }

    // The largest key of the token again and again; top_k + 1 of them, and the value of the next.  If that is not enough
    // to be sure, all 16 that the row has lanes for.
    unsigned candidate = 0;
    int found = 0, wanted = h.top_k + 1, expert, rank;
    bool lives;
    double score;
    unsigned long long unsure;
    sort_fours(key);
    for (;;) {
#pragma unroll 1
        for (; found < wanted; ++found) {
            const unsigned best = row_max(largest_key(key));
            candidate = l16 == found ? best : candidate;
            remove_key(key, best);
        }
        const unsigned rest = row_max(largest_key(key));
        lives = candidate != 0;
        const unsigned place = kIndex - (candidate & kIndex);
        expert = lives ? (int)(place - (place / E >> group_shift) * (unsigned)(group_lanes * E - size)) : 0;
        const float its_bias = biased ? h.bias[expert] : 0.f;
        const float logit = clean_logit(logits[expert]);
        score = h.sigmoid ? sigmoid_score((double)logit) : softmax_part((double)logit, top);
        if (all_sums) score *= scale;
        double order = biased ? score + (double)its_bias : (double)logit;
        if (order != order || !lives) order = -__builtin_inf();
        // They come in the order of their words: nearly always that of their values.
        rank = l16;
        const double next = __shfl(order, row + min(l16 + 1, 15));             // (by all lanes)
        const int next_lives = __shfl((int)lives, row + min(l16 + 1, 15));
        if (__ballot(l16 + 1 < wanted && next_lives && !(order > next))) {
            rank = 0;
            for (int c = 0; c < wanted; ++c) {
                const double o = __shfl(order, row + c);
                const int oe = __shfl(lives ? expert : kNone, row + c);
                rank += oe != kNone && (o > order || (o == order && oe < expert));
            }
        }
        // The last one chosen has to be ahead of everything that is no candidate: the next word's value is at most this.
        // (-infinity is what it is, and equal ones are in order.)
        bool ahead = sure;
        if (ahead && lives && rank == h.top_k - 1 && rest != 0) {
            const float most = key_value(rest | kIndex);
            ahead = order > (double)most + (biased ? (double)error : 0.0) || most == -__builtin_inff();
        }
        unsure = __ballot(!ahead);
        if (!unsure || wanted == 16) break;
        wanted = 16;
    }
    const bool chosen = lives && rank < h.top_k;
    if (h.renormalise) {
        const double total = row_sum(chosen ? score : 0.0);
        score = total > 0.0 ? score / total : 0.0;
    }
    if (chosen && token0 + lane / 16 < h.tokens && !(unsure >> row & 0xFFFF)) {
        h.idx[(size_t)token * h.top_k + rank] = expert;
        h.weight[(size_t)token * h.top_k + rank] = (float)(score * (double)h.scaling);
    }
    if (unsure) {
        for (int c = 0; c < 4; ++c)
            if (unsure >> 16 * c & 0xFFFF && token0 + c < h.tokens)
                route_exactly<(E + 3) / 4>(h, token0 + c, values[w]);
    }
}

template <int E>
__global__ __launch_bounds__(kRouteWaves * 64) void route_exactly_kernel(RouteHostArgs h)
{
    __shared__ double values[kRouteWaves][E * 64];
    const int w = threadIdx.x >> 6, token = blockIdx.x * kRouteWaves + w;
    if (token < h.tokens) route_exactly<E>(h, token, values[w]);
}

}  // namespace

hipError_t launch_route_experts(const RouteHostArgs &args, hipStream_t stream)
{
    RouteHostArgs h = args;
    if (h.top_groups == h.groups) h.groups = h.top_groups = 1;      // all take part
    const int size = h.experts / h.groups;
    int group_lanes = 16, per_lane = 1;        // of a row
    while (group_lanes * h.groups > 16) group_lanes /= 2;
    while (group_lanes * per_lane < size && per_lane <= 32) per_lane *= 2;
    const dim3 block(kRouteWaves * 64);
    if (group_lanes > 0 && per_lane <= 32 && h.top_k < 16) {
        const bool quads = size % 4 == 0 && (reinterpret_cast<uintptr_t>(h.logits) & 15) == 0 &&
                           (reinterpret_cast<uintptr_t>(h.bias) & 15) == 0;
        const dim3 grid((unsigned)((h.tokens + 4 * kRouteWaves - 1) / (4 * kRouteWaves)));
#define TEAL_ROUTE(E) hipLaunchKernelGGL(route_rows_kernel<E>, grid, block, 0, stream, h, group_lanes, quads)
        if (per_lane == 1) TEAL_ROUTE(1);
        else if (per_lane == 2) TEAL_ROUTE(2);
        else if (per_lane == 4) TEAL_ROUTE(4);
        else if (per_lane == 8) TEAL_ROUTE(8);
        else if (per_lane == 16) TEAL_ROUTE(16);
        else TEAL_ROUTE(32);
#undef TEAL_ROUTE
        return hipGetLastError();
    }
    const dim3 grid((unsigned)((h.tokens + kRouteWaves - 1) / kRouteWaves));
#define TEAL_ROUTE(E) hipLaunchKernelGGL(route_exactly_kernel<E>, grid, block, 0, stream, h)
    if (h.experts <= 64) TEAL_ROUTE(1);
    else if (h.experts <= 128) TEAL_ROUTE(2);
    else if (h.experts <= 256) TEAL_ROUTE(4);
    else if (h.experts <= 512) TEAL_ROUTE(8);
    else TEAL_ROUTE(16);
#undef TEAL_ROUTE
    return hipGetLastError();
}

}  // namespace teal
