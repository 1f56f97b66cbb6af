// Routing to experts: scores from a router's logits, the top_k experts of each token and their weights.
//
// The result is defined in binary64, but hardly a token needs all of its scores there.  fp32 values (the score and a
// bias, or the logit), cut to the upper bits of a word above the expert's number, find top_k + 1 candidates, and
// their binary64 scores, which are the weights, put those in order.  What the words left out matters only if a
// third value lies within their error of the last one chosen: such tokens (one in 10^5 of ordinary ones) take a
// wavefront each, by binary64 values throughout, and so do more than 512 experts or 15 of them chosen, and groups that do
// not end with a lane's experts.  Groups whose fp32 values are too near each other are valued again in binary64.
//
// What bounds it is instruction issue.  (us for 16384 tokens of 256 experts in 8 groups, 4 groups and 8 experts taken,
// sigmoid scores and a bias; reading the logits takes 4: a wavefront per token in binary64 46; the selection on fp32
// scores, the place of each maximum found by ballots, 28; a row of lanes per token on words, with all scores in
// binary64, 24; fp32 scores and keys in sorted fours 16.)
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
__device__ __forceinline__ float row_min(float v)
{
    v = fminf(v, row_rotate<1>(v));
    v = fminf(v, row_rotate<2>(v));
    v = fminf(v, row_rotate<4>(v));
    return fminf(v, row_rotate<8>(v));
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

// Order of floats as that of unsigned numbers, none of them zero; -0 and 0 are equal.
__device__ __forceinline__ unsigned order_key(float v)
{
    const unsigned u = __float_as_uint(v + 0.f);
    return u ^ ((int)u < 0 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float key_value(unsigned key)
{
    return __uint_as_float(key ^ ((int)key < 0 ? 0x80000000u : 0xFFFFFFFFu));
}

// A logit as it counts: NaN as -infinity, +infinity as the largest finite number.
__device__ __forceinline__ float clean_logit(float l) { return l != l ? -__builtin_inff() : fminf(l, 3.402823466e38f); }

// exp(x) for x of at most 709.78 to a last place or two: x = k ln 2 + r, the Taylor polynomial of degree 12 at
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
__device__ __forceinline__ double sigmoid_score(double z)
{
    return z < -709.78 ? 0.0 : reciprocal(1.0 + exponential(-fmax(z, -709.78)));
}
__device__ __forceinline__ double softmax_part(double z, double top)
{
    return z == -__builtin_inf() ? 0.0 : exponential(z - top);
}

// fp32 sigmoid from the hardware's exponential and reciprocal.  What a wrong last place of the argument, of at most
// 88 log2 e where it matters, does to s is below s (1 - s) |l| 2^-23 < 2^-25; a few last places of numbers of at most 1
// come on top.
__device__ __forceinline__ float rough_sigmoid(float l)
{
    return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * l));
}
constexpr float kScoreError = 0x1p-20f;

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

// The two largest values of a lane's experts, then of a group in its `lanes` lanes (a power of two up to 16).
template <int E, class V>
__device__ __forceinline__ void largest_two(const V (&v)[E], int lanes, V &first, V &second)
{
    const auto larger = [](V a, V b) { return a > b ? a : b; };
    const auto smaller = [](V a, V b) { return a > b ? b : a; };
    first = v[0];
    second = -__builtin_inff();
#pragma unroll
    for (int j = 1; j < E; ++j) {
        if constexpr (sizeof(V) == 4) second = __builtin_amdgcn_fmed3f(first, second, v[j]);
        else second = larger(second, smaller(first, v[j]));
        first = larger(first, v[j]);
    }
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
    const int lane = threadIdx.x & 63, row = lane & 48, group = (lane & 15) / group_lanes;
    int before = 0;
#pragma unroll 1
    for (int g = 0; g < groups; g += 4) {
        V x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) x[u] = __shfl(value, row + min((g + u) * group_lanes, 15));
#pragma unroll
        for (int u = 0; u < 4; ++u) before += g + u < groups && (x[u] > value || (x[u] == value && g + u < group));
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

// E values from place E * l16 on of the `count` at p, zeros past the end.  quads: by 16 bytes.
template <int E>
__device__ __forceinline__ void lane_values(float (&v)[E], const float *p, int l16, int count, bool quads)
{
    if (E % 4 == 0 && quads) {
#pragma unroll
        for (int j = 0; j < E; j += 4) {
            const float4 q = l16 * E + j < count ? *reinterpret_cast<const float4 *>(p + l16 * E + j)
                                                 : make_float4(0.f, 0.f, 0.f, 0.f);
            v[j] = q.x;
            v[j + 1] = q.y;
            v[j + 2] = q.z;
            v[j + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < E; ++j) v[j] = l16 * E + j < count ? p[l16 * E + j] : 0.f;
    }
}

// A row of 16 lanes has a token, a lane of it experts E l .. E l + E - 1, and after the selection candidate l.
// group_lanes: lanes of a group, a power of two up to 16.  quads: logits and bias begin on 16 bytes, and their number is
// a multiple of four.
template <int E>
__global__ __launch_bounds__(kRouteWaves * 64) void route_rows_kernel(RouteHostArgs h, int group_lanes, bool quads)
{
    __shared__ double values[kRouteWaves][E < 4 ? 64 : 16 * E];
    constexpr unsigned kIndex = 16 * E - 1;    // the lower bits of a key: kIndex - expert, so that of equal values
                                               // the lower number is the larger key
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token0 = ((int)blockIdx.x * kRouteWaves + w) * 4;
    if (token0 >= h.tokens) return;            // no barrier below: a wavefront has its tokens to itself
    const int l16 = lane & 15, row = lane - l16, token = min(token0 + lane / 16, h.tokens - 1);
    const bool biased = h.bias != nullptr, full = h.experts == 16 * E;
    const bool two = h.groups > 1 && h.group_top == 2;
    const bool scored = biased || two;                                  // all of them, not the candidates alone
    const bool all_sums = !h.sigmoid && (scored || !h.renormalise);
    const float *logits = h.logits + (size_t)token * h.experts;
    float l[E];
    lane_values(l, logits, l16, h.experts, quads);
    float bias[E], error = 0.f;
    if (biased) {
        float largest = 0.f;
        lane_values(bias, h.bias, l16, h.experts, quads);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            bias[j] = bias[j] != bias[j] ? -__builtin_inff() : bias[j];
            largest = fmaxf(largest, fabsf(bias[j]));
        }
        error = 0x1p-23f * row_max(largest);             // (of an infinite one: nothing is sure)
    }
    if (scored) error += kScoreError + 0x1p-23f;         // of any value, twice what rounding a sum does
#pragma unroll
    for (int j = 0; j < E; ++j) l[j] = clean_logit(l[j]);
    if (!full) {
#pragma unroll
        for (int j = 0; j < E; ++j) l[j] = l16 * E + j < h.experts ? l[j] : -__builtin_inff();
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
#pragma unroll
    for (int j = 0; j < E; ++j) {
        if (biased) v[j] += bias[j];
        else if (!two) v[j] = l[j];
    }
    unsigned key[E];                                                   // never 0 but for what takes no part
#pragma unroll
    for (int j = 0; j < E; ++j)
        key[j] = (order_key(biased ? v[j] : l[j]) & ~kIndex) | (kIndex - (unsigned)(l16 * E + j));
    if (!full) {
#pragma unroll
        for (int j = 0; j < E; ++j) {
            key[j] = l16 * E + j < h.experts ? key[j] : 0u;
            v[j] = l16 * E + j < h.experts ? v[j] : -__builtin_inff();
        }
    }
    if (h.groups > 1) {
        const bool sum_two = h.group_top == 2 && h.experts > h.groups;
        float first, second;
        largest_two(v, group_lanes, first, second);
        const float value = sum_two ? first + second : first;
        const bool member = l16 / group_lanes < h.groups;
        bool taken = groups_before(value, h.groups, group_lanes) < h.top_groups;
        if (scored && h.top_groups < h.groups) {
            const float in = row_min(taken && member ? value : __builtin_inff());
            const float out = row_max(!taken && member ? value : -__builtin_inff());
            // two values of two scores each
            if (__ballot(!(in - out > 5.f * error))) {
                double z[E], a, b;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    z[j] = h.sigmoid ? sigmoid_score((double)l[j]) : softmax_part((double)l[j], top) * scale;
                    if (biased) z[j] += (double)bias[j];
                    z[j] = full || l16 * E + j < h.experts ? z[j] : -__builtin_inf();
                }
                largest_two(z, group_lanes, a, b);
                double exact = sum_two ? a + b : a;
                exact = exact != exact ? -__builtin_inf() : exact;
                taken = groups_before(exact, h.groups, group_lanes) < h.top_groups;
            }
        }
#pragma unroll
        for (int j = 0; j < E; ++j) key[j] = taken ? key[j] : 0u;
    }

    // The largest key of the token again and again; top_k + 1 of them, and the value of the next.
    unsigned candidate = 0, rest = 0;
    sort_fours(key);
#pragma unroll 1
    for (int c = 0; c <= h.top_k + 1; ++c) {
        rest = row_max(largest_key(key));
        candidate = l16 == c ? rest : candidate;
        remove_key(key, rest);
    }

    const bool lives = candidate != 0 && l16 <= h.top_k;
    const int expert = lives ? (int)(kIndex - (candidate & kIndex)) : 0;
    const float logit = clean_logit(logits[expert]);
    double score = h.sigmoid ? sigmoid_score((double)logit) : softmax_part((double)logit, top);
    if (all_sums) score *= scale;
    double order = biased ? score + (double)h.bias[expert] : (double)logit;
    if (order != order || !lives) order = -__builtin_inf();
    // They come in the order of their words: nearly always that of their values.
    int rank = l16;
    const double next = __shfl(order, row + min(l16 + 1, 15));             // (by all lanes)
    const int next_lives = __shfl((int)lives, row + min(l16 + 1, 15));
    if (__ballot(l16 < h.top_k && next_lives && !(order > next))) {
        rank = 0;
        for (int c = 0; c <= h.top_k; ++c) {
            const double o = __shfl(order, row + c);
            const int oe = __shfl(lives ? expert : kNone, row + c);
            rank += oe != kNone && (o > order || (o == order && oe < expert));
        }
    }
    // The last one chosen has to be ahead of everything that is no candidate: the next word's value is at most this.
    // (-infinity is what it is, and equal ones are in order.)
    bool sure = true;
    if (lives && rank == h.top_k - 1 && rest != 0) {
        const float most = key_value(rest | kIndex);
        sure = order > (double)most + (biased ? (double)error : 0.0) || most == -__builtin_inff();
    }
    const bool chosen = lives && rank < h.top_k;
    if (h.renormalise) {
        const double total = row_sum(chosen ? score : 0.0);
        score = total > 0.0 ? score / total : 0.0;
    }
    const unsigned long long unsure = __ballot(!sure);
    if (chosen && token0 + lane / 16 < h.tokens && !(unsure >> row & 0xFFFF)) {
        h.idx[(size_t)token * h.top_k + rank] = expert;
        h.weight[(size_t)token * h.top_k + rank] = (float)(score * (double)h.scaling);
    }
    for (int c = 0; c < 4; ++c)
        if (unsure >> 16 * c & 0xFFFF && token0 + c < h.tokens)
            route_exactly<(E + 3) / 4>(h, token0 + c, values[w]);
}

template <int E>
__global__ __launch_bounds__(kRouteWaves * 64) void route_exactly_kernel(RouteHostArgs h)
{
    __shared__ double values[kRouteWaves][E * 64];
    const int w = threadIdx.x >> 6, token = blockIdx.x * kRouteWaves + w;
    if (token < h.tokens) route_exactly<E>(h, token, values[w]);
}

}  // namespace

hipError_t launch_route_experts(const RouteHostArgs &h, hipStream_t stream)
{
    int per_lane = 1;                          // of a row
    while (16 * per_lane < h.experts) per_lane *= 2;
    const int size = h.experts / h.groups, lanes = size / per_lane;
    const bool by_lanes = h.groups == 1 || (size % per_lane == 0 && (lanes & (lanes - 1)) == 0);
    const int group_lanes = h.groups == 1 ? 16 : lanes;
    const dim3 block(kRouteWaves * 64);
    if (by_lanes && per_lane <= 32 && h.top_k < 16) {
        const bool quads = h.experts % 4 == 0 && (reinterpret_cast<uintptr_t>(h.logits) & 15) == 0 &&
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
