// Routing to experts: scores from a router's logits, the top_k experts of each token and their weights.
//
// The result is defined in binary64, but hardly a token needs all of its scores there.  Without a bias the experts
// are ranked by their logits as they are; with one, fp32 scores (wrong by at most kScoreError) find the top_k + 1
// candidates, whose binary64 scores (they are the weights) put them in order.  What the fp32 scores left behind
// may still matter only if it lies within their error of the last one chosen, and a group left out only within
// theirs of the last one taken: those tokens (about 1 in 5000 of ordinary ones) and groups that do not end
// with a lane's experts are ranked in binary64 as a whole.
//
// What bounds it is instruction issue: a maximum over a wavefront for every expert chosen.  (16384 tokens of 256
// experts in 8 groups, 4 groups and 8 experts taken, with a bias, all in binary64 with shuffles through LDS: 46 us;
// reading the logits takes 4 us.)
#include <hip/hip_runtime.h>

#include "teal_internal.h"

namespace teal {

namespace {

constexpr int kRouteWaves = 4;
constexpr int kNone = 0x7fffffff;

template <int CTRL, int ROWS>
__device__ __forceinline__ unsigned dpp_or_zero(unsigned v)
{
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true);
}

// Largest of a value over the wavefront (zero is the smallest there is).
__device__ __forceinline__ unsigned wave_umax(unsigned v)
{
    v = max(v, dpp_or_zero<0x111, 0xF>(v));   // row_shr:1, 2, 4, 8
    v = max(v, dpp_or_zero<0x112, 0xF>(v));
    v = max(v, dpp_or_zero<0x114, 0xF>(v));
    v = max(v, dpp_or_zero<0x118, 0xF>(v));
    v = max(v, dpp_or_zero<0x142, 0xA>(v));   // row_bcast:15 -> rows 1, 3
    v = max(v, dpp_or_zero<0x143, 0xC>(v));   // row_bcast:31 -> rows 2, 3
    return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
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

__device__ __forceinline__ double sigmoid_score(double z) { return 1.0 / (1.0 + exp(-z)); }
__device__ __forceinline__ double softmax_part(double z, double top)
{
    return z == -__builtin_inf() ? 0.0 : exp(z - top);
}

// fp32 sigmoid from the hardware's exponential and reciprocal: what a wrong last place of the argument, of at most 88 |log2 e|,
// does to s is below s (1 - s) |l| 2^-23, which is below 2^-25; a few last places of a number of at most 1 come on top.
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
        const double value = h.group_top == 2 && size > 1 ? first + second : first;
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

// The two largest values of a group in its `lanes` lanes (a power of two), in all of them.
template <int CTRL>
__device__ __forceinline__ void merge_two(float &first, float &second)
{
    const float a = __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(first), CTRL, 0xF, 0xF, false));
    const float b = __uint_as_float((unsigned)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(second), CTRL, 0xF, 0xF, false));
    second = fmaxf(fminf(first, a), fmaxf(second, b));
    first = fmaxf(first, a);
}
__device__ __forceinline__ void merge_group(float &first, float &second, int lanes)
{
    if (lanes > 1) merge_two<0xB1>(first, second);      // lane ^ 1, lane ^ 2, the other quad, the other half of a row
    if (lanes > 2) merge_two<0x4E>(first, second);
    if (lanes > 4) merge_two<0x141>(first, second);
    if (lanes > 8) merge_two<0x140>(first, second);
    for (int d = 16; d < lanes; d *= 2) {
        const float a = __shfl_xor(first, d), b = __shfl_xor(second, d);
        second = fmaxf(fminf(first, a), fmaxf(second, b));
        first = fmaxf(first, a);
    }
}

// A wavefront selects the candidates of TOKENS tokens one after the other, lane l with experts E l .. E l + E - 1, and
// leaves those of token k in lanes k * W .. ; then a lane has one candidate, and the binary64 work is done for all of
// them at once.  group_lanes: lanes of a group, a power of two (one group: 64).
template <int E, int TOKENS>
__global__ __launch_bounds__(kRouteWaves * 64) void route_experts_kernel(RouteHostArgs h, int group_lanes)
{
    constexpr int W = 64 / TOKENS;
    __shared__ double values[kRouteWaves][E * 64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int token0 = ((int)blockIdx.x * kRouteWaves + w) * TOKENS;
    if (token0 >= h.tokens) return;            // no barrier below: a wavefront has its tokens to itself
    const bool biased = h.bias != nullptr;
    // whether the order below comes from rounded scores
    const bool rounded = biased, rounded_groups = biased || h.group_top == 2;
    const bool all_sums = !h.sigmoid && (biased || !h.renormalise || (h.groups > 1 && h.group_top == 2));
    const int wanted = h.top_k + (rounded ? 1 : 0);
    float bias[E], error = kScoreError + 0x1p-23f;       // of any rounded s + bias, twice what rounding the sum does
    if (biased) {
        unsigned largest = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int e = lane * E + j;
            bias[j] = e < h.experts ? h.bias[e] : 0.f;
            largest = max(largest, __float_as_uint(fabsf(bias[j])));
        }
        error += 0x1p-23f * __uint_as_float(wave_umax(largest));      // (not a number: nothing is sure)
    }

    int candidate = kNone;                     // of this lane's slot
    double top = 0.0, sum = 1.0;               // of its token
    float rest = -__builtin_inff();            // largest rounded value that is no candidate
    unsigned unsure = 0;                       // bit k: token k
#pragma unroll 1
    for (int k = 0; k < TOKENS; ++k) {
        const int token = token0 + k;
        if (token >= h.tokens) break;
        const float *logits = h.logits + (size_t)token * h.experts;
        float l[E], v[E];
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const int e = lane * E + j;
            l[j] = e < h.experts ? clean_logit(logits[e]) : -__builtin_inff();
        }
        float score[E];
        if (h.sigmoid) {
            if (biased || rounded_groups) {
#pragma unroll
                for (int j = 0; j < E; ++j)
                    score[j] = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-1.44269504f * l[j]));
            }
        } else {
            float m = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < E; ++j) m = fmaxf(m, l[j]);
            const double t = (double)key_value(wave_umax(order_key(m)));
            double total = 0.0, part[E];
            if (all_sums) {
#pragma unroll
                for (int j = 0; j < E; ++j) total += part[j] = softmax_part((double)l[j], t);
                total = wave_sum(total);
#pragma unroll
                for (int j = 0; j < E; ++j) score[j] = total > 0.0 ? (float)(part[j] / total) : 0.f;
            }
            top = lane / W == k ? t : top;
            sum = lane / W == k ? total : sum;
        }
#pragma unroll
        for (int j = 0; j < E; ++j) {
            v[j] = biased ? score[j] + bias[j] : l[j];
            if (v[j] != v[j]) v[j] = -__builtin_inff();
        }
        unsigned key[E];
#pragma unroll
        for (int j = 0; j < E; ++j) key[j] = lane * E + j < h.experts ? order_key(v[j]) : 0u;
        if (h.groups > 1) {
            float first = -__builtin_inff(), second = -__builtin_inff();
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const float x = h.group_top == 2 && !biased ? score[j] : v[j];
                second = fmaxf(second, fminf(first, x));
                first = fmaxf(first, x);
            }
            merge_group(first, second, group_lanes);
            const bool two = h.group_top == 2 && h.experts > h.groups;
            const float value = two ? first + second : first;
            const int group = lane / group_lanes;
            int before = 0;
            for (int g = 0; g < h.groups; ++g) {
                const float x = __uint_as_float((unsigned)__builtin_amdgcn_readlane((int)__float_as_uint(value), g * group_lanes));
                before += x > value || (x == value && g < group);
            }
            const bool taken = before < h.top_groups;
            if (rounded_groups && h.top_groups < h.groups) {
                const bool lives = group < h.groups;
                const unsigned long long last = __ballot(lives && before == h.top_groups - 1);
                const unsigned long long next = __ballot(lives && before == h.top_groups);
                // (a value that is no number leaves a rank without a group)
                bool clear = last != 0 && next != 0;
                if (clear) {
                    const float a = __shfl(value, __ffsll((long long)last) - 1);
                    const float b = __shfl(value, __ffsll((long long)next) - 1);
                    clear = a - b > 5.f * error;          // two values of two scores each
                }
                if (!clear) unsure |= 1u << k;
            }
#pragma unroll
            for (int j = 0; j < E; ++j) key[j] = taken ? key[j] : 0u;
        }
#pragma unroll 1
        for (int c = 0; c < wanted; ++c) {
            unsigned best = key[0];
#pragma unroll
            for (int j = 1; j < E; ++j) best = max(best, key[j]);
            const unsigned largest = wave_umax(best);
            if (largest == 0) break;                                   // fewer than top_k + 1
            int first = E - 1;                                         // the first of this lane's that has it
#pragma unroll
            for (int j = E - 2; j >= 0; --j) first = key[j] == largest ? j : first;
            const int from = __ffsll((long long)__ballot(best == largest)) - 1;
            const int e = from * E + __builtin_amdgcn_readlane(first, from);
            candidate = lane == k * W + c ? e : candidate;
            const int mine = e - lane * E;                             // 0..E - 1 in that lane alone
#pragma unroll
            for (int j = 0; j < E; ++j) key[j] = mine == j ? 0u : key[j];
        }
        if (rounded) {
            unsigned best = key[0];
#pragma unroll
            for (int j = 1; j < E; ++j) best = max(best, key[j]);
            const unsigned largest = wave_umax(best);
            const float r = largest ? key_value(largest) : -__builtin_inff();
            rest = lane / W == k ? r : rest;
        }
    }

    // One candidate a lane.
    const int k = lane / W, slot = lane % W, token = token0 + k, base = lane - slot;
    const bool lives = candidate != kNone;
    double score = 0.0, v = -__builtin_inf();
    if (lives) {
        const double z = (double)clean_logit(h.logits[(size_t)token * h.experts + candidate]);
        score = h.sigmoid ? sigmoid_score(z) : softmax_part(z, top);
        if (all_sums) score = sum > 0.0 ? score / sum : 0.0;
        v = biased ? score + (double)h.bias[candidate] : z;
        if (v != v) v = -__builtin_inf();
    }
    int rank = slot;
    if (rounded) {
        rank = 0;
        for (int c = 0; c < wanted; ++c) {
            const double o = __shfl(v, base + c);
            const int oe = __shfl(candidate, base + c);
            rank += oe != kNone && (o > v || (o == v && oe < candidate));
        }
        // the last one chosen is ahead of everything that is no candidate, whatever the rounding did
        const bool close = lives && rank == h.top_k - 1 && rest > -__builtin_inff() &&
                           !(v > (double)rest + (double)error);
        const unsigned long long near = __ballot(close);
        for (int c = 0; c < TOKENS; ++c)
            if (near >> (c * W) & (W == 64 ? ~0ull : (1ull << (W & 63)) - 1)) unsure |= 1u << c;
    }
    const bool chosen = lives && rank < h.top_k;
    double total = chosen ? score : 0.0;
    if (h.renormalise)
        for (int d = 1; d < W; d *= 2) total += __shfl_xor(total, d);
    if (chosen && !(unsure >> k & 1)) {
        double x = score;
        if (h.renormalise) x = total > 0.0 ? score / total : 0.0;
        h.idx[(size_t)token * h.top_k + rank] = candidate;
        h.weight[(size_t)token * h.top_k + rank] = (float)(x * (double)h.scaling);
    }
    for (int c = 0; unsure; ++c, unsure >>= 1)
        if (unsure & 1) route_exactly<E>(h, token0 + c, values[w]);
}

template <int E>
__global__ __launch_bounds__(kRouteWaves * 64) void route_exactly_kernel(RouteHostArgs h)
{
    __shared__ double values[kRouteWaves][E * 64];
    const int w = threadIdx.x >> 6, token = blockIdx.x * kRouteWaves + w;
    if (token < h.tokens) route_exactly<E>(h, token, values[w]);
}

}  // namespace

// Tokens of a wavefront: four share the binary64 work where there are enough of them to fill the units all the same.
constexpr int kManyTokens = 8192;

hipError_t launch_route_experts(const RouteHostArgs &h, hipStream_t stream)
{
    int per_lane = 1;
    while (64 * per_lane < h.experts) per_lane *= 2;
    const int size = h.experts / h.groups, lanes = size / per_lane;
    const bool by_lanes = h.groups == 1 || (size % per_lane == 0 && (lanes & (lanes - 1)) == 0);
    const int group_lanes = h.groups == 1 ? 64 : lanes;
    const int tokens = by_lanes && h.top_k < 16 && h.tokens >= kManyTokens ? 4 : 1;
    const int per_block = kRouteWaves * tokens;
    const dim3 grid((unsigned)((h.tokens + per_block - 1) / per_block)), block(kRouteWaves * 64);
#define TEAL_ROUTE(E)                                                                          \
    do {                                                                                       \
        if (!by_lanes) hipLaunchKernelGGL(route_exactly_kernel<E>, grid, block, 0, stream, h); \
        else if (tokens == 4)                                                                  \
            hipLaunchKernelGGL((route_experts_kernel<E, 4>), grid, block, 0, stream, h, group_lanes); \
        else hipLaunchKernelGGL((route_experts_kernel<E, 1>), grid, block, 0, stream, h, group_lanes); \
    } while (0)
    if (per_lane == 1) TEAL_ROUTE(1);
    else if (per_lane == 2) TEAL_ROUTE(2);
    else if (per_lane == 4) TEAL_ROUTE(4);
    else if (per_lane == 8) TEAL_ROUTE(8);
    else TEAL_ROUTE(16);
#undef TEAL_ROUTE
    return hipGetLastError();
}

}  // namespace teal
