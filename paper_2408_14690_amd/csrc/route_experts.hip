// Routing to experts: scores from a router's logits, the top_k experts of each token and their weights.
#include <hip/hip_runtime.h>

#include "teal_internal.h"

namespace teal {

namespace {

constexpr int kRouteWaves = 4;

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

// One wavefront per token; lane l has experts l, l + 64, ...  Scores are formed in binary64: two that are next to
// each other decide which expert is chosen, and with a bias on them that is no longer the order of the logits.
template <int E>
__global__ __launch_bounds__(kRouteWaves * 64) void route_experts_kernel(RouteHostArgs h)
{
    __shared__ double shared_values[kRouteWaves][E * 64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int token = blockIdx.x * kRouteWaves + w;
    if (token >= h.tokens) return;             // no barrier below: a wavefront has its token to itself
    double *values = shared_values[w];

    const float *logits = h.logits + (size_t)token * h.experts;
    double z[E], score[E], order[E];
    unsigned available = 0;
    double top = -__builtin_inf();
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const int e = lane + 64 * j;
        float l = e < h.experts ? logits[e] : -__builtin_inff();
        available |= (unsigned)(e < h.experts) << j;
        l = l != l ? -__builtin_inff() : fminf(l, 3.402823466e38f);
        z[j] = l;
        top = fmax(top, z[j]);
    }
    if (h.sigmoid) {
#pragma unroll
        for (int j = 0; j < E; ++j) score[j] = 1.0 / (1.0 + exp(-z[j]));
    } else {
        top = wave_max(top);
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            score[j] = z[j] == -__builtin_inf() ? 0.0 : exp(z[j] - top);
            sum += score[j];
        }
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
        for (int j = 0; j < E; ++j) {
            // two experts' logits say nothing about the sum of their scores
            double v = order[j];
            if (h.group_top == 2 && !h.bias) v = score[j];
            values[lane + 64 * j] = v;
        }
        __builtin_amdgcn_wave_barrier();
        double first = -__builtin_inf(), second = -__builtin_inf();
        if (lane < h.groups)
            for (int k = 0; k < size; ++k) {
                const double v = values[lane * size + k];
                second = fmax(second, fmin(first, v));
                first = fmax(first, v);
            }
        double value = first;
        if (h.group_top == 2 && size > 1) value = first + second;
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
        int at = 0x7fffffff;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const bool free = available >> j & 1;
            if (free && (at == 0x7fffffff || order[j] > best)) {
                best = order[j];
                at = lane + 64 * j;
            }
        }
        for (int d = 32; d; d >>= 1) {
            const double v = __shfl_xor(best, d);
            const int o = __shfl_xor(at, d);
            const bool take = o != 0x7fffffff && (at == 0x7fffffff || v > best || (v == best && o < at));
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

}  // namespace

hipError_t launch_route_experts(const RouteHostArgs &h, hipStream_t stream)
{
    const dim3 grid((unsigned)((h.tokens + kRouteWaves - 1) / kRouteWaves)), block(kRouteWaves * 64);
#define TEAL_ROUTE(E) hipLaunchKernelGGL(route_experts_kernel<E>, grid, block, 0, stream, h)
    if (h.experts <= 64) TEAL_ROUTE(1);
    else if (h.experts <= 128) TEAL_ROUTE(2);
    else if (h.experts <= 256) TEAL_ROUTE(4);
    else if (h.experts <= 512) TEAL_ROUTE(8);
    else TEAL_ROUTE(16);
#undef TEAL_ROUTE
    return hipGetLastError();
}

}  // namespace teal
