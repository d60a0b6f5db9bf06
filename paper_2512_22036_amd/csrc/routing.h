// Routing of tokens to experts: scores, a bias for balance, groups, top-k, weights; and the gradient of the weights.
//
//   s = sigmoid(l) = 1 / (1 + exp(-l)), or exp(l - max l) / sum exp(l - max l)
//   experts compete by b = s + bias (without a bias the softmax's denominator, common to a row, is left out); with groups, a group counts
//   as much as its group_best largest b together, and only experts of the keep_groups best groups compete
//   chosen: the k largest b, descending, ties to the lower index;  w = scale * s / (sum of the chosen s)  or  scale * s
//
// LANES lanes of a wave hold one row, VPL values each: expert e is value e / LANES of lane e % LANES.
#ifndef FUSCO_CSRC_ROUTING_H
#define FUSCO_CSRC_ROUTING_H

#include "common.h"

namespace {

constexpr int kRouteThreads = 256;

struct RouteArgs {
    const char *logits;
    const float *bias;
    int32_t *chosen;       // [N, k]
    float *w;              // [N, k]
    const float *dw;       // backward: [N, k]
    char *dlogits;         // backward: [N, E] of the logits' type
    int64_t stride;        // elements from row to row of the logits
    int32_t N, E, k, groups, keep_groups, group_best, group_size;
    int32_t bf16, sigmoid, renorm;
    float scale;
};

template <int LANES>
__device__ __forceinline__ float lanes_max(float v)
{
#pragma unroll
    for (int d = LANES / 2; d >= 1; d /= 2) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

template <int LANES>
__device__ __forceinline__ float lanes_sum(float v)
{
#pragma unroll
    for (int d = LANES / 2; d >= 1; d /= 2) v += __shfl_xor(v, d);
    return v;
}

template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v)
{
#pragma unroll
    for (int d = LANES / 2; d >= 1; d /= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
        v = o > v ? o : v;
    }
    return v;
}

template <int LANES>
__device__ __forceinline__ uint32_t lanes_min(uint32_t v)
{
#pragma unroll
    for (int d = LANES / 2; d >= 1; d /= 2) {
        const uint32_t o = (uint32_t)__shfl_xor((int)v, d);
        v = o < v ? o : v;
    }
    return v;
}

// Order of the scores as whole numbers.  Below every score: NaN (2), an expert of a group that was not kept (1), an expert that was
// already chosen or does not exist (0).
constexpr uint32_t kKeyGone = 0, kKeyDropped = 1, kKeyNan = 2;
__device__ __forceinline__ uint32_t score_key(float b)
{
    const uint32_t u = __float_as_uint(b);
    return b != b ? kKeyNan : (u & 0x80000000u) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ float load_logit(const RouteArgs &p, int64_t at)
{
    return p.bf16 ? (float)((const __bf16 *)p.logits)[at] : ((const float *)p.logits)[at];
}

// 1 / (1 + e) with every operation rounded on its own: equal logits then score the same wherever they are computed
__device__ __forceinline__ float sigmoid_exact(float l)
{
#pragma clang fp contract(off)
    const float e = expf(-l);
    const float d = 1.0f + e;
    return 1.0f / d;
}

// The row's scores: sigmoids, or exponentials with their sum in `total` (NaN where the row has a NaN or +infinity)
template <int LANES, int VPL>
__device__ __forceinline__ void row_scores(const RouteArgs &p, int n, int sub, float (&s)[VPL], float &total)
{
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        const int e = v * LANES + sub;
        s[v] = e < p.E ? load_logit(p, (int64_t)n * p.stride + e) : -INFINITY;
    }
    total = 1.0f;
    if (p.sigmoid) {
#pragma unroll
        for (int v = 0; v < VPL; ++v) s[v] = sigmoid_exact(s[v]);
        return;
    }
    float m = s[0];
#pragma unroll
    for (int v = 1; v < VPL; ++v) m = fmaxf(m, s[v]);
    m = lanes_max<LANES>(m);
    if (m == -INFINITY) m = 0.0f;   // no expert allowed: all scores 0
    total = 0.0f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        s[v] = expf(s[v] - m);
        total += s[v];
    }
    total = lanes_sum<LANES>(total);
}

template <int LANES, int VPL>
__global__ __launch_bounds__(kRouteThreads) void route_kernel(RouteArgs p)
{
    constexpr int kRows = kRouteThreads / LANES;
    __shared__ float scores[kRows][LANES * VPL];          // s
    __shared__ float by[kRows][LANES * VPL];              // b, where there are groups
    __shared__ float group_score[kRows][FUSCO_MAX_GROUPS];
    __shared__ uint8_t group_kept[kRows][FUSCO_MAX_GROUPS];
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int n_real = blockIdx.x * kRows + slot, n = n_real < p.N ? n_real : p.N - 1;   // rows past the end repeat the last one and store nothing

    float s[VPL], total;
    row_scores<LANES, VPL>(p, n, sub, s, total);
    uint32_t key[VPL];
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        const int e = v * LANES + sub;
        scores[slot][e] = s[v];
        float b = s[v];
        if (p.bias && e < p.E) b = (p.sigmoid ? s[v] : s[v] / total) + p.bias[e];
        key[v] = e < p.E ? score_key(b) : kKeyGone;
        if (p.groups > 1) by[slot][e] = b;
    }
    __syncthreads();
    if (p.groups > 1) {
        for (int g = sub; g < p.groups; g += LANES) {
            // the group's largest and second largest b
            float best = -INFINITY, second = -INFINITY;
            for (int i = 0; i < p.group_size; ++i) {
                const float b = by[slot][g * p.group_size + i];
                if (b > best) {
                    second = best;
                    best = b;
                } else if (b > second) {
                    second = b;
                }
            }
            group_score[slot][g] = p.group_best == 2 ? best + second : best;
        }
        __syncthreads();
        for (int g = sub; g < p.groups; g += LANES) {
            const uint32_t mine = score_key(group_score[slot][g]);
            int ahead = 0;
            for (int o = 0; o < p.groups; ++o) {
                const uint32_t other = score_key(group_score[slot][o]);
                ahead += other > mine || (other == mine && o < g);
            }
            group_kept[slot][g] = ahead < p.keep_groups;
        }
        __syncthreads();
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const int e = v * LANES + sub;
            if (e < p.E && !group_kept[slot][e / p.group_size]) key[v] = kKeyDropped;
        }
    }

    // k times the largest key of the row, the lowest expert among equal ones; lane j % LANES keeps the j-th
    float picked_sum = 0.0f;
    int mine = 0;
    for (int j = 0; j < p.k; ++j) {
        uint32_t best = key[0];
        int at = 0;
#pragma unroll
        for (int v = 1; v < VPL; ++v) {
            if (key[v] > best) {
                best = key[v];
                at = v;
            }
        }
        const uint32_t top = lanes_max<LANES>(best);
        const uint32_t e = lanes_min<LANES>(best == top ? (uint32_t)(at * LANES + sub) : 0xffffffffu);
#pragma unroll
        for (int v = 0; v < VPL; ++v)
            if ((uint32_t)(v * LANES + sub) == e) key[v] = kKeyGone;
        picked_sum += scores[slot][e];
        if (sub == j % LANES) mine = (int)e;
        if ((j % LANES == LANES - 1 || j == p.k - 1) && sub <= j % LANES && n_real < p.N) p.chosen[(int64_t)n * p.k + j - j % LANES + sub] = mine;
    }
    // weights; a row whose scores are all zero (no expert allowed) has weights 0
    const float of = p.renorm ? picked_sum : total;
    for (int j = sub; j < p.k; j += LANES) {
        if (n_real >= p.N) break;
        const int e = p.k <= LANES ? mine : p.chosen[(int64_t)n * p.k + j];
        const float v = p.scale * scores[slot][e];
        float w = of == 0.0f ? 0.0f : v / of;
        if (total != total) w = total;
        p.w[(int64_t)n * p.k + j] = w;
    }
}

// dlogits of w = scale * s[chosen] / of (of: sum of the chosen s, or 1):
//   renormalised: ds_j = scale / of * (dw_j - sum_i dw_i s_i / of), otherwise ds_j = scale * dw_j
//   sigmoid: dl = ds s (1 - s);  softmax: dl = s (ds - sum_i ds_i s_i), where the sum vanishes if the weights are renormalised
template <int LANES, int VPL>
__global__ __launch_bounds__(kRouteThreads) void route_grad_kernel(RouteArgs p)
{
    constexpr int kRows = kRouteThreads / LANES;
    __shared__ float scores[kRows][LANES * VPL];
    __shared__ float dscore[kRows][LANES * VPL];
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int n_real = blockIdx.x * kRows + slot, n = n_real < p.N ? n_real : p.N - 1;
    float s[VPL], total;
    row_scores<LANES, VPL>(p, n, sub, s, total);
    const float inv_total = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        s[v] *= inv_total;
        scores[slot][v * LANES + sub] = s[v];
        dscore[slot][v * LANES + sub] = 0.0f;
    }
    __syncthreads();
    float sum_s = 0.0f, sum_ds = 0.0f;   // of the chosen: s, dw * s
    for (int j = sub; j < p.k; j += LANES) {
        const int e = p.chosen[(int64_t)n * p.k + j];
        if ((uint32_t)e >= (uint32_t)p.E) continue;
        sum_s += scores[slot][e];
        sum_ds += p.dw[(int64_t)n * p.k + j] * scores[slot][e];
    }
    sum_s = lanes_sum<LANES>(sum_s);
    sum_ds = lanes_sum<LANES>(sum_ds);
    const float factor = p.renorm ? (sum_s == 0.0f ? 0.0f : p.scale / sum_s) : p.scale;
    const float mean = p.renorm ? (sum_s == 0.0f ? 0.0f : sum_ds / sum_s) : 0.0f;
    for (int j = sub; j < p.k; j += LANES) {
        const int e = p.chosen[(int64_t)n * p.k + j];
        if ((uint32_t)e >= (uint32_t)p.E) continue;
        atomicAdd(&dscore[slot][e], factor * (p.dw[(int64_t)n * p.k + j] - mean));   // chosen experts of a row are distinct: one addition each
    }
    __syncthreads();
    if (n_real >= p.N) return;
    const float common = p.sigmoid || p.renorm ? 0.0f : factor * sum_ds;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        const int e = v * LANES + sub;
        if (e >= p.E) continue;
        const float d = dscore[slot][e];
        const float dl = p.sigmoid ? d * s[v] * (1.0f - s[v]) : s[v] * (d - common);
        if (p.bf16) ((__bf16 *)p.dlogits)[(int64_t)n * p.E + e] = (__bf16)dl;
        else ((float *)p.dlogits)[(int64_t)n * p.E + e] = dl;
    }
}

}   // namespace

#endif
