// Routing of tokens to experts: scores, a bias for balance, groups, top-k, weights; and the gradient of the weights.
//
//   s = sigmoid(l) = 1 / (1 + exp(-l)), or exp(l - max l) / sum exp(l - max l)
//   experts compete by b = s + bias (without a bias the softmax's denominator, common to a row, is left out); with groups, a group counts
//   as much as its group_best largest b together, and only experts of the keep_groups best groups compete
//   chosen: the k largest b, descending, ties to the lower index;  w = scale * s / (sum of the chosen s)  or  scale * s
//
// LANES lanes of a wave (16 or all 64) hold one row, VPL values each.  WHOLE: a row has LANES * VPL experts and lies on 16-byte boundaries;
// a lane then has neighbours, expert e is value e % VPL of lane e / VPL, which are loaded 16 bytes at a time and often lie in one
// group.  Otherwise expert e is value e / LANES of lane e % LANES, so that no lane is left without.
#ifndef FUSCO_CSRC_ROUTING_H
#define FUSCO_CSRC_ROUTING_H

#include "rows.h"

namespace {

struct RouteArgs {
    const char *logits;
    const float *bias;
    int32_t *chosen;       // [N, k]
    float *w;              // [N, k]
    const float *dw;       // backward: [N, k]
    char *dlogits;         // backward: [N, E] of the logits' type
    int64_t stride;        // elements from row to row of the logits
    int32_t N, E, k, groups, keep_groups, group_best, group_size, group_magic, group_lanes;   // e / group_size == e * group_magic >> 20 for every e < 1024
    int32_t bf16, sigmoid, renorm;
    float scale;
};

template <int LANES, int VPL, bool WHOLE>
__device__ __forceinline__ int expert_at(int v, int sub) { return WHOLE ? sub * VPL + v : v * LANES + sub; }

// Reductions over the LANES lanes of a row, in all of them
template <int LANES, typename T, typename F>
__device__ __forceinline__ T over_lanes(T v, F f)
{
    static_assert(sizeof(T) == 4 && (LANES == 16 || LANES == 64), "");
    auto with = [&](uint32_t o) { v = f(v, __builtin_bit_cast(T, o)); };
    with(turned<8>(__builtin_bit_cast(uint32_t, v)));
    with(turned<4>(__builtin_bit_cast(uint32_t, v)));
    with(turned<2>(__builtin_bit_cast(uint32_t, v)));
    with(turned<1>(__builtin_bit_cast(uint32_t, v)));
    if (LANES == 64) {
        with((uint32_t)__shfl_xor((int)__builtin_bit_cast(uint32_t, v), 16));
        with((uint32_t)__shfl_xor((int)__builtin_bit_cast(uint32_t, v), 32));
    }
    return v;
}
template <int LANES>
__device__ __forceinline__ float lanes_max(float v) { return over_lanes<LANES>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) { return over_lanes<LANES>(v, [](float a, float b) { return a + b; }); }
template <int LANES>
__device__ __forceinline__ uint32_t lanes_max(uint32_t v) { return over_lanes<LANES>(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
template <int LANES>
__device__ __forceinline__ uint32_t lanes_min(uint32_t v) { return over_lanes<LANES>(v, [](uint32_t a, uint32_t b) { return a < b ? a : b; }); }

// Largest value of the wave, as a scalar
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    const uint32_t m = lanes_max<16>(v);
    const uint32_t a = __builtin_amdgcn_readlane(m, 0), b = __builtin_amdgcn_readlane(m, 16), c = __builtin_amdgcn_readlane(m, 32), d = __builtin_amdgcn_readlane(m, 48);
    const uint32_t ab = a > b ? a : b, cd = c > d ? c : d;
    return ab > cd ? ab : cd;
}

// Orders the LDS accesses of a wave's lanes: a row belongs to one wave
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// Order of the scores as whole numbers.  Below every score: NaN (2), an expert of a group that was not kept (1), an expert that was
// already chosen or does not exist (0).
constexpr uint32_t kKeyGone = 0, kKeyDropped = 1, kKeyNan = 2;
__device__ __forceinline__ uint32_t score_key(float b)
{
    const uint32_t u = __float_as_uint(b);
    return b != b ? kKeyNan : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

__device__ __forceinline__ float load_logit(const RouteArgs &p, int64_t at)
{
    return p.bf16 ? (float)((const __bf16 *)p.logits)[at] : ((const float *)p.logits)[at];
}

// Sigmoids, 1 / (1 + exp(-l)) with every operation rounded correctly on its own: equal logits score the same wherever they are computed.
// The reciprocal of 1 <= d < 2^126 comes from the hardware's (one unit in the last place) by one step of Newton's with fused
// multiply-adds, which rounds it correctly for every such d; a wave with a d beyond divides.
template <int n>
__device__ __forceinline__ void sigmoids(float (&l)[n])
{
#pragma clang fp contract(off)
    float largest = 0.0f;
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float e = expf(-l[i]);
        l[i] = 1.0f + e;
        largest = fmaxf(largest, l[i]);
    }
    if (__any(!(largest < 0x1p126f))) {
        asm volatile("");   // rare: not to be worked out beside the other way
#pragma unroll
        for (int i = 0; i < n; ++i) l[i] = 1.0f / l[i];
        return;
    }
#pragma unroll
    for (int i = 0; i < n; ++i) {
        const float r = __builtin_amdgcn_rcpf(l[i]);
        l[i] = __builtin_fmaf(__builtin_fmaf(-l[i], r, 1.0f), r, r);
    }
}

// What an expert of logit l scores in a row whose largest logit is m
__device__ __forceinline__ float score_of(const RouteArgs &p, float l, float m)
{
    if (!p.sigmoid) return expf(l - m);
    float s[1] = {l};
    sigmoids(s);
    return s[0];
}

// The row's scores: sigmoids, or exponentials with their sum in `total` (NaN where the row has a NaN or +infinity)
template <int LANES, int VPL, bool WHOLE>
__device__ __forceinline__ void row_scores(const RouteArgs &p, int n, int sub, float (&s)[VPL], float &total, float &m)
{
    // loads past the row's end are loads of its last logit
    const int64_t row = (int64_t)n * p.stride;
    if constexpr (WHOLE) {
        typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
        const int64_t at = row + sub * VPL;
        if (p.bf16) {
#pragma unroll
            for (int v = 0; v < VPL; v += 4) {
                const bf16x4 l = *(const bf16x4 *)(p.logits + (at + v) * 2);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[v + i] = (float)l[i];
            }
        } else {
#pragma unroll
            for (int v = 0; v < VPL; v += 4) {
                const rows_f32x4 l = *(const rows_f32x4 *)(p.logits + (at + v) * 4);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[v + i] = l[i];
            }
        }
    } else if (p.bf16) {
#pragma unroll
        for (int v = 0; v < VPL; ++v) s[v] = (float)((const __bf16 *)p.logits)[row + min(v * LANES + sub, p.E - 1)];
    } else {
#pragma unroll
        for (int v = 0; v < VPL; ++v) s[v] = ((const float *)p.logits)[row + min(v * LANES + sub, p.E - 1)];
    }
    total = 1.0f;
    m = 0.0f;
    if (p.sigmoid) {   // an expert that does not exist scores what the last one does, and its key says that it does not exist
        sigmoids(s);
        return;
    }
    if (!WHOLE && p.E < LANES * VPL) {
#pragma unroll
        for (int v = 0; v < VPL; ++v) s[v] = v * LANES + sub < p.E ? s[v] : -INFINITY;
    }
    m = s[0];
#pragma unroll
    for (int v = 1; v < VPL; ++v) m = fmaxf(m, s[v]);
    m = lanes_max<LANES>(m);
    if (m == -INFINITY) m = 0.0f;   // no expert allowed: all scores 0
    total = 0.0f;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        s[v] = score_of(p, s[v], m);
        total += s[v];
    }
    total = lanes_sum<LANES>(total);
}

// The two largest of both lanes' two largest
__device__ __forceinline__ void join_best(float &best, float &second, float b, float s)
{
    second = fmaxf(fmaxf(second, s), fminf(best, b));
    best = fmaxf(best, b);
}
template <int control>
__device__ __forceinline__ float moved(float v)
{
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), control, 0xf, 0xf, true));
}

// Scores of groups that are `lanes` whole lanes each, a power of two: the lane's own two largest b, then those of its group's lanes
template <int LANES, int VPL>
__device__ __forceinline__ void score_own_group(const RouteArgs &p, int sub, const float (&b)[VPL], int lanes, float *group_score)
{
    float best = -INFINITY, second = -INFINITY;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        const float some = fmaxf(b[v], -INFINITY);   // a NaN is passed over
        second = __builtin_amdgcn_fmed3f(best, second, some);
        best = fmaxf(best, some);
    }
    if (lanes >= 2) join_best(best, second, moved<0xb1>(best), moved<0xb1>(second));      // lane ^ 1
    if (lanes >= 4) join_best(best, second, moved<0x4e>(best), moved<0x4e>(second));      // lane ^ 2
    if (lanes >= 8) join_best(best, second, moved<0x141>(best), moved<0x141>(second));    // the other four of eight, mirrored
    if (lanes >= 16) join_best(best, second, moved<0x140>(best), moved<0x140>(second));   // the other eight of sixteen
    if (LANES == 64) {
        for (int d = 16; d < lanes; d *= 2) join_best(best, second, __shfl_xor(best, d), __shfl_xor(second, d));
    }
    if (sub % lanes == 0) group_score[sub / lanes] = p.group_best == 2 ? best + second : best;
}

// The same from the row's b in LDS, for groups of any size
template <int LANES>
__device__ __forceinline__ void score_groups(const RouteArgs &p, int sub, const float *by, float *group_score)
{
    wave_sync();
    // as many lanes per group as there are, a power of two; each takes every `share`-th expert, begun at another place per group so that
    // groups of 32 do not meet in one bank
    int share = 1;
    while (share * 2 * p.groups <= LANES) share *= 2;
    const int each = (p.group_size + share - 1) / share;
    for (int base = 0; base < p.groups; base += LANES / share) {
        const int g = base + sub / share, h = sub % share;
        float best = -INFINITY, second = -INFINITY;
        if (g < p.groups) {
            int i = g % each;
#pragma unroll 8
            for (int n = 0; n < each; ++n) {
                const int at = i * share + h;
                const float b = fmaxf(at < p.group_size ? by[g * p.group_size + at] : -INFINITY, -INFINITY);   // a NaN is passed over
                second = __builtin_amdgcn_fmed3f(best, second, b);
                best = fmaxf(best, b);
                i = i + 1 == each ? 0 : i + 1;
            }
        }
        for (int d = 1; d < share; d *= 2) join_best(best, second, __shfl_xor(best, d), __shfl_xor(second, d));
        if (g < p.groups && h == 0) group_score[g] = p.group_best == 2 ? best + second : best;
    }
}

// Which groups are kept, and what of that holds for this lane's experts.  own: all of them are of group `own`, or -1.
template <int LANES, int VPL, bool WHOLE>
__device__ __forceinline__ void drop_groups(const RouteArgs &p, int sub, const float *group_score, int own, uint32_t (&key)[VPL])
{
    wave_sync();
    uint64_t kept = 0;   // bit g: group g of this lane's row is kept
    for (int base = 0; base < p.groups; base += LANES) {
        const int g = base + sub;
        const uint32_t mine = score_key(g < p.groups ? group_score[g] : 0.0f);
        int ahead = 0;
#pragma unroll 8
        for (int o = 0; o < p.groups; ++o) {
            const uint32_t other = score_key(group_score[o]);
            ahead += other > mine || (other == mine && o < g);
        }
        const uint64_t said = __ballot(g < p.groups && ahead < p.keep_groups);
        kept |= LANES == 64 ? said : (said >> (threadIdx.x & 48) & 0xffff) << base;
    }
    if (WHOLE && own >= 0) {
        const uint32_t most = kept >> own & 1 ? 0xffffffffu : kKeyDropped;
#pragma unroll
        for (int v = 0; v < VPL; ++v) key[v] = min(key[v], most);
    } else if (p.groups <= 32) {
        const uint32_t some = (uint32_t)kept;
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const uint32_t g = (uint32_t)expert_at<LANES, VPL, WHOLE>(v, sub) * p.group_magic >> 20;
            key[v] = some >> g & 1 ? key[v] : min(key[v], kKeyDropped);
        }
    } else {
#pragma unroll
        for (int v = 0; v < VPL; ++v) {
            const uint32_t g = (uint32_t)expert_at<LANES, VPL, WHOLE>(v, sub) * p.group_magic >> 20;
            key[v] = kept >> g & 1 ? key[v] : min(key[v], kKeyDropped);
        }
    }
}

// The j-th chosen expert of the row in lane j (of 64 lanes' j % LANES), one after the other: k times the largest key, the lowest expert among
// equal ones
template <int LANES, int VPL, bool WHOLE>
__device__ __forceinline__ int choose_in_turn(const RouteArgs &p, int sub, uint32_t (&key)[VPL])
{
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
        uint32_t e;
        if constexpr (LANES == 64) {
            const uint32_t top = wave_max(best);
            const uint64_t with = __ballot(best == top);
            if (__popcll(with) == 1) {
                const int lane = __ffsll((long long)with) - 1;
                e = (uint32_t)expert_at<LANES, VPL, WHOLE>(__builtin_amdgcn_readlane(at, lane), lane);
            } else {
                e = lanes_min<LANES>(best == top ? (uint32_t)expert_at<LANES, VPL, WHOLE>(at, sub) : 0xffffffffu);
            }
        } else {
            const uint32_t top = lanes_max<LANES>(best);
            e = lanes_min<LANES>(best == top ? (uint32_t)expert_at<LANES, VPL, WHOLE>(at, sub) : 0xffffffffu);
        }
#pragma unroll
        for (int v = 0; v < VPL; ++v)
            if ((uint32_t)expert_at<LANES, VPL, WHOLE>(v, sub) == e) key[v] = kKeyGone;
        if (sub == j) mine = (int)e;
    }
    return mine;
}

constexpr int kListed = 32;   // candidates that choose_at_once ranks

template <int by>
struct RankTurn {
    // how many of the entries (key, expert) that lie 1 .. by lanes on come before this lane's
    static __device__ __forceinline__ void count(uint64_t entry, uint64_t others, int &ahead)
    {
        const uint64_t o = (uint64_t)turned<by>((uint32_t)(others >> 32)) << 32 | turned<by>((uint32_t)others);
        ahead += o > entry;
        if constexpr (by > 1) RankTurn<by - 1>::count(entry, others, ahead);
    }
};
template <int by>
__device__ __forceinline__ void count_larger(uint32_t m, int &larger)
{
    larger += turned<by>(m) > m;
    if constexpr (by > 1) count_larger<by - 1>(m, larger);
}

// The same for 16 lanes without k dependent rounds.  The k-th largest of the lanes' largest keys bounds the k-th largest of all from below;
// what reaches it (about 11 keys of 256 for k = 8) is listed in LDS and ranked, every entry against every other.  False in the whole wave
// if some row has more than kListed candidates (many equal scores): nothing is chosen then.
template <int VPL>
__device__ __forceinline__ bool choose_at_once(const RouteArgs &p, int sub, const uint32_t (&key)[VPL], uint64_t *list, int *order, int &mine)
{
    uint32_t m = key[0];
#pragma unroll
    for (int v = 1; v < VPL; ++v) m = key[v] > m ? key[v] : m;
    int larger = 0;
    count_larger<15>(m, larger);
    uint32_t bound = lanes_min<16>(larger < p.k ? m : 0xffffffffu);
    bound = bound < kKeyDropped ? kKeyDropped : bound;
    int count = 0;
#pragma unroll
    for (int v = 0; v < VPL; ++v) count += key[v] >= bound;
    int before = count;   // inclusive sums over the lanes
#pragma unroll
    for (int d = 1; d < 16; d *= 2) {
        const int o = __shfl_up(before, d, 16);
        if (sub >= d) before += o;
    }
    const int total = __shfl(before, 15, 16);
    if (__any(total > kListed)) return false;
    before -= count;
    list[sub] = 0;
    list[sub + 16] = 0;
    wave_sync();
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        if (key[v] >= bound) list[before++] = (uint64_t)key[v] << 32 | (uint32_t)~(v * 16 + sub);
    }
    wave_sync();
    const uint64_t first = list[sub];
    int rank = 0;
    RankTurn<15>::count(first, first, rank);
    if (__any(total > 16)) {
        asm volatile("");   // one wave in several
        const uint64_t second = list[sub + 16];
        int rank2 = 0;
        RankTurn<15>::count(second, second, rank2);
        RankTurn<15>::count(second, first, rank2);
        rank2 += first > second;
        RankTurn<15>::count(first, second, rank);
        rank += second > first;
        if (second != 0 && rank2 < p.k) order[rank2] = (int)~(uint32_t)second;
    }
    if (first != 0 && rank < p.k) order[rank] = (int)~(uint32_t)first;
    wave_sync();
    mine = order[sub];
    return true;
}

// Bound by vector instructions where there are many rows (32768 x 256 with 8 groups, sigmoids, 8 chosen: 16.5 us, 2.2 TB/s read and written, vector units
// busy for three quarters of it; without groups 13.7), by a wave's chain of dependent steps where there are few (128 x 256: 4.4 us, an empty launch 2).
template <int LANES, int VPL, int THREADS, bool WHOLE>
__global__ __launch_bounds__(THREADS) void route_kernel(RouteArgs p)
{
    constexpr int kRows = THREADS / LANES, kPitch = LANES * VPL + (LANES == 64 ? 0 : WHOLE ? 80 : 16);   // rows of a wave begin in different banks
    __shared__ __align__(16) float by[kRows][kPitch];              // b, where there are groups
    __shared__ float group_score[kRows][FUSCO_MAX_GROUPS];
    __shared__ uint64_t list[LANES == 16 ? kRows : 1][kListed];
    __shared__ int order[LANES == 16 ? kRows : 1][16];
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int n_real = blockIdx.x * kRows + slot, n = n_real < p.N ? n_real : p.N - 1;   // rows past the end repeat the last one and store nothing

    float s[VPL], total, m;
    row_scores<LANES, VPL, WHOLE>(p, n, sub, s, total, m);
    if (p.bias) {
        float by_total = 1.0f;
        if (!p.sigmoid) by_total = total == 0.0f ? 0.0f : 1.0f / total;   // no expert allowed: scores stay 0, the bias decides
#pragma unroll
        for (int v = 0; v < VPL; ++v) s[v] = s[v] * by_total + p.bias[WHOLE ? sub * VPL + v : min(v * LANES + sub, p.E - 1)];
    }
    uint32_t key[VPL];
#pragma unroll
    for (int v = 0; v < VPL; ++v) key[v] = score_key(s[v]);
    if (!WHOLE && p.E < LANES * VPL) {
#pragma unroll
        for (int v = 0; v < VPL; ++v) key[v] = v * LANES + sub < p.E ? key[v] : kKeyGone;
    }
    if (p.groups > 1) {
        const bool own = WHOLE && (LANES == 16 || p.group_lanes > 0);   // a group is some whole lanes of the row
        if (own) {
            score_own_group<LANES, VPL>(p, sub, s, p.group_lanes, group_score[slot]);
        } else {
#pragma unroll
            for (int v = 0; v < VPL; ++v) by[slot][expert_at<LANES, VPL, WHOLE>(v, sub)] = s[v];
            score_groups<LANES>(p, sub, by[slot], group_score[slot]);
        }
        drop_groups<LANES, VPL, WHOLE>(p, sub, group_score[slot], own ? sub / p.group_lanes : -1, key);
    }
    // choose_at_once wants the candidates spread over the lanes, which those of kept groups are not
    constexpr bool kSpread = WHOLE && LANES == 16;
    if constexpr (kSpread) {
        uint32_t *keys = (uint32_t *)by[slot];
#pragma unroll
        for (int v = 0; v < VPL; v += 4) {
            typedef uint32_t words __attribute__((ext_vector_type(4)));
            *(words *)(keys + sub * (VPL + 4) + v) = words{key[v], key[v + 1], key[v + 2], key[v + 3]};
        }
        wave_sync();
#pragma unroll
        for (int v = 0; v < VPL; ++v) key[v] = keys[v * LANES + sub + (v * LANES + sub) / VPL * 4];
    }

    int mine = 0;                                        // lane j has the j-th chosen expert
    if constexpr (LANES == 16) {
        if (!choose_at_once<VPL>(p, sub, key, list[slot], order[slot], mine)) mine = choose_in_turn<LANES, VPL, false>(p, sub, key);
    } else {
        mine = choose_in_turn<LANES, VPL, WHOLE>(p, sub, key);
    }

    // weights; a row whose scores are all zero (no expert allowed) has weights 0
    const float score = sub < p.k ? score_of(p, load_logit(p, (int64_t)n * p.stride + mine), m) : 0.0f;   // once more, for the chosen alone
    const float of = p.renorm ? lanes_sum<LANES>(score) : total;
    float w = of == 0.0f ? 0.0f : p.scale * score / of;
    if (total != total) w = total;
    if (n_real < p.N && sub < p.k) {
        p.chosen[(int64_t)n * p.k + sub] = mine;
        p.w[(int64_t)n * p.k + sub] = w;
    }
}

// dlogits of w = scale * q, with q = s[chosen], or s[chosen] / (sum of the chosen s) if renormalised; d_j is what dw_j gives to the logarithm of s_j:
//   renormalised: d_j = scale * q_j * (dw_j - sum_i dw_i q_i), otherwise d_j = scale * q_j * dw_j
//   sigmoid: dl = d (1 - s), 1 - s = 1 / (1 + exp(l));  softmax: dl = d - s * sum_i d_i, where the sum vanishes if the weights are renormalised
// No factor grows as the scores shrink: with ds = scale * (dw - ...) / (sum of the chosen s) and dl = ds * s (...) it would overflow.
// Bound by latency and vector instructions, busy for two fifths of it: 16384 x 128 bf16, softmax, 8 chosen: 4.8 us; 32768 x 256 fp32, sigmoids: 13.4 us, 5.0 TB/s.
template <int LANES, int VPL, int THREADS>
__global__ __launch_bounds__(THREADS) void route_grad_kernel(RouteArgs p)
{
    constexpr int kRows = THREADS / LANES;
    static_assert(LANES == FUSCO_MAX_K || LANES == 16, "a lane per chosen expert: 16 lanes are taken for at most 10");
    __shared__ float grad[kRows][LANES * VPL];
    const int sub = threadIdx.x % LANES, slot = threadIdx.x / LANES;
    const int n_real = blockIdx.x * kRows + slot, n = n_real < p.N ? n_real : p.N - 1;
    // lane j has the j-th chosen expert, or none
    const int64_t at = (int64_t)n * p.k + sub;
    const int e = sub < p.k ? p.chosen[at] : -1;
    const bool some = (uint32_t)e < (uint32_t)p.E;
    const float dw = some ? p.dw[at] : 0.0f, l = some ? load_logit(p, (int64_t)n * p.stride + e) : 0.0f;
    float s[VPL], total, m;
    row_scores<LANES, VPL, false>(p, n, sub, s, total, m);
    const float inv_total = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        s[v] *= inv_total;
        grad[slot][v * LANES + sub] = 0.0f;
    }
    const float score = score_of(p, l, m);   // as in the row
    float q = some ? score : 0.0f;
    if (p.renorm) {
        const float sum = lanes_sum<LANES>(q);
        q = sum == 0.0f ? 0.0f : q / sum;
    } else {
        q *= inv_total;
    }
    const float mean = lanes_sum<LANES>(dw * q);
    float d = p.scale * q * (p.renorm ? dw - mean : dw);
    if (p.sigmoid) d *= score_of(p, -l, m);   // 1 - s without its cancellation: 1 - s has no bit left from l = 17 on
    wave_sync();
    if (some) atomicAdd(&grad[slot][e], d);   // chosen experts of a row are distinct: one addition each
    wave_sync();
    if (n_real >= p.N) return;
    const float common = p.sigmoid || p.renorm ? 0.0f : p.scale * mean;
#pragma unroll
    for (int v = 0; v < VPL; ++v) {
        const int x = v * LANES + sub;
        if (x >= p.E) continue;
        const float dl = grad[slot][x] - s[v] * common;   // a NaN among the scores stays one
        if (p.bf16) ((__bf16 *)p.dlogits)[(int64_t)n * p.E + x] = (__bf16)dl;
        else ((float *)p.dlogits)[(int64_t)n * p.E + x] = dl;
    }
}

}   // namespace

#endif
