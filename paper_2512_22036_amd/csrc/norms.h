// Norms before and after a block.
//
//   before:  next = x * inv(x) * next_gain,                          inv(x) = 1 / sqrt(mean(x^2) + eps)
//   after:   out = r + scale * gate * (y * inv(y) * gain),           and next of out in the same pass
//
// A workgroup holds one row in registers: every row is read once, both sums of squares are taken over the workgroup, and the row is
// written once.
#ifndef FUSCO_CSRC_NORMS_H
#define FUSCO_CSRC_NORMS_H

#include "rows.h"

namespace {

struct NormArgs {
    const char *r, *y, *gain, *gate, *next_gain;
    char *out, *next;
    int32_t N, chunks;         // chunks of eight elements in a row
    int32_t gate_kind;         // FUSCO_GATE_*
    int32_t gain_bf16;
    float scale, eps, inv_h;
};

// CPT chunks per thread: thread i has the chunks i, i + blockDim, ...
// Bound by memory (norm after a block with the next one: 16384 x 4096 bf16 102 us, 5.3 TB/s; 8192 x 7168 with an fp32 stream 136 us with a gate per
// channel, 130 with one per token, 5.2 and 5.4 TB/s; 4096 x 12288 bf16 74 us, 5.5 TB/s; norm before a block alone, 8192 x 7168 with an fp32 stream 61 us, 5.8 TB/s), by
// latency for a few rows (4 x 7168: 3.6 us).
template <bool STREAM_BF16, bool BLOCK_BF16, int CPT, bool PAST, bool AFTER>
__global__ __launch_bounds__(1024) void norm_kernel(NormArgs p)
{
    __shared__ float part[2][kMaxWaves];
    const int waves = blockDim.x >> 6;
    const size_t row = (size_t)blockIdx.x * p.chunks;
    Eight r[CPT];
    float sums[1];
    if (AFTER) {
        RawEight<STREAM_BF16> rr[CPT];
        RawEight<BLOCK_BF16> ry[CPT];
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = c * blockDim.x + threadIdx.x;
            if (at >= p.chunks) continue;
            ry[c] = load_raw<BLOCK_BF16, PAST>(p.y, (row + at) * kEight);
            rr[c] = load_raw<STREAM_BF16, PAST>(p.r, (row + at) * kEight);
        }
        sums[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            if (c * blockDim.x + threadIdx.x >= p.chunks) continue;
            const Eight y = wide(ry[c]);
#pragma unroll
            for (int i = 0; i < kEight; ++i) sums[0] += y.v[i] * y.v[i];
        }
        group_sums(sums, part[0], waves);
        float factor = p.scale * rsqrtf(sums[0] * p.inv_h + p.eps);
        if (p.gate_kind == FUSCO_GATE_TOKEN) factor *= p.gain_bf16 ? (float)((const __bf16 *)p.gate)[blockIdx.x] : ((const float *)p.gate)[blockIdx.x];
        sums[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = c * blockDim.x + threadIdx.x;
            if (at >= p.chunks) continue;
            const Eight y = wide(ry[c]), gain = load_shared(p.gain, p.gain_bf16, (size_t)at * kEight);
            r[c] = wide(rr[c]);
            Eight gate;
            if (p.gate_kind == FUSCO_GATE_CHANNEL) gate = load_shared(p.gate, p.gain_bf16, (size_t)at * kEight);
#pragma unroll
            for (int i = 0; i < kEight; ++i) {
                float u = y.v[i] * factor * gain.v[i];
                if (p.gate_kind == FUSCO_GATE_CHANNEL) u *= gate.v[i];
                r[c].v[i] += u;
                sums[0] += r[c].v[i] * r[c].v[i];
            }
            store_eight<STREAM_BF16>(p.out, (row + at) * kEight, r[c]);
        }
        if (!p.next) return;
    } else {
        sums[0] = 0.0f;
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = c * blockDim.x + threadIdx.x;
            if (at >= p.chunks) continue;
            r[c] = wide(load_raw<STREAM_BF16, PAST>(p.r, (row + at) * kEight));
        }
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            if (c * blockDim.x + threadIdx.x >= p.chunks) continue;
#pragma unroll
            for (int i = 0; i < kEight; ++i) sums[0] += r[c].v[i] * r[c].v[i];
        }
    }
    group_sums(sums, part[1], waves);
    const float inv = rsqrtf(sums[0] * p.inv_h + p.eps);
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
        const int at = c * blockDim.x + threadIdx.x;
        if (at >= p.chunks) continue;
        const Eight gain = load_shared(p.next_gain, p.gain_bf16, (size_t)at * kEight);
#pragma unroll
        for (int i = 0; i < kEight; ++i) r[c].v[i] *= inv * gain.v[i];
        store_eight<BLOCK_BF16>(p.next, (row + at) * kEight, r[c]);
    }
}

// Gradients.  With u = y * inv(y) * gain and the gradients dout of out and dnext of next:
//   g2 = dnext * next_gain;   dr = dout + inv(out) * (g2 - out * inv(out)^2 * mean(g2 * out));   dnext_gain = sum over rows of dnext * out * inv(out)
//   du = scale * gate * dr;   g1 = du * gain;   dy = inv(y) * (g1 - y * inv(y)^2 * mean(g1 * y));   dgain = sum over rows of du * y * inv(y)
//   dgate = scale * dr * u, summed over the rows (a gate per channel) or over the row (a gate per token)
// A workgroup takes every groups-th row, keeps its part of the sums over rows in registers and writes it to `partial` once;
// norm_join_kernel adds the parts up in a fixed order.
struct NormGradArgs {
    const char *dout, *dnext, *y, *out, *gain, *gate, *next_gain;
    char *dr, *dy;
    float *dgate_token;        // [N], gate per token
    float *partial;            // [groups][sums][H]
    int32_t N, chunks, sums;   // sums: how many of dnext_gain, dgain, dgate (per channel), in this order
    int32_t gate_kind, gain_bf16;
    float scale, eps, inv_h;
};

// Bound by memory up to 8192 columns: 8192 x 7168 with an fp32 stream, both norms, 231 us, 4.6 TB/s over six streams; the norm before a block alone
// 160 us, 5.2 TB/s; the join 5 us.  Beyond, a thread has four chunks: with the row ahead, the row at hand and the sums they need more than the 128 registers of a workgroup
// of 1024, and 340 to 1572 bytes per lane lie in memory, which bounds it: 4096 x 12288 bf16, both norms, 709 us, 0.85 TB/s; with an fp32 stream 1054, 0.86; the norm before
// alone 225 us, 1.8 TB/s.
template <bool STREAM_BF16, bool BLOCK_BF16, int CPT, bool PAST, bool AFTER, bool NEXT, bool GATE_CHANNEL>
__global__ __launch_bounds__(1024) void norm_grad_kernel(NormGradArgs p)
{
    __shared__ float part[2][3 * kMaxWaves];
    const int waves = blockDim.x >> 6;
    Eight dnext_gain[NEXT ? CPT : 1], dgain[AFTER ? CPT : 1], dgate[GATE_CHANNEL ? CPT : 1];
#pragma unroll
    for (int c = 0; c < CPT; ++c)
#pragma unroll
        for (int i = 0; i < kEight; ++i) {
            if (NEXT) dnext_gain[c].v[i] = 0.0f;
            if (AFTER) dgain[c].v[i] = 0.0f;
            if (GATE_CHANNEL) dgate[c].v[i] = 0.0f;
        }
    RawEight<STREAM_BF16> rd[CPT], ro[CPT], rd_next[CPT], ro_next[CPT];
    RawEight<BLOCK_BF16> rn[CPT], ry[CPT], rn_next[CPT], ry_next[CPT];
    auto ask = [&](int n) {   // a row's loads, a row ahead of their use: the waits of the sums then cost no bandwidth
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = c * blockDim.x + threadIdx.x;
            if (at >= p.chunks) continue;
            const size_t el = ((size_t)n * p.chunks + at) * kEight;
            if (NEXT) {
                rn_next[c] = load_raw<BLOCK_BF16, PAST>(p.dnext, el);
                ro_next[c] = load_raw<STREAM_BF16, PAST>(p.out, el);
            }
            if (AFTER) ry_next[c] = load_raw<BLOCK_BF16, PAST>(p.y, el);
            if (p.dout) rd_next[c] = load_raw<STREAM_BF16, PAST>(p.dout, el);
        }
    };
    if ((int)blockIdx.x < p.N) ask(blockIdx.x);
    for (int n = blockIdx.x; n < p.N; n += gridDim.x) {
        const size_t row = (size_t)n * p.chunks;
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            rd[c] = rd_next[c];
            ro[c] = ro_next[c];
            rn[c] = rn_next[c];
            ry[c] = ry_next[c];
        }
        if (n + (int)gridDim.x < p.N) ask(n + gridDim.x);
        float s[3] = {0.0f, 0.0f, 0.0f};   // out^2, g2 * out, y^2
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = c * blockDim.x + threadIdx.x;
            if (at >= p.chunks) continue;
            if (NEXT) {
                const Eight o = wide(ro[c]), d = wide(rn[c]), g = load_shared(p.next_gain, p.gain_bf16, (size_t)at * kEight);
#pragma unroll
                for (int i = 0; i < kEight; ++i) {
                    s[0] += o.v[i] * o.v[i];
                    s[1] += d.v[i] * g.v[i] * o.v[i];
                }
            }
            if (AFTER) {
                const Eight y = wide(ry[c]);
#pragma unroll
                for (int i = 0; i < kEight; ++i) s[2] += y.v[i] * y.v[i];
            }
        }
        group_sums(s, part[0], waves);
        const float inv2 = rsqrtf(s[0] * p.inv_h + p.eps), inv1 = rsqrtf(s[2] * p.inv_h + p.eps);
        const float pull = s[1] * p.inv_h * inv2 * inv2;
        float gate_row = p.scale;
        if (AFTER && p.gate_kind == FUSCO_GATE_TOKEN) gate_row *= p.gain_bf16 ? (float)((const __bf16 *)p.gate)[n] : ((const float *)p.gate)[n];
        Eight dr[CPT];
        float t[2] = {0.0f, 0.0f};         // g1 * y and, for a gate per token, dr * gain * y
#pragma unroll
        for (int c = 0; c < CPT; ++c) {
            const int at = c * blockDim.x + threadIdx.x;
            if (at >= p.chunks) continue;
            if (p.dout) dr[c] = wide(rd[c]);
            else
#pragma unroll
                for (int i = 0; i < kEight; ++i) dr[c].v[i] = 0.0f;
            if (NEXT) {
                const Eight o = wide(ro[c]), d = wide(rn[c]), g = load_shared(p.next_gain, p.gain_bf16, (size_t)at * kEight);
#pragma unroll
                for (int i = 0; i < kEight; ++i) {
                    dnext_gain[c].v[i] += d.v[i] * o.v[i] * inv2;
                    dr[c].v[i] += inv2 * (d.v[i] * g.v[i] - o.v[i] * pull);
                }
            }
            store_eight<STREAM_BF16>(p.dr, (row + at) * kEight, dr[c]);
            if (AFTER) {
                const Eight y = wide(ry[c]), g = load_shared(p.gain, p.gain_bf16, (size_t)at * kEight);
                Eight gate;
                if (GATE_CHANNEL) gate = load_shared(p.gate, p.gain_bf16, (size_t)at * kEight);
#pragma unroll
                for (int i = 0; i < kEight; ++i) {
                    const float unit = y.v[i] * inv1;
                    float du = dr[c].v[i] * gate_row;
                    if (GATE_CHANNEL) {
                        dgate[c].v[i] += du * unit * g.v[i];
                        du *= gate.v[i];
                    }
                    dgain[c].v[i] += du * unit;
                    t[0] += du * g.v[i] * y.v[i];
                    t[1] += dr[c].v[i] * g.v[i] * y.v[i];
                    dr[c].v[i] = du * g.v[i];
                }
            }
        }
        if (AFTER) {
            group_sums(t, part[1], waves);
            const float pull1 = t[0] * p.inv_h * inv1 * inv1;
#pragma unroll
            for (int c = 0; c < CPT; ++c) {
                const int at = c * blockDim.x + threadIdx.x;
                if (at >= p.chunks) continue;
                const Eight y = wide(ry[c]);
#pragma unroll
                for (int i = 0; i < kEight; ++i) dr[c].v[i] = inv1 * (dr[c].v[i] - y.v[i] * pull1);
                store_eight<BLOCK_BF16>(p.dy, (row + at) * kEight, dr[c]);
            }
            if (p.dgate_token && threadIdx.x == 0) p.dgate_token[n] = p.scale * inv1 * t[1];
        }
        if (!AFTER) __syncthreads();   // part[0] is used again
    }
    float *mine = p.partial + (size_t)blockIdx.x * p.sums * p.chunks * kEight;
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
        const int at = c * blockDim.x + threadIdx.x;
        if (at >= p.chunks) continue;
        size_t el = (size_t)at * kEight;
        const size_t step = (size_t)p.chunks * kEight;
        if (NEXT) {
            store_eight<false>((char *)mine, el, dnext_gain[c]);
            el += step;
        }
        if (AFTER) {
            store_eight<false>((char *)mine, el, dgain[c]);
            el += step;
        }
        if (GATE_CHANNEL) store_eight<false>((char *)mine, el, dgate[c]);
    }
}

constexpr int kJoinThreads = 256, kJoinCols = 64;

// total[s][h] = sum over the groups of partial[g][s][h]: 16 threads share a column and take every 16th group each, in ascending order
__global__ __launch_bounds__(kJoinThreads) void norm_join_kernel(const float *partial, int groups, int sums, int H, float *a, float *b, float *c)
{
    constexpr int kShare = kJoinThreads / (kJoinCols / 4);
    __shared__ rows_f32x4 part[kShare][kJoinCols / 4];
    const int quad = threadIdx.x % (kJoinCols / 4), share = threadIdx.x / (kJoinCols / 4), col = blockIdx.x * kJoinCols + quad * 4;
    const int s = blockIdx.y;
    rows_f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < H) {
#pragma unroll 8
        for (int g = share; g < groups; g += kShare) v += *(const rows_f32x4 *)(partial + ((size_t)g * sums + s) * H + col);
    }
    part[share][quad] = v;
    __syncthreads();
    if (share != 0 || col >= H) return;
    for (int w = 1; w < kShare; ++w) v += part[w][quad];
    *(rows_f32x4 *)((s == 0 ? a : s == 1 ? b : c) + col) = v;
}

}   // namespace

#endif
