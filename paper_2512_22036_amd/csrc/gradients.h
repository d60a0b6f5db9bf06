// Gradient of the weighted combine out[t] = sum_j w[t, j] * y[slot(t, j)]:
//   dy[slot(t, j)] = w[t, j] * dout[t],   dw[t, j] = sum over the row of dout[t] * y[slot(t, j)]
// A workgroup holds dout[t] in registers; each of the token's k rows of y is read once and its row of dy written once.
#ifndef FUSCO_CSRC_GRADIENTS_H
#define FUSCO_CSRC_GRADIENTS_H

#include "rows.h"

namespace {

struct CombineGradArgs {
    const int32_t *pair_slot;
    const char *y, *dout;
    const float *w;
    char *dy;
    float *dw;
    int32_t N, k, chunks;
};

// CPT chunks of eight elements per thread, rows of y taken JU at a time
// Bound by memory, rows read and written all over the tensors at once: 8192 x 8 x 14336 B 401 us, 5.0 TB/s; 1537 x 6 x 5760 B 20 us.
template <bool Y_BF16, bool DOUT_BF16, int CPT, int JU, bool PAST>
__global__ __launch_bounds__(1024) void combine_grad_kernel(CombineGradArgs p)
{
    __shared__ float part[FUSCO_MAX_K][kMaxWaves];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int64_t t = blockIdx.x;
    const int32_t *slots = p.pair_slot + t * p.k;
    const float *w = p.w + t * p.k;
    Eight d[CPT];
#pragma unroll
    for (int c = 0; c < CPT; ++c) {
        const int at = c * blockDim.x + threadIdx.x;
        if (at < p.chunks) d[c] = wide(load_raw<DOUT_BF16, PAST>(p.dout, ((size_t)t * p.chunks + at) * kEight));
    }
    for (int j0 = 0; j0 < p.k; j0 += JU) {
        RawEight<Y_BF16> y[JU][CPT];
        int slot[JU];
#pragma unroll
        for (int u = 0; u < JU; ++u) {
            slot[u] = j0 + u < p.k ? slots[j0 + u] : -1;
            if (slot[u] < 0) continue;
#pragma unroll
            for (int c = 0; c < CPT; ++c) {
                const int at = c * blockDim.x + threadIdx.x;
                if (at < p.chunks) y[u][c] = load_raw<Y_BF16, PAST>(p.y, ((size_t)slot[u] * p.chunks + at) * kEight);
            }
        }
#pragma unroll
        for (int u = 0; u < JU; ++u) {
            if (j0 + u >= p.k) break;
            float dot = 0.0f;
            if (slot[u] >= 0) {
                const float weight = w[j0 + u];
#pragma unroll
                for (int c = 0; c < CPT; ++c) {
                    const int at = c * blockDim.x + threadIdx.x;
                    if (at >= p.chunks) continue;
                    const Eight row = wide(y[u][c]);
                    Eight g;
#pragma unroll
                    for (int i = 0; i < kEight; ++i) {
                        dot += row.v[i] * d[c].v[i];
                        g.v[i] = weight * d[c].v[i];
                    }
                    store_eight<Y_BF16>(p.dy, ((size_t)slot[u] * p.chunks + at) * kEight, g);
                }
            }
            dot = wave_sum(dot);
            if (lane == 0) part[j0 + u][wave] = dot;
        }
    }
    __syncthreads();
    for (int j = threadIdx.x; j < p.k; j += blockDim.x) {
        float dot = 0.0f;
        for (int v = 0; v < waves; ++v) dot += part[j][v];
        p.dw[t * p.k + j] = dot;
    }
}

}   // namespace

#endif
