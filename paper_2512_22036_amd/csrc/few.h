// The whole layer for a few tokens: out[t] = sum over j of w[t, j] * W_out[e] (silu(g) * u), g and u = W_in[e] x[t], e = topk_idx[t, j].
//
// Bound by the weights of the chosen experts, every one of which is read once: few_gated_kernel reads those of the gated product, finds an expert's tokens in the
// routing itself and leaves h in scratch memory; few_linear_kernel reads those of the down product and adds up a token's experts in registers.
// Nothing is moved or planned in between.  h is kept as three numbers of bf16, its rounding and those of what is left, which hold an fp32 number: nothing is rounded to fewer
// bits but a result of bf16.  (Two of them, 17 bits, were 2.5e-6 off in the norm where fp32 throughout is 8e-7.)
//
// Weights of e4m3 become bf16 on their way to the matrix instructions, which is exact; their scales are applied to the fp32 sums of 128 columns.
#ifndef FUSCO_CSRC_FEW_H
#define FUSCO_CSRC_FEW_H

#include "products.h"

namespace {

struct FewArgs {
    const char *x;                     // [N, H] bf16
    const int32_t *chosen;             // [N, k]
    const float *w;                    // [N, k]
    const char *w_in, *w_out;          // [E, 2 I, H], [E, H, I]
    const float *w_in_scale, *w_out_scale;
    char *out;                         // [N, H]
    int32_t *used;                     // scratch: how many experts any token has, and which, ascending
    char *h;                           // scratch: [kParts, N k, I] bf16
    int32_t N, E, k, H, I, out_f32;
};

constexpr int kParts = 3;
constexpr int kUsedInts = FUSCO_MAX_E + 4;
constexpr int kFewTokens = FUSCO_MAX_FEW_TOKENS;

// A wave's part of 16 weight rows and the rows that they are multiplied with, one piece of the sum: CHUNKS times 64 bytes of a row, within one block of scales.
// Lane l holds, of weight row l % 16 and of column l % 16, the elements that the matrix instructions of the piece take from it.
template <bool EIGHT, int CHUNKS>
struct FewPiece {
    static constexpr int kElements = (EIGHT ? 64 : 32) * CHUNKS;
    static constexpr int kSteps = kElements / 32;        // matrix instructions: 32 elements of the sum each
    // first element of a lane's eight of a step
    static __device__ __forceinline__ int element(int lane, int step)
    {
        return EIGHT ? (step / 2) * 64 + (lane >> 4) * 16 + (step % 2) * 8 : step * 32 + (lane >> 4) * 8;
    }
    bf16x8 raw[CHUNKS];                                  // weights as they lie in memory
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, uint32_t row, int lane, int c0, int C)
    {
#pragma unroll
        for (int i = 0; i < CHUNKS; ++i) {
            const int c = c0 + element(lane, EIGHT ? 2 * i : i);
            raw[i] = load_fragment(from, c < C ? row + c * (EIGHT ? 1 : 2) : kNowhere);
        }
    }
    __device__ __forceinline__ bf16x8 operand(int step) const
    {
        if constexpr (EIGHT) {
            typedef __bf16 pair __attribute__((ext_vector_type(2)));
            const words4 q = __builtin_bit_cast(words4, raw[step / 2]);
            const int lo = (int)q[2 * (step % 2)], hi = (int)q[2 * (step % 2) + 1];
            const pair a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
            const pair c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
            return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
        } else {
            return raw[step];
        }
    }
};

// A workgroup per expert and block of 8 * F units, whose gate and up rows make F fragments.  An expert is looked for by the pair that names it where there are fewer
// pairs than experts (the first one stays, the others leave at once), else by its number.  Its pairs, 16 * G at a time, are the columns.
template <bool EIGHT, int F, int WAVES, int G>
__global__ __launch_bounds__(WAVES *kWave) void few_gated_kernel(FewArgs p)
{
    typedef FewPiece<EIGHT, 2> Piece;
    constexpr int kUnits = 8 * F, kOut = F / 2, kCols = 16 * G;
    __shared__ int pairs[kFewTokens * FUSCO_MAX_K];
    __shared__ f32x4 sums[WAVES][F][G][kWave];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int P = p.N * p.k, blocks = (p.I + kUnits - 1) / kUnits;
    const int slot = blockIdx.x / blocks, block = blockIdx.x - slot * blocks, a0 = block * kUnits;
    const int slots = P < p.E ? P : p.E;
    if (slot == slots) {   // the workgroup behind them lists the experts that have tokens
        int *seen = pairs;
        for (int e = tid; e < p.E; e += WAVES * kWave) seen[e] = 0;
        __syncthreads();
        for (int i = tid; i < P; i += WAVES * kWave)
            if ((uint32_t)p.chosen[i] < (uint32_t)p.E) seen[p.chosen[i]] = 1;
        __syncthreads();
        if (wave > 0) return;
        int n = 0;
        for (int e0 = 0; e0 < p.E; e0 += kWave) {
            const bool here = e0 + lane < p.E && seen[e0 + lane];
            const uint64_t all = __ballot(here);
            if (here) p.used[1 + n + __popcll(all & ((1ull << lane) - 1))] = e0 + lane;
            n += __popcll(all);
        }
        if (lane == 0) p.used[0] = n;
        return;
    }
    const int e = __builtin_amdgcn_readfirstlane(P < p.E ? p.chosen[slot] : slot);
    if ((uint32_t)e >= (uint32_t)p.E) return;
    int n = 0;
    for (int base = 0; base < P; base += kWave) {
        const bool mine = base + lane < P && p.chosen[base + lane] == e;
        const uint64_t all = __ballot(mine);
        if (n == 0 && all && P < p.E && base + __ffsll((unsigned long long)all) - 1 != slot) return;
        if (wave == 0 && mine) pairs[n + __popcll(all & ((1ull << lane) - 1))] = base + lane;
        n += __popcll(all);
    }
    if (n == 0) return;
    __syncthreads();

    const int ld = p.H * (EIGHT ? 1 : 2);
    const int pieces = (p.H + Piece::kElements - 1) / Piece::kElements, mine = (pieces - wave + WAVES - 1) / WAVES;
    const __amdgpu_buffer_rsrc_t vx = view(p.x, (int64_t)p.N * p.H * 2);
    const __amdgpu_buffer_rsrc_t vw = view(p.w_in + ((int64_t)e * 2 * p.I + a0) * ld, (int64_t)(2 * p.I - a0) * ld);
    uint32_t w_at[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int unit = f % kOut * 16 + (lane & 15);
        w_at[f] = a0 + unit < p.I ? (uint32_t)((unit + (f >= kOut ? p.I : 0)) * ld) : kNowhere;
    }
    const int scale_rows = (p.I + 127) / 128;
    const float *scales = EIGHT ? p.w_in_scale + ((int64_t)e * 2 * scale_rows + a0 / 128) * pieces : nullptr;
    const int turn = mine > 0 ? (int)(((uint32_t)(block + e * blocks) * 2654435761u >> 12) % (uint32_t)mine) : 0;   // as in few_rows_kernel

    for (int first = 0; first < n; first += kCols) {
        uint32_t x_at[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int col = first + g * 16 + (lane & 15);
            x_at[g] = col < n ? (uint32_t)(pairs[col] / p.k * (p.H * 2)) : kNowhere;
        }
        Piece w[F];
        bf16x8 x[G][Piece::kSteps];
        float scale[2] = {1.0f, 1.0f};
        auto load = [&](int i) {
            int j = i + turn;
            j = j >= mine ? j - mine : j;
            const int piece = wave + j * WAVES, c0 = i < mine ? piece * Piece::kElements : p.H;
#pragma unroll
            for (int f = 0; f < F; ++f) w[f].load(vw, w_at[f], lane, c0, p.H);
#pragma unroll
            for (int s = 0; s < Piece::kSteps; ++s) {
                const int c = c0 + Piece::element(lane, s);
#pragma unroll
                for (int g = 0; g < G; ++g) x[g][s] = load_fragment(vx, c < p.H && x_at[g] != kNowhere ? x_at[g] + c * 2 : kNowhere);
            }
            if (EIGHT && i < mine) {
                scale[0] = scales[piece];
                scale[1] = scales[scale_rows * pieces + piece];
            }
        };
        load(0);
        f32x4 acc[F][G];
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int g = 0; g < G; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int i = 0; i < mine; ++i) {
            Piece wn[F];
            bf16x8 xn[G][Piece::kSteps];
#pragma unroll
            for (int f = 0; f < F; ++f) wn[f] = w[f];
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int s = 0; s < Piece::kSteps; ++s) xn[g][s] = x[g][s];
            const float now[2] = {scale[0], scale[1]};
            if (i + 1 < mine) load(i + 1);
#pragma unroll
            for (int f = 0; f < F; ++f) {
                bf16x8 a[Piece::kSteps];
#pragma unroll
                for (int s = 0; s < Piece::kSteps; ++s) a[s] = wn[f].operand(s);
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    f32x4 part = EIGHT ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[f][g];
#pragma unroll
                    for (int s = 0; s < Piece::kSteps; ++s) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s], xn[g][s], part, 0, 0, 0);
#pragma unroll
                    for (int q = 0; q < 4; ++q) acc[f][g][q] = EIGHT ? fmaf(now[f >= kOut], part[q], acc[f][g][q]) : part[q];
                }
            }
        }
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int g = 0; g < G; ++g) sums[wave][f][g][lane] = acc[f][g];
        __syncthreads();
        for (int fg = wave; fg < kOut * G; fg += WAVES) {
            const int f = fg / G, g = fg % G, col = first + g * 16 + (lane & 15), a = a0 + f * 16 + (lane >> 4) * 4;
            f32x4 gate = sums[0][f][g][lane], up = sums[0][f + kOut][g][lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) {
                gate += sums[v][f][g][lane];
                up += sums[v][f + kOut][g][lane];
            }
            if (col >= n || a >= p.I) continue;
            f32x4 rest;
#pragma unroll
            for (int q = 0; q < 4; ++q) rest[q] = silu(gate[q]) * up[q];
            const int64_t at = (int64_t)pairs[col] * p.I + a;
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                bf16x4 part;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    part[q] = (__bf16)rest[q];
                    rest[q] -= (float)part[q];
                }
                *(bf16x4 *)(p.h + ((int64_t)i * P * p.I + at) * 2) = part;
            }
        }
        __syncthreads();
    }
}

// A workgroup per block of 16 outputs and up to 16 * G tokens, which are the columns (the workgroups of one block's other tokens run on the same XCD at the same time and find
// the weights in its L2).  Its waves share the pieces of all experts that have tokens, each a run of them; a wave that goes on to another expert
// adds what it has of the last one, times the tokens' weights, to the tokens that chose it and to no others.
template <bool EIGHT, int WAVES, int G, int CHUNKS>
__global__ __launch_bounds__(WAVES *kWave) void few_linear_kernel(FewArgs p)
{
    typedef FewPiece<EIGHT, CHUNKS> Piece;
    __shared__ int chosen[16 * G * FUSCO_MAX_K];
    __shared__ f32x4 sums[WAVES][G][kWave];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int P = p.N * p.k, ld = p.I * (EIGHT ? 1 : 2);
    const int groups = (p.N + 16 * G - 1) / (16 * G), block = (int)blockIdx.x / (kXcds * groups) * kXcds + (int)blockIdx.x % kXcds;
    const int a0 = block * 16, t0 = (int)blockIdx.x / kXcds % groups * (16 * G), tokens = min(p.N - t0, 16 * G);
    if (a0 >= p.H) return;
    for (int i = tid; i < tokens * p.k; i += WAVES * kWave) chosen[i] = p.chosen[t0 * p.k + i];
    const int pieces = (p.I + Piece::kElements - 1) / Piece::kElements;
    const int64_t total = (int64_t)__builtin_amdgcn_readfirstlane(p.used[0]) * pieces;
    // blocks begin at different experts: the waves' runs are dealt out from another place in every block
    const int run = (wave + block) % WAVES;
    const int begin = (int)(total * run / WAVES), end = (int)(total * (run + 1) / WAVES);
    __syncthreads();

    __amdgpu_buffer_rsrc_t vh[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i) vh[i] = view(p.h + (int64_t)i * P * p.I * 2, (int64_t)P * p.I * 2);
    const uint32_t w_row = a0 + (lane & 15) < p.H ? (uint32_t)((lane & 15) * ld) : kNowhere;
    Piece w;
    bf16x8 h[G][Piece::kSteps][kParts];
    float scale = 1.0f, weight[G];
    uint32_t h_at[G];
    int e = 0, piece = begin % (pieces > 0 ? pieces : 1), at = begin / (pieces > 0 ? pieces : 1);
    // expert number `at` of those that have tokens: a column's row of h, and the weight that its token gives it
    auto open = [&] {
        e = __builtin_amdgcn_readfirstlane(p.used[1 + at]);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int t = g * 16 + (lane & 15);
            h_at[g] = kNowhere;
            weight[g] = 0.0f;
            for (int j = 0; j < p.k && t < tokens; ++j) {
                if (chosen[t * p.k + j] != e) continue;
                const int pair = (t0 + t) * p.k + j;
                if (h_at[g] == kNowhere) h_at[g] = (uint32_t)(pair * (p.I * 2));
                weight[g] += p.w[pair];
            }
        }
    };
    auto load = [&] {
        const int c0 = piece * Piece::kElements;
        w.load(view(p.w_out + ((int64_t)e * p.H + a0) * ld, (int64_t)(p.H - a0) * ld), w_row, lane, c0, p.I);
#pragma unroll
        for (int s = 0; s < Piece::kSteps; ++s) {
            const int c = c0 + Piece::element(lane, s);
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const uint32_t place = c < p.I && h_at[g] != kNowhere ? h_at[g] + c * 2 : kNowhere;
#pragma unroll
                for (int i = 0; i < kParts; ++i) h[g][s][i] = load_fragment(vh[i], place);
            }
        }
        if (EIGHT) scale = p.w_out_scale[((int64_t)e * ((p.H + 127) / 128) + a0 / 128) * ((p.I + 127) / 128) + c0 / 128];
    };
    f32x4 acc[G], out[G];
#pragma unroll
    for (int g = 0; g < G; ++g) acc[g] = out[g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    if (begin < end) {
        open();
        load();
    }
    for (int i = begin; i < end; ++i) {
        const Piece wn = w;
        bf16x8 hn[G][Piece::kSteps][kParts];
        float weight_now[G];
        bool chose[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            weight_now[g] = weight[g];
            chose[g] = h_at[g] != kNowhere;
#pragma unroll
            for (int s = 0; s < Piece::kSteps; ++s)
#pragma unroll
                for (int i = 0; i < kParts; ++i) hn[g][s][i] = h[g][s][i];
        }
        const float scale_now = scale;
        const bool last = piece == pieces - 1 || i == end - 1;   // of this expert here
        if (++piece == pieces) {
            piece = 0;
            ++at;
            if (i + 1 < end) open();
        }
        if (i + 1 < end) load();
        bf16x8 a[Piece::kSteps];
#pragma unroll
        for (int s = 0; s < Piece::kSteps; ++s) a[s] = wn.operand(s);
#pragma unroll
        for (int g = 0; g < G; ++g) {
            f32x4 part = EIGHT ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[g];
#pragma unroll
            for (int s = 0; s < Piece::kSteps; ++s)
#pragma unroll
                for (int i = 0; i < kParts; ++i) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s], hn[g][s][i], part, 0, 0, 0);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                acc[g][q] = EIGHT ? fmaf(scale_now, part[q], acc[g][q]) : part[q];
                if (last) {
                    out[g][q] = chose[g] ? fmaf(weight_now[g], acc[g][q], out[g][q]) : out[g][q];
                    acc[g][q] = 0.0f;
                }
            }
        }
    }
#pragma unroll
    for (int g = 0; g < G; ++g) sums[wave][g][lane] = out[g];
    __syncthreads();
    for (int g = wave; g < G; g += WAVES) {
        const int t = g * 16 + (lane & 15), a = a0 + (lane >> 4) * 4;
        f32x4 v = sums[0][g][lane];
#pragma unroll
        for (int s = 1; s < WAVES; ++s) v += sums[s][g][lane];
        if (t >= tokens || a >= p.H) continue;
        const int64_t to = (int64_t)(t0 + t) * p.H + a;
        if (p.out_f32) *(f32x4 *)(p.out + to * 4) = v;
        else store4(p.out, to, v);
    }
}

}   // namespace

#endif
