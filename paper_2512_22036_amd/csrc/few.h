// The whole layer for a few tokens: out[t] = sum over j of w[t, j] * W_out[e] (silu(g) * u), g and u = W_in[e] x[t], e = topk_idx[t, j].
//
// Bound by the weights of the chosen experts where those have few tokens: few_gated_kernel reads those of the gated product, finds an expert's tokens in the
// routing itself and leaves h in scratch memory; few_linear_kernel reads those of the down product and adds up a token's experts in registers.  Both pass over an expert's weights once for as
// many of its pairs as a matrix instruction has columns for, 16 or 32 and 5 or 15, from the caches if they still hold them, and few_linear_kernel reads all of h for every 16 outputs: with
// more pairs than that it is these passes that bound (e4m3, 4096 x 1280, 64 tokens: 8 experts, two per token, 71 us, eight per token 210, where the weights take 20; 128 experts 516, weights 312).
// Nothing is moved in between; the pairs are sorted by expert beside the first product.  h is kept as three numbers of bf16, its rounding and those of what is left, which hold an fp32 number: nothing is rounded to fewer
// bits but a result of bf16.  (Two of them, 17 bits, were 2.5e-6 off in the norm where fp32 throughout is 8e-7.)
//
// Weights of e4m3 become bf16 on their way to the matrix instructions, which is exact; their scales are applied to the fp32 sums of 128 columns.
#ifndef FUSCO_CSRC_FEW_H
#define FUSCO_CSRC_FEW_H

#include "products.h"
#include <float.h>

namespace {

struct FewArgs {
    const char *x;                     // [N, H] bf16
    const int32_t *chosen;             // [N, k]
    const float *w;                    // [N, k]
    const char *w_in, *w_out;          // [E, 2 I, H], [E, H, I]
    const float *w_in_scale, *w_out_scale;
    char *out;                         // [N, H]
    int32_t *groups;                   // scratch: how many groups there are; [N k] groups: expert | pairs << 10 | place of the first pair << 14
    int32_t *listed;                   // scratch: [N k] pairs, group by group
    float *listed_w;                   // scratch: [N k] their weights
    float *partial;                    // scratch: [blocks of outputs, parts, N, 16] sums of the parts of the groups, where there is more than one
    uint32_t *arrived;                 // scratch: [blocks of outputs] parts that are done
    char *h;                           // scratch: [kParts, N k, I] bf16
    int32_t N, E, k, H, I, out_f32;
    int32_t parts;                     // of the list of groups, a workgroup of few_linear_kernel each
    int32_t group;                     // pairs of a group: kFive, or kManyFives times that
};

constexpr int kParts = 3;
constexpr float kMaxBf16 = 0x1.fep127f;
constexpr int kFive = 5;       // pairs: kParts columns each of the sixteen of a matrix instruction
constexpr int kManyFives = 3;
static_assert(FUSCO_MAX_E <= 1 << 10 && kFive * kManyFives < 1 << 4 && FUSCO_MAX_FEW_TOKENS * FUSCO_MAX_K <= 1 << 17, "a group in 31 bits");
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

// The pairs by expert, in groups of up to p.group of one expert, in ascending order throughout, for few_linear_kernel.  Pairs that name no expert are left out; a token that names
// one several times is in its list once, with the weights together.  `key` and `lists` are LDS.
template <int WAVES>
__device__ __forceinline__ void few_groups(const FewArgs &p, int16_t *__restrict__ key, int (*__restrict__ lists)[FUSCO_MAX_E])
{
    constexpr int kThreads = WAVES * kWave;
    int *count = lists[0], *groups_before = lists[1], *pairs_before = lists[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, P = p.N * p.k;
    for (int i = tid; p.parts > 1 && i * 16 < p.H; i += kThreads) p.arrived[i] = 0;
    for (int i = tid; i < P; i += kThreads) {
        const int e = p.chosen[i], first = i / p.k * p.k;
        bool again = (uint32_t)e >= (uint32_t)p.E;
        for (int j = first; j < i; ++j) again |= p.chosen[j] == e;
        key[i] = (int16_t)(again ? -1 : e);
    }
    __syncthreads();
    for (int e = wave; e < p.E; e += WAVES) {
        int n = 0;
        for (int base = 0; base < P; base += kWave) n += __popcll(__ballot(base + lane < P && key[base + lane] == e));
        if (lane == 0) count[e] = n;
    }
    __syncthreads();
    if (wave == 0) {
        int groups = 0, pairs = 0;
        for (int e0 = 0; e0 < p.E; e0 += kWave) {
            const int n = e0 + lane < p.E ? count[e0 + lane] : 0, g = (n + p.group - 1) / p.group;
            int g_sum = g, n_sum = n;
#pragma unroll
            for (int d = 1; d < kWave; d *= 2) {
                const int og = __shfl_up(g_sum, d), on = __shfl_up(n_sum, d);
                if (lane >= d) {
                    g_sum += og;
                    n_sum += on;
                }
            }
            if (e0 + lane < p.E) {
                groups_before[e0 + lane] = groups + g_sum - g;
                pairs_before[e0 + lane] = pairs + n_sum - n;
            }
            groups += __shfl(g_sum, 63);
            pairs += __shfl(n_sum, 63);
        }
        if (lane == 0) p.groups[0] = groups;
    }
    __syncthreads();
    for (int e = wave; e < p.E; e += WAVES) {
        const int n = count[e], first = pairs_before[e];
        for (int g = lane; g * p.group < n; g += kWave) p.groups[1 + groups_before[e] + g] = e | min(n - g * p.group, p.group) << 10 | (first + g * p.group) << 14;
        int done = 0;
        for (int base = 0; base < P && done < n; base += kWave) {
            const bool mine = base + lane < P && key[base + lane] == e;
            const uint64_t all = __ballot(mine);
            if (mine) {
                const int i = base + lane, to = first + done + __popcll(all & ((1ull << lane) - 1));
                float w = 0.0f;
                for (int j = i; j < (i / p.k + 1) * p.k; ++j)
                    if (p.chosen[j] == e) w += p.w[j];
                p.listed[to] = i;
                p.listed_w[to] = w;
            }
            done += __popcll(all);
        }
    }
}

// A workgroup per expert and block of 8 * F units, whose gate and up rows make F fragments (with one, its first and its last eight rows).  An expert is looked for by the
// pair that names it where there are fewer pairs than experts (the first one stays, the others leave at once), else by its number.  Its pairs,
// 16 * G at a time, are the columns.  The waves share the sum piece by piece; weights are DEPTH pieces ahead of their use, rows of x, from the L2, one.
template <bool EIGHT, int F, int WAVES, int G, int DEPTH, int SIMD>
__global__ __launch_bounds__(WAVES *kWave, SIMD) void few_gated_kernel(FewArgs p)
{
    typedef FewPiece<EIGHT, 2> Piece;
    constexpr int kUnits = 8 * F, kCols = 16 * G, kFragments = F == 1 ? 1 : F / 2;   // of gate rows
    static_assert(F == 1 || F % 2 == 0, "gate and up rows");
    typedef f32x4 Sums[WAVES][F][G][kWave];
    __shared__ int16_t pairs[kFewTokens * FUSCO_MAX_K];
    __shared__ __align__(16) char lds[sizeof(Sums) > 3 * FUSCO_MAX_E * 4 ? sizeof(Sums) : 3 * FUSCO_MAX_E * 4];
    Sums &sums = *(Sums *)lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int P = p.N * p.k, blocks = (p.I + kUnits - 1) / kUnits;
    if (blockIdx.x == 0) {   // makes the groups, while the others multiply
        few_groups<WAVES>(p, pairs, (int (*)[FUSCO_MAX_E])lds);
        return;
    }
    const int slot = ((int)blockIdx.x - 1) / blocks, block = (int)blockIdx.x - 1 - slot * blocks, a0 = block * kUnits;
    const int ahead = lane < P ? p.chosen[lane] : -1;   // asked for together with the expert
    const int e = __builtin_amdgcn_readfirstlane(P < p.E ? p.chosen[slot] : slot);
    if ((uint32_t)e >= (uint32_t)p.E) return;
    int n = 0;
    for (int base = 0; base < P; base += kWave) {
        const bool mine = base + lane < P && (base == 0 ? ahead : p.chosen[base + lane]) == e;
        const uint64_t all = __ballot(mine);
        if (n == 0 && all && P < p.E && base + __ffsll((unsigned long long)all) - 1 != slot) return;
        if (wave == 0 && mine) pairs[n + __popcll(all & ((1ull << lane) - 1))] = (int16_t)(base + lane);
        n += __popcll(all);
    }
    if (n == 0) return;

    const int ld = p.H * (EIGHT ? 1 : 2);
    const int pieces = (p.H + Piece::kElements - 1) / Piece::kElements, mine = (pieces - wave + WAVES - 1) / WAVES;
    const __amdgpu_buffer_rsrc_t vx = view(p.x, (int64_t)p.N * p.H * 2);
    const __amdgpu_buffer_rsrc_t vw = view(p.w_in + ((int64_t)e * 2 * p.I + a0) * ld, (int64_t)(2 * p.I - a0) * ld);
    uint32_t w_at[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int unit = F == 1 ? lane & 7 : f % kFragments * 16 + (lane & 15);
        const bool up = F == 1 ? (lane & 8) != 0 : f >= F / 2;
        w_at[f] = a0 + unit < p.I ? (uint32_t)((unit + (up ? p.I : 0)) * ld) : kNowhere;
    }
    const int scale_rows = (p.I + 127) / 128;
    const float *scales = EIGHT ? p.w_in_scale + ((int64_t)e * 2 * scale_rows + a0 / 128) * pieces : nullptr;
    const int turn = mine > 0 ? (int)(((uint32_t)(block + e * blocks) * 2654435761u >> 12) % (uint32_t)mine) : 0;   // as in few_rows_kernel
    auto piece_of = [&](int i) {
        const int j = i + turn;
        return wave + (j >= mine ? j - mine : j) * WAVES;
    };

    for (int first = 0; first < n; first += kCols) {
        Piece w[DEPTH][F];
        float scale[DEPTH][2];
        auto load = [&](int i, int d) {
            const int piece = i < mine ? piece_of(i) : pieces;
#pragma unroll
            for (int f = 0; f < F; ++f) w[d][f].load(vw, w_at[f], lane, piece * Piece::kElements, p.H);
            if (EIGHT) {
                const int at = i < mine ? piece : 0;
                scale[d][0] = scales[at];
                scale[d][1] = scales[scale_rows * pieces + at];
            }
        };
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) load(d, d);
        __syncthreads();   // pairs
        uint32_t x_at[G];
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const int col = first + g * 16 + (lane & 15);
            x_at[g] = col < n ? (uint32_t)(pairs[col] / p.k * (p.H * 2)) : kNowhere;
        }
        bf16x8 x[G][Piece::kSteps];
        auto load_x = [&](int i) {
            const int c0 = i < mine ? piece_of(i) * Piece::kElements : p.H;
#pragma unroll
            for (int s = 0; s < Piece::kSteps; ++s) {
                const int c = c0 + Piece::element(lane, s);
#pragma unroll
                for (int g = 0; g < G; ++g) x[g][s] = load_fragment(vx, c < p.H && x_at[g] != kNowhere ? x_at[g] + c * 2 : kNowhere);
            }
        };
        load_x(0);
        f32x4 acc[F][G];
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int g = 0; g < G; ++g) acc[f][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        for (int i0 = 0; i0 < mine; i0 += DEPTH) {
#pragma unroll
            for (int d = 0; d < DEPTH; ++d) {   // pieces past the last one are zeros, and so is their scale: another one's may be infinite
                bf16x8 xn[G][Piece::kSteps];
#pragma unroll
                for (int g = 0; g < G; ++g)
#pragma unroll
                    for (int s = 0; s < Piece::kSteps; ++s) xn[g][s] = x[g][s];
                Piece wn[F];
#pragma unroll
                for (int f = 0; f < F; ++f) wn[f] = w[d][f];
                // of both scales, that of this lane's four rows of the results
                const bool in = i0 + d < mine;
                const float now[2] = {!EIGHT || !in ? 0.0f : F == 1 && lane >= 32 ? scale[d][1] : scale[d][0], EIGHT && in ? scale[d][1] : 0.0f};
                load_x(i0 + d + 1);
                load(i0 + d + DEPTH, d);
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
                        for (int q = 0; q < 4; ++q) acc[f][g][q] = EIGHT ? fmaf(now[F > 1 && f >= F / 2], part[q], acc[f][g][q]) : part[q];
                    }
                }
            }
        }
#pragma unroll
        for (int f = 0; f < F; ++f)
#pragma unroll
            for (int g = 0; g < G; ++g) sums[wave][f][g][lane] = acc[f][g];
        __syncthreads();
        for (int fg = wave; fg < kFragments * G; fg += WAVES) {
            const int f = fg / G, g = fg % G, col = first + g * 16 + (lane & 15), a = a0 + f * 16 + (lane >> 4) * 4;
            const int up_f = F == 1 ? 0 : f + kFragments, up_lane = F == 1 ? lane ^ 32 : lane;
            f32x4 gate = sums[0][f][g][lane], up = sums[0][up_f][g][up_lane];
#pragma unroll
            for (int v = 1; v < WAVES; ++v) {
                gate += sums[v][f][g][lane];
                up += sums[v][up_f][g][up_lane];
            }
            if (col >= n || a >= p.I || (F == 1 && lane >= 32)) continue;
            f32x4 rest;
#pragma unroll
            for (int q = 0; q < 4; ++q) rest[q] = silu(gate[q]) * up[q];
            const int64_t at = (int64_t)pairs[col] * p.I + a;
#pragma unroll
            for (int i = 0; i < kParts; ++i) {
                bf16x4 part;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    // the largest number of bf16 for what would round to infinity; of an infinity, nothing is left
                    const bool finite = fabsf(rest[q]) <= FLT_MAX;
                    part[q] = (__bf16)(finite ? __builtin_amdgcn_fmed3f(rest[q], -kMaxBf16, kMaxBf16) : rest[q]);
                    rest[q] = fabsf(rest[q]) == INFINITY ? 0.0f : rest[q] - (float)part[q];
                }
                *(bf16x4 *)(p.h + ((int64_t)i * P * p.I + at) * 2) = part;
            }
        }
        __syncthreads();
    }
}

// A workgroup per block of 16 outputs of all tokens and part of the pieces of all groups.  Its waves share them, each a run of them.  The three parts of h of a group's pairs are columns of
// their own, five by five, so that one load and one matrix instruction take them all (in columns of the tokens, with a load and an instruction for each part: 16 tokens
// with 8 of 128 experts of 4096 x 1280 in e4m3 147 us, a quarter of the memory's rate).  A wave that goes on to another group adds up the parts of the last one and adds them, times
// the tokens' weights, to sums of its own in LDS, of the group's tokens and no others.  Weights are DEPTH pieces ahead of their use, h, from the L2, one.  A group has up to
// FIVES times five pairs.
template <bool EIGHT, int WAVES, int TOKENS, int FIVES, int CHUNKS, int DEPTH, int SIMD>
__global__ __launch_bounds__(WAVES *kWave, SIMD) void few_linear_kernel(FewArgs p)
{
    typedef FewPiece<EIGHT, CHUNKS> Piece;
    __shared__ int groups[TOKENS * FUSCO_MAX_K + 1], listed[TOKENS * FUSCO_MAX_K];
    __shared__ f32x4 sums[WAVES][TOKENS][4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int P = p.N * p.k, ld = p.I * (EIGHT ? 1 : 2), block = (int)blockIdx.x / p.parts, of_list = (int)blockIdx.x - block * p.parts, a0 = block * 16;
    for (int i = tid; i <= P; i += WAVES * kWave) {   // whatever lies behind the groups is not looked at
        groups[i] = p.groups[i];
        if (i < P) listed[i] = p.listed[i];
    }
    for (int i = lane; i < p.N * 4; i += kWave) sums[wave][i / 4][i % 4] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    __syncthreads();
    const int pieces = (p.I + Piece::kElements - 1) / Piece::kElements;
    const int64_t total = (int64_t)__builtin_amdgcn_readfirstlane(groups[0]) * pieces;
    // blocks begin at different experts: the waves' runs are dealt out from another place in every block
    const int runs = WAVES * p.parts, run = (of_list * WAVES + wave + block) % runs;
    const int begin = (int)(total * run / runs), end = (int)(total * (run + 1) / runs);

    const __amdgpu_buffer_rsrc_t vh = view(p.h, (int64_t)kParts * P * p.I * 2);
    const uint32_t w_row = a0 + (lane & 15) < p.H ? (uint32_t)((lane & 15) * ld) : kNowhere;
    const int column = lane & 15, in_five = column % kFive, part = column / kFive;
    // a place in the list of all groups' pieces
    struct Place {
        int at, piece;
        __device__ __forceinline__ void next(int pieces)
        {
            if (++piece == pieces) {
                piece = 0;
                ++at;
            }
        }
    };
    Place weights = {begin / pieces, begin % pieces}, rows = weights;
    Piece w[DEPTH];
    float scale[DEPTH];
    auto load = [&](bool more, int d) {
        const int e = __builtin_amdgcn_readfirstlane(more ? groups[1 + weights.at] & 1023 : 0), c0 = more ? weights.piece * Piece::kElements : p.I;
        w[d].load(view(p.w_out + ((int64_t)e * p.H + a0) * ld, (int64_t)(p.H - a0) * ld), w_row, lane, c0, p.I);
        if (EIGHT) scale[d] = p.w_out_scale[((int64_t)e * ((p.H + 127) / 128) + a0 / 128) * ((p.I + 127) / 128) + (more ? c0 / 128 : 0)];
        weights.next(pieces);
    };
    bf16x8 h[FIVES][Piece::kSteps];
    uint32_t h_at[FIVES];       // this lane's columns in h
    int token[FIVES];           // lanes of the first part: the token of their pair, and the weight that it gives the expert
    float weight[FIVES];
    bool chose[FIVES];
    int fives = 0;              // of this group
    auto open = [&] {
        const int group = __builtin_amdgcn_readfirstlane(groups[1 + rows.at]), n = group >> 10 & 15;
        fives = (n + kFive - 1) / kFive;
#pragma unroll
        for (int b = 0; b < FIVES; ++b) {
            const int i = b * kFive + in_five;
            chose[b] = i < n && part < kParts;
            h_at[b] = kNowhere;
            if (!chose[b]) continue;
            const int place = (group >> 14) + i, pair = listed[place];
            token[b] = pair / p.k;
            weight[b] = p.listed_w[place];
            h_at[b] = (uint32_t)((part * P + pair) * (p.I * 2));
        }
    };
    auto load_h = [&](bool more) {
        const int c0 = more ? rows.piece * Piece::kElements : p.I;
#pragma unroll
        for (int b = 0; b < FIVES; ++b) {
            if (b > 0 && b >= fives) break;
#pragma unroll
            for (int s = 0; s < Piece::kSteps; ++s) {
                const int c = c0 + Piece::element(lane, s);
                h[b][s] = load_fragment(vh, c < p.I && h_at[b] != kNowhere ? h_at[b] + c * 2 : kNowhere);
            }
        }
    };
    f32x4 acc[FIVES];
#pragma unroll
    for (int b = 0; b < FIVES; ++b) {
        acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        h_at[b] = kNowhere;
        token[b] = 0;
        weight[b] = 0.0f;
        chose[b] = false;
#pragma unroll
        for (int s = 0; s < Piece::kSteps; ++s) h[b][s] = {};
    }
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) load(begin + d < end, d);
    if (begin < end) open();
    load_h(begin < end);
    for (int i0 = begin; i0 < end; i0 += DEPTH) {
#pragma unroll
        for (int d = 0; d < DEPTH; ++d) {
            const int i = i0 + d;
            if (i >= end) break;
            const Piece wn = w[d];
            bf16x8 hn[FIVES][Piece::kSteps];
            float weight_now[FIVES];
            int token_now[FIVES];
            bool chose_now[FIVES];
#pragma unroll
            for (int b = 0; b < FIVES; ++b) {
                weight_now[b] = weight[b];
                token_now[b] = token[b];
                chose_now[b] = chose[b];
#pragma unroll
                for (int s = 0; s < Piece::kSteps; ++s) hn[b][s] = h[b][s];
            }
            const float scale_now = scale[d];
            const int at = rows.at, fives_now = fives;
            rows.next(pieces);
            const bool more = i + 1 < end;
            if (more && rows.at != at) open();
            load_h(more);
            load(i + DEPTH < end, d);
            bf16x8 a[Piece::kSteps];
#pragma unroll
            for (int s = 0; s < Piece::kSteps; ++s) a[s] = wn.operand(s);
#pragma unroll
            for (int b = 0; b < FIVES; ++b) {
                if (b > 0 && b >= fives_now) break;
                f32x4 sum = EIGHT ? f32x4{0.0f, 0.0f, 0.0f, 0.0f} : acc[b];
#pragma unroll
                for (int s = 0; s < Piece::kSteps; ++s) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[s], hn[b][s], sum, 0, 0, 0);
#pragma unroll
                for (int q = 0; q < 4; ++q) acc[b][q] = EIGHT ? fmaf(scale_now, sum[q], acc[b][q]) : sum[q];
                if (rows.at != at || !more) {   // the last piece of this group here
                    f32x4 v = acc[b];
#pragma unroll
                    for (int j = 1; j < kParts; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) v[q] += __shfl(acc[b][q], (lane & 48) | ((column + j * kFive) & 15));
                    if (chose_now[b] && part == 0) {
                        f32x4 &to = sums[wave][token_now[b]][lane >> 4];
#pragma unroll
                        for (int q = 0; q < 4; ++q) to[q] = fmaf(weight_now[b], v[q], to[q]);
                    }
                    acc[b] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
                }
            }
        }
    }
    __syncthreads();
    const int threads = WAVES * kWave;
    // The last of a block's parts to end adds them all up, in their order.  Sums are stored past the L2s (at agent scope); every thread waits for its own before the
    // workgroup counts itself, so that no cache has to be written back (a fence at agent scope, which does that, takes over 100 us here).
    if (p.parts > 1) {
        float *mine = p.partial + ((int64_t)block * p.parts + of_list) * p.N * 16;
        for (int i = tid; i < p.N * 16; i += threads) {
            float v = 0.0f;
#pragma unroll
            for (int s = 0; s < WAVES; ++s) v += ((const float *)sums[s])[i];
            __hip_atomic_store(mine + i, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        if (tid == 0) listed[0] = (int)__hip_atomic_fetch_add(p.arrived + block, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        __syncthreads();
        if (listed[0] != p.parts - 1) return;
        const float *all = p.partial + (int64_t)block * p.parts * p.N * 16;
        for (int i = tid; i < p.N * 16; i += threads) {
            float v = 0.0f;
            for (int s = 0; s < p.parts; ++s) v += __hip_atomic_load(all + (int64_t)s * p.N * 16 + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            ((float *)sums[0])[i] = v;
        }
        __syncthreads();
    }
    for (int i = tid; i < p.N * 4; i += threads) {
        const int t = i / 4, a = a0 + i % 4 * 4;
        f32x4 v = sums[0][t][i % 4];
#pragma unroll
        for (int s = 1; s < WAVES; ++s)
            if (p.parts == 1) v += sums[s][t][i % 4];
        if (a >= p.H) continue;
        const int64_t to = (int64_t)t * p.H + a;
        if (p.out_f32) *(f32x4 *)(p.out + to * 4) = v;
        else store4(p.out, to, v);
    }
}

}   // namespace

#endif
