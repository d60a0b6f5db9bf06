// The MoE block in 8 bits for MI355X (gfx950): rows and weights to e4m3 and back (eight.h), the experts' products on them and the gradients from kept rows (products.h);
// and the whole layer for a few tokens with weights of either type (few.h).  C entry points, declared in fusco.h.
#include "block_host.h"
#include "eight.h"
#include "few.h"

namespace {

// rows of e4m3 that the kernels take
bool eight_row_ok(int32_t elements) { return elements > 0 && elements % 16 == 0 && (size_t)elements <= FUSCO_MAX_ROW_BYTES; }
int32_t blocks_of(int32_t n) { return (n + kBlockColumns - 1) / kBlockColumns; }
// scales of a row: loads inside a tile's are addressed with 31 bits
bool scale_stride_ok(int32_t stride, int32_t columns) { return stride >= blocks_of(columns) && stride <= FUSCO_MAX_SCALE_STRIDE; }

int fp8_check(const fusco_fp8 *f)
{
    if (!f || f->rows < 0 || !eight_row_ok(f->columns) || f->matrix_rows < 0 || !scale_stride_ok(f->scale_stride, f->columns)) return FUSCO_ERR_INVALID_ARG;
    if (f->rows > INT32_MAX) return FUSCO_ERR_INVALID_ARG;
    if (f->matrix_rows && (f->rows % f->matrix_rows != 0 || f->scale_stride != blocks_of(f->columns))) return FUSCO_ERR_INVALID_ARG;
    // a launch has fewer than 2^32 threads, in whole workgroups
    constexpr int kEach = kEightGroups * kEightEach;   // blocks of a workgroup
    if (f->rows * blocks_of(f->columns) > UINT32_MAX / kEightThreads * kEach) return FUSCO_ERR_INVALID_ARG;
    if (f->matrix_rows && f->rows / f->matrix_rows * blocks_of(f->matrix_rows) * blocks_of(f->columns) >= ((int64_t)1 << 32) / kMatrixThreads) return FUSCO_ERR_INVALID_ARG;
    return dtype_ok(f->dtype) ? FUSCO_OK : FUSCO_ERR_UNSUPPORTED;
}

EightArgs eight_args(const fusco_fp8 *f, const void *in, void *out, const float *scale)
{
    const int32_t per_row = blocks_of(f->columns);
    return {(const char *)in, (char *)out, const_cast<float *>(scale), (uint32_t)(f->rows * per_row), (uint32_t)per_row, f->columns, f->scale_stride,
            f->matrix_rows, blocks_of(f->matrix_rows)};
}

dim3 block_grid(const EightArgs &a) { return dim3((a.blocks + kEightGroups * kEightEach - 1) / (kEightGroups * kEightEach)); }

template <bool BF16, bool PAST, bool STREAMED>
void launch_to_eight(const fusco_fp8 *f, const EightArgs &a, hipStream_t s)
{
    if (f->matrix_rows) hipLaunchKernelGGL((matrix_to_eight_kernel<BF16, PAST, STREAMED>), dim3((unsigned)(f->rows / f->matrix_rows * a.scale_rows * a.per_row)), dim3(kMatrixThreads), 0, s, a);
    else hipLaunchKernelGGL((rows_to_eight_kernel<BF16, PAST, STREAMED>), block_grid(a), dim3(kEightThreads), 0, s, a);
}

// x past the caches where they cannot hold it, q where little of it would still be there when it is read, rows by the next call, matrices later.  To and back, q through / past the caches,
// us: rows 131072 x 4096 549 / 512, 131072 x 1280 (q 168 MB) 153 / 162; fp32 matrices 64 x 1408 x 2048 (q 185 MB) 261 / 251, 128 x 4096 x 1280 1053 / 975, 8 x 2560 x 4096 (q 84 MB) 110 / 115.
template <bool BF16>
void launch_to_eight(const fusco_fp8 *f, const EightArgs &a, hipStream_t s)
{
    const int64_t elements = f->rows * f->columns;
    if (elements > (f->matrix_rows ? kCacheBytes / 2 : kCacheBytes)) launch_to_eight<BF16, true, true>(f, a, s);
    else if (elements * (BF16 ? 2 : 4) > kCacheBytes) launch_to_eight<BF16, true, false>(f, a, s);
    else launch_to_eight<BF16, false, false>(f, a, s);
}

// arguments of a product of e4m3 rows [P, C] with e4m3 weights; gated: `outputs` units
ProductArgs eight_product(const fusco_layout *L, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, const void *d_w, const float *d_w_scale, void *d_out, void *d_pre,
                          int32_t outputs, int32_t C, bool gated)
{
    ProductArgs a = {L->exp_off, (const char *)d_x, (const char *)d_w, (char *)d_out, (char *)d_pre, L->E, outputs, 0, C / 2};
    a.row_scale = d_x_scale;
    a.weight_scale = d_w_scale;
    a.row_scales = x_scale_stride;
    a.scale_rows = blocks_of(outputs) * (gated ? 2 : 1);
    a.scales = blocks_of(C);
    return a;
}

// ---- the layer for a few tokens

int few_check(const fusco_few *f)
{
    if (!f || f->N < 0 || f->N > FUSCO_MAX_FEW_TOKENS || f->E < 1 || f->E > FUSCO_MAX_E || f->k < 1 || f->k > FUSCO_MAX_K) return FUSCO_ERR_INVALID_ARG;
    if ((f->weight_dtype != FUSCO_BF16 && f->weight_dtype != FUSCO_E4M3) || !dtype_ok(f->out_dtype)) return FUSCO_ERR_UNSUPPORTED;
    const bool eight = f->weight_dtype == FUSCO_E4M3;
    if (!row_ok(f->H) || !row_ok(f->I) || (eight && (f->H % 16 != 0 || f->I % 16 != 0))) return FUSCO_ERR_INVALID_ARG;
    // loads inside one expert's weights, inside x and inside h are addressed with 31 bits
    if (2 * (int64_t)f->I * f->H * (eight ? 1 : 2) >= (int64_t)kNowhere || (int64_t)f->N * f->k * f->I * 2 * kParts >= (int64_t)kNowhere || (int64_t)f->N * f->H * 2 >= (int64_t)kNowhere)
        return FUSCO_ERR_INVALID_ARG;
    // blocks of eight units of all experts that can be chosen, a workgroup of 256 threads each: fewer than 2^32 threads
    const int64_t experts = f->N * f->k < f->E ? f->N * f->k : f->E;
    if (experts * ((f->I + 7) / 8) >= ((int64_t)1 << 24) - 1) return FUSCO_ERR_INVALID_ARG;
    return FUSCO_OK;
}

constexpr int kFewOutputs = 16;   // of a workgroup's block

// Parts of the list of groups: where there are fewer blocks of outputs than compute units, as many (up to four) as leave the fewest units without work.  Down
// product, parts 1 / 2 / 4, us: 128 blocks of 1408 (16 tokens, 64 experts, bf16) 77 / 47 / 47; 180 blocks of 1040 (5 tokens, 30 experts, bf16) 39 / 41 / 38; 256
// blocks of 1280 (16 tokens, 83 experts, e4m3) 89 / 97 / 100.
constexpr int kFewPartial = 4 * kCus;   // workgroups that leave sums
int few_parts(int32_t H)
{
    const int blocks = (H + kFewOutputs - 1) / kFewOutputs;
    if (blocks >= kCus) return 1;
    int best = 1;
    double most = 0.0;
    for (int parts = 1; parts <= 4; ++parts) {
        const double busy = (double)blocks * parts / (ceil((double)blocks * parts / kCus) * kCus);
        if (busy > most + 0.05) {
            most = busy;
            best = parts;
        }
    }
    return best;
}

// scratch: groups, listed pairs and their weights, parts that are done, h, sums of the parts, each on a boundary of 16 bytes
struct FewScratch {
    size_t listed, listed_w, arrived, h, partial, bytes;
    FewScratch(int32_t N, int32_t k, int32_t I)
    {
        const size_t list = ((size_t)N * k + 4) / 4 * 16;
        listed = list;
        listed_w = 2 * list;
        arrived = 3 * list;
        h = arrived + kFewPartial * 4;
        partial = h + (size_t)N * k * I * 2 * kParts;
        bytes = partial + (size_t)kFewPartial * N * kFewOutputs * 4;
    }
};

int few_slots(const FewArgs &a) { return a.N * a.k < a.E ? a.N * a.k : a.E; }

template <bool EIGHT, int F, int G>
void launch_few_gated(const FewArgs &a, hipStream_t s)
{
    constexpr int kUnits = 8 * F, kWaves = 4, kSimd = F == 4 ? 2 : G == 2 ? 3 : 4;
    const int64_t grid = (int64_t)few_slots(a) * ((a.I + kUnits - 1) / kUnits) + 1;   // and the one that makes the groups
    hipLaunchKernelGGL((few_gated_kernel<EIGHT, F, kWaves, G, 2, kSimd>), dim3((unsigned)grid), dim3(kWaves * kWave), 0, s, a);
}

// Gated product, experts of 4096 x (2 x 1280), us: blocks of 8 units in bf16 where those of 16 would leave less than four workgroups per compute unit (one token with 8
// experts, 640 blocks of 16: 32 / 35 with 16; 5 tokens with 30 experts of 2880 x (2 x 1040): 60 / 55; e4m3 for one token 20.7 / 19.5); blocks of 32, which take a row of x
// half as often, where there are more than eight (64 tokens with all of 128 experts, e4m3 281 / 318, bf16 452 / 484; 16 tokens with 83, e4m3 158 / 160; but bf16 with one pair per
// expert, 16 tokens with 41 of 64 experts of 2048 x (2 x 1408), 89 / 84); 2 x 16 columns at a time from eight pairs per expert on (64 tokens with 8 experts 44 / 51; 64 tokens with
// 128 experts 474 / 452).  The four waves hold two pieces each: 16 tokens with 83 experts in e4m3, one, two, three pieces 159 / 160 / 183, eight waves 177 / 186.
// Down product: eight waves with two pieces of e4m3 or three of bf16: 16 tokens with 83 experts of 1280 x 4096 in e4m3, one, two, three pieces 103 / 91 / 89, sixteen waves 91 /
// 95 / 95; one token 17.0 / 15.7 / 16.3; bf16, 5 tokens with 30 experts of 1040 x 2880 46 / 40 / 39.  Groups of fifteen pairs from three per expert on: 64 tokens with 32 experts of
// 1280 x 4096 in e4m3 79 / 93 with five.
template <bool EIGHT>
int launch_moe_few(const FewArgs &a, hipStream_t s)
{
    const int64_t blocks = (int64_t)few_slots(a) * ((a.I + 15) / 16);
    const int pairs = a.N * a.k / a.E;   // per expert
    if (pairs >= 8) launch_few_gated<EIGHT, 2, 2>(a, s);
    else if (!EIGHT && blocks < 4 * kCus) launch_few_gated<EIGHT, EIGHT ? 2 : 1, 1>(a, s);
    else if (blocks > 8 * kCus && (EIGHT || pairs >= 3)) launch_few_gated<EIGHT, 4, 1>(a, s);
    else launch_few_gated<EIGHT, 2, 1>(a, s);
    const dim3 grid((unsigned)((a.H + kFewOutputs - 1) / kFewOutputs * a.parts)), block(8 * kWave);
    constexpr int kDepth = EIGHT ? 2 : 3;
    if (a.group > kFive) hipLaunchKernelGGL((few_linear_kernel<EIGHT, 8, 64, kManyFives, 2, kDepth, 2>), grid, block, 0, s, a);
    else if (a.N <= 16) hipLaunchKernelGGL((few_linear_kernel<EIGHT, 8, 16, 1, 2, kDepth, 4>), grid, block, 0, s, a);
    else hipLaunchKernelGGL((few_linear_kernel<EIGHT, 8, 64, 1, 2, kDepth, 4>), grid, block, 0, s, a);
    return launch_status();
}

}   // namespace

extern "C" {

int fusco_to_fp8(const fusco_fp8 *f, const void *d_x, void *d_q, float *d_scale, void *stream)
{
    const int rc = fp8_check(f);
    if (rc != FUSCO_OK) return rc;
    const void *const p[] = {d_x, d_q, d_scale};
    if (check_pointers(f->rows == 0, p, 3) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (f->rows == 0) return FUSCO_OK;
    const EightArgs a = eight_args(f, d_x, d_q, d_scale);
    if (f->dtype == FUSCO_BF16) launch_to_eight<true>(f, a, (hipStream_t)stream);
    else launch_to_eight<false>(f, a, (hipStream_t)stream);
    return launch_status();
}

int fusco_from_fp8(const fusco_fp8 *f, const void *d_q, const float *d_scale, void *d_x, void *stream)
{
    const int rc = fp8_check(f);
    if (rc != FUSCO_OK) return rc;
    const void *const p[] = {d_q, d_scale, d_x};
    if (check_pointers(f->rows == 0, p, 3) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (f->rows == 0) return FUSCO_OK;
    const EightArgs a = eight_args(f, d_q, d_x, d_scale);
    if (f->dtype == FUSCO_BF16) hipLaunchKernelGGL(from_eight_kernel<true>, block_grid(a), dim3(kEightThreads), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(from_eight_kernel<false>, block_grid(a), dim3(kEightThreads), 0, (hipStream_t)stream, a);
    return launch_status();
}

int fusco_experts_gated_fp8(const fusco_layout *L, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, const void *d_w, const float *d_w_scale, void *d_h, void *d_pre,
                            int32_t H, int32_t I, void *stream)
{
    if (!layout_ok(L) || !eight_row_ok(H) || !row_ok(I) || !row_ok(2 * I) || 2 * (int64_t)I * H >= (int64_t)kNowhere || !scale_stride_ok(x_scale_stride, H)) return FUSCO_ERR_INVALID_ARG;
    const void *const p[] = {d_x, d_x_scale, d_w, d_w_scale, d_h};
    if (check_pointers(L->N == 0, p, 5) != FUSCO_OK || !aligned16(d_pre)) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    const ProductArgs a = eight_product(L, d_x, d_x_scale, x_scale_stride, d_w, d_w_scale, d_h, d_pre, I, H, true);
    return launch_by_rows<kAlongC, kStoreGated, true>(L, a, (hipStream_t)stream);
}

int fusco_experts_linear_fp8(const fusco_layout *L, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, const void *d_w, const float *d_w_scale, void *d_y, int32_t C, int32_t M,
                             void *stream)
{
    if (!layout_ok(L) || !eight_row_ok(C) || !row_ok(M) || (int64_t)M * C >= (int64_t)kNowhere || !scale_stride_ok(x_scale_stride, C)) return FUSCO_ERR_INVALID_ARG;
    const void *const p[] = {d_x, d_x_scale, d_w, d_w_scale, d_y};
    if (check_pointers(L->N == 0, p, 5) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    const ProductArgs a = eight_product(L, d_x, d_x_scale, x_scale_stride, d_w, d_w_scale, d_y, nullptr, M, C, false);
    return launch_by_rows<kAlongC, kStoreBf16, true>(L, a, (hipStream_t)stream);
}

int fusco_experts_input_grad_fp8(const fusco_layout *L, const void *d_dy, const void *d_w, void *d_dpre, const void *d_pre, const float *d_pre_scale, int32_t pre_scale_stride, int32_t M,
                                 int32_t C, void *stream)
{
    if (!layout_ok(L) || !row_ok(M) || !row_ok(2 * C) || !weights_ok(M, C) || C % 16 != 0 || !scale_stride_ok(pre_scale_stride, 2 * C)) return FUSCO_ERR_INVALID_ARG;
    const void *const p[] = {d_dy, d_w, d_dpre, d_pre, d_pre_scale};
    if (check_pointers(L->N == 0, p, 5) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    ProductArgs a = {L->exp_off, (const char *)d_dy, (const char *)d_w, (char *)d_dpre, (char *)const_cast<void *>(d_pre), L->E, C, 0, M};
    a.row_scale = d_pre_scale;
    a.row_scales = pre_scale_stride;
    return launch_by_rows<kAcross, kStoreGatedGradKept>(L, a, (hipStream_t)stream);
}

int fusco_experts_weight_grad_fp8(const fusco_layout *L, const void *d_dy, const void *d_x, const float *d_x_scale, int32_t x_scale_stride, void *d_dw, int dw_dtype, int32_t M, int32_t C,
                                  void *stream)
{
    if (!layout_ok(L) || !row_ok(M) || !row_ok(C) || !eight_row_ok(C) || !weights_ok(M, C) || !scale_stride_ok(x_scale_stride, C)) return FUSCO_ERR_INVALID_ARG;
    if (!dtype_ok(dw_dtype)) return FUSCO_ERR_UNSUPPORTED;
    const void *const rows[] = {d_dy, d_x, d_x_scale}, *const weights[] = {d_dw};
    if (check_pointers(L->N == 0, rows, 3) != FUSCO_OK || check_pointers(false, weights, 1) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (((int64_t)L->E * ((M + 255) / 256)) * ((C + 255) / 256) >= (int64_t)1 << 30) return FUSCO_ERR_INVALID_ARG;
    ProductArgs a = {L->exp_off, (const char *)d_x, (const char *)d_dy, (char *)d_dw, nullptr, L->E, C, M, 0};
    a.row_scale = d_x_scale;
    a.row_scales = x_scale_stride;
    if (dw_dtype == FUSCO_F32) launch_product(product_kernel<kAcross, kAcross, 256, 4, 2, kStoreF32, false, true>, a, (hipStream_t)stream);
    else launch_product(product_kernel<kAcross, kAcross, 256, 4, 2, kStoreBf16, false, true>, a, (hipStream_t)stream);
    return launch_status();
}

size_t fusco_moe_few_scratch_bytes(int32_t N, int32_t k, int32_t I)
{
    if (N < 0 || N > FUSCO_MAX_FEW_TOKENS || k < 1 || k > FUSCO_MAX_K || !row_ok(I)) return 0;
    return FewScratch(N, k, I).bytes;
}

int fusco_moe_few(const fusco_few *f, const void *d_x, const int32_t *d_topk_idx, const float *d_w, const void *d_w_in, const float *d_w_in_scale, const void *d_w_out,
                  const float *d_w_out_scale, void *d_out, void *d_scratch, size_t scratch_bytes, void *stream)
{
    const int rc = few_check(f);
    if (rc != FUSCO_OK) return rc;
    const bool empty = f->N == 0, eight = f->weight_dtype == FUSCO_E4M3;
    const void *const p[] = {d_x, d_topk_idx, d_w, d_w_in, d_w_out, d_out, d_scratch}, *const scales[] = {d_w_in_scale, d_w_out_scale};
    if (check_pointers(empty, p, 7) != FUSCO_OK || check_pointers(empty || !eight, scales, 2) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (empty) return FUSCO_OK;
    if (scratch_bytes < fusco_moe_few_scratch_bytes(f->N, f->k, f->I)) return FUSCO_ERR_WORKSPACE;
    FewArgs a = {};
    a.x = (const char *)d_x; a.chosen = d_topk_idx; a.w = d_w;
    a.w_in = (const char *)d_w_in; a.w_out = (const char *)d_w_out; a.w_in_scale = d_w_in_scale; a.w_out_scale = d_w_out_scale;
    a.out = (char *)d_out;
    const FewScratch at(f->N, f->k, f->I);
    char *scratch = (char *)d_scratch;
    a.groups = (int32_t *)scratch; a.listed = (int32_t *)(scratch + at.listed); a.listed_w = (float *)(scratch + at.listed_w); a.arrived = (uint32_t *)(scratch + at.arrived);
    a.h = scratch + at.h; a.partial = (float *)(scratch + at.partial);
    a.parts = few_parts(f->H);
    a.group = f->N * f->k >= 3 * f->E ? kFive * kManyFives : kFive;
    a.N = f->N; a.E = f->E; a.k = f->k; a.H = f->H; a.I = f->I; a.out_f32 = f->out_dtype == FUSCO_F32;
    return eight ? launch_moe_few<true>(a, (hipStream_t)stream) : launch_moe_few<false>(a, (hipStream_t)stream);
}

}   // extern "C"
