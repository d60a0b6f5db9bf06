// The operators around the token shuffle of an MoE block for MI355X (gfx950): the experts' products on the dispatched rows
// (products.h).  C entry points, declared in fusco.h.
#include "products.h"

namespace {

// rows of `elements` bf16 that the kernels take
bool row_ok(int32_t elements) { return elements > 0 && elements % 8 == 0 && (size_t)elements * 2 <= FUSCO_MAX_ROW_BYTES; }

// one expert's weights: loads inside them are addressed with 31 bits
bool weights_ok(int64_t rows, int64_t cols) { return rows * cols * 2 < (int64_t)kNowhere; }

int check_pointers(bool empty, const void *const *p, int n)
{
    for (int i = 0; i < n; ++i)
        if ((!empty && !p[i]) || !aligned16(p[i])) return FUSCO_ERR_INVALID_ARG;
    return FUSCO_OK;
}

template <typename K>
void launch_product(K kernel, int64_t tiles, int per_cu, const ProductArgs &a, hipStream_t s)
{
    // whole sets of compute units, so that the tile list is dealt to the XCDs in runs
    const int sets = tiles > (int64_t)kCus && per_cu > 1 ? per_cu : 1;
    hipLaunchKernelGGL(kernel, dim3(kCus * sets), dim3(kTileThreads), 0, s, a);
}

// Products whose tiles are rows of one expert: the tile's height goes by the mean number of rows of an expert
template <int AMODE, int STORE>
int launch_by_rows(const fusco_layout *L, const ProductArgs &a, hipStream_t s)
{
    const int64_t mean = L->P / L->E, tiles_a = (a.NA + kTileA - 1) / kTileA;
    if (mean >= 160) launch_product(product_kernel<AMODE, kAlongC, 256, 8, 4, STORE>, (L->P / 256 + L->E) * tiles_a, 1, a, s);
    else if (mean >= 48) launch_product(product_kernel<AMODE, kAlongC, 128, 4, 4, STORE>, (L->P / 128 + L->E) * tiles_a, 1, a, s);
    else launch_product(product_kernel<AMODE, kAlongC, 64, 4, 2, STORE>, (L->P / 64 + L->E) * tiles_a, 1, a, s);
    return launch_status();
}

}   // namespace

extern "C" {

int fusco_experts_gated(const fusco_layout *L, const void *d_x, const void *d_w, void *d_h, void *d_pre, int32_t H, int32_t I, void *stream)
{
    if (!layout_ok(L) || !row_ok(H) || !row_ok(I) || !row_ok(2 * I) || !weights_ok(2 * (int64_t)I, H)) return FUSCO_ERR_INVALID_ARG;
    const void *const p[] = {d_x, d_w, d_h};
    if (check_pointers(L->N == 0, p, 3) != FUSCO_OK || !aligned16(d_pre)) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    ProductArgs a = {L->exp_off, (const char *)d_x, (const char *)d_w, (char *)d_h, (char *)d_pre, L->E, I, 0, H};
    return launch_by_rows<kAlongC, kStoreGated>(L, a, (hipStream_t)stream);
}

int fusco_experts_linear(const fusco_layout *L, const void *d_x, const void *d_w, void *d_y, int32_t C, int32_t M, void *stream)
{
    if (!layout_ok(L) || !row_ok(C) || !row_ok(M) || !weights_ok(M, C)) return FUSCO_ERR_INVALID_ARG;
    const void *const p[] = {d_x, d_w, d_y};
    if (check_pointers(L->N == 0, p, 3) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    ProductArgs a = {L->exp_off, (const char *)d_x, (const char *)d_w, (char *)d_y, nullptr, L->E, M, 0, C};
    return launch_by_rows<kAlongC, kStoreBf16>(L, a, (hipStream_t)stream);
}

int fusco_experts_input_grad(const fusco_layout *L, const void *d_dy, const void *d_w, void *d_dx, const void *d_pre, int32_t M, int32_t C, void *stream)
{
    if (!layout_ok(L) || !row_ok(M) || !row_ok(C) || !weights_ok(M, C)) return FUSCO_ERR_INVALID_ARG;
    if (d_pre && !row_ok(2 * C)) return FUSCO_ERR_INVALID_ARG;
    const void *const p[] = {d_dy, d_w, d_dx};
    if (check_pointers(L->N == 0, p, 3) != FUSCO_OK || !aligned16(d_pre)) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    ProductArgs a = {L->exp_off, (const char *)d_dy, (const char *)d_w, (char *)d_dx, (char *)d_pre, L->E, C, 0, M};
    return d_pre ? launch_by_rows<kAcross, kStoreGatedGrad>(L, a, (hipStream_t)stream) : launch_by_rows<kAcross, kStoreBf16>(L, a, (hipStream_t)stream);
}

int fusco_experts_weight_grad(const fusco_layout *L, const void *d_dy, const void *d_x, void *d_dw, int dw_dtype, int32_t M, int32_t C, void *stream)
{
    if (!layout_ok(L) || !row_ok(M) || !row_ok(C) || !weights_ok(M, C)) return FUSCO_ERR_INVALID_ARG;
    if (dw_dtype != FUSCO_BF16 && dw_dtype != FUSCO_F32) return FUSCO_ERR_UNSUPPORTED;
    const void *const rows[] = {d_dy, d_x}, *const weights[] = {d_dw};
    if (check_pointers(L->N == 0, rows, 2) != FUSCO_OK || check_pointers(false, weights, 1) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (((int64_t)L->E * ((M + 255) / 256)) * ((C + 255) / 256) >= (int64_t)1 << 30) return FUSCO_ERR_INVALID_ARG;
    ProductArgs a = {L->exp_off, (const char *)d_x, (const char *)d_dy, (char *)d_dw, nullptr, L->E, C, M, 0};
    const int64_t tiles = (int64_t)L->E * ((M + 255) / 256) * ((C + 255) / 256);
    if (dw_dtype == FUSCO_F32) launch_product(product_kernel<kAcross, kAcross, 256, 8, 4, kStoreF32>, tiles, 1, a, (hipStream_t)stream);
    else launch_product(product_kernel<kAcross, kAcross, 256, 8, 4, kStoreBf16>, tiles, 1, a, (hipStream_t)stream);
    return launch_status();
}

}   // extern "C"
