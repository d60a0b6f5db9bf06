// The operators around the token shuffle of an MoE block for MI355X (gfx950): the experts' products on the dispatched rows
// (products.h), routing (routing.h), the norms around the block (norms.h) and the gradient of the combine (gradients.h).  C entry
// points, declared in fusco.h.
#include "products.h"
#include "routing.h"
#include "norms.h"
#include "gradients.h"
#include "fusco_probe.h"
#include <math.h>

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
void launch_product(K kernel, const ProductArgs &a, hipStream_t s)
{
    // a workgroup per compute unit, also where there are fewer tiles: the list is dealt to the XCDs in runs
    hipLaunchKernelGGL(kernel, dim3(kCus), dim3(kTileThreads), 0, s, a);
}

// Few rows per expert: a workgroup per tile of 16 token rows and block of weight rows; tiles that do not exist leave at once
constexpr int kFewF = 2;
template <int STORE>
int64_t few_workgroups(const fusco_layout *L, const ProductArgs &a)
{
    constexpr int kUnits = STORE == kStoreGated ? 8 * kFewF : 16 * kFewF;
    const int64_t blocks = (a.NA + kUnits - 1) / kUnits, spread = L->P / 16 + L->E, tiles = spread < L->P ? spread : L->P;
    return tiles * blocks;
}
// eight waves share a long row, four a short one: 1280 x 4096, 32 tokens 217 us / 231 with eight; 4096 x (2 x 1280) 398 / 383
int few_waves(const ProductArgs &a) { return a.C >= 2048 ? 8 : 4; }

template <int WAVES, int STORE>
int launch_few(const fusco_layout *L, const ProductArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((few_rows_kernel<kFewF, WAVES, STORE>), dim3((unsigned)few_workgroups<STORE>(L, a)), dim3(WAVES * kWave), 0, s, a);
    return launch_status();
}

// Products whose tiles are rows of one expert.  From eight rows per expert on, the tile's height is the one whose rounds of tiles over the compute units
// take least: an expert's rows end inside a tile, two fifths of one on average, and a tile of 64, 128 or 256 rows takes 1 : 1.2 : 1.4 (fitted to
// 130 products of 8 to 128 experts with 8 to 1000 rows, where the choice is 3 % slower than the best one; by the mean number of rows alone, from 48 and from
// 96 on, it was 20 %).  Measured with 64 / 128 / 256, us: 128 experts of 4096 x (2 x 1280) gated, 8 rows 455 / 531 / 591, 64 rows 671 / 511 / 619, 128 rows 996 / 826 /
// 601; 16 of 2048 x 1408 with 128 rows, gradient of the pre-activations 32 / 48 / 61; 16 of 4096 x (2 x 1280) with 230 rows 224 / 185 / 127, its
// gradient of the pre-activations 120 / 90 / 136.
template <int STORE>
int tile_rows(const fusco_layout *L, const ProductArgs &a)
{
    const int units = STORE == kStoreGated ? kTileA / 2 : kTileA;
    const double across = (a.NA + units - 1) / units, takes[] = {1.0, 1.2, 1.4};
    int best = 256;
    double least = INFINITY;
    for (int i = 2; i >= 0; --i) {
        const int rows = 64 << i;
        const double tiles = fmax((double)L->E, (double)L->P / rows + 0.4 * L->E) * across;
        const double time = ceil(tiles / kCus) * takes[i];
        if (time < least) {
            least = time;
            best = rows;
        }
    }
    return best;
}

// Rows per tile, 16 for few_rows_kernel: below eight rows per expert (4 rows: 437 us, 441 in tiles of 64; 8 rows: 482 / 455), unless its
// workgroups for very many outputs come to more threads than a launch may have
template <int AMODE, int STORE>
int rows_per_tile(const fusco_layout *L, const ProductArgs &a)
{
    if (AMODE == kAlongC && L->P / L->E < 8 && few_workgroups<STORE>(L, a) * few_waves(a) * kWave <= UINT32_MAX) return 16;
    return tile_rows<STORE>(L, a);
}

template <int AMODE, int STORE>
int launch_by_rows(const fusco_layout *L, const ProductArgs &a, hipStream_t s)
{
    const int rows = rows_per_tile<AMODE, STORE>(L, a);
    if constexpr (AMODE == kAlongC) {
        if (rows == 16) return few_waves(a) == 8 ? launch_few<8, STORE>(L, a, s) : launch_few<4, STORE>(L, a, s);
    }
    if (rows == 256) launch_product(product_kernel<AMODE, kAlongC, 256, 4, 2, STORE>, a, s);
    else if (rows == 128) launch_product(product_kernel<AMODE, kAlongC, 128, 2, 2, STORE>, a, s);
    else launch_product(product_kernel<AMODE, kAlongC, 64, 2, 1, STORE>, a, s);
    return launch_status();
}

// ---- rows of one workgroup each

bool dtype_ok(int t) { return t == FUSCO_BF16 || t == FUSCO_F32; }

// threads of a workgroup whose threads take `cpt` chunks each
unsigned row_threads(int chunks, int cpt) { return (unsigned)((chunks + cpt * kWave - 1) / (cpt * kWave) * kWave); }

// chunks per thread: few rows spread each over as many threads as there are chunks, up to 512; more in flight per thread otherwise
int row_cpt(int chunks, bool few)
{
    if (few) return chunks <= 512 ? 1 : chunks <= 1024 ? 2 : 4;
    return chunks <= 64 ? 1 : chunks <= 1024 ? 2 : 4;
}

// calls f(integral constant CPT)
template <typename F>
void with_cpt(int cpt, F f)
{
    if (cpt == 1) f(std::integral_constant<int, 1>());
    else if (cpt == 2) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 4>());
}

// calls f(stream is bf16, block is bf16, loads go past the caches) for the pairs of types that are offered.  Rows of bf16 go past the caches if
// the call's tensors exceed the memory-side cache, rows of fp32, whose two halves a thread loads one after the other, never.  Norm after a
// block, past / through, us: 16384 x 4096 bf16 102.4 / 104.4, 512 x 7168 6.3 / 6.3; with an fp32 stream 8192 x 7168 146 / 137, 1537 x 2880
// 13.0 / 9.5; gradients 8192 x 7168 with an fp32 stream 245 / 230.
template <typename F>
void with_types(const fusco_norm *n, int64_t bytes_per_element, F f)
{
    if (n->stream_dtype == FUSCO_BF16 && bytes_per_element * n->N * n->H > kCacheBytes) f(std::true_type(), std::true_type(), std::true_type());
    else if (n->stream_dtype == FUSCO_BF16) f(std::true_type(), std::true_type(), std::false_type());
    else if (n->block_dtype == FUSCO_BF16) f(std::false_type(), std::true_type(), std::false_type());
    else f(std::false_type(), std::false_type(), std::false_type());
}

int norm_check(const fusco_norm *n)
{
    if (!n || n->N < 0 || n->H < 8 || n->H % 8 != 0 || n->H > FUSCO_MAX_NORM_H || !(n->eps > 0.0f) || !isfinite(n->eps)) return FUSCO_ERR_INVALID_ARG;
    if (!dtype_ok(n->stream_dtype) || !dtype_ok(n->block_dtype) || !dtype_ok(n->gain_dtype)) return FUSCO_ERR_UNSUPPORTED;
    if (n->stream_dtype == FUSCO_BF16 && n->block_dtype != FUSCO_BF16) return FUSCO_ERR_UNSUPPORTED;
    return FUSCO_OK;
}

int gate_check(const fusco_norm *n, const void *d_gate)
{
    if (n->gate_kind != FUSCO_GATE_NONE && n->gate_kind != FUSCO_GATE_CHANNEL && n->gate_kind != FUSCO_GATE_TOKEN) return FUSCO_ERR_UNSUPPORTED;
    const bool empty = n->N == 0 && n->gate_kind == FUSCO_GATE_TOKEN;
    return (n->gate_kind == FUSCO_GATE_NONE || empty || d_gate) && aligned16(d_gate) ? FUSCO_OK : FUSCO_ERR_INVALID_ARG;
}

// Norms' gradients: one chunk per thread where the row allows it (up to 1024 threads), and as many workgroups as the compute units hold at
// 16 waves each, every one of which leaves a row of partial sums per parameter.  Measured with 256 / 512 / 1024 workgroups, us: with an
// fp32 stream 8192 x 7168 231 / 241 / 258, 16384 x 4096 271 / 236 / 243, 32768 x 2048 335 / 236 / 247; bf16 16384 x 4096 214 / 174 / 183, 32768 x 2048 298 / 193 / 178.
int grad_cpt(int chunks) { return chunks <= 1024 ? 1 : 4; }
int norm_groups(int N, int H)
{
    const int waves = (int)row_threads(H / kEight, grad_cpt(H / kEight)) / kWave, each = 16 / waves;
    const int groups = kCus * (each > 4 ? 4 : each);
    return N < groups ? (N < 1 ? 1 : N) : groups;
}

template <bool AFTER>
int launch_norm(const fusco_norm *n, const NormArgs &a, hipStream_t s)
{
    const int cpt = row_cpt(a.chunks, n->N < 1024);
    const dim3 grid((unsigned)n->N), block(row_threads(a.chunks, cpt));
    with_types(n, AFTER ? 8 : 4, [&](auto st, auto bl, auto past) {
        with_cpt(cpt, [&](auto c) { hipLaunchKernelGGL((norm_kernel<decltype(st)::value, decltype(bl)::value, decltype(c)::value, decltype(past)::value, AFTER>), grid, block, 0, s, a); });
    });
    return launch_status();
}

template <bool AFTER, bool NEXT, bool CHANNEL>
void launch_norm_grad(const fusco_norm *n, const NormGradArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)norm_groups(n->N, n->H)), block(row_threads(a.chunks, grad_cpt(a.chunks)));
    with_types(n, (NEXT ? 4 : 0) + (AFTER ? 4 : 0) + 4, [&](auto st, auto bl, auto past) {
        constexpr bool kS = decltype(st)::value, kB = decltype(bl)::value, kPast = decltype(past)::value;
        if (grad_cpt(a.chunks) == 1) hipLaunchKernelGGL((norm_grad_kernel<kS, kB, 1, kPast, AFTER, NEXT, CHANNEL>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((norm_grad_kernel<kS, kB, 4, kPast, AFTER, NEXT, CHANNEL>), grid, block, 0, s, a);
    });
}

void launch_norm_join(const fusco_norm *n, const NormGradArgs &a, float *first, float *second, float *third, hipStream_t s)
{
    hipLaunchKernelGGL(norm_join_kernel, dim3((unsigned)((n->H + kJoinCols - 1) / kJoinCols), (unsigned)a.sums), dim3(kJoinThreads), 0, s, a.partial, norm_groups(n->N, n->H), a.sums,
                       n->H, first, second, third);
}

// ---- routing

int route_check(const fusco_router *R)
{
    if (!R || R->N < 0 || R->E < 1 || R->E > FUSCO_MAX_E || R->k < 1 || R->k > FUSCO_MAX_K || R->k > R->E || (int64_t)R->N * R->k >= (int64_t)1 << 31) return FUSCO_ERR_INVALID_ARG;
    if (R->logits_stride < R->E || !isfinite(R->scale)) return FUSCO_ERR_INVALID_ARG;
    if (!dtype_ok(R->logits_dtype) || (R->score != FUSCO_SCORE_SOFTMAX && R->score != FUSCO_SCORE_SIGMOID) || (R->renorm != 0 && R->renorm != 1)) return FUSCO_ERR_UNSUPPORTED;
    if (R->groups < 1 || R->groups > FUSCO_MAX_GROUPS || R->E % R->groups != 0 || R->keep_groups < 1 || R->keep_groups > R->groups) return FUSCO_ERR_INVALID_ARG;
    if (R->group_best < 1 || R->group_best > 2 || R->group_best > R->E / R->groups || R->k > R->keep_groups * (R->E / R->groups)) return FUSCO_ERR_INVALID_ARG;
    return FUSCO_OK;
}

RouteArgs route_args(const fusco_router *R, const void *d_logits)
{
    RouteArgs a = {};
    a.logits = (const char *)d_logits;
    a.stride = R->logits_stride;
    a.N = R->N; a.E = R->E; a.k = R->k;
    a.groups = R->groups; a.keep_groups = R->keep_groups; a.group_best = R->group_best; a.group_size = R->E / R->groups;
    a.group_magic = ((1 << 20) + a.group_size - 1) / a.group_size;
    a.bf16 = R->logits_dtype == FUSCO_BF16;
    a.sigmoid = R->score == FUSCO_SCORE_SIGMOID;
    a.renorm = R->renorm;
    a.scale = R->scale;
    return a;
}

// calls f(lanes per row, values per lane, threads per workgroup).  A wave per row where rows are few and long, for its latency (8 of E, sigmoids, 8 groups, us,
// 16 lanes / 64: 128 x 256 5.1 / 4.5, 128 x 512 7.1 / 5.2, 2048 x 256 5.7 / 5.3, 4096 x 256 5.8 / 7.0, 1024 x 128 4.3 / 5.1).  Else 16 lanes
// where every lane then has at most 32 values and k of the lanes' largest values say enough; single waves per workgroup for few rows, which
// spreads them over the compute units.
template <typename F>
void with_route_shape(const fusco_router *R, F f)
{
    const int by16 = (R->E + 15) / 16, by64 = (R->E + 63) / 64;
    auto go = [&](auto lanes, auto values) {
        if (R->N <= 4096) f(lanes, values, std::integral_constant<int, 64>());
        else f(lanes, values, std::integral_constant<int, 256>());
    };
    const std::integral_constant<int, 16> some;
    const std::integral_constant<int, 64> all;
    if (R->N <= 2048 && R->E > 128 && by64 <= 4) go(all, std::integral_constant<int, 4>());
    else if (R->N <= 2048 && R->E > 128 && by64 <= 8) go(all, std::integral_constant<int, 8>());
    else if (R->k <= 10 && by16 <= 4) go(some, std::integral_constant<int, 4>());
    else if (R->k <= 10 && by16 <= 8) go(some, std::integral_constant<int, 8>());
    else if (R->k <= 10 && by16 <= 16) go(some, std::integral_constant<int, 16>());
    else if (R->k <= 10 && by16 <= 32) go(some, std::integral_constant<int, 32>());
    else if (by64 <= 1) go(all, std::integral_constant<int, 1>());
    else if (by64 <= 2) go(all, std::integral_constant<int, 2>());
    else if (by64 <= 4) go(all, std::integral_constant<int, 4>());
    else if (by64 <= 8) go(all, std::integral_constant<int, 8>());
    else go(all, std::integral_constant<int, 16>());
}

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

}   // namespace

extern "C" {

int fusco_route(const fusco_router *R, const void *d_logits, const float *d_bias, int32_t *d_topk_idx, float *d_w, void *stream)
{
    const int rc = route_check(R);
    if (rc != FUSCO_OK) return rc;
    const bool empty = R->N == 0;
    if ((!empty && (!d_logits || !d_topk_idx || !d_w)) || !aligned(d_logits, R->logits_dtype == FUSCO_BF16 ? 2 : 4) || !aligned(d_bias, 4) || !aligned16(d_topk_idx) || !aligned16(d_w))
        return FUSCO_ERR_INVALID_ARG;
    if (empty) return FUSCO_OK;
    RouteArgs a = route_args(R, d_logits);
    a.bias = d_bias;
    a.chosen = d_topk_idx;
    a.w = d_w;
    with_route_shape(R, [&](auto lanes, auto values, auto threads) {
        constexpr int kLanes = decltype(lanes)::value, kValues = decltype(values)::value, kThreads = decltype(threads)::value, kRows = kThreads / kLanes;
        const dim3 grid((unsigned)((R->N + kRows - 1) / kRows));
        // Rows held in whole lanes spare the groups their way through LDS (8 groups, us, without / with: 32768 x 256 21.2 / 16.5, 32768 x 512 35.4 / 29.0);
        // 16 lanes without groups gain nothing worth an instance.
        if constexpr (kValues >= 4) {
            a.group_lanes = a.group_size % kValues == 0 && ((a.group_size / kValues) & (a.group_size / kValues - 1)) == 0 ? a.group_size / kValues : 0;
            const bool boundaries = aligned16(d_logits) && R->logits_stride * (a.bf16 ? 2 : 4) % 16 == 0 && aligned16(d_bias);
            if (boundaries && R->E == kLanes * kValues && (kLanes == 64 || (R->groups > 1 && a.group_lanes > 0))) {
                hipLaunchKernelGGL((route_kernel<kLanes, kValues, kThreads, true>), grid, dim3(kThreads), 0, (hipStream_t)stream, a);
                return;
            }
        }
        hipLaunchKernelGGL((route_kernel<kLanes, kValues, kThreads, false>), grid, dim3(kThreads), 0, (hipStream_t)stream, a);
    });
    return launch_status();
}

int fusco_route_backward(const fusco_router *R, const void *d_logits, const int32_t *d_topk_idx, const float *d_dw, void *d_dlogits, void *stream)
{
    const int rc = route_check(R);
    if (rc != FUSCO_OK) return rc;
    const bool empty = R->N == 0;
    if ((!empty && (!d_logits || !d_topk_idx || !d_dw || !d_dlogits)) || !aligned(d_logits, R->logits_dtype == FUSCO_BF16 ? 2 : 4) || !aligned16(d_topk_idx) || !aligned16(d_dw) ||
        !aligned16(d_dlogits))
        return FUSCO_ERR_INVALID_ARG;
    if (empty) return FUSCO_OK;
    RouteArgs a = route_args(R, d_logits);
    a.chosen = const_cast<int32_t *>(d_topk_idx);
    a.dw = d_dw;
    a.dlogits = (char *)d_dlogits;
    with_route_shape(R, [&](auto lanes, auto values, auto threads) {
        constexpr int kLanes = decltype(lanes)::value, kThreads = decltype(threads)::value, kRows = kThreads / kLanes;
        hipLaunchKernelGGL((route_grad_kernel<kLanes, decltype(values)::value, kThreads>), dim3((unsigned)((R->N + kRows - 1) / kRows)), dim3(kThreads), 0, (hipStream_t)stream, a);
    });
    return launch_status();
}

int fusco_norm_before(const fusco_norm *n, const void *d_x, const void *d_gain, void *d_out, void *stream)
{
    const int rc = norm_check(n);
    if (rc != FUSCO_OK) return rc;
    const void *const rows[] = {d_x, d_out}, *const shared[] = {d_gain};
    if (check_pointers(n->N == 0, rows, 2) != FUSCO_OK || check_pointers(false, shared, 1) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (n->N == 0) return FUSCO_OK;
    NormArgs a = {};
    a.r = (const char *)d_x; a.next_gain = (const char *)d_gain; a.next = (char *)d_out;
    a.N = n->N; a.chunks = n->H / kEight; a.gain_bf16 = n->gain_dtype == FUSCO_BF16;
    a.eps = n->eps; a.inv_h = 1.0f / n->H;
    return launch_norm<false>(n, a, (hipStream_t)stream);
}

int fusco_norm_after(const fusco_norm *n, const void *d_r, const void *d_y, const void *d_gain, const void *d_gate, void *d_out, const void *d_next_gain, void *d_next, void *stream)
{
    int rc = norm_check(n);
    if (rc == FUSCO_OK) rc = gate_check(n, d_gate);
    if (rc != FUSCO_OK) return rc;
    if (!isfinite(n->scale)) return FUSCO_ERR_INVALID_ARG;
    const void *const rows[] = {d_r, d_y, d_out}, *const shared[] = {d_gain};
    if (check_pointers(n->N == 0, rows, 3) != FUSCO_OK || check_pointers(false, shared, 1) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (!aligned16(d_next) || !aligned16(d_next_gain) || (d_next && !d_next_gain)) return FUSCO_ERR_INVALID_ARG;
    if (n->N == 0) return FUSCO_OK;
    NormArgs a = {};
    a.r = (const char *)d_r; a.y = (const char *)d_y; a.gain = (const char *)d_gain; a.gate = (const char *)d_gate; a.next_gain = (const char *)d_next_gain;
    a.out = (char *)d_out; a.next = (char *)d_next;
    a.N = n->N; a.chunks = n->H / kEight; a.gate_kind = n->gate_kind; a.gain_bf16 = n->gain_dtype == FUSCO_BF16;
    a.scale = n->scale; a.eps = n->eps; a.inv_h = 1.0f / n->H;
    return launch_norm<true>(n, a, (hipStream_t)stream);
}

size_t fusco_norm_scratch_bytes(int32_t N, int32_t H)
{
    if (N < 0 || H < 8 || H % 8 != 0 || H > FUSCO_MAX_NORM_H) return 0;
    return (size_t)norm_groups(N, H) * 3 * (size_t)H * 4;
}

int fusco_norm_before_backward(const fusco_norm *n, const void *d_dout, const void *d_x, const void *d_gain, const void *d_dres, void *d_dx, float *d_dgain, void *d_scratch,
                               size_t scratch_bytes, void *stream)
{
    const int rc = norm_check(n);
    if (rc != FUSCO_OK) return rc;
    const void *const rows[] = {d_dout, d_x, d_dx}, *const shared[] = {d_gain, d_dgain, d_scratch};
    if (check_pointers(n->N == 0, rows, 3) != FUSCO_OK || check_pointers(false, shared, 3) != FUSCO_OK || !aligned16(d_dres)) return FUSCO_ERR_INVALID_ARG;
    if (scratch_bytes < fusco_norm_scratch_bytes(n->N, n->H)) return FUSCO_ERR_WORKSPACE;
    NormGradArgs a = {};
    a.dout = (const char *)d_dres; a.dnext = (const char *)d_dout; a.out = (const char *)d_x; a.next_gain = (const char *)d_gain;
    a.dr = (char *)d_dx;
    a.partial = (float *)d_scratch;
    a.N = n->N; a.chunks = n->H / kEight; a.sums = 1; a.gain_bf16 = n->gain_dtype == FUSCO_BF16;
    a.scale = 1.0f; a.eps = n->eps; a.inv_h = 1.0f / n->H;
    launch_norm_grad<false, true, false>(n, a, (hipStream_t)stream);
    launch_norm_join(n, a, d_dgain, nullptr, nullptr, (hipStream_t)stream);
    return launch_status();
}

int fusco_norm_after_backward(const fusco_norm *n, const void *d_dout, const void *d_dnext, const void *d_y, const void *d_out, const void *d_gain, const void *d_gate,
                              const void *d_next_gain, void *d_dr, void *d_dy, float *d_dgain, float *d_dgate, float *d_dnext_gain, void *d_scratch, size_t scratch_bytes, void *stream)
{
    int rc = norm_check(n);
    if (rc == FUSCO_OK) rc = gate_check(n, d_gate);
    if (rc != FUSCO_OK) return rc;
    if (!isfinite(n->scale)) return FUSCO_ERR_INVALID_ARG;
    const bool empty = n->N == 0, channel = n->gate_kind == FUSCO_GATE_CHANNEL, token = n->gate_kind == FUSCO_GATE_TOKEN, next = d_dnext != nullptr || (empty && d_dnext_gain);
    const void *const rows[] = {d_y, d_dr, d_dy}, *const shared[] = {d_gain, d_dgain, d_scratch};
    if (check_pointers(empty, rows, 3) != FUSCO_OK || check_pointers(false, shared, 3) != FUSCO_OK || !aligned16(d_dout)) return FUSCO_ERR_INVALID_ARG;
    const void *const after[] = {d_out}, *const after_shared[] = {d_next_gain, d_dnext_gain}, *const gates[] = {d_dgate};
    if (next && (check_pointers(empty, after, 1) != FUSCO_OK || check_pointers(false, after_shared, 2) != FUSCO_OK || !aligned16(d_dnext))) return FUSCO_ERR_INVALID_ARG;
    if ((channel || token) && check_pointers(empty && token, gates, 1) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (!next && !d_dout && !empty) return FUSCO_ERR_INVALID_ARG;
    if (scratch_bytes < fusco_norm_scratch_bytes(n->N, n->H)) return FUSCO_ERR_WORKSPACE;
    NormGradArgs a = {};
    a.dout = (const char *)d_dout; a.dnext = (const char *)d_dnext; a.y = (const char *)d_y; a.out = (const char *)d_out;
    a.gain = (const char *)d_gain; a.gate = (const char *)d_gate; a.next_gain = (const char *)d_next_gain;
    a.dr = (char *)d_dr; a.dy = (char *)d_dy;
    a.dgate_token = token ? d_dgate : nullptr;
    a.partial = (float *)d_scratch;
    a.N = n->N; a.chunks = n->H / kEight; a.sums = 1 + (next ? 1 : 0) + (channel ? 1 : 0);
    a.gate_kind = n->gate_kind; a.gain_bf16 = n->gain_dtype == FUSCO_BF16;
    a.scale = n->scale; a.eps = n->eps; a.inv_h = 1.0f / n->H;
    hipStream_t s = (hipStream_t)stream;
    if (next && channel) launch_norm_grad<true, true, true>(n, a, s);
    else if (next) launch_norm_grad<true, true, false>(n, a, s);
    else if (channel) launch_norm_grad<true, false, true>(n, a, s);
    else launch_norm_grad<true, false, false>(n, a, s);
    if (next) launch_norm_join(n, a, d_dnext_gain, d_dgain, d_dgate, s);
    else launch_norm_join(n, a, d_dgain, d_dgate, nullptr, s);
    return launch_status();
}

int fusco_combine_backward(const fusco_layout *L, const void *d_y, int y_dtype, const float *d_w, const void *d_dout, int dout_dtype, void *d_dy, float *d_dw, int32_t H, void *stream)
{
    if (!layout_ok(L) || H < 8 || H % 8 != 0 || H > FUSCO_MAX_NORM_H) return FUSCO_ERR_INVALID_ARG;
    if (!dtype_ok(y_dtype) || !dtype_ok(dout_dtype)) return FUSCO_ERR_UNSUPPORTED;
    const void *const p[] = {d_y, d_w, d_dout, d_dy, d_dw};
    if (check_pointers(L->N == 0, p, 5) != FUSCO_OK) return FUSCO_ERR_INVALID_ARG;
    if (L->N == 0) return FUSCO_OK;
    const CombineGradArgs a = {L->pair_slot, (const char *)d_y, (const char *)d_dout, d_w, (char *)d_dy, d_dw, L->N, L->k, H / kEight};
    const int cpt = row_cpt(a.chunks, L->N < 1024);
    const dim3 grid((unsigned)L->N), block(row_threads(a.chunks, cpt));
    // tensors that the memory-side cache cannot hold are read past it: 16384 x 8 x 8 KiB 448 us / 455 through it, 1537 x 6 x 5760 B 25.9 / 20.9
    const int64_t y_bytes = y_dtype == FUSCO_BF16 ? 2 : 4, bytes = ((int64_t)2 * L->P * y_bytes + (int64_t)L->N * (dout_dtype == FUSCO_BF16 ? 2 : 4)) * H;
    with_cpt(cpt, [&](auto c) {
        constexpr int kCpt = decltype(c)::value, kJu = kCpt == 4 ? 2 : 4;
        auto go = [&](auto y, auto dout) {
            constexpr bool kY = decltype(y)::value, kD = decltype(dout)::value;
            if (bytes > kCacheBytes) hipLaunchKernelGGL((combine_grad_kernel<kY, kD, kCpt, kJu, true>), grid, block, 0, (hipStream_t)stream, a);
            else hipLaunchKernelGGL((combine_grad_kernel<kY, kD, kCpt, kJu, false>), grid, block, 0, (hipStream_t)stream, a);
        };
        if (y_dtype == FUSCO_BF16 && dout_dtype == FUSCO_BF16) go(std::true_type(), std::true_type());
        else if (y_dtype == FUSCO_BF16) go(std::true_type(), std::false_type());
        else if (dout_dtype == FUSCO_BF16) go(std::false_type(), std::true_type());
        else go(std::false_type(), std::false_type());
    });
    return launch_status();
}

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
    if (dw_dtype == FUSCO_F32) launch_product(product_kernel<kAcross, kAcross, 256, 4, 2, kStoreF32>, a, (hipStream_t)stream);
    else launch_product(product_kernel<kAcross, kAcross, 256, 4, 2, kStoreBf16>, a, (hipStream_t)stream);
    return launch_status();
}

int fusco_probe_experts_tile_rows(const fusco_layout *L, int which, int32_t outputs, int32_t sum)
{
    const bool gated = which == FUSCO_PROBE_PRODUCT_GATED, activation = which == FUSCO_PROBE_PRODUCT_INPUT_GRAD_ACTIVATION;
    if (!layout_ok(L) || which < 0 || which > FUSCO_PROBE_PRODUCT_INPUT_GRAD_ACTIVATION || !row_ok(outputs) || !row_ok(sum)) return FUSCO_ERR_INVALID_ARG;
    if (((gated || activation) && !row_ok(2 * outputs)) || !weights_ok((gated ? 2 : 1) * (int64_t)outputs, sum)) return FUSCO_ERR_INVALID_ARG;
    ProductArgs a = {};
    a.E = L->E; a.NA = outputs; a.C = sum;
    if (gated) return rows_per_tile<kAlongC, kStoreGated>(L, a);
    if (which == FUSCO_PROBE_PRODUCT_LINEAR) return rows_per_tile<kAlongC, kStoreBf16>(L, a);
    return activation ? rows_per_tile<kAcross, kStoreGatedGrad>(L, a) : rows_per_tile<kAcross, kStoreBf16>(L, a);
}

}   // extern "C"
