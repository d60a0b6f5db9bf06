// Host side that the operators around the shuffle share (block.hip, eight.hip): checks of arguments, and which instance of the experts' products runs.
#ifndef FUSCO_CSRC_BLOCK_HOST_H
#define FUSCO_CSRC_BLOCK_HOST_H

#include "products.h"
#include <math.h>

namespace {

// rows of `elements` bf16 that the kernels take
inline bool row_ok(int32_t elements) { return elements > 0 && elements % 8 == 0 && (size_t)elements * 2 <= FUSCO_MAX_ROW_BYTES; }

// one expert's weights: loads inside them are addressed with 31 bits
inline bool weights_ok(int64_t rows, int64_t cols) { return rows * cols * 2 < (int64_t)kNowhere; }

inline int check_pointers(bool empty, const void *const *p, int n)
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
inline int few_waves(const ProductArgs &a) { return a.C >= 2048 ? 8 : 4; }

template <int WAVES, int STORE, bool EIGHT>
int launch_few(const fusco_layout *L, const ProductArgs &a, hipStream_t s)
{
    hipLaunchKernelGGL((few_rows_kernel<kFewF, WAVES, STORE, EIGHT>), dim3((unsigned)few_workgroups<STORE>(L, a)), dim3(WAVES * kWave), 0, s, a);
    return launch_status();
}

// Products whose tiles are rows of one expert.  From eight rows per expert on, the tile's height is the one whose rounds of tiles over the compute units
// take least: an expert's rows end inside a tile, two fifths of one on average, and a tile of 64, 128 or 256 rows takes 1 : 1.2 : 1.4 (fitted to
// 130 products of 8 to 128 experts with 8 to 1000 rows, where the choice is 3 % slower than the best one; by the mean number of rows alone, from 48 and from
// 96 on, it was 20 %).  Measured with 64 / 128 / 256, us: 128 experts of 4096 x (2 x 1280) gated, 8 rows 455 / 531 / 591, 64 rows 671 / 511 / 619, 128 rows 996 / 826 /
// 601; 16 of 2048 x 1408 with 128 rows, gradient of the pre-activations 32 / 48 / 61; 16 of 4096 x (2 x 1280) with 230 rows 224 / 185 / 127, its
// gradient of the pre-activations 120 / 90 / 136.  E4m3 keeps the rule (20 products measured, of evenly spread rows, the worst choice 8 % slower): 128 experts of
// 4096 x (2 x 1280) gated, 8 rows 232 / 248 / 283, 64 rows 268 / 267 / 294, 256 rows 806 / 513 / 392.
inline double tiles_of_rows(const fusco_layout *L, int rows) { return fmax((double)L->E, (double)L->P / rows + 0.4 * L->E); }
template <int STORE>
int tile_rows(const fusco_layout *L, const ProductArgs &a)
{
    const int units = STORE == kStoreGated ? kTileA / 2 : kTileA;
    const double across = (a.NA + units - 1) / units, takes[] = {1.0, 1.2, 1.4};
    int best = 256;
    double least = INFINITY;
    for (int i = 2; i >= 0; --i) {
        const int rows = 64 << i;
        const double tiles = tiles_of_rows(L, rows) * across;
        const double time = ceil(tiles / kCus) * takes[i];
        if (time < least) {
            least = time;
            best = rows;
        }
    }
    return best;
}

// Rows per tile, 16 for few_rows_kernel: below eight rows per expert (4 rows: 437 us, 441 in tiles of 64; 8 rows: 482 / 455), unless its
// workgroups for very many outputs come to more threads than a launch may have.  E4m3, 128 experts, 1 token of 8 choices 22 us, 42 in tiles of 64; 32 tokens
// 202 / 221, 64 tokens 232 / 228; 8 experts, 7 rows each 24 / 43.
template <int AMODE, int STORE>
int rows_per_tile(const fusco_layout *L, const ProductArgs &a)
{
    if (AMODE == kAlongC && L->P / L->E < 8 && few_workgroups<STORE>(L, a) * few_waves(a) * kWave <= UINT32_MAX) return 16;
    return tile_rows<STORE>(L, a);
}

// Input gradients: tiles of 64 rows and 128 outputs, where a compute unit has one of them at the most.  Their stages take 64 elements of the sum, three of them under way, where a stage of 256
// outputs has room for 32, and a single tile waits for its loads; sums keep their order.  Tiles are counted in two ways, by the mean as above and as if all experts had equally many rows (a few more
// than 64 make two tiles of each), and the larger count decides.  Through the activation / without it, us, 256 outputs / 128: 8 experts, 2048 x 768, 32 rows each, 48 tiles 29 / 21 and 24 / 19; 16 of 1040 x 528, 38 rows,
// 80 tiles 20 / 15 and 15.6 / 12.6; 8 of 4096 x 1280, 64 rows, 80 tiles 71 / 46 and 65 / 43; 64 of 1024 x 512, 32 rows, 256 tiles 28 / 20 and 24 / 17; 64 of 1024 x 256, 66 rows, 256 tiles
// 22 / 15 and 17 / 12.  More tiles than compute units: 88 of 336 x 256, 66 rows, 352 tiles 15.8 / 17.9 and 9.5 / 13.4; 40 of 1024 x 512, 66 rows, 320 tiles 22 / 23 and 15.8 / 18.3.  Segments so uneven
// that the count is too low lose less than one so counted gains: 120 of 1024 x 256, 66 and 14 rows in turn, 360 tiles counted as 246, 25 / 25 and 19.7 / 20.9.
inline bool narrow(const fusco_layout *L, const ProductArgs &a)
{
    const int64_t even = L->E * (((int64_t)L->P + 64 * (int64_t)L->E - 1) / (64 * (int64_t)L->E));
    return fmax((double)even, tiles_of_rows(L, 64)) * ((a.NA + 127) / 128) <= kCus;
}

// E4m3 in tiles of 64 rows: three stages in LDS instead of two, where filling up the last turn costs hardly a stage.  Gated / linear, us, two / three: 60 experts of 2880 x (2 x 1040) with 12 rows 112
// / 93 and 55 / 47; 256 of 7168 x (2 x 1024) with 9 664 / 614 and 361 / 358; 128 of 4096 x (2 x 1280) with 8 228 / 225; 64 of 2048 x 1408 with 20 linear 44.4 / 42.2; where a turn is filled up, sums of
// 512 19.4 / 22.2, of 1024 31.3 / 32.9, of 2048 27.3 / 26.6, 73.6 / 75.0 and 22.3 / 23.0.
inline bool three(const ProductArgs &a)
{
    const int stages = (a.C + 63) / 64;   // of 128 elements of one byte
    return 100 * ((stages + 2) / 3 * 3) <= 107 * ((stages + 1) / 2 * 2);
}

// Outputs of a tile (gated: units)
template <int AMODE, int STORE>
int outputs_per_tile(const fusco_layout *L, const ProductArgs &a)
{
    const int rows = rows_per_tile<AMODE, STORE>(L, a), whole = rows == 16 ? 16 * kFewF : AMODE == kAcross && rows == 64 && narrow(L, a) ? 128 : kTileA;
    return STORE == kStoreGated ? whole / 2 : whole;
}

template <int AMODE, int STORE, bool EIGHT = false>
int launch_by_rows(const fusco_layout *L, const ProductArgs &a, hipStream_t s)
{
    const int rows = rows_per_tile<AMODE, STORE>(L, a);
    if constexpr (AMODE == kAlongC) {
        if (rows == 16) return few_waves(a) == 8 ? launch_few<8, STORE, EIGHT>(L, a, s) : launch_few<4, STORE, EIGHT>(L, a, s);
    }
    if (rows == 256) launch_product(product_kernel<AMODE, kAlongC, 256, 4, 2, STORE, EIGHT>, a, s);
    else if (rows == 128) launch_product(product_kernel<AMODE, kAlongC, 128, 2, 2, STORE, EIGHT>, a, s);
    else if constexpr (AMODE == kAcross) launch_product(narrow(L, a) ? product_kernel<AMODE, kAlongC, 64, 1, 1, STORE, false, false, 128> : product_kernel<AMODE, kAlongC, 64, 2, 1, STORE>, a, s);
    else if constexpr (EIGHT) launch_product(three(a) ? product_kernel<AMODE, kAlongC, 64, 2, 1, STORE, true, false, kTileA, true> : product_kernel<AMODE, kAlongC, 64, 2, 1, STORE, true>, a, s);
    else launch_product(product_kernel<AMODE, kAlongC, 64, 2, 1, STORE>, a, s);
    return launch_status();
}

inline bool dtype_ok(int t) { return t == FUSCO_BF16 || t == FUSCO_F32; }

}   // namespace

#endif
