// Rows and weights in 8-bit floating point (e4m3: four significant bits from 2^-6 to 448, none infinite) with a scale per block, and back.
//
//     s = 2^n, n the smallest whole number with max |x| <= 448 * 2^n over the block        q = x / s rounded to e4m3 (nearest even)
//
// Powers of two, so that x / s is exact and q * s is a number of bf16 (four significant bits; from s = 2^-124 on, below which it may be smaller than the smallest of them): the only rounding is
// that to e4m3, and another scale between s / 2 and s would keep no more bits of any value that is not among the block's smallest.  A block is 128 columns of a row, or 128 x 128 of a matrix.
// Infinities and NaN become NaN and take no part in the maximum; a block of zeros has scale 1.  Scales are at least 2^-126.
//
// Bound by memory: x read once, q and scales written once, or the other way round; of a few rows by the launch (128 rows of 4096 4 us).
#ifndef FUSCO_CSRC_EIGHT_H
#define FUSCO_CSRC_EIGHT_H

#include "rows.h"

namespace {

constexpr int kBlockColumns = 128;
constexpr int kBlockLanes = kBlockColumns / kEight;   // lanes that hold one row of a block
constexpr int kEightThreads = 256;
constexpr int kEightGroups = kEightThreads / kBlockLanes;
constexpr int kEightEach = 2;                         // blocks per group of lanes

struct EightArgs {
    const char *in;
    char *out;
    float *scale;
    uint32_t blocks, per_row;          // of 128 columns, in all rows and in one
    int32_t columns, scale_stride;
    int32_t matrix_rows, scale_rows;   // rows of a matrix and of its scales, 0 where every row has scales of its own
};

// largest of the absolute values that are finite, as ordered integers; and over a row of 16 lanes
__device__ __forceinline__ uint32_t largest(const Eight &e)
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kEight; ++i) {
        const uint32_t bits = __float_as_uint(e.v[i]) & 0x7fffffffu;
        m = max(m, bits < 0x7f800000u ? bits : 0u);
    }
    return m;
}
__device__ __forceinline__ uint32_t sixteen_max(uint32_t v)
{
    v = max(v, turned<8>(v));
    v = max(v, turned<4>(v));
    v = max(v, turned<2>(v));
    return max(v, turned<1>(v));
}

// The exponent field of the scale: 448 is 1.75 * 2^8, and a significand above 1.75 takes the next power
__device__ __forceinline__ uint32_t scale_exponent(uint32_t largest)
{
    if (largest == 0) return 127;
    const int e = (int)((largest + 0x1fffffu) >> 23) - 8;
    return (uint32_t)(e < 1 ? 1 : e);
}

// e4m3 of eight values times 2^(127 - exponent)
__device__ __forceinline__ u32x2 to_eight(const Eight &e, uint32_t exponent)
{
    const float inverse = __uint_as_float((254u - exponent) << 23);
    float v[kEight];
#pragma unroll
    for (int i = 0; i < kEight; ++i) v[i] = (__float_as_uint(e.v[i]) & 0x7fffffffu) < 0x7f800000u ? e.v[i] * inverse : __uint_as_float(0x7fc00000u);
    u32x2 q;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i], v[4 * i + 1], 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(v[4 * i + 2], v[4 * i + 3], w, true);
        q[i] = (uint32_t)w;
    }
    return q;
}

__device__ __forceinline__ Eight from_eight(u32x2 q, float scale)
{
    Eight e;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)q[i], true);
        e.v[4 * i] = lo[0] * scale;
        e.v[4 * i + 1] = lo[1] * scale;
        e.v[4 * i + 2] = hi[0] * scale;
        e.v[4 * i + 3] = hi[1] * scale;
    }
    return e;
}

// STREAMED: past the caches
template <bool STREAMED>
__device__ __forceinline__ void put_eight(char *to, u32x2 q)
{
    if (STREAMED) __builtin_nontemporal_store(q, (u32x2 *)to);
    else *(u32x2 *)to = q;
}

// Block b of a row-major list of rows: its row, and the column of this lane's eight values; false where there are none
struct EightPlace {
    uint32_t row, block;
    int column;
    bool in;
    __device__ __forceinline__ EightPlace(const EightArgs &a, uint32_t b)
    {
        row = b / a.per_row;
        block = b - row * a.per_row;
        column = (int)block * kBlockColumns + (int)(threadIdx.x % kBlockLanes) * kEight;
        in = b < a.blocks && column < a.columns;
    }
    __device__ __forceinline__ size_t element(const EightArgs &a) const { return (size_t)row * a.columns + column; }
};

// Rows: 16 lanes per block, two blocks per group of lanes (bf16, one / two / four / eight, us: 2048 rows of 4096 6.6 / 6.4 / 6.9 / 7.8, 9222 of 1040 7.3 / 7.5 / 8.3 / 9.3, 131072 of
// 4096 284 / 271 / 278 / 278, 5.9 TB/s; back 269 / 265 / 273 / 280)
template <bool BF16, bool PAST, bool STREAMED>
__global__ __launch_bounds__(kEightThreads) void rows_to_eight_kernel(EightArgs a)
{
    const uint32_t first = blockIdx.x * (kEightGroups * kEightEach) + threadIdx.x / kBlockLanes;
    RawEight<BF16> raw[kEightEach];
#pragma unroll
    for (int i = 0; i < kEightEach; ++i) {
        const EightPlace at(a, first + i * kEightGroups);
        raw[i] = {};
        if (at.in) raw[i] = load_raw<BF16, PAST>(a.in, at.element(a));
    }
#pragma unroll
    for (int i = 0; i < kEightEach; ++i) {
        const EightPlace at(a, first + i * kEightGroups);
        const Eight e = wide<BF16>(raw[i]);
        const uint32_t exponent = scale_exponent(sixteen_max(largest(e)));
        if (!at.in) continue;
        put_eight<STREAMED>(a.out + at.element(a), to_eight(e, exponent));
        if (threadIdx.x % kBlockLanes == 0) a.scale[(size_t)at.row * a.scale_stride + at.block] = __uint_as_float(exponent << 23);
    }
}

// Matrices: a workgroup per block of 128 x 128, which it holds in registers, so that x is read once (64 fp32 matrices of 2048 x 1408 with 256 / 512 / 1024 threads 178 / 175 / 173 us, q
// past the caches 512 / 1024 165 / 171, 5.6 TB/s; of bf16 107 / 97 / 96 and 93 / 96; back to bf16 87, 6.3)
constexpr int kMatrixThreads = 512;
template <bool BF16, bool PAST, bool STREAMED>
__global__ __launch_bounds__(kMatrixThreads) void matrix_to_eight_kernel(EightArgs a)
{
    constexpr int kGroups = kMatrixThreads / kBlockLanes, kRows = kBlockColumns / kGroups;   // per thread
    __shared__ uint32_t part[kMatrixThreads / kWave];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t block = blockIdx.x % a.per_row, down = blockIdx.x / a.per_row, matrix = down / a.scale_rows;
    const int row0 = (int)(down - matrix * a.scale_rows) * kBlockColumns + (int)threadIdx.x / kBlockLanes;
    const int column = (int)block * kBlockColumns + (int)(threadIdx.x % kBlockLanes) * kEight;
    auto element = [&](int i) { return ((size_t)matrix * a.matrix_rows + row0 + i * kGroups) * a.columns + column; };
    auto in = [&](int i) { return column < a.columns && row0 + i * kGroups < a.matrix_rows; };
    RawEight<BF16> raw[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        raw[i] = {};
        if (in(i)) raw[i] = load_raw<BF16, PAST>(a.in, element(i));
    }
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) m = max(m, largest(wide<BF16>(raw[i])));
    m = sixteen_max(m);
    const uint32_t here = max(max((uint32_t)__builtin_amdgcn_readlane((int)m, 0), (uint32_t)__builtin_amdgcn_readlane((int)m, 16)),
                              max((uint32_t)__builtin_amdgcn_readlane((int)m, 32), (uint32_t)__builtin_amdgcn_readlane((int)m, 48)));
    if (lane == 0) part[wave] = here;
    __syncthreads();
    uint32_t all = part[0];
#pragma unroll
    for (int v = 1; v < kMatrixThreads / kWave; ++v) all = max(all, part[v]);
    const uint32_t exponent = scale_exponent(all);
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (in(i)) put_eight<STREAMED>(a.out + element(i), to_eight(wide<BF16>(raw[i]), exponent));
    if (threadIdx.x == 0) a.scale[(size_t)down * a.scale_stride + block] = __uint_as_float(exponent << 23);
}

// Back, for rows and matrices: values times their block's scale, whatever it is, rounded once
template <bool BF16>
__global__ __launch_bounds__(kEightThreads) void from_eight_kernel(EightArgs a)
{
    const uint32_t first = blockIdx.x * (kEightGroups * kEightEach) + threadIdx.x / kBlockLanes;
    u32x2 q[kEightEach];
    float scale[kEightEach];
#pragma unroll
    for (int i = 0; i < kEightEach; ++i) {
        const EightPlace at(a, first + i * kEightGroups);
        q[i] = u32x2{0, 0};
        scale[i] = 0.0f;
        if (!at.in) continue;
        uint32_t row = at.row;
        if (a.matrix_rows) {
            const uint32_t matrix = row / a.matrix_rows;
            row = matrix * a.scale_rows + (row - matrix * a.matrix_rows) / kBlockColumns;
        }
        q[i] = *(const u32x2 *)(a.in + at.element(a));
        scale[i] = a.scale[(size_t)row * a.scale_stride + at.block];
    }
#pragma unroll
    for (int i = 0; i < kEightEach; ++i) {
        const EightPlace at(a, first + i * kEightGroups);
        if (at.in) store_eight<BF16>(a.out, at.element(a), from_eight(q[i], scale[i]));
    }
}

}   // namespace

#endif
