// What the kernels that work row by row share: eight elements of bf16 or fp32 at a time, sums over a wave and a workgroup.
#ifndef FUSCO_CSRC_ROWS_H
#define FUSCO_CSRC_ROWS_H

#include "common.h"

namespace {

constexpr int64_t kCacheBytes = (int64_t)256 << 20;   // the memory-side cache
constexpr int kEight = 8;   // elements per thread and access: 16 bytes of bf16, two times 16 bytes of fp32

typedef __bf16 rows_bf16x8 __attribute__((ext_vector_type(8)));
typedef float rows_f32x4 __attribute__((ext_vector_type(4)));

struct Eight {
    float v[kEight];
};

template <bool BF16>
struct RawEight;                     // as it lies in memory
template <>
struct RawEight<true> {
    rows_bf16x8 a;
};
template <>
struct RawEight<false> {
    rows_f32x4 a, b;
};

// PAST: past the caches, for tensors that they cannot hold (kCacheBytes); otherwise rows that were just written are read from there
template <bool BF16, bool PAST>
__device__ __forceinline__ RawEight<BF16> load_raw(const char *p, size_t element)
{
    RawEight<BF16> r;
    if constexpr (BF16) {
        const rows_bf16x8 *at = (const rows_bf16x8 *)(p + element * 2);
        r.a = PAST ? __builtin_nontemporal_load(at) : *at;
    } else {
        const rows_f32x4 *at = (const rows_f32x4 *)(p + element * 4);
        r.a = PAST ? __builtin_nontemporal_load(at) : at[0];
        r.b = PAST ? __builtin_nontemporal_load(at + 1) : at[1];
    }
    return r;
}

template <bool BF16>
__device__ __forceinline__ Eight wide(const RawEight<BF16> &r)
{
    Eight e;
#pragma unroll
    for (int i = 0; i < kEight; ++i) {
        if constexpr (BF16) e.v[i] = (float)r.a[i];
        else e.v[i] = i < 4 ? r.a[i & 3] : r.b[i & 3];
    }
    return e;
}

// eight parameters that every row uses again (cached): bf16 or fp32 by a value that is the same for the whole launch
__device__ __forceinline__ Eight load_shared(const char *p, bool bf16, size_t element)
{
    Eight e;
    if (bf16) {
        const rows_bf16x8 a = *(const rows_bf16x8 *)(p + element * 2);
#pragma unroll
        for (int i = 0; i < kEight; ++i) e.v[i] = (float)a[i];
    } else {
        const rows_f32x4 a = *(const rows_f32x4 *)(p + element * 4), b = *(const rows_f32x4 *)(p + element * 4 + 16);
#pragma unroll
        for (int i = 0; i < kEight; ++i) e.v[i] = i < 4 ? a[i & 3] : b[i & 3];
    }
    return e;
}

template <bool BF16>
__device__ __forceinline__ void store_eight(char *p, size_t element, const Eight &e)
{
    if constexpr (BF16) {
        rows_bf16x8 a;
#pragma unroll
        for (int i = 0; i < kEight; ++i) a[i] = (__bf16)e.v[i];
        __builtin_nontemporal_store(a, (rows_bf16x8 *)(p + element * 2));
    } else {
        rows_f32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = e.v[i];
            b[i] = e.v[i + 4];
        }
        __builtin_nontemporal_store(a, (rows_f32x4 *)(p + element * 4));
        __builtin_nontemporal_store(b, (rows_f32x4 *)(p + element * 4 + 16));
    }
}

// Values of the lanes `by` places on in the row of 16 lanes, round and round: no LDS, one instruction
template <int by>
__device__ __forceinline__ uint32_t turned(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x120 + by, 0xf, 0xf, true);
}

// Sums over 16 neighbouring lanes and over the wave, in all of their lanes
__device__ __forceinline__ float sixteen_sum(float v)
{
    v += __uint_as_float(turned<8>(__float_as_uint(v)));
    v += __uint_as_float(turned<4>(__float_as_uint(v)));
    v += __uint_as_float(turned<2>(__float_as_uint(v)));
    v += __uint_as_float(turned<1>(__float_as_uint(v)));
    return v;
}
__device__ __forceinline__ float wave_sum(float v)
{
    const int s = (int)__float_as_uint(sixteen_sum(v));
    const float a = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(s, 0)), b = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(s, 16));
    const float c = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(s, 32)), d = __uint_as_float((uint32_t)__builtin_amdgcn_readlane(s, 48));
    return (a + b) + (c + d);
}

constexpr int kMaxWaves = 16;   // of a workgroup

// Sums of n values over the workgroup, in every thread; `part` is LDS of n * kMaxWaves floats.  The same part may be used again once
// every thread has passed another barrier.
template <int n>
__device__ __forceinline__ void group_sums(float (&v)[n], float *part, int waves)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = wave_sum(v[i]);
    if (waves == 1) return;
    if (lane == 0) {
#pragma unroll
        for (int i = 0; i < n; ++i) part[i * kMaxWaves + wave] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < n; ++i) v[i] = sixteen_sum((lane & 15) < waves ? part[i * kMaxWaves + (lane & 15)] : 0.0f);
}

}   // namespace

#endif
