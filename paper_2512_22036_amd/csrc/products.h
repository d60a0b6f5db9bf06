// Products of the experts' rows with the experts' weights on the matrix cores.
//
// One kernel computes, expert by expert, D[a, b] = sum over c of A(a, c) * B(b, c) and stores it with a contiguous:
//   forward          a = weight row, b = token row,  c = column of both      (both operands are contiguous along c)
//   input gradient   a = weight column, b = token row, c = weight row        (A is contiguous along a)
//   weight gradient  a = weight column, b = weight row, c = token row        (both are contiguous along a and b)
// Rows lie expert-major (layout's exp_off); an expert's segment is cut into tiles of BB rows.
#ifndef FUSCO_CSRC_PRODUCTS_H
#define FUSCO_CSRC_PRODUCTS_H

#include "common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __attribute__((address_space(3))) char lds_byte;
typedef __attribute__((address_space(3))) bf16x4 lds_bf16x4;

constexpr int kCus = 256;              // compute units of an MI355X
constexpr int kTileThreads = 512;
constexpr int kTileA = 256;
constexpr uint32_t kNowhere = 0x7f000000u;   // byte offset past every buffer: such a load gives zeros

// How the tiles of one product lie in memory
enum { kAlongC, kAcross };             // operand contiguous along the summed dimension, or across it
enum { kStoreBf16, kStoreF32, kStoreGated, kStoreGatedGrad };

struct ProductArgs {
    const int32_t *exp_off;            // [E + 1]
    const char *rows;                  // B operand of forward and input gradient, [P, C]; A operand of the weight gradient, [P, NA]
    const char *other;                 // weights [E, ...]; B operand of the weight gradient, [P, NB]
    char *out;                         // [P, NA], or [E, NB, NA]
    char *pre;                         // gated forms: pre-activations [P, 2 * units] (written by forward where not null, read by the gradient)
    int32_t E, NA, NB, C;              // NA: outputs along a (gated forward: units); NB, C: weight gradient has NB outputs along b, others sum over C
};

// 1 / (1 + exp(-g)) from the hardware's exponential and reciprocal: off by some (|g| + 4) * 2^-23 of itself, below 2^-16 where it is not 0 (g > -87), and what comes
// of it is rounded to bf16, 2^-8
__device__ __forceinline__ float sigmoid(float g) { return __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }
__device__ __forceinline__ float silu(float g) { return g * sigmoid(g); }

// The bounds-checked view of `bytes` bytes from p: loads outside give zeros
__device__ __forceinline__ __amdgpu_buffer_rsrc_t view(const char *p, int64_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc((void *)p, 0, (int)(bytes < 0 ? 0 : bytes), 0x00020000);
}

// 16 bytes per lane straight to LDS: the wave's 64 chunks lie behind one another from `to` on
__device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t from, char *to, uint32_t offset, int uniform)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (lds_byte *)to, 16, (int)offset, uniform, 0, 0);
}

// One operand of a tile: where a stage of it (KC elements of the summed dimension) comes from and how it lies in LDS.  A fragment is 32 outputs
// by 16 elements of the sum, slice `ks` of the stage; lane l has output l % 32 and elements l / 32 * 8 + 0 .. 7.
//   OUT (operand A): the outputs of a fragment are dealt out so that the 16 results of a lane are neighbours: output i of the matrix
//   instruction is the fragment's row (i >> 2 & 1) * 16 + (i >> 3) * 4 + (i & 3).  Operand B keeps its order.
//   kAlongC: LDS rows of KC elements, the 16-byte chunk q of row r at place q ^ swizzle(r): the 16 lanes that are
//            served together (0-3, 12-15, 20-27 and so on) hit all banks in either order of the rows.
//   kAcross: LDS rows of W elements, one per c; windows of 32 outputs (64 bytes) of row c at place window ^ (c & 3): the transposing read of 32
//            lanes takes one window of each of four rows.
template <int MODE, int W, int KC, bool OUT>
struct Operand {
    static constexpr int kBytes = W * KC * 2;
    static constexpr int kRowLanes = KC / 8;   // kAlongC: lanes that load one row
    static constexpr int kChunks = kBytes / 16, kLoads = (kChunks + kTileThreads - 1) / kTileThreads;   // loads per thread and stage
    static constexpr int kLoadWaves = kChunks < kTileThreads ? kChunks / kWave : kTileThreads / kWave;  // waves that take part in a load
    const char *base;
    int64_t ld;            // bytes from row to row
    int64_t limit;         // kAlongC: readable bytes from base; kAcross: bytes that are missing from a whole last row
    int32_t c_size;        // elements (kAlongC) or rows (kAcross) of the summed dimension
    uint32_t at[kLoads];   // this thread's byte offsets
    int32_t chunk;         // kAlongC: the chunk of its row that this thread loads

    __device__ __forceinline__ void load(int stage, int i, char *lds, int wave) const
    {
        if (kLoadWaves < kTileThreads / kWave && wave >= kLoadWaves) return;
        if (MODE == kAlongC) {
            const bool in = stage * KC + chunk * 8 < c_size;
            to_lds(view(base, limit), lds + (i * kTileThreads + wave * kWave) * 16, in ? at[i] : kNowhere, stage * KC * 2);
        } else {
            const int left = min(max(c_size - stage * KC, 0), KC);
            const int bytes = __builtin_amdgcn_readfirstlane(max(left * (int)ld - (int)limit, 0));
            to_lds(__builtin_amdgcn_make_buffer_rsrc((void *)(base + (int64_t)stage * (int64_t)(KC * (int)ld)), 0, bytes, 0x00020000),
                   lds + (i * kTileThreads + wave * kWave) * 16, at[i], 0);
        }
    }

    // Load i of thread tid: which row of the stage's LDS (an output for kAlongC, a c for kAcross), and the first output (kAcross)
    static __device__ __forceinline__ int row_of(int i, int tid) { return MODE == kAlongC ? (i * kTileThreads + tid) / kRowLanes : (i * kTileThreads + tid) / (W / 8); }
    static __device__ __forceinline__ int swizzle(int row) { return KC == 64 ? row >> 1 & 7 : row >> 2 & 3; }
    static __device__ __forceinline__ int chunk_of(int tid) { return (tid & (kRowLanes - 1)) ^ swizzle(tid / kRowLanes); }
    static __device__ __forceinline__ int output_of(int i, int tid) { return ((tid & (W / 8 - 1)) ^ ((row_of(i, tid) & 3) << 2)) * 8; }

    // byte offset of this lane's part of the wave's first fragment, which begins at output `first`, a multiple of all its outputs
    static __device__ __forceinline__ uint32_t lane_at(int lane, int first)
    {
        if (MODE == kAlongC) {
            const int i = lane & 31, row = OUT ? (i >> 2 & 1) * 16 + (i >> 3) * 4 + (i & 3) : i;
            return (first + row) * (KC * 2) + (((lane >> 5) ^ swizzle(row)) << 4);
        }
        // a group of 16 lanes reads 4 outputs of 4 rows each, which the transposition gives to 16 outputs of one lane each
        const int c = (lane >> 5) * 8 + (lane >> 2 & 3), m = lane & 3, half = lane >> 4 & 1;
        const int output = OUT ? (m & 1) * 16 + (half * 2 + (m >> 1)) * 4 : half * 16 + m * 4;
        return c * (W * 2) + (((first >> 5) ^ (c & 3)) << 6) + output * 2;
    }

    static __device__ __forceinline__ bf16x8 fragment(const char *lds, uint32_t at, int f, int ks)
    {
        if (MODE == kAlongC) return *(const bf16x8 *)(lds + (at ^ (ks << 5)) + f * 32 * KC * 2);
        const char *p = lds + (at ^ (f << 6)) + ks * 16 * W * 2;
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)p);
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(p + 4 * W * 2));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// Everything a wave keeps over a tile.  Of the stages in LDS one is multiplied while the others are on their way.  Operands along c come in
// rows of 128 bytes, whole lines of the L2, which leaves room for two stages; rows of operands across c are long anyway, and four stages of
// half the length keep more in flight (8 experts of 16384 rows, 4096 x 2560, TF/s: two of 64 / four of 32: forward 1225 / 1190, input
// gradient 1103 / 1150, weight gradient 1206 / 1345).
template <int AMODE, int BMODE, int BB, int FA, int FB>
struct TileState {
    static constexpr int kStageC = AMODE == kAlongC ? 64 : 32, kSlices = kStageC / 16, kSlots = AMODE == kAlongC ? 2 : 4;
    typedef Operand<AMODE, kTileA, kStageC, true> A;
    typedef Operand<BMODE, BB, kStageC, false> B;
    static constexpr int kStageBytes = A::kBytes + B::kBytes, kLoads = A::kLoads;
    static_assert(A::kLoads >= B::kLoads, "the wider operand");
    A a;
    B b;
    uint32_t a_lane, b_lane;
    int wave;
    int stages, turn;

    // turns through the slots of a tile: a tile has whole turns, at least one, and what is missing is filled up with stages of zeros
    __device__ __forceinline__ int turns() const { return stages > 0 ? (stages + kSlots - 1) / kSlots : 1; }

    // stages are taken in the order turn, turn + 1, ..., turn - 1; past the last one loads fetch nothing, but they are made, so that
    // the number of loads behind a stage is always the same
    __device__ __forceinline__ int stage_of(int s) const
    {
        const int i = s + turn;
        return s >= stages ? stages : i >= stages ? i - stages : i;
    }
    __device__ __forceinline__ void load(int s, int i, char *slot) const
    {
        const int at = stage_of(s);
        if (i < A::kLoads) a.load(at, i, slot, wave);
        if (i < B::kLoads) b.load(at, i, slot + A::kBytes, wave);
    }
    // waits until at most the loads of `behind` stages and `more` stores are on their way and nothing is being read from LDS
    template <int behind, int more = 0>
    __device__ __forceinline__ void wait() const
    {
        constexpr int kAll = (A::kLoads + B::kLoads) * behind + more, kSome = A::kLoads * behind + more;
        static_assert(kAll < 64, "what the hardware counts");
        if (B::kLoadWaves == kTileThreads / kWave || wave < B::kLoadWaves) __builtin_amdgcn_s_waitcnt((kAll & 15) | (kAll >> 4) << 14 | 0x70);
        else __builtin_amdgcn_s_waitcnt((kSome & 15) | (kSome >> 4) << 14 | 0x70);
    }
};

// One stage, slice by slice: a slice is multiplied while the next one's fragments are read.  Before the last one comes the barrier behind which
// `cur` is free and `nxt` is whole: nxt's first fragments are read then, and the stage that will take cur's place is asked for.  Every
// matrix instruction is followed by what can be issued while it runs.
template <int FA, int FB>
struct Slice {
    bf16x8 a[FA], b[FB];
};

// what comes after matrix instruction m of FA * FB: fragment reads, those of b first, spread evenly
template <int FA, int FB, typename S>
__device__ __forceinline__ void read_after(const S &t, const char *slot, uint32_t a_at, uint32_t b_at, int ks, int m, Slice<FA, FB> &to)
{
    constexpr int kReads = FA + FB, kEach = (kReads + FA * FB - 1) / (FA * FB);
#pragma unroll
    for (int i = m * kEach; i < (m + 1) * kEach && i < kReads; ++i) {
        if (i < FB) to.b[i] = t.b.fragment(slot + S::A::kBytes, b_at, i, ks);
        else to.a[i - FB] = t.a.fragment(slot, a_at, i - FB, ks);
    }
}

template <bool ACTIVE, int STORES, int FA, int FB, typename S>
__device__ __forceinline__ void tile_stage(const S &t, char *cur, const char *nxt, int ask, Slice<FA, FB> (&x)[2], f32x16 (&acc)[FA][FB])
{
    uint32_t a_at = t.a_lane, b_at = t.b_lane;
    asm volatile("" : "+v"(a_at), "+v"(b_at));   // fragments' places are worked out where they are used, not kept in registers over the loop
#pragma unroll
    for (int ks = 0; ks < S::kSlices; ++ks) {
        const bool last = ks == S::kSlices - 1;
        if (last) {
            t.template wait<S::kSlots - 2, STORES>();
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_sched_barrier(0);
        }
        if (!ACTIVE && !last) continue;
        const int next = (ks + 1) % S::kSlices;
#pragma unroll
        for (int m = 0; m < FA * FB; ++m) {
            if (ACTIVE) acc[m / FB][m % FB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[ks % 2].a[m / FB], x[ks % 2].b[m % FB], acc[m / FB][m % FB], 0, 0, 0);
            read_after(t, last ? nxt : cur, a_at, b_at, next, m, x[next % 2]);
            if (last) {                  // loads behind the last matrix instructions
                constexpr int kEach = (S::kLoads + FA * FB - 1) / (FA * FB), kBegin = FA * FB - S::kLoads / kEach;
#pragma unroll
                for (int i = 0; i < kEach; ++i)
                    if (m >= kBegin) t.load(ask, (m - kBegin) * kEach + i, cur);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
}

// One turn through the slots, while stage ask, ask + 1, ... of this tile or the next are asked for.  STORES: stores that were issued after
// the loads of the stages that are under way, which the turn need not wait for.  The slots are arrays of their own: the compiler then
// knows that a fragment's read waits for its own slot's loads only.
template <bool ACTIVE, int STORES, int FA, int FB, typename S>
__device__ __forceinline__ void tile_turn(const S &t, char *slot0, char *slot1, char *slot2, char *slot3, int ask, Slice<FA, FB> (&x)[2], f32x16 (&acc)[FA][FB])
{
    if constexpr (S::kSlots == 2) {
        tile_stage<ACTIVE, STORES>(t, slot0, slot1, ask, x, acc);
        tile_stage<ACTIVE, 0>(t, slot1, slot0, ask + 1, x, acc);
    } else {
        tile_stage<ACTIVE, STORES>(t, slot0, slot1, ask, x, acc);
        tile_stage<ACTIVE, STORES>(t, slot1, slot2, ask + 1, x, acc);
        tile_stage<ACTIVE, STORES>(t, slot2, slot3, ask + 2, x, acc);
        tile_stage<ACTIVE, 0>(t, slot3, slot0, ask + 3, x, acc);
    }
}

typedef uint32_t words4 __attribute__((ext_vector_type(4)));

// Outputs of a wave.  Stores go through a bounds-checked view, so that their number is the same for every tile: what lies outside is dropped.
struct Target {
    __amdgpu_buffer_rsrc_t to;
    uint32_t ld;           // bytes from row to row
    __device__ __forceinline__ void open(char *p, int64_t row0, int64_t row_bytes, int64_t column_bytes, int rows)
    {
        ld = (uint32_t)row_bytes;
        to = view(p + row0 * row_bytes + column_bytes, rows > 0 ? rows * row_bytes - column_bytes : 0);
    }
    __device__ __forceinline__ void put8(const float *v, uint32_t offset) const
    {
        bf16x8 o;
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = (__bf16)v[q];
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(words4, o), to, (int)offset, 0, 0);
    }
};

// Part k of a lane's sixteen results as it is stored: four of fp32 or eight of bf16
template <bool F32>
__device__ __forceinline__ words4 packed(const f32x16 &v, int k)
{
    if constexpr (F32) {
        const f32x4 o = {v[4 * k], v[4 * k + 1], v[4 * k + 2], v[4 * k + 3]};
        return __builtin_bit_cast(words4, o);
    } else {
        bf16x8 o;
#pragma unroll
        for (int q = 0; q < 8; ++q) o[q] = (__bf16)v[8 * k + q];
        return __builtin_bit_cast(words4, o);
    }
}

// Transposes two values over two lanes of four neighbours: the lower keeps its first and gets the other's first as its second, the upper (upper != 0)
// gets the other's second as its first
template <int control>
__device__ __forceinline__ void exchange(int upper, words4 &first, words4 &second)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t of_first = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)first[i], control, 0xf, 0xf, true);
        const uint32_t of_second = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)second[i], control, 0xf, 0xf, true);
        first[i] = upper ? of_second : first[i];
        second[i] = upper ? second[i] : of_first;
    }
}

__device__ __forceinline__ void store4(char *out, int64_t element, f32x4 v)
{
    bf16x4 o;
#pragma unroll
    for (int q = 0; q < 4; ++q) o[q] = (__bf16)v[q];
    *(bf16x4 *)(out + element * 2) = o;
}

__device__ __forceinline__ bf16x8 load_fragment(__amdgpu_buffer_rsrc_t from, uint32_t offset)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(bf16x8, (words)__builtin_amdgcn_raw_buffer_load_b128(from, (int)offset, 0, 0));
}

// Exclusive prefix sums of the experts' tile counts, [E + 1] ints in LDS
__device__ __forceinline__ void tile_prefix(const int *__restrict__ exp_off, int E, int BB, int *__restrict__ prefix, int *__restrict__ part)
{
    static_assert(FUSCO_MAX_E <= 2 * kTileThreads, "two experts per thread");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, e = 2 * tid;
    const int o0 = exp_off[e < E ? e : E], o1 = exp_off[e + 1 < E ? e + 1 : E], o2 = exp_off[e + 2 < E ? e + 2 : E];
    const int n0 = (o1 - o0 + BB - 1) / BB, n1 = (o2 - o1 + BB - 1) / BB;
    int sum = n0 + n1;
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int other = __shfl_up(sum, d);
        if (lane >= d) sum += other;
    }
    if (lane == 63) part[wave] = sum;
    __syncthreads();
    int before = sum - n0 - n1;
    for (int w = 0; w < wave; ++w) before += part[w];
    if (e <= E) prefix[e] = before;
    if (e + 1 <= E) prefix[e + 1] = before + n0;
    if (E == 2 * kTileThreads && tid == kTileThreads - 1) prefix[E] = before + n0 + n1;
    __syncthreads();
}

// Tiles of BB token rows of one expert are taken in groups of four with all tiles along a: 32 neighbours (what one XCD's compute units
// work on at a time) then share 4 tiles of rows and 8 tiles of weights in their L2.
constexpr int kGroupB = 4;

// The i-th tile of a workgroup: in each round an XCD has 32 tiles that follow one another, and workgroups are dealt to the XCDs in turn.
__device__ __forceinline__ int tile_in_list(int i)
{
    return (i * kXcds + blockIdx.x % kXcds) * (kCus / kXcds) + blockIdx.x / kXcds;
}

// FA x FB fragments of 32 x 32 outputs per wave, kTileA / (32 * FA) waves along a
//
// Bound by the matrix instructions under the card's power limit where experts have many rows (8 experts of 16384 rows, 4096 x 2560: 1.21 to 1.29 PFLOP/s
// forward, 1.15 to 1.20 input gradient, 1.20 to 1.38 weight gradient; 128 uneven ones of 1024 rows gated 1.13), by the weights where they have few (128 experts
// with 32 rows, 4096 x (2 x 1280): 470 us, 5.7 TB/s).  Tiles of 256 x 256 read an operand half as often as those of 128; the list and the loads
// of the next tile under the last turn of one leave no gap between tiles (gated 2447 us with one, 2361 without).
template <int AMODE, int BMODE, int BB, int FA, int FB, int STORE>
__global__ __launch_bounds__(kTileThreads, 2) void product_kernel(ProductArgs p)
{
    typedef TileState<AMODE, BMODE, BB, FA, FB> State;
    constexpr int kWavesA = kTileA / (32 * FA), kWavesB = BB / (32 * FB);
    constexpr bool kByRows = BMODE == kAlongC;             // b is a token row (forward, input gradient), or a weight row
    constexpr bool kGated = STORE == kStoreGated;
    constexpr int kUnitsA = kGated ? kTileA / 2 : kTileA;  // outputs along a per tile: a gated tile holds both rows of a unit
    static_assert(kWavesA * kWavesB * kWave == kTileThreads, "eight waves");
    static_assert(!kGated || FA % 2 == 0, "gate and up rows of a unit in one wave");
    constexpr int kMore = State::kSlots == 4 ? State::kStageBytes : 16;
    __shared__ __align__(1024) char slot0[State::kStageBytes], slot1[State::kStageBytes], slot2[kMore], slot3[kMore];
    __shared__ int offsets[FUSCO_MAX_E + 1], prefix[kByRows ? FUSCO_MAX_E + 1 : 1];
    __shared__ int part[kTileThreads / kWave];

    const int tid = threadIdx.x, lane = tid & 63;
    for (int e = tid; e <= p.E; e += kTileThreads) offsets[e] = p.exp_off[e];
    __syncthreads();
    // Where a slot is written and read from is hidden from the compiler: as long as it cannot tell one place in a slot from another, it lets
    // reads wait for the loads to their slot; where it could, it would let them wait for all loads.
    int hidden = tid >> 6;
    asm volatile("" : "+v"(hidden));
    const int wave = __builtin_amdgcn_readfirstlane(hidden);
    const int wa = wave % kWavesA, wb = wave / kWavesA;
    const int tiles_a = (p.NA + kUnitsA - 1) / kUnitsA;
    const int tiles_b = kByRows ? 0 : (p.NB + BB - 1) / BB;
    int total;
    if (kByRows) {
        tile_prefix(offsets, p.E, BB, prefix, part);
        total = prefix[p.E] * tiles_a;
    } else {
        total = p.E * tiles_a * tiles_b;
    }

    State s;
    s.wave = wave;
    s.a_lane = State::A::lane_at(lane, wa * FA * 32);
    s.b_lane = State::B::lane_at(lane, wb * FB * 32);
    asm volatile("" : "+v"(s.a_lane), "+v"(s.b_lane));

    // the tile at hand
    int a0 = 0, a_left = 0, b_left = 0;
    int64_t row0 = 0;
    auto begin = [&](int t) {
        int tid = threadIdx.x;
        asm volatile("" : "+v"(tid));    // as in store
        const int lane = tid & 63;
        // which expert, which tiles
        int e, ta, tb, first, rows;
        {
            int at, in_e;
            if (kByRows) {
                int lo = 0, hi = p.E;   // the last expert whose first tile is not behind t
                while (hi - lo > 1) {
                    const int mid = (lo + hi) / 2;
                    if (prefix[mid] * tiles_a <= t) lo = mid;
                    else hi = mid;
                }
                e = __builtin_amdgcn_readfirstlane(lo);
                at = t - __builtin_amdgcn_readfirstlane(prefix[e]) * tiles_a;
                in_e = __builtin_amdgcn_readfirstlane(prefix[e + 1] - prefix[e]);
            } else {
                e = t / (tiles_a * tiles_b);
                at = t - e * tiles_a * tiles_b;
                in_e = tiles_b;
            }
            const int g = at / (kGroupB * tiles_a), wide = in_e - g * kGroupB < kGroupB ? in_e - g * kGroupB : kGroupB;
            at -= g * kGroupB * tiles_a;
            ta = at / wide;
            tb = g * kGroupB + at % wide;
            first = __builtin_amdgcn_readfirstlane(offsets[e]);
            rows = __builtin_amdgcn_readfirstlane(offsets[e + 1]) - first;
        }
        a0 = ta * kUnitsA;
        const int b0 = tb * BB;
        b_left = (kByRows ? rows : p.NB) - b0;
        a_left = p.NA - a0;
        row0 = kByRows ? (int64_t)first + b0 : (int64_t)e * p.NB + b0;
        // operand A
        if (AMODE == kAlongC) {   // forward: weight rows
            const int rows_e = kGated ? 2 * p.NA : p.NA;
            s.a.ld = (int64_t)p.C * 2;
            s.a.base = p.other + ((int64_t)e * rows_e + a0) * s.a.ld;
            s.a.limit = (rows_e - a0) * s.a.ld;
            s.a.c_size = p.C;
            s.a.chunk = State::A::chunk_of(tid);
#pragma unroll
            for (int j = 0; j < State::A::kLoads; ++j) {
                const int r = State::A::row_of(j, tid);
                int unit = r, up = 0;
                if (kGated) {   // a wave's rows: FA * 16 gate rows, then the up rows of the same units
                    unit = r / (32 * FA) * (16 * FA) + r % (16 * FA);
                    up = r / (16 * FA) % 2;
                }
                s.a.at[j] = unit < a_left ? (uint32_t)((unit + up * p.NA) * s.a.ld) + (s.a.chunk << 4) : kNowhere;
            }
        } else {
            s.a.ld = (int64_t)p.NA * 2;
            s.a.limit = (int64_t)a0 * 2;
            s.a.c_size = kByRows ? p.C : rows;
            s.a.base = (kByRows ? p.other + (int64_t)e * p.C * s.a.ld : p.rows + first * s.a.ld) + s.a.limit;
#pragma unroll
            for (int j = 0; j < State::A::kLoads; ++j) {
                const int output = State::A::output_of(j, tid);
                s.a.at[j] = output < a_left ? (uint32_t)(State::A::row_of(j, tid) * s.a.ld) + output * 2 : kNowhere;
            }
        }
        // operand B
        if (BMODE == kAlongC) {
            s.b.ld = (int64_t)p.C * 2;
            s.b.base = p.rows + ((int64_t)first + b0) * s.b.ld;
            s.b.limit = (b_left < BB ? b_left : BB) * s.b.ld;
            s.b.c_size = p.C;
            s.b.chunk = State::B::chunk_of(tid);
#pragma unroll
            for (int j = 0; j < State::B::kLoads; ++j) s.b.at[j] = (uint32_t)(State::B::row_of(j, tid) * s.b.ld) + (s.b.chunk << 4);
            s.stages = (p.C + State::kStageC - 1) / State::kStageC;
        } else {
            s.b.ld = (int64_t)p.NB * 2;
            s.b.limit = (int64_t)b0 * 2;
            s.b.base = p.other + first * s.b.ld + s.b.limit;
            s.b.c_size = rows;
#pragma unroll
            for (int j = 0; j < State::B::kLoads; ++j) {
                const int output = State::B::output_of(j, tid);
                s.b.at[j] = output < b_left ? (uint32_t)(State::B::row_of(j, tid) * s.b.ld) + output * 2 : kNowhere;
            }
            s.stages = (rows + State::kStageC - 1) / State::kStageC;
        }
        // tiles begin at different stages, as in few_rows_kernel; neighbours along a, which share rows in an L2, at the same one
        s.turn = s.stages > 0 ? (int)(((uint32_t)(e * 64 + ta / 8) * 2654435761u >> 12) % (uint32_t)s.stages) : 0;
    };

    // Lane l holds, of fragment (f, j), the outputs a = 32 * f + l / 32 * 16 + 0 .. 15 of b = 32 * j + l % 32.
    constexpr int kOutA = kGated ? FA / 2 : FA;
    f32x16 acc[FA][FB];
    auto store = [&](int a0, int a_left, int b_left, int64_t row0) {
        constexpr int kSize = STORE == kStoreF32 ? 4 : 2;
        const int rows = b_left < BB ? b_left : BB;
        Target out, pre;
        out.open(p.out, row0, (int64_t)p.NA * (STORE == kStoreGatedGrad ? 2 : 1) * kSize, (int64_t)a0 * kSize, rows);
        if ((kGated && p.pre) || STORE == kStoreGatedGrad) pre.open(p.pre, row0, (int64_t)p.NA * 2 * kSize, (int64_t)a0 * kSize, rows);
        const uint32_t second = (uint32_t)p.NA * kSize;
        int lane = tid & 63;
        asm volatile("" : "+v"(lane));   // places are worked out here, not kept in registers over the sums
#pragma unroll
        for (int j = 0; j < FB; ++j) {
            const int b = (wb * FB + j) * 32 + (lane & 31);
            bf16x8 gates[STORE == kStoreGatedGrad ? kOutA : 1][2], ups[STORE == kStoreGatedGrad ? kOutA : 1][2];
            if constexpr (STORE == kStoreGatedGrad) {   // all pre-activations at once, not one after the other
#pragma unroll
                for (int f = 0; f < kOutA; ++f)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int a = (wa * kOutA + f) * 32 + (lane >> 5) * 16 + h * 8;
                        const uint32_t at = a < a_left && b < b_left ? b * out.ld + a * kSize : kNowhere;
                        gates[f][h] = load_fragment(pre.to, at);
                        ups[f][h] = load_fragment(pre.to, at + second);
                    }
            }
#pragma unroll
            for (int f = 0; f < kOutA; ++f) {
                if constexpr (STORE == kStoreF32 || STORE == kStoreBf16) {
                    // 64 (fp32) or 32 bytes of a lane's row are dealt out to as many neighbours, so that a store meets whole pieces of a row
                    constexpr int kParts = STORE == kStoreF32 ? 4 : 2;
                    words4 v[kParts];
#pragma unroll
                    for (int k = 0; k < kParts; ++k) v[k] = packed<STORE == kStoreF32>(acc[f][j], k);
#pragma unroll
                    for (int k = 0; k < kParts; k += 2) exchange<0xb1>(lane & 1, v[k], v[k + 1]);
                    if constexpr (kParts == 4) {
                        exchange<0x4e>(lane & 2, v[0], v[2]);
                        exchange<0x4e>(lane & 2, v[1], v[3]);
                    }
                    const int a = (wa * kOutA + f) * 32 + (lane >> 5) * 16 + (lane & (kParts - 1)) * (16 / kParts);
#pragma unroll
                    for (int k = 0; k < kParts; ++k) {
                        const int row = (wb * FB + j) * 32 + (lane & 32 - kParts) + k;
                        __builtin_amdgcn_raw_buffer_store_b128(v[k], out.to, (int)(a < a_left && row < b_left ? row * out.ld + a * kSize : kNowhere), 0, 0);
                    }
                    continue;
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int a = (wa * kOutA + f) * 32 + (lane >> 5) * 16 + h * 8;
                    const bool in = a < a_left && b < b_left;
                    const uint32_t at = in ? b * out.ld + a * kSize : kNowhere;
                    float v[8];
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] = acc[f][j][h * 8 + q];
                    if (STORE == kStoreGated) {
                        float up[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) up[q] = acc[f + FA / 2][j][h * 8 + q];
                        if (p.pre) {
                            const uint32_t to = in ? b * pre.ld + a * kSize : kNowhere;
                            pre.put8(v, to);
                            pre.put8(up, to + second);
                        }
#pragma unroll
                        for (int q = 0; q < 8; ++q) v[q] = silu(v[q]) * up[q];
                        out.put8(v, at);
                    } else {
                        float dup[8];
#pragma unroll
                        for (int q = 0; q < 8; ++q) {
                            const float g = (float)gates[f][h][q], sig = sigmoid(g);
                            dup[q] = v[q] * g * sig;
                            v[q] = v[q] * (float)ups[f][h][q] * sig * (1.0f + g * (1.0f - sig));
                        }
                        out.put8(v, at);
                        out.put8(dup, at + second);
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    auto clear = [&] {
#pragma unroll
        for (int f = 0; f < FA; ++f)
#pragma unroll
            for (int j = 0; j < FB; ++j)
#pragma unroll
                for (int q = 0; q < 16; ++q) acc[f][j][q] = 0.0f;
    };
    // stores of one tile and wave; the activation's gradient waits for loads in between and counts as none
    constexpr int kStores = STORE == kStoreGatedGrad ? 0 : FB * kOutA * (STORE == kStoreF32 ? 4 : 2);

    // Tiles follow one another without a pause: the last turn of one asks for the first stages of the next, whose first fragments it reads.
    int t = tile_in_list(0);
    if (t >= total) return;
    clear();
    begin(t);
#pragma unroll
    for (int i = 0; i < State::kLoads; ++i) s.load(0, i, slot0);
#pragma unroll
    for (int i = 0; i < State::kLoads; ++i) s.load(1, i, slot1);
    if constexpr (State::kSlots == 4) {
#pragma unroll
        for (int i = 0; i < State::kLoads; ++i) s.load(2, i, slot2);
#pragma unroll
        for (int i = 0; i < State::kLoads; ++i) s.load(3, i, slot3);
    }
    __builtin_amdgcn_sched_barrier(0);
    store(0, 0, 0, 0);   // nothing, but the stores are counted
    s.template wait<State::kSlots - 1, kStores>();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    Slice<FA, FB> x[2];
#pragma unroll
    for (int m = 0; m < FA * FB; ++m) read_after(s, slot0, s.a_lane, s.b_lane, 0, m, x[0]);
    for (int i = 1;; ++i) {
        const int now_a0 = a0, now_a = a_left, now_b = b_left;
        const int64_t now_row = row0;
        const bool active = wb * FB * 32 < b_left;   // or all of this wave's rows lie past the segment: loads and barriers only
        const int turns = s.turns();
        int ask = State::kSlots;
        if (turns > 1) {
            if (active) {
                tile_turn<true, kStores>(s, slot0, slot1, slot2, slot3, ask, x, acc);
                for (ask += State::kSlots; ask < turns * State::kSlots; ask += State::kSlots) tile_turn<true, 0>(s, slot0, slot1, slot2, slot3, ask, x, acc);
            } else {
                tile_turn<false, kStores>(s, slot0, slot1, slot2, slot3, ask, x, acc);
                for (ask += State::kSlots; ask < turns * State::kSlots; ask += State::kSlots) tile_turn<false, 0>(s, slot0, slot1, slot2, slot3, ask, x, acc);
            }
        }
        t = tile_in_list(i);
        const bool more = t < total;   // later tiles of this workgroup lie behind it
        if (more) {
            begin(t);
        } else {
            s.stages = s.a.c_size = s.b.c_size = 0;
        }
        if (active) tile_turn<true, 0>(s, slot0, slot1, slot2, slot3, 0, x, acc);
        else tile_turn<false, 0>(s, slot0, slot1, slot2, slot3, 0, x, acc);
        store(now_a0, now_a, now_b, now_row);
        if (!more) break;
        clear();
    }
    __builtin_amdgcn_s_waitcnt(0x0070);   // nothing may be on its way to LDS when the workgroup gives it up
}

// ---- Few rows per expert: bound by the weights, every one of which is read once for a handful of rows.
//
// A block is 16 * F weight rows (gated: 16 * F / 2 units with their gate and up rows) of one expert for up to 16 of its token rows.  The
// WAVES waves of a workgroup share the summed dimension: wave v has the pieces v, v + WAVES, ... of 64 elements, and the waves' sums are
// added up in LDS in the order of the waves.  Fragments go straight from memory to registers, a piece ahead of their use: many waves keep
// enough bytes in flight, and deeper prefetch costs waves (measured 6.1 TB/s with one piece ahead, 5.8 with three).  One block per
// workgroup: with two to eight neighbouring blocks, the next one's first piece under way while the sums are added up, 5.8 to 5.6 TB/s.
// Measured, 128 experts of 4096 x (2 x 1280), 32 tokens with 8 experts each: 383 us, 6.14 TB/s of weights; a single token 36 us, 4.7 TB/s.
constexpr int kPiece = 64;   // elements

template <int WAVES>
struct FewTile {
    int e, first, rows;

    // Which rows of which expert: the tiles of 16 rows of all experts lie one after the other.  False if there are fewer tiles.
    __device__ __forceinline__ bool find(const int32_t *__restrict__ exp_off, int E, int tile, int *__restrict__ part)
    {
        // every thread counts the tiles of a few neighbouring experts; the one whose range holds `tile` says so
        constexpr int kThreads = WAVES * kWave, kEach = FUSCO_MAX_E / kThreads;
        const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
        int at[kEach + 1];
#pragma unroll
        for (int i = 0; i <= kEach; ++i) {
            const int x = tid * kEach + i;
            at[i] = exp_off[x < E ? x : E];
        }
        int own = 0;
#pragma unroll
        for (int i = 0; i < kEach; ++i) own += (at[i + 1] - at[i] + 15) / 16;
        int sum = own;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int other = __shfl_up(sum, d);
            if (lane >= d) sum += other;
        }
        if (lane == 63) part[wave] = sum;
        if (tid == 0) part[WAVES] = -1;
        __syncthreads();
        int before = sum - own;
        for (int w = 0; w < wave; ++w) before += part[w];
        if (tile >= before && tile < before + own) {
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                const int n = (at[i + 1] - at[i] + 15) / 16;
                if (tile >= before && tile < before + n) {
                    part[WAVES] = tid * kEach + i;
                    part[WAVES + 1] = at[i] + (tile - before) * 16;
                    part[WAVES + 2] = at[i + 1];
                }
                before += n;
            }
        }
        __syncthreads();
        e = __builtin_amdgcn_readfirstlane(part[WAVES]);
        first = __builtin_amdgcn_readfirstlane(part[WAVES + 1]);
        rows = __builtin_amdgcn_readfirstlane(part[WAVES + 2]) - first;
        rows = rows < 16 ? rows : 16;
        return e >= 0;
    }
};

template <int F, int WAVES, int STORE>
__global__ __launch_bounds__(WAVES *kWave) void few_rows_kernel(ProductArgs p)
{
    constexpr bool kGated = STORE == kStoreGated;
    constexpr int kUnits = kGated ? 8 * F : 16 * F;       // outputs along a of a block
    constexpr int kOut = kGated ? F / 2 : F;
    __shared__ int part[WAVES + 3];
    __shared__ f32x4 sums[WAVES][F][kWave];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int blocks = (p.NA + kUnits - 1) / kUnits;
    const int tile = blockIdx.x / blocks, block = blockIdx.x - tile * blocks, a0 = block * kUnits;
    FewTile<WAVES> at;
    if (!at.find(p.exp_off, p.E, tile, part)) return;

    const int64_t ld = (int64_t)p.C * 2;
    const int rows_e = kGated ? 2 * p.NA : p.NA;
    const int pieces = (p.C + kPiece - 1) / kPiece, mine = (pieces - wave + WAVES - 1) / WAVES;
    const __amdgpu_buffer_rsrc_t vx = view(p.rows + at.first * ld, at.rows * ld);
    const uint32_t in_row = (lane >> 4) * 16, x_at = (uint32_t)((lane & 15) * ld) + in_row;
    const __amdgpu_buffer_rsrc_t vw = view(p.other + ((int64_t)at.e * rows_e + a0) * ld, (rows_e - a0) * ld);
    uint32_t w_at[F];
#pragma unroll
    for (int f = 0; f < F; ++f) {
        const int unit = (kGated ? f % kOut : f) * 16 + (lane & 15);
        w_at[f] = a0 + unit < p.NA ? (uint32_t)((unit + (kGated && f >= kOut ? p.NA : 0)) * ld) + in_row : kNowhere;
    }
    // Blocks begin at different pieces: rows whose size is a multiple of a large power of two lie on the same memory channels piece by
    // piece (rows of 8 KiB: 6.1 TB/s, 5.0 without).  The order of a sum depends on the weights' place alone, not on the batch.
    const int turn = mine > 0 ? (int)(((uint32_t)(block + at.e * blocks) * 2654435761u >> 12) % (uint32_t)mine) : 0;
    bf16x8 w[F][2], x[2];
    auto load = [&](int i) {
        int j = i + turn;
        j = j >= mine ? j - mine : j;
        const int c0 = (wave + j * WAVES) * kPiece;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            const int c = c0 + ks * 32;
            const bool in = i < mine && c + (lane >> 4) * 8 < p.C;   // past the end: zeros, and no traffic
#pragma unroll
            for (int f = 0; f < F; ++f) w[f][ks] = load_fragment(vw, in ? w_at[f] + c * 2 : kNowhere);
            x[ks] = load_fragment(vx, in ? x_at + c * 2 : kNowhere);
        }
    };
    load(0);
    f32x4 acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0; i < mine; ++i) {
        bf16x8 wn[F][2], xn[2];
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
            for (int f = 0; f < F; ++f) wn[f][ks] = w[f][ks];
            xn[ks] = x[ks];
        }
        if (i + 1 < mine) load(i + 1);
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int f = 0; f < F; ++f) acc[f] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wn[f][ks], xn[ks], acc[f], 0, 0, 0);
    }
#pragma unroll
    for (int f = 0; f < F; ++f) sums[wave][f][lane] = acc[f];
    __syncthreads();
    for (int f = wave; f < kOut; f += WAVES) {
        const int b = lane & 15, a = a0 + f * 16 + (lane >> 4) * 4;
        f32x4 v = sums[0][f][lane], up = v;
#pragma unroll
        for (int s = 1; s < WAVES; ++s) v += sums[s][f][lane];
        if (kGated) {
            up = sums[0][f + kOut][lane];
#pragma unroll
            for (int s = 1; s < WAVES; ++s) up += sums[s][f + kOut][lane];
        }
        if (b >= at.rows || a >= p.NA) continue;
        const int64_t row = (int64_t)at.first + b;
        if (kGated) {
            f32x4 h;
#pragma unroll
            for (int q = 0; q < 4; ++q) h[q] = silu(v[q]) * up[q];
            store4(p.out, row * p.NA + a, h);
            if (p.pre) {
                store4(p.pre, row * 2 * p.NA + a, v);
                store4(p.pre, (row * 2 + 1) * p.NA + a, up);
            }
        } else {
            store4(p.out, row * p.NA + a, v);
        }
    }
}

}   // namespace

#endif
