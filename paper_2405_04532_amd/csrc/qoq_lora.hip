// Low-rank adapters of many requests beside a projection that they share:
//   out[m] = base[m] + s_a (x[m] A_a^T) B_a^T,   a = the adapter of row m;   out[m] = base[m] where it has none
// with A_a [r, K], B_a [N, r] FP16, sums in FP32, one rounding at the end.
//
// Plan.  Which rows belong to which adapter is the same for every projection of a step, so it is worked out once: the rows ordered by
// adapter, and tiles of up to tile_rows(M) of them that share one, so that an adapter's matrices are read once for a tile.
//
// The first launch forms h = x A^T, tile by tile, K cut over workgroups.  h enters the second product as pairs of FP16 numbers hi + lo of h
// scaled by a power of two for each row (and 64 ranks): within 2^-22 of h, or 2^-39 of the row's largest; hi B^T + lo B^T is one product whose k
// runs over the pairs, B's columns taken twice (and, where that gives NaN, done again with hi alone: an infinity of B).  Where few sums meet, the
// launch of the second product adds the slices of K up and forms the pairs itself; else that is a launch between.  (Joined by the last workgroup of a tile, past the caches, a slice of 4096 x 64 sums took 3 us.)
//
// Many rows are bound by the trips to memory that a wave makes one after the other: 4096 rows of 64 ranks beside 28672 x 8192 take 172 us, 34 in the first
// launch (2.0 TB/s: one workgroup to a compute unit) and 138 in the second (470 MB in and out, 3.4 TB/s).  It is not the bytes that the second waits for (136
// took 127 without base, 134 without the stores), nor arithmetic (matrix unit 0.10 of the cycles, vector unit 0.13): of two waves to a SIMD, none has the next
// block's operands in flight while it multiplies and stores.  Few rows are launches: 64 of 16 ranks beside 6144 x 4096 8.5 us, 4.0 + 5.0 by a profiler.  More
// than 64 ranks: the pairs are read again for every 64 channels, by one wave to a SIMD where rows are many (2048 rows beside 8192 x 8192: 56 ranks 41 us,
// 128 89, 256 166; 64 rows of 256 ranks beside 6144 x 4096 23.6).  (In one launch, every workgroup forming h by itself, one row of 4096 x 4096 and 16 ranks took 7.9 us,
// 7.0 in two: a compute unit needs 5 us for its 128 KB of A.)
#include <hip/hip_fp16.h>

#include <algorithm>
#include <type_traits>

#include "qoq_internal.h"
#include "qoq_kv4_common.h"

namespace qoq {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kMaxAdapters = 4096;
constexpr int kPlanHead = 16;                            // words: the number of tiles, then what the plan was made for
constexpr int kPlanMagic = 0x4C6F5241;
constexpr int kRankChunk = 64;                           // ranks with a scale of their own

// rows of a tile
int64_t tile_rows(int64_t M) { return M <= 512 ? 16 : 64; }
// Tiles of a plan at most: every adapter in use, and the rows of none, may end in a part of one.
int64_t most_tiles(int64_t M, int64_t adapters) { return M / tile_rows(M) + std::min(M, adapters + 1); }

struct PlanArgs {
    const int32_t* adapter;                              // [M]
    int M, adapters, tile;
    int* head;
    int4* tiles;                                         // adapter (-1: none), first place, rows
    int* rows;                                           // row of each place
};

__global__ __launch_bounds__(kPlanThreads) void lora_plan_kernel(PlanArgs p)
{
    __shared__ int s_count[kMaxAdapters + 1], s_start[kMaxAdapters + 1];
    __shared__ int2 s_wave[kPlanThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, n = p.adapters + 1;
    for (int a = tid; a < n; a += kPlanThreads) s_count[a] = 0;
    __syncthreads();
    auto of_row = [&](int m) { const int a = p.adapter[m]; return a >= 0 && a < p.adapters ? a : p.adapters; };
    for (int m = tid; m < p.M; m += kPlanThreads) atomicAdd(&s_count[of_row(m)], 1);
    __syncthreads();
    // places and tiles in front of this thread's adapters
    const int each = (n + kPlanThreads - 1) / kPlanThreads, a0 = min(tid * each, n), a1 = min(a0 + each, n);
    int2 mine = make_int2(0, 0);
    for (int a = a0; a < a1; ++a) { mine.x += s_count[a]; mine.y += (s_count[a] + p.tile - 1) / p.tile; }
    int2 upto = mine;
    for (int o = 1; o < 64; o <<= 1) {
        const int x = __shfl_up(upto.x, o, 64), y = __shfl_up(upto.y, o, 64);
        if (lane >= o) { upto.x += x; upto.y += y; }
    }
    if (lane == 63) s_wave[wave] = upto;
    __syncthreads();
    int place = upto.x - mine.x, tile = upto.y - mine.y;
    for (int w = 0; w < wave; ++w) { place += s_wave[w].x; tile += s_wave[w].y; }
    for (int a = a0; a < a1; ++a) {
        const int c = s_count[a];
        s_start[a] = place;
        for (int at = 0; at < c; at += p.tile) p.tiles[tile++] = make_int4(a < p.adapters ? a : -1, place + at, min(p.tile, c - at), 0);
        place += c;
    }
    if (tid == kPlanThreads - 1) {
        p.head[0] = tile;
        p.head[1] = p.M;
        p.head[2] = p.adapters;
        p.head[3] = kPlanMagic;
    }
    __syncthreads();
    // (the order of an adapter's rows is whichever arrives first: each row's result is its own, whatever the others of its tile are)
    for (int m = tid; m < p.M; m += kPlanThreads) p.rows[atomicAdd(&s_start[of_row(m)], 1)] = m;
}

// Tiles of a plan for these rows and adapters; none of anything else, whose rows and adapters could be any.
__device__ __forceinline__ int tiles_of(const int* head, int M, int adapters)
{
    return head[1] == M && head[2] == adapters && head[3] == kPlanMagic ? head[0] : 0;
}

struct ShrinkArgs {
    const __half* x;
    const __half* a;                                     // [adapters, rank, K]
    const int* head;
    const int4* tiles;
    const int* rows;
    float* parts;                                        // [slices][M][rank]
    int64_t x_stride;
    int M, adapters, K, rank, slice;                     // slice: elements of K, a multiple of 128
};

// 2^shift that brings a row's largest number to 2^14 .. 2^15, the last whole binade of FP16: half of its smallest step, 2^-25, is 2^-39 of that at most
__device__ __forceinline__ int shift_of(float most) { return most > 0.f ? min(141 - (int)(__float_as_uint(most) >> 23), 100) : 0; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ float finite_size(float v) { return fabsf(v) < __builtin_inff() ? fabsf(v) : 0.f; }
// (a number below half of the smallest step keeps that step and its sign, which the low part takes back: an infinity of B that meets it is one, not 0 times that)
__device__ __forceinline__ _Float16 high_part(float y)
{
    const _Float16 hi = (_Float16)y;
    return hi == (_Float16)0.f && y != 0.f ? __builtin_bit_cast(_Float16, (unsigned short)((__float_as_uint(y) >> 16 & 0x8000u) | 1u)) : hi;
}
__device__ __forceinline__ _Float16 low_part(float y, _Float16 hi)
{
    const float back = (float)hi;
    return fabsf(back) < __builtin_inff() ? (_Float16)(y - back) : (_Float16)0.f;
}

// The sums of a tile over a slice of K.  Bound by x and A where rows are many, else by the trips to memory one after the other: a wave has all of its steps in flight.
template <int CT, int RT>
__global__ __launch_bounds__(256) void lora_shrink_kernel(ShrinkArgs p)
{
    __shared__ float s_part[4][RT * 16][17];
    const int tile = blockIdx.x, part = blockIdx.y, z = blockIdx.z;
    const int4 t = p.tiles[tile];                        // (whatever it holds, beside the head)
    if (tile >= tiles_of(p.head, p.M, p.adapters) || t.x < 0) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r16 = lane & 15, kb = lane >> 4;
    const int first_rank = z * kRankChunk, ranks = min(p.rank - first_rank, kRankChunk);

    const __half* x_row[CT];
    const __half* a_row[RT];
#pragma unroll
    for (int c = 0; c < CT; ++c) x_row[c] = p.x + (int64_t)p.rows[t.y + min(c * 16 + r16, t.z - 1)] * p.x_stride;
#pragma unroll
    for (int i = 0; i < RT; ++i) a_row[i] = p.a + ((int64_t)t.x * p.rank + first_rank + min(i * 16 + r16, ranks - 1)) * p.K;
    f4 acc[CT][RT];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int i = 0; i < RT; ++i) acc[c][i] = (f4){0.f, 0.f, 0.f, 0.f};

    // (a quarter of the slice for each wave: side by side, the waves' and slices' places in a row are spread over the memory channels, which rows of
    // a power of two apart are not)
    const int k0 = part * p.slice + wave * (p.slice / 4), k1 = min(k0 + p.slice / 4, p.K);
    constexpr int kTurn = CT * RT >= 8 ? 1 : CT * RT >= 4 ? 2 : 4;       // steps requested together; twice that are in flight where rows are many
    struct Turn { uint4 x[kTurn][CT], a[kTurn][RT]; };
    auto load = [&](Turn& v, int k) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < kTurn; ++s) {                // (elements behind the slice are read inside the row, and left out below)
            const int at = min(k + 32 * s + kb * 8, p.K - 8);
#pragma unroll
            for (int i = 0; i < RT; ++i) v.a[s][i] = *reinterpret_cast<const uint4*>(a_row[i] + at);
#pragma unroll
            for (int c = 0; c < CT; ++c) v.x[s][c] = *reinterpret_cast<const uint4*>(x_row[c] + at);
        }
    };
    auto multiply = [&](Turn& v, int k) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < kTurn; ++s) {
            if (k + 32 * s >= k1) break;
            if (k + 32 * s + 32 > k1) {
                const uint32_t some = k + 32 * s + kb * 8 < k1 ? ~0u : 0u;
                auto kept = [&](uint4 v) { return make_uint4(v.x & some, v.y & some, v.z & some, v.w & some); };
#pragma unroll
                for (int c = 0; c < CT; ++c) v.x[s][c] = kept(v.x[s][c]);
#pragma unroll
                for (int i = 0; i < RT; ++i) v.a[s][i] = kept(v.a[s][i]);
            }
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int i = 0; i < RT; ++i)
                    acc[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, v.a[s][i]), __builtin_bit_cast(h8, v.x[s][c]), acc[c][i], 0, 0, 0);
        }
    };
    Turn now;
    if (k0 < k1) {
        load(now, k0);
        if constexpr (CT > 1) {
            Turn next;
#pragma unroll 1
            for (int k = k0; k < k1; k += 64 * kTurn) {
                load(next, k + 32 * kTurn);
                multiply(now, k);
                load(now, k + 64 * kTurn);
                multiply(next, k + 32 * kTurn);
            }
        } else {
#pragma unroll 1
            for (int k = k0;;) {
                multiply(now, k);
                k += 32 * kTurn;
                if (k >= k1) break;
                load(now, k);
            }
        }
    }

    // ---- the waves' sums meet in LDS, sixteen rows at a time; sixteen lanes to a row, RT neighbouring ranks to a lane ----
    const int w = tid & 15, g = tid >> 4, rank0 = w * RT;
#pragma unroll 1
    for (int c = 0; c < CT; ++c) {
        if (c * 16 >= t.z) break;
        if (c) __syncthreads();
#pragma unroll
        for (int q = 0; q < CT; ++q)                     // (registers have no index)
            if (q == c)
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int x = 0; x < 4; ++x) s_part[wave][i * 16 + 4 * kb + x][r16] = acc[q][i][x];
        __syncthreads();
        const int row = c * 16 + g;
        if (row >= t.z || rank0 >= ranks) continue;      // (ranks come in eights)
        float v[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) v[i] = (s_part[0][rank0 + i][g] + s_part[1][rank0 + i][g]) + (s_part[2][rank0 + i][g] + s_part[3][rank0 + i][g]);
        float* to = p.parts + ((int64_t)part * p.M + t.y + row) * p.rank + first_rank + rank0;
        if constexpr (RT == 4) *reinterpret_cast<float4*>(to) = make_float4(v[0], v[1], v[2], v[3]);
        else if constexpr (RT == 2) *reinterpret_cast<float2*>(to) = make_float2(v[0], v[1]);
        else *to = v[0];
    }
}

// The slices' sums of a place and 64 ranks added up, in their order, and left as pairs: sixteen lanes to a place, four ranks to a lane.
struct PairArgs {
    const float* parts;
    __half* h;                                           // [M][2 rank]: 64 ranks at a time, hi then lo
    float* scales;                                       // [M][chunks]
    int M, rank, chunks, slices;
};
__global__ __launch_bounds__(256) void lora_pair_kernel(PairArgs p)
{
    const int w = threadIdx.x & 15, place = min((int)(blockIdx.x * 16 + (threadIdx.x >> 4)), p.M - 1), z = blockIdx.y;
    const int first = z * kRankChunk, ranks = min(p.rank - first, kRankChunk), rank = min(4 * w, ranks - 4);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    constexpr int kInFlight = 8;
#pragma unroll 1
    for (int s0 = 0; s0 < p.slices; s0 += kInFlight) {
        float4 got[kInFlight];
#pragma unroll
        for (int s = 0; s < kInFlight; ++s) got[s] = *reinterpret_cast<const float4*>(p.parts + ((int64_t)min(s0 + s, p.slices - 1) * p.M + place) * p.rank + first + rank);
#pragma unroll
        for (int s = 0; s < kInFlight; ++s) {
            const bool some = s0 + s < p.slices;
            v[0] += some ? got[s].x : 0.f; v[1] += some ? got[s].y : 0.f; v[2] += some ? got[s].z : 0.f; v[3] += some ? got[s].w : 0.f;
        }
    }
    const int shift = shift_of(row_max16(fmaxf(fmaxf(finite_size(v[0]), finite_size(v[1])), fmaxf(finite_size(v[2]), finite_size(v[3])))));
    if (4 * w >= ranks || blockIdx.x * 16 + (threadIdx.x >> 4) >= (unsigned)p.M) return;
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    h4 hi, lo;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float y = v[e] * power_of_two(shift);
        hi[e] = high_part(y);
        lo[e] = low_part(y, hi[e]);
    }
    _Float16* to = reinterpret_cast<_Float16*>(p.h) + (int64_t)place * 2 * p.rank + 2 * first + rank;
    *reinterpret_cast<h4*>(to) = hi;
    *reinterpret_cast<h4*>(to + ranks) = lo;
    if (w == 0) p.scales[(int64_t)place * p.chunks + z] = power_of_two(-shift);
}

struct ExpandArgs {
    const __half *base, *b;                              // b [adapters, N, rank]
    __half* out;
    const __half* h;
    const float *scales, *adapter_scales;                // adapter_scales may be null
    const float* parts;
    const int* head;
    const int4* tiles;
    const int* rows;
    int64_t base_stride, out_stride;
    int M, adapters, N, rank, chunks, slices, blocks;    // blocks of 64 channels for each wave
};

// STEPS matrix instructions for the pairs of a chunk of ranks, which `FULL` fill; WIDE: several chunks.  SUM: the pairs are formed here from the
// slices' sums, which for few rows takes less than to join them first.
// Bound by base and out; B of an adapter comes from the L2 for all but its first tile.
template <int CT, int STEPS, bool FULL, bool WIDE, bool SUM>
__global__ __launch_bounds__(64) __attribute__((amdgpu_waves_per_eu(WIDE ? 1 : 2))) void lora_expand_kernel(ExpandArgs p)
{
    const int tile = blockIdx.y;
    const int4 t = p.tiles[tile];                        // (whatever it holds, beside the head)
    if (tile >= tiles_of(p.head, p.M, p.adapters)) return;
    const int lane = threadIdx.x, r16 = lane & 15, kb = lane >> 4;
    const bool in_place = p.base == p.out;
    if (t.x < 0 && in_place) return;
    const __half* from[CT];
    __half* to[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int64_t row = p.rows[t.y + min(c * 16 + r16, t.z - 1)];
        from[c] = p.base + row * p.base_stride;
        to[c] = p.out + row * p.out_stride;
    }
    uint4 hv[CT][STEPS];
    float scale[CT];
    const float of_adapter = p.adapter_scales && t.x >= 0 ? p.adapter_scales[t.x] : 1.f;
    auto load_h = [&](int z) __attribute__((always_inline)) {
        const int ranks = min(p.rank - z * kRankChunk, kRankChunk);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int64_t place = t.y + min(c * 16 + r16, t.z - 1);
            if constexpr (SUM) {
                float v[STEPS][8], most = 0.f;
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[s][e] = 0.f;
#pragma unroll 4
                for (int q = 0; q < p.slices; ++q) {
                    const float* at = p.parts + ((int64_t)q * p.M + place) * p.rank + z * kRankChunk;
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        const int pair = s * 32 + kb * 8, rank = pair < ranks ? pair : min(pair, 2 * ranks - 8) - ranks;
                        const float4 a = *reinterpret_cast<const float4*>(at + rank), b = *reinterpret_cast<const float4*>(at + rank + 4);
                        v[s][0] += a.x; v[s][1] += a.y; v[s][2] += a.z; v[s][3] += a.w;
                        v[s][4] += b.x; v[s][5] += b.y; v[s][6] += b.z; v[s][7] += b.w;
                    }
                }
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int e = 0; e < 8; ++e) most = fmaxf(most, finite_size(v[s][e]));
                const int shift = shift_of(max_other_half(max_other_row(most)));
                scale[c] = power_of_two(-shift) * of_adapter;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const int pair = s * 32 + kb * 8;
                    _Float16 o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float y = v[s][e] * power_of_two(shift);
                        const _Float16 hi = high_part(y);
                        o[e] = pair < ranks ? hi : low_part(y, hi);
                        if (!FULL && pair >= 2 * ranks) o[e] = (_Float16)0.f;
                    }
                    hv[c][s] = __builtin_bit_cast(uint4, (h8){o[0], o[1], o[2], o[3], o[4], o[5], o[6], o[7]});
                }
            } else {
                const __half* at = p.h + place * 2 * p.rank + 2 * z * kRankChunk;
                scale[c] = p.scales[place * p.chunks + z] * of_adapter;
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    const int pair = s * 32 + kb * 8;
                    hv[c][s] = *reinterpret_cast<const uint4*>(at + (FULL ? pair : min(pair, 2 * ranks - 8)));
                    if (!FULL && pair >= 2 * ranks) hv[c][s] = make_uint4(0, 0, 0, 0);
                }
            }
        }
    };
    if (t.x >= 0 && !WIDE) load_h(0);
    const __half* b = p.b + (int64_t)max(t.x, 0) * p.N * p.rank;
    // two neighbouring channels of `base` and the products: words k of the lane's eight channels e
    auto added = [](uint32_t base, const f4 (&sum)[4], int e, int k) __attribute__((always_inline)) {
        const h2 o = __builtin_bit_cast(h2, base);
        return (h2){(_Float16)((float)o.x + sum[2 * e + k / 2][2 * (k & 1)]), (_Float16)((float)o.y + sum[2 * e + k / 2][2 * (k & 1) + 1])};
    };
    // h B^T of 64 channels from n0 on; HIGH: of the pairs' high parts alone
    auto products = [&](auto high, int n0, f4 (&sum)[CT][4]) __attribute__((always_inline)) {
        constexpr bool HIGH = decltype(high)::value;
#pragma unroll 1
        for (int z = 0; z < (WIDE ? p.chunks : 1); ++z) {
            if (WIDE) load_h(z);
            const int ranks = min(p.rank - z * kRankChunk, kRankChunk);
            uint4 w[STEPS][4];
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if constexpr (FULL && STEPS % 2 == 0 && !HIGH) {          // (16 STEPS ranks: the second half of the steps takes B as the first)
                    if (s >= STEPS / 2) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[s][j] = w[s - STEPS / 2][j];
                        continue;
                    }
                }
                const int pair = s * 32 + kb * 8, rank = pair < ranks ? pair : (FULL ? pair : min(pair, 2 * ranks - 8)) - ranks;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = min(n0 + (j >> 1) * 32 + (r16 >> 2) * 8 + (j & 1) * 4 + (r16 & 3), p.N - 1);
                    w[s][j] = *reinterpret_cast<const uint4*>(b + (int64_t)row * p.rank + z * kRankChunk + rank);
                    if (HIGH ? pair >= ranks : !FULL && pair >= 2 * ranks) w[s][j] = make_uint4(0, 0, 0, 0);
                }
            }
            f4 acc[CT][4];
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, w[s][j]), __builtin_bit_cast(h8, hv[c][s]), s ? acc[c][j] : (f4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sum[c][j][x] = !WIDE || z == 0 ? acc[c][j][x] * scale[c] : fmaf(acc[c][j][x], scale[c], sum[c][j][x]);
        }
    };
#pragma unroll 1
    for (int i = 0; i < p.blocks; ++i) {
        const int n0 = (i * gridDim.x + blockIdx.x) * 64;            // neighbouring workgroups go through neighbouring channels together
        if (n0 >= p.N) return;
        // a lane's results: channels n .. n + 7 and n + 32 .. n + 39 of its row, 4 of each matrix product j, so that four lanes take 64 bytes of a row
        // together (what lies behind the last channel is computed from the last ones' operands, and not stored)
        const int n = n0 + kb * 8;
        uint4 bv[CT][2];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) bv[c][e] = *reinterpret_cast<const uint4*>(from[c] + min(n + 32 * e, p.N - 8));
        f4 sum[CT][4];
        h2 any = {(_Float16)0.f, (_Float16)0.f};         // NaN where a result is
        if (t.x >= 0) {
            products(std::false_type(), n0, sum);
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t v[4] = {bv[c][e].x, bv[c][e].y, bv[c][e].z, bv[c][e].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const h2 y = added(v[k], sum[c], e, k);
                        any = __builtin_elementwise_maximum(any, y);
                        v[k] = __builtin_bit_cast(uint32_t, y);
                    }
                    bv[c][e] = make_uint4(v[0], v[1], v[2], v[3]);
                }
            // An infinity of B meets both parts of a pair, of which the low one may be 0 or of the other sign: NaN, where h B is the high part's infinity.
            if (__builtin_amdgcn_ballot_w64(any.x != any.x || any.y != any.y) != 0) {
                int again = n0;                          // (operands are requested again, not kept until here)
                asm volatile("" : "+s"(again));
                products(std::true_type(), again, sum);
#pragma unroll
                for (int c = 0; c < CT; ++c)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const uint4 base = *reinterpret_cast<const uint4*>(from[c] + min(again + kb * 8 + 32 * e, p.N - 8));
                        const uint32_t old[4] = {base.x, base.y, base.z, base.w};
                        uint32_t v[4] = {bv[c][e].x, bv[c][e].y, bv[c][e].z, bv[c][e].w};
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            h2 y = __builtin_bit_cast(h2, v[k]);
                            const h2 by_high = added(old[k], sum[c], e, k);
                            y.x = y.x != y.x ? by_high.x : y.x;
                            y.y = y.y != y.y ? by_high.y : y.y;
                            v[k] = __builtin_bit_cast(uint32_t, y);
                        }
                        bv[c][e] = make_uint4(v[0], v[1], v[2], v[3]);
                    }
            }
        }
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e)
                if (c * 16 + r16 < t.z && n + 32 * e < p.N) *reinterpret_cast<uint4*>(to[c] + n + 32 * e) = bv[c][e];
    }
}

bool large_tiles(int64_t M) { return tile_rows(M) == 64; }
// Slices of K.  Few rows: workgroups enough to fill the chip twice, of 512 elements at least (four steps of each wave, which are in flight together).
// Many rows: one workgroup to a compute unit; the tiles' sums are 16 KB a slice (4096 rows of 8192 elements and 64 ranks 33.8 us with 3 slices, 33.6 with 7,
// 41 with 10, 77 with one; 1733 of 4096 and 8 ranks 9.1 with 7, 10.1 with 14, 10.5 with 3).
int shrink_slices(int64_t M, int64_t K, int64_t rank, int64_t adapters)
{
    const int64_t chunks = (rank + kRankChunk - 1) / kRankChunk, tiles = most_tiles(M, adapters);
    if (tiles <= 0) return 1;
    if (large_tiles(M)) return (int)std::max<int64_t>(1, std::min<int64_t>(256 / (tiles * chunks), (K + 255) / 256));
    return (int)std::max<int64_t>(1, std::min<int64_t>({512 / (tiles * chunks), (K + 511) / 512, 16}));
}

// Whether a launch of its own forms the pairs: where a wave of the second product would read more than 16 KB of sums for them (473 rows of 32 ranks beside
// 8192 x 8192 in 30 tiles of 15 slices 41.0 us, 18.0 with the launch; 64 rows of 16 ranks beside 6144 x 4096 8.4 and 10.0).
bool pair_first(int64_t M, int64_t K, int64_t rank, int64_t adapters)
{
    return large_tiles(M) || shrink_slices(M, K, rank, adapters) * rank > 256;
}

typedef void (*ExpandKernel)(ExpandArgs);
struct Shape { bool big, pairs; };
template <int STEPS, bool FULL, bool WIDE>
ExpandKernel pick_expand(Shape s)
{
    if (s.big) return lora_expand_kernel<4, STEPS, FULL, WIDE, false>;
    return s.pairs ? lora_expand_kernel<1, STEPS, FULL, WIDE, false> : lora_expand_kernel<1, STEPS, FULL, WIDE, true>;
}
ExpandKernel pick_expand_of(int64_t rank, Shape big)
{
    switch (rank / 8) {
        case 1: return pick_expand<1, false, false>(big);
        case 2: return pick_expand<1, true, false>(big);
        case 3: return pick_expand<2, false, false>(big);
        case 4: return pick_expand<2, true, false>(big);
        case 5: return pick_expand<3, false, false>(big);
        case 6: return pick_expand<3, true, false>(big);
        case 7: return pick_expand<4, false, false>(big);
        default: return pick_expand<4, true, false>(big);
    }
}

struct Layout { size_t h, parts, all; };                  // of the workspace: scales, pairs, the slices' sums
Layout workspace_layout(int64_t M, int64_t K, int64_t rank, int64_t adapters)
{
    auto up = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    const int64_t chunks = (rank + kRankChunk - 1) / kRankChunk;
    Layout l;
    const bool pairs = pair_first(M, K, rank, adapters);
    l.h = pairs ? up(M * chunks * 4) : 0;
    l.parts = l.h + (pairs ? up(M * rank * 4) : 0);
    l.all = l.parts + up(shrink_slices(M, K, rank, adapters) * M * rank * 4);
    return l;
}

}  // namespace

size_t lora_plan_bytes(int64_t M, int64_t adapters) { return (size_t)(kPlanHead + 4 * most_tiles(M, adapters) + (M + 3) / 4 * 4) * 4; }
int64_t lora_max_adapters() { return kMaxAdapters; }

hipError_t launch_lora_plan(const int32_t* row_adapter, int64_t M, int64_t adapters, void* plan, hipStream_t s)
{
    PlanArgs p{};
    p.adapter = row_adapter; p.M = (int)M; p.adapters = (int)adapters; p.tile = (int)tile_rows(M);
    p.head = static_cast<int*>(plan);
    p.tiles = reinterpret_cast<int4*>(p.head + kPlanHead);
    p.rows = p.head + kPlanHead + 4 * most_tiles(M, adapters);
    lora_plan_kernel<<<1, kPlanThreads, 0, s>>>(p);
    return hipGetLastError();
}

size_t lora_workspace_bytes(int64_t M, int64_t N, int64_t K, int64_t rank, int64_t adapters) { return workspace_layout(M, K, rank, adapters).all; }

hipError_t launch_lora_add(const LoraAdd& l, hipStream_t s)
{
    const int64_t chunks = (l.rank + kRankChunk - 1) / kRankChunk, tiles = most_tiles(l.M, l.adapters), slices = shrink_slices(l.M, l.K, l.rank, l.adapters);
    const Layout at = workspace_layout(l.M, l.K, l.rank, l.adapters);
    char* ws = static_cast<char*>(l.workspace);
    ShrinkArgs a{};
    a.x = static_cast<const __half*>(l.x); a.a = static_cast<const __half*>(l.a);
    a.head = static_cast<const int*>(l.plan);
    a.tiles = reinterpret_cast<const int4*>(a.head + kPlanHead);
    a.rows = a.head + kPlanHead + 4 * tiles;
    a.parts = reinterpret_cast<float*>(ws + at.parts);
    a.x_stride = l.x_stride;
    a.M = (int)l.M; a.adapters = (int)l.adapters; a.K = (int)l.K; a.rank = (int)l.rank;
    a.slice = (int)(((l.K + slices - 1) / slices + 127) / 128 * 128);
    const bool big = large_tiles(l.M), pairs = pair_first(l.M, l.K, l.rank, l.adapters);
    const int rt = l.rank <= 16 ? 1 : l.rank <= 32 ? 2 : 4;
    const int64_t blocks64 = (l.N + 63) / 64;
    // blocks of 64 channels for each wave, which keeps h meanwhile
    const int64_t each = std::max<int64_t>(1, std::min<int64_t>(8, tiles * blocks64 / 8192)), groups = (blocks64 + each - 1) / each;
    if (tiles * groups >= (int64_t)1 << 24) return hipErrorInvalidValue;    // (tiles and slices are at most 20481 and, with the chunks, 163848)
    const dim3 grid((unsigned)tiles, (unsigned)slices, (unsigned)chunks);
    auto* shrink = big ? (rt == 1 ? lora_shrink_kernel<4, 1> : rt == 2 ? lora_shrink_kernel<4, 2> : lora_shrink_kernel<4, 4>)
                       : (rt == 1 ? lora_shrink_kernel<1, 1> : rt == 2 ? lora_shrink_kernel<1, 2> : lora_shrink_kernel<1, 4>);
    shrink<<<grid, 256, 0, s>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    __half* h = reinterpret_cast<__half*>(ws + at.h);
    float* scales = reinterpret_cast<float*>(ws);
    if (pairs) {
        PairArgs q{};
        q.parts = a.parts; q.h = h; q.scales = scales;
        q.M = (int)l.M; q.rank = (int)l.rank; q.chunks = (int)chunks; q.slices = (int)slices;
        lora_pair_kernel<<<dim3((unsigned)((l.M + 15) / 16), (unsigned)chunks), 256, 0, s>>>(q);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    ExpandArgs e{};
    e.base = static_cast<const __half*>(l.base); e.b = static_cast<const __half*>(l.b); e.out = static_cast<__half*>(l.out);
    e.h = h; e.scales = scales; e.parts = a.parts; e.adapter_scales = l.scales;
    e.head = a.head; e.tiles = a.tiles; e.rows = a.rows;
    e.base_stride = l.base_stride; e.out_stride = l.out_stride;
    e.M = (int)l.M; e.adapters = (int)l.adapters; e.N = (int)l.N; e.rank = (int)l.rank; e.chunks = (int)chunks; e.slices = (int)slices; e.blocks = (int)each;
    auto* expand = chunks > 1 ? pick_expand<4, false, true>({big, pairs}) : pick_expand_of(l.rank, {big, pairs});
    expand<<<dim3((unsigned)groups, (unsigned)tiles), 64, 0, s>>>(e);
    return hipGetLastError();
}

}  // namespace qoq
