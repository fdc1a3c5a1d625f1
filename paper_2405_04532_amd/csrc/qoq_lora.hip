// Low-rank adapters of many requests beside a projection that they share:
//   out[m] = base[m] + s_a (x[m] A_a^T) B_a^T,   a = the adapter of row m;   out[m] = base[m] where it has none
// with A_a [r, K], B_a [N, r] FP16, sums in FP32, one rounding at the end.
//
// Plan.  Which rows belong to which adapter is the same for every projection of a step, so it is worked out once: the rows ordered by
// adapter, and tiles of up to tile_rows(M) of them that share one, so that an adapter's matrices are read once for a tile.
//
// Two launches.  The first forms h = x A^T, tile by tile, K cut over workgroups where there are few tiles; the last workgroup of a tile adds the
// partial sums up, in their order whichever arrives when, and leaves h as pairs of FP16 numbers hi + lo of h scaled by a power of two for each
// row (and 64 ranks): within 2^-22 of h, or 2^-39 of the row's largest.  The second forms hi B^T + lo B^T: one product whose k runs over the
// pairs, B's columns taken twice.
#include <hip/hip_fp16.h>

#include <algorithm>

#include "qoq_gemm_common.h"
#include "qoq_internal.h"
#include "qoq_kv4_common.h"
#include "qoq_workspace.h"

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
    __half* h;                                           // [M][2 rank]: 64 ranks at a time, hi then lo
    float* scales;                                       // [M][chunks]
    int* counters;
    int64_t x_stride;
    int M, adapters, K, rank, chunks, slice;             // slice: elements of K, a multiple of 32
};

template <int CT, int RT>
__global__ __launch_bounds__(256) void lora_shrink_kernel(ShrinkArgs p)
{
    __shared__ __align__(16) float s_part[4][RT * 16][17];
    __shared__ int s_last;
    const int tile = blockIdx.x, part = blockIdx.y, parts = gridDim.y, z = blockIdx.z;
    if (tile >= tiles_of(p.head, p.M, p.adapters)) return;
    const int4 t = p.tiles[tile];
    if (t.x < 0) return;
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

    const int k0 = part * p.slice, k1 = min(k0 + p.slice, p.K);
    constexpr int kTurn = CT * RT >= 8 ? 1 : CT * RT >= 4 ? 2 : 4;       // steps in flight
    auto load = [&](const __half* row, int k) __attribute__((always_inline)) {
        return k < k1 ? *reinterpret_cast<const uint4*>(row + k) : make_uint4(0, 0, 0, 0);
    };
    for (int k = k0 + wave * 32 + kb * 8; k - kb * 8 < k1; k += 128 * kTurn) {
        uint4 xv[kTurn][CT], av[kTurn][RT];
#pragma unroll
        for (int s = 0; s < kTurn; ++s) {
#pragma unroll
            for (int c = 0; c < CT; ++c) xv[s][c] = load(x_row[c], k + 128 * s);
#pragma unroll
            for (int i = 0; i < RT; ++i) av[s][i] = load(a_row[i], k + 128 * s);
        }
#pragma unroll
        for (int s = 0; s < kTurn; ++s)
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int i = 0; i < RT; ++i)
                    acc[c][i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, av[s][i]), __builtin_bit_cast(h8, xv[s][c]), acc[c][i], 0, 0, 0);
    }

    // ---- the waves' sums meet in LDS, sixteen rows at a time; sixteen lanes to a row, lane w its ranks w, w + 16, ... ----
    const int w = tid & 15, g = tid >> 4;
    auto finish = [&](int row, const float (&v)[RT]) __attribute__((always_inline)) {       // row of the tile, whole sums
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const float m = fabsf(v[i]);
            most = fmaxf(most, i * 16 + w < ranks && m < __builtin_inff() ? m : 0.f);
        }
        most = row_max16(most);
        // 2^shift brings the largest to 2^13 .. 2^14, with room for the others' sums in FP16's range
        const int shift = most > 0.f ? min(140 - (int)(__float_as_uint(most) >> 23), 100) : 0;
        const float up = __uint_as_float((uint32_t)(127 + shift) << 23);
        if (row >= t.z) return;
        __half* to = p.h + (int64_t)(t.y + row) * 2 * p.rank + 2 * first_rank;
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            const int rank = i * 16 + w;
            if (rank >= ranks) continue;
            const float y = v[i] * up;
            const __half hi = __float2half_rn(y);
            const float back = __half2float(hi);
            to[rank] = hi;
            to[ranks + rank] = fabsf(back) < __builtin_inff() ? __float2half_rn(y - back) : __float2half_rn(0.f);
        }
        if (w == 0) p.scales[(int64_t)(t.y + row) * p.chunks + z] = __uint_as_float((uint32_t)(127 - shift) << 23);
    };
    auto place = [&](int s, int row) { return p.parts + ((int64_t)s * p.M + t.y + row) * p.rank + first_rank; };
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        if (c * 16 >= t.z) break;
        if (c) __syncthreads();
#pragma unroll
        for (int i = 0; i < RT; ++i)
#pragma unroll
            for (int x = 0; x < 4; ++x) s_part[wave][i * 16 + 4 * kb + x][r16] = acc[c][i][x];
        __syncthreads();
        float v[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) v[i] = (s_part[0][i * 16 + w][g] + s_part[1][i * 16 + w][g]) + (s_part[2][i * 16 + w][g] + s_part[3][i * 16 + w][g]);
        if (parts == 1) {
            finish(c * 16 + g, v);
        } else if (c * 16 + g < t.z) {
            float* to = place(part, c * 16 + g);
#pragma unroll
            for (int i = 0; i < RT; ++i)
                if (i * 16 + w < ranks) __hip_atomic_store(to + i * 16 + w, v[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
    }
    if (parts == 1) return;
    // The stores above went past the caches that other workgroups do not share; they have arrived when the counter is raised.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        int* counter = p.counters + tile * p.chunks + z;
        const int old = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = old == parts - 1;
        if (old == parts - 1) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        if (c * 16 >= t.z) break;
        const int row = min(c * 16 + g, t.z - 1);
        float v[RT];
#pragma unroll
        for (int i = 0; i < RT; ++i) v[i] = 0.f;
        constexpr int kInFlight = 32 / RT;
        for (int s0 = 0; s0 < parts; s0 += kInFlight) {
            float got[kInFlight][RT];
#pragma unroll
            for (int s = 0; s < kInFlight; ++s)
#pragma unroll
                for (int i = 0; i < RT; ++i)
                    got[s][i] = __hip_atomic_load(place(min(s0 + s, parts - 1), row) + min(i * 16 + w, ranks - 1), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
            for (int s = 0; s < kInFlight; ++s)
#pragma unroll
                for (int i = 0; i < RT; ++i) v[i] += s0 + s < parts ? got[s][i] : 0.f;
        }
        finish(c * 16 + g, v);
    }
}

struct ExpandArgs {
    const __half *base, *b;                              // b [adapters, N, rank]
    __half* out;
    const __half* h;
    const float *scales, *adapter_scales;                // adapter_scales may be null
    const int* head;
    const int4* tiles;
    const int* rows;
    int64_t base_stride, out_stride;
    int M, adapters, N, rank, chunks, blocks;            // blocks of 64 channels for each wave
};

// STEPS matrix instructions for the pairs of a chunk of ranks; WIDE: several chunks.
template <int CT, int STEPS, bool WIDE>
__global__ __launch_bounds__(64) void lora_expand_kernel(ExpandArgs p)
{
    const int tile = blockIdx.x;
    if (tile >= tiles_of(p.head, p.M, p.adapters)) return;
    const int4 t = p.tiles[tile];
    const int lane = threadIdx.x, r16 = lane & 15, kb = lane >> 4;
    const bool in_place = p.base == p.out;
    if (t.x < 0 && in_place) return;
    const __half* from[CT];
    __half* to[CT];
    bool there[CT];
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        there[c] = c * 16 + r16 < t.z;
        const int64_t row = p.rows[t.y + min(c * 16 + r16, t.z - 1)];
        from[c] = p.base + row * p.base_stride;
        to[c] = p.out + row * p.out_stride;
    }
    uint4 hv[STEPS][CT];
    float scale[CT];
    auto load_h = [&](int z) __attribute__((always_inline)) {
        const int ranks = min(p.rank - z * kRankChunk, kRankChunk);
#pragma unroll
        for (int c = 0; c < CT; ++c) {
            const int64_t place = t.y + min(c * 16 + r16, t.z - 1);
            const __half* at = p.h + place * 2 * p.rank + 2 * z * kRankChunk;
            scale[c] = p.scales[place * p.chunks + z] * (p.adapter_scales ? p.adapter_scales[t.x] : 1.f);
#pragma unroll
            for (int s = 0; s < STEPS; ++s) hv[s][c] = s * 32 + kb * 8 < 2 * ranks ? *reinterpret_cast<const uint4*>(at + s * 32 + kb * 8) : make_uint4(0, 0, 0, 0);
        }
    };
    if (t.x >= 0 && !WIDE) load_h(0);
    const __half* b = p.b + (int64_t)max(t.x, 0) * p.N * p.rank;
    for (int i = 0; i < p.blocks; ++i) {
        const int n0 = (blockIdx.y * p.blocks + i) * 64;
        if (n0 >= p.N) return;
        // a lane's results: 16 channels n0 + 16 kb .. of its row, 4 of each matrix product j
        const int n = n0 + kb * 16;
        uint4 bv[CT][2];
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) bv[c][e] = there[c] && n + 8 * e < p.N ? *reinterpret_cast<const uint4*>(from[c] + n + 8 * e) : make_uint4(0, 0, 0, 0);
        if (t.x < 0) {
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (there[c] && n + 8 * e < p.N) *reinterpret_cast<uint4*>(to[c] + n + 8 * e) = bv[c][e];
            continue;
        }
        f4 sum[CT][4];
        for (int z = 0; z < (WIDE ? p.chunks : 1); ++z) {
            if (WIDE) load_h(z);
            const int ranks = min(p.rank - z * kRankChunk, kRankChunk);
            f4 acc[CT][4];
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[c][j] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                const int pair = s * 32 + kb * 8, rank = pair < ranks ? pair : pair - ranks;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int row = n0 + (r16 >> 2) * 16 + j * 4 + (r16 & 3);
                    const uint4 w = pair < 2 * ranks ? *reinterpret_cast<const uint4*>(b + (int64_t)min(row, p.N - 1) * p.rank + z * kRankChunk + rank) : make_uint4(0, 0, 0, 0);
#pragma unroll
                    for (int c = 0; c < CT; ++c)
                        acc[c][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, w), __builtin_bit_cast(h8, hv[s][c]), acc[c][j], 0, 0, 0);
                }
            }
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x) sum[c][j][x] = z == 0 ? acc[c][j][x] * scale[c] : fmaf(acc[c][j][x], scale[c], sum[c][j][x]);
        }
#pragma unroll
        for (int c = 0; c < CT; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint32_t old[4] = {bv[c][e].x, bv[c][e].y, bv[c][e].z, bv[c][e].w};
                uint32_t now[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const h2 o = __builtin_bit_cast(h2, old[k]);
                    const float y0 = (float)o.x + sum[c][2 * e + k / 2][2 * (k & 1)], y1 = (float)o.y + sum[c][2 * e + k / 2][2 * (k & 1) + 1];
                    now[k] = __builtin_bit_cast(uint32_t, (h2){(_Float16)y0, (_Float16)y1});
                }
                if (there[c] && n + 8 * e < p.N) *reinterpret_cast<uint4*>(to[c] + n + 8 * e) = make_uint4(now[0], now[1], now[2], now[3]);
            }
    }
}

// Slices of K: workgroups enough to fill the chip, of 128 elements at least (a step of each wave).
int shrink_slices(int64_t M, int64_t K, int64_t rank, int64_t adapters)
{
    const int64_t chunks = (rank + kRankChunk - 1) / kRankChunk, tiles = most_tiles(M, adapters);
    if (tiles <= 0 || tiles * chunks > kMaxCounters) return 1;
    return (int)std::max<int64_t>(1, std::min<int64_t>(512 / (tiles * chunks), (K + 127) / 128));
}

struct Layout { size_t scales, h, parts, all; };          // of the workspace, behind the counters
Layout workspace_layout(int64_t M, int64_t K, int64_t rank, int64_t adapters)
{
    auto up = [](int64_t n) { return (size_t)((n + 255) / 256 * 256); };
    const int64_t chunks = (rank + kRankChunk - 1) / kRankChunk, slices = shrink_slices(M, K, rank, adapters);
    Layout l;
    l.scales = kCounterBytes;
    l.h = l.scales + up(M * chunks * 4);
    l.parts = l.h + up(M * rank * 4);
    l.all = l.parts + (slices > 1 ? up(slices * M * rank * 4) : 0);
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
    a.counters = reinterpret_cast<int*>(ws);
    a.scales = reinterpret_cast<float*>(ws + at.scales);
    a.h = reinterpret_cast<__half*>(ws + at.h);
    a.parts = reinterpret_cast<float*>(ws + at.parts);
    a.x_stride = l.x_stride;
    a.M = (int)l.M; a.adapters = (int)l.adapters; a.K = (int)l.K; a.rank = (int)l.rank; a.chunks = (int)chunks;
    a.slice = (int)(((l.K + slices - 1) / slices + 31) / 32 * 32);
    const bool big = tile_rows(l.M) == 64;
    const int rt = l.rank <= 16 ? 1 : l.rank <= 32 ? 2 : 4;
    const int64_t blocks64 = (l.N + 63) / 64;
    // blocks of 64 channels for each wave, which keeps h meanwhile
    const int64_t each = std::max<int64_t>(1, std::min<int64_t>(8, tiles * blocks64 / 4096)), groups = (blocks64 + each - 1) / each;
    if (tiles >= (int64_t)1 << 22 || tiles * slices * chunks >= (int64_t)1 << 24 || tiles * groups >= (int64_t)1 << 24 || groups > 65535) return hipErrorInvalidValue;
    const dim3 grid((unsigned)tiles, (unsigned)slices, (unsigned)chunks);
    auto* shrink = big ? (rt == 1 ? lora_shrink_kernel<4, 1> : rt == 2 ? lora_shrink_kernel<4, 2> : lora_shrink_kernel<4, 4>)
                       : (rt == 1 ? lora_shrink_kernel<1, 1> : rt == 2 ? lora_shrink_kernel<1, 2> : lora_shrink_kernel<1, 4>);
    shrink<<<grid, 256, 0, s>>>(a);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    ExpandArgs e{};
    e.base = static_cast<const __half*>(l.base); e.b = static_cast<const __half*>(l.b); e.out = static_cast<__half*>(l.out);
    e.h = a.h; e.scales = a.scales; e.adapter_scales = l.scales;
    e.head = a.head; e.tiles = a.tiles; e.rows = a.rows;
    e.base_stride = l.base_stride; e.out_stride = l.out_stride;
    e.M = (int)l.M; e.adapters = (int)l.adapters; e.N = (int)l.N; e.rank = (int)l.rank; e.chunks = (int)chunks; e.blocks = (int)each;
    const int steps = chunks > 1 ? 4 : (int)((2 * l.rank + 31) / 32);
    auto* expand = chunks > 1   ? (big ? lora_expand_kernel<4, 4, true> : lora_expand_kernel<1, 4, true>)
                   : steps == 1 ? (big ? lora_expand_kernel<4, 1, false> : lora_expand_kernel<1, 1, false>)
                   : steps == 2 ? (big ? lora_expand_kernel<4, 2, false> : lora_expand_kernel<1, 2, false>)
                   : steps == 3 ? (big ? lora_expand_kernel<4, 3, false> : lora_expand_kernel<1, 3, false>)
                                : (big ? lora_expand_kernel<4, 4, false> : lora_expand_kernel<1, 4, false>);
    expand<<<dim3((unsigned)tiles, (unsigned)groups), 64, 0, s>>>(e);
    return hipGetLastError();
}

}  // namespace qoq
