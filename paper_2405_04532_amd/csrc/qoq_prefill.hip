// Causal attention over ragged prompts in FP16, with a sliding window and first tokens that stay visible.
//
//   out[i, h] = softmax_t( q[i, h] . k[t, h / r] / sqrt(128) ) v[t, h / r],  t <= p and (t > p - window or t < sinks),
//   p = Tk - Tq + i the position of a sequence's i-th query: the queries are the last Tq of its Tk tokens.
//
// The rows of a (sequence, KV head) are its queries times the r heads that share the KV head, query by query; a workgroup
// takes 128 of them, a wave 32.  Keys and values pass in tiles of 64, through LDS, one tile ahead of the arithmetic.  Both products run on
// v_mfma_f32_32x32x16_f16 with the rows in the columns of the results:
//   S[key][row]  = sum_d k[key][d] q[row][d]           a lane has 16 keys of every 32 for its one row, so maximum and sum of a
//                                                       row are the lane's own but for one exchange between the halves
//   O[d][row]   += sum_key v[key][d] p[key][row]       p's registers are the operand as they stand: the order of the keys in
//                                                       the sum is free, and v is read transposed from LDS in that order
// Softmax in base 2, FP32; the weights are rounded to FP16 for the second product (2^-11 relative, each on its own), sums stay FP32.
// The running maximum is raised only when a score passes it by more than kSlack: weights then reach 2^kSlack, their FP16 numbers
// have the same relative precision there, and the sums' 64 registers are rarely rescaled.
#include <algorithm>
#include <type_traits>

#include "qoq_gemm_common.h"
#include "qoq_kv4_common.h"
#include "qoq_ragged.h"

namespace qoq {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kBM = 128, kBN = 64, kPrefillThreads = 256;
constexpr int kRowBytes = kD * 2;                        // 256: sixteen 16-byte chunks
constexpr int kTileBytes = kBN * kRowBytes;              // 16 KiB of keys, as much of values
constexpr float kScale = 1.4426950408889634f * 0.08838834764831845f;      // log2(e) / sqrt(128)
constexpr float kSlack = 8.f / kScale;                   // in units of the scores

struct PrefillArgs {
    const __half *q, *k, *v;
    __half* out;
    const int32_t *cu_q, *cu_k;
    int64_t q_stride, k_stride, v_stride;                // elements per token
    int M, Mk, B, H, Hkv, r, window, sinks;
    uint32_t slots;
};

// LDS position of chunk c of row `row`.  Keys are read 32 rows at a time, the same chunk of each: c ^ row % 16 spreads 16
// rows over all chunk positions.  Values are read by lanes that take four rows of the same 64 bytes: those go to different quarters.
__device__ __forceinline__ int k_place(int row, int c) { return c ^ (row & 15); }
__device__ __forceinline__ int v_place(int row, int c) { return c ^ ((row & 3) << 2); }

__device__ __forceinline__ h8 v_operand(const uint8_t* lo, const uint8_t* hi)      // two transposed reads of four keys each
{
    typedef __attribute__((address_space(3))) s4 lds_s4;
    struct { s4 a, b; } t = {__builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)lo), __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)hi)};
    return __builtin_bit_cast(h8, t);
}

__global__ __launch_bounds__(kPrefillThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void prefill_kernel(PrefillArgs p)
{
    __shared__ __align__(256) uint8_t s_tiles[2][2][kTileBytes];           // [buffer][keys | values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hl = lane >> 5, col = lane & 31;
    // the last tiles of a sequence, which see the most keys, come first
    const uint32_t slot = p.slots - 1 - blockIdx.x / (uint32_t)p.Hkv;
    const int hk = (int)(blockIdx.x % (uint32_t)p.Hkv);
    const int b = count_before(p.B, lane, [&](int i) { return ((int64_t)p.cu_q[i] * p.r >> 7) + i <= (int64_t)slot; });
    if (b >= p.B) return;
    auto bounded = [](int v, int most) { return min(max(v, 0), most); };
    const int q0 = bounded(p.cu_q[b], p.M), q1 = bounded(p.cu_q[b + 1], p.M), k0 = bounded(p.cu_k[b], p.Mk), k1 = bounded(p.cu_k[b + 1], p.Mk);
    const int Tq = q1 - q0, Tk = max(k1 - k0, 0);
    const int64_t tile = (int64_t)slot - (((int64_t)p.cu_q[b] * p.r >> 7) + b);
    if (Tq <= 0 || tile < 0 || tile * kBM >= (int64_t)Tq * p.r) return;
    const int first = (int)(tile * kBM);                                   // row of the (sequence, KV head); below 2^31
    // this lane's row
    const int rho = first + wave * 32 + col, i = rho / p.r, j = rho - i * p.r;
    const bool there = i < Tq;
    const int pos = Tk - Tq + i;
    // the wave's and the workgroup's positions
    const int i_wave = (first + wave * 32) / p.r, i_wave_end = min((first + wave * 32 + 31) / p.r, Tq - 1);
    const int lo_wave = Tk - Tq + i_wave, hi_wave = Tk - Tq + i_wave_end;  // hi < lo: no row
    const int lo_pos = Tk - Tq + first / p.r, hi_pos = Tk - Tq + min((first + kBM - 1) / p.r, Tq - 1);
    // the list of key tiles: those of the sinks, then those of the window
    const int end = max(hi_pos + 1, 0), from = p.window ? max(lo_pos - p.window + 1, 0) : 0;
    const int tiles = (end + kBN - 1) / kBN, n_first = min((p.sinks + kBN - 1) / kBN, tiles), gap = max(min(from / kBN, tiles) - n_first, 0);
    const int n = tiles - gap;

    // tiles of the list that hold a key which some row of the wave sees
    const int tiles_wave = hi_wave < max(lo_wave, 0) ? 0 : hi_wave / kBN + 1;
    const int n_wave = tiles_wave <= n_first ? tiles_wave : max(tiles_wave - gap, n_first);

    const __half* k_rows = p.k + (int64_t)k0 * p.k_stride + hk * kD;
    const __half* v_rows = p.v + (int64_t)k0 * p.v_stride + hk * kD;
    auto tile_of = [&](int it) __attribute__((always_inline)) { return it < n_first ? it : it + gap; };
    // A wave copies 16 rows of a tile, four at a time; rows past the end repeat the last one.  Within a tile that is whole the lanes' offsets
    // never change: row 16 wave + 4 x + lane / 16 has its chunks at place ^ 4 x (keys), or where every fourth row has them (values).
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&s_tiles[0][0][0] + wave * 4096;
    const int row0 = wave * 16 + (lane >> 4), k_chunk = k_place(lane >> 4, lane & 15) * 16, v_chunk = v_place(lane >> 4, lane & 15) * 16;
    const uint32_t k_copy = (uint32_t)(row0 * (int)p.k_stride * 2), v_copy = (uint32_t)(row0 * (int)p.v_stride * 2 + v_chunk);
    auto fetch = [&](int it, bool values) __attribute__((always_inline)) {
        const int t0 = tile_of(it) * kBN, most = Tk - 1 - t0;
        const int64_t stride = values ? p.v_stride : p.k_stride;
        const __half* rows = (values ? v_rows : k_rows) + t0 * stride;
        const uint32_t to = lds + ((it & 1) * 2 + (values ? 1 : 0)) * kTileBytes;
        if (most >= kBN - 1) {
#pragma unroll
            for (int x = 0; x < 4; ++x) dma16(rows + 4 * x * stride, values ? v_copy : k_copy + (uint32_t)(k_chunk ^ (64 * x)), to + x * 1024);
        } else {
            int r = row0;
            asm volatile("" : "+v"(r));                                    // (nothing of this in registers outside)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                dma16(rows, (uint32_t)(min(r + 4 * x, most) * (int)stride * 2 + (values ? v_chunk : k_chunk ^ (64 * x))), to + x * 1024);
        }
    };
    if (n > 0) {
        fetch(0, false);
        fetch(0, true);
    }
    if (n > 1) fetch(1, false);

    h8 qf[8];                                                              // elements 16 s + 8 hl .. of this lane's row
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(q0 + (there ? i : 0)) * p.q_stride + (hk * p.r + (there ? j : 0)) * kD);
        const uint32_t some = there ? ~0u : 0u;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const uint4 t = src[2 * s + hl];
            qf[s] = __builtin_bit_cast(h8, make_uint4(t.x & some, t.y & some, t.z & some, t.w & some));
        }
    }
    float m = -1e30f, l[4] = {0.f, 0.f, 0.f, 0.f};                         // l: of this lane's keys
    f16v acc[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = (f16v)(0.f);

    // lane offsets of the operands in a tile
    uint32_t k_off[8], v_off[4];
#pragma unroll
    for (int s = 0; s < 8; ++s) k_off[s] = (uint32_t)(col * kRowBytes + k_place(col, 2 * s + hl) * 16);
    const int key = 4 * hl + ((lane & 15) >> 2);                           // of the 8-key groups: the row this lane addresses
    const int within = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);          // 16-byte chunk of the 64 bytes of 32 elements
#pragma unroll
    for (int d = 0; d < 4; ++d) v_off[d] = (uint32_t)(key * kRowBytes + v_place(key, 4 * d + within) * 16 + (lane & 1) * 8);

    // sc[x][y]: key 32 x + 8 (y / 4) + 4 hl + y % 4 of the tile
    auto scores = [&](int it, f16v (&sc)[2]) __attribute__((always_inline)) {
        const uint8_t* ks = s_tiles[it & 1][0];
        sc[0] = sc[1] = (f16v)(0.f);
#pragma unroll
        for (int s = 0; s < 8; ++s)
#pragma unroll
            for (int x = 0; x < 2; ++x)
                sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(ks + 32 * x * kRowBytes + k_off[s]), qf[s], sc[x], 0, 0, 0);
    };
    auto top_of = [&](const f16v (&sc)[2]) __attribute__((always_inline)) {
        float t[4] = {m, m, m, m};
#pragma unroll
        for (int y = 0; y < 16; ++y) t[y & 3] = fmaxf(fmaxf(t[y & 3], sc[0][y]), sc[1][y]);
        return max_other_half(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])));
    };
    auto values = [&](int it, int s, int d) __attribute__((always_inline)) {   // v's operand: 16 keys of step s, 32 elements of block d
        const uint8_t* at = s_tiles[it & 1][1] + 16 * s * kRowBytes + v_off[d];
        return v_operand(at, at + 8 * kRowBytes);
    };
    auto not_finite = [&](const h8& a, float bad) __attribute__((always_inline)) {  // NaN if some element is not finite
        struct { h2 v[4]; } t = __builtin_bit_cast(decltype(t), a);
#pragma unroll
        for (int x = 0; x < 4; ++x) bad = __builtin_amdgcn_fdot2(t.v[x], (h2){(_Float16)0.f, (_Float16)0.f}, bad, false);
        return bad;
    };
    bool odd = false;                                                      // some value that not every row sees is not finite
    // One tile: the weights of scores `sc` (with their maximum `top`, m among them) and their product with the values, while the
    // matrix cores form the next tile's scores (behind the last tile those of whatever the buffer holds, for nobody).  The order of
    // the instructions is set here, step by step: a step's products run while the next step's operands come from LDS and a share of the
    // softmax is computed.
    auto tile_step = [&](int it, f16v (&sc)[2], float& top, f16v (&next)[2]) __attribute__((always_inline)) {
        const int t0 = tile_of(it) * kBN, t1 = t0 + kBN - 1;
        const bool masked = !(t1 <= lo_wave && (!p.window || t0 > hi_wave - p.window || t1 < p.sinks));
        // of the tile's keys this row sees those up to at_most that lie above `above` or below `below`; a lane's first key is 4 hl (counted
        // from there, the keys are constants)
        const int at_most = (there ? pos - t0 : -1) - 4 * hl, above = (p.window ? pos - p.window - t0 : -1) - 4 * hl, below = p.sinks - t0 - 4 * hl;
        auto seen = [&](int e) { return e <= at_most && (e > above || e < below); };
        if (masked) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 16; ++y) sc[x][y] = seen(32 * x + 8 * (y >> 2) + (y & 3)) ? sc[x][y] : -__builtin_inff();
            top = top_of(sc);
            float bad = 0.f;
#pragma unroll 1
            for (int s = 0; s < 4; ++s)
#pragma unroll
                for (int d = 0; d < 4; ++d) bad = not_finite(values(it, s, d), bad);
            if (__builtin_amdgcn_ballot_w64(bad != bad) != 0) odd = true;
        }
        if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0) {
            const float alpha = __builtin_amdgcn_exp2f((m - top) * kScale);
            m = top;
#pragma unroll
            for (int x = 0; x < 4; ++x) l[x] *= alpha;
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[d] *= alpha;
        }
        const float shift = -m * kScale;
        const uint8_t* ks = s_tiles[(it + 1) & 1][0];
        auto keys = [&](int st, int x) __attribute__((always_inline)) { return *reinterpret_cast<const h8*>(ks + 32 * x * kRowBytes + k_off[st]); };
        h8 w[4], kf[3][2], vf[2][4];                                       // w: weights of 16 keys each
        h2 o[4];
#pragma unroll
        for (int st = 0; st < 2; ++st)
#pragma unroll
            for (int x = 0; x < 2; ++x) kf[st][x] = keys(st, x);
        next[0] = next[1] = (f16v)(0.f);
#pragma unroll
        for (int st = 0; st < 8; ++st) {
            if (st < 6) {
                kf[(st + 2) % 3][0] = keys(st + 2, 0);
                kf[(st + 2) % 3][1] = keys(st + 2, 1);
            } else {
#pragma unroll
                for (int d = 0; d < 2; ++d) vf[0][2 * (st - 6) + d] = values(it, 0, 2 * (st - 6) + d);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                next[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kf[st % 3][x], qf[st], next[x], 0, 0, 0);
                // two weights
                const int y = 4 * (st & 3) + 2 * x;
                const float a = __builtin_amdgcn_exp2f(fmaf(sc[st >> 2][y], kScale, shift));
                const float c = __builtin_amdgcn_exp2f(fmaf(sc[st >> 2][y + 1], kScale, shift));
                const h2 ac = {(_Float16)a, (_Float16)c};
                // the sum of the rounded weights: a row that sees one key returns its values exactly
                l[y / 2 & 3] = __builtin_amdgcn_fdot2(ac, (h2){(_Float16)1.f, (_Float16)1.f}, l[y / 2 & 3], false);
                o[y / 2 & 3] = ac;
            }
            if (st & 1) w[st >> 1] = join(o[0], o[1], o[2], o[3]);
            __builtin_amdgcn_sched_barrier(0);
        }
        float t4[4] = {m, m, m, m};
#pragma unroll
        for (int st = 0; st < 4; ++st) {
            if (st < 3)
#pragma unroll
                for (int d = 0; d < 4; ++d) vf[(st + 1) & 1][d] = values(it, st + 1, d);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[st & 1][d], w[st], acc[d], 0, 0, 0);
                t4[d] = fmaxf(fmaxf(t4[d], next[0][4 * st + d]), next[1][4 * st + d]);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        top = max_other_half(fmaxf(fmaxf(t4[0], t4[1]), fmaxf(t4[2], t4[3])));
    };
    f16v sa[2], sb[2];
    float top = m;
    if (n > 0) {
        if (n > 1) wait_vmcnt<8>();                                        // the first tile's keys; its values and the second's keys are on their way
        else wait_vmcnt<4>();
        __syncthreads();
        scores(0, sa);
        top = top_of(sa);
    }
    // Keys run one tile ahead of the values: turn `it` multiplies the values of tile it and forms the scores of tile it + 1.  At its start
    // everyone has left the keys of tile it and the values of tile it - 1, whose places the next copies take.
    auto turn = [&](int it, f16v (&sc)[2], f16v (&next)[2]) __attribute__((always_inline)) {
        wait_vmcnt<0>();
        __syncthreads();
        if (it + 2 < n) fetch(it + 2, false);
        if (it + 1 < n) fetch(it + 1, true);
        if (it < n_wave) tile_step(it, sc, top, next);
    };
    for (int it = 0; it < n; it += 2) {
        turn(it, sa, sb);
        if (it + 1 < n) turn(it + 1, sb, sa);
    }
    if (odd) {
        // A zero weight times infinity or NaN is NaN, in rows that do not see that value.  Such a wave's rows are done again here, one after
        // the other, with the keys they see and no others: 64 scores at a time, a lane each, then two elements of the values a lane.
        for (int x = 0; x < 32; ++x) {
            const int row = first + wave * 32 + x, qi = row / p.r, h = hk * p.r + row - qi * p.r, at = Tk - Tq + qi;
            if (qi >= Tq) break;
            const __half* q_row = p.q + (int64_t)(q0 + qi) * p.q_stride + h * kD;
            float top = -1e30f, sum = 0.f, o0 = 0.f, o1 = 0.f;
            for (int it = 0; it < n; ++it) {
                const int t = tile_of(it) * kBN + lane;
                const bool sees = t <= at && (!p.window || t > at - p.window || t < p.sinks);
                float s = 0.f;
                if (sees)
                    for (int d = 0; d < kD; ++d) s = fmaf(__half2float(k_rows[(int64_t)t * p.k_stride + d]), __half2float(q_row[d]), s);
                float most = sees ? s : -__builtin_inff();
                for (int step = 32; step; step >>= 1) most = fmaxf(most, __shfl_xor(most, step, 64));
                most = fmaxf(most, top);
                const float keep = __builtin_amdgcn_exp2f((top - most) * kScale), weight = sees ? __builtin_amdgcn_exp2f((s - most) * kScale) : 0.f;
                top = most;
                sum = sum * keep + weight;
                o0 *= keep;
                o1 *= keep;
                for (uint64_t left = __builtin_amdgcn_ballot_w64(sees); left; left &= left - 1) {
                    const int from = __ffsll((unsigned long long)left) - 1;
                    const float wt = __shfl(weight, from, 64);
                    const __half* v_row = v_rows + (int64_t)(tile_of(it) * kBN + from) * p.v_stride + 2 * lane;
                    o0 = fmaf(wt, __half2float(v_row[0]), o0);
                    o1 = fmaf(wt, __half2float(v_row[1]), o1);
                }
            }
            for (int step = 32; step; step >>= 1) sum += __shfl_xor(sum, step, 64);
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const h2 pair = {(_Float16)(o0 * inv), (_Float16)(o1 * inv)};
            reinterpret_cast<uint32_t*>(p.out + ((int64_t)(q0 + qi) * p.H + h) * kD)[lane] = __builtin_bit_cast(uint32_t, pair);
        }
        return;
    }
    float total = (l[0] + l[1]) + (l[2] + l[3]);
    total += __shfl_xor(total, 32, 64);
    if (!there) return;
    const float inv = total == 0.f ? 0.f : 1.f / total;                    // a row that sees nothing is zero (NaN stays)
    __half* dst = p.out + ((int64_t)(q0 + i) * p.H + hk * p.r + j) * kD + 4 * hl;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const h2 a = {(_Float16)(acc[d][4 * y] * inv), (_Float16)(acc[d][4 * y + 1] * inv)};
            const h2 c = {(_Float16)(acc[d][4 * y + 2] * inv), (_Float16)(acc[d][4 * y + 3] * inv)};
            *reinterpret_cast<uint2*>(dst + 32 * d + 8 * y) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c));
        }
}

}  // namespace

size_t prefill_workspace_bytes(int64_t, int64_t, int64_t, int64_t, int64_t, int64_t, int64_t) { return 0; }

hipError_t launch_prefill(const Prefill& a, hipStream_t s)
{
    PrefillArgs p{};
    p.q = static_cast<const __half*>(a.q); p.k = static_cast<const __half*>(a.k); p.v = static_cast<const __half*>(a.v);
    p.out = static_cast<__half*>(a.out);
    p.cu_q = a.cu_q; p.cu_k = a.cu_k;
    p.q_stride = a.q_stride; p.k_stride = a.k_stride; p.v_stride = a.v_stride;
    p.M = (int)a.M; p.Mk = (int)a.Mk; p.B = (int)a.B; p.H = (int)a.H; p.Hkv = (int)a.Hkv; p.r = (int)(a.H / a.Hkv);
    p.window = (int)a.window; p.sinks = a.window ? (int)a.sinks : 0;
    const int64_t slots = a.M * p.r / kBM + a.B;
    if (slots * a.Hkv >= (int64_t)1 << 31) return hipErrorInvalidValue;
    p.slots = (uint32_t)slots;
    prefill_kernel<<<(unsigned)(slots * a.Hkv), kPrefillThreads, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace qoq
