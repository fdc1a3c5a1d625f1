// The 4-bit KV cache in pages of a pool: norm, rotation and quantization of new tokens, tokens back as FP16, decode attention.
//
// Pool.  `pages` pages of 64 tokens; a page holds, for each KV head, the 8704 bytes that the contiguous cache holds per 64
// tokens (qoq_kv4.hip): codes of the keys, their scales and zeros, codes of the values, theirs.  A block table [B, width] names
// the page of each 64 tokens of a sequence; an entry outside 0 .. pages - 1 is no page: nothing is read or written there.
#include <algorithm>
#include <type_traits>

#include "qoq_gemm_common.h"
#include "qoq_kv4_common.h"
#include "qoq_ragged.h"
#include "qoq_workspace.h"

namespace qoq {
namespace {

// ------------------------------------------------------------------------------------------
// Norm, rotation and quantization of new tokens.  One pass over queries, keys and values: a row of 16 lanes holds one head of one
// token, 8 elements (16 bytes) a lane, so that a head's sum of squares, the other half of a rotated pair, and the quantizer's range
// are exchanges inside the row.
//   y = x gamma r,  r = 1 / sqrt(mean(x^2) + eps)   (with gamma);   pairs (a, b) -> (a cos - b sin, b cos + a sin)
// x gamma is exact in FP32 (two 11-bit numbers), its product with the FP32 cosine exact in FP64, whose multiply-add runs at
// FP32's rate here, so everything behind x gamma is FP64 up to the conversion to FP16.
// Bound by memory: a wave keeps two KV heads' or four queries' loads in flight and looks its rows and angles up once for up to eight heads.
// 5 x 1733 tokens of 64 / 8 heads 53 us, 5.0 TB/s (a large copy: 5.2), with norms 60; one token of 32 / 32 heads 4.1, 64 of 32 / 8 with norms 5.2.
// ------------------------------------------------------------------------------------------
struct AppendArgs {
    const __half *q, *k, *v;                     // token rows, their strides in elements
    int64_t q_stride, k_stride, v_stride;
    const __half *q_gamma, *k_gamma;             // [128] or null
    double eps;
    const float* angles;                         // [angle_rows, rot]: cosines, sines
    int angle_rows, rot, interleaved;
    const int32_t *cu, *starts;                  // starts may be null
    int M, B, H, Hkv;
    uint8_t* pool;
    uint32_t pages;
    const int32_t* table;
    int width;
    __half *q_out, *k_out;                       // k_out may be null
    int64_t q_out_stride, k_out_stride;
    uint32_t kv_items, kv_groups, kv_heads;      // waves for keys and values: groups of kv_heads heads per aligned quad of positions
    uint32_t q_items, q_groups, q_heads;         // waves for queries: groups of q_heads heads per four rows
};

// FP64 to FP16 through FP32, as programs convert (there is no direct instruction): within 1/2 + 2^-14 of a step, and the bits of a
// plain FP64 evaluation that is converted so.  One rounding instead costs a look for midpoints at every element, and one key in 16000
// is then another neighbour of such a midpoint than theirs, which now and then moves a 4-bit code by one.
__device__ __forceinline__ uint4 halves_of(const double (&y)[8])
{
    float f[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        f[e] = (float)y[e];
        asm("" : "+v"(f[e]));                                              // else the two conversions become one in software
    }
    uint32_t o[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] = __builtin_bit_cast(uint32_t, (h2){(_Float16)f[2 * e], (_Float16)f[2 * e + 1]});
    return make_uint4(o[0], o[1], o[2], o[3]);
}

template <int CTRL>
__device__ __forceinline__ uint32_t row_word(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, false); }
template <int CTRL>
__device__ __forceinline__ double row_double(double v)
{
    const uint64_t b = (uint64_t)__double_as_longlong(v);
    return __longlong_as_double((int64_t)((uint64_t)row_word<CTRL>((uint32_t)(b >> 32)) << 32 | row_word<CTRL>((uint32_t)b)));
}
__device__ __forceinline__ double row_sum16(double v)
{
    v += row_double<0x128>(v);                                             // rotations by 8, 4, 2, 1 lanes
    v += row_double<0x124>(v);
    v += row_double<0x122>(v);
    return v + row_double<0x121>(v);
}
// 1 / sqrt(v), v >= 0, to a few units in the last place: the instruction is good to 2^-23, each step doubles that
__device__ __forceinline__ double inverse_root(double v)
{
    double r = __builtin_amdgcn_rsq(v);
#pragma unroll
    for (int i = 0; i < 2; ++i) r = r * fma(-0.5 * v * r, r, 1.5);
    return v == 0.0 ? __builtin_inf() : v == __builtin_inf() ? 0.0 : r;
}

// Angles of a token for a lane's 8 elements, and the weights of a norm.  NEAR: pairs of neighbours, else of halves (i, i + rot / 2).
// WHOLE: all 128 elements are turned, so a lane's other halves lie 8 lanes further on.
template <bool NEAR, bool WHOLE>
struct Turn {
    double c[NEAR ? 4 : 8], s[NEAR ? 4 : 8];     // s: with the sign that the lane's elements take it with
    int partner;
    bool turned;

    __device__ __forceinline__ void load(const AppendArgs& p, int64_t pos, int lane)
    {
        const int w = lane & 15, half = p.rot / 2;
        turned = WHOLE || 8 * w < p.rot;
        const bool first = 8 * w < half;
        partner = NEAR || !turned ? lane : first ? lane + p.rot / 16 : lane - p.rot / 16;
#pragma unroll
        for (int e = 0; e < (NEAR ? 4 : 8); ++e) { c[e] = 1.0; s[e] = 0.0; }
        if (!turned) return;
        const int64_t row = pos < 0 ? 0 : pos < p.angle_rows ? pos : p.angle_rows - 1;
        const float* at = p.angles + row * p.rot + (NEAR ? 4 * w : first ? 8 * w : 8 * w - half);
        const float sign = NEAR || !first ? 1.f : -1.f;
#pragma unroll
        for (int e = 0; e < (NEAR ? 1 : 2); ++e) {
            const float4 cc = reinterpret_cast<const float4*>(at)[e], ss = reinterpret_cast<const float4*>(at + half)[e];
            c[4 * e] = cc.x; c[4 * e + 1] = cc.y; c[4 * e + 2] = cc.z; c[4 * e + 3] = cc.w;
            s[4 * e] = ss.x * sign; s[4 * e + 1] = ss.y * sign; s[4 * e + 2] = ss.z * sign; s[4 * e + 3] = ss.w * sign;
        }
    }

    // one head of a token; every lane of the row takes part.  g, gp: the norm's weights of the lane's and of its partner's elements
    __device__ __forceinline__ uint4 head(const uint4& raw, bool norm, const uint4& g, const uint4& gp, const AppendArgs& p) const
    {
        if (!norm && p.rot == 0) return raw;
        const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w}, gw[4] = {g.x, g.y, g.z, g.w};
        auto element = [](const uint32_t (&v)[4], int e) { return (float)half_of(v[e >> 1] >> (16 * (e & 1))); };
        float x[8];                                                        // x gamma, exact
        double r = 1.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = element(rw, e);
        if (norm) {
            double sum = 0.0;
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = fma((double)x[e], (double)x[e], sum);
            r = inverse_root(fma(row_sum16(sum), 1.0 / kD, p.eps));
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] *= element(gw, e);
        }
        double y[8];
        if constexpr (NEAR) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const double a = x[2 * e], b = x[2 * e + 1];
                y[2 * e] = turned ? fma(a, c[e], -(b * s[e])) : a;         // (0 times a neighbour's infinity is no zero)
                y[2 * e + 1] = turned ? fma(b, c[e], a * s[e]) : b;
            }
        } else {
            uint32_t pw[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) pw[e] = WHOLE ? row_word<0x128>(rw[e]) : (uint32_t)__shfl((int)rw[e], partner, 64);
            const uint32_t gq[4] = {gp.x, gp.y, gp.z, gp.w};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float o = element(pw, e);
                if (norm) o *= element(gq, e);
                y[e] = fma((double)x[e], c[e], (double)o * s[e]);
            }
        }
        if (norm)
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] *= r;
        const uint4 out = halves_of(y);
        if (!WHOLE && !norm && !turned) return raw;                        // (its bits, whatever they are)
        return out;
    }
    __device__ __forceinline__ void gammas(const __half* gamma, int lane, uint4& g, uint4& gp) const
    {
        g = gp = make_uint4(0, 0, 0, 0);
        if (!gamma) return;
        g = reinterpret_cast<const uint4*>(gamma)[lane & 15];
        gp = reinterpret_cast<const uint4*>(gamma)[partner & 15];
    }
};

template <bool NEAR, bool WHOLE>
__global__ __launch_bounds__(256) void rope_append_kernel(AppendArgs p)
{
    __shared__ uint4 s_block[4][16];                                       // per wave: the value codes of its quad
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, w = lane & 15;
    uint32_t item = blockIdx.x * 4 + (uint32_t)wave;
    Window window;
    Turn<NEAR, WHOLE> turn;
    uint4 gamma, gamma_partner;
    if (item < p.kv_items) {
        // keys and values: an aligned quad of token positions of one sequence, a group of KV heads
        const uint32_t slot = item / p.kv_groups, group = item - slot * p.kv_groups;
        auto before = [&](int end, int i) { return (uint32_t)(end >> 2) + 2u * (uint32_t)i <= slot; };
        window.load(p.cu, p.starts, p.B, near_before(p.B, lane, [&](int i) { return before(p.cu[i], i); }), lane);
        const int c = __popcll(__builtin_amdgcn_ballot_w64(lane < window.held && before(window.end, window.lo + lane + 1)));
        if (c >= window.held) return;
        const int b = window.lo + c;
        const int64_t row0 = window.first_row(b, false), T = (int64_t)window.end_row(b) - row0, p0 = window.start_of(b, false);
        const int64_t j = (int64_t)slot - ((row0 >> 2) + 2 * (int64_t)b);
        const int64_t pos = ((p0 >> 2) + j) * 4 + g, t = pos - p0, row = row0 + t;
        const bool there = t >= 0 && t < T && row >= 0 && row < p.M;       // a token of the call
        if (__builtin_amdgcn_ballot_w64(there) == 0) return;
        const bool held = there && pos >= 0 && pos < (int64_t)p.width * kPageTokens;
        const uint32_t id = held ? (uint32_t)p.table[(int64_t)b * p.width + pos / kPageTokens] : ~0u;
        const int64_t at = there ? row : 0;
        const uint4* k_src = reinterpret_cast<const uint4*>(p.k + at * p.k_stride) + w;
        const uint4* v_src = reinterpret_cast<const uint4*>(p.v + at * p.v_stride) + w;
        const int h0 = (int)(group * p.kv_heads), h1 = min(h0 + (int)p.kv_heads, p.Hkv);
        uint4 next_k[2], next_v[2];                                        // two heads on their way
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            next_k[x] = k_src[min(h0 + x, h1 - 1) * (kD / 8)];
            next_v[x] = v_src[min(h0 + x, h1 - 1) * (kD / 8)];
        }
        turn.load(p, pos, lane);
        turn.gammas(p.k_gamma, lane, gamma, gamma_partner);
        const bool valid = held && id < p.pages;
        const uint64_t written = __builtin_amdgcn_ballot_w64(valid);
        uint8_t* page = p.pool + (int64_t)(valid ? id : 0) * p.Hkv * kPageBytes;
        const int tin = (int)(pos & (kPageTokens - 1));
        for (int h = h0; h < h1; h += 2) {
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const uint4 rk = next_k[x], rv = next_v[x];
                const int ahead = min(h + x + 2, h1 - 1) * (kD / 8);
                next_k[x] = k_src[ahead];
                next_v[x] = v_src[ahead];
                if (h + x >= h1) break;
                const uint4 k = turn.head(rk, p.k_gamma != nullptr, gamma, gamma_partner, p);
                if (p.k_out && there) reinterpret_cast<uint4*>(p.k_out + row * p.k_out_stride + (h + x) * kD)[w] = k;
                if (written == 0) continue;
                uint8_t* at_page = page + (int64_t)(h + x) * kPageBytes;
                write_token<false>(k, at_page, tin, w, lane, written == ~0ull, valid, s_block[wave]);
                write_token<true>(rv, at_page, tin, w, lane, written == ~0ull, valid, s_block[wave]);
            }
        }
        return;
    }
    // queries: four rows, a group of heads
    item -= p.kv_items;
    if (item >= p.q_items) return;
    const uint32_t quad = item / p.q_groups, group = item - quad * p.q_groups;
    window.load(p.cu, p.starts, p.B, near_before(p.B, lane, [&](int x) { return p.cu[x] <= (int)(4 * quad); }), lane);
    int b = 0;
    bool far = false;                                                      // so many empty sequences that a row lies past the window
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int c = __popcll(__builtin_amdgcn_ballot_w64(lane < window.held && window.end <= (int)(4 * quad) + i));
        far |= c == 64;
        b = g == i ? window.lo + c : b;
    }
    if (far)
        for (int i = 0; i < 4; ++i) {
            const int c = count_before(p.B, lane, [&](int x) { return p.cu[x] <= (int)(4 * quad) + i; });
            b = g == i ? c : b;
        }
    const int64_t row = 4 * (int64_t)quad + g;
    const int b_in = min(b, p.B - 1);
    const int64_t row0 = window.first_row(b_in, far);
    const bool there = b < p.B && row >= row0 && row < p.M;
    const int64_t pos = window.start_of(b_in, far) + row - row0;
    const int64_t at = there ? row : 0;
    const int h0 = (int)(group * p.q_heads), h1 = min(h0 + (int)p.q_heads, p.H);
    const uint4* src = reinterpret_cast<const uint4*>(p.q + at * p.q_stride) + w;
    uint4* dst = reinterpret_cast<uint4*>(p.q_out + at * p.q_out_stride) + w;
    constexpr int kAhead = 4;                                              // heads on their way
    uint4 next[kAhead];
#pragma unroll
    for (int x = 0; x < kAhead; ++x) next[x] = src[min(h0 + x, h1 - 1) * (kD / 8)];
    turn.load(p, there ? pos : 0, lane);
    turn.gammas(p.q_gamma, lane, gamma, gamma_partner);
    for (int h = h0; h < h1; h += kAhead) {
#pragma unroll
        for (int x = 0; x < kAhead; ++x) {
            const uint4 raw = next[x];
            next[x] = src[min(h + x + kAhead, h1 - 1) * (kD / 8)];
            if (h + x >= h1) break;
            const uint4 y = turn.head(raw, p.q_gamma != nullptr, gamma, gamma_partner, p);
            if (there) dst[(h + x) * (kD / 8)] = y;
        }
    }
}

// ------------------------------------------------------------------------------------------
// Tokens of the cache back as FP16, (code - z) s rounded once: one wave per aligned 16 positions of a sequence and KV head, all its loads
// at once, keys and values stored in whole rows.  Bound by the stores: 6 x 6000 tokens of 8 heads 23-30 us, 4.7-6 TB/s; 389 tokens of 32 heads 4.7.
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ uint2 values_of(uint32_t c4, float z, float s)     // four codes in the low 16 bits
{
    float x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = ((float)((c4 >> (4 * j)) & 15u) + z) * s;
    return make_uint2(__builtin_bit_cast(uint32_t, (h2){(_Float16)x[0], (_Float16)x[1]}), __builtin_bit_cast(uint32_t, (h2){(_Float16)x[2], (_Float16)x[3]}));
}

__global__ __launch_bounds__(256) void paged_gather_kernel(const uint8_t* __restrict__ pool, const int32_t* __restrict__ table,
                                                           const int32_t* __restrict__ cu, const int32_t* __restrict__ starts,
                                                           __half* __restrict__ k_out, __half* __restrict__ v_out, uint32_t pages, int width,
                                                           int M, int B, int Hkv, uint32_t items)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int g = lane >> 4, w = lane & 15;
    const uint32_t item = blockIdx.x * 4 + (uint32_t)wave;
    if (item >= items) return;
    const uint32_t slot = item / (uint32_t)Hkv;
    const int h = (int)(item - slot * (uint32_t)Hkv);
    auto before = [&](int end, int i) { return (uint32_t)(end >> 4) + 2u * (uint32_t)i <= slot; };
    Window window;
    window.load(cu, starts, B, near_before(B, lane, [&](int i) { return before(cu[i], i); }), lane);
    const int c = __popcll(__builtin_amdgcn_ballot_w64(lane < window.held && before(window.end, window.lo + lane + 1)));
    if (c >= window.held) return;
    const int b = window.lo + c;
    const int64_t row0 = window.first_row(b, false), T = (int64_t)window.end_row(b) - row0, p0 = window.start_of(b, false);
    const int64_t j = (int64_t)slot - ((row0 >> 4) + 2 * (int64_t)b);
    const int64_t pos0 = ((p0 >> 4) + j) * 16;                             // floor(p0 / 16) also for negative p0
    if (pos0 >= p0 + T || pos0 + 16 <= p0) return;
    const bool held = pos0 >= 0 && pos0 < (int64_t)width * kPageTokens;
    const uint32_t id = held ? (uint32_t)table[(int64_t)b * width + pos0 / kPageTokens] : ~0u;
    const bool on = id < pages;                                            // else zeros
    const uint8_t* page = pool + ((int64_t)(on ? id : 0) * Hkv + h) * kPageBytes;
    const int tin = (int)(pos0 & (kPageTokens - 1));
    uint32_t kw[4], kp[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {                                          // token 4 i + g, elements 8 w ..
        kw[i] = on ? reinterpret_cast<const uint32_t*>(page + (tin + 4 * i + g) * (kD / 2))[w] : 0u;
        kp[i] = on ? reinterpret_cast<const uint32_t*>(page + kCodeBytes)[tin + 4 * i + g] : 0xE4000000u;
    }
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 vc = on ? reinterpret_cast<const uint4*>(page + kHalfPage + tin * (kD / 2))[lane] : none;
    const uint4 vp = on ? reinterpret_cast<const uint4*>(page + kHalfPage + kCodeBytes + tin * 4)[g]
                        : make_uint4(0xE4000000u, 0xE4000000u, 0xE4000000u, 0xE4000000u);
    auto there = [&](int64_t t) { return t >= 0 && t < T && row0 + t >= 0 && row0 + t < M; };
    auto zero_of = [](uint32_t prm) { return (float)half_of(prm >> 16) + 1024.0f; };      // -z
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t t = pos0 + 4 * i + g - p0;
        const float z = zero_of(kp[i]), s = (float)half_of(kp[i]);
        // element 8w + 2j in nibble j of the low half, 8w + 2j + 1 of the high half
        uint32_t lo = 0, hi = 0;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            lo |= ((kw[i] >> (4 * x)) & 15u) << (8 * x) | ((kw[i] >> (16 + 4 * x)) & 15u) << (8 * x + 4);
            hi |= ((kw[i] >> (8 + 4 * x)) & 15u) << (8 * x) | ((kw[i] >> (24 + 4 * x)) & 15u) << (8 * x + 4);
        }
        const uint2 a = values_of(lo, z, s), c = values_of(hi, z, s);
        if (there(t)) reinterpret_cast<uint4*>(k_out + ((row0 + t) * Hkv + h) * kD)[w] = make_uint4(a.x, a.y, c.x, c.y);
    }
    const uint32_t vw[4] = {vc.x, vc.y, vc.z, vc.w}, prm[4] = {vp.x, vp.y, vp.z, vp.w};
#pragma unroll
    for (int x = 0; x < 4; ++x) {                                          // token 4 g + x: dword 2u + (x >> 1), half x & 1
        const int64_t t = pos0 + 4 * g + x - p0;
        const float z = zero_of(prm[x]), s = (float)half_of(prm[x]);
#pragma unroll
        for (int u = 0; u < 2; ++u)                                        // elements 4 (w + 16 u) ..
            if (there(t))
                reinterpret_cast<uint2*>(v_out + ((row0 + t) * Hkv + h) * kD)[w + 16 * u] = values_of(vw[2 * u + (x >> 1)] >> (16 * (x & 1)), z, s);
    }
}

// ------------------------------------------------------------------------------------------
// Decode attention over pages.  The arithmetic of a chunk of 32 tokens is that of the contiguous cache's kernel (qoq_kv4.hip): both
// products on the matrix cores, codes unpacked in registers, softmax in place; but the weights' reference follows the values' scales too.
//
// What a sequence's query sees is a list of chunks: those of the sinks, then those of the window (without a window all of them).
// `ns` workgroups stand by for each (sequence, KV head); nwg of them attend, as few as leave each wave `deal` chunks
// at most (all of them if that is not enough), and their waves take the chunks in turn.  Unnormalised sums, references and weight sums meet in the workspace; the last workgroup to
// arrive adds them up, in the order of the workgroups whichever arrives when, and leaves the counter at zero.
//
// The second product's operand is weight x value scale in FP16: off by 2^-11 of itself, or by 2^-39 of the largest weight x scale where that is
// more (a lane's largest weight times its largest scale, of four or eight tokens at a time, or 2^-15 where that is less: a subnormal scale's exponent
// no longer tells its size).
//
// Bound by memory where there are pairs enough, 64 x 1024 tokens of 32 heads 39 us (5.4 TB/s); else by the trips to memory one after the
// other: table, page, a wave's chunks, and the join's (parts out, counter, parts in: about 4 us); 8192 tokens of 8 KV heads 10.7 us, 40 tokens 4.0.
// ------------------------------------------------------------------------------------------
constexpr int kPartial = kD + 4;                         // floats per head: 128 sums, their reference, the weight sum (rows of 16 bytes)
constexpr int kChunk = 32;                               // tokens per chunk: two tiles of 16 (divides the page)
constexpr int kMaxRatio = 16;                            // query heads per KV head: the columns of one matrix instruction
constexpr int kWaves = 4;                                // of a workgroup
// Chunks per wave up to which one workgroup attends alone: the join costs as much.  8 x 300 tokens of 64 / 8 heads 5.4 us alone, 8.1 shared;
// 1000 tokens of 8 or 32 KV heads 8.8 alone, 7.5 and 8.0 shared.
constexpr int kAlone = 5;
constexpr int kInFlight = 8;                             // sums of a thread of the join
constexpr int kMaxSplits = 64;                           // workgroups to a (sequence, KV head): the lanes of a wave

struct DecodeTail {                                      // arguments that are not needed at once
    const __half* q;
    __half* out;
    int* counters;
    float* parts;
    int64_t q_stride;
    int R, sinks;
};

// pages are addressed by a base in scalar registers, which comes out of the block table, and a lane's offset
typedef const __attribute__((address_space(1))) uint8_t* global_bytes;
typedef const __attribute__((address_space(1))) u32x4* global_u32x4;
typedef unsigned short us2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float4 load_part(const float* at)
{
    const v4i v = load_through(reinterpret_cast<const int4*>(at));
    return make_float4(__int_as_float(v.x), __int_as_float(v.y), __int_as_float(v.z), __int_as_float(v.w));
}

template <int PK, bool NT>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(3))) void paged_decode_kernel(
    const uint8_t* __restrict__ pool, const int32_t* __restrict__ table, const int32_t* __restrict__ seq_lens, uint32_t pages, int width,
    int Hkv, int ns, int window, DecodeTail p)
{
    extern __shared__ __align__(16) float s_part[];      // [wave][column][kPartial], then as the join needs it
    __shared__ int s_last;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, kb = lane >> 4;
    const int R = p.R, head = PK == 2 ? r16 & 7 : r16;
    const bool second = PK == 2 && r16 >= 8;
    const uint32_t bh = blockIdx.x, b = bh / (uint32_t)Hkv, hk = bh - b * (uint32_t)Hkv;
    const int split = blockIdx.y;

    const int32_t* pages_of = table + (int64_t)b * width;
    const int i0 = split * kWaves + wave;                    // without a window the wave's first chunk, whose page is looked up beside the length
    const uint32_t first_id = window ? 0u : (uint32_t)pages_of[min(i0, 2 * width - 1) >> 1];
    struct Chunk {
        uint4 kc[2];        // keys: token r16 of the tile, elements 32 kb ..
        uint4 vc[2];        // values: this lane's 16 bytes of the tile
        uint32_t kz[2];     // (s, z) of token r16 (zero point for unpacking)
        uint4 ks[2 / PK];   // (s, z) of tokens 4 kb .. 4 kb + 3 (scales of the scores this lane keeps)
        uint4 vp[2];        // (s, z) of tokens 4 kb .. 4 kb + 3 of the values
    };
    uint32_t off_kc = (uint32_t)(r16 * (kD / 2) + kb * 16), off_kz = (uint32_t)(kCodeBytes + r16 * 4);
    uint32_t off_ks = (uint32_t)(kCodeBytes + kb * 16 + (second ? 64 : 0)), off_vc = (uint32_t)(kHalfPage + lane * 16);
    uint32_t off_vp = (uint32_t)(kHalfPage + kCodeBytes + kb * 16);
    auto words = [](global_bytes at) __attribute__((always_inline)) { return __builtin_bit_cast(uint4, *(global_u32x4)at); };
    auto code_words = [&](global_bytes at) __attribute__((always_inline)) {
        return NT ? __builtin_bit_cast(uint4, __builtin_nontemporal_load((global_u32x4)at)) : words(at);
    };
    auto load_chunk = [&](Chunk& c, int chunk, uint32_t id) __attribute__((always_inline)) {
        const uint32_t held = id < pages ? id : 0;                       // (no page: any, and nothing of it counts)
        const auto page = (global_bytes)(uintptr_t)to_sgpr(pool + ((int64_t)held * Hkv + hk) * kPageBytes);
        const int tin = (chunk & 1) * kChunk;
        const auto codes = page + tin * (kD / 2), prm = page + tin * 4;
        // (extended to 64 bits outside the loop, the offsets would take register pairs and an addition for each load)
        asm("" : "+v"(off_kc), "+v"(off_kz), "+v"(off_ks), "+v"(off_vc), "+v"(off_vp));
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            c.kc[tt] = code_words(codes + tt * 1024 + off_kc);
            c.kz[tt] = *(const __attribute__((address_space(1))) uint32_t*)(prm + tt * 64 + off_kz);
            if (tt < 2 / PK) c.ks[tt] = words(prm + tt * 64 + off_ks);
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            c.vc[tt] = code_words(codes + tt * 1024 + off_vc);
            c.vp[tt] = words(prm + tt * 64 + off_vp);
        }
    };
    Chunk A, Bf;
    // what is seen: tokens below `sinks`, and from `lo` to L
    const int L = min(max(seq_lens[b], 0), width * kPageTokens);
    const int lo = window ? max(L - window, 0) : 0, sinks = p.sinks;
    const int chunks = (L + kChunk - 1) / kChunk;
    const int n_first = min((sinks + kChunk - 1) / kChunk, chunks);        // chunks of the sinks
    const int gap = max(lo / kChunk - n_first, 0);                         // chunks behind them that nothing sees
    const int n = chunks - gap;                                            // the list: i < n_first ? i : i + gap
    // more workgroups shorten the waves' chains and lengthen the join: chunks to a wave grow with the root of their number
    // (8192 tokens of 8 KV heads 10.6 us; 1 to a wave 12.5, 6 11.2; 32000 of one KV head 22.9; 1 to a wave 27.5)
    const int deal = max(2, (int)(__builtin_sqrtf((float)n) * 0.25f));
    const int nwg = n <= kAlone * kWaves ? 1 : min(ns, (n + kWaves * deal - 1) / (kWaves * deal));
    if (split >= nwg) return;
    __half* out_bh = p.out + (size_t)bh * R * kD;
    if (n == 0) {
        for (int x = threadIdx.x; x < R * kD; x += 64 * kWaves) out_bh[x] = __float2half_rn(0.f);
        return;
    }
    const int stride = nwg * kWaves;
    const int n_iter = i0 < n ? (n - i0 + stride - 1) / stride : 0;

    auto chunk_of = [&](int it) __attribute__((always_inline)) {           // of the wave's it-th turn, or its last
        const int i = min(i0 + max(min(it, n_iter - 1), 0) * stride, n - 1);
        return __builtin_amdgcn_readfirstlane(i < n_first ? i : i + gap);
    };
    auto page_of = [&](int it) __attribute__((always_inline)) { return (uint32_t)pages_of[chunk_of(it) >> 1]; };
    uint32_t id_a = window ? page_of(0) : first_id, id_b = page_of(1);
    load_chunk(A, chunk_of(0), id_a);

    // B operand of S = K q^T: column = head (both halves of the columns with PK = 2; heads >= R: zero), k-block kb = elements 32 kb ..
    uint4 qv[4];
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_stride + ((int)hk * R + min(head, R - 1)) * kD + kb * 32);
        const uint32_t some = head < R ? ~0u : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint4 t = src[e];
            qv[e] = make_uint4(t.x & some, t.y & some, t.z & some, t.w & some);
        }
    }

    // of this lane's column, over the tokens it has seen: the reference that scores are taken from before they become weights, and the weights'
    // sum.  It follows the largest (score + exponent of the value's scale): weight x scale, which is rounded to FP16 for the matrix cores, then has
    // its largest numbers below 2^15 whatever the values' size, and 29 binades lie between those and the first that loses bits.  (37 x 700 10.2 us
    // without the scales, 10.5 with them, 64 x 4000 39.3 and 39.6, 8192 tokens 10.8 and 10.9.)
    float m = -1e29f, l = 0.f;
    f4 acc[8];                                           // acc[4u + j][x]: element d = 16 kb + 4x + 64u + j of the column
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[i] = (f4){0.f, 0.f, 0.f, 0.f};
    const float kScale = 1.4426950408889634f * 0.08838834764831845f;      // log2(e) / sqrt(128)
    const h2 k960 = {(_Float16)960.0f, (_Float16)960.0f};

    // A chunk of which not every token is seen: the parameters of the others are whatever the cache holds and must not enter the
    // arithmetic.  Their codes become small numbers, their scales zero, and their scores fall to -1e30 by `bias`, whose weight is 0
    // against any maximum (which starts at -1e29).
    auto hide = [&](Chunk& cur, int chunk, bool held, f4 (&bias)[2 / PK]) __attribute__((always_inline)) {
        const int end = held ? L : 0, end_first = held ? sinks : 0;
        auto seen = [&](int t) { return t < end && (t >= lo || t < end_first); };
        auto kept = [&](uint4 v, int t, uint32_t none) {                   // parameters of tokens t .. t + 3
            return make_uint4(seen(t) ? v.x : none, seen(t + 1) ? v.y : none, seen(t + 2) ? v.z : none, seen(t + 3) ? v.w : none);
        };
        const int t0 = chunk * kChunk;
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            cur.kz[tt] = seen(t0 + tt * 16 + r16) ? cur.kz[tt] : 0xE4000000u;                     // -(1024 + 0)
            cur.vp[tt] = kept(cur.vp[tt], t0 + tt * 16 + 4 * kb, 0xE4000000u);
        }
#pragma unroll
        for (int tt = 0; tt < 2 / PK; ++tt) {
            const int t = t0 + (second ? 16 : 0) + tt * 16 + 4 * kb;
            cur.ks[tt] = kept(cur.ks[tt], t, 0u);
#pragma unroll
            for (int x = 0; x < 4; ++x) bias[tt][x] = seen(t + x) ? 0.f : -1e30f;
        }
    };
    auto process = [&](Chunk& cur, int it, uint32_t id) __attribute__((always_inline)) {
        constexpr int NS = 2 / PK;
        const int chunk = chunk_of(it);
        f4 bias[NS];
#pragma unroll
        for (int tt = 0; tt < NS; ++tt) bias[tt] = (f4){0.f, 0.f, 0.f, 0.f};
        if (!(id < pages && chunk * kChunk + kChunk <= L && (chunk * kChunk >= lo || chunk * kChunk + kChunk <= sinks)))
            hide(cur, chunk, id < pages, bias);
        f4 d[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const uint32_t kz = cur.kz[tt];
            const h2 c = __builtin_bit_cast(h2, __builtin_amdgcn_perm(kz, kz, 0x07060706u));   // high half in both halves
            const h2 c16 = c + k960;
            const uint32_t kw[4] = {cur.kc[tt].x, cur.kc[tt].y, cur.kc[tt].z, cur.kc[tt].w};
            d[tt] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                h2 kh[4];
                unpack4(kw[w], c, c16, kh);              // kh[j] = elements 8w + 2j, 8w + 2j + 1 of this lane's 32
                d[tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(kh[0], kh[1], kh[2], kh[3]),
                                                               __builtin_bit_cast(h8, qv[w]), d[tt], 0, 0, 0);
            }
        }
        f4 sc[NS];                                       // [x] = token 4 kb + x of the lane's tile (of both tiles with PK = 1)
        if (PK == 2) {
#pragma unroll
            for (int x = 0; x < 4; ++x) sc[0][x] = second ? d[1][x] : d[0][x];
        } else {
#pragma unroll
            for (int tt = 0; tt < NS; ++tt) sc[tt] = d[tt];
        }
        uint32_t pw[NS][4];                              // parameters of the values of the tokens whose scores this lane keeps
#pragma unroll
        for (int tt = 0; tt < NS; ++tt) {
            const uint4 a = PK == 2 && second ? cur.vp[1] : cur.vp[tt];
            pw[tt][0] = a.x; pw[tt][1] = a.y; pw[tt][2] = a.z; pw[tt][3] = a.w;
        }
        float top = -1e30f;
        us2 largest = {0, 0};
#pragma unroll
        for (int tt = 0; tt < NS; ++tt) {
            const uint32_t sw[4] = {cur.ks[tt].x, cur.ks[tt].y, cur.ks[tt].z, cur.ks[tt].w};
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                sc[tt][x] = fmaf(sc[tt][x], (float)half_of(sw[x]) * kScale, bias[tt][x]);
                top = fmaxf(top, sc[tt][x]);
                largest = __builtin_elementwise_max(largest, __builtin_bit_cast(us2, pw[tt][x]));
            }
        }
        // the largest scale is below 2^(its exponent's bits - 14), so with this reference weight x scale stays below 2^15
        // (where FP32 no longer holds a score's units, the sum would be rounded by more than there is room: the score itself)
        const float below = fabsf(top) < 0x1p23f ? (float)((largest.x >> 10) & 31u) - 29.f : 0.f;
        // the four k-blocks of a column agree on the reference
        const float m_new = max_other_half(max_other_row(fmaxf(m, top + below)));
        if (__builtin_amdgcn_ballot_w64(m_new != m) != 0) {                  // rare once a few chunks have been seen
            const float alpha = __builtin_amdgcn_exp2f(m - m_new);
            m = m_new;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] *= alpha;
        }
        uint32_t bw[2][2];                               // B operand: softmax weight * value scale, tokens 4 kb .. of both tiles
#pragma unroll
        for (int tt = 0; tt < NS; ++tt) {
            float wf[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
                const float pr = __builtin_amdgcn_exp2f(sc[tt][x] - m);
                l += pr;
                wf[x] = pr * (float)half_of(pw[tt][x]);
            }
            const uint32_t b_lo = __builtin_bit_cast(uint32_t, (h2){(_Float16)wf[0], (_Float16)wf[1]});
            const uint32_t b_hi = __builtin_bit_cast(uint32_t, (h2){(_Float16)wf[2], (_Float16)wf[3]});
            if (PK == 2) {                               // a column takes part with its own tile only
                bw[0][0] = second ? 0u : b_lo; bw[0][1] = second ? 0u : b_hi;
                bw[1][0] = second ? b_lo : 0u; bw[1][1] = second ? b_hi : 0u;
            } else {
                bw[tt][0] = b_lo; bw[tt][1] = b_hi;
            }
        }
        h2 cz[2][2], cz16[2][2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const uint32_t zw[4] = {cur.vp[tt].x, cur.vp[tt].y, cur.vp[tt].z, cur.vp[tt].w};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                cz[tt][h] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(zw[2 * h + 1], zw[2 * h], 0x07060302u));
                cz16[tt][h] = cz[tt][h] + k960;
            }
        }
        const h8 b8 = join(__builtin_bit_cast(h2, bw[0][0]), __builtin_bit_cast(h2, bw[0][1]), __builtin_bit_cast(h2, bw[1][0]),
                           __builtin_bit_cast(h2, bw[1][1]));
#pragma unroll
        for (int u = 0; u < 2; ++u) {                    // (one half of the elements after the other: registers)
            __builtin_amdgcn_sched_barrier(0);
            h2 vh[2][2][4];                              // [tile][h][j]: (token 4 kb + 2h, + 1) of element 4 (r16 + 16 u) + j
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const uint32_t vw[4] = {cur.vc[tt].x, cur.vc[tt].y, cur.vc[tt].z, cur.vc[tt].w};
#pragma unroll
                for (int h = 0; h < 2; ++h) unpack4(vw[2 * u + h], cz[tt][h], cz16[tt][h], vh[tt][h]);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[4 * u + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(join(vh[0][0][j], vh[0][1][j], vh[1][0][j], vh[1][1][j]), b8, acc[4 * u + j], 0, 0, 0);
        }
    };

    // Two copies of the arithmetic and no more: a call on short sequences runs through its code once, and pays for fetching it.  The wave's
    // last turn therefore requests its own chunk again (which is in the caches), as does a wave without chunks the list's last.
    int it = 0;
    for (; it + 2 < n_iter; it += 2) {
        load_chunk(Bf, chunk_of(it + 1), id_b);
        const uint32_t now = id_a;
        id_a = page_of(it + 2);
        process(A, it, now);
        load_chunk(A, chunk_of(it + 2), id_a);
        const uint32_t then = id_b;
        id_b = page_of(it + 3);
        process(Bf, it + 1, then);
    }
    if (it + 2 == n_iter) {
        load_chunk(Bf, chunk_of(it + 1), id_b);
        process(A, it, id_a);
        process(Bf, it + 1, id_b);
    } else if (n_iter > 0) {
        process(A, it, id_a);
    }

    // ---- the partial results of the waves (and of the column halves) meet in LDS --------------
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    const int columns = PK * R;
    if (head < R) {
        float* part = s_part + (wave * columns + (second ? R : 0) + head) * kPartial;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                *reinterpret_cast<float4*>(part + 16 * kb + 4 * x + 64 * u) = make_float4(acc[4 * u][x], acc[4 * u + 1][x], acc[4 * u + 2][x], acc[4 * u + 3][x]);
        if (kb == 0) *reinterpret_cast<float2*>(part + kD) = make_float2(m, l);
    }
    __syncthreads();
    constexpr int N = kWaves * PK;                           // partial results of a head
    const int n4 = R * (kD / 4);                         // results, four elements each
    float* mine = p.parts + ((size_t)bh * ns + split) * R * kPartial;
    auto write_out = [&](int x, float4 num, float den) {
        float inv = den > 0.f ? 1.f / den : 1.f;         // nothing seen: zero, as the sums are (NaN stays)
        if (den == 0.f)                                  // tokens seen all the same: their scores are minus infinity, and this is no softmax
            for (int i = 0; i < n; ++i)
                if ((uint32_t)pages_of[(i < n_first ? i : i + gap) >> 1] < pages) {
                    inv = __builtin_nanf("");
                    break;
                }
        const h2 a = {(_Float16)(num.x * inv), (_Float16)(num.y * inv)}, c = {(_Float16)(num.z * inv), (_Float16)(num.w * inv)};
        reinterpret_cast<uint2*>(out_bh)[x] = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c));
    };
    for (int x = threadIdx.x; x < n4; x += 64 * kWaves) {
        const int r = x / (kD / 4), d = x % (kD / 4) * 4;
        const float* part = s_part + r * kPartial;
        float mm = -1e29f;
#pragma unroll
        for (int i = 0; i < N; ++i) mm = fmaxf(mm, part[i * R * kPartial + kD]);
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        float den = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float2 ml = *reinterpret_cast<const float2*>(part + i * R * kPartial + kD);
            const float4 a = *reinterpret_cast<const float4*>(part + i * R * kPartial + d);
            const float f = __builtin_amdgcn_exp2f(ml.x - mm);
            num.x = fmaf(a.x, f, num.x); num.y = fmaf(a.y, f, num.y); num.z = fmaf(a.z, f, num.z); num.w = fmaf(a.w, f, num.w);
            den = fmaf(ml.y, f, den);
        }
        if (nwg == 1) {
            write_out(x, num, den);
        } else {
            auto put = [&](int at, float4 v) {
                store_through(reinterpret_cast<int4*>(mine + r * kPartial + at), __float_as_int(v.x), __float_as_int(v.y), __float_as_int(v.z), __float_as_int(v.w));
            };
            put(d, num);
            if (d == 0) put(kD, make_float4(mm, den, 0.f, 0.f));
        }
    }
    if (nwg == 1) return;
    // The stores above went past the caches that other workgroups do not share; they have arrived when the counter is raised.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0) {
        const int old = __hip_atomic_fetch_add(p.counters + bh, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = old == nwg - 1;
        if (old == nwg - 1) __hip_atomic_store(p.counters + bh, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    __syncthreads();
    if (!s_last) return;
    // The join: `groups` groups of n4 threads take the workgroups' sums in turn, kInFlight in flight beside the
    // maxima; the groups' own sums meet in LDS.
    const float* parts = p.parts + (size_t)bh * ns * R * kPartial;
    float* s_factor = s_part;                            // [nwg][R]: 2^(reference - the largest)
    float* s_den = s_factor + kMaxSplits * kMaxRatio;    // [R]
    float4* s_sum = reinterpret_cast<float4*>(s_den + kMaxRatio);          // [groups][n4]
    const int groups = max(1, 64 * kWaves / n4);
    const int g0 = groups > 1 ? (int)threadIdx.x / n4 : 0;
    int x = groups > 1 ? (int)threadIdx.x - g0 * n4 : (int)threadIdx.x, s0 = g0;
    bool some = g0 < groups && x < n4;
    float4 a[kInFlight];
    auto fetch = [&]() __attribute__((always_inline)) {
        const float* at = parts + (size_t)(some ? x / (kD / 4) : 0) * kPartial + (some ? x % (kD / 4) * 4 : 0);
#pragma unroll
        for (int i = 0; i < kInFlight; ++i) {
            a[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s0 + i * groups < nwg) a[i] = load_part(at + (size_t)(s0 + i * groups) * R * kPartial);
        }
    };
    unsigned long long ml[kMaxRatio / kWaves];           // a wave per head, a lane per workgroup: reference and weight sum
#pragma unroll
    for (int i = 0; i < kMaxRatio / kWaves; ++i)
        ml[i] = __hip_atomic_load(reinterpret_cast<unsigned long long*>(const_cast<float*>(parts) + ((size_t)min(lane, nwg - 1) * R + min(wave + i * kWaves, R - 1)) * kPartial + kD),
                                  __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    fetch();
#pragma unroll
    for (int i = 0; i < kMaxRatio / kWaves; ++i) {
        const int r = wave + i * kWaves;
        if (r >= R) break;
        const float ms = __uint_as_float((uint32_t)ml[i]);
        float top = ms;
#pragma unroll
        for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
        const float f = lane < nwg ? __builtin_amdgcn_exp2f(ms - top) : 0.f;
        float den = lane < nwg ? __uint_as_float((uint32_t)(ml[i] >> 32)) * f : 0.f;
#pragma unroll
        for (int o = 32; o; o >>= 1) den += __shfl_xor(den, o, 64);
        s_factor[lane * R + r] = f;
        if (lane == 0) s_den[r] = den;
    }
    __syncthreads();
    while (true) {                                       // (once, unless a KV head serves more heads than the threads have sums for)
        const int r = some ? x / (kD / 4) : 0;
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        while (true) {
#pragma unroll
            for (int i = 0; i < kInFlight; ++i) {
                const int s = s0 + i * groups;
                const float f = s < nwg ? s_factor[s * R + r] : 0.f;
                num.x = fmaf(a[i].x, f, num.x); num.y = fmaf(a[i].y, f, num.y); num.z = fmaf(a[i].z, f, num.z); num.w = fmaf(a[i].w, f, num.w);
            }
            s0 += kInFlight * groups;
            if (s0 >= nwg) break;
            fetch();
        }
        if (groups > 1) {
            if (some) s_sum[g0 * n4 + x] = num;
            break;
        }
        if (some) write_out(x, num, s_den[r]);
        x += 64 * kWaves;
        s0 = 0;
        some = x < n4;
        if (!some) return;
        fetch();
    }
    __syncthreads();
    for (int y = threadIdx.x; y < n4; y += 64 * kWaves) {
        float4 num = s_sum[y];
        for (int g = 1; g < groups; ++g) {
            const float4 c = s_sum[g * n4 + y];
            num.x += c.x; num.y += c.y; num.z += c.z; num.w += c.w;
        }
        write_out(y, num, s_den[y / (kD / 4)]);
    }
}

}  // namespace

int64_t kv4_page_bytes(int64_t Hkv) { return Hkv * kPageBytes; }

constexpr int64_t kFill = 1024;                          // (5 x 1733 tokens of 64 / 8 heads 53.6 us, with 4096 56.5; 1 x 1000 of 32 heads 15.3 and 20.3)
hipError_t launch_rope_append(const RopeAppend& a, hipStream_t s)
{
    AppendArgs p{};
    p.q = static_cast<const __half*>(a.q); p.k = static_cast<const __half*>(a.k); p.v = static_cast<const __half*>(a.v);
    p.q_stride = a.q_stride; p.k_stride = a.k_stride; p.v_stride = a.v_stride;
    p.q_gamma = static_cast<const __half*>(a.q_gamma); p.k_gamma = static_cast<const __half*>(a.k_gamma);
    p.eps = a.eps;
    p.angles = a.angles; p.angle_rows = (int)a.angle_rows; p.rot = (int)a.rot; p.interleaved = a.interleaved;
    p.cu = a.cu; p.starts = a.starts;
    p.M = (int)a.M; p.B = (int)a.B; p.H = (int)a.H; p.Hkv = (int)a.Hkv;
    p.pool = a.pool; p.pages = (uint32_t)a.pages; p.table = a.table; p.width = (int)a.width;
    p.q_out = static_cast<__half*>(a.q_out); p.k_out = static_cast<__half*>(a.k_out);
    p.q_out_stride = a.q_out_stride; p.k_out_stride = a.k_out_stride;
    const int64_t slots = a.M / 4 + 2 * a.B;             // a sequence of T tokens touches at most (T + 2) / 4 + 1 aligned quads
    const int64_t quads = (a.M + 3) / 4;
    // heads to a wave: as many as leave kFill waves, since they share the look-up of the rows and the angles
    auto heads_to_a_wave = [](int64_t rows, int64_t heads) {
        uint32_t n = 1;
        while (n < 8 && rows * heads / (2 * n) >= kFill) n *= 2;
        return n;
    };
    p.q_heads = heads_to_a_wave(quads, a.H);
    p.q_groups = (uint32_t)((a.H + p.q_heads - 1) / p.q_heads);
    p.kv_heads = heads_to_a_wave(quads, a.Hkv);
    p.kv_groups = (uint32_t)((a.Hkv + p.kv_heads - 1) / p.kv_heads);
    const int64_t kv_items = slots * p.kv_groups, q_items = p.q ? quads * p.q_groups : 0;
    if (kv_items + q_items > 4 * kMaxGrid) return hipErrorInvalidValue;
    p.kv_items = (uint32_t)kv_items; p.q_items = (uint32_t)q_items;
    auto* kernel = a.rot == kD ? (a.interleaved ? rope_append_kernel<true, true> : rope_append_kernel<false, true>)
                               : (a.interleaved ? rope_append_kernel<true, false> : rope_append_kernel<false, false>);
    kernel<<<(unsigned)((kv_items + q_items + 3) / 4), 256, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_paged_gather(const uint8_t* pool, int64_t pages, const int32_t* table, int64_t width, const int32_t* cu,
                               const int32_t* starts, int64_t M, int64_t B, int64_t Hkv, void* k_out, void* v_out, hipStream_t s)
{
    const int64_t items = (M / 16 + 2 * B) * Hkv;
    if (items > 4 * kMaxGrid) return hipErrorInvalidValue;
    paged_gather_kernel<<<(unsigned)((items + 3) / 4), 256, 0, s>>>(pool, table, cu, starts, static_cast<__half*>(k_out), static_cast<__half*>(v_out),
                                                                     (uint32_t)pages, (int)width, (int)M, (int)B, (int)Hkv, (uint32_t)items);
    return hipGetLastError();
}

// Workgroups that stand by for each (sequence, KV head), and the tokens that a query can see at most.  Two for each compute unit: with three
// 37 x 700 tokens of 64 / 8 heads 12.3 us, 9.9 with two (its 296 pairs then have one each), 4 x 8192 of 32 / 8 14.0 and 13.3, 16 x 32000 through a window of 4096 19.4 and 18.9.
// Lengths are not known here: this rule, and whether codes pass by the caches below, go by the table's width or the window.  Tables of 512 pages a sequence where 5 are
// used were no slower: 8 x 300 of 64 / 8 heads 5.9 us with either, 64 x 300 of 32 heads 21.3 and 23.1, 4 x 4000 of 32 / 8 11.6 and 11.8.
static int64_t most_seen(int64_t width, int64_t window, int64_t sinks)
{
    const int64_t S = width * kPageTokens;
    return window ? std::min(S, window + sinks) : S;
}
static int paged_splits(int64_t B, int64_t Hkv, int64_t width, int64_t window, int64_t sinks)
{
    const int64_t pairs = B * Hkv;
    if (pairs <= 0 || pairs > kMaxCounters) return 1;
    int64_t ns = 512 / pairs;
    ns = std::min<int64_t>(ns, kMaxSplits);
    ns = std::min<int64_t>(ns, (most_seen(width, window, sinks) / kChunk + 2 + 2 * kWaves - 1) / (2 * kWaves));
    if (most_seen(width, window, sinks) / kChunk + 2 <= kAlone * kWaves) return 1;
    return (int)std::max<int64_t>(ns, 1);
}

size_t paged_decode_workspace_bytes(int64_t B, int64_t H, int64_t Hkv, int64_t width, int64_t window, int64_t sinks)
{
    const int ns = paged_splits(B, Hkv, width, window, sinks);
    return ns <= 1 ? 0 : kCounterBytes + ((size_t)(B * H) * ns * kPartial * sizeof(float) + 15) / 16 * 16;
}

hipError_t launch_paged_decode(const void* q, int64_t q_stride, const uint8_t* pool, int64_t pages, const int32_t* table, int64_t width,
                               const int32_t* seq_lens, int64_t B, int64_t H, int64_t Hkv, int64_t window, int64_t sinks, void* out,
                               void* workspace, hipStream_t s)
{
    DecodeTail p{};
    p.q = static_cast<const __half*>(q); p.q_stride = q_stride;
    p.out = static_cast<__half*>(out);
    p.R = (int)(H / Hkv);
    p.sinks = window ? (int)sinks : 0;
    p.counters = static_cast<int*>(workspace);
    p.parts = workspace ? reinterpret_cast<float*>(static_cast<char*>(workspace) + kCounterBytes) : nullptr;
    const int ns = workspace ? paged_splits(B, Hkv, width, window, sinks) : 1;
    // Codes past the caches where a call reads more than stays in them: 16 x 32000 tokens of 8 KV heads through a window of 4096 (71 MB) 18.5 us,
    // 20.0 through them, 64 x 4000 (279 MB) 39 and 44; level at 27 and 36 MB, slower where the memory-side cache still holds a call's codes
    // (64 x 300 of 32 heads, three caches in turn, 17.5 and 16.5; nine in turn 18.0 and 18.9).
    const bool nt = B * Hkv * most_seen(width, window, sinks) / kPageTokens * kPageBytes >= (int64_t)24 << 20;
    if (B * Hkv > kMaxGrid) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(B * Hkv), (unsigned)ns);
    // Up to eight heads to a KV head, two tiles of tokens share the columns: half of the softmax's instructions for more code.  64 x 4000 tokens of
    // 32 / 8 heads 39.0 us, a tile at a time 39.8, 16 x 8192 26.2 and 27.0; short sequences lose 0.2.
    const int PK = p.R <= 8 ? 2 : 1;
    const size_t lds = std::max((size_t)kWaves * PK * p.R * kPartial * sizeof(float), (kMaxSplits + 1) * kMaxRatio * sizeof(float) + 64 * kWaves * sizeof(float4));
    auto* kernel = PK == 2 ? (nt ? paged_decode_kernel<2, true> : paged_decode_kernel<2, false>)
                           : (nt ? paged_decode_kernel<1, true> : paged_decode_kernel<1, false>);
    kernel<<<grid, 64 * kWaves, lds, s>>>(pool, table, seq_lens, (uint32_t)pages, (int)width, (int)Hkv, ns, (int)window, p);
    return hipGetLastError();
}

}  // namespace qoq
