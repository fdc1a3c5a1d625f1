// Decode attention over the paged 4-bit cache for a batch whose sequences share prefixes: one query token for each sequence,
//   out[b, h] = softmax_t( q[b, h] . K^[t] / sqrt(D) ) V^[t],  t < L_b,
// where tokens t < P_g of a sequence of group g lie in the pages of the group's first sequence, the others in its own.
//
// The columns of a matrix instruction are 16 query vectors; over a sequence's own tokens those are the heads of a KV head, over a
// prefix the heads of all the group's sequences.  So a wave takes 16 CT columns through a chunk of 32 tokens whose codes it unpacks once: a
// prefix is read, and unpacked, once for 16 CT / R sequences, and a workgroup for as many columns of the same KV head finds it in the L2 of its
// chiplet (workgroups of one KV head are 8 apart where the heads are a multiple of 8).
//
// One launch attends, with workgroups for both kinds of work side by side, each writing unnormalised sums, references and weight sums of
// its range of tokens; a second one joins those of each head.  Where the sequences alone fill the chip, the first launch is the prefixes' and the
// second that of the own tokens, which joins.  The arithmetic of a chunk and the weights' reference are those of the
// paged decode kernel (qoq_kv4_paged.hip).
//
// A prefix of many columns is bound by the vector unit beside the matrix unit: 200 sequences of 64 / 8 heads with 100 tokens behind 16000 take 187 us, 0.56
// PFLOP/s, in which the matrix unit is busy for 0.26 of the cycles and the vector unit for 0.49 (exp2, weights, FP16).  Short ones are bound
// by the chain of trips to memory: 4 sequences with 30 tokens behind 1000 10.7 us, 7.8 and 3.6 for the join by a profiler.
//
// Without groups (every sequence reads its prefix itself, qoq_kv4_paged.hip) these two take 432 and 8.1 us: a second launch costs some 3, and columns cost
// arithmetic.  In one group the call is ahead from about 500 000 sequences x tokens of the prefix x KV heads on where a KV head has up to four query
// heads (16 behind 4096 of 32 / 8 heads 15.2 and 17.2, 8 behind 1000 of 32 / 32 10.9 and 12.5; 16 behind 1000 of 32 / 8 11.5 and 10.1), from 2 000 000 on
// where it has eight (64 behind 4096 of 64 / 8 37.3 and 42.7, behind 1000 21.1 and 15.6).
#include <algorithm>

#include "qoq_gemm_common.h"
#include "qoq_kv4_common.h"

namespace qoq {
namespace {

constexpr int kPartial = kD + 4;                         // floats of a part: 128 sums, their reference, the weight sum (rows of 16 bytes)
constexpr int kChunk = 32;                               // tokens: two tiles of 16 (divides the page)
constexpr int kWaves = 4;                                // of a workgroup
constexpr int kMaxParts = 64;                            // of a prefix, and of a sequence's own tokens
constexpr int kInFlight = 8;                             // parts that the join requests together
constexpr int kOwnInFlight = 4;                          // the same where it is part of the work on a sequence's own tokens
constexpr int kColumnTiles = 2;                          // of 16 columns for each wave, over a prefix
constexpr int kPrefixColumns = 16 * kColumnTiles;
constexpr int kWide = 2;                                 // the same where a prefix's columns are many and a workgroup's waves have columns of their own
constexpr int kWideWorkgroups = 512;                     // that share the prefixes then: two on a compute unit
constexpr int kLeastRun = 4;                             // pages of a run
// Units of the wide form (a page for 128 columns) from which it is taken, where no column of a tile is empty: about 24 us and 6.5 ns a unit, and about 15 and
// 10.5 ns for each 128 columns where waves share the tokens (its pages go through LDS one after the other, and a run's first costs three).  64
// sequences of 32 / 8 heads behind 8000 tokens (2000 units) 36.8 and 35.1 us, behind 16000 49.6 and 57.6; 151 of 40 / 8 behind 2000 (1536) 41.0 and 35.7,
// behind 4000 47.7 and 54.8; five groups of 13 of 28 / 4 behind 14485 (4540, of which 0.29 empty) 49.2 and 45.0, four of 17 of 32 / 8 behind 16000 (8000, 0.47)
// 65.5 and 53.7.  Only the device knows the prefixes' lengths.
constexpr int kWideUnits = 2250;

struct SharedArgs {
    const uint8_t* pool;
    const int32_t *table, *seq_lens, *cu, *prefix_lens;
    const __half* q;
    float* parts;                                        // [B][H][prefix_parts + own_parts][kPartial]
    __half* out;
    int64_t q_stride;
    uint32_t pages;
    int width, B, G, Hkv, R;
    int prefix_slots, own_parts;                         // slots of a head for its prefix, and for its own tokens
    int prefix_parts, wide_parts;                        // of a tile of columns of a prefix, by the waves' way of sharing it
    int prefix_workgroups;                               // of the wide form
    uint32_t prefix_blocks, ratio_magic;                 // ceil(2^32 / R)
};
// n / R for n < 2^28
__device__ __forceinline__ int by_ratio(const SharedArgs& p, int n) { return p.R == 1 ? n : (int)__umulhi((uint32_t)n, p.ratio_magic); }

typedef const __attribute__((address_space(1))) uint8_t* global_bytes;
typedef const __attribute__((address_space(1))) u32x4* global_u32x4;
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef unsigned short us2 __attribute__((ext_vector_type(2)));
// the block table, which no kernel here writes: entries at addresses that a wave shares come through the scalar cache, and only their use waits
typedef const __attribute__((address_space(4))) int32_t* constant_ints;
__device__ __forceinline__ constant_ints constant(const int32_t* at) { return (constant_ints)(uintptr_t)at; }

// Workgroups that attend to `chunks` chunks, of the `parts` that stand by: as few as leave each wave two, if there are that many.
__device__ __forceinline__ int attending(int chunks, int parts) { return min(parts, (chunks + 2 * kWaves - 1) / (2 * kWaves)); }

// Group of sequence b with a prefix: its prefix's tokens (0: none).  The 64 lanes look together.
__device__ __forceinline__ int prefix_of(const SharedArgs& p, int b, int lane)
{
    for (int g0 = 0; g0 < p.G; g0 += 64) {
        const int g = g0 + lane;
        int n = 0;
        bool in = false;
        if (g < p.G) {
            in = p.cu[g] <= b && b < p.cu[g + 1];
            n = min(max(p.prefix_lens[g], 0), p.width * kPageTokens);
        }
        const unsigned long long who = __builtin_amdgcn_ballot_w64(in);
        if (who) return __builtin_amdgcn_readfirstlane(__shfl(n, __builtin_ctzll(who), 64));
    }
    return 0;
}

// 1 / the weights' sum of sequence b, of whose L tokens P lie in front of its prefix's end.  Without a weight: a sequence that sees nothing has a zero row,
// as its sums are; one that does has scores of minus infinity only, and NaN.  (Looked up then: no other call pays for it.)
__device__ __forceinline__ float inverse_sum(const SharedArgs& p, float den, int b, int L, int P)
{
    if (den != 0.f || L == 0) return den > 0.f ? 1.f / den : 1.f;           // (a NaN stays)
    int first = b;
    for (int g = 0; P > 0 && g < p.G; ++g)
        if (p.cu[g] <= b && b < p.cu[g + 1]) {
            first = max(p.cu[g], 0);
            break;
        }
    const int shared = min(P, L);
    for (int i = 0; i < L; i = (i / kPageTokens + 1) * kPageTokens) {
        if (i < shared && (uint32_t)p.table[(int64_t)first * p.width + i / kPageTokens] < p.pages) return __builtin_nanf("");
        if (min((i / kPageTokens + 1) * kPageTokens, L) > shared && (uint32_t)p.table[(int64_t)b * p.width + i / kPageTokens] < p.pages) return __builtin_nanf("");
    }
    return 1.f;
}

// sums over the lanes up to each, in registers
__device__ __forceinline__ int upto_lane(int v)
{
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);       // from 1, 2, 4, 8 lanes back in a row of 16
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);       // the last of rows 0 and 2 into 1 and 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);       // the last of row 1 into 2 and 3
    return v;
}
__device__ __forceinline__ int largest_upto_lane(int v)                   // (of numbers that are not negative)
{
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false));
    return v;
}
__device__ __forceinline__ int largest_of_lanes(int v) { return __builtin_amdgcn_readlane(largest_upto_lane(v), 63); }

struct Work {
    const int32_t* pages_of;                             // the block table's row
    int hk, lo, hi;                                      // KV head; tokens lo .. hi - 1
    int part, parts;                                     // this workgroup among those that attend
    int first, column0, columns;                         // column c is head (column0 + c) % R of sequence first + (column0 + c) / R
    int slot;                                            // of the parts
    int total_slots;
    int page, page_end;                                  // of the wide form, in place of part and parts
};

// One workgroup's range of tokens for up to 16 CT columns.  PK = 2: two tiles of tokens share the columns of a matrix instruction (at most
// eight columns).  LIMITS: columns may end in front of `hi`, each at its sequence's length.  finish(row, d, sums, reference, weight sum) takes four
// elements of a column's result each.
template <int CT, int PK, bool LIMITS, class Finish>
__device__ __forceinline__ void attend(const SharedArgs& p, const Work& k, float* s_part, Finish finish)
{
    constexpr int NS = 2 / PK;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, kb = lane >> 4;
    const bool second = PK == 2 && r16 >= 8;
    const int R = p.R;

    struct Chunk {
        uint4 kc[2];        // keys: token r16 of the tile, elements 32 kb ..
        uint4 vc[2];        // values: this lane's 16 bytes of the tile
        uint32_t kz[2];     // (s, z) of token r16 (zero point for unpacking)
        uint4 ks[NS];       // (s, z) of tokens 4 kb .. 4 kb + 3 (scales of the scores this lane keeps)
        uint4 vp[2];        // (s, z) of tokens 4 kb .. 4 kb + 3 of the values
    };
    uint32_t off_kc = (uint32_t)(r16 * (kD / 2) + kb * 16), off_kz = (uint32_t)(kCodeBytes + r16 * 4);
    uint32_t off_ks = (uint32_t)(kCodeBytes + kb * 16 + (second ? 64 : 0)), off_vc = (uint32_t)(kHalfPage + lane * 16);
    uint32_t off_vp = (uint32_t)(kHalfPage + kCodeBytes + kb * 16);
    auto words = [](global_bytes at) __attribute__((always_inline)) { return __builtin_bit_cast(uint4, *(global_u32x4)at); };
    auto load_chunk = [&](Chunk& c, int chunk, uint32_t id) __attribute__((always_inline)) {
        const uint32_t held = id < p.pages ? id : 0;                     // (no page: any, and nothing of it counts)
        const auto page = (global_bytes)(uintptr_t)to_sgpr(p.pool + ((int64_t)held * p.Hkv + k.hk) * kPageBytes);
        const int tin = (chunk & 1) * kChunk;
        const auto codes = page + tin * (kD / 2), prm = page + tin * 4;
        asm("" : "+v"(off_kc), "+v"(off_kz), "+v"(off_ks), "+v"(off_vc), "+v"(off_vp));
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            c.kc[tt] = words(codes + tt * 1024 + off_kc);
            c.kz[tt] = *(const __attribute__((address_space(1))) uint32_t*)(prm + tt * 64 + off_kz);
            if (tt < NS) c.ks[tt] = words(prm + tt * 64 + off_ks);
        }
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            c.vc[tt] = words(codes + tt * 1024 + off_vc);
            c.vp[tt] = words(prm + tt * 64 + off_vp);
        }
    };

    const int c0 = k.lo / kChunk, n = (k.hi + kChunk - 1) / kChunk - c0;   // the chunks
    const int i0 = k.part * kWaves + wave, stride = k.parts * kWaves;
    const int n_iter = i0 < n ? (n - i0 + stride - 1) / stride : 0;
    auto chunk_of = [&](int it) __attribute__((always_inline)) {           // of the wave's it-th turn, or its last
        return __builtin_amdgcn_readfirstlane(c0 + min(i0 + max(min(it, n_iter - 1), 0) * stride, n - 1));
    };
    auto page_of = [&](int it) __attribute__((always_inline)) { return (uint32_t)constant(k.pages_of)[chunk_of(it) >> 1]; };
    Chunk A, Bf;
    uint32_t id_a = page_of(0), id_b = page_of(1);
    load_chunk(A, chunk_of(0), id_a);

    // B operand of S = K q^T: a lane's column of each tile (none: zeros), k-block kb = elements 32 kb ..
    uint4 qv[CT][4];
    int limit[CT];
    int least = k.hi, most = LIMITS ? 0 : k.hi;          // of the columns' limits: what lies behind all of them need not have been written
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int column = c * 16 + (PK == 2 ? r16 & 7 : r16), held = k.column0 + min(column, k.columns - 1), s = by_ratio(p, held), b = k.first + s;
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_stride + (int64_t)(k.hk * R + held - s * R) * kD + kb * 32);
        const uint32_t some = column < k.columns ? ~0u : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint4 t = src[e];
            qv[c][e] = make_uint4(t.x & some, t.y & some, t.z & some, t.w & some);
        }
        limit[c] = k.hi;
        if (LIMITS) {
            limit[c] = min(max(p.seq_lens[b], 0), k.hi);
            least = min(least, limit[c]);
            most = max(most, limit[c]);
        }
    }
    if (LIMITS) {
        least = k.hi - largest_of_lanes(k.hi - least);
        most = largest_of_lanes(most);
    }

    // of a lane's columns, over the tokens they have seen: the reference that scores are taken from before they become weights, and the weights' sum
    float m[CT], l[CT];
    f4 acc[CT][8];                                       // acc[.][4u + j][x]: element d = 16 kb + 4x + 64u + j of the column
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        m[c] = -1e29f; l[c] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[c][i] = (f4){0.f, 0.f, 0.f, 0.f};
    }
    const float kScale = 1.4426950408889634f * 0.08838834764831845f;      // log2(e) / sqrt(128)
    const h2 k960 = {(_Float16)960.0f, (_Float16)960.0f};

    auto process = [&](Chunk& cur, int it, uint32_t id) __attribute__((always_inline)) {
        const int chunk = chunk_of(it), t0 = chunk * kChunk;
        // A chunk of which not every token is seen by all: parameters of tokens that none sees are whatever the cache holds and must not
        // enter the arithmetic; what a column does not see gets a score of -1e30, whose weight is 0 against any maximum (which starts at
        // -1e29), and a value scale of zero.
        const bool partly = !(id < p.pages && t0 >= k.lo && t0 + kChunk <= least);
        const int lo = k.lo, hi = id < p.pages ? most : 0;
        if (partly) {
            auto held = [&](int t) { return t >= lo && t < hi; };
            auto kept = [&](uint4 v, int t, uint32_t none) {               // parameters of tokens t .. t + 3
                return make_uint4(held(t) ? v.x : none, held(t + 1) ? v.y : none, held(t + 2) ? v.z : none, held(t + 3) ? v.w : none);
            };
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                cur.kz[tt] = held(t0 + tt * 16 + r16) ? cur.kz[tt] : 0xE4000000u;                 // -(1024 + 0)
                cur.vp[tt] = kept(cur.vp[tt], t0 + tt * 16 + 4 * kb, 0xE4000000u);
            }
        }
        f4 d[CT][2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const uint32_t kz = cur.kz[tt];
            const h2 c = __builtin_bit_cast(h2, __builtin_amdgcn_perm(kz, kz, 0x07060706u));   // high half in both halves
            const h2 c16 = c + k960;
            const uint32_t kw[4] = {cur.kc[tt].x, cur.kc[tt].y, cur.kc[tt].z, cur.kc[tt].w};
#pragma unroll
            for (int i = 0; i < CT; ++i) d[i][tt] = (f4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                h2 kh[4];
                unpack4(kw[w], c, c16, kh);              // kh[j] = elements 8w + 2j, 8w + 2j + 1 of this lane's 32
                const h8 k8 = join(kh[0], kh[1], kh[2], kh[3]);
#pragma unroll
                for (int i = 0; i < CT; ++i) d[i][tt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k8, __builtin_bit_cast(h8, qv[i][w]), d[i][tt], 0, 0, 0);
            }
        }
        h8 b8[CT];                                       // B operand: softmax weight * value scale, tokens 4 kb .. of both tiles
#pragma unroll
        for (int i = 0; i < CT; ++i) {
            float sc[NS][4];                             // [x] = token 4 kb + x of the lane's tile (of both tiles with PK = 1)
            uint32_t pw[NS][4];                          // parameters of the values of these tokens
#pragma unroll
            for (int tt = 0; tt < NS; ++tt) {
                const uint4 a = PK == 2 && second ? cur.vp[1] : cur.vp[tt];
                pw[tt][0] = a.x; pw[tt][1] = a.y; pw[tt][2] = a.z; pw[tt][3] = a.w;
                const uint32_t sw[4] = {cur.ks[tt].x, cur.ks[tt].y, cur.ks[tt].z, cur.ks[tt].w};
#pragma unroll
                for (int x = 0; x < 4; ++x) sc[tt][x] = (PK == 2 && second ? d[i][1][x] : d[i][tt][x]) * ((float)half_of(sw[x]) * kScale);
            }
            if (partly) {
                const int end = min(hi, limit[i]);
#pragma unroll
                for (int tt = 0; tt < NS; ++tt)
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int t = t0 + (second ? 16 : 0) + tt * 16 + 4 * kb + x;
                        if (!(t >= lo && t < end)) { sc[tt][x] = -1e30f; pw[tt][x] = 0; }
                    }
            }
            float top = -1e30f;
            us2 largest = {0, 0};
#pragma unroll
            for (int tt = 0; tt < NS; ++tt)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    top = fmaxf(top, sc[tt][x]);
                    largest = __builtin_elementwise_max(largest, __builtin_bit_cast(us2, pw[tt][x]));
                }
            // the largest scale is below 2^(its exponent's bits - 14), so with this reference weight x scale stays below 2^15
            // (where FP32 no longer holds a score's units, the sum would be rounded by more than there is room: the score itself)
            const float below = fabsf(top) < 0x1p23f ? (float)((largest.x >> 10) & 31u) - 29.f : 0.f;
            // the four k-blocks of a column agree on the reference
            const float m_new = max_other_half(max_other_row(fmaxf(m[i], top + below)));
            if (__builtin_amdgcn_ballot_w64(m_new != m[i]) != 0) {           // rare once a few chunks have been seen
                const float alpha = __builtin_amdgcn_exp2f(m[i] - m_new);
                m[i] = m_new;
                l[i] *= alpha;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[i][e] *= alpha;
            }
            uint32_t bw[2][2];
#pragma unroll
            for (int tt = 0; tt < NS; ++tt) {
                float wf[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float pr = __builtin_amdgcn_exp2f(sc[tt][x] - m[i]);
                    l[i] += pr;
                    wf[x] = pr * (float)half_of(pw[tt][x]);
                }
                const uint32_t b_lo = __builtin_bit_cast(uint32_t, (h2){(_Float16)wf[0], (_Float16)wf[1]});
                const uint32_t b_hi = __builtin_bit_cast(uint32_t, (h2){(_Float16)wf[2], (_Float16)wf[3]});
                if (PK == 2) {                           // a column takes part with its own tile only
                    bw[0][0] = second ? 0u : b_lo; bw[0][1] = second ? 0u : b_hi;
                    bw[1][0] = second ? b_lo : 0u; bw[1][1] = second ? b_hi : 0u;
                } else {
                    bw[tt][0] = b_lo; bw[tt][1] = b_hi;
                }
            }
            b8[i] = join(__builtin_bit_cast(h2, bw[0][0]), __builtin_bit_cast(h2, bw[0][1]), __builtin_bit_cast(h2, bw[1][0]), __builtin_bit_cast(h2, bw[1][1]));
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
            for (int j = 0; j < 4; ++j) {
                const h8 v8 = join(vh[0][0][j], vh[0][1][j], vh[1][0][j], vh[1][1][j]);
#pragma unroll
                for (int i = 0; i < CT; ++i) acc[i][4 * u + j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(v8, b8[i], acc[i][4 * u + j], 0, 0, 0);
            }
        }
    };

    // One copy of the arithmetic: a call on short sequences runs through its code once, and pays for fetching it.  The last turn requests its own
    // chunk again (which is in the caches).
#pragma unroll 1
    for (int it = 0; it < n_iter; ++it) {
        const uint32_t id_after = page_of(it + 2);
        load_chunk(Bf, chunk_of(it + 1), id_b);
        process(A, it, id_a);
        A = Bf;
        id_a = id_b;
        id_b = id_after;
    }

    // ---- the partial results of the waves (and of the column halves) meet in LDS, a column tile at a time: [wave, half][16 / PK][kPartial] ----
    constexpr int N = kWaves * PK, W = 16 / PK;
#pragma unroll
    for (int i = 0; i < CT; ++i) {
        const int columns = min(k.columns - i * 16, W);
        if (columns <= 0) break;
        if (i) __syncthreads();
        l[i] += __shfl_xor(l[i], 16, 64);
        l[i] += __shfl_xor(l[i], 32, 64);
        const int column = PK == 2 ? r16 & 7 : r16;
        float* mine = s_part + ((wave * PK + (second ? 1 : 0)) * W + column) * kPartial;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                *reinterpret_cast<float4*>(mine + 16 * kb + 4 * x + 64 * u) = make_float4(acc[i][4 * u][x], acc[i][4 * u + 1][x], acc[i][4 * u + 2][x], acc[i][4 * u + 3][x]);
        if (kb == 0) *reinterpret_cast<float2*>(mine + kD) = make_float2(m[i], l[i]);
        __syncthreads();
        for (int x = threadIdx.x; x < columns * (kD / 4); x += 64 * kWaves) {
            const int at = x / (kD / 4), d = x % (kD / 4) * 4;
            const float* part = s_part + at * kPartial;
            float mm = -1e29f;
#pragma unroll
            for (int e = 0; e < N; ++e) mm = fmaxf(mm, part[e * W * kPartial + kD]);
            float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
            float den = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float2 ml = *reinterpret_cast<const float2*>(part + e * W * kPartial + kD);
                const float4 a = *reinterpret_cast<const float4*>(part + e * W * kPartial + d);
                const float f = __builtin_amdgcn_exp2f(ml.x - mm);
                num.x = fmaf(a.x, f, num.x); num.y = fmaf(a.y, f, num.y); num.z = fmaf(a.z, f, num.z); num.w = fmaf(a.w, f, num.w);
                den = fmaf(ml.y, f, den);
            }
            const int held = k.column0 + i * 16 + at, s = by_ratio(p, held);
            const int64_t row = ((int64_t)(k.first + s) * p.Hkv + k.hk) * R + held - s * R;
            finish(row, d, num, mm, den);
        }
    }
}
// ... which becomes a part
template <int CT, int PK, bool LIMITS>
__device__ __forceinline__ void attend(const SharedArgs& p, const Work& k, float* s_part)
{
    attend<CT, PK, LIMITS>(p, k, s_part, [&](int64_t row, int d, float4 num, float mm, float den) __attribute__((always_inline)) {
        float* to = p.parts + (row * k.total_slots + k.slot) * kPartial;
        *reinterpret_cast<float4*>(to + d) = num;
        if (d == 0) *reinterpret_cast<float4*>(to + kD) = make_float4(mm, den, 0.f, 0.f);
    });
}

// ---- A prefix that many columns share: four waves of 16 CT columns each, the pages unpacked once for all of them ----
// A page goes through LDS in the order of the matrix instructions' operands, [fragment][lane] of 16 bytes, a quarter of it unpacked by each
// wave, the next page while this one is used.
constexpr int kPageFragments = 32;                       // of 1 KB: keys [tile][word], values [chunk][u][j]
// Binades that the reference is set above what the largest weight needs, so that it seldom has to follow: each time costs half a chunk's arithmetic.
// Weight times scale is FP16: as many binades less of its range are left below the largest (2^-33 of it, or of a weight
// beside a scale of 2^-15 where there is none as large, and not 2^-39, is its smallest step's half).
constexpr float kSpare = 6.f;
struct WidePage {
    uint4 fragment[kPageFragments][64];
    float ks[kPageTokens], vs[kPageTokens];              // scale of a token's scores, log2(e) / sqrt(128) with it; of its values
    float below;                                         // exponent of the largest of those, as the reference takes it
};

template <int CT>
__device__ __forceinline__ void attend_wide(const SharedArgs& p, const Work& k, WidePage* s_page)
{
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, kb = lane >> 4, R = p.R;
    const int first = k.page, end = k.page_end;

    uint4 qv[CT][4];
    int limit[CT];
    int least = k.hi, most = 0;                          // of this wave's columns' limits; of all, behind which nothing need have been written
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        const int column = (wave * CT + c) * 16 + r16, held = k.column0 + min(column, k.columns - 1), s = by_ratio(p, held), b = k.first + s;
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)b * p.q_stride + (int64_t)(k.hk * R + held - s * R) * kD + kb * 32);
        const uint32_t some = column < k.columns ? ~0u : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint4 t = src[e];
            qv[c][e] = make_uint4(t.x & some, t.y & some, t.z & some, t.w & some);
        }
        limit[c] = min(max(p.seq_lens[b], 0), k.hi);
        least = min(least, limit[c]);
    }
    for (int s = by_ratio(p, k.column0) + lane, last = by_ratio(p, k.column0 + k.columns - 1); s <= last; s += 64) most = max(most, min(max(p.seq_lens[k.first + s], 0), k.hi));
    least = k.hi - largest_of_lanes(k.hi - least);
    most = largest_of_lanes(most);

    // this wave's quarter of a page: the keys of tile `wave`, half u of the values' elements of chunk `wave` / 2
    struct Staged {
        uint4 kc, vp[2];
        uint2 vc[2];
        uint32_t kz, param;                              // of token `lane`: of its key (wave 0), its value (wave 1)
    };
    const int chunk = wave >> 1, u = wave & 1;
    auto page_id = [&](int i) __attribute__((always_inline)) { return (uint32_t)constant(k.pages_of)[min(i, end - 1)]; };
    auto load = [&](Staged& s, uint32_t id) __attribute__((always_inline)) {
        const uint32_t held = id < p.pages ? id : 0;
        const uint8_t* page = p.pool + ((int64_t)held * p.Hkv + k.hk) * kPageBytes;
        s.kc = *reinterpret_cast<const uint4*>(page + wave * 1024 + r16 * (kD / 2) + kb * 16);
        s.kz = *reinterpret_cast<const uint32_t*>(page + kCodeBytes + (wave * 16 + r16) * 4);
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            s.vc[tt] = *reinterpret_cast<const uint2*>(page + kHalfPage + (2 * chunk + tt) * 1024 + lane * 16 + 8 * u);
            s.vp[tt] = *reinterpret_cast<const uint4*>(page + kHalfPage + kCodeBytes + ((2 * chunk + tt) * 16 + 4 * kb) * 4);
        }
        s.param = *reinterpret_cast<const uint32_t*>(page + (wave == 1 ? kHalfPage : 0) + kCodeBytes + lane * 4);
    };
    const float kScale = 1.4426950408889634f * 0.08838834764831845f;      // log2(e) / sqrt(128)
    const h2 k960 = {(_Float16)960.0f, (_Float16)960.0f};
    auto unpack = [&](Staged s, int i, uint32_t id, WidePage& to) __attribute__((always_inline)) {
        const int held = (id < p.pages ? most : 0) - i * kPageTokens;     // tokens of the page that some column sees
        if (held < kPageTokens) {
            s.kz = wave * 16 + r16 < held ? s.kz : 0xE4000000u;           // -(1024 + 0): the others' parameters may be anything
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const int t = (2 * chunk + tt) * 16 + 4 * kb;
                s.vp[tt] = make_uint4(t < held ? s.vp[tt].x : 0xE4000000u, t + 1 < held ? s.vp[tt].y : 0xE4000000u, t + 2 < held ? s.vp[tt].z : 0xE4000000u,
                                      t + 3 < held ? s.vp[tt].w : 0xE4000000u);
            }
            s.param = lane < held ? s.param : 0;
        }
        {
            const h2 c = __builtin_bit_cast(h2, __builtin_amdgcn_perm(s.kz, s.kz, 0x07060706u));
            const h2 c16 = c + k960;
            const uint32_t kw[4] = {s.kc.x, s.kc.y, s.kc.z, s.kc.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                h2 kh[4];
                unpack4(kw[w], c, c16, kh);
                to.fragment[wave * 4 + w][lane] = __builtin_bit_cast(uint4, join(kh[0], kh[1], kh[2], kh[3]));
            }
        }
        h2 vh[2][2][4];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
            const uint32_t zw[4] = {s.vp[tt].x, s.vp[tt].y, s.vp[tt].z, s.vp[tt].w}, vw[2] = {s.vc[tt].x, s.vc[tt].y};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const h2 cz = __builtin_bit_cast(h2, __builtin_amdgcn_perm(zw[2 * h + 1], zw[2 * h], 0x07060302u));
                unpack4(vw[h], cz, cz + k960, vh[tt][h]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) to.fragment[16 + wave * 4 + j][lane] = __builtin_bit_cast(uint4, join(vh[0][0][j], vh[0][1][j], vh[1][0][j], vh[1][1][j]));
        const float scale = (float)half_of(s.param);
        if (wave == 0) to.ks[lane] = scale * kScale;
        if (wave == 1) {
            to.vs[lane] = scale;
            int exponent = (int)((s.param >> 10) & 31u);
#pragma unroll
            for (int o = 32; o; o >>= 1) exponent = max(exponent, __shfl_xor(exponent, o, 64));
            if (lane == 0) to.below = (float)exponent - 29.f;
        }
    };

    float m[CT], l[CT];
    f4 acc[CT][8];                                       // acc[.][4u + j][x]: element d = 16 kb + 4x + 64u + j of the column
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        m[c] = -1e29f; l[c] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[c][i] = (f4){0.f, 0.f, 0.f, 0.f};
    }
    auto process = [&](const WidePage& page, int i, uint32_t id) __attribute__((always_inline)) {
        const bool partly = !(id < p.pages && (i + 1) * kPageTokens <= least);
        const float below = page.below;
#pragma unroll 1
        for (int half = 0; half < 2; ++half) {
            // (the operands of a half are requested together, those of the second product in front of the softmax: requested one at a time, as
            // the compiler orders them, each trip to LDS is waited for, twice what the arithmetic takes)
            uint4 kf[8], vf[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) kf[e] = page.fragment[half * 8 + e][lane];
            __builtin_amdgcn_sched_barrier(0);
            f4 d[CT][2];
            float t[CT][8], over[CT];
            bool follow = partly;
#pragma unroll
            for (int c = 0; c < CT; ++c) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d[c][e >> 2] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, kf[e]), __builtin_bit_cast(h8, qv[c][e & 3]), e & 3 ? d[c][e >> 2] : (f4){0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
            float ks[8], vs[8];                          // [4 tt + x]: of token 4 kb + x of tile tt
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const float4 a = *reinterpret_cast<const float4*>(page.ks + (2 * half + tt) * 16 + 4 * kb), b = *reinterpret_cast<const float4*>(page.vs + (2 * half + tt) * 16 + 4 * kb);
                ks[4 * tt] = a.x; ks[4 * tt + 1] = a.y; ks[4 * tt + 2] = a.z; ks[4 * tt + 3] = a.w;
                vs[4 * tt] = b.x; vs[4 * tt + 1] = b.y; vs[4 * tt + 2] = b.z; vs[4 * tt + 3] = b.w;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) vf[e] = page.fragment[16 + half * 8 + e][lane];
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                over[c] = -1e30f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    t[c][e] = fmaf(d[c][e >> 2][e & 3], ks[e], -m[c]);
                    over[c] = fmaxf(over[c], t[c][e]);
                }
                // The reference has to follow: a weight times the largest scale would pass 2^15.  (Where FP32 no longer holds a score's units, the sum
                // of score and exponent would be rounded by more than there is room: the score itself is the reference.)
                follow |= over[c] + (fabsf(m[c]) < 0x1p23f - 64.f ? below : 0.f) > 0.f;
            }
            // softmax weight times value scale of column tile c, the operand of the second product, and the weights' sum
            auto weights = [&](int c, const float (&by)[8]) __attribute__((always_inline)) {
                uint32_t b[4];
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const float p0 = __builtin_amdgcn_exp2f(t[c][e]), p1 = __builtin_amdgcn_exp2f(t[c][e + 1]);
                    l[c] += p0;
                    l[c] += p1;
                    b[e / 2] = __builtin_bit_cast(uint32_t, (h2){(_Float16)(p0 * by[e]), (_Float16)(p1 * by[e + 1])});
                }
                return __builtin_bit_cast(h8, make_uint4(b[0], b[1], b[2], b[3]));
            };
            float scale[CT][8];                          // of what a column sees
#pragma unroll
            for (int c = 0; c < CT; ++c)
#pragma unroll
                for (int e = 0; e < 8; ++e) scale[c][e] = vs[e];
            if (__builtin_amdgcn_ballot_w64(follow) != 0) {
#pragma unroll
                for (int c = 0; c < CT; ++c) {
                    const int end_c = (id < p.pages ? limit[c] : 0) - i * kPageTokens - half * 32 - 4 * kb;
                    float top = -1e30f, largest = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const bool seen = (e >> 2) * 16 + (e & 3) < end_c;
                        t[c][e] = seen ? d[c][e >> 2][e & 3] * ks[e] : -1e30f;
                        scale[c][e] = seen ? vs[e] : 0.f;
                        top = fmaxf(top, t[c][e]);
                        largest = fmaxf(largest, scale[c][e]);
                    }
                    // (where a column does not see all, its reference rests on what it sees: the page's largest scale may be another token's)
                    const float room = (partly ? (float)(min(max((int)(__float_as_uint(largest) >> 23) - 112, 0), 31) - 29) : below) + kSpare;
                    const float m_new = max_other_half(max_other_row(fmaxf(m[c], top + (fabsf(top) < 0x1p23f ? room : 0.f))));
                    const float alpha = __builtin_amdgcn_exp2f(m[c] - m_new);
                    m[c] = m_new;
                    l[c] *= alpha;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        acc[c][e] *= alpha;
                        t[c][e] -= m_new;
                    }
                }
            }
#pragma unroll
            for (int c = 0; c < CT; ++c) {
                const h8 b8 = weights(c, scale[c]);
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[c][e] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, vf[e]), b8, acc[c][e], 0, 0, 0);
            }
        }
    };

    // (a wave may be a page ahead of the others, which then use the other buffer)
    Staged staged;
    uint32_t id = page_id(first), id_next = page_id(first + 1);
    load(staged, id);
#pragma unroll 1
    for (int i = first; i < end; ++i) {
        const uint32_t id_after = page_id(i + 2);
        WidePage& page = s_page[(i - first) & 1];
        unpack(staged, i, id, page);
        load(staged, id_next);                           // (the last turn its own page again)
        __syncthreads();
        process(page, i, id);
        id = id_next;
        id_next = id_after;
    }
    // The parts leave through LDS, a column tile at a time, in whole rows: stored from the registers, 16 bytes here and there, they took as long as
    // three pages (64 sequences behind 4096 tokens of 32 / 8 heads 41 us, 28 without the stores).
    __syncthreads();                                     // (the pages are done with)
    float* s_rows = reinterpret_cast<float*>(s_page) + wave * 16 * kPartial;
#pragma unroll
    for (int c = 0; c < CT; ++c) {
        l[c] += __shfl_xor(l[c], 16, 64);
        l[c] += __shfl_xor(l[c], 32, 64);
#pragma unroll
        for (int v = 0; v < 2; ++v)
#pragma unroll
            for (int x = 0; x < 4; ++x)
                *reinterpret_cast<float4*>(s_rows + r16 * kPartial + 16 * kb + 4 * x + 64 * v) = make_float4(acc[c][4 * v][x], acc[c][4 * v + 1][x], acc[c][4 * v + 2][x], acc[c][4 * v + 3][x]);
        if (kb == 0) *reinterpret_cast<float4*>(s_rows + r16 * kPartial + kD) = make_float4(m[c], l[c], 0.f, 0.f);
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");           // the wave's own writes, then its reads
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const int column0 = (wave * CT + c) * 16, columns = min(k.columns - column0, 16);
#pragma unroll 1
        for (int i = lane; i < columns * (kPartial / 4); i += 64) {
            const int column = i / (kPartial / 4), held = k.column0 + column0 + column, s = by_ratio(p, held);
            const int64_t row = ((int64_t)(k.first + s) * p.Hkv + k.hk) * R + held - s * R;
            *reinterpret_cast<float4*>(p.parts + (row * k.total_slots + k.slot) * kPartial + (i - column * (kPartial / 4)) * 4) = *reinterpret_cast<const float4*>(s_rows + i * 4);
        }
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();                                     // (the next run begins with the first buffer)
}

// The work over all prefixes where they are wide: units of a page for a tile of columns, by group, KV head, tile and page, dealt to the workgroups in
// equal runs of `run` units, of which none covers a tile in more parts than there are slots.
struct Units {
    int all, run;
    bool wide;                                           // worth their form
    int before;                                          // units of the groups in front of the one looked for
    int first, columns, tokens, pages, tiles;            // that group
};

// Groups g0 .. g0 + 63, one to a lane.  Bounds that descend are taken as ascending ones: no sequence is in two groups, and the units stay within what
// the host counted.
template <int TILE>
struct GroupLanes {
    int first, last, tokens, columns, pages, tiles, units, upto;
    int lost;                                            // units' worth of columns that are none
    int reached;                                         // the largest bound in front of these groups
    __device__ __forceinline__ void load(const SharedArgs& p, int g0)
    {
        const int g = g0 + (int)(threadIdx.x & 63);
        int bound = 0, end = 0;
        tokens = 0;
        if (g < p.G) {
            const int a = p.cu[g], e = p.cu[g + 1], n = p.prefix_lens[g];
            bound = min(max(a, 0), p.B);
            end = min(e, p.B);
            tokens = min(max(n, 0), p.width * kPageTokens);
        }
        if (g0 == 0) reached = 0;
        first = largest_upto_lane(max(bound, reached));
        last = max(end, first);
        reached = __builtin_amdgcn_readlane(first, 63);
        columns = (last - first) * p.R;
        tiles = (columns + TILE - 1) / TILE;
        pages = tiles ? (tokens + kPageTokens - 1) / kPageTokens : 0;
        units = tiles * p.Hkv * pages;
        upto = upto_lane(units);
        lost = (int)((int64_t)(p.Hkv * pages) * (tiles * TILE - columns) / TILE);
    }
    __device__ __forceinline__ void pick(Units& f, unsigned long long who, int before) const
    {
        const int w = __builtin_ctzll(who);
        f.before = before + __builtin_amdgcn_readlane(upto, w) - __builtin_amdgcn_readlane(units, w);
        f.first = __builtin_amdgcn_readlane(first, w);
        f.columns = __builtin_amdgcn_readlane(columns, w);
        f.tokens = __builtin_amdgcn_readlane(tokens, w);
        f.pages = __builtin_amdgcn_readlane(pages, w);
        f.tiles = __builtin_amdgcn_readlane(tiles, w);
    }
};
// All units and the runs they are dealt in; where `b` >= 0, the group of sequence b as well (tokens 0: none).  `g` is left at the last 64 groups.
template <int TILE>
__device__ __forceinline__ void count_units(const SharedArgs& p, GroupLanes<TILE>& g, Units& f, int b)
{
    f.all = 0;
    f.tokens = 0;
    int longest = 0, lost = 0;
    for (int g0 = 0; g0 < p.G; g0 += 64) {
        g.load(p, g0);
        if (b >= 0 && !f.tokens) {
            const unsigned long long who = __builtin_amdgcn_ballot_w64(g.first <= b && b < g.last && g.tokens > 0);
            if (who) g.pick(f, who, f.all);
        }
        f.all += __builtin_amdgcn_readlane(g.upto, 63);
        longest = max(longest, largest_of_lanes(g.pages));
        lost += __builtin_amdgcn_readlane(upto_lane(g.lost), 63);
    }
    f.wide = 8 * (int64_t)f.all - 21 * (int64_t)lost >= 8 * kWideUnits;      // (10.5 (all - lost) - 6.5 all >= 4 kWideUnits)
    f.run = max(max((f.all + p.prefix_workgroups - 1) / p.prefix_workgroups, min(kLeastRun, max(longest, 1))), (longest + p.wide_parts - 3) / (p.wide_parts - 2));
}
template <int TILE>
__device__ __forceinline__ void find_unit(const SharedArgs& p, GroupLanes<TILE>& g, Units& f, int unit)
{
    int before = 0;
    for (int g0 = 0; g0 < p.G; g0 += 64) {
        if (p.G > 64) g.load(p, g0);
        const unsigned long long who = __builtin_amdgcn_ballot_w64(before + g.upto > unit && g.units > 0);
        if (who) {
            g.pick(f, who, before);
            return;
        }
        before += __builtin_amdgcn_readlane(g.upto, 63);
    }
}

// The work of this workgroup where the waves share the tokens of kPrefixColumns: false if there is none.
__device__ __forceinline__ bool narrow_work(const SharedArgs& p, Work& k)
{
    const int lane = threadIdx.x & 63, most = p.width * kPageTokens;
    const uint32_t of_tile = (uint32_t)p.Hkv * p.prefix_parts, rest = blockIdx.x % of_tile;
    int tile = blockIdx.x / of_tile;
    k.hk = rest % p.Hkv;
    k.part = rest / p.Hkv;
    // the tile's group: tiles of the groups in front of each are counted 64 groups at a time
    bool found = false;
    for (int g0 = 0; g0 < p.G && !found; g0 += 64) {
        const int g = g0 + lane;
        int first = 0, columns = 0, tokens = 0;
        if (g < p.G) {
            first = min(max(p.cu[g], 0), p.B);
            columns = max(min(p.cu[g + 1], p.B) - first, 0) * p.R;
            tokens = min(max(p.prefix_lens[g], 0), most);
        }
        const int tiles = tokens ? (columns + kPrefixColumns - 1) / kPrefixColumns : 0;
        int upto = tiles;
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o, 64);
            if (lane >= o) upto += v;
        }
        const unsigned long long who = __builtin_amdgcn_ballot_w64(upto > tile);
        if (who) {
            const int f = __builtin_ctzll(who);
            const int at = tile - (__shfl(upto, f, 64) - __shfl(tiles, f, 64));
            const int group_first = __builtin_amdgcn_readfirstlane(__shfl(first, f, 64));
            k.hi = __builtin_amdgcn_readfirstlane(__shfl(tokens, f, 64));
            k.columns = __builtin_amdgcn_readfirstlane(min(__shfl(columns, f, 64) - at * kPrefixColumns, kPrefixColumns));
            k.first = group_first;
            k.column0 = __builtin_amdgcn_readfirstlane(at * kPrefixColumns);
            k.pages_of = p.table + (int64_t)group_first * p.width;
            found = true;
        } else {
            tile -= __shfl(upto, 63, 64);
        }
    }
    if (!found) return false;
    k.parts = attending((k.hi + kChunk - 1) / kChunk, p.prefix_parts);
    k.slot = k.part;
    return k.part < k.parts;
}

// WIDE: column tiles of a wave where the prefix's columns are many, 0 where a workgroup's waves share the tokens of kPrefixColumns
template <int PK, int WIDE>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(2))) void shared_decode_kernel(SharedArgs p)
{
    constexpr size_t kNarrowBytes = kWaves * 16 * kPartial * sizeof(float), kWideBytes = 2 * sizeof(WidePage);
    __shared__ __align__(16) unsigned char s_bytes[WIDE && kWideBytes > kNarrowBytes ? kWideBytes : kNarrowBytes];
    float* s_part = reinterpret_cast<float*>(s_bytes);
    const int lane = threadIdx.x & 63;
    const int most = p.width * kPageTokens;
    Work k{};
    k.total_slots = p.prefix_slots + p.own_parts;
    if (blockIdx.x < p.prefix_blocks) {
        if constexpr (WIDE != 0) {
            constexpr int kTile = 64 * WIDE;
            // runs of neighbouring units on one chiplet: its L2 then holds the pages of a KV head or two
            const int w = (int)(blockIdx.x % 8) * (p.prefix_workgroups / 8) + (int)(blockIdx.x / 8);
            Units f;
            GroupLanes<kTile> g;
            count_units<kTile>(p, g, f, -1);
            if (!f.wide) {
                if (!narrow_work(p, k)) return;
                attend<kColumnTiles, 1, true>(p, k, s_part);
                return;
            }
            if ((int)blockIdx.x >= p.prefix_workgroups) return;
            int unit = w * f.run;
            const int end = min(unit + f.run, f.all);
#pragma unroll 1
            while (unit < end) {
                find_unit<kTile>(p, g, f, unit);
                const int of_group = unit - f.before, column_tile = of_group / f.pages, hk = column_tile / f.tiles, tile = column_tile - hk * f.tiles;
                k.page = of_group - column_tile * f.pages;
                k.page_end = min(k.page + end - unit, f.pages);
                k.hk = hk;
                k.hi = f.tokens;
                k.first = f.first;
                k.column0 = tile * kTile;
                k.columns = min(f.columns - tile * kTile, kTile);
                k.pages_of = p.table + (int64_t)k.first * p.width;
                k.slot = w - (unit - k.page) / f.run;
                unit += k.page_end - k.page;
                attend_wide<WIDE>(p, k, reinterpret_cast<WidePage*>(s_bytes));
            }
            return;
        } else {
            if (!narrow_work(p, k)) return;
            attend<kColumnTiles, 1, true>(p, k, s_part);
        }
    } else {
        const uint32_t i = blockIdx.x - p.prefix_blocks, pairs = (uint32_t)p.B * p.Hkv, bh = i % pairs;
        const int b = bh / p.Hkv;
        k.hk = bh - b * p.Hkv;
        k.part = i / pairs;
        k.hi = min(max(p.seq_lens[b], 0), most);
        k.lo = min(prefix_of(p, b, lane), k.hi);
        if (k.lo == k.hi) return;
        k.parts = attending((k.hi + kChunk - 1) / kChunk - k.lo / kChunk, p.own_parts);
        if (k.part >= k.parts) return;
        k.pages_of = p.table + (int64_t)b * p.width;
        k.first = b;
        k.columns = p.R;
        k.slot = p.prefix_slots + k.part;
        attend<1, PK, false>(p, k, s_part);
    }
}

// A workgroup for each sequence and KV head, where those fill the chip: its own tokens, and the join with the prefix's parts.
template <int PK>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(3))) void shared_own_kernel(SharedArgs p)
{
    __shared__ __align__(16) float s_part[kWaves * 16 * kPartial];
    const int lane = threadIdx.x & 63, b = blockIdx.x / p.Hkv;
    Work k{};
    k.hk = blockIdx.x - b * p.Hkv;
    k.hi = min(max(p.seq_lens[b], 0), p.width * kPageTokens);
    const int P = prefix_of(p, b, lane), n = P && k.hi ? attending((P + kChunk - 1) / kChunk, p.prefix_parts) : 0;
    k.lo = min(P, k.hi);
    k.parts = 1;
    k.pages_of = p.table + (int64_t)b * p.width;
    k.first = b;
    k.columns = p.R;
    const int64_t row0 = ((int64_t)b * p.Hkv + k.hk) * p.R;
    // (the prefix's parts come a few together, each few against the largest reference so far)
    auto finish = [&](int64_t row, int d, float4 num, float top, float den) __attribute__((always_inline)) {
        const float* parts = p.parts + row * (p.prefix_slots + p.own_parts) * kPartial;
#pragma unroll 1
        for (int i0 = 0; i0 < n; i0 += kOwnInFlight) {
            float4 a[kOwnInFlight];
            float2 ml[kOwnInFlight];
            float most = top;
#pragma unroll
            for (int e = 0; e < kOwnInFlight; ++e) {
                const float* part = parts + (int64_t)min(i0 + e, n - 1) * kPartial;
                ml[e] = *reinterpret_cast<const float2*>(part + kD);
                a[e] = *reinterpret_cast<const float4*>(part + d);
            }
#pragma unroll
            for (int e = 0; e < kOwnInFlight; ++e) most = fmaxf(most, ml[e].x);
            const float alpha = __builtin_amdgcn_exp2f(top - most);
            num.x *= alpha; num.y *= alpha; num.z *= alpha; num.w *= alpha;
            den *= alpha;
            top = most;
#pragma unroll
            for (int e = 0; e < kOwnInFlight; ++e) {
                const float f = i0 + e < n ? __builtin_amdgcn_exp2f(ml[e].x - most) : 0.f;
                num.x = fmaf(a[e].x, f, num.x); num.y = fmaf(a[e].y, f, num.y); num.z = fmaf(a[e].z, f, num.z); num.w = fmaf(a[e].w, f, num.w);
                den = fmaf(ml[e].y, f, den);
            }
        }
        const float inv = inverse_sum(p, den, b, k.hi, P);
        *reinterpret_cast<h4*>(p.out + row * kD + d) = (h4){(_Float16)(num.x * inv), (_Float16)(num.y * inv), (_Float16)(num.z * inv), (_Float16)(num.w * inv)};
    };
    if (k.lo < k.hi) {
        attend<1, PK, false>(p, k, s_part, finish);
    } else {
        for (int x = threadIdx.x; x < p.R * (kD / 4); x += 64 * kWaves) finish(row0 + x / (kD / 4), x % (kD / 4) * 4, make_float4(0.f, 0.f, 0.f, 0.f), -1e29f, 0.f);
    }
}

// The parts of a head, a wave to a head: two elements to a lane, a part's reference to a lane.
template <int WIDE>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedArgs p)
{
    const int lane = threadIdx.x & 63;
    const int H = p.Hkv * p.R;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)p.B * H) return;
    const int b = (int)(row / H);
    const int most = p.width * kPageTokens;
    const int L = min(max(p.seq_lens[b], 0), most);
    int P, n_prefix = 0;
    if constexpr (WIDE != 0) {
        Units f;
        GroupLanes<64 * WIDE> g;
        count_units<64 * WIDE>(p, g, f, b);
        P = f.tokens;
        if (P && L && !f.wide) {
            n_prefix = attending((P + kChunk - 1) / kChunk, p.prefix_parts);
        } else if (P && L) {
            const int h = (int)(row - (int64_t)b * H), hk = by_ratio(p, h), tile = ((b - f.first) * p.R + h - hk * p.R) / (64 * WIDE);
            const int unit = f.before + (hk * f.tiles + tile) * f.pages;
            n_prefix = (unit + f.pages - 1) / f.run - unit / f.run + 1;
        }
    } else {
        P = prefix_of(p, b, lane);
        if (P && L) n_prefix = attending((P + kChunk - 1) / kChunk, p.prefix_parts);
    }
    const int lo = min(P, L);
    const int n_own = L > lo ? attending((L + kChunk - 1) / kChunk - lo / kChunk, p.own_parts) : 0;
    const int total = p.prefix_slots + p.own_parts, n = n_prefix + n_own;
    const float* parts = p.parts + row * total * kPartial;
    auto slot = [&](int i) { return i < n_prefix ? i : p.prefix_slots + i - n_prefix; };
    float f[2], den = 0.f, top = -1e29f;
    float2 ml[2];
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        ml[e] = make_float2(-1e29f, 0.f);
        if (lane + 64 * e < n) ml[e] = *reinterpret_cast<const float2*>(parts + (int64_t)slot(lane + 64 * e) * kPartial + kD);
        top = fmaxf(top, ml[e].x);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        f[e] = __builtin_amdgcn_exp2f(ml[e].x - top);
        den = fmaf(ml[e].y, f[e], den);
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) den += __shfl_xor(den, o, 64);
    float2 sum = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int i0 = 0; i0 < n; i0 += kInFlight) {
        float2 a[kInFlight];
#pragma unroll
        for (int e = 0; e < kInFlight; ++e) a[e] = *reinterpret_cast<const float2*>(parts + (int64_t)slot(min(i0 + e, n - 1)) * kPartial + 2 * lane);
#pragma unroll
        for (int e = 0; e < kInFlight; ++e) {
            const int i = i0 + e;
            const float g = i < n ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(i < 64 ? f[0] : f[1]), i & 63)) : 0.f;
            sum.x = fmaf(a[e].x, g, sum.x); sum.y = fmaf(a[e].y, g, sum.y);
        }
    }
    const float inv = inverse_sum(p, den, b, L, P);
    reinterpret_cast<h2*>(p.out + row * kD)[lane] = (h2){(_Float16)(sum.x * inv), (_Float16)(sum.y * inv)};
}

// Tiles of columns of all prefixes at most: every group may end in a part of one, but no more than B of them hold a sequence (3 sequences in 20000 groups
// 0.15 ms, with workgroups for a tile of each 44).
int64_t prefix_tiles(int64_t B, int64_t G, int64_t R, int64_t columns) { return B * R / columns * (G > 0) + std::min(G, B); }
// Whether prefixes may take the wide form: enough columns to a group, and room in the block table for that many units.
bool wide_prefix(int64_t B, int64_t G, int64_t R, int64_t Hkv, int64_t width)
{
    return G && B * R / G >= 80 && prefix_tiles(B, G, R, 64 * kWide) * Hkv * width >= kWideUnits;
}
// Workgroups that stand by for each tile of columns of a prefix and KV head, and for each sequence and KV head: two to a compute unit.
int parts_for(int64_t items, int64_t width)
{
    if (items <= 0) return 0;
    return (int)std::max<int64_t>(1, std::min<int64_t>({kMaxParts, 512 / items, (2 * width + 2 * kWaves - 1) / (2 * kWaves)}));
}

// Parts of a tile of columns of a prefix where the waves share its tokens, and where they have columns of their own: twice what an even share of
// the workgroups comes to, and the pieces at its ends.
int prefix_parts(int64_t B, int64_t G, int64_t R, int64_t Hkv, int64_t width) { return parts_for(prefix_tiles(B, G, R, kPrefixColumns) * Hkv, width); }
int wide_parts(int64_t B, int64_t G, int64_t R, int64_t Hkv, int64_t width)
{
    return wide_prefix(B, G, R, Hkv, width) ? (int)std::min<int64_t>(kMaxParts, 2 * kWideWorkgroups / (prefix_tiles(B, G, R, 64 * kWide) * Hkv) + 3) : 0;
}
// Whether the own tokens have a launch of their own, behind the prefixes' and in place of the join, with registers and LDS for three workgroups on a
// compute unit, not two.  Side by side with a prefix they fill what it leaves, so few gain nothing, nor do those beside prefixes that may be long for
// the wide form: 64 sequences of 32 / 8 heads with 300 tokens behind 4096 26.5 us in one launch and joined, 28.5 one behind the other; 200 of 40 / 8
// with 100 behind 1000 36.1 and 32.7; 512 of 32 / 8 with 300 behind 100 64.4 and 52.2; 300 of 32 / 8 with 100 behind 8000 in three groups 96 and 103,
// 200 of 64 / 8 with 100 behind 16000 190 and 195.  Without prefixes there is the one launch: 64 of 32 / 8 with 300 tokens 11.5 us joined, 7.6 so.
bool own_launch(int64_t B, int64_t G, int64_t Hkv, int own_parts, bool wide) { return own_parts == 1 && !wide && (!G || B * Hkv > 1000); }

}  // namespace

size_t shared_decode_workspace_bytes(int64_t B, int64_t H, int64_t Hkv, int64_t width, int64_t G)
{
    const int64_t slots = std::max(prefix_parts(B, G, H / Hkv, Hkv, width), wide_parts(B, G, H / Hkv, Hkv, width)) + parts_for(B * Hkv, width);
    return (size_t)(B * H * slots) * kPartial * sizeof(float);
}

hipError_t launch_shared_decode(const void* q, int64_t q_stride, const uint8_t* pool, int64_t pages, const int32_t* table, int64_t width,
                                const int32_t* seq_lens, const int32_t* group_cu, const int32_t* prefix_lens, int64_t B, int64_t G, int64_t H,
                                int64_t Hkv, void* out, void* workspace, hipStream_t s)
{
    SharedArgs p{};
    p.pool = pool; p.table = table; p.seq_lens = seq_lens; p.cu = group_cu; p.prefix_lens = prefix_lens;
    p.q = static_cast<const __half*>(q); p.q_stride = q_stride;
    p.parts = static_cast<float*>(workspace);
    p.out = static_cast<__half*>(out);
    p.pages = (uint32_t)pages; p.width = (int)width; p.B = (int)B; p.G = (int)G; p.Hkv = (int)Hkv; p.R = (int)(H / Hkv);
    const bool wide = wide_prefix(B, G, p.R, Hkv, width);
    p.prefix_parts = prefix_parts(B, G, p.R, Hkv, width);
    p.wide_parts = wide_parts(B, G, p.R, Hkv, width);
    p.prefix_slots = std::max(p.prefix_parts, p.wide_parts);
    p.own_parts = parts_for(B * Hkv, width);
    p.prefix_workgroups = kWideWorkgroups;
    p.ratio_magic = (uint32_t)((((uint64_t)1 << 32) + p.R - 1) / p.R);
    const int64_t prefix_blocks = std::max<int64_t>(wide ? kWideWorkgroups : 0, prefix_tiles(B, G, p.R, kPrefixColumns) * Hkv * p.prefix_parts);
    const bool own = own_launch(B, G, Hkv, p.own_parts, wide);
    const int64_t blocks = prefix_blocks + (own ? 0 : B * Hkv * p.own_parts), joins = (B * H + 3) / 4;
    if (blocks >= (int64_t)1 << 24 || B * Hkv >= (int64_t)1 << 24 || joins >= (int64_t)1 << 24) return hipErrorInvalidValue;    // 2^32 threads
    if (wide && prefix_tiles(B, G, p.R, 64 * kWide) * Hkv * width >= (int64_t)1 << 31) return hipErrorInvalidValue;  // units of work, counted in 32 bits
    p.prefix_blocks = (uint32_t)prefix_blocks;
    const int PK = p.R <= 8 ? 2 : 1;
    auto* kernel = PK == 2 ? (wide ? shared_decode_kernel<2, kWide> : shared_decode_kernel<2, 0>) : (wide ? shared_decode_kernel<1, kWide> : shared_decode_kernel<1, 0>);
    if (blocks) {
        kernel<<<(unsigned)blocks, 64 * kWaves, 0, s>>>(p);
        if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    if (own) {
        auto* rest = PK == 2 ? shared_own_kernel<2> : shared_own_kernel<1>;
        rest<<<(unsigned)(B * Hkv), 64 * kWaves, 0, s>>>(p);
        return hipGetLastError();
    }
    auto* join = wide ? shared_join_kernel<kWide> : shared_join_kernel<0>;
    join<<<(unsigned)joins, 256, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace qoq
