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
// Softmax in base 2, FP32; the weights are rounded to FP16 for the second product, sums stay FP32.  They are taken relative to a reference
// that lies 2^7 (kLead) below a row's largest score when it is set, and is raised only when a score passes it by more than another
// 2^8 (kSlack), so that the sums' 64 registers are rarely rescaled: the largest weight is between 2^7 and 2^15, and each is off by 2^-11 of
// itself or, below FP16's normal numbers, by 2^-25, which is 2^-32 of the largest at most.  (Without the lead the second bound is 2^-25; times were level,
// 3 x 4001 520 to 521 us, 256 alone 8.55 and 8.65.)
// Large batches, 3 x 4001 tokens of 64 / 8 heads 510 us, 933 TFLOP/s (a large product of the library's: 1145), two workgroups to a compute unit, are
// bound by instructions: of the cycles matrix instructions take 55% and vector ones 47%, hardly at once, and the clock falls to
// 1.7 GHz under them (2.3 on one short prompt).  Short ones are bound by a workgroup's own chain of key tiles, 1024 tokens of 32 heads 25 us: 3.7 to the
// first tile, then 1.2 to 1.4 for each of the last rows' 16.  A ring of four tiles was no faster (31), nor are weights spread over both products (27.5).
#include <algorithm>
#include <type_traits>

#include "qoq_gemm_common.h"
#include "qoq_kv4_common.h"
#include "qoq_ragged.h"
#include "qoq_workspace.h"

namespace qoq {
namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr int kBM = 128, kBN = 64, kPrefillThreads = 256;
constexpr int kRows = 32, kKeys = 32;                    // of the narrow kernel's tiles
constexpr int kPart = kD + 4;                            // floats of a row's partial result: sums, reference, weight sum, whether to do it again
constexpr int kRowBytes = kD * 2;                        // 256: sixteen 16-byte chunks
constexpr int kRowPitch = kRowBytes + 16;                // of results in LDS
constexpr int kTileBytes = kBN * kRowBytes;              // 16 KiB of keys, as much of values
constexpr float kScale = 1.4426950408889634f * 0.08838834764831845f;      // log2(e) / sqrt(128)
constexpr int kMaxParts = 64;                            // workgroups to a row tile
constexpr int kWideDeal = 8;                            // key tiles that a workgroup is given before another one attends
constexpr int kNarrowDeal = 2;                          // key tiles that a wave is given before another workgroup attends
constexpr float kLead = 7.f / kScale, kSlack = 8.f / kScale;              // in units of the scores

struct PrefillArgs {
    const __half *q, *k, *v;
    __half* out;
    const int32_t *cu_q, *cu_k;
    int64_t q_stride, k_stride, v_stride;                // elements per token
    int M, Mk, B, H, Hkv, r, window, sinks;
    uint32_t slots;
    // the narrow kernel's: workgroups that stand by for a row tile, and their partial results
    int ns;
    float* parts;
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

// Where a workgroup's rows lie: ROWS rows of a (sequence, KV head), and the list of key tiles of BN keys that some of them see: those of
// the sinks, then those of the window (without one all up to the last row's position).
template <int ROWS, int BN>
struct RowTile {
    int q0, Tq, k0, Tk, first;                           // the sequence's queries and keys; the tile's first row, of Tq r
    int lo_pos, hi_pos;                                  // positions of its first and last row
    int n_first, gap, n;                                 // key tile i of the list: i < n_first ? i : i + gap

    __device__ __forceinline__ bool find(const PrefillArgs& p, uint32_t slot, int lane)
    {
        // 64 sequences' bounds in flight at once, a lane each
        auto before = [&](int end, int i) { return (int64_t)end * p.r / ROWS + i <= (int64_t)slot; };
        const int lo = near_before(p.B, lane, [&](int i) { return before(p.cu_q[i], i); }), held = min(p.B - lo, 64);
        const int ends_q = lane < held ? p.cu_q[lo + lane + 1] : 0, ends_k = lane < held ? p.cu_k[lo + lane + 1] : 0;
        const int begin_q = p.cu_q[lo], begin_k = p.cu_k[lo];
        const int c = __popcll(__builtin_amdgcn_ballot_w64(lane < held && before(ends_q, lo + lane + 1)));
        if (c >= held) return false;
        auto bounded = [](int v, int most) { return min(max(v, 0), most); };
        const int at_q = c ? __builtin_amdgcn_readlane(ends_q, c - 1) : begin_q, at_k = c ? __builtin_amdgcn_readlane(ends_k, c - 1) : begin_k;
        q0 = bounded(at_q, p.M);
        k0 = bounded(at_k, p.Mk);
        Tq = bounded(__builtin_amdgcn_readlane(ends_q, c), p.M) - q0;
        Tk = max(bounded(__builtin_amdgcn_readlane(ends_k, c), p.Mk) - k0, 0);
        const int64_t tile = (int64_t)slot - ((int64_t)at_q * p.r / ROWS + lo + c);
        if (Tq <= 0 || tile < 0 || tile * ROWS >= (int64_t)Tq * p.r) return false;
        first = (int)(tile * ROWS);                      // below 2^31
        lo_pos = Tk - Tq + first / p.r;
        hi_pos = Tk - Tq + min((first + ROWS - 1) / p.r, Tq - 1);
        const int end = max(hi_pos + 1, 0), from = p.window ? max(lo_pos - p.window + 1, 0) : 0, tiles = (end + BN - 1) / BN;
        n_first = min((p.sinks + BN - 1) / BN, tiles);
        gap = max(min(from / BN, tiles) - n_first, 0);
        n = tiles - gap;
        return true;
    }
    __device__ __forceinline__ int rows(const PrefillArgs& p) const { return min(ROWS, Tq * p.r - first); }
    __device__ __forceinline__ int tile_of(int i) const { return i < n_first ? i : i + gap; }
    // query and head of a row of the tile
    __device__ __forceinline__ void row(const PrefillArgs& p, int x, int& query, int& head) const
    {
        query = (first + x) / p.r;
        head = first + x - query * p.r;
    }
};

// workgroups that share the keys of a row tile: as many as stand by, get their deal of key tiles each
template <int ROWS, int BN>
__device__ __forceinline__ int attending(const PrefillArgs& p, const RowTile<ROWS, BN>& t)
{
    constexpr int deal = ROWS == kBM ? kWideDeal : 4 * kNarrowDeal;
    return min(p.ns, max(1, (t.n + deal - 1) / deal));
}

// What a row's sums are multiplied by.  A row in front of position 0 sees nothing and is zero.  From there on it sees a key, and its largest
// weight is at least 1 unless all of its scores are minus infinity: its sums are zero and it is 0 / 0.
__device__ __forceinline__ float factor(float inv, int pos) { return pos < 0 ? 0.f : inv; }

// A zero weight times infinity or NaN is NaN, in rows that do not see that value, and scores past 2^24 can leave a row without weights.  So
// where a wave's results are not all finite, or a row's weights are gone, rows `begin` .. `end` - 1 of its tile are done again, one after the
// other, with the keys they see and no others: 64 scores at a time, a lane each, then two elements of the values a lane.  (Slow: for inputs
// that are broken already, or next to it.)
template <int ROWS, int BN>
__device__ void redo_rows(const PrefillArgs& p, const RowTile<ROWS, BN>& t, int hk, int begin, int end, int lane)
{
    const __half* k_rows = p.k + (int64_t)t.k0 * p.k_stride + hk * kD;
    const __half* v_rows = p.v + (int64_t)t.k0 * p.v_stride + hk * kD;
    for (int x = begin; x < min(end, t.rows(p)); ++x) {
        int query, head;
        t.row(p, x, query, head);
        const int pos = t.Tk - t.Tq + query;
        const __half* q_row = p.q + (int64_t)(t.q0 + query) * p.q_stride + (hk * p.r + head) * kD;
        float top = -1e30f, sum = 0.f, o0 = 0.f, o1 = 0.f;
        for (int i = 0; i < t.n; ++i)
            for (int at = t.tile_of(i) * BN; at < t.tile_of(i) * BN + BN && at <= pos; at += 64) {
                const int key = at + lane, last = min(t.tile_of(i) * BN + BN - 1, pos);
                const bool sees = key <= last && (!p.window || key > pos - p.window || key < p.sinks);
                const uint4* k_row = reinterpret_cast<const uint4*>(k_rows + (int64_t)min(key, last) * p.k_stride);
                float s = 0.f;
#pragma unroll
                for (int d = 0; d < kD / 8; ++d) {
                    const uint4 a = k_row[d], c = reinterpret_cast<const uint4*>(q_row)[d];
                    s = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, a.x), __builtin_bit_cast(h2, c.x), s, false);
                    s = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, a.y), __builtin_bit_cast(h2, c.y), s, false);
                    s = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, a.z), __builtin_bit_cast(h2, c.z), s, false);
                    s = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, a.w), __builtin_bit_cast(h2, c.w), s, false);
                }
                float most = sees ? s : -__builtin_inff();
                for (int step = 32; step; step >>= 1) most = fmaxf(most, __shfl_xor(most, step, 64));
                most = fmaxf(most, top);
                const float keep = __builtin_amdgcn_exp2f((top - most) * kScale), weight = sees ? __builtin_amdgcn_exp2f((s - most) * kScale) : 0.f;
                top = most;
                sum = sum * keep + weight;
                o0 *= keep;
                o1 *= keep;
                const uint64_t seen = __builtin_amdgcn_ballot_w64(sees);
                for (int j = 0; j < 64; j += 8) {
                    if ((seen >> j & 255) == 0) continue;
                    uint32_t v[8];
#pragma unroll
                    for (int x = 0; x < 8; ++x) v[x] = reinterpret_cast<const uint32_t*>(v_rows + (int64_t)min(at + j + x, last) * p.v_stride)[lane];
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        if ((seen >> (j + x) & 1) == 0) continue;
                        const float w = __shfl(weight, j + x, 64);
                        o0 = fmaf(w, (float)half_of(v[x]), o0);
                        o1 = fmaf(w, (float)half_of(v[x] >> 16), o1);
                    }
                }
            }
        for (int step = 32; step; step >>= 1) sum += __shfl_xor(sum, step, 64);
        const float inv = factor(1.f / sum, pos);
        const h2 pair = {(_Float16)(o0 * inv), (_Float16)(o1 * inv)};
        reinterpret_cast<uint32_t*>(p.out + ((int64_t)(t.q0 + query) * p.H + hk * p.r + head) * kD)[lane] = __builtin_bit_cast(uint32_t, pair);
    }
}

// four elements of a row's result
template <int ROWS, int BN>
__device__ __forceinline__ void write_out(const PrefillArgs& p, const RowTile<ROWS, BN>& t, int hk, int x, int d, float4 num, float inv)
{
    int query, head;
    t.row(p, x, query, head);
    inv = factor(inv, t.Tk - t.Tq + query);
    const h2 a = {(_Float16)(num.x * inv), (_Float16)(num.y * inv)}, c = {(_Float16)(num.z * inv), (_Float16)(num.w * inv)};
    *reinterpret_cast<uint2*>(p.out + ((int64_t)(t.q0 + query) * p.H + hk * p.r + head) * kD + d) =
        make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c));
}

// Whether some row of the wave has to be done again: a sum is not finite, or the weights' is small although a score was seen (it is 2^7 at
// least but for rounding).  The product of the reference and kScale is rounded, which is a factor that a row's weights have in common; past
// 2^24 it is not small, and they can overflow or vanish.
__device__ __forceinline__ bool to_redo(const f16v (&acc)[4], float m, float total, bool there)
{
    float bad = total < 0x1p-14f && m > -1e29f ? __builtin_nanf("") : 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int y = 0; y < 16; ++y) bad = fmaf(acc[d][y], 0.f, bad);
    return __builtin_amdgcn_ballot_w64(there && bad != bad) != 0;
}

__global__ __launch_bounds__(kPrefillThreads) __attribute__((amdgpu_waves_per_eu(2, 2))) void prefill_kernel(PrefillArgs p)
{
    __shared__ __align__(256) uint8_t s_tiles[2][2][kTileBytes];           // [buffer][keys | values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hl = lane >> 5, col = lane & 31;
    // the last tiles of a sequence, which see the most keys, come first
    const uint32_t slot = p.slots - 1 - blockIdx.x / (uint32_t)p.Hkv;
    const int hk = (int)(blockIdx.x % (uint32_t)p.Hkv);
    RowTile<kBM, kBN> t;
    if (!t.find(p, slot, lane)) return;
    // workgroups that share the keys take one range of the list after the other
    const int nwg = attending(p, t), split = blockIdx.y, per = (t.n + nwg - 1) / nwg, it0 = min(split * per, t.n), n = min(t.n, it0 + per) - it0;
    if (split >= nwg) return;
    const int q0 = t.q0, Tq = t.Tq, Tk = t.Tk, n_first = t.n_first, gap = t.gap;
    // this lane's row
    int i, j;
    t.row(p, wave * 32 + col, i, j);
    const bool there = i < Tq;
    const int pos = Tk - Tq + i;
    // the wave's positions; hi < lo: no row
    const int lo_wave = Tk - Tq + (t.first + wave * 32) / p.r, hi_wave = Tk - Tq + min((t.first + wave * 32 + 31) / p.r, Tq - 1);
    // tiles of the list that hold a key which some row of the wave sees
    const int tiles_wave = hi_wave < max(lo_wave, 0) ? 0 : hi_wave / kBN + 1;
    const int n_wave = min((tiles_wave <= n_first ? tiles_wave : max(tiles_wave - gap, n_first)) - it0, n);

    const __half* k_rows = p.k + (int64_t)t.k0 * p.k_stride + hk * kD;
    const __half* v_rows = p.v + (int64_t)t.k0 * p.v_stride + hk * kD;
    auto tile_of = [&](int it) __attribute__((always_inline)) { return t.tile_of(it0 + it); };
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
        if (masked) {
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int y = 0; y < 16; ++y) sc[x][y] = 32 * x + 8 * (y >> 2) + (y & 3) <= at_most ? sc[x][y] : -__builtin_inff();
            if (p.window)
#pragma unroll
                for (int x = 0; x < 2; ++x)
#pragma unroll
                    for (int y = 0; y < 16; ++y) {
                        const int e = 32 * x + 8 * (y >> 2) + (y & 3);
                        sc[x][y] = e > above || e < below ? sc[x][y] : -__builtin_inff();
                    }
            top = top_of(sc);
        }
        if (__builtin_amdgcn_ballot_w64(top > m + (kLead + kSlack)) != 0) {
            const float raised = fmaxf(m, top - kLead), alpha = __builtin_amdgcn_exp2f((m - raised) * kScale);
            m = raised;
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
    __syncthreads();                                                       // everyone has left the tiles
    float total = (l[0] + l[1]) + (l[2] + l[3]);
    total += __shfl_xor(total, 32, 64);
    const bool odd = to_redo(acc, m, total, there);
    if (odd && nwg == 1) {
        redo_rows(p, t, hk, wave * 32, wave * 32 + 32, lane);
        return;
    }
    if (nwg > 1) {                                                         // to be added up by the second launch
        if (!there) return;
        float* mine = p.parts + ((((size_t)slot * p.Hkv + hk) * p.ns + split) * kBM + wave * 32 + col) * kPart;
#pragma unroll
        for (int d = 0; d < 4; ++d)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                *reinterpret_cast<float4*>(mine + 32 * d + 8 * y + 4 * hl) = make_float4(acc[d][4 * y], acc[d][4 * y + 1], acc[d][4 * y + 2], acc[d][4 * y + 3]);
        if (hl == 0) *reinterpret_cast<float4*>(mine + kD) = make_float4(m * kScale, total, odd ? 1.f : 0.f, 0.f);
        return;
    }
    // rows leave through LDS, 16 bytes a lane and whole rows of 256 (8 bytes a lane of 64 rows' pieces otherwise)
    const float inv = factor(1.f / total, pos);
    uint8_t* own = reinterpret_cast<uint8_t*>(&s_tiles[0][0][0]) + wave * 32 * kRowPitch;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const h2 a = {(_Float16)(acc[d][4 * y] * inv), (_Float16)(acc[d][4 * y + 1] * inv)};
            const h2 c = {(_Float16)(acc[d][4 * y + 2] * inv), (_Float16)(acc[d][4 * y + 3] * inv)};
            *reinterpret_cast<uint2*>(own + col * kRowPitch + (32 * d + 8 * y + 4 * hl) * 2) = make_uint2(__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, c));
        }
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");                 // the wave's own LDS writes, then its reads
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
#pragma unroll
    for (int x = 0; x < 8; ++x) {
        const int row = 4 * x + (lane >> 4);
        if (wave * 32 + row >= t.rows(p)) break;
        int query, head;
        t.row(p, wave * 32 + row, query, head);
        reinterpret_cast<uint4*>(p.out + ((int64_t)(q0 + query) * p.H + hk * p.r + head) * kD)[lane & 15] =
            *reinterpret_cast<const uint4*>(own + row * kRowPitch + (lane & 15) * 16);
    }
}

// ------------------------------------------------------------------------------------------
// Few rows.  A workgroup takes 32 rows, and its four waves take key tiles of 32 in turn, each through a ring of its own in LDS (two tiles of
// keys and values), without meeting; p.ns workgroups stand by for a row tile, of which as many attend as get kNarrowDeal key tiles a
// wave.  Sums, references and weight sums of the waves meet in LDS, those of the workgroups in the workspace, added up by a second launch.
// ------------------------------------------------------------------------------------------
constexpr int kRing = 2 * kKeys * kRowBytes;             // a key tile's keys and values

__global__ __launch_bounds__(kPrefillThreads) __attribute__((amdgpu_waves_per_eu(1, 1))) void prefill_narrow_kernel(PrefillArgs p)
{
    __shared__ __align__(256) uint8_t s_ring[4][2][kRing];                 // [wave][buffer][keys, values]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int hl = lane >> 5, col = lane & 31;
    const uint32_t slot = p.slots - 1 - blockIdx.x / (uint32_t)p.Hkv;
    const int hk = (int)(blockIdx.x % (uint32_t)p.Hkv), split = blockIdx.y;
    RowTile<kRows, kKeys> t;
    if (!t.find(p, slot, lane)) return;
    const int nwg = attending(p, t);
    if (split >= nwg) return;
    int i, j;
    t.row(p, col, i, j);
    const bool there = i < t.Tq;
    const int pos = t.Tk - t.Tq + i, at_once = 4 * nwg, mine0 = split * 4 + wave;
    const int n = mine0 < t.n ? (t.n - mine0 + at_once - 1) / at_once : 0;

    const __half* k_rows = p.k + (int64_t)t.k0 * p.k_stride + hk * kD;
    const __half* v_rows = p.v + (int64_t)t.k0 * p.v_stride + hk * kD;
    const uint32_t lds = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&s_ring[wave][0][0];
    auto first_key = [&](int it) __attribute__((always_inline)) { return t.tile_of(mine0 + it * at_once) * kKeys; };
    auto fetch = [&](int it) __attribute__((always_inline)) {              // rows past the end repeat the last one
        const int t0 = first_key(it), most = t.Tk - 1 - t0;
        const uint32_t to = lds + (it & 1) * kRing;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int row = 4 * x + (lane >> 4);
            dma16(k_rows + (int64_t)t0 * p.k_stride, (uint32_t)(min(row, most) * (int)p.k_stride * 2 + k_place(row, lane & 15) * 16), to + x * 1024);
        }
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const int row = 4 * x + (lane >> 4);
            dma16(v_rows + (int64_t)t0 * p.v_stride, (uint32_t)(min(row, most) * (int)p.v_stride * 2 + v_place(row, lane & 15) * 16),
                  to + kKeys * kRowBytes + x * 1024);
        }
    };
    h8 qf[8];
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(t.q0 + (there ? i : 0)) * p.q_stride + (hk * p.r + (there ? j : 0)) * kD);
        const uint32_t some = there ? ~0u : 0u;
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const uint4 x = src[2 * s + hl];
            qf[s] = __builtin_bit_cast(h8, make_uint4(x.x & some, x.y & some, x.z & some, x.w & some));
        }
    }
    if (n > 0) fetch(0);
    if (n > 1) fetch(1);
    float m = -1e30f, l[4] = {0.f, 0.f, 0.f, 0.f};
    f16v acc[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = (f16v)(0.f);
    const int key = 4 * hl + ((lane & 15) >> 2), within = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    for (int it = 0; it < n; ++it) {
        if (it + 1 < n) wait_vmcnt<16>();                                  // the next tile may still be on its way
        else wait_vmcnt<0>();
        const uint8_t* ks = s_ring[wave][it & 1];
        const uint8_t* vs = ks + kKeys * kRowBytes;
        auto values = [&](int s, int d) __attribute__((always_inline)) {
            const uint8_t* at = vs + (16 * s + key) * kRowBytes + v_place(key, 4 * d + within) * 16 + (lane & 1) * 8;
            return v_operand(at, at + 8 * kRowBytes);
        };
        f16v sc[2] = {(f16v)(0.f), (f16v)(0.f)};                           // two chains of products
#pragma unroll
        for (int s = 0; s < 8; ++s)
            sc[s & 1] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(ks + col * kRowBytes + k_place(col, 2 * s + hl) * 16), qf[s], sc[s & 1], 0, 0, 0);
        sc[0] += sc[1];
        const int t0 = first_key(it), t1 = t0 + kKeys - 1;
        if (!(t1 <= t.lo_pos && (!p.window || t0 > t.hi_pos - p.window || t1 < p.sinks))) {
            const int at_most = (there ? pos - t0 : -1) - 4 * hl, above = (p.window ? pos - p.window - t0 : -1) - 4 * hl, below = p.sinks - t0 - 4 * hl;
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                const int e = 8 * (y >> 2) + (y & 3);
                sc[0][y] = e <= at_most && (e > above || e < below) ? sc[0][y] : -__builtin_inff();
            }
        }
        float top = m;
#pragma unroll
        for (int y = 0; y < 16; ++y) top = fmaxf(top, sc[0][y]);
        top = max_other_half(top);
        if (__builtin_amdgcn_ballot_w64(top > m + (kLead + kSlack)) != 0) {
            const float raised = fmaxf(m, top - kLead), alpha = __builtin_amdgcn_exp2f((m - raised) * kScale);
            m = raised;
#pragma unroll
            for (int x = 0; x < 4; ++x) l[x] *= alpha;
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[d] *= alpha;
        }
        const float shift = -m * kScale;
        h8 w[2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            h2 o[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                o[y] = (h2){(_Float16)__builtin_amdgcn_exp2f(fmaf(sc[0][8 * s + 2 * y], kScale, shift)),
                            (_Float16)__builtin_amdgcn_exp2f(fmaf(sc[0][8 * s + 2 * y + 1], kScale, shift))};
                l[y] = __builtin_amdgcn_fdot2(o[y], (h2){(_Float16)1.f, (_Float16)1.f}, l[y], false);
            }
            w[s] = join(o[0], o[1], o[2], o[3]);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(values(s, d), w[s], acc[d], 0, 0, 0);
        if (it + 2 < n) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");             // the ring's tile has been read
            fetch(it + 2);
        }
    }
    // ---- the waves meet ----
    float total = (l[0] + l[1]) + (l[2] + l[3]);
    total += __shfl_xor(total, 32, 64);
    const bool odd = to_redo(acc, m, total, there);
    float* own = reinterpret_cast<float*>(&s_ring[wave][0][0]) + col * kPart;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int y = 0; y < 4; ++y)
            *reinterpret_cast<float4*>(own + 32 * d + 8 * y + 4 * hl) = make_float4(acc[d][4 * y], acc[d][4 * y + 1], acc[d][4 * y + 2], acc[d][4 * y + 3]);
    if (hl == 0) *reinterpret_cast<float4*>(own + kD) = make_float4(m * kScale, total, odd ? 1.f : 0.f, 0.f);
    __syncthreads();
    const int rows = t.rows(p);
    float* part = p.parts + (((size_t)slot * p.Hkv + hk) * p.ns + split) * kRows * kPart;
    bool again = false;
    for (int x = threadIdx.x; x < rows * (kD / 4); x += kPrefillThreads) {
        const int row = x / (kD / 4), d = x % (kD / 4) * 4;
        float4 ml[4];
        float most = -1e30f * kScale, sum = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            ml[w] = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(&s_ring[w][0][0]) + row * kPart + kD);
            most = fmaxf(most, ml[w].x);
        }
        float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
        bool redo = false;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float4 a = *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(&s_ring[w][0][0]) + row * kPart + d);
            const float f = __builtin_amdgcn_exp2f(ml[w].x - most);
            num.x = fmaf(a.x, f, num.x); num.y = fmaf(a.y, f, num.y); num.z = fmaf(a.z, f, num.z); num.w = fmaf(a.w, f, num.w);
            sum = fmaf(ml[w].y, f, sum);
            redo |= ml[w].z != 0.f;
        }
        again |= redo;
        if (nwg > 1) {
            *reinterpret_cast<float4*>(part + row * kPart + d) = num;
            if (d == 0) *reinterpret_cast<float4*>(part + row * kPart + kD) = make_float4(most, sum, redo ? 1.f : 0.f, 0.f);
        } else if (!redo) {
            write_out(p, t, hk, row, d, num, 1.f / sum);
        }
    }
    // (a wave's `odd` stands at all of its rows, so every thread that has a row knows)
    if (nwg == 1 && __builtin_amdgcn_ballot_w64(again) != 0) redo_rows(p, t, hk, wave * 8, wave * 8 + 8, lane);
}

// Second launch: the workgroups' partial results of a row tile, added up in their order.
template <int ROWS, int BN>
__global__ __launch_bounds__(kPrefillThreads) void prefill_combine_kernel(PrefillArgs p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t slot = blockIdx.x / (uint32_t)p.Hkv;
    const int hk = (int)(blockIdx.x % (uint32_t)p.Hkv);
    RowTile<ROWS, BN> t;
    if (!t.find(p, slot, lane)) return;
    const int nwg = attending(p, t), rows = t.rows(p);
    if (nwg == 1 || (int)blockIdx.y * 8 >= rows) return;
    const float* parts = p.parts + ((size_t)slot * p.Hkv + hk) * p.ns * ROWS * kPart;
    // eight rows of the tile to a workgroup, two to a wave
    const int row = blockIdx.y * 8 + wave * 2 + (lane >> 5), d = (lane & 31) * 4;
    const bool there = row < rows;
    float most = -1e30f * kScale, sum = 0.f;
    float4 num = make_float4(0.f, 0.f, 0.f, 0.f);
    bool redo = false;
    for (int s0 = 0; s0 < nwg; s0 += 8) {
        float4 a[8], ml[8];
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const float* at = parts + ((size_t)min(s0 + s, nwg - 1) * ROWS + (there ? row : 0)) * kPart;
            a[s] = *reinterpret_cast<const float4*>(at + d);
            ml[s] = *reinterpret_cast<const float4*>(at + kD);
        }
        float top = most;
#pragma unroll
        for (int s = 0; s < 8; ++s) top = fmaxf(top, ml[s].x);
        const float keep = __builtin_amdgcn_exp2f(most - top);
        num.x *= keep; num.y *= keep; num.z *= keep; num.w *= keep;
        sum *= keep;
        most = top;
#pragma unroll
        for (int s = 0; s < 8; ++s)
            if (s0 + s < nwg) {
                const float f = __builtin_amdgcn_exp2f(ml[s].x - top);
                num.x = fmaf(a[s].x, f, num.x); num.y = fmaf(a[s].y, f, num.y); num.z = fmaf(a[s].z, f, num.z); num.w = fmaf(a[s].w, f, num.w);
                sum = fmaf(ml[s].y, f, sum);
                redo |= ml[s].z != 0.f;
            }
    }
    if (there && !redo) write_out(p, t, hk, row, d, num, 1.f / sum);
    if (__builtin_amdgcn_ballot_w64(there && redo) != 0) redo_rows(p, t, hk, blockIdx.y * 8 + wave * 2, blockIdx.y * 8 + wave * 2 + 2, lane);
}

}  // namespace

static int64_t row_tiles(int64_t M, int64_t B, int64_t H, int64_t Hkv, int64_t rows) { return (M * (H / Hkv) / rows + B) * Hkv; }
// Which kernel, and how many workgroups stand by for each of its row tiles.  The host knows the rows and the sequences, not their
// lengths: `seen` is what a row may see, of twice the mean length.
// The narrow kernel reads the keys again for every 32 rows, the wide one for every 128, but has a compute unit's four waves on different
// keys.  Measured, narrow and wide: 32 / 8 heads, 20 tokens behind 3000 15.0 and 17.7 us, 200 behind 4000 45 and 36, 300 behind 2000 48 and 32; 200 alone
// 8.8 and 13.3; 32 / 32 heads, 256 alone 9.0 and 15.2, 512 18.4 and 21.5; 32 / 8 heads, 800 alone 34 and 23.
// The keys of wide tiles are shared while there are less than two for each compute unit: 512 behind 4000 88 us whole, 60 shared; not where a
// workgroup is through them before a second launch pays: 800 alone 23 whole, 28 shared, 1024 alone of 32 / 32 heads 28 and 38.
struct Plan { bool narrow; int ns; int64_t tiles; };
static Plan prefill_plan(int64_t M, int64_t Mk, int64_t B, int64_t H, int64_t Hkv, int64_t window, int64_t sinks)
{
    const int64_t narrow_tiles = row_tiles(M, B, H, Hkv, kRows);
    int64_t seen = std::min(Mk, 2 * (Mk / std::max<int64_t>(B, 1) + 1));
    if (window) seen = std::min(seen, window + sinks + std::min<int64_t>(M, kRows));
    const bool narrow = narrow_tiles <= 128 || (narrow_tiles <= 640 && narrow_tiles * seen <= 512 * 1024);
    const int64_t tiles = narrow ? narrow_tiles : row_tiles(M, B, H, Hkv, kBM);
    const int64_t deal = narrow ? 4 * kNarrowDeal * kKeys : kWideDeal * kBN;
    int64_t ns = 1;
    if (narrow || seen > 1024) {
        ns = std::min<int64_t>((narrow ? 256 : 512) / std::max<int64_t>(tiles, 1), kMaxParts);
        ns = std::min(ns, (seen + 2 * kBN + deal - 1) / deal);
    }
    return {narrow, (int)std::max<int64_t>(ns, 1), tiles};
}

size_t prefill_workspace_bytes(int64_t M, int64_t Mk, int64_t B, int64_t H, int64_t Hkv, int64_t window, int64_t sinks)
{
    const Plan plan = prefill_plan(M, Mk, B, H, Hkv, window, sinks);
    return plan.ns <= 1 ? 0 : kCounterBytes + (size_t)(plan.tiles * plan.ns * (plan.narrow ? kRows : kBM) * kPart) * sizeof(float);
}

hipError_t launch_prefill(const Prefill& a, hipStream_t s)
{
    PrefillArgs p{};
    p.q = static_cast<const __half*>(a.q); p.k = static_cast<const __half*>(a.k); p.v = static_cast<const __half*>(a.v);
    p.out = static_cast<__half*>(a.out);
    p.cu_q = a.cu_q; p.cu_k = a.cu_k;
    p.q_stride = a.q_stride; p.k_stride = a.k_stride; p.v_stride = a.v_stride;
    p.M = (int)a.M; p.Mk = (int)a.Mk; p.B = (int)a.B; p.H = (int)a.H; p.Hkv = (int)a.Hkv; p.r = (int)(a.H / a.Hkv);
    p.window = (int)a.window; p.sinks = a.window ? (int)a.sinks : 0;
    const Plan plan = prefill_plan(a.M, a.Mk, a.B, a.H, a.Hkv, a.window, a.sinks);
    if (plan.tiles > kMaxGrid) return hipErrorInvalidValue;
    p.slots = (uint32_t)(plan.tiles / a.Hkv);
    p.ns = a.workspace ? plan.ns : 1;
    p.parts = p.ns > 1 ? reinterpret_cast<float*>(static_cast<char*>(a.workspace) + kCounterBytes) : nullptr;
    const dim3 grid((unsigned)plan.tiles, (unsigned)p.ns);
    if (plan.narrow) prefill_narrow_kernel<<<grid, kPrefillThreads, 0, s>>>(p);
    else prefill_kernel<<<grid, kPrefillThreads, 0, s>>>(p);
    if (p.ns > 1) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        if (plan.narrow) prefill_combine_kernel<kRows, kKeys><<<dim3((unsigned)plan.tiles, kRows / 8), kPrefillThreads, 0, s>>>(p);
        else prefill_combine_kernel<kBM, kBN><<<dim3((unsigned)plan.tiles, kBM / 8), kPrefillThreads, 0, s>>>(p);
    }
    return hipGetLastError();
}

}  // namespace qoq
