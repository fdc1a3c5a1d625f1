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

    const __half* k_rows = p.k + (int64_t)k0 * p.k_stride + hk * kD;
    const __half* v_rows = p.v + (int64_t)k0 * p.v_stride + hk * kD;
    auto tile_of = [&](int it) __attribute__((always_inline)) { return it < n_first ? it : it + gap; };
    // a wave copies 16 rows of the keys and of the values of a tile; rows past the end repeat the last one
    auto fetch = [&](int it) __attribute__((always_inline)) {
        const int t0 = tile_of(it) * kBN, most = Tk - 1 - t0;
        const uint32_t to = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t*)&s_tiles[it & 1][0][0] + wave * 4096;
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int row = wave * 16 + x * 4 + (lane >> 4), at = min(row, most);
            dma16(k_rows + (int64_t)t0 * p.k_stride, (uint32_t)(at * (int)p.k_stride * 2 + k_place(row, lane & 15) * 16), to + x * 1024);
        }
#pragma unroll
        for (int x = 0; x < 4; ++x) {
            const int row = wave * 16 + x * 4 + (lane >> 4), at = min(row, most);
            dma16(v_rows + (int64_t)t0 * p.v_stride, (uint32_t)(at * (int)p.v_stride * 2 + v_place(row, lane & 15) * 16), to + kTileBytes + x * 1024);
        }
    };
    if (n > 0) fetch(0);

    h8 qf[8];                                                              // elements 16 s + 8 hl .. of this lane's row
    {
        const uint4* src = reinterpret_cast<const uint4*>(p.q + (int64_t)(q0 + (there ? i : 0)) * p.q_stride + (hk * p.r + (there ? j : 0)) * kD);
#pragma unroll
        for (int s = 0; s < 8; ++s) {
            const uint4 t = src[2 * s + hl];
            qf[s] = __builtin_bit_cast(h8, there ? t : make_uint4(0, 0, 0, 0));
        }
    }
    float m = -1e30f, l = 0.f;                                             // l: of this lane's keys
    f16v acc[4];
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = (f16v)(0.f);

    auto compute = [&](int it, auto masked_tag) __attribute__((always_inline)) {
        constexpr bool MASKED = decltype(masked_tag)::value;
        const int t0 = tile_of(it) * kBN;
        const uint8_t* ks = s_tiles[it & 1][0];
        const uint8_t* vs = s_tiles[it & 1][1];
        auto seen = [&](int t) { return there && t <= pos && (!p.window || t > pos - p.window || t < p.sinks); };
        f16v sc[2];                                                        // sc[x][y]: key 32 x + 8 (y / 4) + 4 hl + y % 4
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            sc[x] = (f16v)(0.f);
#pragma unroll
            for (int s = 0; s < 8; ++s) {
                const h8 a = *reinterpret_cast<const h8*>(ks + (32 * x + col) * kRowBytes + k_place(col, 2 * s + hl) * 16);
                sc[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, qf[s], sc[x], 0, 0, 0);
            }
        }
        float top = m;
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int y = 0; y < 16; ++y) {
                if (MASKED) sc[x][y] = seen(t0 + 32 * x + 8 * (y >> 2) + 4 * hl + (y & 3)) ? sc[x][y] : -__builtin_inff();
                top = fmaxf(top, sc[x][y]);
            }
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        if (__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0) {
            const float alpha = __builtin_amdgcn_exp2f((m - top) * kScale);
            m = top;
            l *= alpha;
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[d] *= alpha;
        }
        const float shift = -m * kScale;
        h8 w[4];                                                           // weights of 16 keys each
#pragma unroll
        for (int x = 0; x < 2; ++x)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                h2 o[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float a = __builtin_amdgcn_exp2f(fmaf(sc[x][8 * half + 2 * y], kScale, shift));
                    const float c = __builtin_amdgcn_exp2f(fmaf(sc[x][8 * half + 2 * y + 1], kScale, shift));
                    l += a + c;
                    o[y] = (h2){(_Float16)a, (_Float16)c};
                }
                w[2 * x + half] = join(o[0], o[1], o[2], o[3]);
            }
        const int key = 4 * hl + ((lane & 15) >> 2);                       // of the 8-key groups: the row this lane addresses
        const int within = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);      // 16-byte chunk of the 64 bytes of 32 elements
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            h8 a[4];
#pragma unroll
            for (int d = 0; d < 4; ++d) {
                const uint8_t* at = vs + (16 * s + key) * kRowBytes + v_place(key, 4 * d + within) * 16 + (lane & 1) * 8;
                a[d] = v_operand(at, at + 8 * kRowBytes);
            }
            if (MASKED) {
                // A zero weight times infinity or NaN is NaN: values that are not finite leave the product and reach the rows that
                // see their key by themselves, counted by a product with zeros and ones (+infinity 1, -infinity 128, NaN 16384).
                float bad = 0.f;
#pragma unroll
                for (int d = 0; d < 4; ++d) {
                    struct { h2 v[4]; } t = __builtin_bit_cast(decltype(t), a[d]);
#pragma unroll
                    for (int x = 0; x < 4; ++x) bad = __builtin_amdgcn_fdot2(t.v[x], (h2){(_Float16)0.f, (_Float16)0.f}, bad, false);
                }
                if (__builtin_amdgcn_ballot_w64(bad != bad) != 0) {
                    h8 sees;
#pragma unroll
                    for (int x = 0; x < 8; ++x) sees[x] = (_Float16)(seen(t0 + 16 * s + 8 * (x >> 2) + 4 * hl + (x & 3)) ? 1.f : 0.f);
#pragma unroll
                    for (int d = 0; d < 4; ++d) {
                        h8 clean = a[d], code;
#pragma unroll
                        for (int x = 0; x < 8; ++x) {
                            const uint32_t bits = __builtin_bit_cast(unsigned short, (_Float16)a[d][x]);
                            const bool odd = (bits & 0x7C00u) == 0x7C00u;
                            code[x] = (_Float16)(!odd ? 0.f : (bits & 0x3FFu) ? 16384.f : (bits & 0x8000u) ? 128.f : 1.f);
                            clean[x] = odd ? (_Float16)0.f : a[d][x];
                        }
                        a[d] = clean;
                        const f16v count = __builtin_amdgcn_mfma_f32_32x32x16_f16(code, sees, (f16v)(0.f), 0, 0, 0);
#pragma unroll
                        for (int y = 0; y < 16; ++y) {
                            const int c = (int)count[y];
                            const bool plus = (c & 127) != 0, minus = (c & (16383 - 127)) != 0;
                            if (c) acc[d][y] += c >= 16384 || (plus && minus) ? __builtin_nanf("") : plus ? __builtin_inff() : -__builtin_inff();
                        }
                    }
                }
            }
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[d], w[s], acc[d], 0, 0, 0);
        }
    };
    for (int it = 0; it < n; ++it) {
        wait_vmcnt<0>();
        __syncthreads();                                                   // tile `it` is there, and everyone has left the other buffer
        if (it + 1 < n) fetch(it + 1);
        const int t0 = tile_of(it) * kBN, t1 = t0 + kBN - 1;
        if (t0 > hi_wave || hi_wave < lo_wave || (p.window && t1 <= lo_wave - p.window && t0 >= p.sinks)) continue;    // no row sees any
        if (t1 <= lo_wave && (!p.window || t0 > hi_wave - p.window || t1 < p.sinks)) compute(it, std::false_type{});
        else compute(it, std::true_type{});
    }
    l += __shfl_xor(l, 32, 64);
    if (!there) return;
    const float inv = l == 0.f ? 0.f : 1.f / l;                            // a row that sees nothing is zero (NaN stays)
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
