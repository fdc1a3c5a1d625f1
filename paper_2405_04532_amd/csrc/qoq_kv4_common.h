// What the kernels of the 4-bit KV cache share: the page's layout, the quantizer of a head, the unpacking of codes
// (internal to the library).  The layout is described in qoq_kv4.hip.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "qoq_fp16.h"
#include "qoq_internal.h"

namespace qoq {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ _Float16 half_of(uint32_t v) { return __builtin_bit_cast(_Float16, (unsigned short)v); }

constexpr int kD = 128;                       // head dimension
constexpr int kPageTokens = 64;
constexpr int kCodeBytes = kPageTokens * kD / 2;          // 4096
constexpr int kParamBytes = kPageTokens * 4;              // 256
constexpr int kHalfPage = kCodeBytes + kParamBytes;       // keys (or values) of a page
constexpr int kPageBytes = 2 * kHalfPage;                 // 8704

// byte offset, inside the value codes of a page, of the 16-bit word of token `tin` (0..63) and elements 4 q4 .. 4 q4 + 3
__device__ __forceinline__ int v_word_offset(int tin, int q4)
{
    const int tile = tin >> 4, kb = (tin >> 2) & 3, h = (tin >> 1) & 1, half = tin & 1;
    const int r = q4 & 15, u = q4 >> 4;
    return tile * 1024 + (kb * 16 + r) * 16 + (2 * u + h) * 4 + half * 2;
}

// minimum / maximum over a row of 16 lanes (cross-lane moves without LDS)
template <int CTRL>
__device__ __forceinline__ float row_move(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ float row_min16(float v)
{
    v = fminf(v, row_move<0x128>(v));                                      // rotations by 8, 4, 2, 1 lanes
    v = fminf(v, row_move<0x124>(v));
    v = fminf(v, row_move<0x122>(v));
    return fminf(v, row_move<0x121>(v));
}
__device__ __forceinline__ float row_max16(float v)
{
    v = fmaxf(v, row_move<0x128>(v));
    v = fmaxf(v, row_move<0x124>(v));
    v = fmaxf(v, row_move<0x122>(v));
    return fmaxf(v, row_move<0x121>(v));
}

// the larger of a lane's number and that of the lane 16 (32) further on or back: rows (halves) change places between two registers,
// without the way through LDS that a shuffle takes
__device__ __forceinline__ float max_other_row(float v)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float max_other_half(float v)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// Eq. 1 of one vector of 128 elements spread over a row of 16 lanes, 8 elements (16 bytes) each: this lane's eight codes, the
// scale's FP16 bits, and the FP16 bits of -(1024 + z) (an exact integer), the constant that the decode kernels add to their
// unpacked codes.  Lanes that hold nothing bring any words; every lane of a row has to take part.
//   s = FP16((hi - lo) / 15), the quotient in exact arithmetic rounded once: the FP32 quotient is within 4 * 2^-24 of it, so
//     where both ends of that interval round to the same FP16 number that is it; else (1 in 2000) the FP64 quotient decides
//   codes and z = floor(x / s + 1/2) + integer: |x / s| < 256 is on a half-integer or at least 2^-12 away from every one;
//     x * fl(1 / s) is within 3e-5 of it, and pushed 1e-4 upwards it lands on the side that rounding half up takes.
__device__ __forceinline__ void quantize_head(const uint4& raw, uint32_t (&c)[8], uint16_t& s_bits, uint32_t& z_bits)
{
    uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
    h2 mn = {(_Float16)0.f, (_Float16)0.f}, mx = mn;                   // the range is widened to contain 0
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        mn = __builtin_elementwise_min(mn, __builtin_bit_cast(h2, rw[e]));
        mx = __builtin_elementwise_max(mx, __builtin_bit_cast(h2, rw[e]));
    }
    const float lo = row_min16(fminf((float)mn.x, (float)mn.y)), hi = row_max16(fmaxf((float)mx.x, (float)mx.y));
    const float quot = (hi - lo) * (1.0f / 15.0f);
    float q_lo = quot * (1.0f - 4 * 0x1p-24f), q_hi = quot * (1.0f + 4 * 0x1p-24f);
    asm("" : "+v"(q_lo), "+v"(q_hi));                                  // no mixed-precision merging of product and conversion
    s_bits = __half_as_ushort(__float2half_rn(q_lo));
    if (s_bits != __half_as_ushort(__float2half_rn(q_hi))) s_bits = double_to_half_rne(((double)hi - (double)lo) / 15.0);
    if ((s_bits & 0x7FFFu) == 0) s_bits = 0x3C00u;                     // all-zero vector: s = 1
    const float inv = 1.0f / __half2float(__ushort_as_half(s_bits));
    const float z = __builtin_amdgcn_fmed3f(floorf(fmaf(-lo, inv, 0.5f + 1e-4f)), 0.f, 15.f);
    const float offset = z + (0.5f + 1e-4f);
    // NaN, and infinity over an infinite scale, are quotient 0 (code z); times zero they leave NaN in the sum
    float bad = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) bad = __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, rw[e]), (h2){(_Float16)0.f, (_Float16)0.f}, bad, false);
    if (bad != bad)
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if ((~(rw[e >> 1] >> (16 * (e & 1))) & 0x7C00u) == 0) rw[e >> 1] &= 0xFFFFu << (16 * (~e & 1));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = (float)half_of(rw[e >> 1] >> (16 * (e & 1)));
        c[e] = (uint32_t)(int)__builtin_amdgcn_fmed3f(fmaf(x, inv, offset), 0.f, 15.f);
    }
    z_bits = __half_as_ushort(__float2half_rn(-1024.0f - z));
}

// Quantizes one head of four consecutive tokens, 16 lanes each (lane w of them holds elements 8w .. 8w+7), and writes it into the page at
// token `tin` of it where `valid`.  `whole`: the wave holds all four tokens of an aligned quad; `block`: 16 x 16 bytes of LDS of the wave.
template <bool VALUE>
__device__ __forceinline__ void write_token(const uint4& raw, uint8_t* page, int tin, int w, int lane, bool whole, bool valid, uint4* block)
{
    const int g = lane >> 4;                                               // token of the quad
    uint32_t c[8], z_bits;
    uint16_t s_bits;
    quantize_head(raw, c, s_bits, z_bits);
    if constexpr (!VALUE) {
        // keys: dword w = elements 8w .. 8w+7, element 8w+2j in nibble j of the low half, 8w+2j+1 of the high half
        uint32_t word = 0;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) word |= (c[2 * jj] << (4 * jj)) | (c[2 * jj + 1] << (16 + 4 * jj));
        if (valid) reinterpret_cast<uint32_t*>(page + tin * (kD / 2))[w] = word;
    } else {
        // values: 16-bit words of element quads 2w (elements 8w .. 8w+3) and 2w+1
        const uint32_t h0 = c[0] | (c[1] << 4) | (c[2] << 8) | (c[3] << 12);
        const uint32_t h1 = c[4] | (c[5] << 4) | (c[6] << 8) | (c[7] << 12);
        if (whole) {
            // inside the quad's 256-byte block: chunk r = q4 % 16, dword 2 (q4 / 16) + (g >> 1), half g & 1
            uint16_t* blk = reinterpret_cast<uint16_t*>(block);
            const int q4a = 2 * w, q4b = 2 * w + 1;
            blk[(q4a & 15) * 8 + (2 * (q4a >> 4) + (g >> 1)) * 2 + (g & 1)] = (uint16_t)h0;
            blk[(q4b & 15) * 8 + (2 * (q4b >> 4) + (g >> 1)) * 2 + (g & 1)] = (uint16_t)h1;
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");     // the wave's own LDS writes, then its reads
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            if (lane < 16) {
                const int tin0 = tin & ~3;                             // lanes 0..15 are token 0 of the quad: tin % 4 == 0
                uint8_t* dst = page + kHalfPage + (tin0 >> 4) * 1024 + (((tin0 >> 2) & 3) * 16 + lane) * 16;
                *reinterpret_cast<uint4*>(dst) = block[lane];
            }
        } else if (valid) {
            *reinterpret_cast<uint16_t*>(page + kHalfPage + v_word_offset(tin, 2 * w)) = (uint16_t)h0;
            *reinterpret_cast<uint16_t*>(page + kHalfPage + v_word_offset(tin, 2 * w + 1)) = (uint16_t)h1;
        }
    }
    if (valid && w == 0) {
        reinterpret_cast<uint32_t*>(page + (VALUE ? kHalfPage : 0) + kCodeBytes)[tin] = (uint32_t)s_bits | (z_bits << 16);
    }
}

// the four FP16 pairs of a code dword, minus the zero point: out[j] = (nibble j of the low half, of the high half)
// c = -(1024 + z), c16 = -(64 + z) = c + 960, per half
// (x & mask) | bits in one instruction.  All three sources are vector registers: with the two constants in scalar
// registers the instruction would exceed its one-scalar-operand limit and the compiler splits it in two.
__device__ __forceinline__ h2 and_or(uint32_t x, uint32_t mask, uint32_t bits)
{
    uint32_t r;
    asm("v_and_or_b32 %0, %1, %2, %3" : "=v"(r) : "v"(x), "v"(mask), "v"(bits));
    return __builtin_bit_cast(h2, r);
}
__device__ __forceinline__ void unpack4(uint32_t word, h2 c, h2 c16, h2 (&out)[4])
{
    const h2 sixteenth = {(_Float16)0.0625f, (_Float16)0.0625f};
    const uint32_t hi = word >> 8;
    out[0] = and_or(word, 0x000F000Fu, 0x64006400u) + c;
    out[1] = and_or(word, 0x00F000F0u, 0x64006400u) * sixteenth + c16;
    out[2] = and_or(hi, 0x000F000Fu, 0x64006400u) + c;
    out[3] = and_or(hi, 0x00F000F0u, 0x64006400u) * sixteenth + c16;
}

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ h8 join(h2 a, h2 b, h2 c, h2 d)
{
    struct { h2 v[4]; } t = {{a, b, c, d}};
    return __builtin_bit_cast(h8, t);
}
}  // namespace qoq
