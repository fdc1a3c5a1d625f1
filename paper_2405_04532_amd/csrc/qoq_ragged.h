// Finding a row's sequence in a ragged batch (internal to the library).
//
// A batch of B sequences is described by cu[0 .. B]: sequence b owns the rows cu[b] .. cu[b + 1] - 1.  A grid is sized on the host,
// which knows the rows and B but not cu.  Where sequence b takes units of `unit` rows, its first unit has the number
// cu[b] / unit + extra * b, and every sequence has room: units(b) <= (cu[b + 1] / unit) - (cu[b] / unit) + extra.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qoq {

// Number of b in 1 .. B for which before(b) holds, a condition that is true up to some b and false from there on: a search by the
// 64 lanes of a wave, one round of loads for up to 64 sequences, two up to 4096.  The result lies in 0 .. B whatever before() says.
template <class F>
__device__ __forceinline__ int count_before(int B, int lane, F&& before)
{
    int lo = 0, n = B;                                       // the result lies in lo .. lo + n
    while (n > 64) {
        const int step = (n + 63) / 64, at = lo + (lane + 1) * step;
        const int c = __popcll(__builtin_amdgcn_ballot_w64(at <= lo + n && before(at)));
        n = min(step - 1, n - c * step);
        lo += c * step;
    }
    return lo + __popcll(__builtin_amdgcn_ballot_w64(lane < n && before(lo + lane + 1)));
}

}  // namespace qoq
