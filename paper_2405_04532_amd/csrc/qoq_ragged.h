// Finding a row's sequence in a ragged batch (internal to the library).
//
// A batch of B sequences is described by cu[0 .. B]: sequence b owns the rows cu[b] .. cu[b + 1] - 1.  A grid is sized on the host,
// which knows the rows and B but not cu.  Where sequence b takes units of `unit` rows, its first unit has the number
// cu[b] / unit + extra * b, and every sequence has room: units(b) <= (cu[b + 1] / unit) - (cu[b] / unit) + extra.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "qoq_ragged_search.h"

namespace qoq {

constexpr int64_t kMaxGrid = (1 << 24) - 1;                 // workgroups of 256 threads: a grid's dimension has less than 2^32 threads

// Number of b in 1 .. B for which before(b) holds, a condition that is true up to some b and false from there on: a search by the
// 64 lanes of a wave, no round of loads for up to 64 sequences, one up to 4096.  The result is an `lo` in 0 .. B (whatever before() says) such that
// the number is lo plus the count of lanes below B - lo for which before(lo + lane + 1) holds; a count of 64 means that the number is B.
template <class F>
__device__ __forceinline__ int near_before(int B, int lane, F&& before)
{
    LaneSearch s{0, B};
    while (!s.near(B)) s.narrow(__popcll(__builtin_amdgcn_ballot_w64(s.asks(lane) && before(s.candidate(lane)))));
    return s.lo;
}
template <class F>
__device__ __forceinline__ int count_before(int B, int lane, F&& before)
{
    const int lo = near_before(B, lane, before);
    return lo + __popcll(__builtin_amdgcn_ballot_w64(lane < B - lo && before(lo + lane + 1)));
}

// 64 sequences from `lo` on, one to a lane, in flight at once: where their rows end and where those are placed.
struct Window {
    const int32_t *cu, *starts;
    int lo, held, end, start, begin;                         // end past the last sequence: above every row

    __device__ __forceinline__ void load(const int32_t* cu_, const int32_t* starts_, int B, int lo_, int lane)
    {
        cu = cu_;
        starts = starts_;
        lo = lo_;
        held = min(B - lo, 64);
        end = lane < held ? cu[lo + lane + 1] : INT32_MAX;
        start = lane < held && starts ? starts[lo + lane] : 0;
        begin = cu[lo];
    }
    // by every lane of the wave (a lane that is off gives no other its numbers); b: inside the window, or anywhere up to B - 1 with `far`
    __device__ __forceinline__ int first_row(int b, bool far) const
    {
        if (far) return cu[b];
        const int before = __shfl(end, max(b - lo - 1, 0), 64);
        return b > lo ? before : begin;
    }
    __device__ __forceinline__ int end_row(int b) const { return __shfl(end, b - lo, 64); }
    __device__ __forceinline__ int start_of(int b, bool far) const
    {
        if (far) return starts ? starts[b] : 0;
        return __shfl(start, b - lo, 64);
    }
};

}  // namespace qoq
