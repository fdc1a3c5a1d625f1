// Log probabilities of given tokens, entropy and the most likely tokens of rows of logits [M, V].
//
//   lse = log sum_j e^{x_j},  logprob = x_t - lse,  entropy = lse - sum_j p_j x_j,  rank = 1 + #{j in front of t}
// in the order of the logits, equal ones by their index.
//
// One pass over the row.  A lane holds a reference r, T = sum 2^(t_j) and U = sum 2^(t_j) t_j of the elements it has seen, t_j =
// log2(e) x_j - r: p_j = 2^(t_j) / T whatever r is, so r only has to keep the powers in range and follows the largest element in steps of
// more than kSlack.  entropy = ln T - ln 2 U / T, a sum of two terms that are not negative when r is the maximum.
//
// The most likely tokens: a lane remembers its largest element's vector.  Where n lanes of a wave have a largest element at or above
// some (value, index), there are n elements of that kind in the row, so nothing below it counts.  The wave finds its n-th largest in
// registers by ballots, bit by bit; the vectors of the lanes at or above the best wave's are looked through again (they are in the L2), and
// what is found is ranked by counting.
#include <hip/hip_fp16.h>

#include <algorithm>

#include "qoq_gemm_common.h"
#include "qoq_internal.h"
#include "qoq_workspace.h"

namespace qoq {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kInTurn = 4;                       // vectors of a lane in flight
constexpr int kMaxRowSplits = 64;                // workgroups to a row: the lanes of a wave
constexpr int kFound = 2048;                     // candidates that are ranked at once: all of a join's
constexpr float kSlack = 4.f;
constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.69314718055994530942;
constexpr double kLog2eOff = (double)kLog2e * kLn2 - 1.0;     // what FP32's log2(e) is off by, relative

struct LogprobArgs {
    const void* logits;
    int64_t stride;
    const int32_t* tokens;                       // or null
    float *logprob, *entropy;                    // or null
    int32_t* rank;                               // or null
    int32_t* top_ids;
    float* top_logprobs;
    int* counters;
    char* parts;
    int V, top, part_bytes;
};

struct Sums { float r, T, U; int count; };       // r in units of log2(e) x (FP16), of x (FP32)

// an element's (value, index): in front of another?
__device__ __forceinline__ bool in_front(float v, int i, float w, int j) { return v > w || (v == w && i < j); }

template <class T> struct Logit;
template <> struct Logit<__half> {
    static constexpr int kVec = 8;
    static constexpr float kLowest = -94600.f;                       // below log2(e) * -65504
    static __device__ __forceinline__ float unit(float x) { return x * kLog2e; }
    static __device__ __forceinline__ float term(float x, float r) { return fmaf(x, kLog2e, -r); }
    static __device__ __forceinline__ float step(float from, float to) { return from - to; }       // in units of log2
    static __device__ __forceinline__ void take(uint4 w, float (&x)[8])
    {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)__builtin_bit_cast(_Float16, (unsigned short)(u[e >> 1] >> (16 * (e & 1))));
    }
    static constexpr uint32_t kNone = 0xFC00FC00u;                   // minus infinity
    // ln sum e^x and the mean of x
    static __device__ double lse(const Sums& s, double mean_t) { return log((double)s.T) + s.r * kLn2 - kLog2eOff * (mean_t + s.r) / kLog2e; }
    static __device__ double logprob(float x, const Sums&, double lse) { return (double)x - lse; }
};
template <> struct Logit<float> {
    static constexpr int kVec = 4;
    static constexpr float kLowest = -3.402823466e38f;               // a row of the type's lowest value is a uniform one
    static __device__ __forceinline__ float unit(float x) { return x; }
    static __device__ __forceinline__ float term(float x, float r) { return (x - r) * kLog2e; }
    static __device__ __forceinline__ float step(float from, float to) { return (from - to) * kLog2e; }
    static __device__ __forceinline__ void take(uint4 w, float (&x)[4])
    {
        x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w);
    }
    static constexpr uint32_t kNone = 0xFF800000u;
    static __device__ double lse(const Sums& s, double mean_t) { return log((double)s.T) - kLog2eOff * mean_t / kLog2e; }      // of x - r
    static __device__ double logprob(float x, const Sums& s, double lse) { return ((double)x - (double)s.r) - lse; }
};

template <class T>
__device__ __forceinline__ Sums rebased(const Sums& s, float r)
{
    const float d = fmaxf(Logit<T>::step(s.r, r), -1e30f), f = __builtin_amdgcn_exp2f(d);
    return {r, s.T * f, f * fmaf(s.T, d, s.U), s.count};
}
template <class T>
__device__ __forceinline__ Sums all_lanes(Sums s)                    // of the wave, the same in every lane
{
    float r = s.r;
#pragma unroll
    for (int o = 32; o; o >>= 1) r = fmaxf(r, __shfl_xor(r, o, 64));
    s = rebased<T>(s, r);
#pragma unroll
    for (int o = 32; o; o >>= 1) {
        s.T += __shfl_xor(s.T, o, 64);
        s.U += __shfl_xor(s.U, o, 64);
        s.count += __shfl_xor(s.count, o, 64);
    }
    return s;
}

__device__ __forceinline__ uint32_t ascending(float v)               // unsigned numbers in the order of floats (no NaN, one zero)
{
    const uint32_t u = __float_as_uint(v + 0.f);
    return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
}

// The n-th in order of the (value, index) that the wave's lanes with `has` hold; the last of all where there are fewer.
__device__ __forceinline__ void nth_of_wave(float v, int i, bool has, int n, float& tau_v, int& tau_i)
{
    unsigned long long alive = __builtin_amdgcn_ballot_w64(has);
    tau_v = -__builtin_inff();
    tau_i = 0x7FFFFFFF;
    if (__builtin_popcountll(alive) < n) return;
    const uint32_t key = ascending(v);
    for (int bit = 31; bit >= 0; --bit) {
        const unsigned long long one = __builtin_amdgcn_ballot_w64((key >> bit) & 1) & alive;
        const int c = __builtin_popcountll(one);
        if (c >= n) alive = one;
        else { n -= c; alive &= ~one; }
    }
    tau_v = __shfl(v, __builtin_ctzll(alive), 64);
    for (int bit = 30; bit >= 0 && __builtin_popcountll(alive) > 1; --bit) {
        const unsigned long long zero = __builtin_amdgcn_ballot_w64(!((i >> bit) & 1)) & alive;
        const int c = __builtin_popcountll(zero);
        if (c >= n) alive = zero;
        else { n -= c; alive &= ~zero; }
    }
    tau_i = __shfl(i, __builtin_ctzll(alive), 64);
}

struct Shared {
    Sums sums[kRowWaves];
    float tau_v[kRowWaves];
    int tau_i[kRowWaves];
    int lanes, found, last;
    int lane[kRowThreads];
    float2 item[kFound];                                             // value, index
};

__device__ __forceinline__ void best_tau(const Shared& sh, float& v, int& i)
{
    v = sh.tau_v[0]; i = sh.tau_i[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w)
        if (in_front(sh.tau_v[w], sh.tau_i[w], v, i)) { v = sh.tau_v[w]; i = sh.tau_i[w]; }
}

// the found items ranked: put(place, value, index) for the first n places, an index of -1 where there is nothing
template <class Put>
__device__ __forceinline__ void put_ranked(const Shared& sh, int found, int n, Put put)
{
    for (int c = threadIdx.x; c < found; c += kRowThreads) {
        const float2 me = sh.item[c];
        int place = 0;
        for (int o = 0; o < found; ++o) {
            const float2 other = sh.item[o];
            place += in_front(other.x, __float_as_int(other.y), me.x, __float_as_int(me.y));
        }
        if (place < n) put(place, me.x, __float_as_int(me.y));
    }
    for (int c = found + threadIdx.x; c < n; c += kRowThreads) put(c, -__builtin_inff(), -1);
}

template <class T, bool TOP>
__global__ __launch_bounds__(kRowThreads) void logprobs_kernel(LogprobArgs p)
{
    using L = Logit<T>;
    constexpr int N = L::kVec;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x, split = blockIdx.y, splits = gridDim.y, V = p.V, n = p.top;
    const T* x_row = static_cast<const T*>(p.logits) + (int64_t)row * p.stride;
    // vectors of 16 aligned bytes, the first of which may begin in front of the row and the last end behind it
    const int before = (int)(((uintptr_t)x_row & 15) / sizeof(T));
    const uint4* vectors = reinterpret_cast<const uint4*>(x_row - before);
    const int all = (int)(((int64_t)before + V + N - 1) / N), share = (all + splits - 1) / splits;
    const int v0 = split * share, v1 = min(all, v0 + share);

    const int token = p.tokens ? p.tokens[row] : -1;
    const bool is_token = token >= 0 && token < V;
    const float xt = is_token ? (float)x_row[token] + 0.f : __builtin_inff();
    const int token_vector = is_token ? (token + before) / N : 0;
    // x > xt as x >= the next number
    const uint32_t xb = __float_as_uint(xt);
    const float xt_next = is_token ? __uint_as_float(xt >= 0.f ? xb + 1 : xb - 1) : __builtin_inff();

    auto load = [&](int v) __attribute__((always_inline)) {
        const int first = v * N - before;
        if (first >= 0 && first + N <= V) return vectors[v];
        uint32_t w[4] = {L::kNone, L::kNone, L::kNone, L::kNone};        // the ends of the row, an element at a time
        for (int e = 0; e < N; ++e)
            if (first + e >= 0 && first + e < V) {
                if constexpr (N == 8) {
                    const uint32_t u = __half_as_ushort(x_row[first + e]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k == e >> 1) w[k] = e & 1 ? (w[k] & 0xFFFFu) | u << 16 : (w[k] & 0xFFFF0000u) | u;
                } else {
                    const uint32_t u = __float_as_uint(x_row[first + e]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k == e) w[k] = u;
                }
            }
        return make_uint4(w[0], w[1], w[2], w[3]);
    };

    Sums s = {L::kLowest, 0.f, 0.f, 0};
    float best = -__builtin_inff();
    int best_vector = v0 + tid < v1 ? v0 + tid : -1;
    auto take = [&](uint4 w, int v) __attribute__((always_inline)) {
        float x[N];
        L::take(w, x);
        float most = fmaxf(x[0], x[1]);
#pragma unroll
        for (int e = 2; e < N; ++e) most = fmaxf(most, x[e]);
        if (TOP && most > best) { best = most; best_vector = v; }
        const float unit = L::unit(most);
        if (__builtin_amdgcn_ballot_w64(unit > s.r + kSlack) != 0)
            if (unit > s.r + kSlack) s = rebased<T>(s, unit);
        const float from = v < token_vector ? xt : xt_next;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float t = L::term(x[e], s.r), q = __builtin_amdgcn_exp2f(t);
            s.T += q;
            s.U = fmaf(q, fmaxf(t, -1e4f), s.U);                      // (minus infinity: 0 times a finite number)
            s.count += x[e] >= from;
        }
        if (v == token_vector)                                        // equal ones beside the token
#pragma unroll
            for (int e = 0; e < N; ++e) s.count += x[e] == xt && v * N - before + e < token && v * N - before + e >= 0;
    };
    int v = v0 + tid;
    for (; v + (kInTurn - 1) * kRowThreads < v1; v += kInTurn * kRowThreads) {
        uint4 w[kInTurn];
#pragma unroll
        for (int k = 0; k < kInTurn; ++k) w[k] = load(v + k * kRowThreads);
#pragma unroll
        for (int k = 0; k < kInTurn; ++k) take(w[k], v + k * kRowThreads);
    }
    for (; v < v1; v += kRowThreads) take(load(v), v);

    const Sums of_wave = all_lanes<T>(s);
    if (lane == 0) sh.sums[wave] = of_wave;
    if constexpr (TOP) {
        if (tid == 0) sh.lanes = sh.found = 0;
        float tau_v;
        int tau_i;
        nth_of_wave(best, min(best_vector * N - before + N - 1, V - 1), best_vector >= 0, n, tau_v, tau_i);
        if (lane == 0) { sh.tau_v[wave] = tau_v; sh.tau_i[wave] = tau_i; }
    }
    __syncthreads();
    Sums sum = sh.sums[0];
#pragma unroll
    for (int w = 1; w < kRowWaves; ++w) {
        const Sums o = sh.sums[w];
        const float r = fmaxf(sum.r, o.r);
        const Sums a = rebased<T>(sum, r), b = rebased<T>(o, r);
        sum = {r, a.T + b.T, a.U + b.U, a.count + b.count};
    }
    char* mine = p.parts + ((int64_t)row * splits + split) * p.part_bytes;
    double lse = 0;
    bool whole = true;                                                // not: the row holds NaN, plus infinity or nothing
    auto finish = [&]() {                                             // with `sum` that of the row
        whole = sum.T > 0.f && sum.T < __builtin_inff();
        const double mean = (double)sum.U / sum.T;
        lse = L::lse(sum, mean);
        if (tid == 0) {
            const float nan = __builtin_nanf("");
            if (p.logprob) p.logprob[row] = is_token && whole ? (float)L::logprob(xt, sum, lse) : nan;
            // (a token of minus infinity: what stands for the elements in front of the row was counted with its equals)
            const int extra = token_vector > 0 && xt == -__builtin_inff() ? before : 0;
            if (p.rank) p.rank[row] = is_token && whole ? sum.count + 1 - extra : 0;
            if (p.entropy) p.entropy[row] = whole ? fmaxf((float)(log((double)sum.T) - kLn2 * mean), 0.f) : nan;
        }
    };
    auto put_result = [&](int place, float value, int index) {
        p.top_ids[(int64_t)row * n + place] = whole ? index : -1;
        p.top_logprobs[(int64_t)row * n + place] = whole ? (float)L::logprob(value, sum, lse) : __builtin_nanf("");
    };
    auto put_part = [&](int place, float value, int index) {
        __hip_atomic_store(reinterpret_cast<unsigned long long*>(mine + 16) + place, (unsigned long long)__float_as_uint(value) | (unsigned long long)(uint32_t)index << 32,
                           __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    };
    if (splits == 1) finish();
    if constexpr (TOP) {
        float tau_v;
        int tau_i;
        best_tau(sh, tau_v, tau_i);
        if (best_vector >= 0 && (best > tau_v || (best == tau_v && best_vector * N - before <= tau_i))) sh.lane[atomicAdd(&sh.lanes, 1)] = tid;
        __syncthreads();
        const int steps = (share + kRowThreads - 1) / kRowThreads, items = sh.lanes * steps;
        for (int c = tid; c < items; c += kRowThreads) {
            const int q = c / steps, at = v0 + sh.lane[q] + (c - q * steps) * kRowThreads;
            if (at >= v1) continue;
            float x[N];
            L::take(load(at), x);
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int i = at * N - before + e;
                if (i >= 0 && i < V && (x[e] > tau_v || (x[e] == tau_v && i <= tau_i))) {
                    const int place = atomicAdd(&sh.found, 1);
                    if (place < kFound) sh.item[place] = make_float2(x[e], __int_as_float(i));
                }
            }
        }
        __syncthreads();
        const int found = sh.found;
        if (found <= kFound) {
            if (splits == 1) put_ranked(sh, found, n, put_result);
            else put_ranked(sh, found, n, put_part);
        } else {
            // More than can be ranked, as where large elements lie a workgroup's stride apart: one after the other, the row read for each.
            float last_v = __builtin_inff();
            int last_i = -1;
            for (int k = 0; k < n; ++k) {
                float bv = -__builtin_inff();
                int bi = 0x7FFFFFFF;
                for (int at = v0 + tid; at < v1; at += kRowThreads) {
                    float x[N];
                    L::take(load(at), x);
#pragma unroll
                    for (int e = 0; e < N; ++e) {
                        const int i = at * N - before + e;
                        if (i >= 0 && i < V && in_front(last_v, last_i, x[e], i) && in_front(x[e], i, bv, bi)) { bv = x[e]; bi = i; }
                    }
                }
#pragma unroll
                for (int o = 32; o; o >>= 1) {
                    const float ov = __shfl_xor(bv, o, 64);
                    const int oi = __shfl_xor(bi, o, 64);
                    if (in_front(ov, oi, bv, bi)) { bv = ov; bi = oi; }
                }
                __syncthreads();
                if (lane == 0) { sh.tau_v[wave] = bv; sh.tau_i[wave] = bi; }
                __syncthreads();
                best_tau(sh, last_v, last_i);
                if (tid == 0) {
                    if (splits == 1) put_result(k, last_v, last_i);
                    else put_part(k, last_v, last_i);
                }
            }
        }
    }
    if (splits == 1) return;
    if (tid == 0) store_through(reinterpret_cast<int4*>(mine), __float_as_int(sum.r), __float_as_int(sum.T), __float_as_int(sum.U), sum.count);
    // The stores above went past the caches that other workgroups do not share; they have arrived when the counter is raised.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (tid == 0) {
        const int old = __hip_atomic_fetch_add(p.counters + row, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh.last = old == splits - 1;
        if (old == splits - 1) __hip_atomic_store(p.counters + row, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh.found = 0;
    }
    __syncthreads();
    if (!sh.last) return;
    // The join, by the last workgroup of the row: a lane to a workgroup's sums, then the first n of their lists.
    const char* parts = p.parts + (int64_t)row * splits * p.part_bytes;
    const v4i part = load_through(reinterpret_cast<const int4*>(parts + (int64_t)min(lane, splits - 1) * p.part_bytes));
    constexpr int kEach = kMaxRowSplits * 32 / kRowThreads;
    float cv[kEach];
    int ci[kEach];
    if constexpr (TOP) {
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const int c = tid + k * kRowThreads, of = c / n;
            cv[k] = -__builtin_inff();
            ci[k] = -1;
            if (of < splits) {
                unsigned long long* at = reinterpret_cast<unsigned long long*>(const_cast<char*>(parts) + (int64_t)of * p.part_bytes + 16) + (c - of * n);
                const unsigned long long u = __hip_atomic_load(at, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                cv[k] = __uint_as_float((uint32_t)u);
                ci[k] = (int)(uint32_t)(u >> 32);
            }
        }
    }
    Sums mine_of = {__int_as_float(part.x), __int_as_float(part.y), __int_as_float(part.z), part.w};
    if (lane >= splits) mine_of = {L::kLowest, 0.f, 0.f, 0};
    sum = all_lanes<T>(mine_of);
    finish();
    if constexpr (TOP) {
        float bv = -__builtin_inff();
        int bi = -1;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (ci[k] >= 0 && (bi < 0 || in_front(cv[k], ci[k], bv, bi))) { bv = cv[k]; bi = ci[k]; }
        float tau_v;
        int tau_i;
        nth_of_wave(bv, bi, bi >= 0, n, tau_v, tau_i);
        if (lane == 0) { sh.tau_v[wave] = tau_v; sh.tau_i[wave] = tau_i; }
        __syncthreads();
        best_tau(sh, tau_v, tau_i);
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            if (ci[k] >= 0 && (cv[k] > tau_v || (cv[k] == tau_v && ci[k] <= tau_i))) sh.item[atomicAdd(&sh.found, 1)] = make_float2(cv[k], __int_as_float(ci[k]));
        __syncthreads();
        put_ranked(sh, sh.found, n, put_result);
    }
}

// Workgroups to a row: enough to fill the chip, none without vectors for its lanes.
int row_splits(int64_t M, int64_t V, int wide)
{
    if (M > kMaxCounters) return 1;
    const int64_t vectors = (V + (wide ? 3 : 7)) / (wide ? 4 : 8);
    return (int)std::max<int64_t>(1, std::min<int64_t>({kMaxRowSplits, 1024 / M, (vectors + kRowThreads - 1) / kRowThreads}));
}
int64_t row_part_bytes(int64_t top) { return (16 + 8 * top + 15) / 16 * 16; }

}  // namespace

size_t logprobs_workspace_bytes(int64_t M, int64_t V, int64_t top, int wide)
{
    const int splits = M > 0 ? row_splits(M, V, wide) : 1;
    return splits <= 1 ? 0 : kCounterBytes + (size_t)(M * splits * row_part_bytes(top));
}

hipError_t launch_logprobs(const TokenLogprobs& a, hipStream_t s)
{
    LogprobArgs p{};
    p.logits = a.logits; p.stride = a.stride;
    p.tokens = a.tokens; p.logprob = a.logprob; p.entropy = a.entropy; p.rank = a.rank;
    p.top_ids = a.top_ids; p.top_logprobs = a.top_logprobs;
    p.counters = static_cast<int*>(a.workspace);
    p.parts = a.workspace ? static_cast<char*>(a.workspace) + kCounterBytes : nullptr;
    p.V = (int)a.V; p.top = (int)a.top; p.part_bytes = (int)row_part_bytes(a.top);
    const int splits = a.workspace ? row_splits(a.M, a.V, a.wide) : 1;
    if (a.M * splits >= (int64_t)1 << 24) return hipErrorInvalidValue;           // 2^32 threads
    auto* kernel = a.wide ? (a.top ? logprobs_kernel<float, true> : logprobs_kernel<float, false>)
                          : (a.top ? logprobs_kernel<__half, true> : logprobs_kernel<__half, false>);
    kernel<<<dim3((unsigned)a.M, (unsigned)splits), kRowThreads, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace qoq
