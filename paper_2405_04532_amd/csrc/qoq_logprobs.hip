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
//
// Many rows are bound by memory, a workgroup to each: 4001 of 32000 FP16 46 us without alternatives, 5.5 TB/s, 54 with the largest where the same logits
// are read again and again, 58.7 where each pass has others (the vector unit is active for nearly all of that).  Few rows are shared by workgroups
// whose parts a second launch joins, and are bound by the chain of steps: one of 32000 with 5 alternatives 11.5 us, 64 of 128256 with 20 17.3.
#include <hip/hip_fp16.h>

#include <algorithm>

#include "qoq_gemm_common.h"
#include "qoq_internal.h"

namespace qoq {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kInTurn = 4;                       // vectors of a lane in flight
constexpr int kMaxRowSplits = 64;                // workgroups to a row: the lanes of a wave
constexpr int kFound = 2048;                     // candidates that are ranked at once: all that a join can have
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
    char* parts;                                 // of each row and workgroup: its sums, then its first `top` (value, index)
    int V, top, part_bytes, splits;
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
    // unsigned numbers in the order of the logits (no NaN, one zero)
    static constexpr int kKeyBits = 16;
    static __device__ __forceinline__ uint32_t key(float v)
    {
        const uint32_t u = __half_as_ushort(__float2half_rn(v + 0.f));
        return (u ^ (u & 0x8000u ? 0xFFFFu : 0x8000u)) & 0xFFFFu;
    }
    static __device__ __forceinline__ float of_key(uint32_t k)       // (below that of minus infinity: that)
    {
        k = k < 0x03FFu ? 0x03FFu : k;
        return (float)__builtin_bit_cast(_Float16, (unsigned short)(k & 0x8000u ? k ^ 0x8000u : ~k));
    }
    // ln sum e^x: ln T, without the part by which log2(e) is off, which is as good as proportional to the mean of x
    static __device__ double lse(const Sums& s, double mean_t, double ln) { return ln + s.r * kLn2 - kLog2eOff / kLog2e * (mean_t + s.r); }
    static __device__ double logprob(float x, float, double lse) { return (double)x - lse; }
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
    static constexpr int kKeyBits = 32;
    static __device__ __forceinline__ uint32_t key(float v)
    {
        const uint32_t u = __float_as_uint(v + 0.f);
        return u ^ ((uint32_t)((int)u >> 31) | 0x80000000u);
    }
    static __device__ __forceinline__ float of_key(uint32_t k)
    {
        k = k < 0x007FFFFFu ? 0x007FFFFFu : k;
        return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
    }
    static __device__ double lse(const Sums&, double mean_t, double ln) { return ln - kLog2eOff / kLog2e * mean_t; }      // of x - r
    static __device__ double logprob(float x, float r, double lse) { return ((double)x - (double)r) - lse; }
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

// A (value, index) at or in front of which there are n of the 64 J (key, index) that a wave's lanes hold, and at most `most`, unless there are
// no more at all (key 0: none).  The key's bits are settled from the highest one down, by ballots, then where more than that
// are equal the index's, until few enough are left.
template <class T, int J>
__device__ __forceinline__ void threshold(const uint32_t (&key)[J], const int (&index)[J], int n, int most, float& tau_v, int& tau_i)
{
    unsigned long long alive[J], part[J];
    int left = 0, in_front = 0, need = n;                            // lanes that are not settled, those in front of them
#pragma unroll
    for (int j = 0; j < J; ++j) {
        alive[j] = __builtin_amdgcn_ballot_w64(key[j] != 0);
        left += __builtin_popcountll(alive[j]);
    }
    tau_v = -__builtin_inff();
    tau_i = 0x7FFFFFFF;
    if (left < n) return;
    // goes on with those of a part if they are enough, else with the others behind them
    auto settle = [&]() __attribute__((always_inline)) {
        int c = 0;
#pragma unroll
        for (int j = 0; j < J; ++j) c += __builtin_popcountll(part[j]);
        const bool enough = c >= need;
#pragma unroll
        for (int j = 0; j < J; ++j) alive[j] = enough ? part[j] : alive[j] & ~part[j];
        left = enough ? c : left - c;
        need -= enough ? 0 : c;
        in_front += enough ? 0 : c;
        return enough;
    };
    uint32_t prefix = 0;
#pragma unroll 1
    for (uint32_t bit = 1u << (Logit<T>::kKeyBits - 1); bit && in_front + left > most; bit >>= 1) {
#pragma unroll
        for (int j = 0; j < J; ++j) part[j] = __builtin_amdgcn_ballot_w64((key[j] & bit) != 0) & alive[j];
        if (settle()) prefix |= bit;
    }
    tau_v = Logit<T>::of_key(prefix);
    if (in_front + left <= most) return;
    tau_i = 0;
#pragma unroll 1
    for (int bit = 1 << 24; bit; bit >>= 1) {
#pragma unroll
        for (int j = 0; j < J; ++j) part[j] = __builtin_amdgcn_ballot_w64((index[j] & bit) == 0) & alive[j];
        if (!settle()) tau_i |= bit;
        if (in_front + left <= most) {
            tau_i |= bit - 1;
            break;
        }
    }
}

struct Shared {
    Sums sums[kRowWaves];
    int lanes, found, whole;
    double lse;
    float row_r;
    uint32_t best_key[kRowThreads];                                  // of each lane's largest element, and where it lies at the latest
    int latest[kRowThreads];
    int lane[kRowThreads];                                           // lanes that may hold one of the first n
    float2 wave_best[kRowWaves];
    float2 item[kFound];                                             // value, index
};

__device__ __forceinline__ void append(Shared& sh, float x, int i)
{
    const int place = atomicAdd(&sh.found, 1);
    if (place < kFound) sh.item[place] = make_float2(x, __int_as_float(i));
}

// the found items ranked: put(place, value, index) for the first n places, an index of -1 where there is nothing
template <class Put>
__device__ __forceinline__ void put_ranked(const Shared& sh, int found, int n, Put put)
{
    // as many lanes to an item as there are threads for
    int shift = 0;
    while (shift < 4 && found << (shift + 1) <= kRowThreads) ++shift;
    const int group = 1 << shift, part = threadIdx.x & (group - 1);
#pragma unroll 1
    for (int c0 = 0; c0 < max(found, n); c0 += kRowThreads >> shift) {
        const int c = c0 + (threadIdx.x >> shift);
        float2 me = make_float2(-__builtin_inff(), __int_as_float(-1));
        int place = c;                                               // (what was not found stands behind the others)
        if (c < found) {
            me = sh.item[c];
            place = 0;
#pragma unroll 4
            for (int o = part; o < found; o += group) {
                const float2 other = sh.item[o];
                place += in_front(other.x, __float_as_int(other.y), me.x, __float_as_int(me.y));
            }
#pragma unroll 1
            for (int o = group >> 1; o; o >>= 1) place += __shfl_xor(place, o, 64);          // (a group's lanes share c)
        }
        if (part == 0 && place < n) put(place, me.x, __float_as_int(me.y));
    }
}

// ln T = k ln 2 + 2 artanh((m - 1) / (m + 1)), T = 2^k m with m in 0.70 .. 1.42: the series to the thirteenth power is good to 5e-13
__device__ __forceinline__ double ln_of(float T)
{
    const uint32_t u = __float_as_uint(T);
    const int k = (int)(u - 0x3F350000u) >> 23;
    const double m = (double)__uint_as_float(u - ((uint32_t)k << 23)), s = (m - 1.0) / (m + 1.0), q = s * s;
    double y = 1.0 / 13;
#pragma unroll
    for (int i = 11; i > 0; i -= 2) y = fma(y, q, 1.0 / i);
    return fma((double)k, kLn2, 2.0 * s * y);
}

// The results of a row, by one wave; they are read behind the next barrier.
template <class T>
__device__ __forceinline__ void finish_row(const LogprobArgs& p, Shared& sh, int row, const Sums& sum, bool is_token, float xt)
{
    using L = Logit<T>;
    const bool whole = sum.T > 0x1p-126f && sum.T < __builtin_inff();        // not: the row holds NaN, plus infinity or nothing
    const double mean = (double)(sum.U / sum.T), ln = ln_of(sum.T), lse = L::lse(sum, mean, ln);
    if ((threadIdx.x & 63) == 0) {
        const float nan = __builtin_nanf("");
        if (p.logprob) p.logprob[row] = is_token && whole ? (float)L::logprob(xt, sum.r, lse) : nan;
        if (p.rank) p.rank[row] = is_token && whole ? sum.count + 1 : 0;
        if (p.entropy) p.entropy[row] = whole ? fmaxf((float)(ln - kLn2 * mean), 0.f) : nan;
        sh.lse = lse;
        sh.row_r = sum.r;
        sh.whole = whole;
    }
}
template <class T>
__device__ __forceinline__ void put_result(const LogprobArgs& p, const Shared& sh, int row, int place, float value, int index)
{
    p.top_ids[(int64_t)row * p.top + place] = sh.whole ? index : -1;
    p.top_logprobs[(int64_t)row * p.top + place] = sh.whole ? (float)Logit<T>::logprob(value, sh.row_r, sh.lse) : __builtin_nanf("");
}

// ALONE: a workgroup to a row, which ends with the results; else its part goes to the join below.
template <class T, bool TOP, bool ALONE>
__global__ __launch_bounds__(kRowThreads) void logprobs_kernel(LogprobArgs p)
{
    using L = Logit<T>;
    constexpr int N = L::kVec;
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x, split = ALONE ? 0 : blockIdx.y, splits = ALONE ? 1 : p.splits, V = p.V, n = p.top;
    const T* x_row = static_cast<const T*>(p.logits) + (int64_t)row * p.stride;
    // vectors of 16 aligned bytes: the whole ones are dealt to the row's workgroups, the elements in front of them and behind are the first one's
    const int before = (int)(((uintptr_t)x_row & 15) / sizeof(T));
    const uint4* vectors = reinterpret_cast<const uint4*>(x_row - before);
    const int whole0 = before ? 1 : 0, whole1 = max((int)(((int64_t)before + V) / N), whole0);
    const int share = (whole1 - whole0 + splits - 1) / splits;
    const int v0 = whole0 + split * share, v1 = min(whole1, v0 + share);
    const int front = min(whole0 * N - before, V), tail = max(whole1 * N - before, front);     // elements 0 .. front - 1 and tail .. V - 1

    const int token = p.tokens ? p.tokens[row] : -1;
    const bool is_token = token >= 0 && token < V;
    const float xt = is_token ? (float)x_row[token] + 0.f : __builtin_inff();
    const int token_vector = is_token ? (token + before) / N : 0;
    // x > xt as x >= the next number
    const uint32_t xb = __float_as_uint(xt);
    const float xt_next = is_token ? __uint_as_float(xt >= 0.f ? xb + 1 : xb - 1) : __builtin_inff();

    // The sums of up to eight turns, to which each vector's own are added; in FP32 those of 64 times as many before, and in FP64 those before them.  Terms
    // alike are rounded to the same side, and a lane of a row of 2^24 has 65536 (logits 2.7 above the first ones, off by 7e-7; one sum in FP32 4e-4, and of a
    // row of 2^20 2e-5.  4001 rows of 32000 54.2 us, with one sum 53.5, with FP64 for each turn 55.7).
    Sums s = {L::kLowest, 0.f, 0.f, 0}, past = s;
    double far_T = 0.0, far_U = 0.0;                                  // against past's reference
    int turn = 0;
    auto keep = [&](float r) __attribute__((always_inline)) {         // past's reference becomes r
        if (turn > 512) {
            const float d = fmaxf(L::step(past.r, r), -1e30f), f = __builtin_amdgcn_exp2f(d);
            far_U = f * fma(far_T, (double)d, far_U);
            far_T *= f;
        }
        past = rebased<T>(past, r);
        past.T += s.T;
        past.U += s.U;
    };
    int count = 0;                                                    // of the wave
    float end_x = -__builtin_inff();
    int end_i = -1;
    if (split == 0 && wave == 0) {                                    // the elements at the ends, one to a lane
        const int i = lane < front ? lane : tail + lane - front;
        if (i < V) {
            end_i = i;
            end_x = (float)x_row[i];
            s.r = fmaxf(s.r, L::unit(end_x));
            const float t = L::term(end_x, s.r);
            s.T = __builtin_amdgcn_exp2f(t);
            s.U = s.T * fmaxf(t, -1e4f);
        }
        count = __builtin_popcountll(__builtin_amdgcn_ballot_w64(is_token && end_i >= 0 && (end_x > xt || (end_x == xt && i < token))));
    }
    float best = -__builtin_inff();
    int best_vector = v0 + tid < v1 ? v0 + tid : -1;
    // (the loop is the same code for whole turns and for the last: a call on few rows runs through its code once, and pays for fetching it)
#pragma unroll 1
    for (int v = v0 + tid; __builtin_amdgcn_ballot_w64(v < v1) != 0; v += kInTurn * kRowThreads) {
        uint4 w[kInTurn];
#pragma unroll
        for (int k = 0; k < kInTurn; ++k) w[k] = vectors[min(v + k * kRowThreads, v1 - 1)];
#pragma unroll
        for (int k = 0; k < kInTurn; ++k) {
            const int at = v + k * kRowThreads;
            const bool real = at < v1;
            if (!real) w[k] = make_uint4(L::kNone, L::kNone, L::kNone, L::kNone);
            float x[N];
            L::take(w[k], x);
            float most = fmaxf(x[0], x[1]);
#pragma unroll
            for (int e = 2; e < N; ++e) most = fmaxf(most, x[e]);
            if (TOP && most > best) { best = most; best_vector = at; }
            const float unit = L::unit(most);
            if (__builtin_amdgcn_ballot_w64(unit > s.r + kSlack) != 0)
                if (unit > s.r + kSlack) s = rebased<T>(s, unit);
            const float from = !real ? __builtin_inff() : at < token_vector ? xt : xt_next;
            float sum_T = 0.f, sum_U = 0.f;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const float t = L::term(x[e], s.r), q = __builtin_amdgcn_exp2f(t), by = fmaxf(t, -1e4f);      // (minus infinity: 0 times a finite number)
                sum_T = e ? sum_T + q : q;
                sum_U = e ? fmaf(q, by, sum_U) : q * by;
            }
            s.T += sum_T;
            s.U += sum_U;
            // (a token that was drawn is mostly among the largest, and few vectors hold one in front of it: 1024 rows of 128256 57.5 us, 54.6 so)
            if (__builtin_amdgcn_ballot_w64(most >= from) != 0)
#pragma unroll
                for (int e = 0; e < N; ++e) count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(x[e] >= from));
            if (__builtin_amdgcn_ballot_w64(real && at == token_vector) != 0)         // equal ones in front of the token in its vector
#pragma unroll
                for (int e = 0; e < N - 1; ++e)
                    count += __builtin_popcountll(__builtin_amdgcn_ballot_w64(real && at == token_vector && x[e] == xt && e < token + before - token_vector * N));
        }
        if ((++turn & 7) == 0) {
            keep(s.r);
            s.T = s.U = 0.f;
            if ((turn & 511) == 0) {
                far_T += past.T;
                far_U += past.U;
                past.T = past.U = 0.f;
            }
        }
    }
    if (turn >= 8) {
        keep(s.r);
        s.T = turn < 512 ? past.T : (float)(far_T + past.T);
        s.U = turn < 512 ? past.U : (float)(far_U + past.U);
    }

    Sums of_wave = all_lanes<T>(s);
    of_wave.count = count;
    if (lane == 0) sh.sums[wave] = of_wave;
    if constexpr (TOP) {
        if (tid == 0) sh.lanes = sh.found = 0;
        sh.best_key[tid] = best_vector >= 0 ? L::key(best) : 0;
        sh.latest[tid] = min(best_vector * N - before + N - 1, V - 1);
    }
    __syncthreads();
    char* mine = p.parts + ((int64_t)row * splits + split) * p.part_bytes;
    if (wave == kRowWaves - 1) {
        Sums of_lane = sh.sums[min(lane, kRowWaves - 1)];
        if (lane >= kRowWaves) of_lane = {L::kLowest, 0.f, 0.f, 0};
        const Sums sum = all_lanes<T>(of_lane);
        if constexpr (ALONE) finish_row<T>(p, sh, row, sum, is_token, xt);
        else if (lane == 0) *reinterpret_cast<float4*>(mine) = make_float4(sum.r, sum.T, sum.U, __int_as_float(sum.count));
    }
    if constexpr (TOP) {
        float tau_v;
        int tau_i;
        uint32_t key[kRowWaves];
        int at_latest[kRowWaves];
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) {
            key[w] = sh.best_key[w * 64 + lane];
            at_latest[w] = sh.latest[w * 64 + lane];
        }
        threshold<T, kRowWaves>(key, at_latest, n, n + n / 2 + 4, tau_v, tau_i);
        if (best_vector >= 0 && (best > tau_v || (best == tau_v && best_vector * N - before <= tau_i))) sh.lane[atomicAdd(&sh.lanes, 1)] = tid;
        __syncthreads();
        const int lanes = sh.lanes;
        auto counts = [&](float x, int i) { return x > tau_v || (x == tau_v && i <= tau_i); };
        const int steps = (share + kRowThreads - 1) / kRowThreads, bits = steps > 1 ? 32 - __builtin_clz(steps - 1) : 0, items = lanes << bits;
#pragma unroll 1
        for (int c = tid; c < items; c += kRowThreads) {
            const int q = c >> bits, at = v0 + sh.lane[q] + (c & ((1 << bits) - 1)) * kRowThreads;
            if (at >= v1) continue;
            float x[N];
            L::take(vectors[at], x);
            uint32_t hits = 0;
#pragma unroll
            for (int e = 0; e < N; ++e) hits |= counts(x[e], at * N - before + e) ? 1u << e : 0;
            while (hits) {
                const int e = __builtin_ctz(hits);
                hits &= hits - 1;
                float y = x[0];
#pragma unroll
                for (int k = 1; k < N; ++k) y = e == k ? x[k] : y;
                append(sh, y, at * N - before + e);
            }
        }
        if (end_i >= 0 && counts(end_x, end_i)) append(sh, end_x, end_i);
        __syncthreads();
        auto put = [&](int place, float value, int index) __attribute__((always_inline)) {
            if constexpr (ALONE) put_result<T>(p, sh, row, place, value, index);
            else *(reinterpret_cast<float2*>(mine + 16) + place) = make_float2(value, __int_as_float(index));
        };
        const int found = sh.found;
        if (found <= kFound) {
            put_ranked(sh, found, n, put);
        } else {
            // More than can be ranked, as where large elements lie a workgroup's stride apart: one after the other, the row read for each.
            float last_v = __builtin_inff();
            int last_i = -1;
#pragma unroll 1
            for (int k = 0; k < n; ++k) {
                float bv = -__builtin_inff();
                int bi = 0x7FFFFFFF;
                auto look = [&](float x, int i) __attribute__((always_inline)) {
                    if (in_front(last_v, last_i, x, i) && in_front(x, i, bv, bi)) { bv = x; bi = i; }
                };
#pragma unroll 1
                for (int at = v0 + tid; at < v1; at += kRowThreads) {
                    float x[N];
                    L::take(vectors[at], x);
#pragma unroll
                    for (int e = 0; e < N; ++e) look(x[e], at * N - before + e);
                }
                if (end_i >= 0) look(end_x, end_i);
#pragma unroll 1
                for (int o = 32; o; o >>= 1) {
                    const float ov = __shfl_xor(bv, o, 64);
                    const int oi = __shfl_xor(bi, o, 64);
                    if (in_front(ov, oi, bv, bi)) { bv = ov; bi = oi; }
                }
                __syncthreads();
                if (lane == 0) sh.wave_best[wave] = make_float2(bv, __int_as_float(bi));
                __syncthreads();
                last_v = bv;
                last_i = bi;
                for (int w = 0; w < kRowWaves; ++w) {
                    const float2 o = sh.wave_best[w];
                    if (in_front(o.x, __float_as_int(o.y), last_v, last_i)) { last_v = o.x; last_i = __float_as_int(o.y); }
                }
                if (tid == 0) put(k, last_v, last_i);
            }
        }
    }
}

// The parts of a row: a lane to a workgroup's sums, then the first n of their lists, which are in order.
template <class T, bool TOP>
__global__ __launch_bounds__(kRowThreads) void logprobs_join_kernel(LogprobArgs p)
{
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int row = blockIdx.x, splits = p.splits, n = p.top;
    const char* parts = p.parts + (int64_t)row * splits * p.part_bytes;
    auto item = [&](int split, int k) { return *(reinterpret_cast<const float2*>(parts + (int64_t)split * p.part_bytes + 16) + k); };
    if constexpr (TOP) {
        // 64 of the foremost of all lists: as many of each as there are lanes for, which come to n at least
        const int each = min(64 / splits, n), k = lane / splits;
        const float2 head = item(lane - k * splits, min(k, each - 1));
        float tau_v;
        int tau_i;
        const uint32_t key[1] = {k < each && __float_as_int(head.y) >= 0 ? Logit<T>::key(head.x) : 0};
        const int index[1] = {__float_as_int(head.y)};
        threshold<T, 1>(key, index, n, n, tau_v, tau_i);      // (exactly: behind each of these stands the rest of its list)
        if (tid == 0) sh.found = 0;
        __syncthreads();
#pragma unroll 1
        for (int c = tid; c < splits * n; c += kRowThreads) {
            const int of = c / n;
            const float2 it = item(of, c - of * n);
            const int i = __float_as_int(it.y);
            if (i >= 0 && (it.x > tau_v || (it.x == tau_v && i <= tau_i))) append(sh, it.x, i);
        }
    }
    if (wave == kRowWaves - 1 || !TOP) {
        const float4 part = *reinterpret_cast<const float4*>(parts + (int64_t)min(lane, splits - 1) * p.part_bytes);
        const int token = p.tokens ? p.tokens[row] : -1;
        const bool is_token = token >= 0 && token < p.V;
        const float xt = is_token ? (float)(static_cast<const T*>(p.logits) + (int64_t)row * p.stride)[token] + 0.f : 0.f;
        Sums s = {part.x, part.y, part.z, __float_as_int(part.w)};
        if (lane >= splits) s = {Logit<T>::kLowest, 0.f, 0.f, 0};
        finish_row<T>(p, sh, row, all_lanes<T>(s), is_token, xt);
    }
    if constexpr (TOP) {
        __syncthreads();
        put_ranked(sh, sh.found, n, [&](int place, float value, int index) { put_result<T>(p, sh, row, place, value, index); });
    }
}

// Workgroups to a row: as few as bring the work of a compute unit down to the least there is, with at most 1024 in all and two turns of their lanes each
// (at least two on a compute unit, so that is counted for one).  64 rows of 128256 with 20 alternatives 16.3 us with 8, 18.7 with 7 or 12 (three on
// some compute units), 17.0 with 16; 200 rows 27.1 with 5, 31 with 2 or 3; 512 of 32000 16.7 with one, 21.2 with two; one of 128256 14.1 with 31, 15.7 with 62.
int row_splits(int64_t M, int64_t V, int wide)
{
    const int64_t vectors = (V + (wide ? 3 : 7)) / (wide ? 4 : 8);
    const int64_t most = M > 0 ? std::min<int64_t>({kMaxRowSplits, 1024 / M, vectors / (2 * kRowThreads)}) : 1;
    int64_t best = 1;
    auto rounds = [&](int64_t s) { return std::max<int64_t>(2, (M * s + 255) / 256); };
    for (int64_t s = 2; s <= most; ++s)
        if (rounds(s) * best < rounds(best) * s) best = s;
    return (int)best;
}
int64_t row_part_bytes(int64_t top) { return (16 + 8 * top + 15) / 16 * 16; }

}  // namespace

size_t logprobs_workspace_bytes(int64_t M, int64_t V, int64_t top, int wide)
{
    const int splits = M > 0 ? row_splits(M, V, wide) : 1;
    return splits <= 1 ? 0 : (size_t)(M * splits * row_part_bytes(top));
}

hipError_t launch_logprobs(const TokenLogprobs& a, hipStream_t s)
{
    LogprobArgs p{};
    p.logits = a.logits; p.stride = a.stride;
    p.tokens = a.tokens; p.logprob = a.logprob; p.entropy = a.entropy; p.rank = a.rank;
    p.top_ids = a.top_ids; p.top_logprobs = a.top_logprobs;
    p.parts = static_cast<char*>(a.workspace);
    p.V = (int)a.V; p.top = (int)a.top; p.part_bytes = (int)row_part_bytes(a.top);
    p.splits = a.workspace ? row_splits(a.M, a.V, a.wide) : 1;
    if (a.M * p.splits >= (int64_t)1 << 24) return hipErrorInvalidValue;           // 2^32 threads
    const dim3 grid((unsigned)a.M, (unsigned)p.splits);
    if (p.splits == 1) {
        auto* kernel = a.wide ? (a.top ? logprobs_kernel<float, true, true> : logprobs_kernel<float, false, true>)
                              : (a.top ? logprobs_kernel<__half, true, true> : logprobs_kernel<__half, false, true>);
        kernel<<<grid, kRowThreads, 0, s>>>(p);
        return hipGetLastError();
    }
    auto* kernel = a.wide ? (a.top ? logprobs_kernel<float, true, false> : logprobs_kernel<float, false, false>)
                          : (a.top ? logprobs_kernel<__half, true, false> : logprobs_kernel<__half, false, false>);
    kernel<<<grid, kRowThreads, 0, s>>>(p);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    auto* join = a.wide ? (a.top ? logprobs_join_kernel<float, true> : logprobs_join_kernel<float, false>)
                        : (a.top ? logprobs_join_kernel<__half, true> : logprobs_join_kernel<__half, false>);
    join<<<(unsigned)a.M, a.top ? kRowThreads : 64, 0, s>>>(p);
    return hipGetLastError();
}

}  // namespace qoq
