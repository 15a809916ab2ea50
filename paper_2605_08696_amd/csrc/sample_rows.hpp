// One token for each row of logits, with that row's temperature, top-k, top-p, min-p and a random number given by the caller.
//
// With w_v = exp((l_v - max) / T), in the order of the logits from the largest down, equal ones by their index, the tokens that may be
// drawn are a prefix: at most top_k of them, none with w < min_p, and of these the shortest prefix whose weights reach top_p of theirs.
// The token is the first one, by index, whose running sum of weights over the kept tokens exceeds u times their sum.
//
// A sum that is rounded differently chooses another token where it passes near a border, so weights are formed in 64 bits and held as
// whole numbers of 2^-43: their sums are exact and do not depend on their order.  (V <= 2^20 of them fit 64 bits.)
#pragma once
#include "fp8.hpp"

typedef unsigned long long sr_mass;
constexpr int kSampleThreads = 1024, kSampleVocab = 1 << 20;
constexpr double kSampleUnit = 8796093022208.0;      // 2^43

struct SampleRows {
    int64_t ld;
    int V;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *tok;
    float *logprob;
};

// Unsigned integers ordered as the floats are; -0 and +0 share a key, a NaN has that of -infinity.
__device__ __forceinline__ uint32_t sample_key(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

template <int NW>
__device__ __forceinline__ sr_mass sample_sum(sr_mass v, sr_mass *red)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v += __shfl_xor(v, off, kWave);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    sr_mass t = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) t += red[i];
    __syncthreads();
    return t;
}

// One work-group per row; every search is a bisection with a pass over the row for each step.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads)
sample_rows_kernel(const T *__restrict__ logits, SampleRows p)
{
    constexpr int NT = kSampleThreads, NW = NT / 64;
    __shared__ sr_mass red[NW];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, V = p.V;
    const T *L = logits + row * p.ld;
    auto value = [&](int v) {
        const float x = (float)L[v];
        return x == x ? x : -INFINITY;
    };
    uint32_t top = 0;
    for (int v = tid; v < V; v += NT) top = max(top, sample_key(value(v)));
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, off, kWave));
    if ((tid & 63) == 0) red[tid >> 6] = top;
    __syncthreads();
    for (int i = 0; i < NW; ++i) top = max(top, (uint32_t)red[i]);
    __syncthreads();
    const float most = __uint_as_float((top & 0x80000000u) ? top & 0x7fffffffu : ~top);
    if (most == -INFINITY) {
        if (tid == 0) {
            p.tok[row] = -1;
            if (p.logprob) p.logprob[row] = -INFINITY;
        }
        return;
    }
    const float t = p.temperature ? p.temperature[row] : 1.0f;
    const bool greedy = !(t > 0.0f);
    const double inv = 1.0 / (double)t;
    const float mp = p.min_p ? p.min_p[row] : 0.0f;
    const double least = greedy ? 1.0 : mp > 0.0f ? fmin((double)mp, 1.0) : 0.0;
    auto mass = [&](float x) -> sr_mass {
        if (x == most) return (sr_mass)kSampleUnit;
        if (x == -INFINITY || greedy) return 0;
        const double w = exp(((double)x - (double)most) * inv);
        return w >= least ? (sr_mass)(w * kSampleUnit + 0.5) : 0;
    };
    // tokens of key >= from: their number and mass
    auto above = [&](uint32_t from, sr_mass &count, sr_mass &sum) {
        sr_mass c = 0, m = 0;
        for (int v = tid; v < V; v += NT) {
            const float x = value(v);
            const sr_mass w = mass(x);
            if (sample_key(x) >= from && w) { ++c; m += w; }
        }
        count = sample_sum<NW>(c, red);
        sum = sample_sum<NW>(m, red);
    };
    sr_mass count, sum;
    above(0, count, sum);
    // the cut: all tokens of larger keys, and of those with this key the first `ties`
    uint32_t cut = 0;
    sr_mass ties = ~0ull;
    auto shorten = [&](sr_mass most_count, sr_mass target) {
        uint32_t lo = 0, hi = top;                   // the limit is reached by {key >= lo}, or nowhere; the largest such key
        while (lo < hi) {
            const uint32_t mid = lo + ((hi - lo) >> 1) + 1;
            sr_mass c, m;
            above(mid, c, m);
            if (c >= most_count || m >= target) lo = mid; else hi = mid - 1;
        }
        sr_mass c, m, c1 = 0, m1 = 0;
        above(lo, c, m);
        if (lo < top) above(lo + 1, c1, m1);
        if (c == c1) return;
        const sr_mass one = (m - m1) / (c - c1);
        sr_mass n = min(c - c1, most_count - c1);
        if (target > m1) n = min(n, (target - m1 + one - 1) / one);
        if (lo > cut) { cut = lo; ties = n; }
        else if (lo == cut) ties = min(ties, n);
        sum = m1 + n * one;
    };
    const int k = greedy ? 1 : p.top_k ? p.top_k[row] : 0;
    if (k > 0 && (sr_mass)k < count) shorten((sr_mass)k, 1ull << 63);
    const float tp = p.top_p ? p.top_p[row] : 1.0f;
    if (tp < 1.0f && !greedy) {
        const sr_mass target = (sr_mass)ceil((double)fmaxf(tp, 0.0f) * (double)sum);
        shorten(~0ull, max(target, (sr_mass)1));
    }
    // the draw: bisection over the index for the first whose running sum exceeds the target
    const float u = p.uniform[row];
    const sr_mass target = min((sr_mass)((double)(u > 0.0f ? u : 0.0f) * (double)sum), sum - 1);
    auto upto = [&](int end) {                       // the kept mass of indices < end
        sr_mass m = 0, c = 0;
        for (int v = tid; v < end; v += NT) {
            const float x = value(v);
            const uint32_t key = sample_key(x);
            if (key > cut) m += mass(x);
            else if (key == cut && mass(x)) ++c;
        }
        m = sample_sum<NW>(m, red);
        c = sample_sum<NW>(c, red);
        const sr_mass one = mass(__uint_as_float((cut & 0x80000000u) ? cut & 0x7fffffffu : ~cut));
        return m + min(c, ties) * one;
    };
    int lo = 0, hi = V - 1;                          // upto(lo + 1) > target at the end
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (upto(mid + 1) > target) hi = mid; else lo = mid + 1;
    }
    if (tid == 0) {
        p.tok[row] = lo;
        if (p.logprob) {
            const float x = value(lo);
            const double lw = x == most ? 0.0 : ((double)x - (double)most) * inv;
            p.logprob[row] = greedy ? 0.0f : (float)(lw - log((double)sum / kSampleUnit));
        }
    }
}
