// One token for each row of logits, with that row's temperature, top-k, top-p, min-p and a random number given by the caller.
//
// With w_v = exp((l_v - max) / T), in the order of the logits from the largest down, equal ones by their index, the tokens that may be
// drawn are a prefix: at most top_k of them, none with w < min_p, and of these the shortest prefix whose weights reach top_p of theirs.
// The token is the first one, by index, whose running sum of weights over the kept tokens exceeds u times their sum.
//
// A sum that is rounded differently chooses another token where it passes near a border, so weights are formed in 64 bits (fp64
// instructions issue as fast as fp32 ones here) and held as whole numbers of 2^-43 of the largest: their sums are exact and do not
// depend on their order, LDS atomics included.  (V <= 2^20 of them fit 64 bits.)  Tokens whose weight rounds to zero are never drawn and
// may be left out of every list: they come last in the order.
//
// A work-group of 1024 threads takes a row; a thread reads eight consecutive logits, a wavefront 512, a segment.  Passes over the row:
//   the largest logit;
//   for top-k a histogram of counts, for top-p one of weights, over 1024 equal steps of logit value; the step in which the limit is
//   reached is divided again by key until it holds a few members, which are compared with each other (or one value: its first ones);
//   sums of the kept weights by segment, one of which holds the token.
// Later passes evaluate only vectors that hold a logit at or above the smallest that may still be drawn.
#pragma once
#include "fp8.hpp"

typedef unsigned long long sr_mass;
constexpr int kSampleThreads = 1024, kSampleVocab = 1 << 20, kSampleSegment = 512, kSampleSteps = 1024, kSampleMembers = 256;
constexpr double kSampleUnit = 8796093022208.0;      // 2^43

struct SampleRows {
    int64_t ld;
    int V;
    const float *temperature, *top_p, *min_p, *uniform;
    const int32_t *top_k;
    int32_t *tok;
    float *logprob;
};

// Unsigned integers ordered as the floats are; -0 and +0 share a key.
__device__ __forceinline__ uint32_t sample_key(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float sample_value(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key); }

// round(2^43 2^y) for y <= 0, 0 for y <= -44 and for a NaN.  2^f on [-1/2, 1/2] by the polynomial that interpolates it at Chebyshev's
// points, of degree 10 (below 1e-15 of the value), its constant term 1 so that y = 0 gives the unit.
__device__ __forceinline__ sr_mass sample_mass(double y)
{
    y = __builtin_fmax(y, -44.0);
    const double magic = 6755399441055744.0;         // 1.5 2^52: its sum with y holds y's nearest integer in the low bits
    const double t = y + magic;
    const double f = y - (t - magic);
    double p = 7.070977866508138e-09;
    p = __builtin_fma(p, f, 1.0205905413765595e-07);
    p = __builtin_fma(p, f, 1.3215451633221434e-06);
    p = __builtin_fma(p, f, 1.5252672924850737e-05);
    p = __builtin_fma(p, f, 0.00015403530424776529);
    p = __builtin_fma(p, f, 0.0013333558200794592);
    p = __builtin_fma(p, f, 0.009618129107618665);
    p = __builtin_fma(p, f, 0.05550410866465167);
    p = __builtin_fma(p, f, 0.24022650695910075);
    p = __builtin_fma(p, f, 0.6931471805599462);
    p = __builtin_fma(p, f, 1.0);
    // p 2^(43 + n), then its nearest integer in the mantissa of 2^52 + it
    const int n = (int)(uint32_t)__builtin_bit_cast(unsigned long long, t);
    const unsigned long long bits = __builtin_bit_cast(unsigned long long, p) + ((unsigned long long)(unsigned)(n + 43) << 52);
    return __builtin_bit_cast(unsigned long long, __builtin_bit_cast(double, bits) + 4503599627370496.0) & 0xFFFFFFFFFFFFFull;
}

template <typename T>
__global__ void __launch_bounds__(kSampleThreads)
sample_rows_kernel(const T *__restrict__ logits, SampleRows p)
{
    constexpr int NT = kSampleThreads, NW = NT / 64, PER = kSampleVocab / kSampleSegment / NT;
    __shared__ sr_mass red[NW];
    __shared__ sr_mass mass_of[kSampleSteps];
    __shared__ uint32_t count_of[kSampleSteps];
    __shared__ sr_mass segment[PER * NT];
    __shared__ uint32_t member_key[kSampleMembers];
    __shared__ int member_at[kSampleMembers];
    __shared__ sr_mass member_mass[kSampleMembers];
    __shared__ sr_mass found_before;
    __shared__ uint32_t found, low_s, high_s, n_members;
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = p.V;
    const T *L = logits + row * p.ld;

    // fn(values, index of the first, how many exist); the next vector is on its way meanwhile
    auto pass = [&](auto &&fn) {
        int at = wave * kSampleSegment + lane * 8;
        float v[8];
        load8(L + at, V - at, v);
        while (at - lane * 8 < V) {                  // wave-uniform
            const int next = at + NW * kSampleSegment;
            float w[8];
            load8(L + next, V - next, w);
            fn(v, at, V - at);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = w[i];
            at = next;
        }
    };
    // exclusive prefix sum over the threads; total: of all
    auto scan = [&](sr_mass v, sr_mass &total) {
        sr_mass s = v;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const sr_mass o = __shfl_up(s, off, kWave);
            if (lane >= off) s += o;
        }
        __syncthreads();
        if (lane == 63) red[wave] = s;
        __syncthreads();
        sr_mass before = 0;
        total = 0;
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const sr_mass r = red[i];
            before += i < wave ? r : 0;
            total += r;
        }
        return before + s - v;
    };

    float most = -INFINITY;
    pass([&](const float (&v)[8], int, int n) {
#pragma unroll
        for (int i = 0; i < 8; ++i) most = fmaxf(most, i < n ? v[i] : -INFINITY);
    });
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) most = fmaxf(most, __shfl_xor(most, off, kWave));
    if (lane == 0) red[wave] = __float_as_uint(most);
    __syncthreads();
    for (int i = 0; i < NW; ++i) most = fmaxf(most, __uint_as_float((uint32_t)red[i]));
    if (most == -INFINITY) {                         // nothing to draw from
        if (tid == 0) {
            p.tok[row] = -1;
            if (p.logprob) p.logprob[row] = -INFINITY;
        }
        return;
    }

    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    const float top_p = p.top_p ? p.top_p[row] : 1.0f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    if (!(temp > 0.0f) || top_k == 1 || top_p <= 0.0f) {                // one token: the first of the largest
        int first = V;
        pass([&](const float (&v)[8], int at, int n) {
#pragma unroll
            for (int i = 7; i >= 0; --i)
                if (i < n && v[i] == most) first = min(first, at + i);
        });
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) first = min(first, __shfl_xor(first, off, kWave));
        __syncthreads();
        if (lane == 0) red[wave] = (sr_mass)first;
        __syncthreads();
        for (int i = 0; i < NW; ++i) first = min(first, (int)red[i]);
        if (tid == 0) {
            p.tok[row] = first;
            if (p.logprob) p.logprob[row] = 0.0f;
        }
        return;
    }

    // an infinite logit leaves all others without weight: the row is read as 0 where it is infinite and -infinity elsewhere
    const bool hot = most == INFINITY;
    if (hot) most = 0.0f;
    auto seen = [&](float x) { return hot ? (x == INFINITY ? 0.0f : -INFINITY) : x; };
    const double c = 1.4426950408889634 / (double)temp;
    const float min_p = p.min_p && p.min_p[row] > 0.0f ? fminf(p.min_p[row], 1.0f) : 0.0f;
    const sr_mass least = max((sr_mass)1, min_p > 0.0f ? (sr_mass)ceil((double)min_p * kSampleUnit) : (sr_mass)0);
    auto mass = [&](float x) {
        const sr_mass m = sample_mass(((double)x - (double)most) * c);
        return m >= least ? m : 0;
    };
    // The smallest logit that may be drawn: below `floor_v` nothing has weight (a little too low: weights decide); of value
    // `cut_v` only indices up to cut_at are kept.
    double lowest = (double)most + (fmax(-44.0, log2((double)least / kSampleUnit)) - 0.001) / c;
    float floor_v = (float)(lowest - fabs(lowest) * 1e-6);
    float cut_v = -INFINITY;
    int cut_at = V;
    auto kept = [&](float x, int at) { return x > cut_v || (x == cut_v && at <= cut_at); };
    // fn(value, index) for the logits that may still be kept
    auto each = [&](auto &&fn) {
        pass([&](const float (&v)[8], int at, int n) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, i < n ? seen(v[i]) : -INFINITY);
            if (__ballot(top >= floor_v) == 0) return;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = seen(v[i]);
                if (i < n && x >= floor_v && kept(x, at + i)) fn(x, at + i);
            }
        });
    };
    // The first index at which the running sum of weight(value, index) exceeds target(sum of all); the sum of all in `total`.
    auto index_of = [&](auto &&weight, auto &&target, sr_mass &total) {
        const int segments = (V + kSampleSegment - 1) / kSampleSegment;
        for (int i = tid; i < PER * NT; i += NT) segment[i] = 0;
        __syncthreads();
        pass([&](const float (&v)[8], int at, int n) {
            float top = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) top = fmaxf(top, i < n ? seen(v[i]) : -INFINITY);
            if (__ballot(top >= floor_v) == 0) return;
            sr_mass s = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = seen(v[i]);
                if (i < n && x >= floor_v) s += weight(x, at + i);
            }
#pragma unroll
            for (int off = 32; off >= 1; off >>= 1) s += __shfl_xor(s, off, kWave);
            if (lane == 0) segment[at / kSampleSegment] = s;
        });
        __syncthreads();
        sr_mass own = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) own += segment[tid * PER + i];
        sr_mass before = scan(own, total);
        const sr_mass t = target(total);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const sr_mass s = segment[tid * PER + i];
            if (t >= before && t - before < s) { found = tid * PER + i; found_before = before; }
            before += s;
        }
        __syncthreads();
        const int at = min((int)found, segments - 1) * kSampleSegment + lane * 8;
        if (wave == 0) {
            float v[8];
            load8(L + at, V - at, v);
            sr_mass w[8], s = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = seen(v[i]);
                w[i] = at + i < V && x >= floor_v ? weight(x, at + i) : 0;
                s += w[i];
            }
            sr_mass upto = s;
#pragma unroll
            for (int off = 1; off < 64; off <<= 1) {
                const sr_mass o = __shfl_up(upto, off, kWave);
                if (lane >= off) upto += o;
            }
            sr_mass run = found_before + upto - s;
            if (t >= run && t - run < s) {
                int k = 0;
#pragma unroll
                for (int i = 0; i < 7; ++i) {
                    run += w[i];
                    if (k == i && t >= run) k = i + 1;
                }
                found = at + k;
            }
        }
        __syncthreads();
        return (int)found;
    };

    // Cuts the kept tokens at the first one with which their number or their mass reaches a limit.
    auto cut = [&](bool by_mass, auto &&limit_of) {
        uint32_t key_low = 0, key_high = 0;          // of the step being divided, once it is one of keys
        int shift = -1;                              // -1: steps of value
        const float scale = (float)kSampleSteps / (most - floor_v);
        auto step_of = [&](float x) -> uint32_t {
            if (shift < 0) return (uint32_t)fminf((most - x) * scale, (float)(kSampleSteps - 1));
            return (key_high - sample_key(x)) >> shift;
        };
        sr_mass limit = 0, before = 0;
        uint32_t step = 0;
        int value_step = -1;
        auto inside = [&](float x) {                 // of the step being divided
            if (value_step < 0) return true;
            const uint32_t key = sample_key(x);
            return shift < 0 || (key >= key_low && key <= key_high);
        };
        for (int round = 0;; ++round) {
            __syncthreads();
            mass_of[tid] = 0;
            count_of[tid] = 0;
            if (tid == 0) { found = ~0u; n_members = 0; low_s = ~0u; high_s = 0; }
            __syncthreads();
            each([&](float x, int) {
                if (!inside(x)) return;
                const uint32_t s = step_of(x);
                if (by_mass) {
                    const sr_mass m = mass(x);
                    if (m == 0) return;
                    atomicAdd(&mass_of[s], m);
                }
                atomicAdd(&count_of[s], 1u);
            });
            __syncthreads();
            const sr_mass own = by_mass ? mass_of[tid] : count_of[tid];
            sr_mass total;
            const sr_mass up = before + scan(own, total);
            if (round == 0) {
                limit = limit_of(total);
                if (limit > total) return;           // never reached
            }
            if (up < limit && limit - up <= own) { found = tid; found_before = up; }
            __syncthreads();
            step = found;
            before = found_before;
            const uint32_t n = count_of[step];
            if (n <= kSampleMembers) break;
            // the keys of this step's members
            uint32_t lo = ~0u, hi = 0;
            each([&](float x, int) {
                if (inside(x) && step_of(x) == step) {
                    const uint32_t key = sample_key(x);
                    lo = min(lo, key);
                    hi = max(hi, key);
                }
            });
            if (lo <= hi) { atomicMin(&low_s, lo); atomicMax(&high_s, hi); }
            __syncthreads();
            key_low = low_s;
            key_high = high_s;
            value_step = 0;
            if (key_low == key_high) {               // one value: its first ones, by index
                const float x0 = sample_value(key_low);
                const sr_mass one = by_mass ? mass(x0) : 1;
                const sr_mass n_kept = (limit - before + one - 1) / one;
                sr_mass all;
                const int at = index_of([&](float x, int i) -> sr_mass { return x == x0 && kept(x, i) ? 1 : 0; },
                                        [&](sr_mass) { return n_kept - 1; }, all);
                cut_v = floor_v = x0;
                cut_at = at;
                return;
            }
            shift = 0;
            while (((key_high - key_low) >> shift) >= (uint32_t)kSampleSteps) ++shift;
        }
        each([&](float x, int at) {
            if (!inside(x) || step_of(x) != step) return;
            const sr_mass m = by_mass ? mass(x) : 1;
            if (m == 0) return;
            const uint32_t i = atomicAdd(&n_members, 1u);
            member_key[i] = sample_key(x);
            member_at[i] = at;
            member_mass[i] = m;
        });
        __syncthreads();
        const int n = (int)n_members;
        if (tid < n) {
            const uint32_t key = member_key[tid];
            const int at = member_at[tid];
            sr_mass up = before;
            for (int j = 0; j < n; ++j) {
                const uint32_t k = member_key[j];
                up += k > key || (k == key && member_at[j] < at) ? member_mass[j] : 0;
            }
            if (up < limit && limit - up <= member_mass[tid]) { low_s = key; high_s = (uint32_t)at; }
        }
        __syncthreads();
        cut_v = floor_v = sample_value(low_s);
        cut_at = (int)high_s;
    };
    if (top_k > 0 && top_k < V) cut(false, [&](sr_mass) { return (sr_mass)top_k; });
    if (top_p < 1.0f) cut(true, [&](sr_mass total) { return max((sr_mass)ceil((double)top_p * (double)total), (sr_mass)1); });

    const float u = p.uniform[row];
    sr_mass total;
    const int tok = index_of([&](float x, int at) -> sr_mass { return kept(x, at) ? mass(x) : 0; },
                             [&](sr_mass sum) { return min((sr_mass)((double)(u > 0.0f ? fminf(u, 1.0f) : 0.0f) * (double)sum), sum - 1); }, total);
    if (tid == 0) {
        p.tok[row] = tok;
        if (p.logprob) {
            const float x = seen((float)L[tok]);
            p.logprob[row] = (float)(((double)x - (double)most) / (double)temp - log((double)total / kSampleUnit));
        }
    }
}
