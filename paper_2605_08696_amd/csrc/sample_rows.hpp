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
// A work-group takes a row; a thread reads eight consecutive logits, a wavefront 512, a segment.  Passes over the row:
//   the largest logit, and each thread's own largest: the top_k-th largest of those is a lower bound of the row's;
//   top-k: the logits above that bound are listed; top-p: a histogram of weights over 2048 equal steps of logit value, and a list of the
//   step in which the limit is reached;
//   the list (LDS) is divided by key until a few members are left, which are compared with each other, or one value, of which the
//   first ones by index are kept;
//   sums of the kept weights by segment, one of which holds the token.
// A list that is too long (nearly equal logits) and a top_k above 512 take the histogram again, of the step's keys or of counts.
//
// bf16 logits have few values.  Their weights are formed once per value, not per logit, into a table in LDS, and a row with top-p alone
// counts its logits by value in its first pass: the counts times the table give the last kept value and how many of it are kept, and the
// second pass is the last one.
//
// What bounds it (us, rows x logits, normal logits): fp32 rows the instructions of the weights, some 30 per logit and pass that forms them
// (one, two with top-p), eight independent chains at a time; bf16 rows the LDS, 18 clocks of a CU for a wavefront's 64 additions to the counts
// and as many for its 64 looks into the table; below that the row's passes through the last-level cache.
//   greedy | no limit | top-p 0.95 | top-k 50 | min-p 0.05: 256 x 32000 fp32 6.3 | 18 | 40 | 17 | 14, bf16 5.7 | 17 | 24 | 16 | 13;
//   1000 x 128001 fp32 105 | 190 | 427 | 162 | 160, bf16, the logits in the last-level cache 61 (4.2 TB/s) | 124 | 177 | 97 | 97, from memory
//   83 | 145 | 190 | 115 | 117; one row of 32000 fp32 3.9 | 14 | 32 | 14 | 10.
//   With weights of bf16 logits formed one by one 1000 x 128001 took 441 with top-p, with a table but a histogram of weights 397, counted in a
//   pass of its own 205.  A table of the limit's region only (guessed from one segment in eight, fewer LDS additions): 421.
#pragma once
#include "fp8.hpp"
#include <cstddef>
#include <type_traits>

typedef unsigned long long sr_mass;
typedef __attribute__((ext_vector_type(2))) uint16_t sr_codes;
constexpr int kSampleVocab = 1 << 20, kSampleSegment = 512, kSampleSteps = kSampleVocab / kSampleSegment;
// The table of bf16 weights: magnitudes from 2^-11 up to 2^9, twenty octaves of 128 codes, of both signs.  Forming it is a good part of
// a short row's work: with it | without, us, 2000 rows with top-p of 4096 logits 63 | 56, 8192: 73 | 84, 32000: 127 | 220; without limits 16384:
// 56 | 55, 24576: 69 | 72, 32000: 83 | 90.
constexpr int kCodeSign = 2560, kCodeFrom = 0x3A00, kSampleCodes = 2 * kCodeSign, kSampleCounted = 6144, kSampleTabled = 20480;
constexpr float kTinyLogit = 0.00048828125f, kHugeLogit = 512.0f;
constexpr int kSampleList = 1024, kSampleFew = 64, kSampleBound = 512, kSampleDense = 256;
#define SR_INLINE __attribute__((always_inline))
constexpr double kSampleUnit = 8796093022208.0;      // 2^43

struct SampleRows {
    int64_t rows, ld;
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

// round(2^43 2^(d c)) for d c from -900 to 0 (0 below -44).  2^f on [-1/2, 1/2] by the polynomial of degree 9 with the constant term 1
// (so that d = 0 gives the unit) whose other part interpolates (2^f - 1) / f at Chebyshev's points: below 2^-44 of the value.
// (N at a time, stage by stage: a chain of dependent fp64 instructions takes twice the clocks that issuing them does, and left alone the
// compiler forms one chain behind the other.)
template <int N>
__device__ __forceinline__ void sample_mass(const double (&d)[N], double c, sr_mass (&m)[N])
{
    constexpr double magic = 6755399441055744.0 + 43.0;                // 1.5 2^52 + 43: a sum with it holds 43 + the nearest integer n in the low bits
    constexpr double coef[9] = {1.0203121063391729e-07, 1.3255224878668817e-06, 1.525268684626772e-05, 0.00015403455852453838, 0.0013333558179043112, 0.009618129159402558, 0.055504108664760424, 0.2402265069581299, 0.6931471805599453};
    double t[N], f[N], p[N];
#pragma unroll
    for (int i = 0; i < N; ++i) t[i] = __builtin_fma(d[i], c, magic);
    if constexpr (N > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = t[i] - magic;
    if constexpr (N > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = __builtin_fma(d[i], c, -f[i]);
    if constexpr (N > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) p[i] = coef[0];
#pragma unroll
    for (int k = 1; k < 10; ++k) {
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = __builtin_fma(p[i], f[i], k < 9 ? coef[k] : 1.0);
        if constexpr (N > 1) __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {                    // p 2^(43 + n), then its nearest integer in the mantissa of 2^52 + it
        const unsigned long long bits = __builtin_bit_cast(unsigned long long, p[i]);
        uint32_t high = (uint32_t)(bits >> 32) + ((uint32_t)__builtin_bit_cast(unsigned long long, t[i]) << 20);
        asm("" : "+v"(high));                        // (one 32-bit instruction; a 64-bit sum otherwise)
        p[i] = __builtin_bit_cast(double, (unsigned long long)high << 32 | (uint32_t)bits) + 4503599627370496.0;
    }
    if constexpr (N > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < N; ++i) m[i] = __builtin_bit_cast(unsigned long long, p[i]) & 0xFFFFFFFFFFFFFull;
}

// Lane exchanges by DPP: through the LDS crossbar a scan or sum of 64 bits is a chain of twelve trips of some hundred clocks.
template <int CTRL, int ROWS = 0xF>
__device__ __forceinline__ sr_mass sample_moved(sr_mass x)              // 0 where no lane is the source
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)x, CTRL, ROWS, 0xF, false);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(x >> 32), CTRL, ROWS, 0xF, false);
    return (sr_mass)hi << 32 | lo;
}
__device__ __forceinline__ sr_mass sample_lane(sr_mass x, int lane)
{
    return (sr_mass)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane);
}
// Running sum over the wavefront's lanes, this one's included.
__device__ __forceinline__ sr_mass sample_wave_scan(sr_mass v)
{
    v += sample_moved<0x111>(v);                     // row_shr:1, 2, 4, 8
    v += sample_moved<0x112>(v);
    v += sample_moved<0x114>(v);
    v += sample_moved<0x118>(v);
    v += sample_moved<0x142, 0xA>(v);                // row_bcast:15 into rows 1 and 3
    v += sample_moved<0x143, 0xC>(v);                // row_bcast:31 into rows 2 and 3
    return v;
}
__device__ __forceinline__ uint32_t sample_wave_scan32(uint32_t v)
{
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xF, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xA, 0xF, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xC, 0xF, false);
    return v;
}
// Sum over the wavefront, in every lane.
__device__ __forceinline__ sr_mass sample_wave_sum(sr_mass v)
{
    v += sample_moved<0xB1>(v);                      // quad_perm [1,0,3,2], [2,3,0,1], row_half_mirror, row_mirror
    v += sample_moved<0x4E>(v);
    v += sample_moved<0x141>(v);
    v += sample_moved<0x140>(v);
    return (sample_lane(v, 0) + sample_lane(v, 16)) + (sample_lane(v, 32) + sample_lane(v, 48));
}
// The same of values below 2^52, whose low 26 and high 26 bits do not leave 32 bits: half the instructions.
__device__ __forceinline__ sr_mass sample_wave_sum52(sr_mass v)
{
    auto sum = [](uint32_t x) {
        x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xF, 0xF, true);
        x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xF, 0xF, true);
        x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x141, 0xF, 0xF, true);
        x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x140, 0xF, 0xF, true);
        return ((uint32_t)__builtin_amdgcn_readlane((int)x, 0) + (uint32_t)__builtin_amdgcn_readlane((int)x, 16)) +
               ((uint32_t)__builtin_amdgcn_readlane((int)x, 32) + (uint32_t)__builtin_amdgcn_readlane((int)x, 48));
    };
    return (sr_mass)sum((uint32_t)v & 0x3ffffffu) + ((sr_mass)sum((uint32_t)(v >> 26)) << 26);
}
__device__ __forceinline__ uint32_t sample_wave_max(uint32_t v)
{
    const int r = (int)row16_max_u32(v);
    return max(max((uint32_t)__builtin_amdgcn_readlane(r, 0), (uint32_t)__builtin_amdgcn_readlane(r, 16)),
               max((uint32_t)__builtin_amdgcn_readlane(r, 32), (uint32_t)__builtin_amdgcn_readlane(r, 48)));
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT, 4)
sample_rows_kernel(const T *__restrict__ logits, SampleRows p)
{
    constexpr int NW = NT / 64, PER = kSampleSteps / NT;
    static_assert(NW * kSampleDense >= 2 * kSampleSegment, "the weights of a segment fit");
    __shared__ sr_mass red[NW];
    struct Lds {
        sr_mass table[kSampleSteps];                 // sums by step or by segment
        uint32_t list_key[kSampleList];
        int list_at[kSampleList];
    };
    __shared__ Lds lds;
    sr_mass *const table = lds.table;
    uint32_t *const list_key = lds.list_key;
    int *const list_at = lds.list_at;
    __shared__ __align__(8) float dense[NW * kSampleDense];             // kept logits of the wavefronts' segments; the weights of a segment
    __shared__ sr_mass few_rank[kSampleFew], few_mass[kSampleFew], few_sum[kSampleFew];
    constexpr bool CODES = sizeof(T) == 2;
    __shared__ sr_mass by_code[CODES ? kSampleCodes + 1 : 1];
    __shared__ sr_mass found_before;
    __shared__ uint32_t found, low_s, high_s, n_list;
    const int64_t row = work_group();
    if (row >= p.rows) return;
    int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = p.V;
    const T *L = logits + row * p.ld;
    auto scalar = [](float x) SR_INLINE { return __uint_as_float((uint32_t)__builtin_amdgcn_readfirstlane((int)__float_as_uint(x))); };
    auto uniform = [](bool x) SR_INLINE { return __builtin_amdgcn_readfirstlane((int)x) != 0; };
    bool hot = false;                                // an infinite logit leaves all others without weight: see below

    // eight logits from `at` on, -infinity behind the row
    auto complete = [&](const Raw8<T> &raw, int at, float (&v)[8]) SR_INLINE {
        widen8(raw, at, V, v);
        if (__ballot(at + 8 > V)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at + i < V ? v[i] : -INFINITY;
        }
        if (hot) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = v[i] == INFINITY ? 0.0f : -INFINITY;
        }
    };
    // fn(values, index of the first); the next vector is on its way meanwhile
    auto first_raw = [&]() SR_INLINE { return raw8(L, wave * kSampleSegment + lane * 8, V); };
    auto pass_from = [&](Raw8<T> raw, auto &&fn) SR_INLINE {
        constexpr int STEP = NW * kSampleSegment;
        int at = wave * kSampleSegment + lane * 8;
        for (int first = wave * kSampleSegment; first < V; first += STEP) {
            const Raw8<T> next = raw8(L, at + STEP, V);
            float v[8];
            complete(raw, at, v);
            fn(v, at);
            raw = next;
            at += STEP;
        }
    };
    auto pass = [&](auto &&fn) SR_INLINE { pass_from(first_raw(), fn); };
    // exclusive prefix sum over the threads; total: of all
    auto scan = [&](sr_mass v, sr_mass &total) SR_INLINE {
        const sr_mass s = sample_wave_scan(v);
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
    auto clear = [&]() SR_INLINE {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PER; ++i) table[i * NT + tid] = 0;
        if (tid == 0) { found = ~0u; n_list = 0; low_s = ~0u; high_s = 0; }
        __syncthreads();
    };
    // The entry of the table in which before + its running sum reaches limit_of(sum of all): its number, and `before` becomes the sum in
    // front of it.  ~0u if none does.
    auto reached = [&](sr_mass &before, auto &&limit_of, sr_mass &total) SR_INLINE {
        __syncthreads();
        sr_mass own = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i) own += table[tid * PER + i];
        sr_mass up = before + scan(own, total);
        const sr_mass limit = limit_of(total);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const sr_mass s = table[tid * PER + i];
            if (up < limit && limit - up <= s) { found = tid * PER + i; found_before = up; }
            up += s;
        }
        __syncthreads();
        before = found_before;
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)found);
    };
    // low_s and high_s: the smallest and the largest of the threads' keys.  (A wavefront's first: the compiler turns an atomic of 64
    // lanes on one word into a loop over the lanes.)
    auto range = [&](uint32_t lo, uint32_t hi) SR_INLINE {
        lo = ~sample_wave_max(~lo);
        hi = sample_wave_max(hi);
        if (lane == 0 && lo <= hi) { atomicMin(&low_s, lo); atomicMax(&high_s, hi); }
    };

    const Raw8<T> raw = first_raw();                 // (on its way while the parameters are read)
    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    const float top_p = p.top_p ? p.top_p[row] : 1.0f;
    const float min_w = p.min_p ? p.min_p[row] : 0.0f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const bool by_count = uniform(top_k > 0 && top_k < V), by_sum = uniform(top_p < 1.0f);

    // A logit's place in the table of bf16 weights is its code minus the first one of its sign's part, in 16 bits modulo 2^16; logits
    // that are not in the table have its end for a place, of which those from kHugeLogit up have to be absent and those of a magnitude
    // below kTinyLogit to be told apart.  Places of N logits times 2^SHIFT:
    auto places = [&](const auto &v, auto &&at, auto shift) SR_INLINE {
        constexpr uint16_t pos = kCodeFrom, neg = 0x8000 + kCodeFrom - kCodeSign, end = kSampleCodes;
#pragma unroll
        for (unsigned i = 0; i < sizeof(v) / sizeof(v[0]); i += 2) {
            const sr_codes x = __builtin_bit_cast(sr_codes, __builtin_amdgcn_perm(__float_as_uint(v[i + 1]), __float_as_uint(v[i]), 0x07060302u));
            const sr_codes y = __builtin_elementwise_min(__builtin_elementwise_min((sr_codes)(x - pos), (sr_codes)(x - neg)), sr_codes{end, end}) << (uint16_t)decltype(shift)::value;
            at[i] = y[0];
            at[i + 1] = y[1];
        }
    };
    auto tiny = [&](const auto &v) SR_INLINE {       // one of the wavefront's logits is
        float small = fabsf(v[0]);
#pragma unroll
        for (unsigned i = 1; i < sizeof(v) / sizeof(v[0]); ++i) small = fminf(small, fabsf(v[i]));
        return __ballot(small < kTinyLogit) != 0;
    };
    // Rows of bf16 logits with top-p alone are counted by code while their largest is looked for; the tiny ones are listed.
    uint32_t *const count = reinterpret_cast<uint32_t *>(&lds);
    static_assert(offsetof(Lds, list_at) == kSampleCodes * 4 && kSampleCodes % NT == 0, "the counts fit in front of the list");
    const bool counted = CODES && V >= kSampleCounted && by_sum && !by_count && uniform(temp > 0.0f && top_p > 0.0f && !(min_w > 0.0f));
    if (counted) {
#pragma unroll
        for (int i = 0; i < kSampleCodes / NT; ++i) count[i * NT + tid] = 0;
        if (tid == 0) n_list = 0;
        __syncthreads();
    }
    float own_most = -INFINITY;
    pass_from(raw, [&](const float (&v)[8], int) SR_INLINE {
#pragma unroll
        for (int i = 0; i < 8; ++i) own_most = fmaxf(own_most, v[i]);
        if constexpr (CODES) {
            if (!counted) return;
            uint32_t at[8];
            places(v, at, std::integral_constant<int, 2>{});
            if (tiny(v)) {
#pragma unroll
                for (int i = 0; i < 8; ++i) at[i] = fabsf(v[i]) < kTinyLogit ? 4 * kSampleCodes : at[i];
#pragma unroll 1
                for (int i = 0; i < 8; ++i) {
                    float x = v[0];
#pragma unroll
                    for (int k = 1; k < 8; ++k) x = i == k ? v[k] : x;
                    if (fabsf(x) < kTinyLogit) {
                        const uint32_t k = atomicAdd(&n_list, 1u);
                        if (k < (uint32_t)kSampleList) list_at[k] = (int)__float_as_uint(x);
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (at[i] < 4 * kSampleCodes) atomicAdd(reinterpret_cast<uint32_t *>(reinterpret_cast<char *>(count) + at[i]), 1u);
        }
    });
    const uint32_t wave_most = sample_wave_max(sample_key(own_most));
    if (lane == 0) red[wave] = wave_most;
    __syncthreads();
    uint32_t most_key = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) most_key = max(most_key, (uint32_t)red[i]);
    float most = sample_value((uint32_t)__builtin_amdgcn_readfirstlane((int)most_key));
    if (most == -INFINITY) {                         // nothing to draw from
        if (tid == 0) {
            p.tok[row] = -1;
            if (p.logprob) p.logprob[row] = -INFINITY;
        }
        return;
    }

    if (!(temp > 0.0f) || top_k == 1 || top_p <= 0.0f) {                // one token: the first of the largest
        int first = V;
        if (own_most == most)
            for (int at = wave * kSampleSegment + lane * 8; at < V && first == V; at += NW * kSampleSegment) {
                float v[8];
                complete(raw8(L, at, V), at, v);
#pragma unroll
                for (int i = 7; i >= 0; --i)
                    if (v[i] == most) first = at + i;
            }
        first = ~(int)sample_wave_max(~(uint32_t)first);
        __syncthreads();
        if (lane == 0) red[wave] = (sr_mass)first;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < NW; ++i) first = min(first, (int)red[i]);
        if (tid == 0) {
            p.tok[row] = first;
            if (p.logprob) p.logprob[row] = 0.0f;
        }
        return;
    }

    // (a row with an infinite logit is read as 0 where it is infinite and -infinity elsewhere)
    hot = uniform(most == INFINITY);
    if (hot) { own_most = own_most == INFINITY ? 0.0f : -INFINITY; most = 0.0f; }
    const double most_d = (double)most, per_bit = (double)fminf(temp, 1e30f) * 0.6931471805599453, c = 1.0 / per_bit;
    // (2^-900 and less are alike; also what a NaN counts as)
    const double clamp_d = -900.0 * per_bit;
    const float min_p = min_w > 0.0f ? fminf(min_w, 1.0f) : 0.0f;
    const sr_mass least = min_p > 0.0f ? max((sr_mass)1, (sr_mass)ceil((double)min_p * kSampleUnit)) : 1;
    const bool has_least = uniform(least > 1);
    auto mass = [&](float x) SR_INLINE {
        const double d[1] = {fmax((double)x - most_d, clamp_d)};
        sr_mass m[1];
        sample_mass(d, c, m);
        return m[0] >= least ? m[0] : 0;
    };
    // Nothing below floor_v has weight (it lies a little too low: weights decide); of value cut_v only indices up to cut_at are kept.
    const double lowest = (double)most + (has_least ? log2((double)least / kSampleUnit) - 0.001 : -44.001) * per_bit;
    float floor_v = scalar((float)(lowest - fabs(lowest) * 1e-6));
    float cut_v = -INFINITY;
    int cut_at = V;
    bool cut = false, summed = false, in_list = false;                  // summed: the table holds the segments' sums; in_list: the list holds all kept logits (and others, which kept() tells)
    uint32_t n = 0;                                  // of the list
    auto kept = [&](float x, int at) SR_INLINE { return x > cut_v || (x == cut_v && at <= cut_at); };
    // vectors that hold a logit from floor_v up
    auto live = [&](const float (&v)[8]) SR_INLINE {
        float top = v[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, v[i]);
        return __ballot(top >= floor_v) != 0;
    };
    // bf16 logits have few values, whose weights fit a table (codes above the largest logit's count as that)
    bool tabled = false, cut_in_table = false;       // cut_in_table: logits from cut_v down have no weight there
    auto tabulate = [&]() SR_INLINE {
        if constexpr (CODES) {
            if (tabled || hot || !(most < kHugeLogit && floor_v > -kHugeLogit)) return;
            for (int i0 = tid; i0 <= kSampleCodes; i0 += 8 * NT) {
                double d[8];
                sr_mass m[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = i0 + k * NT;
                    const uint32_t bits = (uint32_t)(i + (i < kCodeSign ? kCodeFrom : 0x8000 + kCodeFrom - kCodeSign)) << 16;
                    d[k] = fmin(fmax((double)__uint_as_float(bits) - most_d, clamp_d), 0.0);
                }
                sample_mass(d, c, m);
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int i = i0 + k * NT;
                    if (i <= kSampleCodes) by_code[i] = i < kSampleCodes && m[k] >= least ? m[k] : 0;
                }
            }
            tabled = true;
            __syncthreads();
        }
    };
    // the weights of N logits from the table; false if one of the wavefront's is not in it
    auto looked_up = [&](auto &v, auto &m) SR_INLINE {
        if constexpr (CODES) {
            constexpr int N = sizeof(v) / sizeof(v[0]);
            if (!tabled) return false;
            if (tiny(v)) return false;
            uint32_t at[N];
            places(v, at, std::integral_constant<int, 3>{});
#pragma unroll
            for (int i = 0; i < N; ++i) m[i] = *reinterpret_cast<const sr_mass *>(reinterpret_cast<const char *>(by_code) + at[i]);
            return true;
        }
        return false;
    };
    // the weights of a vector's kept logits, in chains that do not wait for each other
    auto masses = [&](const float (&v)[8], int at, sr_mass (&m)[8]) SR_INLINE {
        const bool from_table = looked_up(v, m);
        if (!from_table) {
            double d[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = (double)v[i];
#pragma unroll
            for (int i = 0; i < 8; ++i) d[i] = fmax(d[i] - most_d, clamp_d);
            sample_mass(d, c, m);
            if (has_least) {
#pragma unroll
                for (int i = 0; i < 8; ++i) m[i] = m[i] >= least ? m[i] : 0;
            }
        }
        if (cut && !(from_table && cut_in_table)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) m[i] = kept(v[i], at + i) ? m[i] : 0;
        }
    };
    // The first index at which the running sum of weights exceeds target(sum of all): one_of(value, index) gives a kept logit's,
    // of(values, index, weights) those of a vector, and sum_of(values, index) the sum of the wavefront's vectors.
    auto index_of = [&](auto &&one_of, auto &&of, auto &&sum_of, auto &&target, sr_mass &total) SR_INLINE {
        if (!summed) clear();
        if (summed) {
        } else if (in_list) {
            for (uint32_t i = tid; i < n; i += NT) {
                const float x = sample_value(list_key[i]);
                const int at = list_at[i];
                if (kept(x, at)) atomicAdd(&table[at / kSampleSegment], one_of(x, at));
            }
        } else {
            pass([&](const float (&v)[8], int at) SR_INLINE {
                if (!live(v)) return;
                const sr_mass s = sum_of(v, at);
                if (lane == 0) table[at / kSampleSegment] = s;
            });
        }
        sr_mass before = 0, goal = 0;
        const uint32_t seg = min(reached(before, [&](sr_mass sum) SR_INLINE { goal = target(sum); return goal + 1; }, total),
                                 (uint32_t)(V - 1) / kSampleSegment);
        sr_mass *weights = reinterpret_cast<sr_mass *>(dense);
        if (in_list) {
            for (int i = tid; i < kSampleSegment; i += NT) weights[i] = 0;
            __syncthreads();
            for (uint32_t i = tid; i < n; i += NT) {
                const float x = sample_value(list_key[i]);
                const int at = list_at[i];
                if ((uint32_t)at / kSampleSegment == seg && kept(x, at)) weights[at % kSampleSegment] = one_of(x, at);
            }
        }
        __syncthreads();
        if (wave == 0) {
            const int at = (int)seg * kSampleSegment + lane * 8;
            sr_mass m[8], s = 0;
            if (in_list) {
#pragma unroll
                for (int i = 0; i < 8; ++i) m[i] = weights[lane * 8 + i];
            } else {
                float v[8];
                complete(raw8(L, at, V), at, v);
                of(v, at, m);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) s += m[i];
            sr_mass run = before + sample_wave_scan(s) - s;
            if (goal >= run && goal - run < s) {
                int k = 0;
#pragma unroll
                for (int i = 0; i < 7; ++i) {
                    run += m[i];
                    if (k == i && goal >= run) k = i + 1;
                }
                found = at + k;
            }
        }
        __syncthreads();
        return (int)found;
    };
    // Lists the logits from `from` to `to`: how many there are, or more than kSampleList if they do not fit (what is listed is no use then).
    auto gather = [&](float from, float to) SR_INLINE {
        __syncthreads();
        if (tid == 0) n_list = 0;
        __syncthreads();
        from = fmaxf(from, floor_v);
        bool full = false;
        pass([&](const float (&v)[8], int at) SR_INLINE {
            if (full) return;
            uint32_t own = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) own += v[i] >= from && v[i] <= to ? 1u : 0u;
            if (__ballot(own != 0) == 0) return;
            const uint32_t upto = sample_wave_scan32(own), sum = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
            uint32_t k = 0;
            if (lane == 0) k = atomicAdd(&n_list, sum);
            k = (uint32_t)__builtin_amdgcn_readfirstlane((int)k);
            full = k + sum > (uint32_t)kSampleList;
            if (full) return;
            k += upto - own;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] >= from && v[i] <= to) { list_key[k] = sample_key(v[i]); list_at[k] = at + i; ++k; }
        });
        __syncthreads();
        return (uint32_t)__builtin_amdgcn_readfirstlane((int)n_list);
    };

    if (has_least) {                                 // min-p leaves few of most rows: those are listed
        n = gather(floor_v, INFINITY);
        in_list = n <= (uint32_t)kSampleList;
    }
    auto top_p_limit = [&](sr_mass sum) SR_INLINE { return max((sr_mass)ceil((double)top_p * (double)sum), (sr_mass)1); };
    // top-p of counted rows: from the counts follow the last kept value and how many of it are kept; then the segments' sums and their
    // numbers of that value, in one pass.  false if the limit is reached among the tiny ones.
    auto top_p_by_code = [&]() SR_INLINE {
        if constexpr (CODES) {
            constexpr int PERC = kSampleCodes / NT;
            if (tid == 0) { few_sum[0] = 0; found = ~0u; }
            __syncthreads();
            for (uint32_t i = tid; i < n_list; i += NT) atomicAdd(&few_sum[0], mass(__uint_as_float((uint32_t)list_at[i])));
            __syncthreads();
            const sr_mass tiny_sum = few_sum[0];
            // the k-th code from the largest down: positive ones lie the other way round
            auto place = [&](int k) SR_INLINE { return k < kCodeSign ? kCodeSign - 1 - k : k; };
            sr_mass own = 0, total;
#pragma unroll
            for (int i = 0; i < PERC; ++i) {
                const int k = tid * PERC + i;
                own += (sr_mass)count[place(k)] * by_code[place(k)];
            }
            sr_mass up = scan(own, total);
            const sr_mass limit = top_p_limit(total + tiny_sum);
#pragma unroll
            for (int i = 0; i < PERC; ++i) {
                const int k = tid * PERC + i;
                const sr_mass one = by_code[place(k)], all_of = (sr_mass)count[place(k)] * one, before = up + (k >= kCodeSign ? tiny_sum : 0);
                if (before < limit && limit - before <= all_of) {
                    found = (uint32_t)k;
                    low_s = (uint32_t)((limit - before + one - 1) / one);
                    high_s = count[place(k)];
                }
                up += all_of;
            }
            __syncthreads();
            const int last = __builtin_amdgcn_readfirstlane((int)found), last_at = place(last);
            if (last < 0) return false;
            const uint32_t n_kept = (uint32_t)__builtin_amdgcn_readfirstlane((int)low_s);
            const bool some = uniform(n_kept < high_s);          // not all of the value
            cut_v = __uint_as_float((uint32_t)(last_at + (last < kCodeSign ? kCodeFrom : 0x8000 + kCodeFrom - kCodeSign)) << 16);
            cut_at = some ? -1 : V;
            cut = cut_in_table = true;
            floor_v = scalar(fmaxf(floor_v, cut_v));
            const sr_mass one = by_code[last_at];
            __syncthreads();
            for (int k = last + (some ? 0 : 1) + tid; k < kSampleCodes; k += NT) by_code[place(k)] = 0;
            clear();
            pass([&](const float (&v)[8], int at) SR_INLINE {
                if (!live(v)) return;
                sr_mass m[8], s = 0;
                masses(v, at, m);
#pragma unroll
                for (int i = 0; i < 8; ++i) s += m[i];
                s = sample_wave_sum52(s);
                uint32_t ties = 0;
                if (some) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) ties += (uint32_t)__popcll(__ballot(v[i] == cut_v));
                }
                if (lane == 0) table[at / kSampleSegment] = s | (sr_mass)ties << 53;         // (512 2^43 < 2^53)
            });
            if (some) {
                __syncthreads();
                sr_mass ties = 0;
#pragma unroll
                for (int i = 0; i < PER; ++i) ties += table[tid * PER + i] >> 53;
                sr_mass before = scan(ties, total);
#pragma unroll
                for (int i = 0; i < PER; ++i) {
                    const sr_mass s = table[tid * PER + i], here = s >> 53;
                    const sr_mass kept_here = before < n_kept ? min(here, n_kept - before) : 0;
                    table[tid * PER + i] = (s & ((1ull << 53) - 1)) + kept_here * one;
                    if (before < n_kept && n_kept - before <= here) { found = (uint32_t)(tid * PER + i); low_s = n_kept - (uint32_t)before; }
                    before += here;
                }
                __syncthreads();
                if (wave == 0) {                     // of this segment the low_s first ones
                    const int first = (int)found * kSampleSegment + lane * 8;
                    float v[8];
                    complete(raw8(L, first, V), first, v);
                    uint32_t own_ties = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) own_ties += v[i] == cut_v ? 1u : 0u;
                    uint32_t rank = low_s - (sample_wave_scan32(own_ties) - own_ties);         // of this lane's
                    if (rank - 1 < own_ties) {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (v[i] == cut_v && --rank == 0) high_s = (uint32_t)(first + i);
                    }
                    if (lane == 0) by_code[last_at] = one;
                }
                __syncthreads();
                cut_at = __builtin_amdgcn_readfirstlane((int)high_s);
                cut_in_table = false;
            }
            __syncthreads();
            if (tid == 0) found = ~0u;
            return true;
        }
        return false;
    };
    // top-k (their number), then top-p (their mass): the kept tokens end at the first one with which a limit is reached
    if (counted && uniform(n_list <= (uint32_t)kSampleList)) {
        tabulate();
        summed = tabled && top_p_by_code();
    }
    for (int by_mass = summed ? 2 : 0; by_mass < 2; ++by_mass) {
        if (by_mass ? !by_sum : !by_count) continue;
        asm volatile("" : "+v"(tid), "+v"(lane));    // (addresses formed from them are not held in registers from here to the end)
        auto limit_of = [&](sr_mass sum) SR_INLINE {
            return by_mass ? top_p_limit(sum) : (sr_mass)top_k;
        };
        const float scale = (float)kSampleSteps / (most - floor_v), scaled = most * scale;
        auto value_step = [&](float x) SR_INLINE { return (uint32_t)fminf(fmaf(x, -scale, scaled), (float)(kSampleSteps - 1)); };
        uint32_t low = 0, high = ~0u, step = 0;      // the keys that are left; the step of the table, of value while shift < 0
        int shift = -1;
        sr_mass before = 0, limit = 0, total;
        auto step_of = [&](float x) SR_INLINE { return shift < 0 ? value_step(x) : (high - sample_key(x)) >> shift; };
        auto in_keys = [&](uint32_t key) SR_INLINE { return key >= low && key <= high; };
        bool listed = false, all = false, whole = false;     // whole: all of the list is divided, not a step
        if (in_list) {
            clear();
            for (uint32_t i = tid; i < n; i += NT) {
                const float x = sample_value(list_key[i]);
                if (kept(x, list_at[i])) {
                    const sr_mass m = mass(x);
                    if (m) atomicAdd(&table[value_step(x)], by_mass ? m : (sr_mass)1);
                }
            }
            step = reached(before, [&](sr_mass sum) SR_INLINE { return limit = limit_of(sum); }, total);
            all = step == ~0u;
            listed = true;
        } else if (!by_mass && top_k <= kSampleBound) {
            // top_k threads whose largest logit is at least a bound hold top_k logits that are: those above it are listed
            clear();
            uint32_t mine = ~0u;
            if (own_most >= floor_v) {
                mine = value_step(own_most);
                atomicAdd(&table[mine], (sr_mass)1);
            }
            const uint32_t last = reached(before, limit_of, total);
            before = 0;
            if (last != ~0u) {
                const uint32_t own_key = sample_key(own_most);
                range(mine <= last ? own_key : ~0u, mine <= last ? own_key : 0);
                __syncthreads();
                const float bound = fmaxf(floor_v, sample_value((uint32_t)__builtin_amdgcn_readfirstlane((int)low_s)));
                n = gather(bound, INFINITY);
                listed = in_list = whole = n <= (uint32_t)kSampleList;
                limit = (sr_mass)top_k;
                if (listed) floor_v = bound;
            }
        }
        if (by_mass && !listed && V >= kSampleTabled) tabulate();
        while (!listed) {
            clear();
            pass([&](const float (&v)[8], int at) SR_INLINE {
                if (!live(v)) return;
                sr_mass m[8];
                if (by_mass) {
                    masses(v, at, m);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) m[i] = kept(v[i], at + i) ? 1 : 0;
                }
                if (shift < 0) {
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (v[i] >= floor_v) atomicAdd(&table[value_step(v[i])], m[i]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const uint32_t key = sample_key(v[i]);
                        if (v[i] >= floor_v && in_keys(key)) atomicAdd(&table[(high - key) >> shift], m[i]);
                    }
                }
            });
            step = reached(before, [&](sr_mass sum) SR_INLINE { return shift < 0 ? limit = limit_of(sum) : limit; }, total);
            all = step == ~0u;                       // never reached
            if (all) break;
            // about where the step lies (no bound where the scale is not finite)
            float from = -INFINITY, to = INFINITY;
            if (shift < 0) {
                const float width = 1.0f / scale, slack = fabsf(most) * 1e-6f;
                if (step + 1 < (uint32_t)kSampleSteps && width < 1e30f) from = most - ((float)step + 1.01f) * width - slack;
                if (width < 1e30f) to = most - ((float)step - 0.01f) * width + slack;
            } else {
                from = sample_value(low);
                to = sample_value(high);
            }
            for (int narrow = 0; narrow < 2 && !listed; ++narrow) {          // everything from there up, else the step alone
                n = gather(from, narrow ? to : INFINITY);
                listed = n <= (uint32_t)kSampleList;
                in_list = listed && narrow == 0;
            }
            if (listed) break;
            // the step is divided by the keys of its members
            uint32_t lo = ~0u, hi = 0;
            pass([&](const float (&v)[8], int at) SR_INLINE {
                if (!live(v)) return;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t key = sample_key(v[i]);
                    if (v[i] >= from && v[i] <= to && v[i] >= floor_v && in_keys(key) && step_of(v[i]) == step) { lo = min(lo, key); hi = max(hi, key); }
                }
            });
            range(lo, hi);
            __syncthreads();
            low = (uint32_t)__builtin_amdgcn_readfirstlane((int)low_s);
            high = (uint32_t)__builtin_amdgcn_readfirstlane((int)high_s);
            if (low == high) break;
            shift = 0;
            while (((high - low) >> shift) >= (uint32_t)kSampleSteps) ++shift;
        }
        if (all) continue;
        // the step's members in the list, by key, until a few or one value is left
        bool few = false;
        auto member = [&](uint32_t i) SR_INLINE {
            const uint32_t key = list_key[i];
            const float x = sample_value(key);
            return in_keys(key) && (whole || step_of(x) == step) && kept(x, list_at[i]);
        };
        while (listed) {
            __syncthreads();
            if (tid == 0) { n_list = 0; low_s = ~0u; high_s = 0; }
            __syncthreads();
            uint32_t lo = ~0u, hi = 0, in = 0;
            for (uint32_t i = tid; i < n; i += NT)
                if (member(i)) { lo = min(lo, list_key[i]); hi = max(hi, list_key[i]); ++in; }
            range(lo, hi);
            in = (uint32_t)sample_wave_sum(in);
            if (lane == 0 && in) atomicAdd(&n_list, in);
            __syncthreads();
            low = (uint32_t)__builtin_amdgcn_readfirstlane((int)low_s);
            high = (uint32_t)__builtin_amdgcn_readfirstlane((int)high_s);
            whole = true;
            few = uniform(n_list <= (uint32_t)kSampleFew);
            if (few || low == high) break;
            clear();
            shift = 0;
            while (((high - low) >> shift) >= (uint32_t)kSampleSteps) ++shift;
            for (uint32_t i = tid; i < n; i += NT)
                if (member(i)) {
                    const uint32_t key = list_key[i];
                    atomicAdd(&table[(high - key) >> shift], by_mass ? mass(sample_value(key)) : (sr_mass)1);
                }
            step = reached(before, [&](sr_mass) SR_INLINE { return limit; }, total);
            const uint32_t top = high - (step << shift), size = (1u << shift) - 1;
            low = top - low > size ? top - size : low;
            high = top;
        }
        if (few) {
            __syncthreads();
            if (tid == 0) n_list = 0;
            if (tid < kSampleFew) few_sum[tid] = 0;
            __syncthreads();
            for (uint32_t i = tid; i < n; i += NT)
                if (member(i)) {
                    const uint32_t k = atomicAdd(&n_list, 1u), key = list_key[i];
                    few_rank[k] = (sr_mass)key << 32 | (uint32_t)~list_at[i];            // larger: earlier in the order
                    few_mass[k] = by_mass ? mass(sample_value(key)) : (sr_mass)1;
                }
            __syncthreads();
            // lane: a member; wavefront w compares it with members w, w + NW, ...
            const int m = (int)n_list;
            const sr_mass rank = few_rank[min(lane, m - 1)], own = few_mass[min(lane, m - 1)];
            sr_mass sum = 0;
            for (int j = wave; j < m; j += NW) sum += few_rank[j] > rank ? few_mass[j] : 0;
            atomicAdd(&few_sum[lane], sum);
            __syncthreads();
            if (wave == 0 && lane < m) {
                const sr_mass up = before + few_sum[lane];
                if (up < limit && limit - up <= own) { low_s = (uint32_t)(rank >> 32); high_s = ~(uint32_t)rank; }
            }
            __syncthreads();
            cut_v = scalar(sample_value((uint32_t)__builtin_amdgcn_readfirstlane((int)low_s)));
            cut_at = __builtin_amdgcn_readfirstlane((int)high_s);
        } else {
            // of one value the first ones, by index
            const float x0 = sample_value(low);
            const sr_mass one = by_mass ? mass(x0) : 1, n_kept = (limit - before + one - 1) / one;
            const int last = x0 > cut_v ? V : cut_at;
            floor_v = fmaxf(floor_v, x0);
            const int at = index_of([&](float x, int) SR_INLINE { return (sr_mass)(x == x0); },
                                    [&](const float (&v)[8], int at, sr_mass (&m)[8]) SR_INLINE {
#pragma unroll
                for (int i = 0; i < 8; ++i) m[i] = v[i] == x0 && at + i <= last ? 1 : 0;
            }, [&](const float (&v)[8], int at) SR_INLINE {
                uint32_t s = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) s += (uint32_t)__popcll(__ballot(v[i] == x0 && at + i <= last));
                return (sr_mass)s;
            }, [&](sr_mass) SR_INLINE { return n_kept - 1; }, total);
            cut_v = x0;
            cut_at = __builtin_amdgcn_readfirstlane(at);
        }
        cut = true;
        floor_v = scalar(fmaxf(floor_v, cut_v));
    }

    if (V >= kSampleTabled && !in_list && !cut) tabulate();
    const float u = p.uniform[row];
    sr_mass total;
    const int tok = index_of([&](float x, int) SR_INLINE { return mass(x); }, masses, [&](const float (&v)[8], int at) SR_INLINE {
        sr_mass s = 0;
        uint32_t own = 8, upto = 8, some = kSampleSegment;
        bool equal = false;                          // some logit of the vector equals cut_v
        if (cut) {
            own = 0;
            unsigned long long eq = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                own += v[i] > cut_v ? 1u : 0u;
                eq |= __ballot(v[i] == cut_v);
            }
            equal = eq != 0;
            if (equal) {
#pragma unroll
                for (int i = 0; i < 8; ++i) own += v[i] == cut_v && at + i <= cut_at ? 1u : 0u;
            }
            upto = sample_wave_scan32(own);
            some = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
        if (some > (uint32_t)kSampleDense) {
            sr_mass m[8];
            masses(v, at, m);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += m[i];
        } else {                                     // few of the segment's logits are kept: side by side they take fewer evaluations
            float *to = dense + wave * kSampleDense + (upto - own);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] > cut_v || (equal && v[i] == cut_v && at + i <= cut_at)) *to++ = v[i];
            __builtin_amdgcn_wave_barrier();
            for (uint32_t j = lane; j < some + lane; j += 128) {
                const float *at2 = dense + wave * kSampleDense;
                const float x[2] = {j < some ? at2[j] : -INFINITY, j + 64 < some ? at2[j + 64] : -INFINITY};
                sr_mass m[2];
                if (!looked_up(x, m)) {
                    const double d[2] = {fmax((double)x[0] - most_d, clamp_d), fmax((double)x[1] - most_d, clamp_d)};
                    sample_mass(d, c, m);
#pragma unroll
                    for (int i = 0; i < 2; ++i) m[i] = m[i] >= least ? m[i] : 0;
                }
                s += m[0] + m[1];
            }
            __builtin_amdgcn_wave_barrier();
        }
        return sample_wave_sum52(s);                 // (a lane adds eight weights of 2^43 at most)
    }, [&](sr_mass sum) SR_INLINE { return min((sr_mass)((double)(u > 0.0f ? fminf(u, 1.0f) : 0.0f) * (double)sum), sum - 1); }, total);
    if (tid == 0) {
        p.tok[row] = tok;
        if (p.logprob) {
            const float x = hot ? 0.0f : (float)L[tok], t = fminf(p.temperature ? p.temperature[row] : 1.0f, 1e30f);
            p.logprob[row] = (float)(((double)x - most_d) / (double)t - log((double)total / kSampleUnit));
        }
    }
}

// ------------------------------------------------------------------ short rows
// The same of rows of up to 512 R logits: a wavefront takes a row, lane by lane eight consecutive logits of each segment, and keeps them and
// their weights in registers.  The last kept key is searched for by halves, of the values and every third time of the keys (which ends
// after 32 of those whatever the values), until one logit or one value is left; there is no list, no table and no barrier.
// (us, this | work-groups of 512 threads, without limits, top-p 0.9, top-k 20: 4000 x 512 5.6 | 48, 24 | 93, 16 | 83; 300 x 512 3.4 | 8.1,
// 13.3 | 14.3, 9.5 | 12.6; two segments 4000 x 1000 9.5 | 51, 41 | 97, 28 | 84, 300 x 1000 4.7 | 8.5, 18.5 | 15.1, 13.7 | 12.8; four, in 297
// registers, 4000 x 2000 22 | 51, 108 | 96, 81 | 82: not kept.  Halving by one of the keys that are left takes fewer, but slower steps: 26 us
// instead of 24.)
template <typename T, int R>
__global__ void __launch_bounds__(256)
sample_short_rows_kernel(const T *__restrict__ logits, SampleRows p)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), V = p.V;
    const int64_t row = (int64_t)work_group() * 4 + wave;
    if (row >= p.rows) return;
    const T *L = logits + row * p.ld;
    Raw8<T> raw[R];
#pragma unroll
    for (int j = 0; j < R; ++j) raw[j] = raw8(L, j * kSampleSegment + lane * 8, V);
    const float temp = p.temperature ? p.temperature[row] : 1.0f;
    const float top_p = p.top_p ? p.top_p[row] : 1.0f;
    const float min_w = p.min_p ? p.min_p[row] : 0.0f;
    const int top_k = p.top_k ? p.top_k[row] : 0;
    const float u = p.uniform[row];
    float v[R][8], most = -INFINITY;
#pragma unroll
    for (int j = 0; j < R; ++j) {
        const int at = j * kSampleSegment + lane * 8;
        widen8(raw[j], at, V, v[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[j][i] = at + i < V ? fmaxf(v[j][i], -INFINITY) : -INFINITY;      // (a NaN becomes -infinity)
            most = fmaxf(most, v[j][i]);
        }
    }
    most = sample_value(sample_wave_max(sample_key(most)));
    if (most == -INFINITY) {
        if (lane == 0) {
            p.tok[row] = -1;
            if (p.logprob) p.logprob[row] = -INFINITY;
        }
        return;
    }
    if (__builtin_amdgcn_readfirstlane((int)(!(temp > 0.0f) || top_k == 1 || top_p <= 0.0f))) {
        int first = V;
#pragma unroll
        for (int j = R - 1; j >= 0; --j)
#pragma unroll
            for (int i = 7; i >= 0; --i) first = v[j][i] == most ? j * kSampleSegment + lane * 8 + i : first;
        first = ~(int)sample_wave_max(~(uint32_t)first);
        if (lane == 0) {
            p.tok[row] = first;
            if (p.logprob) p.logprob[row] = 0.0f;
        }
        return;
    }
    if (most == INFINITY) {
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) v[j][i] = v[j][i] == INFINITY ? 0.0f : -INFINITY;
        most = 0.0f;
    }
    const double most_d = (double)most, temp_d = (double)fminf(temp, 1e30f), per_bit = temp_d * 0.6931471805599453, c = 1.0 / per_bit;
    const double clamp_d = -900.0 * per_bit;         // (2^-900 and less are alike)
    const sr_mass least = min_w > 0.0f ? max((sr_mass)1, (sr_mass)ceil((double)fminf(min_w, 1.0f) * kSampleUnit)) : 1;
    sr_mass m[R][8];
    uint32_t key[R][8];                              // 0: not to be drawn
#pragma unroll
    for (int j = 0; j < R; ++j) {
        double d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = fmax((double)v[j][i] - most_d, clamp_d);
        sample_mass(d, c, m[j]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            m[j][i] = m[j][i] >= least ? m[j][i] : 0;
            key[j][i] = m[j][i] ? sample_key(v[j][i]) : 0;
        }
    }
    auto count_from = [&](uint32_t from) SR_INLINE {
        int n = 0;
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) n += __popcll(__ballot(key[j][i] >= from));
        return n;
    };
    auto sum_from = [&](uint32_t from) SR_INLINE {
        sr_mass s = 0;
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) s += key[j][i] >= from ? m[j][i] : 0;
        return sample_wave_sum52(s);
    };
    // the largest key that enough() finds enough logits to have or exceed
    auto last_key = [&](auto &&enough) SR_INLINE {
        uint32_t least_key = ~0u;
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) least_key = min(least_key, key[j][i] - 1);        // (0 wraps)
        uint32_t lo = ~sample_wave_max(~least_key) + 1, hi = sample_key(most);
        int n_lo = count_from(lo), n_hi = 0;         // logits from lo up, above hi
        for (int half = 0; lo < hi && n_lo - n_hi > 1; half = half == 2 ? 0 : half + 1) {
            uint32_t mid = lo + (hi - lo + 1) / 2;
            if (half != 2) {
                const uint32_t k = sample_key(0.5f * sample_value(lo) + 0.5f * sample_value(hi));
                mid = k > lo && k <= hi ? k : mid;
            }
            mid = (uint32_t)__builtin_amdgcn_readfirstlane((int)mid);
            const int n = count_from(mid);
            if (enough(mid, n)) { lo = mid; n_lo = n; }
            else { hi = mid - 1; n_hi = n; }
        }
        uint32_t t = 0;
#pragma unroll
        for (int j = 0; j < R; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) t = max(t, key[j][i] <= hi ? key[j][i] : 0);
        return sample_wave_max(t);
    };
    // of the logits of key t the first ones are kept, as long as stays(how many are in front, the weight of one); none of a smaller key
    auto keep = [&](uint32_t t, auto &&stays) SR_INLINE {
        uint32_t before = 0;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            uint32_t own = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) own += key[j][i] == t ? 1u : 0u;
            const uint32_t upto = sample_wave_scan32(own);
            uint32_t rank = before + upto - own;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool equal = key[j][i] == t;
                if (key[j][i] < t || (equal && !stays(rank, m[j][i]))) { m[j][i] = 0; key[j][i] = 0; }
                rank += equal ? 1u : 0u;
            }
            before += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        }
    };
    if (__builtin_amdgcn_readfirstlane((int)(top_k > 0)) && top_k < count_from(1)) {
        const uint32_t t = last_key([&](uint32_t, int n) SR_INLINE { return n >= top_k; });
        const uint32_t ties = (uint32_t)(top_k - count_from(t + 1));
        keep(t, [&](uint32_t rank, sr_mass) SR_INLINE { return rank < ties; });
    }
    if (__builtin_amdgcn_readfirstlane((int)(top_p < 1.0f))) {
        const sr_mass limit = max((sr_mass)ceil((double)top_p * (double)sum_from(1)), (sr_mass)1);
        const uint32_t t = last_key([&](uint32_t from, int) SR_INLINE { return sum_from(from) >= limit; });
        const sr_mass rest = limit - sum_from(t + 1);
        keep(t, [&](uint32_t rank, sr_mass one) SR_INLINE { return rank * one < rest; });     // (equal ones have one weight)
    }
    sr_mass before = 0;
    const sr_mass total = sum_from(1), goal = min((sr_mass)((double)(u > 0.0f ? fminf(u, 1.0f) : 0.0f) * (double)total), total - 1);
#pragma unroll
    for (int j = 0; j < R; ++j) {
        sr_mass s = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += m[j][i];
        const sr_mass upto = before + sample_wave_scan(s);
        sr_mass run = upto - s;
        if (goal >= run && goal < upto) {            // in one lane
            int k = 0;
            float x = v[j][0];
#pragma unroll
            for (int i = 0; i < 7; ++i) {
                run += m[j][i];
                if (goal >= run) { k = i + 1; x = v[j][i + 1]; }
            }
            p.tok[row] = j * kSampleSegment + lane * 8 + k;
            if (p.logprob) p.logprob[row] = (float)(((double)x - most_d) / temp_d - log((double)total / kSampleUnit));
        }
        before = sample_lane(upto, 63);
    }
}
