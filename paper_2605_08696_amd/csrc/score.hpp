// Log probabilities of given tokens, the entropy of each row of logits and its most likely tokens, in one reading of the row and a second
// one from the caches.
//
// With m the largest logit, d = (m - l) / T >= 0 and w = e^-d:
//   Z = sum w      log p(v) = -d_v - log Z      entropy = log Z + (sum w d) / Z
// (both parts of the entropy are positive: nothing cancels).  A thread keeps its largest logit and the two sums relative to it, 32 logits at
// a time, and rescales them when a larger one comes; the threads' sums are joined in a fixed order.  d counts in factors of two and is
// held at 1000, beyond which w is 0 in fp32: a logit of -infinity, and a NaN, then add nothing without being looked for.
//
// The k most likely tokens: the k-th largest of 64 disjoint groups' largest logits is at or below the k-th largest of the row, so the
// logits from it on (some 1.3 k of them where the groups are alike) hold all that are wanted.  A row's first 32 logits a thread, which stay
// in registers, give such a bound; from there on every logit above it is listed as it comes, and a few hundred of 128000 are.  A list that
// overflows is made again, in a second reading, with the bound that the whole row gives.  The listed ones are put in order by counting,
// equal ones by their index.  A list that overflows again (equal logits in bulk) is not used: the tokens are then looked for one after the
// other, a reading each.
//
// What bounds it: the row is read once; for bf16 rows about as much the ten instruction slots that a logit takes, four of them its
// exponential's: 2001 x 128001 bf16 139 us, 512 MB at 3.7 TB/s, 600 x 150000 fp32 74 us, 4.9 TB/s.  One row: one CU's share of both, 32000 fp32
// logits 8.6 us, 150000 bf16 ones 22.  (With two readings, the threads' sums joined one by one and a compare for each exponential 189, 80, 15, 33.)
#pragma once
#include "fp8.hpp"

constexpr int kScoreTop = 32, kScoreList = 1024, kScoreVocab = 1 << 30;

struct ScoreCall {
    int64_t rows, ld;
    int V, k;
    const int32_t *token;
    const float *temperature;
    float *logprob, *entropy, *top_logprob;
    int32_t *top_token;
};

// Unsigned integers ordered as the floats are; -0 and +0 share a key.
__device__ __forceinline__ uint32_t score_key(float f)
{
    const uint32_t u = __float_as_uint(f + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float score_value(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key); }

struct ScoreSums {
    float m, z, e;                                   // the largest logit, sum of w, sum of w d relative to it
};
__device__ __forceinline__ float score_weight(float d) { return __builtin_amdgcn_exp2f(-d * 1.44269504088896340736f); }
// Sums relative to a's largest logit -> relative to `m`, at or above it.
__device__ __forceinline__ ScoreSums score_rescaled(const ScoreSums &a, float m, float inv)
{
    if (a.m == m || a.m == -INFINITY) return {m, a.z, a.e};
    const float d = (m - a.m) * inv, f = score_weight(d);
    return {m, f * a.z, f > 0.0f ? f * fmaf(d, a.z, a.e) : 0.0f};
}
__device__ __forceinline__ uint32_t score_wave_max(uint32_t v)
{
    const int r = (int)row16_max_u32(v);
    return max(max((uint32_t)__builtin_amdgcn_readlane(r, 0), (uint32_t)__builtin_amdgcn_readlane(r, 16)),
               max((uint32_t)__builtin_amdgcn_readlane(r, 32), (uint32_t)__builtin_amdgcn_readlane(r, 48)));
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT)
token_logprobs_kernel(const T *__restrict__ logits, ScoreCall c)
{
    constexpr int NW = NT / 64, STEP = NT * 8, PER = 4, G = NT / 64;    // PER vectors of eight logits at a time; G lanes of a group
    __shared__ float wave_m[NW], wave_z[NW], wave_e[NW];
    __shared__ __align__(16) unsigned long long listed[kScoreList + 2];  // key of the logit, behind it its index upside down
    __shared__ uint32_t group[64], bound_s, found_key[NW];
    __shared__ int n_list, found_at[NW];
    const int64_t row = work_group();
    if (row >= c.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), V = c.V, k = c.k;
    const T *L = logits + row * c.ld;
    const int token = c.token ? c.token[row] : -1;
    const bool given = token >= 0 && token < V;
    float t = c.temperature ? c.temperature[row] : 1.0f;
    t = t > 0.0f ? fminf(fmaxf(t, 1e-30f), 1e30f) : 1.0f;
    const float inv = 1.0f / t, inv2 = inv * 1.44269504088896340736f;
    float l_given = given ? (float)L[token] : 0.0f;
    if (l_given != l_given) l_given = -INFINITY;

    // eight logits from `at` on (NaN among them), -infinity behind the row
    auto values = [&](const Raw8<T> &raw, int at, float (&v)[8]) __attribute__((always_inline)) {
        raw8_values(raw, v);
        if (__ballot(at + 8 > V)) {
            if (V >= 8) {
                const int late = at + 8 - V;
#pragma unroll
                for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (late > 0 && (late & s)) v[i] = i + s < 8 ? v[i + s] : 0.0f;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at + i < V ? v[i] : -INFINITY;
        }
    };
    // The largest of eight, -infinity of none but NaN.  (Written out, as three at a time; the compiler would quiet each value first.  Of a NaN
    // that signals the instruction makes a quiet one, which the next instruction drops with all that went into it: each one's result is
    // looked at.)
    auto largest = [](const float (&v)[8]) __attribute__((always_inline)) {
        float a, b, d, m;
        asm("v_max3_f32 %0, %1, %2, %3" : "=v"(a) : "v"(v[0]), "v"(v[1]), "v"(v[2]));
        asm("v_max3_f32 %0, %1, %2, %3" : "=v"(b) : "v"(a), "v"(v[3]), "v"(v[4]));
        asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(b), "v"(v[5]), "v"(v[6]));
        asm("v_max_f32 %0, %1, %2" : "=v"(m) : "v"(d), "v"(v[7]));
        if (__builtin_isunordered(a, b) || __builtin_isunordered(d, m)) {
            m = -INFINITY;
#pragma unroll
            for (int i = 0; i < 8; ++i) m = v[i] > m ? v[i] : m;
        }
        return m;
    };
    ScoreSums s = {-INFINITY, 0.0f, 0.0f};
    // 32 logits join the thread's sums
    float tops[PER];                                 // the vectors' largest
    auto take = [&](const float (&v)[PER][8]) __attribute__((always_inline)) {
        float m = s.m;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            tops[j] = largest(v[j]);
            m = tops[j] > m ? tops[j] : m;
        }
        s = score_rescaled(s, m, inv);
        if (m == -INFINITY) return;
        if (m == INFINITY) {                         // leaves all others without weight
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) s.z += v[j][i] == INFINITY ? 1.0f : 0.0f;
            return;
        }
        float z[2] = {0.0f, 0.0f}, e[2] = {0.0f, 0.0f};
        const float at_m = m * inv2;
        if (fabsf(at_m) < 1e6f) {
            // One multiply-add to the logit's distance from the rounded product; what the rounding took is the same for all of them.
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = fminf(fmaf(v[j][i], -inv2, at_m), 1000.0f), w = __builtin_amdgcn_exp2f(-d);
                    z[i & 1] += w;
                    e[i & 1] = fmaf(w, d, e[i & 1]);
                }
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float d = fminf((m - v[j][i]) * inv2, 1000.0f), w = __builtin_amdgcn_exp2f(-d);
                    z[i & 1] += w;
                    e[i & 1] = fmaf(w, d, e[i & 1]);
                }
        }
        const float off = fabsf(at_m) < 1e6f ? fmaf(m, inv2, -at_m) : 0.0f, f = __builtin_amdgcn_exp2f(-off), zs = z[0] + z[1];
        s.z = fmaf(f, zs, s.z);
        s.e = fmaf(f * 0.69314718055994530942f, fmaf(off, zs, e[0] + e[1]), s.e);
    };
    // the k-th largest of the groups' largest, equal ones by number; -infinity is no alternative
    float least = INFINITY;
    auto bound = [&]() __attribute__((always_inline)) {
        uint32_t top = score_key(s.m);
        if constexpr (G > 1) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));
        if constexpr (G > 2) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
        if constexpr (G > 4) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xF, 0xF, true));
        if constexpr (G > 8) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x140, 0xF, 0xF, true));
        if (lane % G == 0) group[tid / G] = top;
        if (tid == 0) n_list = 0;
        __syncthreads();
        if (wave == 0) {
            const uint32_t mine = group[lane];
            int before = 0;
#pragma unroll
            for (int j = 0; j < 64; ++j) {
                const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)mine, j);
                before += o > mine || (o == mine && j < lane);
            }
            if (before == k - 1) bound_s = max(mine, score_key(-INFINITY) + 1);
        }
        __syncthreads();
        least = score_value(bound_s);
    };
    auto list = [&](const float (&v)[8], float top, int at) __attribute__((always_inline)) {
        if (top >= least) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (v[i] >= least) {
                    const int to = atomicAdd(&n_list, 1);
                    if (to < kScoreList) listed[to] = (unsigned long long)score_key(v[i]) << 32 | (uint32_t)~(at + i);
                }
        }
    };
    auto fetch = [&](Raw8<T> (&raw)[PER], int at) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < PER; ++j) raw[j] = raw8(L, at + j * STEP, V);
    };
    auto widen = [&](const Raw8<T> (&raw)[PER], int at, float (&v)[PER][8]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < PER; ++j) values(raw[j], at + j * STEP, v[j]);
    };
    const int mine = tid * 8, ours = mine - lane * 8;                   // a thread's, its wavefront's first logit
    {
        Raw8<T> raw[PER], next[PER];
        float v[PER][8];
        fetch(raw, mine);
        if (ours + PER * STEP < V) fetch(next, mine + PER * STEP);
        widen(raw, mine, v);
        take(v);
        if (k > 0) {
            bound();
#pragma unroll
            for (int j = 0; j < PER; ++j) list(v[j], tops[j], mine + j * STEP);
        }
        for (int at = PER * STEP; ours + at < V; at += PER * STEP) {
#pragma unroll
            for (int j = 0; j < PER; ++j) raw[j] = next[j];
            if (ours + at + PER * STEP < V) fetch(next, mine + at + PER * STEP);
            widen(raw, mine + at, v);
            take(v);
            if (k > 0) {
#pragma unroll
                for (int j = 0; j < PER; ++j) list(v[j], tops[j], mine + at + j * STEP);
            }
        }
    }
    // the row's largest, then the sums relative to it
    const float own_m = s.m;
    {
        const float top = score_value(score_wave_max(score_key(s.m)));
        if (lane == 0) wave_m[wave] = top;
        __syncthreads();
        float m = wave_m[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, wave_m[w]);
        s = score_rescaled(s, m, inv);
        s.z = wave_sum(s.z);
        s.e = wave_sum(s.e);
        if constexpr (NW > 1) {
            if (lane == 0) {
                wave_z[wave] = s.z;
                wave_e[wave] = s.e;
            }
            __syncthreads();
            s.z = s.e = 0.0f;
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                s.z += wave_z[w];
                s.e += wave_e[w];
            }
        }
    }
    const float log_z = logf(s.z);                   // (a row of -infinity: z is 0)
    auto logprob = [&](float l) {
        if (l == -INFINITY || s.z == 0.0f) return -INFINITY;
        return (l == s.m ? 0.0f : (0.5f * l - 0.5f * s.m) * (2.0f * inv)) - log_z;   // (l - m may leave fp32's range)
    };
    if (tid == 0) {
        if (c.logprob) c.logprob[row] = given ? logprob(l_given) : 0.0f;
        if (c.entropy) c.entropy[row] = s.z > 0.0f ? log_z + s.e / s.z : 0.0f;
    }
    if (k == 0) return;

    int n = n_list;
    if (n > kScoreList) {
        __syncthreads();                             // (all have read it)
        const ScoreSums whole = s;
        s.m = own_m;
        bound();
        s = whole;
        for (int at = 0; ours + at < V; at += STEP) {
            float v[8];
            values(raw8(L, mine + at, V), mine + at, v);
            list(v, largest(v), mine + at);
        }
        __syncthreads();
        n = n_list;
    }
    float *const top_logprob = c.top_logprob + row * k;
    int32_t *const top_token = c.top_token + row * k;
    if (n <= kScoreList) {
        if (tid < 2) listed[n + tid] = 0;            // (behind the last, for the reads in pairs)
        __syncthreads();
        typedef __attribute__((ext_vector_type(2))) unsigned long long pair;
        for (int i = tid; i < n; i += NT) {
            const unsigned long long own = listed[i];
            int before = 0;
#pragma unroll 4
            for (int j = 0; j < n; j += 2) {
                const pair o = *reinterpret_cast<const pair *>(listed + j);
                before += (int)(o[0] > own) + (int)(o[1] > own);
            }
            if (before < k) {
                top_token[before] = (int)~(uint32_t)own;
                top_logprob[before] = logprob(score_value((uint32_t)(own >> 32)));
            }
        }
        for (int i = n + tid; i < k; i += NT) {
            top_token[i] = -1;
            top_logprob[i] = -INFINITY;
        }
        return;
    }
    // one after the other: the best logit behind the last one found
    uint32_t last_key = 0xffffffffu;
    int last_at = -1;
    for (int i = 0; i < k; ++i) {
        uint32_t key = 0;
        int where = V;
        for (int at = 0; ours + at < V; at += STEP) {
            float v[8];
            values(raw8(L, mine + at, V), mine + at, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const int index = mine + at + q;
                const uint32_t u = score_key(fmaxf(v[q], -INFINITY));
                const bool behind = u < last_key || (u == last_key && index > last_at);
                if (index < V && behind && (u > key || (u == key && index < where))) { key = u; where = index; }
            }
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t u = (uint32_t)__shfl_xor((int)key, off);
            const int w = __shfl_xor(where, off);
            if (u > key || (u == key && w < where)) { key = u; where = w; }
        }
        __syncthreads();
        if (lane == 0) { found_key[wave] = key; found_at[wave] = where; }
        __syncthreads();
        for (int w = 0; w < NW; ++w)
            if (found_key[w] > key || (found_key[w] == key && found_at[w] < where)) { key = found_key[w]; where = found_at[w]; }
        last_key = key;
        last_at = where;
        if (tid == 0) {
            top_token[i] = where;                    // (there are more than kScoreList finite ones)
            top_logprob[i] = logprob(score_value(key));
        }
    }
}
