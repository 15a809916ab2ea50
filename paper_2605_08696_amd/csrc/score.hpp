// Log probabilities of given tokens, the entropy of each row of logits and its most likely tokens, in one reading of the row and a second
// one from the caches.
//
// With m the largest logit, d = (m - l) / T >= 0 and w = e^-d:
//   Z = sum w      log p(v) = -d_v - log Z      entropy = log Z + (sum w d) / Z
// (both parts of the entropy are positive: nothing cancels).  A thread keeps its largest logit and the two sums relative to it, 32 logits at
// a time, and rescales them when a larger one comes; the threads' sums are joined in a fixed order.
//
// The k most likely tokens: the k-th largest of 64 disjoint groups' largest logits is at or below the k-th largest of the row, so the
// logits from it on (some 1.3 k of them where the groups are alike) hold all that are wanted; the second reading lists them, and they are
// put in order by counting, equal ones by their index.  A list that overflows (equal logits in bulk) is not used: the tokens are then looked
// for one after the other, a reading each.
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
__device__ __forceinline__ ScoreSums score_join(const ScoreSums &a, const ScoreSums &b, float inv)
{
    const float m = fmaxf(a.m, b.m);
    const ScoreSums x = score_rescaled(a, m, inv), y = score_rescaled(b, m, inv);
    return {m, x.z + y.z, x.e + y.e};
}

template <typename T, int NT>
__global__ void __launch_bounds__(NT)
token_logprobs_kernel(const T *__restrict__ logits, ScoreCall c)
{
    constexpr int NW = NT / 64, STEP = NT * 8;
    __shared__ ScoreSums sums[NW];
    __shared__ uint32_t group[64], list_key[kScoreList], bound_s, found_key[NW];
    __shared__ int list_at[kScoreList], n_list, found_at[NW];
    const int64_t row = work_group();
    if (row >= c.rows) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, V = c.V;
    const T *L = logits + row * c.ld;
    const int token = c.token ? c.token[row] : -1;
    const bool given = token >= 0 && token < V;
    float t = c.temperature ? c.temperature[row] : 1.0f;
    t = t > 0.0f ? fminf(fmaxf(t, 1e-30f), 1e30f) : 1.0f;
    const float inv = 1.0f / t;
    float l_given = given ? (float)L[token] : 0.0f;
    if (l_given != l_given) l_given = -INFINITY;

    // eight logits from `at` on; a NaN, or what lies behind the row, counts as -infinity
    auto values = [&](const Raw8<T> &raw, int at, float (&v)[8]) {
        widen8(raw, at, V, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaxf(v[i], -INFINITY);
        if (__ballot(at + 8 > V)) {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at + i < V ? v[i] : -INFINITY;
        }
    };
    ScoreSums s = {-INFINITY, 0.0f, 0.0f};
    bool hot = false;                                // an infinite logit leaves all others without weight
    for (int at = tid * 8; at - lane * 8 < V; at += STEP * 4) {
        Raw8<T> raw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[j] = raw8(L, at + j * STEP, V);
        float v[4][8], m = s.m;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            values(raw[j], at + j * STEP, v[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) m = fmaxf(m, v[j][i]);
        }
        s = score_rescaled(s, m, inv);
        if (m == INFINITY || m == -INFINITY) {
            if (m == INFINITY) {
                if (!hot) s.z = s.e = 0.0f;
                hot = true;
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) s.z += v[j][i] == INFINITY ? 1.0f : 0.0f;
            }
            continue;
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float d = (m - v[j][i]) * inv, w = score_weight(d);
                s.z += w;
                s.e = w > 0.0f ? fmaf(w, d, s.e) : s.e;
            }
    }
    // the largest of each group of NT / 64 threads, then the sums of all
    {
        const uint32_t mine = score_key(s.m);
        uint32_t top = mine;
        constexpr int G = NT / 64;                   // lanes of a group: 4, 8 or 16
        if constexpr (G > 1) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0xB1, 0xF, 0xF, true));
        if constexpr (G > 2) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x4E, 0xF, 0xF, true));
        if constexpr (G > 4) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x141, 0xF, 0xF, true));
        if constexpr (G > 8) top = max(top, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)top, 0x140, 0xF, 0xF, true));
        if (lane % G == 0) group[tid / G] = top;
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const ScoreSums o = {__shfl_xor(s.m, off), __shfl_xor(s.z, off), __shfl_xor(s.e, off)};
        s = score_join(s, o, inv);
    }
    if (lane == 0) sums[wave] = s;
    if (tid == 0) n_list = 0;
    __syncthreads();
    s = sums[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) s = score_join(s, sums[w], inv);
    const float log_z = logf(s.z);                   // (a row of -infinity: z is 0)
    auto logprob = [&](float l) {
        if (l == -INFINITY || s.z == 0.0f) return -INFINITY;
        return (l == s.m ? 0.0f : (0.5f * l - 0.5f * s.m) * (2.0f * inv)) - log_z;   // (l - m may leave fp32's range)
    };
    if (tid == 0) {
        if (c.logprob) c.logprob[row] = given ? logprob(l_given) : 0.0f;
        if (c.entropy) c.entropy[row] = s.z > 0.0f ? log_z + s.e / s.z : 0.0f;
    }
    if (c.k == 0) return;

    if (wave == 0) {                                 // the k-th largest of the groups', equal ones by number
        const uint32_t mine = group[lane];
        int before = 0;
#pragma unroll
        for (int j = 0; j < 64; ++j) {
            const uint32_t o = (uint32_t)__builtin_amdgcn_readlane((int)mine, j);
            before += o > mine || (o == mine && j < lane);
        }
        if (before == c.k - 1) bound_s = mine;
    }
    __syncthreads();
    // (-infinity is no alternative)
    const uint32_t bound = max(bound_s, score_key(-INFINITY) + 1);
    const float least = score_value(bound);
    for (int at = tid * 8; at - lane * 8 < V; at += STEP * 4) {
        Raw8<T> raw[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) raw[j] = raw8(L, at + j * STEP, V);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float v[8];
            values(raw[j], at + j * STEP, v);
            float m = v[0];
#pragma unroll
            for (int i = 1; i < 8; ++i) m = fmaxf(m, v[i]);
            if (m >= least) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (v[i] >= least) {
                        const int to = atomicAdd(&n_list, 1);
                        if (to < kScoreList) {
                            list_key[to] = score_key(v[i]);
                            list_at[to] = at + j * STEP + i;
                        }
                    }
            }
        }
    }
    __syncthreads();
    const int n = n_list;
    float *const top_logprob = c.top_logprob + row * c.k;
    int32_t *const top_token = c.top_token + row * c.k;
    if (n <= kScoreList) {
        for (int i = tid; i < n; i += NT) {
            const uint32_t key = list_key[i];
            const int at = list_at[i];
            int before = 0;
            for (int j = 0; j < n; ++j) before += list_key[j] > key || (list_key[j] == key && list_at[j] < at);
            if (before < c.k) {
                top_token[before] = at;
                top_logprob[before] = logprob(score_value(key));
            }
        }
        for (int i = n + tid; i < c.k; i += NT) {
            top_token[i] = -1;
            top_logprob[i] = -INFINITY;
        }
        return;
    }
    // one after the other: the best logit behind the last one found
    uint32_t last_key = 0xffffffffu;
    int last_at = -1;
    for (int i = 0; i < c.k; ++i) {
        uint32_t key = 0;
        int where = V;
        for (int at = tid * 8; at - lane * 8 < V; at += STEP) {
            float v[8];
            values(raw8(L, at, V), at, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const uint32_t k = score_key(v[q]);
                const bool behind = k < last_key || (k == last_key && at + q > last_at);
                if (at + q < V && behind && (k > key || (k == key && at + q < where))) { key = k; where = at + q; }
            }
        }
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
            const uint32_t k = (uint32_t)__shfl_xor((int)key, off);
            const int w = __shfl_xor(where, off);
            if (k > key || (k == key && w < where)) { key = k; where = w; }
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
