// The short causal convolution of packed sequences, each channel by itself:
//   out[t, c] = act(bias[c] + sum_k w[c, k] x[t - (W - 1) + k, c])
// A slot keeps the last W rows of x, position p in row p % W: a single token then overwrites the one row that none of its taps reads, which
// lets the kernel of single tokens read and write the ring without an order among its work-groups.
//
// A thread takes eight channels of a run of tokens, R tokens at a time: their rows' loads are in flight together, without a branch
// between them, while the R in front of them are worked on, and the filter's W - 1 rows in front of a row stay in registers.  A sequence
// that begins inside a run is a piece of its own; its first W - 1 tokens, whose taps reach into the slot's ring, all belong to the run that
// holds the first of them, in which the same thread writes the ring behind them.
// What bounds it: memory, x read once, out written once, and the way it is walked, a kilobyte of each of eight rows at a time: of 32768 x 4352
// bf16 one tap without an activation takes 119 us (torch's copy 106, a copy in one stream of addresses 92), three more taps 9, the activation
// 4; vector instructions issue for a fifth of the time.  With four taps 133 us, 571 MB at 4.3 TB/s, fp32 16384 x 4352 129 us, 4.4 TB/s (124
// with the activation of bf16 outputs); 37 x 2304, which is a launch and three trips to memory, 6.3.  With runs of eight tokens, each of
// which reads its filter, and branches around the loads at a sequence's begin: 193 and 15.
#pragma once
#include "fp8.hpp"
#include "packed.hpp"

constexpr int kConvTaps = 8;                         // the widest filter

struct ConvCall {
    Packed seqs;
    int64_t ldx, ld_out;
    const float *weight, *bias;
    int channels, units, per_run, silu, run;         // units of eight channels; lanes that share a run (a power of two), tokens of a run
    int64_t runs;
    void *ring;
};

// e^-w for w >= 0, to an ulp: its argument in steps of a factor of two keeps what its product is rounded by, which the fast exponential drops
// (w 2^-24 of the value).  Below 2^-126 it is 0.
__device__ __forceinline__ float exp_minus(float w)
{
    w = fminf(w, 104.0f);                            // (a NaN's as well: what uses it keeps the NaN by another way)
    const float at = w * -1.44269504f, left = fmaf(w, -1.92596299e-8f, fmaf(w, -1.44269504f, -at)), e = __builtin_amdgcn_exp2f(at);
    return fmaf(e, left * 0.69314718f, e);
}
// v / (1 + e^-v) to a few ulp; what is below 2^-119 may be 0.  For values that stay in fp32.
__device__ __forceinline__ float silu_f32(float v)
{
    const float u = exp_minus(fabsf(v)), d = 1.0f + u, r0 = __builtin_amdgcn_rcpf(d), r = fmaf(fmaf(-d, r0, 1.0f), r0, r0);
    return (v < 0.0f ? v * u : v) * r;
}
// ... as an output of type T: five instructions and (|v| + 4) 2^-24 of the value for what is rounded to bf16 (2^-9 of it).
template <typename T>
__device__ __forceinline__ float silu(float v)
{
    if constexpr (sizeof(T) == 4) return silu_f32(v);
    return v * __builtin_amdgcn_rcpf(1.0f + __expf(-v));
}

template <typename T, int W, int R>
__global__ void __launch_bounds__(256)
causal_conv_kernel(const T *__restrict__ x, T *__restrict__ out, ConvCall c)
{
    constexpr int HIST = W > 1 ? W - 1 : 1;
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)work_group() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // a wavefront: 64 units of one run, or, of few channels, several runs
    const int groups = c.units > 64 ? (c.units + 63) >> 6 : 1, shift = __builtin_ctz(c.per_run);
    const int64_t run0 = wave / groups * (64 >> shift), run = run0 + (lane >> shift);
    const int unit = (int)(wave % groups) * 64 + (lane & (c.per_run - 1)), col = unit * 8, C = c.channels;
    if (run0 >= c.runs) return;
    const bool there = run < c.runs && unit < c.units;
    const int t0 = c.seqs.lo + (int)min(run, c.runs - 1) * c.run, t1 = min(t0 + c.run, c.seqs.hi), n_cols = min(8, C - col);

    float w[W][8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ch = min(col + i, C - 1);
        b[i] = c.bias ? c.bias[ch] : 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = c.weight[(int64_t)ch * W + k];
    }
    // this lane's sequence: between those of the wavefront's first and last run
    int n = 0;
    if (c.seqs.n > 1) {
        const int first = __builtin_amdgcn_readfirstlane(t0), last = __builtin_amdgcn_readlane(t0, 63);
        n = packed_find(c.seqs, first, lane);
        if (last != first) {
            int up = packed_find(c.seqs, last, lane) + 1;
            while (up - n > 1) {
                const int mid = (n + up) >> 1;
                if (c.seqs.offsets[mid] <= t0) n = mid;
                else up = mid;
            }
        }
    }
    if (!there) return;
    const int late = C >= 8 ? max(col + 8 - C, 0) : 0;                  // the row's last eight are moved to their places
    auto values = [&](const Raw8<T> &raw, float (&v)[8]) {
        raw8_values(raw, v);
        if (late > 0) {
#pragma unroll
            for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (late & s) v[i] = i + s < 8 ? v[i + s] : 0.0f;
        }
    };
    auto put = [&](int t, float (&v)[8]) {
        T *to = out + (int64_t)t * c.ld_out + col;
        store8(to, n_cols, v);
    };
    auto row_of = [&](int t) { return x + (int64_t)t * c.ldx; };

    for (int t = t0; t < t1;) {
        Sequence s = packed_sequence(c.seqs, n);
        while (t >= s.end && n + 1 < c.seqs.n) s = packed_sequence(c.seqs, ++n);
        if (t >= s.end) break;                       // (offsets that are not the host's)
        int u = t, until = min(s.end, t1);
        if (s.begin < t0 && t - s.begin < W - 1) u = min(until, s.begin + W - 1);      // an earlier run's
        const bool starts = u == s.begin;
        if (starts) until = max(until, min(s.end, s.begin + W - 1));
        t = max(until, t + 1);
        if (u >= until) continue;
        if (s.pos < 0) {
            for (; u < until; ++u) {
                float zero[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                put(u, zero);
            }
            continue;
        }
        T *ring = s.slot >= 0 && c.ring ? static_cast<T *>(c.ring) + s.slot * W * C : nullptr;
        Raw8<T> next[R], hist[HIST];
        bool none[HIST];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            const int at = u - (W - 1) + j;
            const int64_t p = (int64_t)s.pos + at - s.begin;
            const bool old = at < s.begin;
            none[j] = old && (p < 0 || !ring);
            hist[j] = raw8(!old ? row_of(at) : none[j] ? row_of(u) : ring + p % W * C, col, C);
        }
#pragma unroll
        for (int j = 0; j < R; ++j) next[j] = raw8(row_of(min(u + j, until - 1)), col, C);
        float v[W][8];
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            values(hist[j], v[j]);
            if (none[j]) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[j][i] = 0.0f;
            }
        }
        if (starts && ring) {
            Raw8<T> last[W];
#pragma unroll
            for (int j = 0; j < W; ++j) last[j] = raw8(row_of(max(s.end - W + j, s.begin)), col, C);
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const int e = s.end - W + j;
                float q[8];
                values(last[j], q);
                if (e >= s.begin) store8(ring + ((int64_t)s.pos + e - s.begin) % W * C + col, n_cols, q);
            }
        }
        for (; u < until; u += R) {
            Raw8<T> now[R];
#pragma unroll
            for (int j = 0; j < R; ++j) now[j] = next[j];
            if (u + R < until) {
#pragma unroll
                for (int j = 0; j < R; ++j) next[j] = raw8(row_of(min(u + R + j, until - 1)), col, C);
            }
#pragma unroll
            for (int j = 0; j < R; ++j) {
                values(now[j], v[(W - 1 + j) % W]);
                float acc[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    acc[i] = b[i];
#pragma unroll
                    for (int k = 0; k < W; ++k) acc[i] = fmaf(w[k][i], v[(j + k) % W][i], acc[i]);
                }
                if (c.silu) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] = silu<T>(acc[i]);
                }
                if (u + j < until) put(u + j, acc);
            }
            if constexpr (R % W != 0) {              // the window begins at its first row again
                float q[HIST][8];
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) q[j][i] = v[(R + j) % W][i];
#pragma unroll
                for (int j = 0; j < W - 1; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[j][i] = q[j][i];
            }
        }
    }
}
