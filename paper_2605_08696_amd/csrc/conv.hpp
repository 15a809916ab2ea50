// The short causal convolution of packed sequences, each channel by itself:
//   out[t, c] = act(bias[c] + sum_k w[c, k] x[t - (W - 1) + k, c])
// A slot keeps the last W rows of x, position p in row p % W: a single token then overwrites the one row that none of its taps reads, which
// lets the kernel of single tokens read and write the ring without an order among its work-groups.
//
// A thread takes eight channels of R consecutive tokens: R + W - 1 loads without a branch between them, then the products from registers.
// What bounds it is memory: x is read once (the W - 1 rows in front of a run come from the caches) and out written once.
#pragma once
#include "fp8.hpp"
#include "packed.hpp"

constexpr int kConvTaps = 8;                         // the widest filter

struct ConvCall {
    Packed seqs;
    int64_t ldx, ld_out;
    const float *weight, *bias;
    int channels, units, per_run, silu;              // units of eight channels; lanes that share a run of tokens (a power of two)
    int64_t runs;
    void *ring;
};

__device__ __forceinline__ float silu(float v) { return v * __builtin_amdgcn_rcpf(1.0f + __expf(-v)); }

template <typename T>
__device__ __forceinline__ void store_part(T *p, int n, const float (&v)[8])
{
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = v[i];
    store8(p, n, w);
}

template <typename T, int W, int R>
__global__ void __launch_bounds__(256)
causal_conv_kernel(const T *__restrict__ x, T *__restrict__ out, ConvCall c)
{
    const int lane = threadIdx.x & 63;
    const int64_t wave = (int64_t)work_group() * 4 + (threadIdx.x >> 6);
    // a wavefront: 64 units of one run, or, of few channels, several runs
    const int groups = c.units > 64 ? (c.units + 63) >> 6 : 1, shift = __builtin_ctz(c.per_run);
    const int64_t run = wave / groups * (64 >> shift) + (c.units > 64 ? 0 : lane >> shift);
    const int unit = (int)(wave % groups) * 64 + (lane & (c.per_run - 1)), col = unit * 8, C = c.channels;
    const bool there = run < c.runs && unit < c.units;
    if (!__ballot(there)) return;
    const int t0 = there ? c.seqs.lo + (int)(run * R) : c.seqs.lo, n_cols = min(8, C - col);

    float w[W][8], b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int ch = min(max(col, 0) + i, C - 1);
        b[i] = c.bias ? c.bias[ch] : 0.0f;
#pragma unroll
        for (int k = 0; k < W; ++k) w[k][i] = c.weight[(int64_t)ch * W + k];
    }
    // this lane's sequence: by all lanes together where they share a run or few sequences do, else by halves
    int n = 0;
    if (c.seqs.n > 1) {
        if (c.units > 64 || c.per_run == 64) {
            n = packed_find(c.seqs, __builtin_amdgcn_readfirstlane(t0), lane);
        } else {
            int lo = 0, hi = c.seqs.n;               // the last n in [lo, hi) that begins at or before t0
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (c.seqs.offsets[mid] <= t0) lo = mid;
                else hi = mid;
            }
            n = lo;
        }
    }
    if (!there) return;
    auto load = [&](const T *row, float (&v)[8]) {
        raw8_values(raw8(row, col, C), v);
        const int late = C >= 8 ? col + 8 - C : 0;   // the row's last eight: moved to their places
        if (late > 0) {
#pragma unroll
            for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (late & s) v[i] = i + s < 8 ? v[i + s] : 0.0f;
        }
    };
    auto row_of = [&](int t) { return x + (int64_t)t * c.ldx; };
    auto put = [&](int t, float (&acc)[8]) {
        if (c.silu) {
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[i] = silu(acc[i]);
        }
        store_part(out + (int64_t)t * c.ld_out + col, n_cols, acc);
    };

    Sequence s = packed_sequence(c.seqs, n);
    const int t1 = min(t0 + R, c.seqs.hi);
    if (t0 - max(W - 1, 1) >= s.begin && t0 + R <= s.end && s.pos >= 0) {
        // the run and the rows in front of it lie in one sequence
        Raw8<T> raw[R + W - 1];
#pragma unroll
        for (int j = 0; j < R + W - 1; ++j) raw[j] = raw8(row_of(t0 - (W - 1) + j), col, C);
        float v[W][8];
        auto values = [&](int j, float (&to)[8]) {
            raw8_values(raw[j], to);
            const int late = C >= 8 ? col + 8 - C : 0;
            if (late > 0) {
#pragma unroll
                for (int sh = 4; sh >= 1; sh >>= 1)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        if (late & sh) to[i] = i + sh < 8 ? to[i + sh] : 0.0f;
            }
        };
#pragma unroll
        for (int j = 0; j < W - 1; ++j) values(j, v[j]);
#pragma unroll
        for (int j = 0; j < R; ++j) {
            values(W - 1 + j, v[(W - 1 + j) % W]);
            float acc[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                acc[i] = b[i];
#pragma unroll
                for (int k = 0; k < W; ++k) acc[i] = fmaf(w[k][i], v[(j + k) % W][i], acc[i]);
            }
            put(t0 + j, acc);
        }
        return;
    }
    // A sequence begins or ends here.  The W - 1 first tokens of a sequence, whose taps reach into the slot's ring, belong to the run that
    // holds the first of them, in which the same thread writes the ring behind them.
    T *const ring_all = static_cast<T *>(c.ring);
    for (int t = t0; t < t1;) {
        while (t >= s.end && n + 1 < c.seqs.n) s = packed_sequence(c.seqs, ++n);
        if (t >= s.end) break;                       // (offsets that are not the host's)
        const bool starts = t == s.begin;
        if (!starts && t - s.begin < W - 1 && s.begin < t0) { ++t; continue; }
        T *ring = s.slot >= 0 && ring_all ? ring_all + s.slot * W * C : nullptr;
        const int until = starts && W > 2 ? min(s.end, s.begin + W - 1) : t + 1;
        for (int u = t; u < until; ++u) {
            float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (s.pos >= 0) {
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[i] = b[i];
#pragma unroll
                for (int k = 0; k < W; ++k) {
                    const int at = u - (W - 1) + k;
                    const int64_t p = (int64_t)s.pos + at - s.begin;
                    float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
                    if (at >= s.begin) load(row_of(at), v);
                    else if (p >= 0 && ring) load(ring + p % W * C, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) acc[i] = fmaf(w[k][i], v[i], acc[i]);
                }
                put(u, acc);
            } else {
                store_part(out + (int64_t)u * c.ld_out + col, n_cols, acc);
            }
        }
        if (starts && ring && s.pos >= 0)
            for (int u = max(s.begin, s.end - W); u < s.end; ++u) {
                const int64_t p = (int64_t)s.pos + u - s.begin;
                float v[8];
                load(row_of(u), v);
                store_part(ring + p % W * C + col, n_cols, v);
            }
        t = until;
    }
}
