// The selective recurrence: for each head a matrix of state S [P][N] whose decay and input depend on the token,
//   dt = softplus(dt_raw + dt_bias[h])     S <- exp(dt A[h]) S + dt x[h] B[g]^T     y = S C[g] + D[h] x[h]     out = y silu(z)
// with x [H][P] | B [G][N] | C [G][N] in a row and g = h / (H / G).  Here: what its kernels share, the kernel for operands in fp32,
// and the kernel of single tokens.
//
// Work over time.  A work-group takes one head (a part of its P rows) of one sequence from its first token to its last, the state in
// registers.  Where there are too few of those, the packed tokens are cut into segments of equal length, whatever sequences they hold:
// a first pass leaves, for each segment that a sequence runs on from, the state at its end that the segment itself brings (`carry`) and
// the factor by which it decays what came before (`decay`); a second one makes of these the states at the segments' ends; the third starts
// each segment from the one in front of it and writes the outputs.  (Joined by the third pass itself, every segment adding up all carries in
// front of it, 16384 tokens of 32 heads took 146 us where this took 115.)
#pragma once
#include "conv.hpp"
#include "tile.hpp"

#define SCAN_INLINE __attribute__((always_inline))

struct StepSizes {                                   // dt_raw [tokens][H] and what dt is made of
    const void *raw;
    int64_t ld;
    const float *bias;
    int is_bf16, softplus;
};
struct ScanCall {
    Packed seqs;
    StepSizes dt;
    int64_t ld, ld_z, ld_out;                        // of x | B | C, z, out
    const void *z;
    const float *a, *skip;
    int H, P, G, N;
    int chunks;                                      // eight divides N and P
    float *state;                                    // [slots][H][P][N]
    int seg, parts;                                  // tokens of a segment; parts of a head's P rows
    float *carry, *held, *decay;                     // [segments][H][P][N] twice, [segments][H]
};
// Work-groups are dealt to the eight XCDs in turn, each with an L2 of its own.  Runs of kScanRun heads, which share B and C or whose rows
// lie side by side, go to one of them.  (The last runs may lie behind the last head: their `work` is behind the last sequence or segment.)
constexpr int kScanRun = 8;
__device__ __forceinline__ int64_t scan_unit()
{
    const uint32_t id = work_group(), j = id >> 3;
    return (int64_t)(j / kScanRun * 8 + (id & 7)) * kScanRun + j % kScanRun;
}
enum { SCAN_WHOLE = 0, SCAN_CARRY = 1, SCAN_SEGMENTS = 2 };

__device__ __forceinline__ float dt_raw(const StepSizes &c, int64_t t, int h)
{
    const int64_t at = t * c.ld + h;
    return c.is_bf16 ? (float)static_cast<const bf16 *>(c.raw)[at] : static_cast<const float *>(c.raw)[at];
}
__device__ __forceinline__ float dt_of(const StepSizes &c, float raw, float bias)
{
    const float v = raw + bias;
    if (!c.softplus) return v;
    // log(1 + e^v) = max(v, 0) + log(1 + u), u = e^-|v|, to an ulp or two and in few registers, which the scans' widest forms do not have for
    // expf and log1pf.  The logarithm without the sum 1 + u, which would drop digits of u (2^-24 of a dt of 0.06): twice the area tangent of
    // s = u / (2 + u), at most a third, by its series s (1 + s^2 / 3 + s^4 / 5 ..), whose first term left out is below 2^-29 of the sum.
    // (A dt below 2^-126 is 0.  A NaN stays one.)
    const float u = exp_minus(fabsf(v)), d = 2.0f + u, r = __builtin_amdgcn_rcpf(d), s0 = u * r, s = fmaf(fmaf(-d, s0, u), r, s0), q = s * s;
    float p = 1.0f / 15.0f;
    p = fmaf(p, q, 1.0f / 13.0f);
    p = fmaf(p, q, 1.0f / 11.0f);
    p = fmaf(p, q, 1.0f / 9.0f);
    p = fmaf(p, q, 1.0f / 7.0f);
    p = fmaf(p, q, 0.2f);
    p = fmaf(p, q, 1.0f / 3.0f);
    return (v > 0.0f ? v : v == v ? 0.0f : v) + 2.0f * fmaf(p * q, s, s);
}
// The decay's exponent in steps of a factor of two, in 64 bits: rounded to fp32, an exponent of -100 would lose 4e-6 of its decay, and a sum of
// exponents what is behind a few large ones.  2^-200 is 0 in fp32 as every smaller decay is; the limit keeps sums of exponents in the range
// of which 64 bits hold all that matters.  (Formed of products in fp32 with what they are rounded by: constants of 64 bits cost registers.
// A comparison, so that a NaN stays one.)
__device__ __forceinline__ double decay_exponent(float dt, float a)
{
    const float p = dt * a, high = p * 1.44269504f;
    const float low = fmaf(fmaf(dt, a, -p), 1.44269504f, fmaf(p, 1.92596299e-8f, fmaf(p, 1.44269504f, -high)));
    return high < -200.0f ? -200.0 : (double)high + (double)low;
}
// 2^(high + low) of an exponent in two parts, low what fp32 leaves of it.
__device__ __forceinline__ float exp2_of(float high, float low)
{
    const float f = __builtin_amdgcn_exp2f(high);
    return fmaf(f, low * 0.69314718f, f);
}
__device__ __forceinline__ float exp2_of(double e)
{
    const float high = (float)e;
    return exp2_of(high, (float)(e - high));
}

// Sum over groups of NL neighbouring lanes, in every lane of a group.
template <int NL>
__device__ __forceinline__ float lanes_sum(float v)
{
    auto step = [](float x, int moved) { return x + __builtin_bit_cast(float, moved); };
    if constexpr (NL > 1) v = step(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));
    if constexpr (NL > 2) v = step(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
    if constexpr (NL > 4) v = step(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x141, 0xF, 0xF, true));
    if constexpr (NL > 8) v = step(v, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x140, 0xF, 0xF, true));
    return v;
}

// What a work-group does over time, whatever its kernel: `work` is a sequence or a segment; clear, load(from) and store(to) act on the
// state that it holds of a head's part (whose first element lies at head_at in a slot), run(t0, t1, sum) takes
// it over tokens of one sequence and adds their decay exponents to sum, zeros(t0, t1) writes an idle sequence's output.
template <int MODE, typename Clear, typename Load, typename Store, typename Run, typename Zeros>
__device__ __forceinline__ void scan_drive(const ScanCall &c, int64_t work, int h, int p0, int64_t head_at, int lane, Clear &&clear, Load &&load,
                                           Store &&store, Run &&run, Zeros &&zeros)
{
    const int64_t slot_size = (int64_t)c.H * c.P * c.N;
    auto slot_of = [&](const Sequence &s) { return c.state + s.slot * slot_size + head_at; };
    double sum = 0.0;
    if constexpr (MODE == SCAN_WHOLE) {
        const Sequence s = packed_sequence(c.seqs, (int)work);
        if (s.begin == s.end) return;
        if (s.pos < 0) return zeros(s.begin, s.end);
        clear();
        if (s.slot >= 0 && s.pos > 0) load(slot_of(s));
        run(s.begin, s.end, sum);
        if (s.slot >= 0) store(slot_of(s));
    } else if constexpr (MODE == SCAN_CARRY) {
        const int t0 = c.seqs.lo + (int)work * c.seg, t1 = t0 + c.seg;
        if (t1 >= c.seqs.hi) return;
        const Sequence s = packed_sequence(c.seqs, packed_find(c.seqs, t1 - 1, lane));
        const Span span = packed_carried({s.begin, s.end}, t0, t1);
        if (span.begin == span.end || s.pos < 0) return;
        const int64_t at = work * slot_size + head_at;
        clear();
        if (s.begin >= t0 && s.slot >= 0 && s.pos > 0) {
            load(slot_of(s));
            store(c.held + at);                      // (the slot may be written before the second pass comes to read it)
        }
        run(span.begin, span.end, sum);
        store(c.carry + at);
        if (threadIdx.x == 0 && p0 == 0) c.decay[work * c.H + h] = s.begin >= t0 ? -1.0f : exp2_of(sum);
    } else {
        const int t0 = c.seqs.lo + (int)work * c.seg, t1 = min(t0 + c.seg, c.seqs.hi);
        auto get = [&](int n) SCAN_INLINE { return packed_sequence(c.seqs, n); };
        packed_pieces(t0, t1, packed_find(c.seqs, t0, lane), c.seqs.n, get, [&](const Sequence &s, int t, int e) SCAN_INLINE {
            if (s.pos < 0) return zeros(t, e);
            clear();
            if (t <= s.begin) {
                if (s.slot >= 0 && s.pos > 0) load(s.end > t1 ? c.held + work * slot_size + head_at : slot_of(s));
            } else if (work > 0) {                   // (always, with the host's offsets)
                load(c.carry + (work - 1) * slot_size + head_at);
            }
            run(t, e, sum);
            if (e == s.end && s.slot >= 0) store(slot_of(s));
        });
    }
}

// The states at the segments' ends, in the carries' place, an element a thread.  (Decay -1: the sequence begins in the segment.  What a
// segment leaves from which no sequence runs on is not read.)
__global__ void __launch_bounds__(256)
selective_scan_join_kernel(float *__restrict__ carry, const float *__restrict__ decay, int segments, int H, int head_size)
{
    const int64_t slot_size = (int64_t)H * head_size, i = (int64_t)work_group() * 256 + threadIdx.x;
    if (i >= slot_size) return;
    const float *d = decay + i / head_size;
    float *at = carry + i, s = 0.0f;
    constexpr int AHEAD = 4;
    for (int k = 0; k < segments; k += AHEAD) {
        float v[AHEAD], f[AHEAD];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int64_t q = min(k + j, segments - 1);
            v[j] = at[q * slot_size];
            f[j] = d[q * H];
        }
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            s = f[j] < 0.0f ? v[j] : fmaf(f[j], s, v[j]);
            if (k + j < segments) at[(k + j) * slot_size] = s;
        }
    }
}

// One wavefront takes PR rows of P a lane, NL lanes with NR elements of N each: 64 / NL * PR rows, NL NR >= N.  Sixteen tokens at a time
// are brought to LDS, the next sixteen on their way in registers; then for every token each lane updates its PR x NR elements (multiply,
// multiply-add) and adds their products with C.  (Eight at a time of the widest rows, for the registers' sake.)
// What bounds it: three vector instructions for each element of state and token: 8192 tokens in eight prompts of 32 heads of 64 x 128 take
// 447 us, of which those are 224.  (With the rows of a tile fetched when it is its turn, 1667 tokens of 10 heads of 50 x 37 took 123 us, now 65.)
template <typename T, int NL, int NR, int MODE>
__global__ void __launch_bounds__(64, NL * NR > 128 ? 1 : 2)
selective_scan_kernel(const T *__restrict__ xbc, T *__restrict__ out, ScanCall c)
{
    constexpr int PR = 4, PW = 64 / NL * PR, NP = NL * NR, TT = NP > 128 || PW > 64 ? 8 : 16;
    __shared__ __align__(16) float sb[TT][NP + 4], sc[TT][NP + 4], sx[TT][PW + 4], sy[TT][PW + 4];
    __shared__ float2 sd[TT];
    __shared__ double se[MODE == SCAN_CARRY ? TT : 1];
    const int lane = threadIdx.x, ln = lane % NL, lp = lane / NL;
    const int64_t id = scan_unit();
    const int per = c.H * c.parts;
    const int64_t work = id / per;
    const int h = (int)(id % per) / c.parts, p0 = (int)(id % per) % c.parts * PW, g = h / (c.H / c.G);
    const int P = c.P, N = c.N, np = min(PW, P - p0);
    const int segments = (c.seqs.hi - c.seqs.lo + c.seg - 1) / c.seg;
    if (MODE == SCAN_WHOLE ? work >= c.seqs.n : work >= segments) return;
    const float a = c.a[h], skip = c.skip ? c.skip[h] : 0.0f, bias = c.dt.bias ? c.dt.bias[h] : 0.0f;
    const int64_t head_at = ((int64_t)h * P + p0) * N;

    float S[PR][NR];
    auto clear = [&]() SCAN_INLINE {
#pragma unroll
        for (int i = 0; i < PR; ++i)
#pragma unroll
            for (int j = 0; j < NR; ++j) S[i][j] = 0.0f;
    };
    auto each = [&](auto &&fn) SCAN_INLINE {                     // fn(element, offset from the head's first) of those that exist
#pragma unroll
        for (int i = 0; i < PR; ++i)
#pragma unroll
            for (int j = 0; j < NR; ++j)
                if (lp * PR + i < np && ln * NR + j < N) fn(S[i][j], (int64_t)(lp * PR + i) * N + ln * NR + j);
    };
    // Sixteen tokens' rows in registers: element 64 i + lane of [TT][NP] or [TT][PW] (rows behind the last are the last one again).
    constexpr int LB = TT * NP / 64, LX = TT * PW / 64;
    float rb[LB], rc[MODE != SCAN_CARRY ? LB : 1], rx[LX], raw = 0.0f;
    const T *const rows = xbc + (int64_t)c.H * P + (int64_t)g * N, *const xs = xbc + (int64_t)h * P + p0;
    const int64_t to_c = (int64_t)c.G * N;
    auto fetch = [&](int t, int t1) SCAN_INLINE {
        static_for<0, LB>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            const int e = 64 * i + lane, n = e % NP;
            const T *row = rows + (int64_t)min(t + e / NP, t1 - 1) * c.ld + (n < N ? n : 0);
            rb[i] = (float)row[0];
            if constexpr (MODE != SCAN_CARRY) rc[i] = (float)row[to_c];
        });
        static_for<0, LX>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            const int e = 64 * i + lane, p = e % PW;
            rx[i] = (float)xs[(int64_t)min(t + e / PW, t1 - 1) * c.ld + (p < np ? p : 0)];
        });
        raw = dt_raw(c.dt, min(t + lane % TT, t1 - 1), h);
    };
    // Tokens [t0, t1) of one sequence; adds their decay exponents to `sum`.
    auto run = [&](int t0, int t1, double &sum) SCAN_INLINE {
        fetch(t0, t1);
        for (int t = t0; t < t1; t += TT) {
            const int nt = min(TT, t1 - t);
            bool far = false;                        // dt x may be infinite, of which the zeros behind the last of N would make NaN of y
            __syncthreads();
            static_for<0, LB>([&](auto i_) SCAN_INLINE {
                constexpr int i = decltype(i_)::value;
                const int e = 64 * i + lane, n = e % NP;
                sb[e / NP][n] = n < N ? rb[i] : 0.0f;
                if constexpr (MODE != SCAN_CARRY) sc[e / NP][n] = n < N ? rc[i] : 0.0f;
            });
            static_for<0, LX>([&](auto i_) SCAN_INLINE {
                constexpr int i = decltype(i_)::value;
                const int e = 64 * i + lane;
                sx[e / PW][e % PW] = e % PW < np ? rx[i] : 0.0f;
                if (MODE != SCAN_CARRY) far |= !(fabsf(rx[i]) < 1e28f);
            });
            if (lane < TT) {
                const float dt = dt_of(c.dt, raw, bias);
                const double ex = decay_exponent(dt, a);
                sd[lane] = make_float2(exp2_of(ex), dt);
                if (MODE == SCAN_CARRY) se[lane] = ex;
                else far |= !(fabsf(dt) < 1e10f);
            }
            if (t + TT < t1) fetch(t + TT, t1);
            float gate[MODE != SCAN_CARRY ? LX : 1]; // z of these tokens
            if (MODE != SCAN_CARRY && c.z)
                static_for<0, LX>([&](auto i_) SCAN_INLINE {
                    constexpr int i = decltype(i_)::value;
                    const int e = 64 * i + lane, p = e % PW;
                    gate[i] = (float)static_cast<const T *>(c.z)[(int64_t)min(t + e / PW, t1 - 1) * c.ld_z + (int64_t)h * P + p0 + (p < np ? p : 0)];
                });
            __syncthreads();
            auto token = [&](int r, auto far_) SCAN_INLINE {
                constexpr bool far = decltype(far_)::value;
                const float2 d = sd[r];
                if (MODE == SCAN_CARRY) sum += se[r];
                float y[PR];
#pragma unroll
                for (int i = 0; i < PR; ++i) {
                    const float x = sx[r][lp * PR + i] * d.y;
                    y[i] = 0.0f;
#pragma unroll
                    for (int j = 0; j < NR; ++j) {
                        S[i][j] = fmaf(x, sb[r][ln * NR + j], d.x * S[i][j]);
                        if (far && ln * NR + j >= N) S[i][j] = 0.0f;
                        if (MODE != SCAN_CARRY) y[i] = fmaf(S[i][j], sc[r][ln * NR + j], y[i]);
                    }
                }
                if (MODE != SCAN_CARRY) {
#pragma unroll
                    for (int i = 0; i < PR; ++i) y[i] = lanes_sum<NL>(y[i]);
                    if (ln == 0) *reinterpret_cast<f32x4_t *>(&sy[r][lp * PR]) = f32x4_t{y[0], y[1], y[2], y[3]};
                }
            };
            if (!__ballot(far)) {
#pragma unroll 2
                for (int r = 0; r < nt; ++r) token(r, std::false_type{});
            } else {
#pragma unroll 1
                for (int r = 0; r < nt; ++r) token(r, std::true_type{});
            }
            if (MODE != SCAN_CARRY) {
                __syncthreads();
                static_for<0, LX>([&](auto i_) SCAN_INLINE {
                    constexpr int i = decltype(i_)::value;
                    const int e = 64 * i + lane, r = e / PW, p = e % PW;
                    float y = sy[r][p];
                    if (c.skip) y = fmaf(skip, sx[r][p], y);      // (0 times an infinite x would be NaN)
                    if (c.z) y *= silu<T>(gate[i]);
                    if (r < nt && p < np) store1(out + (int64_t)(t + r) * c.ld_out + (int64_t)h * P + p0 + p, y);
                });
            }
        }
    };
    auto zeros = [&](int t0, int t1) SCAN_INLINE {
        for (int t = t0; t < t1; ++t)
            for (int p = lane; p < np; p += 64) store1(out + (int64_t)t * c.ld_out + (int64_t)h * P + p0 + p, 0.0f);
    };
    auto load = [&](const float *from) SCAN_INLINE { each([&](float &v, int64_t at) SCAN_INLINE { v = from[at]; }); };
    auto store = [&](float *to) SCAN_INLINE { each([&](float &v, int64_t at) SCAN_INLINE { to[at] = v; }); };
    scan_drive<MODE>(c, work, h, p0, head_at, lane, clear, load, store, run, zeros);
}

// ------------------------------------------------------------------ single tokens
// Four wavefronts of a work-group, or one, take PW rows of P of one head of one request.  The state's loads start as soon as the slot is
// known, the convolution of the head's x and its group's B and C runs while they travel.  B and C are formed anew for every head of a group;
// the ring's row of the new token, which none of the taps reads, is written for the group's first head alone.
// What bounds it: the state is read and written once: 300 requests of 32 heads of 64 x 128 take 131 us, 640 MB at 4.9 TB/s, one request 6 (a launch
// and its trips to memory; with the taps one by one 8.8).  1024 requests of 32 heads of 16 x 16: 30 us, 92 with four wavefronts to a head.
struct StepCall {
    StepSizes dt;
    int64_t rows, slots, ld, ld_z, ld_out;
    const int32_t *pos, *slot;
    const float *weight, *bias;                      // weight NULL: x | B | C as they are
    int width, silu;
    void *ring;
    const void *z;
    const float *a, *skip;
    int H, P, G, N, parts;
    float *state;
};
typedef f32x4_t __attribute__((aligned(4))) f32x4_any;

// NL lanes with four elements of N each hold a row of P, a wavefront U rows of them in each lane; WAVES of them (4 or 1) share a head.
template <typename T, int NL, int U, int WAVES>
__global__ void __launch_bounds__(256)
selective_step_kernel(const T *__restrict__ xbc, T *__restrict__ out, StepCall c)
{
    constexpr int PL = 64 / NL, PW = WAVES * PL * U, NT = 64 * WAVES, TAPS = 3;
    __shared__ __align__(16) float shared_x[4 / WAVES][PW], shared_bc[4 / WAVES][2][4 * NL];
    const int lane = threadIdx.x & 63, in_group = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), ln = lane % NL;
    const int wave = WAVES == 4 ? in_group : 0, mine = WAVES == 4 ? 0 : in_group, tid = wave * 64 + lane;
    float *const sx = shared_x[mine], *const sb = shared_bc[mine][0], *const sc = shared_bc[mine][1];
    const int64_t id = (int64_t)work_group() * (4 / WAVES) + mine;
    const int per = c.H * c.parts;
    const int64_t r = id / per;
    if (r >= c.rows) return;                         // (wavefronts that share nothing meet no barrier)
    const int h = (int)(id % per) / c.parts, p0 = (int)(id % per) % c.parts * PW, g = h / (c.H / c.G);
    const int P = c.P, N = c.N, np = min(PW, P - p0), C = c.H * P + 2 * c.G * N;
    const int pos = c.pos[r];
    const int64_t at = c.slot ? c.slot[r] : r;
    const bool kept = at >= 0 && at < c.slots;
    T *o = out + r * c.ld_out + (int64_t)h * P + p0;
    if (pos < 0) {
        for (int p = tid; p < np; p += NT) store1(o + p, 0.0f);
        return;
    }
    float *S = kept ? c.state + ((at * c.H + h) * P + p0) * (int64_t)N : nullptr;
    auto row_of = [&](int u) { return (u * WAVES + wave) * PL + lane / NL; };
    f32x4_t v[U];
    const bool whole = ln * 4 + 4 <= N;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        v[u] = f32x4_t{0, 0, 0, 0};
        if (kept && pos > 0 && row_of(u) < np && ln * 4 < N) {
            const float *from = S + (int64_t)row_of(u) * N + ln * 4;
            if (whole) v[u] = __builtin_nontemporal_load(reinterpret_cast<const f32x4_any *>(from));
            else
                for (int i = 0; i < 3; ++i)
                    if (ln * 4 + i < N) v[u][i] = from[i];
        }
    }
    const float dt = dt_of(c.dt, dt_raw(c.dt, r, h), c.dt.bias ? c.dt.bias[h] : 0.0f);
    const float decay = exp2_of(decay_exponent(dt, c.a[h])), skip = c.skip ? c.skip[h] : 0.0f;
    const bool first = h % (c.H / c.G) == 0 && p0 == 0;
    const T *x = xbc + r * c.ld;
    T *ring = c.ring && kept ? static_cast<T *>(c.ring) + at * c.width * (int64_t)C : nullptr;
    // (the filter's first taps: loads without a branch between them, further ones one by one)
    for (int e = tid; e < PW + 8 * NL; e += NT) {
        const int which = e < PW ? 0 : (e - PW) / (4 * NL), n = (e - PW) % (4 * NL);
        const bool there = e < PW ? e < np : n < N;
        const int ch = !there ? 0 : e < PW ? h * P + p0 + e : c.H * P + which * c.G * N + g * N + n;
        const T now = x[ch];
        float q = (float)now;
        if (c.weight) {
            const float *w = c.weight + (int64_t)ch * c.width;
            float acc = c.bias ? c.bias[ch] : 0.0f, u[TAPS], f[TAPS];
            const float last = w[c.width - 1];
#pragma unroll
            for (int k = 0; k < TAPS; ++k) {         // k + 1 tokens ago
                const bool tap = k + 1 < c.width && pos > k && ring;
                u[k] = tap ? (float)ring[(int64_t)((pos - 1 - k) % c.width) * C + ch] : 0.0f;
                f[k] = tap ? w[c.width - 2 - k] : 0.0f;
            }
            for (int k = TAPS; k + 1 < c.width; ++k)
                if (pos > k && ring) acc = fmaf(w[c.width - 2 - k], (float)ring[(int64_t)((pos - 1 - k) % c.width) * C + ch], acc);
#pragma unroll
            for (int k = TAPS - 1; k >= 0; --k) acc = fmaf(f[k], u[k], acc);
            acc = fmaf(last, q, acc);
            if (ring && there && (e < PW || first)) ring[(int64_t)(pos % c.width) * C + ch] = now;
            q = c.silu ? silu_f32(acc) : acc;                 // (not rounded to T: it goes into the state)
        }
        (e < PW ? sx + e : (which ? sc : sb) + n)[0] = there ? q : 0.0f;
    }
    if constexpr (WAVES == 4) __syncthreads();
    else __builtin_amdgcn_wave_barrier();
    const f32x4_t b = *reinterpret_cast<const f32x4_t *>(sb + ln * 4), cc = *reinterpret_cast<const f32x4_t *>(sc + ln * 4);
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const int p = row_of(u);
        const float xd = sx[p] * dt;
        float y = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[u][i] = fmaf(xd, b[i], decay * v[u][i]);
            y = ln * 4 + i < N ? fmaf(v[u][i], cc[i], y) : y;         // (behind the last of N an infinite x leaves NaN, infinity times 0)
        }
        if (kept && p < np && ln * 4 < N) {
            float *to = S + (int64_t)p * N + ln * 4;
            if (whole) __builtin_nontemporal_store(v[u], reinterpret_cast<f32x4_any *>(to));
            else
                for (int i = 0; i < 3; ++i)
                    if (ln * 4 + i < N) to[i] = v[u][i];
        }
        y = lanes_sum<(NL < 16 ? NL : 16)>(y);
        if constexpr (NL > 16) y += __shfl_xor(y, 16);
        if constexpr (NL > 32) y += __shfl_xor(y, 32);
        if (ln == 0 && p < np) {
            if (c.skip) y = fmaf(skip, sx[p], y);    // (0 times an infinite x would be NaN)
            if (c.z) y *= silu<T>((float)static_cast<const T *>(c.z)[r * c.ld_z + (int64_t)h * P + p0 + p]);
            store1(o + p, y);
        }
    }
}
