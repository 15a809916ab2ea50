// The selective recurrence over packed prompts and single tokens with its short convolution, and the scores of given tokens: operators of
// libsrm that need no model.  (A translation unit of its own, so that the code objects of the others stay as they are.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "srm.h"
#include "conv.hpp"
#include "selective.hpp"
#include "selective_mfma.hpp"
#include "score.hpp"
#include "status.hpp"

static hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }
// blocks < 2^31
static dim3 grid_of(int64_t blocks) { return dim3((unsigned)std::min<int64_t>(blocks, kGridRow), (unsigned)cdiv(blocks, kGridRow)); }
static bool misaligned(const void *p, unsigned to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
static bool known(int32_t dtype) { return dtype == SRM_BF16 || dtype == SRM_FP32; }
static unsigned size_of(int32_t dtype) { return dtype == SRM_BF16 ? 2 : 4; }
static const char *const kNotWhole = "an operand does not lie at a whole element";
constexpr int kChipCus = 256;
constexpr int64_t kMaxRows = 1ll << 30, kMaxBlocks = 1ll << 31;

// ------------------------------------------------------------------ packed sequences
static int check_offsets(const char *who, const int32_t *h, int32_t n, int32_t &longest)
{
    if (n <= 0 || n >= kMaxRows) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (h[0] < 0) return fail(SRM_EINVAL, "%s: offsets must not be negative", who);
    longest = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (h[i + 1] < h[i]) return fail(SRM_EINVAL, "%s: offsets must not fall (sequence %d)", who, i);
        longest = std::max(longest, h[i + 1] - h[i]);
    }
    if (h[n] >= kMaxRows) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    return SRM_OK;
}
static int check_packed(const char *who, const int32_t *h_offsets, const int32_t *d_offsets, int32_t n, const int32_t *d_pos, const int32_t *d_slot,
                        int64_t slots, const void *d_state, Packed &packed, int32_t &longest)
{
    if (!h_offsets || !d_offsets) return fail(SRM_EINVAL, "%s: null argument", who);
    SRM_TRY(check_offsets(who, h_offsets, n, longest));
    if (slots < 0 || (d_state && slots == 0)) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (misaligned(d_offsets, 4) || misaligned(d_pos, 4) || misaligned(d_slot, 4)) return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    packed = Packed{d_offsets, d_pos, d_slot, n, h_offsets[0], h_offsets[n], d_state ? slots : 0};
    return SRM_OK;
}

// ------------------------------------------------------------------ the short convolution
// Runs of 32 tokens, over which a thread's filter (32 W bytes) is read once, as long as they are two rounds of the chip's wavefronts; four
// tokens at a time of a short filter where the shortest runs are less than one.  (Four | eight, us: 37 x 2304 7.7 | 8.9, 300 x 2304 10.4 | 12.6, 32768 x 4352 135 |
// 135, fp32 16384 x 4352 141 | 128, 4000 x 2304 of eight taps 39 | 32; 300 x 2304 in 300 sequences 17, in runs of one 10.)
template <typename T, int W>
static void launch_conv(const void *d_x, void *d_out, ConvCall c, int64_t tokens, hipStream_t st)
{
    auto waves = [&](int run) {
        c.runs = cdiv(tokens, c.run = run);
        return c.units > 64 ? c.runs * cdiv(c.units, 64) : cdiv(c.runs, 64 / c.per_run);
    };
    const bool few = W <= 4 && waves(8) < 4096;
    int64_t n;
    int run = few ? 4 : 32;
    while (run > 8 && waves(run) < 8192) run /= 2;
    // (the sequences of a run are worked on one after the other: shorter runs of sequences that are shorter still)
    while (run > 1 && (int64_t)run * c.seqs.n > tokens && waves(run / 2) <= 16384) run /= 2;
    n = waves(run);
    hipLaunchKernelGGL((few ? causal_conv_kernel<T, W, 4> : causal_conv_kernel<T, W, 8>), grid_of(cdiv(n, 4)), dim3(256), 0, st, static_cast<const T *>(d_x),
                       static_cast<T *>(d_out), c);
}
template <typename T>
static void conv(int width, const void *d_x, void *d_out, const ConvCall &c, int64_t tokens, hipStream_t st)
{
    switch (width) {
    case 1: return launch_conv<T, 1>(d_x, d_out, c, tokens, st);
    case 2: return launch_conv<T, 2>(d_x, d_out, c, tokens, st);
    case 3: return launch_conv<T, 3>(d_x, d_out, c, tokens, st);
    case 4: return launch_conv<T, 4>(d_x, d_out, c, tokens, st);
    case 5: return launch_conv<T, 5>(d_x, d_out, c, tokens, st);
    case 6: return launch_conv<T, 6>(d_x, d_out, c, tokens, st);
    case 7: return launch_conv<T, 7>(d_x, d_out, c, tokens, st);
    default: return launch_conv<T, 8>(d_x, d_out, c, tokens, st);
    }
}

extern "C" int srm_causal_conv(int32_t dtype, const void *d_x, int64_t ldx, const float *d_weight, const float *d_bias, int32_t activation,
                               int32_t channels, int32_t width, const int32_t *h_offsets, const int32_t *d_offsets, int32_t N, const int32_t *d_pos,
                               const int32_t *d_slot, int64_t slots, void *d_state, void *d_out, int64_t ld_out, void *hip_stream)
{
    const char *who = "srm_causal_conv";
    if (!d_weight) return fail(SRM_EINVAL, "%s: null argument", who);
    if (!known(dtype)) return fail(SRM_EINVAL, "%s: unknown dtype %d", who, dtype);
    if (channels <= 0 || channels > (1 << 24) || width <= 0 || width > kConvTaps) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (activation != 0 && activation != 1) return fail(SRM_EINVAL, "%s: unknown activation %d", who, activation);
    if (ldx < channels || ld_out < channels) return fail(SRM_EINVAL, "%s: a row stride is less than %d", who, channels);
    ConvCall c{};
    int32_t longest;
    SRM_TRY(check_packed(who, h_offsets, d_offsets, N, d_pos, d_slot, slots, d_state, c.seqs, longest));
    const unsigned size = size_of(dtype);
    const int64_t tokens = c.seqs.hi - c.seqs.lo;
    if (tokens > 0 && (!d_x || !d_out)) return fail(SRM_EINVAL, "%s: null argument", who);      // (arrays of no rows may lie nowhere)
    if (misaligned(d_x, size) || misaligned(d_out, size) || misaligned(d_state, size) || misaligned(d_weight, 4) || misaligned(d_bias, 4))
        return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    if (tokens * cdiv(channels, 512) >= kMaxBlocks) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (tokens == 0) return SRM_OK;
    c.ldx = ldx;
    c.ld_out = ld_out;
    c.weight = d_weight;
    c.bias = d_bias;
    c.channels = channels;
    c.silu = activation;
    c.units = (int)cdiv(channels, 8);
    for (c.per_run = 1; c.per_run < std::min(c.units, 64); c.per_run *= 2) {}
    c.ring = d_state;
    if (dtype == SRM_BF16) conv<bf16>(width, d_x, d_out, c, tokens, as_stream(hip_stream));
    else conv<float>(width, d_x, d_out, c, tokens, as_stream(hip_stream));
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}

// ------------------------------------------------------------------ the selective recurrence
struct HeadSizes {
    int32_t H, P, G, N;
};
static bool fits(const HeadSizes &s)
{
    return s.H > 0 && s.H <= 65536 && s.P > 0 && s.P <= 4096 && s.N > 0 && s.N <= 256 && s.G > 0 && s.H % s.G == 0 &&
           (int64_t)s.H * s.P + 2ll * s.G * s.N < (1 << 30);
}
static int check_heads(const char *who, int32_t dtype, int32_t dt_dtype, const HeadSizes &s, int64_t rows, const void *xbc, int64_t ld, const void *dt, int64_t ld_dt,
                       const float *a, const float *dt_bias, const float *skip, const void *z, int64_t ld_z, const void *out, int64_t ld_out,
                       const float *state)
{
    if (!a || (rows > 0 && (!xbc || !dt || !out))) return fail(SRM_EINVAL, "%s: null argument", who);        // (arrays of no rows may lie nowhere)
    if (!known(dtype) || !known(dt_dtype)) return fail(SRM_EINVAL, "%s: unknown dtype %d, %d", who, dtype, dt_dtype);
    if (!fits(s)) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    const int64_t inner = (int64_t)s.H * s.P;
    if (ld < inner + 2ll * s.G * s.N || ld_dt < s.H || (z && ld_z < inner) || ld_out < inner) return fail(SRM_EINVAL, "%s: a row stride is less than its row", who);
    const unsigned size = size_of(dtype);
    if (misaligned(xbc, size) || misaligned(z, size) || misaligned(out, size) || misaligned(dt, size_of(dt_dtype)) || misaligned(a, 4) ||
        misaligned(dt_bias, 4) || misaligned(skip, 4) || misaligned(state, 4))
        return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    return SRM_OK;
}

// How a scan is cut over time.  A work-group holds `rows` rows of P; `chip` of them run at the chip's full rate together.  Segments cost a
// pass of their own that forms the states at their ends (about half of the work again), so that whole sequences are taken up to three times a
// segment's length (us, whole | segments: 8192 tokens in eight prompts of 32 heads 59 | 80; one prompt of 16384, 32 work-groups, 799 as a whole, with
// 256 | 384 | 512 | 768 | 1024 work-groups of segments 173 | 154 | 126 | 128 | 138).
struct ScanPlan {
    int parts, seg, segments;                        // segments 0: every sequence as a whole
};
// The form of the fp32 kernel for heads of P x N, as form(lanes along N, elements of N in each): as few lanes along N, which share a row of P
// and its sums, as leave none along P without rows.  (That form | the next with twice the lanes, us, 8192 tokens of 32 heads: in 64 prompts, as many
// wavefronts as the chip takes, 64 x 16 73 | 73, 128 x 16 129 | 145, 64 x 32 92 | 102, 64 x 64 157 | 171, 64 x 128 315 | 438; in eight, with whole
// sequences and few wavefronts, more lanes would be faster: 64 x 16 401 | 311, 64 x 32 498 | 351, 64 x 64 463 | 332, 64 x 128 455 | 427.)
template <int NL, int NR>
struct ScanForm {
    static constexpr int lanes = NL, elements = NR, rows = 64 / NL * 4;
};
template <typename Form>
static auto scan_f32_form(int P, int N, Form &&form)
{
    if (N <= 8) return P > 64 ? form(ScanForm<1, 8>{}) : form(ScanForm<4, 2>{});
    if (N <= 16) return P > 64 ? form(ScanForm<2, 8>{}) : P > 32 ? form(ScanForm<4, 4>{}) : form(ScanForm<8, 2>{});
    if (N <= 32) return P > 32 ? form(ScanForm<4, 8>{}) : form(ScanForm<8, 4>{});
    if (N <= 64) return P > 16 ? form(ScanForm<8, 8>{}) : form(ScanForm<16, 4>{});
    return N <= 128 ? form(ScanForm<16, 8>{}) : form(ScanForm<16, 16>{});
}
static int scan_rows(int32_t dtype, const HeadSizes &s)
{
    return dtype == SRM_BF16 ? kScanRows : scan_f32_form(s.P, s.N, [](auto form) { return decltype(form)::rows; });
}
static ScanPlan scan_plan(int32_t dtype, const HeadSizes &s, int64_t tokens, int32_t longest)
{
    ScanPlan p{(int)cdiv(s.P, scan_rows(dtype, s)), 0, 0};
    const int64_t chip = dtype == SRM_BF16 ? 768 : 2048, units = (int64_t)s.H * p.parts, least = 64;
    const int64_t seg = std::max(least, cdiv(cdiv(tokens * units, chip), 64) * 64);
    if (longest > 3 * seg + 3 * least) {
        p.seg = (int)seg;
        p.segments = (int)cdiv(tokens, seg);
    }
    return p;
}
static size_t segment_bytes(const HeadSizes &s) { return ((size_t)2 * s.P * s.N + 1) * s.H * 4; }

extern "C" size_t srm_selective_scan_workspace_bytes(int32_t dtype, const int32_t *h_offsets, int32_t N, int32_t heads, int32_t head_dim,
                                                     int32_t state_dim)
{
    const HeadSizes s{heads, head_dim, 1, state_dim};
    int32_t longest;
    if (!h_offsets || !known(dtype) || !fits(s) || check_offsets("srm_selective_scan_workspace_bytes", h_offsets, N, longest) != SRM_OK) return 0;
    return scan_plan(dtype, s, h_offsets[N] - h_offsets[0], longest).segments * segment_bytes(s);
}

template <typename T, auto WHOLE, auto CARRY, auto SEGMENTS>
static int launch_scan(const void *d_xbc, void *d_out, const ScanCall &c, const ScanPlan &p, int threads, hipStream_t st)
{
    const int64_t units = (int64_t)c.H * c.parts;
    const T *x = static_cast<const T *>(d_xbc);
    T *out = static_cast<T *>(d_out);
    const dim3 grid = grid_of(cdiv((p.segments ? p.segments : c.seqs.n) * units, 8 * kScanRun) * 8 * kScanRun);
    if (p.segments == 0) {
        hipLaunchKernelGGL(WHOLE, grid, dim3(threads), 0, st, x, out, c);
    } else {
        hipLaunchKernelGGL(CARRY, grid, dim3(threads), 0, st, x, out, c);
        HIP_TRY(hipGetLastError());
        const int head_size = c.P * c.N;
        hipLaunchKernelGGL(selective_scan_join_kernel, grid_of(cdiv((int64_t)c.H * head_size, 256)), dim3(256), 0, st, c.carry, c.decay, p.segments - 1, c.H,
                           head_size);
        HIP_TRY(hipGetLastError());
        hipLaunchKernelGGL(SEGMENTS, grid, dim3(threads), 0, st, x, out, c);
    }
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}
static int scan_f32(const void *d_xbc, void *d_out, const ScanCall &c, const ScanPlan &p, hipStream_t st)
{
    return scan_f32_form(c.P, c.N, [&](auto form) {
        constexpr int NL = decltype(form)::lanes, NR = decltype(form)::elements;
        return launch_scan<float, selective_scan_kernel<float, NL, NR, SCAN_WHOLE>, selective_scan_kernel<float, NL, NR, SCAN_CARRY>,
                           selective_scan_kernel<float, NL, NR, SCAN_SEGMENTS>>(d_xbc, d_out, c, p, 64, st);
    });
}
template <bool W>
static int scan_bf16(const void *d_xbc, void *d_out, const ScanCall &c, const ScanPlan &p, hipStream_t st)
{
#define SCAN_CASE(NP)                                                                                                                         \
    return launch_scan<bf16, selective_scan_mfma_kernel<NP, SCAN_WHOLE, W>, selective_scan_mfma_kernel<NP, SCAN_CARRY, W>,                  \
                       selective_scan_mfma_kernel<NP, SCAN_SEGMENTS, W>>(d_xbc, d_out, c, p, 256, st)
    if (c.N <= 32) SCAN_CASE(32);
    if (c.N <= 64) SCAN_CASE(64);
    if (c.N <= 128) SCAN_CASE(128);
    SCAN_CASE(256);
#undef SCAN_CASE
}

extern "C" int srm_selective_scan(int32_t dtype, const void *d_xbc, int64_t ld_xbc, int32_t dt_dtype, const void *d_dt, int64_t ld_dt, const float *d_a,
                                  const float *d_dt_bias, const float *d_skip, int32_t softplus, const void *d_z, int64_t ld_z, int32_t heads,
                                  int32_t head_dim, int32_t groups, int32_t state_dim, const int32_t *h_offsets, const int32_t *d_offsets, int32_t N,
                                  const int32_t *d_pos, const int32_t *d_slot, int64_t slots, float *d_state, void *d_out, int64_t ld_out,
                                  void *d_workspace, size_t workspace_bytes, void *hip_stream)
{
    const char *who = "srm_selective_scan";
    const HeadSizes s{heads, head_dim, groups, state_dim};
    ScanCall c{};
    int32_t longest;
    SRM_TRY(check_packed(who, h_offsets, d_offsets, N, d_pos, d_slot, slots, d_state, c.seqs, longest));
    const int64_t tokens = c.seqs.hi - c.seqs.lo;
    SRM_TRY(check_heads(who, dtype, dt_dtype, s, tokens, d_xbc, ld_xbc, d_dt, ld_dt, d_a, d_dt_bias, d_skip, d_z, ld_z, d_out, ld_out, d_state));
    if (misaligned(d_workspace, 4)) return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    ScanPlan p = scan_plan(dtype, s, tokens, longest);
    const int64_t room = d_workspace ? (int64_t)(workspace_bytes / segment_bytes(s)) : 0;
    if (p.segments > room) {                         // fewer and longer segments, or none
        p.segments = 0;
        if (room > 1) {
            p.seg = (int)((cdiv(tokens, room) + 63) / 64 * 64);
            p.segments = (int)cdiv(tokens, p.seg);
        }
    }
    if (std::max<int64_t>(p.segments, N) * heads * p.parts >= kMaxBlocks - 64) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (tokens == 0) return SRM_OK;
    c.dt = StepSizes{d_dt, ld_dt, d_dt_bias, dt_dtype == SRM_BF16, softplus != 0};
    c.ld = ld_xbc;
    c.ld_z = ld_z;
    c.ld_out = ld_out;
    c.z = d_z;
    c.a = d_a;
    c.skip = d_skip;
    c.H = heads;
    c.P = head_dim;
    c.G = groups;
    c.N = state_dim;
    // (offsets inside a block of rows are 32 bits)
    auto lies_whole = [](const void *q, int64_t ld) { return !q || (!misaligned(q, 16) && ld % 8 == 0 && ld < (1 << 23)); };
    c.chunks = state_dim % 8 == 0 && head_dim % 8 == 0;
    const bool whole = c.chunks && lies_whole(d_xbc, ld_xbc) && lies_whole(d_z, ld_z) && lies_whole(d_out, ld_out);
    c.state = d_state;
    c.seg = p.segments ? p.seg : 1;
    c.parts = p.parts;
    if (p.segments) {
        const size_t all = (size_t)p.segments * heads * head_dim * state_dim;
        c.carry = static_cast<float *>(d_workspace);
        c.held = c.carry + all;
        c.decay = c.held + all;
    }
    if (dtype == SRM_BF16 && whole) return scan_bf16<true>(d_xbc, d_out, c, p, as_stream(hip_stream));
    return dtype == SRM_BF16 ? scan_bf16<false>(d_xbc, d_out, c, p, as_stream(hip_stream)) : scan_f32(d_xbc, d_out, c, p, as_stream(hip_stream));
}

// ------------------------------------------------------------------ single tokens
// A head's state takes `need` rounds of a wavefront's 64 / NL rows of P.  Many heads: up to eight rounds are one wavefront's, further ones four
// wavefronts' of a work-group, up to eight each.  Few: four wavefronts with as few rounds each as leave two work-groups a CU, so that the state's loads
// start on as many CUs as there are.  (One wavefront | four with as many rounds | the best of other forms, us, four taps, bf16: 1024 requests of 32 heads
// of 16 x 16 30 | 92, 64 x 16 63 | 110 | 63, 128 x 16 112 | 145, 64 x 32 108 | 140, 32 x 64 113 | 143, 16 x 128 127 | 168; from sixteen rounds on
// 64 x 64 257 | 193, 128 x 32 201 | 194, 32 x 128 233 | 215, 64 x 128 449 | 378.  512 heads, as few rounds as leave two work-groups a CU | as many: 64 x 32
// 5.9 | 8.0, 32 x 64 5.9 | 8.7, 128 x 16 5.8 | 8.9, 64 x 16 5.1 | 6.4; 2048 heads 11.5 | 9.6, 11.6 | 10.2, 11.9 | 10.9, 9.8 | 7.9; one request of 64 x 128
// 4.9 | 7.8.  Over 119 sizes and numbers of requests the rule is 0.7 % off the best of eight forms in the mean, 12 % at most; fp32 0.9 and 16.)
template <typename T, int NL, int U, int WAVES>
static void launch_step(const void *d_xbc, void *d_out, StepCall c, hipStream_t st)
{
    c.parts = (int)cdiv(c.P, WAVES * (64 / NL) * U);
    hipLaunchKernelGGL((selective_step_kernel<T, NL, U, WAVES>), grid_of(cdiv(c.rows * c.H * c.parts, 4 / WAVES)), dim3(256), 0, st,
                       static_cast<const T *>(d_xbc), static_cast<T *>(d_out), c);
}
template <typename T, int NL, int WAVES>
static void step_rounds(int rounds, const void *d_xbc, void *d_out, const StepCall &c, hipStream_t st)
{
    if (rounds <= 1) return launch_step<T, NL, 1, WAVES>(d_xbc, d_out, c, st);
    if (rounds <= 2) return launch_step<T, NL, 2, WAVES>(d_xbc, d_out, c, st);
    if (rounds <= 4) return launch_step<T, NL, 4, WAVES>(d_xbc, d_out, c, st);
    launch_step<T, NL, 8, WAVES>(d_xbc, d_out, c, st);
}
template <typename T, int NL>
static void step_lanes(const void *d_xbc, void *d_out, const StepCall &c, hipStream_t st)
{
    const int64_t heads = c.rows * c.H, need = cdiv(c.P, 64 / NL), two_each = 2 * kChipCus;
    if (heads <= two_each && need > 1) {
        int rounds = 1;
        while (rounds < 8 && heads * cdiv(need, 4 * rounds) > two_each) rounds *= 2;
        step_rounds<T, NL, 4>(rounds, d_xbc, d_out, c, st);
    } else if (need <= 8) {
        step_rounds<T, NL, 1>((int)need, d_xbc, d_out, c, st);
    } else {
        step_rounds<T, NL, 4>((int)cdiv(need, 4), d_xbc, d_out, c, st);
    }
}
template <typename T>
static void step(const void *d_xbc, void *d_out, const StepCall &c, hipStream_t st)
{
    if (c.N <= 16) return step_lanes<T, 4>(d_xbc, d_out, c, st);
    if (c.N <= 32) return step_lanes<T, 8>(d_xbc, d_out, c, st);
    if (c.N <= 64) return step_lanes<T, 16>(d_xbc, d_out, c, st);
    if (c.N <= 128) return step_lanes<T, 32>(d_xbc, d_out, c, st);
    step_lanes<T, 64>(d_xbc, d_out, c, st);
}

extern "C" int srm_selective_step(int32_t dtype, const void *d_xbc, int64_t ld_xbc, const float *d_weight, const float *d_bias, int32_t activation,
                                  int32_t width, void *d_conv_state, int32_t dt_dtype, const void *d_dt, int64_t ld_dt, const float *d_a,
                                  const float *d_dt_bias, const float *d_skip, int32_t softplus, const void *d_z, int64_t ld_z, int32_t heads,
                                  int32_t head_dim, int32_t groups, int32_t state_dim, int64_t rows, const int32_t *d_pos, const int32_t *d_slot,
                                  int64_t slots, float *d_state, void *d_out, int64_t ld_out, void *hip_stream)
{
    const char *who = "srm_selective_step";
    const HeadSizes s{heads, head_dim, groups, state_dim};
    SRM_TRY(check_heads(who, dtype, dt_dtype, s, 1, d_xbc, ld_xbc, d_dt, ld_dt, d_a, d_dt_bias, d_skip, d_z, ld_z, d_out, ld_out, d_state));
    if (!d_state || !d_pos) return fail(SRM_EINVAL, "%s: null argument", who);
    if (rows <= 0 || rows >= kMaxRows || slots <= 0) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (d_weight) {
        if (width <= 0 || width > kConvTaps) return fail(SRM_EINVAL, "%s: sizes out of range", who);
        if (width > 1 && !d_conv_state) return fail(SRM_EINVAL, "%s: null argument", who);
        if (activation != 0 && activation != 1) return fail(SRM_EINVAL, "%s: unknown activation %d", who, activation);
    }
    if (misaligned(d_weight, 4) || misaligned(d_bias, 4) || misaligned(d_conv_state, size_of(dtype)) || misaligned(d_pos, 4) || misaligned(d_slot, 4))
        return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    if (rows * heads * cdiv(head_dim, 8) >= kMaxBlocks) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    StepCall c{};
    c.dt = StepSizes{d_dt, ld_dt, d_dt_bias, dt_dtype == SRM_BF16, softplus != 0};
    c.rows = rows;
    c.slots = slots;
    c.ld = ld_xbc;
    c.ld_z = ld_z;
    c.ld_out = ld_out;
    c.pos = d_pos;
    c.slot = d_slot;
    c.weight = d_weight;
    c.bias = d_bias;
    c.width = d_weight ? width : 1;
    c.silu = activation;
    c.ring = d_weight ? d_conv_state : nullptr;
    c.z = d_z;
    c.a = d_a;
    c.skip = d_skip;
    c.H = heads;
    c.P = head_dim;
    c.G = groups;
    c.N = state_dim;
    c.state = d_state;
    if (dtype == SRM_BF16) step<bf16>(d_xbc, d_out, c, as_stream(hip_stream));
    else step<float>(d_xbc, d_out, c, as_stream(hip_stream));
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}

// ------------------------------------------------------------------ scores of given tokens
// Work-groups of 1024 threads while every row has a CU, behind that of 512, two of which a CU holds; few logits by fewer threads.
// (1024 | 512 threads, us: 1 x 32000 fp32 8.8 | 11.0, 37 x 128001 bf16 22 | 29, 300 x 32000 fp32 20.5 | 19.1, 2001 x 128001 bf16 161 | 140;
// 4096 x 512 fp32 by 256 threads 25, by a wavefront a row 11.7.)
template <typename T>
static void launch_score(const void *d_logits, const ScoreCall &c, hipStream_t st)
{
    const T *logits = static_cast<const T *>(d_logits);
    const int threads = c.V <= 2048 ? 64 : c.V <= 8192 ? 256 : c.rows > kChipCus ? 512 : 1024;
    const auto kernel = threads == 64    ? token_logprobs_kernel<T, 64>
                        : threads == 256 ? token_logprobs_kernel<T, 256>
                        : threads == 512 ? token_logprobs_kernel<T, 512>
                                         : token_logprobs_kernel<T, 1024>;
    hipLaunchKernelGGL(kernel, grid_of(c.rows), dim3(threads), 0, st, logits, c);
}

extern "C" int srm_token_logprobs(int32_t dtype, const void *d_logits, int64_t ld, int64_t rows, int32_t vocab, const float *d_temperature,
                                  const int32_t *d_token, float *d_logprob, float *d_entropy, int32_t top, int32_t *d_top_token,
                                  float *d_top_logprob, void *hip_stream)
{
    const char *who = "srm_token_logprobs";
    if (!d_logits || (d_token && !d_logprob) || (d_logprob && !d_token)) return fail(SRM_EINVAL, "%s: null argument", who);
    if (!known(dtype)) return fail(SRM_EINVAL, "%s: unknown dtype %d", who, dtype);
    if (rows <= 0 || rows >= kMaxRows || vocab <= 0 || vocab > kScoreVocab || top < 0 || top > kScoreTop)
        return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (top > 0 && (!d_top_token || !d_top_logprob)) return fail(SRM_EINVAL, "%s: null argument", who);
    if (!d_token && !d_entropy && top == 0) return fail(SRM_EINVAL, "%s: nothing to compute", who);
    if (ld < vocab) return fail(SRM_EINVAL, "%s: row stride %lld is less than %d", who, (long long)ld, vocab);
    const void *const words[] = {d_temperature, d_token, d_logprob, d_entropy, d_top_token, d_top_logprob};
    bool whole = !misaligned(d_logits, size_of(dtype));
    for (const void *w : words) whole = whole && !misaligned(w, 4);
    if (!whole) return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    const ScoreCall c{rows, ld, vocab, top, d_token, d_temperature, d_logprob, d_entropy, d_top_logprob, d_top_token};
    if (dtype == SRM_BF16) launch_score<bf16>(d_logits, c, as_stream(hip_stream));
    else launch_score<float>(d_logits, c, as_stream(hip_stream));
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}
