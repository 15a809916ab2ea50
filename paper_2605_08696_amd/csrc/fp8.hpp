// Rows in 8 bits: e4m3 values (OCP: 448 largest, no infinities) with one E8M0 scale, a power of two, for each block of 128 along
// a row.  A block's scale is the smallest power of two that brings its largest finite magnitude to 448 or less, so that it lands in
// (224, 448]; e4m3 is a floating-point type, so a scale between the powers of two would win at most part of a bit for values near the
// type's subnormals, and the matrix cores multiply by an E8M0 scale at no cost (v_mfma_scale), which a factor in fp32 is not.
//
// A wavefront takes 512 elements of a row at a time, four blocks: sixteen lanes (a DPP row) with eight consecutive elements each hold a
// block, whose largest magnitude is four DPP steps away, and the four scales are one 32-bit word of the scales' array
// [ceil(d / 512)][rows].  What bounds both kernels is the memory's rate, or for few rows the launch and one trip to memory.
#pragma once
#include "common.hpp"

constexpr int kFp8Block = 128, kFp8Group = 512;      // elements of a block, of a word of scales

// A dimension of a grid holds less than 2^32 threads, which tens of millions of rows exceed: work-groups behind the first 2^21 are further
// rows of the grid, the last of which may have more than there is work for.
constexpr uint32_t kGridRow = 1u << 21;
__device__ __forceinline__ uint32_t work_group() { return blockIdx.y * kGridRow + blockIdx.x; }

__device__ __forceinline__ uint32_t row16_max_u32(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xF, 0xF, true));   // quad_perm [1,0,3,2]
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xF, 0xF, true));   // quad_perm [2,3,0,1]
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xF, 0xF, true));  // row_half_mirror
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x140, 0xF, 0xF, true));  // row_mirror
    return v;
}

// Eight consecutive elements of a row from index `col` on, in two steps, so that several requests travel together: a load without a
// branch (16 bytes from any address of whole elements, which gfx950 allows; the row's last eight where it ends before), and behind it
// their values, zeros behind the row.  (With a branch around each load, the compiler waits for every load at its end: 16384 x 1024
// fp32 rows + bf16 40.6 us, 35 without.)  ONCE: what nothing reads again soon, with the streaming hint.
template <typename T>
struct Raw8;
template <>
struct Raw8<float> {
    f32x4_t a, b;
};
template <>
struct Raw8<bf16> {
    bf16x8_t a;
};
template <bool ONCE = false>
__device__ __forceinline__ Raw8<float> raw8(const float *row, int col, int d)
{
    typedef f32x4_t __attribute__((aligned(4))) unaligned;
    Raw8<float> r;
    if (d < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = col + i < d ? row[col + i] : 0.0f;
            if (i < 4) r.a[i] = x; else r.b[i - 4] = x;
        }
        return r;
    }
    const unaligned *q = reinterpret_cast<const unaligned *>(row + min(col, d - 8));
    if constexpr (ONCE) {
        r.a = __builtin_nontemporal_load(q);
        r.b = __builtin_nontemporal_load(q + 1);
    } else {
        r.a = q[0];
        r.b = q[1];
    }
    return r;
}
template <bool ONCE = false>
__device__ __forceinline__ Raw8<bf16> raw8(const bf16 *row, int col, int d)
{
    typedef bf16x8_t __attribute__((aligned(2))) unaligned;
    Raw8<bf16> r;
    if (d < 8) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.a[i] = col + i < d ? row[col + i] : (bf16)0.0f;
        return r;
    }
    const unaligned *q = reinterpret_cast<const unaligned *>(row + min(col, d - 8));
    if constexpr (ONCE) r.a = __builtin_nontemporal_load(q);
    else r.a = *q;
    return r;
}
__device__ __forceinline__ void raw8_values(const Raw8<float> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[i] = r.a[i]; v[4 + i] = r.b[i]; }
}
__device__ __forceinline__ void raw8_values(const Raw8<bf16> &r, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)r.a[i];
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T> &r, int col, int d, float (&v)[8])
{
    raw8_values(r, v);
    if (d >= 8 && __ballot(col + 8 > d)) {           // some lane's eight are the row's last: moved to their places
        const int late = col + 8 - d;                // by which they lie too high
#pragma unroll
        for (int s = 4; s >= 1; s >>= 1)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (late > 0 && (late & s)) v[i] = i + s < 8 ? v[i + s] : 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = col + i < d ? v[i] : 0.0f;
    }
}
// v as it is stored at p, rounded to p's type
__device__ __forceinline__ void store8(float *p, int n, float (&v)[8])
{
    if (n >= 8) {
        const f32x4_t a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        __builtin_memcpy(p, &a, 16);
        __builtin_memcpy(p + 4, &b, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = v[i];
    }
}
__device__ __forceinline__ void store8(bf16 *p, int n, float (&v)[8])
{
    bf16x8_t a;
#pragma unroll
    for (int i = 0; i < 8; ++i) { a[i] = (bf16)v[i]; v[i] = (float)a[i]; }
    if (n >= 8) {
        __builtin_memcpy(p, &a, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = a[i];
    }
}

// This lane's eight values of the block of its sixteen lanes -> their e4m3 codes and the block's scale.  Infinities and NaN do not count
// for the scale and become NaN.  Absent elements are zeros.
__device__ __forceinline__ uint2 fp8_of_block(const float (&v)[8], uint32_t &scale)
{
    constexpr uint32_t kInf = 0x7f800000u;
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t a = __float_as_uint(v[i]) & 0x7fffffffu;
        top = max(top, a < kInf ? a : 0u);
    }
    top = row16_max_u32(top);
    // top / 448 rounded up to a power of two: 448 = 1.75 2^8.  Biased exponents; 1 (2^-126) at least, 127 for zeros
    int s = (int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u ? 1 : 0);
    s = top == 0 ? 127 : max(s, 1);
    const float inv = __uint_as_float((uint32_t)(254 - s) << 23);
    float q[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        q[i] = (__float_as_uint(v[i]) & 0x7fffffffu) < kInf ? v[i] * inv : __uint_as_float(0x7fc00000u);
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[0], q[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[4], q[5], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(q[2], q[3], lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(q[6], q[7], hi, true);
    scale = (uint32_t)s;
    return make_uint2((uint32_t)lo, (uint32_t)hi);
}
// The same of a group's four blocks; their scales in every lane.
__device__ __forceinline__ uint2 fp8_of_8(const float (&v)[8], uint32_t &scales)
{
    uint32_t s;
    const uint2 codes = fp8_of_block(v, s);
    scales = (uint32_t)__builtin_amdgcn_readlane((int)s, 0) | (uint32_t)__builtin_amdgcn_readlane((int)s, 16) << 8 |
             (uint32_t)__builtin_amdgcn_readlane((int)s, 32) << 16 | (uint32_t)__builtin_amdgcn_readlane((int)s, 48) << 24;
    return codes;
}
// The word of a row of one or two blocks, of 16 or 32 lanes, from its blocks' scales.
template <int LANES>
__device__ __forceinline__ uint32_t fp8_narrow_word(uint32_t s)
{
    return LANES == 16 ? s | 0x7f7f7f00u : s | (uint32_t)__shfl_down((int)s, 16) << 8 | 0x7f7f0000u;
}

// x [rows][d], row stride ldx -> q [rows][dp], dp = d rounded up to 128, and scales [groups][rows].  A wavefront takes a group of R rows,
// requested together; the groups of a row lie side by side.  (us, R = 1 | 2 | 4: 16384 x 1024 fp32 16.6 | 17 | 17.7, with the groups of a
// column of rows side by side instead 18.2; 16384 x 4096 bf16 40.4 | 36.9 | 36.9 (5.5 TB/s), 3001 x 4001 bf16 8.9 | 8.4 | 9.4, 300 x 4096 bf16
// 2.6 | 2.9 | 3.6.  With the streaming hint what the caches hold is read from memory: 3001 x 4001 9.5.)
template <typename T, int R>
__global__ void __launch_bounds__(256)
quantize_fp8_kernel(const T *__restrict__ x, int64_t ldx, uint32_t rows, int d, unsigned char *__restrict__ q, uint32_t *__restrict__ scales)
{
    const uint32_t groups = (uint32_t)(d + kFp8Group - 1) / kFp8Group, unit = work_group() * 4 + (threadIdx.x >> 6);    // < 2^32
    const uint32_t row0 = unit / groups * R, g = unit % groups;
    const int dp = (d + kFp8Block - 1) / kFp8Block * kFp8Block, lane = threadIdx.x & 63, col = (int)g * kFp8Group + lane * 8;
    Raw8<T> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r] = raw8(x + (int64_t)min(row0 + r, rows - 1) * ldx, col, d);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float v[8];
        widen8(raw[r], col, d, v);
        uint32_t s;
        const uint2 codes = fp8_of_8(v, s);
        const uint32_t row = row0 + r;
        if (row >= rows) return;                     // wave-uniform
        if (col < dp) *reinterpret_cast<uint2 *>(q + (int64_t)row * dp + col) = codes;
        if (lane == 0) scales[(int64_t)g * rows + row] = s;
    }
}

// x += add (if there is one), then y = x / sqrt(mean(x^2) + eps) * gain of the row as it is stored -> q, scales.  NW wavefronts hold a
// row in registers, wavefront w its groups w, w + NW, ..., G of them at most.  16384 x 1024 fp32 + bf16 33.5 us (5.5 TB/s, the rate of a copy of
// as many bytes), one row 2.6 us, a launch and a trip to memory.  Not kept: two rows a wavefront (39 .. 42).
template <typename T, typename TAdd, int NW, int G>
__global__ void __launch_bounds__(NW > 4 ? NW * 64 : 256)
rmsnorm_fp8_kernel(T *__restrict__ x, int64_t ldx, const TAdd *__restrict__ add, int64_t ld_add, const float *__restrict__ gain, float eps,
                   int64_t rows, int d, unsigned char *__restrict__ q, uint32_t *__restrict__ scales)
{
    constexpr int ROWS = NW > 4 ? 1 : 4 / NW;        // rows of a work-group
    __shared__ float part[ROWS * NW];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, w = wave % NW;
    const int64_t row = (int64_t)work_group() * ROWS + wave / NW;
    const int groups = (d + kFp8Group - 1) / kFp8Group, dp = (d + kFp8Block - 1) / kFp8Block * kFp8Block;
    const bool in = row < rows;
    const int64_t at = in ? row : rows - 1;
    float v[G][8], sum = 0.0f;
    Raw8<T> rx[G];
    Raw8<TAdd> ra[G];
    // up to 1024 elements a wavefront the gain is requested with the row, so that its latency does not follow the sum
    constexpr bool EARLY = G <= 2;
    Raw8<float> rg[G];
#pragma unroll
    for (int i = 0; i < G; ++i) rx[i] = raw8(x + at * ldx, (w + i * NW) * kFp8Group + lane * 8, d);
    if (add) {
#pragma unroll
        for (int i = 0; i < G; ++i) ra[i] = raw8<true>(add + at * ld_add, (w + i * NW) * kFp8Group + lane * 8, d);
    }
    if constexpr (EARLY) {
#pragma unroll
        for (int i = 0; i < G; ++i) rg[i] = raw8(gain, (w + i * NW) * kFp8Group + lane * 8, d);
    }
#pragma unroll
    for (int i = 0; i < G; ++i) widen8(rx[i], (w + i * NW) * kFp8Group + lane * 8, d, v[i]);
    if (add) {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int col = (w + i * NW) * kFp8Group + lane * 8;
            float t[8];
            widen8(ra[i], col, d, t);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] += t[k];
            store8(x + at * ldx + col, in ? d - col : 0, v[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < G; ++i)
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(v[i][k], v[i][k], sum);
    sum = wave_sum(sum);
    if constexpr (NW > 1) {
        if (lane == 0) part[wave] = sum;
        __syncthreads();
        sum = 0.0f;
#pragma unroll
        for (int k = 0; k < NW; ++k) sum += part[wave / NW * NW + k];
    }
    if (!in) return;
    const float r = 1.0f / sqrtf(sum / (float)d + eps);
#pragma unroll
    for (int i = 0; i < G; ++i) {
        const int g = w + i * NW, col = g * kFp8Group + lane * 8;
        if (g >= groups) break;                      // wave-uniform
        float t[8];
        if constexpr (!EARLY) rg[i] = raw8(gain, col, d);
        widen8(rg[i], col, d, t);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[i][k] = col + k < d ? v[i][k] * r * t[k] : 0.0f;          // (r may be a NaN)
        uint32_t s;
        const uint2 codes = fp8_of_8(v[i], s);
        if (col < dp) *reinterpret_cast<uint2 *>(q + row * dp + col) = codes;
        if (lane == 0) scales[(int64_t)g * rows + row] = s;
    }
}

// Rows of up to 256 elements take a part of a wavefront: LANES lanes, 16 for one block, 32 for two.  (us, a wavefront a row | this: 45726 x 64
// fp32 norm 20.8 | 6.9, 48376 x 64 bf16 quantize 15.3 | 5.2; 131072 x 128 fp32 quantize 13.6, 6.2 TB/s.)
template <typename T, int LANES, int R>
__global__ void __launch_bounds__(256)
quantize_fp8_narrow_kernel(const T *__restrict__ x, int64_t ldx, uint32_t rows, int d, unsigned char *__restrict__ q, uint32_t *__restrict__ scales)
{
    constexpr int DP = LANES * 8, AT_ONCE = 64 / LANES;
    const uint32_t unit = work_group() * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, row0 = unit * (R * AT_ONCE) + lane / LANES;
    const int col = (int)(lane % LANES) * 8;
    Raw8<T> raw[R];
#pragma unroll
    for (int r = 0; r < R; ++r) raw[r] = raw8(x + (int64_t)min(row0 + r * AT_ONCE, rows - 1) * ldx, col, d);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float v[8];
        widen8(raw[r], col, d, v);
        uint32_t s;
        const uint2 codes = fp8_of_block(v, s);
        const uint32_t row = row0 + r * AT_ONCE, word = fp8_narrow_word<LANES>(s);
        if (row >= rows) continue;
        *reinterpret_cast<uint2 *>(q + (int64_t)row * DP + col) = codes;
        if (col == 0) scales[row] = word;
    }
}
template <typename T, typename TAdd, int LANES, int R>
__global__ void __launch_bounds__(256)
rmsnorm_fp8_narrow_kernel(T *__restrict__ x, int64_t ldx, const TAdd *__restrict__ add, int64_t ld_add, const float *__restrict__ gain, float eps,
                          uint32_t rows, int d, unsigned char *__restrict__ q, uint32_t *__restrict__ scales)
{
    constexpr int DP = LANES * 8, AT_ONCE = 64 / LANES;
    const uint32_t unit = work_group() * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, row0 = unit * (R * AT_ONCE) + lane / LANES;
    const int col = (int)(lane % LANES) * 8;
    Raw8<T> rx[R];
    Raw8<TAdd> ra[R];
    const Raw8<float> rg = raw8(gain, col, d);
#pragma unroll
    for (int r = 0; r < R; ++r) rx[r] = raw8(x + (int64_t)min(row0 + r * AT_ONCE, rows - 1) * ldx, col, d);
    if (add) {
#pragma unroll
        for (int r = 0; r < R; ++r) ra[r] = raw8<true>(add + (int64_t)min(row0 + r * AT_ONCE, rows - 1) * ld_add, col, d);
    }
    float g[8];
    widen8(rg, col, d, g);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t row = row0 + r * AT_ONCE;
        float v[8], sum = 0.0f;
        widen8(rx[r], col, d, v);
        if (add) {
            float t[8];
            widen8(ra[r], col, d, t);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += t[k];
            store8(x + (int64_t)min(row, rows - 1) * ldx + col, row < rows ? d - col : 0, v);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) sum = fmaf(v[k], v[k], sum);
        sum = row16_sum(sum);
        if constexpr (LANES == 32) sum += __shfl_xor(sum, 16);
        const float scale = 1.0f / sqrtf(sum / (float)d + eps);
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = col + k < d ? v[k] * scale * g[k] : 0.0f;              // (scale may be a NaN)
        uint32_t s;
        const uint2 codes = fp8_of_block(v, s);
        const uint32_t word = fp8_narrow_word<LANES>(s);
        if (row >= rows) continue;
        *reinterpret_cast<uint2 *>(q + (int64_t)row * DP + col) = codes;
        if (col == 0) scales[row] = word;
    }
}
