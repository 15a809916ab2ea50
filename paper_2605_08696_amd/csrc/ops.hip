// The operators of libsrm that need no model: rows in 8 bits with scales, their products, and sampling by request.
// (A translation unit of its own, so that the code object of the generation kernels stays as it is.)
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>

#include "srm.h"
#include "fp8.hpp"
#include "gemm_fp8.hpp"
#include "sample_rows.hpp"
#include "status.hpp"

static hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }
// blocks < 2^30
static dim3 grid_of(int64_t blocks) { return dim3((unsigned)std::min<int64_t>(blocks, kGridRow), (unsigned)cdiv(blocks, kGridRow)); }
static bool misaligned(const void *p, unsigned to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }

// ------------------------------------------------------------------ 8-bit rows
extern "C" size_t srm_fp8_row_bytes(int32_t K) { return K > 0 ? align_up((size_t)K, kFp8Block) : 0; }
extern "C" size_t srm_fp8_scale_bytes(int64_t rows, int32_t K)
{
    return rows > 0 && K > 0 ? (size_t)cdiv(K, kFp8Group) * (size_t)rows * 4 : 0;
}

static int check_fp8(const char *who, const void *d_q, const void *d_scales)
{
    if (!d_q || !d_scales) return fail(SRM_EINVAL, "%s: null argument", who);
    if (misaligned(d_q, 16) || misaligned(d_scales, 4))
        return fail(SRM_EINVAL, "%s: 8-bit rows must lie at multiples of 16 bytes, their scales at multiples of 4", who);
    return SRM_OK;
}
static unsigned size_of(int32_t dtype) { return dtype == SRM_BF16 ? 2 : 4; }
static const char *const kNotWhole = "an operand does not lie at a whole element";
constexpr int64_t kMaxRows = 1ll << 30;
constexpr int32_t kNarrow = 256;                      // rows of up to so many elements share wavefronts
constexpr int32_t kMaxWidth = 1 << 22;                // (256 rows of a tile are addressed by 32 bits)

template <typename T, int R>
static int launch_quantize(const void *d_x, int64_t ldx, int64_t rows, int32_t K, void *d_q, void *d_scales, hipStream_t st)
{
    const int64_t blocks = cdiv(cdiv(rows, R) * cdiv(K, kFp8Group), 4);
    hipLaunchKernelGGL((quantize_fp8_kernel<T, R>), grid_of(blocks), dim3(256), 0, st, static_cast<const T *>(d_x), ldx, (uint32_t)rows, K,
                       static_cast<unsigned char *>(d_q), static_cast<uint32_t *>(d_scales));
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}
// (two bf16 rows a wavefront, whose eight elements are half the bytes of fp32 ones, once there are some tens of wavefronts a CU)
template <typename T>
static int quantize(const void *d_x, int64_t ldx, int64_t rows, int32_t K, void *d_q, void *d_scales, hipStream_t st)
{
    if (K <= kNarrow) {
        constexpr int R = 2;
        const bool two = K > kFp8Block;
        const auto kernel = two ? quantize_fp8_narrow_kernel<T, 32, R> : quantize_fp8_narrow_kernel<T, 16, R>;
        hipLaunchKernelGGL(kernel, grid_of(cdiv(rows, (two ? 8 : 16) * R)), dim3(256), 0, st, static_cast<const T *>(d_x), ldx, (uint32_t)rows, K,
                           static_cast<unsigned char *>(d_q), static_cast<uint32_t *>(d_scales));
        HIP_TRY(hipGetLastError());
        return SRM_OK;
    }
    const int64_t units = rows * cdiv(K, kFp8Group);
    if (units >= 1ll << 31) return fail(SRM_EINVAL, "srm_quantize_fp8: sizes out of range");
    if constexpr (sizeof(T) == 2) {
        if (units >= 8192) return launch_quantize<T, 2>(d_x, ldx, rows, K, d_q, d_scales, st);
    }
    return launch_quantize<T, 1>(d_x, ldx, rows, K, d_q, d_scales, st);
}

extern "C" int srm_quantize_fp8(int32_t dtype, const void *d_x, int64_t ldx, int64_t rows, int32_t K, void *d_q, void *d_scales,
                                void *hip_stream)
{
    const char *who = "srm_quantize_fp8";
    if (!d_x) return fail(SRM_EINVAL, "%s: null argument", who);
    SRM_TRY(check_fp8(who, d_q, d_scales));
    if (rows <= 0 || rows >= kMaxRows || K <= 0 || K > kMaxWidth) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (ldx < K) return fail(SRM_EINVAL, "%s: row stride %lld is less than %d", who, (long long)ldx, K);
    if (misaligned(d_x, size_of(dtype))) return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    if (dtype == SRM_FP32) return quantize<float>(d_x, ldx, rows, K, d_q, d_scales, as_stream(hip_stream));
    if (dtype == SRM_BF16) return quantize<bf16>(d_x, ldx, rows, K, d_q, d_scales, as_stream(hip_stream));
    return fail(SRM_EINVAL, "%s: unknown dtype %d", who, dtype);
}

template <typename T, typename TAdd, int NW, int G>
static int launch_rmsnorm(void *d_x, int64_t ldx, const void *d_add, int64_t ld_add, const float *d_gain, float eps, int64_t rows, int32_t d,
                          void *d_q, void *d_scales, hipStream_t st)
{
    constexpr int ROWS = NW > 4 ? 1 : 4 / NW;
    hipLaunchKernelGGL((rmsnorm_fp8_kernel<T, TAdd, NW, G>), grid_of(cdiv(rows, ROWS)), dim3(NW > 4 ? NW * 64 : 256), 0, st,
                       static_cast<T *>(d_x), ldx, static_cast<const TAdd *>(d_add), ld_add, d_gain, eps, rows, d,
                       static_cast<unsigned char *>(d_q), static_cast<uint32_t *>(d_scales));
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}
constexpr int32_t kMaxNorm = 32768;
// (by the width alone: a row's sum is formed in the same order whatever the number of rows)
template <typename T, typename TAdd>
static int rmsnorm(void *d_x, int64_t ldx, const void *d_add, int64_t ld_add, const float *d_gain, float eps, int64_t rows, int32_t d,
                   void *d_q, void *d_scales, hipStream_t st)
{
    const int groups = (int)cdiv(d, kFp8Group);
    if (d <= kNarrow) {
        constexpr int R = 2;
        const bool two = d > kFp8Block;
        const auto kernel = two ? rmsnorm_fp8_narrow_kernel<T, TAdd, 32, R> : rmsnorm_fp8_narrow_kernel<T, TAdd, 16, R>;
        hipLaunchKernelGGL(kernel, grid_of(cdiv(rows, (two ? 8 : 16) * R)), dim3(256), 0, st, static_cast<T *>(d_x), ldx,
                           static_cast<const TAdd *>(d_add), ld_add, d_gain, eps, (uint32_t)rows, d, static_cast<unsigned char *>(d_q),
                           static_cast<uint32_t *>(d_scales));
        HIP_TRY(hipGetLastError());
        return SRM_OK;
    }
#define RMS_CASE(NW, G) return launch_rmsnorm<T, TAdd, NW, G>(d_x, ldx, d_add, ld_add, d_gain, eps, rows, d, d_q, d_scales, st)
    if (groups <= 1) RMS_CASE(1, 1);
    if (groups <= 2) RMS_CASE(1, 2);
    if (groups <= 4) RMS_CASE(2, 2);
    if (groups <= 8) RMS_CASE(4, 2);
    if (groups <= 16) RMS_CASE(8, 2);
    if (groups <= 32) RMS_CASE(16, 2);
    RMS_CASE(16, 4);
#undef RMS_CASE
}

extern "C" int srm_rmsnorm_fp8(int32_t dtype, void *d_x, int64_t ldx, int32_t add_dtype, const void *d_add, int64_t ld_add,
                               const float *d_gain, float eps, int64_t rows, int32_t d, void *d_q, void *d_scales, void *hip_stream)
{
    const char *who = "srm_rmsnorm_fp8";
    if (!d_x || !d_gain) return fail(SRM_EINVAL, "%s: null argument", who);
    SRM_TRY(check_fp8(who, d_q, d_scales));
    if (rows <= 0 || rows >= kMaxRows || d <= 0 || d > kMaxNorm) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (ldx < d || (d_add && ld_add < d)) return fail(SRM_EINVAL, "%s: a row stride is less than %d", who, d);
    if (!(eps >= 0.0f)) return fail(SRM_EINVAL, "%s: eps must not be negative", who);
    if (!d_add) add_dtype = dtype;
    if ((dtype != SRM_FP32 && dtype != SRM_BF16) || (add_dtype != SRM_FP32 && add_dtype != SRM_BF16))
        return fail(SRM_EINVAL, "%s: unknown dtype %d, %d", who, dtype, add_dtype);
    if (misaligned(d_x, size_of(dtype)) || misaligned(d_add, size_of(add_dtype)) || misaligned(d_gain, 4)) return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    hipStream_t st = as_stream(hip_stream);
    if (dtype == SRM_FP32)
        return add_dtype == SRM_FP32 ? rmsnorm<float, float>(d_x, ldx, d_add, ld_add, d_gain, eps, rows, d, d_q, d_scales, st)
                                     : rmsnorm<float, bf16>(d_x, ldx, d_add, ld_add, d_gain, eps, rows, d, d_q, d_scales, st);
    return add_dtype == SRM_FP32 ? rmsnorm<bf16, float>(d_x, ldx, d_add, ld_add, d_gain, eps, rows, d, d_q, d_scales, st)
                                 : rmsnorm<bf16, bf16>(d_x, ldx, d_add, ld_add, d_gain, eps, rows, d, d_q, d_scales, st);
}

// ------------------------------------------------------------------ their products
struct Fp8Call {
    const unsigned char *a;
    const uint32_t *sa;
    const unsigned char *w;
    const uint32_t *sw;
    int64_t M;
    int N, Kp;
    Fp8Epi ep;
    hipStream_t st;
};
static int device_cus()
{
    static thread_local int dev_of = -1, cus_of = 0;
    int dev = 0;
    if (hipGetDevice(&dev) != hipSuccess) return 0;
    if (dev != dev_of) {
        int cus = 0;
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess) return 0;
        dev_of = dev;
        cus_of = cus;
    }
    return cus_of;
}

template <auto KERN>
static int launch_fp8(int64_t blocks, int threads, int lds, const Fp8Call &c)
{
    if (blocks >= (1 << 30)) return fail(SRM_EINVAL, "srm_linear_fp8: sizes out of range");
    static std::atomic<uint64_t> set_on{0};          // devices, by number
    int dev = 0;
    HIP_TRY(hipGetDevice(&dev));
    if (!(set_on.load(std::memory_order_acquire) >> (dev & 63) & 1)) {
        HIP_TRY(hipFuncSetAttribute(reinterpret_cast<const void *>(KERN), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
        set_on.fetch_or(1ull << (dev & 63), std::memory_order_release);
    }
    hipLaunchKernelGGL(KERN, grid_of(blocks), dim3(threads), lds, c.st, c.a, c.sa, c.w, c.sw, c.M, c.N, c.Kp, c.ep);
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}
template <int BM, int BN, int WM, int WN, int NS, int EPI>
static int launch_fp8_tile(const Fp8Call &c)
{
    return launch_fp8<gemm_fp8_tile_kernel<BM, BN, WM, WN, NS, EPI>>(cdiv(c.M, BM) * cdiv(c.N, BN), WM * WN * 64, NS * fp8_stage_bytes<BM, BN>(), c);
}
template <int EPI>
static int launch_fp8_persist(const Fp8Call &c, int64_t cus)
{
    if (cdiv(c.M, 256) * cdiv(c.N, 256) >= (1 << 30)) return fail(SRM_EINVAL, "srm_linear_fp8: sizes out of range");
    return launch_fp8<gemm_fp8_persist_kernel<EPI>>(std::min(cdiv(c.M, 256) * cdiv(c.N, 256), cus), 512, kFp8PersistLds, c);
}
template <int RT, int CT, int NS, int EPI>
static int launch_fp8_slices(const Fp8Call &c)
{
    return launch_fp8<gemm_fp8_slices_kernel<RT, CT, NS, EPI>>(cdiv(c.M, 16 * RT) * cdiv(c.N, 16 * CT), kFp8SliceWaves * 64,
                                                              kFp8SliceWaves * fp8_slice_lds<RT, CT, NS>(), c);
}
// Which kernel.  Measured (graphs of launches over matrices in turn, us, rows x columns x K):
//   K cut over the wavefronts while a launch is one round of the chip: 16x16 | 32x32 | 64x64 | 64x64 tile of four wavefronts:
//     64 x 1024 x 4096 4.2 | 5.4 | 9.0 | 14.0; 37 x 4096 x 1024 4.9 | 3.6 | 5.2 | 5.3; 700 x 1024 x 4096 21 | 11.7 | 9.6 | 14.3;
//     300 x 4096 x 1024 20 | 9.4 | 9.3 | 6.7 (two rounds of the 64x64 form)
//   up to 16 rows of many columns are bound by reading W: 16x32 | 16x16 | 32x32: 16 x 32000 x 4096 28.3 | 30.0 | 29.5, 1 x 32000 x 1024
//     8.4 | 11.4 | 9.2 (W at 3.9 to 5.9 TB/s)
//   64x64 with a ring of two | four | 128x128: 300 x 4096 x 1024 6.7 | 6.9 | 8.6, 2048 x 1024 x 4096 18.1 | 17.5 | 23.8, 700 x 4096 x 1024
//     9.0 | 11.1 | 9.4, 1024 x 4096 x 4096 33.0 | 36.6 | 30.4; 64x128 once there are three for each two CUs: 3755 x 872 x 1152 9.7 | 11.0 with 64x64,
//     2620 x 1446 x 1024 with fp32 output 14.8 | 15.1 (882 x 1584 x 768, one for each 1.4: 12.4 | 9.5)
//   256x256 persistent | 128x128 by eight wavefronts: 8192^3 412 | 582, 4096^3 55.5 | 85, 3001 x 4001 x 1024 18.2 | 19.7, but 2048 x 4096 x 4096
//     (128 tiles for 256 CUs) 47.5 | 39.7: a tile of 256x256 takes 0.7 of the time of four tiles of 128x128, two of which a CU holds;
//     with two blocks of K 0.5: 10837 x 1721 x 256 19.5 | 15.7, 8192 x 2048 x 256 13.2 | 13.1
//   fp32 outputs, 128x128 by four | eight wavefronts: 8192^3 892 | 1010, 16384 x 1024 x 4096 (+=) 133 | 143, 3001 x 4001 x 1024 (+=) 39.9 | 35.4;
//     64x128 while three of them on each CU take a launch in one round, or else 128x64 | the better of those two: 1500 x 4096 x 2048 29.7 | 33.3,
//     (+=) 34.7 | 38.8, 3000 x 2048 x 8192 106 | 115, 26464 x 156 x 6016 81 | 88 (9000 x 700 x 1024, not one round: 21.9 | 20.1);
//     two blocks of K, 64x64 | 64x128 | 128x128: 8192 x 2048 x 256 18.8 | 17.8 | 20.3, (+=) 25.2 | 27.6 | 31.1, 16384 x 1024 x 128 (+=) 23.5 | 25.2 | 24.0
template <int EPI>
static int linear_fp8(const Fp8Call &c)
{
    const int64_t cus = device_cus();
    if (cus <= 0) return fail(SRM_EHIP, "cannot read the number of compute units");
    auto tiles = [&](int bm, int bn) { return cdiv(c.M, bm) * cdiv(c.N, bn); };
    if (tiles(16, 16) <= cus) return launch_fp8_slices<1, 1, 2, EPI>(c);
    if (c.M <= 16) return launch_fp8_slices<1, 2, 1, EPI>(c);
    if (tiles(32, 32) <= 2 * cus) return launch_fp8_slices<2, 2, 1, EPI>(c);
    if (tiles(64, 64) <= cus) return launch_fp8_slices<4, 4, 1, EPI>(c);
    const int64_t rounds = cdiv(tiles(128, 128), 2 * cus);
    if constexpr (!kFp8Exact<EPI>) {
        if (c.Kp >= 256 && 10 * cdiv(tiles(256, 256), cus) <= (c.Kp > 256 ? 7 : 5) * rounds) return launch_fp8_persist<EPI>(c, cus);
    }
    if (tiles(128, 128) >= cus) {
        if constexpr (kFp8Exact<EPI>) {
            if (c.Kp <= 256) return EPI == EPI_RESID ? launch_fp8_tile<64, 64, 2, 2, 2, EPI>(c) : launch_fp8_tile<64, 128, 2, 2, 2, EPI>(c);
            if (tiles(64, 128) <= 3 * cus) return launch_fp8_tile<64, 128, 2, 2, 2, EPI>(c);
            if (tiles(128, 64) <= 3 * cus) return launch_fp8_tile<128, 64, 2, 2, 2, EPI>(c);
            if (tiles(128, 128) >= 2 * cus && (EPI == EPI_F32 || c.Kp >= 2048)) return launch_fp8_tile<128, 128, 2, 2, 2, EPI>(c);
        }
        return launch_fp8_tile<128, 128, 2, 4, 2, EPI>(c);
    }
    if (2 * tiles(64, 128) >= 3 * cus) return launch_fp8_tile<64, 128, 2, 2, 2, EPI>(c);
    return tiles(64, 64) <= 2 * cus ? launch_fp8_tile<64, 64, 2, 2, 4, EPI>(c) : launch_fp8_tile<64, 64, 2, 2, 2, EPI>(c);
}

extern "C" int srm_linear_fp8(int32_t epilogue, const void *d_a, const void *d_a_scales, const void *d_w, const void *d_w_scales,
                              const float *d_bias, int64_t M, int32_t N, int32_t K, void *d_out, void *hip_stream)
{
    const char *who = "srm_linear_fp8";
    SRM_TRY(check_fp8(who, d_a, d_a_scales));
    SRM_TRY(check_fp8(who, d_w, d_w_scales));
    if (!d_out) return fail(SRM_EINVAL, "%s: null output", who);
    if (M <= 0 || M >= kMaxRows || N <= 0 || N >= kMaxRows || K <= 0 || K > kMaxWidth) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (misaligned(d_out, epilogue == 0 || epilogue == 1 ? 2 : 4) || misaligned(d_bias, 4))
        return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    const Fp8Call c{static_cast<const unsigned char *>(d_a), static_cast<const uint32_t *>(d_a_scales), static_cast<const unsigned char *>(d_w),
                    static_cast<const uint32_t *>(d_w_scales), M, N, (int)align_up(K, kFp8Block), Fp8Epi{d_bias, d_out, N},
                    as_stream(hip_stream)};
    switch (epilogue) {
    case 0: return linear_fp8<EPI_STORE>(c);
    case 1: return linear_fp8<EPI_GELU>(c);
    case 2: return linear_fp8<EPI_RESID>(c);
    case 4: return linear_fp8<EPI_F32>(c);
    default: return fail(SRM_EINVAL, "%s: unknown epilogue %d", who, epilogue);
    }
}

// ------------------------------------------------------------------ sampling by request
// Work-groups of 1024 threads while each row has a CU of its own, behind that of 512, of which a CU holds two; rows of up to
// 512 logits by a wavefront each, and of up to 1024 where there are more than those work-groups take at once.
template <typename T>
static void launch_sample(const void *d_logits, const SampleRows &p, hipStream_t st)
{
    const T *logits = static_cast<const T *>(d_logits);
    if (p.V <= kSampleSegment) hipLaunchKernelGGL((sample_short_rows_kernel<T, 1>), grid_of(cdiv(p.rows, 4)), dim3(256), 0, st, logits, p);
    else if (p.V <= 2 * kSampleSegment && p.rows > 2 * device_cus()) hipLaunchKernelGGL((sample_short_rows_kernel<T, 2>), grid_of(cdiv(p.rows, 4)), dim3(256), 0, st, logits, p);
    else if (p.rows <= device_cus()) hipLaunchKernelGGL((sample_rows_kernel<T, 1024>), grid_of(p.rows), dim3(1024), 0, st, logits, p);
    else hipLaunchKernelGGL((sample_rows_kernel<T, 512>), grid_of(p.rows), dim3(512), 0, st, logits, p);
}

extern "C" int srm_sample_rows(int32_t dtype, const void *d_logits, int64_t ld, int64_t rows, int32_t vocab, const float *d_temperature,
                               const int32_t *d_top_k, const float *d_top_p, const float *d_min_p, const float *d_uniform,
                               int32_t *d_tok_out, float *d_logprob, void *hip_stream)
{
    const char *who = "srm_sample_rows";
    if (!d_logits || !d_uniform || !d_tok_out) return fail(SRM_EINVAL, "%s: null argument", who);
    if (rows <= 0 || rows >= kMaxRows || vocab <= 0 || vocab > kSampleVocab) return fail(SRM_EINVAL, "%s: sizes out of range", who);
    if (ld < vocab) return fail(SRM_EINVAL, "%s: row stride %lld is less than %d", who, (long long)ld, vocab);
    const void *const words[] = {d_temperature, d_top_k, d_top_p, d_min_p, d_uniform, d_tok_out, d_logprob};
    bool whole = !misaligned(d_logits, size_of(dtype));
    for (const void *w : words) whole = whole && !misaligned(w, 4);
    if (!whole) return fail(SRM_EINVAL, "%s: %s", who, kNotWhole);
    const SampleRows p{rows, ld, vocab, d_temperature, d_top_p, d_min_p, d_uniform, d_top_k, d_tok_out, d_logprob};
    hipStream_t st = as_stream(hip_stream);
    if (dtype == SRM_FP32) launch_sample<float>(d_logits, p, st);
    else if (dtype == SRM_BF16) launch_sample<bf16>(d_logits, p, st);
    else return fail(SRM_EINVAL, "%s: unknown dtype %d", who, dtype);
    HIP_TRY(hipGetLastError());
    return SRM_OK;
}
