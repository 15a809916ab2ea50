// What the matrix kernels of all types share: epilogue codes, the order of output tiles, the LDS layout of operand tiles.
#pragma once
#include "common.hpp"
#include <type_traits>

enum { EPI_STORE = 0, EPI_GELU = 1, EPI_RESID = 2, EPI_ARGMAX = 3, EPI_F32 = 4, EPI_MIX = 5, EPI_RESID_LN = 6 };

// Block -> tile mapping.  Workgroups are dealt round-robin to the 8 XCDs, each
// with its own L2: give every XCD one contiguous run of tiles, and inside a run
// walk groups of GM row-tiles column by column so the A rows of a group and the
// W tile being shared stay L2-resident.
__device__ __forceinline__ void tile_of_pid(int pid, int nbm, int nbn, int &bm, int &bn)
{
    constexpr int GM = 8;
    const int nblk = nbm * nbn;
    if ((nblk & 7) == 0) pid = (pid & 7) * (nblk >> 3) + (pid >> 3);
    const int gsz = GM * nbn;
    const int g = pid / gsz;
    const int first_m = g * GM;
    const int gm = min(nbm - first_m, GM);
    const int in_g = pid - g * gsz;
    bm = first_m + in_g % gm;
    bn = in_g / gm;
}

// LDS chunk swizzle: 16-byte chunk c of row r sits at chunk c ^ ((r >> 1) & 7);
// with 64 banks this makes both the tile writes and the fragment reads
// conflict-free (measured: SQ_LDS_BANK_CONFLICT ~1% of SQ_LDS_IDX_ACTIVE).
__device__ __forceinline__ int swz_of_row(int r) { return (r >> 1) & 7; }

// f(integral_constant<int, I>) for I = FIRST .. LAST-1, unrolled by construction
template <int FIRST, int LAST, typename F>
__device__ __forceinline__ void static_for(F &&f)
{
    if constexpr (FIRST < LAST) {
        f(std::integral_constant<int, FIRST>{});
        static_for<FIRST + 1, LAST>(f);
    }
}

// Exact (erf) GELU for bf16 outputs: x * Phi(x) with erfc(|x| / sqrt(2)) / 2 = 2^-P(|x|), |x| clamped to
// 4.3 * sqrt(2) (beyond it Phi is 0 or 1 to 1e-9), P a degree-6 polynomial fitted to
// -log2(erfc(z) / 2), z = |x| / sqrt(2) (minimax in the absolute error of erfc: 2.2e-7; |error| of the
// GELU value <= 6.5e-7 in fp32 evaluation; the 1 / sqrt(2) is folded into the coefficients), so one exp2
// and six FMAs, no reciprocal.  With q = 2^-P: x * (1 - q) for x >= 0 and x * q for x < 0 are both
// max(x, 0) - |x| * q, one max and one FMA instead of a subtraction, a compare, a select and a
// product.  The result is rounded to bf16 (relative 2^-8) right after, so the approximation error is
// invisible there.  |x| is the clamped one in the product too: beyond the clamp the result is max(x, 0) - 3.3e-9, for
// infinities as for finite values (the magnitude itself times q would grow without bound, and be NaN for +infinity).
// The minimum is the instruction that keeps a NaN, which then is all that follows from it.
__device__ __forceinline__ float gelu_bf16out(float x)
{
    // Ten instructions, written out: from the C form the compiler made 14 to 18 per element (a
    // NaN-quieting max in front of each min / max, whose inputs come straight from LDS, and a move per
    // constant in every other Horner chain), and this epilogue is bound by its instruction count.
    //   w = min(|x|, 6.0811183)                       P(w) by Horner, coefficients high to low:
    //   -1.917465077776602e-05, 0.0006586045579087176, -0.00775440879176911, 0.05296539231773387,
    //   0.4590602540550674, 1.1511220519383694, 0.9999996936263803
    //   q = 2^-P ;  result = max(x, 0) - w * q
    float w, p, q, r;
    const float c5 = 0.0006586045579087176f, clamp = 6.0811183f;
    asm("v_minimum3_f32 %0, |%4|, %6, %6\n\t"
        "v_fmamk_f32 %1, %0, 0xb7a0d940, %5\n\t"
        "v_fmaak_f32 %1, %0, %1, 0xbbfe18b2\n\t"
        "v_fmaak_f32 %1, %0, %1, 0x3d58f23d\n\t"
        "v_fmaak_f32 %1, %0, %1, 0x3eeb09f2\n\t"
        "v_fmaak_f32 %1, %0, %1, 0x3f9357f8\n\t"
        "v_fmaak_f32 %1, %0, %1, 0x3f7ffffb\n\t"
        "v_exp_f32_e64 %2, -%1\n\t"
        "v_max_f32 %3, 0, %4\n\t"
        "v_fma_f32 %3, -%0, %2, %3"
        : "=&v"(w), "=&v"(p), "=&v"(q), "=&v"(r)
        : "v"(x), "v"(c5), "s"(clamp));
    return r;
}
