// GEMMs of 8-bit rows: out = epilogue(A W^T + bias), A [M][Kp] and W [N][Kp] in e4m3 with E8M0 scales for blocks of 128 (fp8.hpp):
//   out[m][n] = epi(sum_b 2^(sa[m][b] + sw[n][b] - 254) sum_{k in block b} a[m][k] w[n][k] + bias[n])
//
// Two ways to the sum, by the type of the output:
//   bf16 (EPI_STORE, EPI_GELU): v_mfma_scale_f32_16x16x128_f8f6f4, whose K is a block; a lane hands it the scales of its row of A and of
//     its row of W with the operands, and the fp32 accumulation runs on over all of K.  The instruction adds the eight products of a
//     lane's 64-bit words in a window of some 14 bits below the largest (2^16 + 2^3 is held, 2^16 + 2^2 is not, whichever fp8
//     instruction; random rows: 1.3e-5 of the result's norm), which a bf16 output's rounding of 2^-9 hides.
//   fp32 (EPI_RESID, EPI_F32): the operands are widened to bf16 with their scales (v_cvt_scalef32_pk_bf16_fp8: exact for scales from
//     2^-117 to 2^119) and multiplied by v_mfma_f32_16x16x32_bf16, which holds products and sums in fp32 (random rows: 8e-8), at half
//     the rate.
// Products are formed transposed (W as the first operand), so that a lane holds four consecutive columns of one row.
#pragma once
#include "fp8.hpp"
#include "tile.hpp"

typedef __attribute__((ext_vector_type(8))) int i32x8_t;

struct Fp8Epi {
    const float *bias;                               // [N] or nullptr
    void *out;                                       // [M][N]: bf16 (EPI_STORE, EPI_GELU), fp32 (EPI_RESID: +=, EPI_F32)
    int N;
};
template <int EPI>
constexpr bool kFp8Exact = EPI == EPI_RESID || EPI == EPI_F32;

// Columns col .. col + 3 of a row, those that exist; at any multiple of an element.
template <int EPI>
__device__ __forceinline__ void fp8_store4(const Fp8Epi &ep, int64_t row, int col, f32x4_t v)
{
    if (col >= ep.N) return;
    const int64_t at = row * ep.N + col;
    if constexpr (EPI == EPI_GELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gelu_bf16out(v[i]);
    }
    if (col + 4 <= ep.N) {
        if constexpr (kFp8Exact<EPI>) {
            float *p = static_cast<float *>(ep.out) + at;
            if constexpr (EPI == EPI_RESID) {
                f32x4_t o;
                __builtin_memcpy(&o, p, 16);
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] += o[i];
            }
            __builtin_memcpy(p, &v, 16);
        } else {
            const bf16x4_t o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
            __builtin_memcpy(static_cast<bf16 *>(ep.out) + at, &o, 8);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (col + i >= ep.N) break;
        if constexpr (EPI == EPI_RESID) static_cast<float *>(ep.out)[at + i] += v[i];
        else if constexpr (EPI == EPI_F32) static_cast<float *>(ep.out)[at + i] = v[i];
        else static_cast<bf16 *>(ep.out)[at + i] = (bf16)v[i];
    }
}
__device__ __forceinline__ f32x4_t fp8_bias4(const Fp8Epi &ep, int col)
{
    f32x4_t b = {0.f, 0.f, 0.f, 0.f};
    if (ep.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = ep.bias[min(col + i, ep.N - 1)];
    }
    return b;
}

// Sixteen e4m3 values (four words) -> two operands of eight bf16, times the scale of byte `s`.
__device__ __forceinline__ void fp8_widen(u32x4_t x, uint32_t s, bf16x8_t (&out)[2])
{
    const float f = __uint_as_float(s << 23);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const bf16x2_t lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[2 * h + i], f, false);
            const bf16x2_t hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x[2 * h + i], f, true);
            out[h][4 * i] = lo[0]; out[h][4 * i + 1] = lo[1]; out[h][4 * i + 2] = hi[0]; out[h][4 * i + 3] = hi[1];
        }
}

// acc[i][j] += the products of one block (128 of K): rows i of A, columns j of W, raw operands and scale bytes of this lane's rows.
// A lane holds the chunks lane / 16 and lane / 16 + 4 of 16 bytes of its row: the order of k within a block is the same in A and W.
template <bool EXACT, int TM, int TN>
__device__ __forceinline__ void fp8_products(f32x4_t (&acc)[TM][TN], const u32x4_t (&a)[TM][2], const u32x4_t (&w)[TN][2],
                                             const uint32_t (&sa)[TM], const uint32_t (&sw)[TN])
{
    if constexpr (EXACT) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            bf16x8_t fw[TN][2];
#pragma unroll
            for (int j = 0; j < TN; ++j) fp8_widen(w[j][h], sw[j], fw[j]);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                bf16x8_t fa[2];
                fp8_widen(a[i][h], sa[i], fa);
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int q = 0; q < 2; ++q) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(fw[j][q], fa[q], acc[i][j], 0, 0, 0);
            }
        }
    } else {
        auto whole = [](const u32x4_t (&x)[2]) {
            return i32x8_t{(int)x[0][0], (int)x[0][1], (int)x[0][2], (int)x[0][3], (int)x[1][0], (int)x[1][1], (int)x[1][2], (int)x[1][3]};
        };
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)             // formats 0: e4m3; byte 0 of the scales' registers
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(whole(w[j]), whole(a[i]), acc[i][j], 0, 0, 0, (int)sw[j], 0, (int)sa[i]);
    }
}

// A buffer descriptor of `bytes` bytes: loads behind them arrive as zeros.
__device__ __forceinline__ u32x4_t fp8_descriptor(const void *base, int bytes)
{
    u32x4_t rs;
    const unsigned long long a = reinterpret_cast<unsigned long long>(base);
    rs[0] = __builtin_amdgcn_readfirstlane((unsigned)a);
    rs[1] = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));                 // stride 0: raw buffer
    rs[2] = __builtin_amdgcn_readfirstlane((unsigned)bytes);
    rs[3] = 0x00020000u;
    return rs;
}
// Loads from memory to LDS are issued from asm statements: a load that the compiler knows to write LDS makes it wait for all
// outstanding loads in front of the next LDS read that it cannot prove disjoint.  The waits are explicit (FP8_WAIT_LOADS).
// 16 bytes of every lane to 1024 bytes at LDS address `dst`, in the lanes' order.
__device__ __forceinline__ void fp8_dma16(unsigned dst, const u32x4_t &rs, int voff, int soff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(dst), "v"(voff), "s"(rs), "s"(soff) : "memory");
}
// 4 bytes of every lane to 256 bytes.
__device__ __forceinline__ void fp8_dma4(unsigned dst, const u32x4_t &rs, int voff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" : : "s"(dst), "v"(voff), "s"(rs) : "memory");
}
// all but the youngest n loads have landed
#define FP8_WAIT_LOADS(n) asm volatile("s_waitcnt vmcnt(%0)" : : "i"(n) : "memory")

__device__ __forceinline__ unsigned fp8_lds_address(const void *p)
{
    typedef __attribute__((address_space(3))) const unsigned char lds_byte;
    return __builtin_amdgcn_readfirstlane((unsigned)reinterpret_cast<unsigned long long>((lds_byte *)p));
}

// ------------------------------------------------------------------ tiles
// A BM x BN tile by WM x WN wavefronts; blocks of K (128 bytes of a row) pass through a ring of NS stages in LDS, NS - 1 of them on their
// way.  A stage holds BM + BN rows of 128 bytes, 16-byte chunk c of row r at chunk c ^ swz(r), and behind them the word of scales of each
// row (the word of four blocks, loaded again for each of them).
template <int BM, int BN>
constexpr int fp8_stage_bytes() { return (BM + BN) * (128 + 4); }

template <int BM, int BN, int WM, int WN, int NS, int EPI>
__global__ void __launch_bounds__(WM *WN * 64, 2)
gemm_fp8_tile_kernel(const unsigned char *__restrict__ A, const uint32_t *__restrict__ sa, const unsigned char *__restrict__ W,
                     const uint32_t *__restrict__ sw, int64_t M, int N, int Kp, Fp8Epi ep)
{
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int LOADS = (BM + BN) / 8 / NW, WORDS = (BM + BN) / 64;            // tile loads of a wavefront, scale loads of the work-group
    static_assert((BM + BN) % (8 * NW) == 0 && BM % 64 == 0 && BN % 64 == 0 && WORDS % NW == 0 && BM % (8 * NW) == 0, "whole loads");
    constexpr int PER_STAGE = LOADS + WORDS / NW;
    extern __shared__ __align__(16) unsigned char fp8_smem[];
    const unsigned lds = fp8_lds_address(fp8_smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, lr = lane & 15, lq = lane >> 4;
    int bm, bn;
    tile_of_pid(blockIdx.x, (int)((M + BM - 1) / BM), (N + BN - 1) / BN, bm, bn);
    const int64_t m0 = (int64_t)bm * BM;
    const int n0 = bn * BN, rows = (int)min((int64_t)BM, M - m0), cols = min(BN, N - n0), KT = Kp / 128;
    const u32x4_t ra = fp8_descriptor(A + m0 * Kp, rows * Kp), rw = fp8_descriptor(W + (int64_t)n0 * Kp, cols * Kp);
    const int ld_r = lane >> 3, ld_c = lane & 7;

    auto load = [&](int kt) {
        const unsigned stage = lds + (unsigned)(kt % NS) * fp8_stage_bytes<BM, BN>();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            // eight rows of A or W: lane (r, slot) fetches chunk slot ^ swz(r)
            const int r0 = (i * NW + wave) * 8, r = r0 + ld_r;
            const bool is_a = i < BM / 8 / NW;
            const int row = is_a ? r : r - BM;
            fp8_dma16(stage + r0 * 128, is_a ? ra : rw, row * Kp + ((ld_c ^ swz_of_row(r)) << 4), kt * 128);
        }
#pragma unroll
        for (int i = 0; i < WORDS / NW; ++i) {
            const int g0 = (i * NW + wave) * 64;
            const bool is_a = g0 < BM;
            const int64_t at = is_a ? (int64_t)(kt >> 2) * M + m0 : (int64_t)(kt >> 2) * N + n0;
            fp8_dma4(stage + (BM + BN) * 128 + g0 * 4, fp8_descriptor((is_a ? sa : sw) + at, (is_a ? rows : cols) * 4),
                     (g0 - (is_a ? 0 : BM) + lane) * 4);
        }
    };
    f32x4_t acc[TM][TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const f32x4_t b = fp8_bias4(ep, n0 + wn * (BN / WN) + j * 16 + 4 * lq);
#pragma unroll
        for (int i = 0; i < TM; ++i) acc[i][j] = b;
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);              // the bias has arrived: loads are counted from here on
    __builtin_amdgcn_sched_barrier(0);
    for (int kt = 0; kt < NS - 1 && kt < KT; ++kt) load(kt);
    for (int kt = 0; kt < KT; ++kt) {
        if (kt + NS - 2 < KT) FP8_WAIT_LOADS((NS - 2) * PER_STAGE);
        else FP8_WAIT_LOADS(0);
        __syncthreads();                             // the stage has landed for everyone, and the one before has been read
        if (kt + NS - 1 < KT) load(kt + NS - 1);
        const unsigned char *stage = fp8_smem + kt % NS * fp8_stage_bytes<BM, BN>();
        const uint32_t *words = reinterpret_cast<const uint32_t *>(stage + (BM + BN) * 128);
        u32x4_t fa[TM][2], fw[TN][2];
        uint32_t va[TM], vw[TN];
        auto read = [&](int r, u32x4_t (&f)[2], uint32_t &s) {
#pragma unroll
            for (int h = 0; h < 2; ++h) f[h] = *reinterpret_cast<const u32x4_t *>(stage + r * 128 + (((h * 4 + lq) ^ swz_of_row(r)) << 4));
            s = words[r] >> (kt & 3) * 8 & 255;
        };
#pragma unroll
        for (int j = 0; j < TN; ++j) read(BM + wn * (BN / WN) + j * 16 + lr, fw[j], vw[j]);
#pragma unroll
        for (int i = 0; i < TM; ++i) read(wm * (BM / WM) + i * 16 + lr, fa[i], va[i]);
        fp8_products<kFp8Exact<EPI>>(acc, fa, fw, va, vw);
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int64_t row = m0 + wm * (BM / WM) + i * 16 + lr;
        if (row >= M) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) fp8_store4<EPI>(ep, row, n0 + wn * (BN / WN) + j * 16 + 4 * lq, acc[i][j]);
    }
}

// ------------------------------------------------------------------ few tiles: K cut over the wavefronts
// A launch with at most a tile for each CU takes as long as one tile's trip through K.  Here eight wavefronts cut K between them, each
// with its own blocks for the whole (16 RT) x (16 CT) tile through a ring of NS stages of its own, without a barrier; the partial
// tiles meet in LDS and are added in the wavefronts' order.
template <int RT, int CT>
constexpr int fp8_slice_stage() { return 16 * (RT + CT) * 128 + 512; }           // two loads of 64 words of scales
template <int RT, int CT, int NS>
constexpr int fp8_slice_lds()
{
    constexpr int ring = NS * fp8_slice_stage<RT, CT>(), part = 16 * RT * (16 * CT + 4) * 4;
    return ring > part ? ring : part;
}
constexpr int kFp8SliceWaves = 8;
template <int RT, int CT, int NS, int EPI>
__global__ void __launch_bounds__(kFp8SliceWaves * 64, 2)
gemm_fp8_slices_kernel(const unsigned char *__restrict__ A, const uint32_t *__restrict__ sa, const unsigned char *__restrict__ W,
                       const uint32_t *__restrict__ sw, int64_t M, int N, int Kp, Fp8Epi ep)
{
    constexpr int NW = kFp8SliceWaves, BM = 16 * RT, BN = 16 * CT, RS = BN + 4;  // row stride of a partial tile, floats
    constexpr int LOADS = (BM + BN) / 8, PER_STAGE = LOADS + 2, WAVE = fp8_slice_lds<RT, CT, NS>();
    extern __shared__ __align__(16) unsigned char fp8_smem[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lr = lane & 15, lq = lane >> 4;
    int bm, bn;
    tile_of_pid(blockIdx.x, (int)((M + BM - 1) / BM), (N + BN - 1) / BN, bm, bn);
    const int64_t m0 = (int64_t)bm * BM;
    const int n0 = bn * BN, rows = (int)min((int64_t)BM, M - m0), cols = min(BN, N - n0), KT = Kp / 128;
    const u32x4_t ra = fp8_descriptor(A + m0 * Kp, rows * Kp), rw = fp8_descriptor(W + (int64_t)n0 * Kp, cols * Kp);
    unsigned char *ring = fp8_smem + wave * WAVE;
    const unsigned lds = fp8_lds_address(fp8_smem) + wave * WAVE;
    const int first = wave * KT / NW, steps = (wave + 1) * KT / NW - first;
    auto load = [&](int s) {
        const int kt = first + s;
        const unsigned stage = lds + (unsigned)(s % NS) * fp8_slice_stage<RT, CT>();
#pragma unroll
        for (int i = LOADS - 1; i >= 0; --i) {       // W first
            const int r = i * 8 + (lane >> 3);
            const bool is_a = i * 8 < BM;
            fp8_dma16(stage + i * 1024, is_a ? ra : rw, (is_a ? r : r - BM) * Kp + (((lane & 7) ^ swz_of_row(r)) << 4), kt * 128);
        }
        fp8_dma4(stage + LOADS * 1024, fp8_descriptor(sa + (int64_t)(kt >> 2) * M + m0, rows * 4), lane * 4);
        fp8_dma4(stage + LOADS * 1024 + 256, fp8_descriptor(sw + (int64_t)(kt >> 2) * N + n0, cols * 4), lane * 4);
    };
    f32x4_t acc[RT][CT];
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < NS && s < steps; ++s) load(s);
    for (int s = 0; s < steps; ++s) {
        if (s + NS <= steps) FP8_WAIT_LOADS((NS - 1) * PER_STAGE);
        else FP8_WAIT_LOADS(0);
        const unsigned char *stage = ring + s % NS * fp8_slice_stage<RT, CT>();
        const uint32_t *words = reinterpret_cast<const uint32_t *>(stage + LOADS * 1024);
        u32x4_t fa[RT][2], fw[CT][2];
        uint32_t va[RT], vw[CT];
        const int shift = ((first + s) & 3) * 8;
        auto read = [&](int r, u32x4_t (&f)[2]) {
#pragma unroll
            for (int h = 0; h < 2; ++h) f[h] = *reinterpret_cast<const u32x4_t *>(stage + r * 128 + (((h * 4 + lq) ^ swz_of_row(r)) << 4));
        };
#pragma unroll
        for (int j = 0; j < CT; ++j) { read(BM + j * 16 + lr, fw[j]); vw[j] = words[64 + j * 16 + lr] >> shift & 255; }
#pragma unroll
        for (int i = 0; i < RT; ++i) { read(i * 16 + lr, fa[i]); va[i] = words[i * 16 + lr] >> shift & 255; }
        fp8_products<kFp8Exact<EPI>>(acc, fa, fw, va, vw);
        __builtin_amdgcn_sched_barrier(0);
        if (s + NS < steps) {
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");       // the stage has been read
            load(s + NS);
        }
    }
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");               // the ring becomes the partial tile
    float *mine = reinterpret_cast<float *>(ring);
#pragma unroll
    for (int i = 0; i < RT; ++i)
#pragma unroll
        for (int j = 0; j < CT; ++j) *reinterpret_cast<f32x4_t *>(mine + (16 * i + lr) * RS + 16 * j + 4 * lq) = acc[i][j];
    __syncthreads();
    const float *part = reinterpret_cast<const float *>(fp8_smem);
    for (int g = tid; g < BM * (BN / 4); g += NW * 64) {
        const int r = g / (BN / 4), c = g % (BN / 4) * 4;
        if (m0 + r >= M || n0 + c >= N) continue;
        f32x4_t v = fp8_bias4(ep, n0 + c);
#pragma unroll
        for (int w = 0; w < NW; ++w) v += *reinterpret_cast<const f32x4_t *>(part + w * (WAVE / 4) + r * RS + c);
        fp8_store4<EPI>(ep, m0 + r, n0 + c, v);
    }
}
