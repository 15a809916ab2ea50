// GEMMs of 8-bit rows: out = epilogue(A W^T + bias), A [M][Kp] and W [N][Kp] in e4m3 with E8M0 scales for blocks of 128 (fp8.hpp):
//   out[m][n] = epi(sum_b 2^(sa[m][b] + sw[n][b] - 254) sum_{k in block b} a[m][k] w[n][k] + bias[n])
//
// Two ways to the sum, by the type of the output:
//   bf16 (EPI_STORE, EPI_GELU): v_mfma_scale_f32_16x16x128_f8f6f4, whose K is a block; a lane hands it the scales of its row of A and of
//     its row of W with the operands, and the fp32 accumulation runs on over all of K.  The instruction adds the eight products of a
//     lane's 64-bit words (eight consecutive k) without what lies below 2^-13 of the largest (2^16 + 2^3 is held, 2^16 + 2^2 is not,
//     whichever fp8 instruction), and those sums to each other and to what is accumulated in fp32 (2^16 + 2^-7 is held).  Taken for
//     its rate: on random rows it costs 1.3e-5 of the results' norm, beside 1.7e-3 of a bf16 output's rounding (2^-8 at most), so
//     that the error against 64 bits stays the same and one output in ninety is the neighbouring bf16 value of that from fp32 sums.
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

// Columns col .. col + 3 of a row, those that exist; at any multiple of an element.  What a store adds to is requested apart from it,
// so that several requests travel together.
template <int EPI>
__device__ __forceinline__ f32x4_t fp8_old4(const Fp8Epi &ep, int64_t row, int col)
{
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    if constexpr (EPI == EPI_RESID) {
        const float *p = static_cast<const float *>(ep.out) + row * ep.N + col;
        if (col + 4 <= ep.N) {
            __builtin_memcpy(&o, p, 16);
        } else {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (col + i < ep.N) o[i] = p[i];
        }
    }
    return o;
}
template <int EPI>
__device__ __forceinline__ void fp8_store4(const Fp8Epi &ep, int64_t row, int col, f32x4_t v, f32x4_t old)
{
    const int64_t at = row * ep.N + col;
    if constexpr (EPI == EPI_RESID) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] += old[i];
    }
    if constexpr (EPI == EPI_GELU) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gelu_bf16out(v[i]);
    }
    if (col + 4 <= ep.N) {
        if constexpr (kFp8Exact<EPI>) {
            __builtin_memcpy(static_cast<float *>(ep.out) + at, &v, 16);
        } else {
            const bf16x4_t o = {(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
            __builtin_memcpy(static_cast<bf16 *>(ep.out) + at, &o, 8);
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        if (col + i >= ep.N) break;
        if constexpr (kFp8Exact<EPI>) static_cast<float *>(ep.out)[at + i] = v[i];
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
// Bound by the trip through L2 and the LDS reads between two barriers, of which other work-groups on the CU fill part: two of 128x128, three of
// 64x128.  fp32 outputs besides by widening, two values an instruction: 8192^3 892 .. 967 us (1.1 .. 1.2 PFLOP/s; the bf16 product of the same
// size 1.46), 3001 x 4001 x 1000 with addition 36 us (matrix pipes busy for a quarter of it: 768 tiles are one and a half rounds, and the
// stored rows are read and written behind the last product; 39 .. 44 with operands and output from memory).  Not kept: the operands of the next block in registers meanwhile
// (128x128 spills, 128x64 gains nothing), what is added to requested in front of the first loads (+-2%).
template <int BM, int BN>
constexpr int fp8_stage_bytes() { return (BM + BN) * (128 + 4); }

template <int BM, int BN, int WM, int WN, int NS, int EPI>
__global__ void __launch_bounds__(WM *WN * 64, 2)
gemm_fp8_tile_kernel(const unsigned char *__restrict__ A, const uint32_t *__restrict__ sa, const unsigned char *__restrict__ W,
                     const uint32_t *__restrict__ sw, int64_t M, int N, int Kp, Fp8Epi ep)
{
    constexpr int NW = WM * WN, TM = BM / WM / 16, TN = BN / WN / 16;
    // tile loads of a wavefront; scale loads of the work-group and of a wavefront (where there are fewer than wavefronts, several of them
    // make the same one: every wavefront counts the same loads)
    constexpr int LOADS = (BM + BN) / 8 / NW, WORDS = (BM + BN) / 64, WORD_LOADS = (WORDS + NW - 1) / NW, PER_STAGE = LOADS + WORD_LOADS;
    static_assert((BM + BN) % (8 * NW) == 0 && BM % 64 == 0 && BN % 64 == 0 && BM % (8 * NW) == 0, "whole loads");
    extern __shared__ __align__(16) unsigned char fp8_smem[];
    const unsigned lds = fp8_lds_address(fp8_smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, lr = lane & 15, lq = lane >> 4;
    int bm, bn;
    const int nbm = (int)((M + BM - 1) / BM), nbn = (N + BN - 1) / BN, pid = (int)work_group();                       // < 2^30 + 2^21
    if (pid >= nbm * nbn) return;
    tile_of_pid(pid, nbm, nbn, bm, bn);
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
        for (int i = 0; i < WORD_LOADS; ++i) {
            const int g0 = (i * NW + wave) % WORDS * 64;
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
    // Sixteen rows at a time pass through a wave-private stage in LDS, 16-byte chunk c of row r at chunk c ^ r, so that a row's columns
    // are read and written side by side.
    constexpr int CHUNKS = TN * 4, AT_ONCE = 64 / CHUNKS;
    static_assert(NW * 16 * CHUNKS * 16 <= NS * fp8_stage_bytes<BM, BN>(), "the stages fit the ring");
    __syncthreads();                                 // the ring has been read
    f32x4_t *out_stage = reinterpret_cast<f32x4_t *>(fp8_smem) + wave * 16 * CHUNKS;
    const int o_row = lane / CHUNKS, o_chunk = lane % CHUNKS;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
#pragma unroll
        for (int j = 0; j < TN; ++j) out_stage[lr * CHUNKS + ((4 * j + lq) ^ (lr & (CHUNKS - 1)))] = acc[i][j];
        __builtin_amdgcn_wave_barrier();
        f32x4_t v[16 / AT_ONCE], old[16 / AT_ONCE];
        const int col = n0 + wn * (BN / WN) + o_chunk * 4;
#pragma unroll
        for (int it = 0; it < 16 / AT_ONCE; ++it)
            old[it] = fp8_old4<EPI>(ep, min(m0 + wm * (BM / WM) + i * 16 + it * AT_ONCE + o_row, M - 1), min(col, N - 1));
#pragma unroll
        for (int it = 0; it < 16 / AT_ONCE; ++it) {
            const int r = it * AT_ONCE + o_row;
            v[it] = out_stage[r * CHUNKS + (o_chunk ^ (r & (CHUNKS - 1)))];
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int it = 0; it < 16 / AT_ONCE; ++it) {
            const int64_t row = m0 + wm * (BM / WM) + i * 16 + it * AT_ONCE + o_row;
            if (row < M && col < N) fp8_store4<EPI>(ep, row, col, v[it], old[it]);
        }
    }
}

// ------------------------------------------------------------------ few tiles: K cut over the wavefronts
// A launch with at most a tile for each CU takes as long as one tile's trip through K.  Here eight wavefronts cut K between them, each
// with its own blocks for the whole (16 RT) x (16 CT) tile through a ring of NS stages of its own, without a barrier; the partial
// tiles meet in LDS and are added in the wavefronts' order.  Bound by latency (37 x 4096 x 1024: 3.7 us, of which an empty launch is 2), for
// one row by reading W: 1 x 32000 x 1024 5.2 us where the caches hold it, 8.4 (3.9 TB/s) where not.
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
    const int nbm = (int)((M + BM - 1) / BM), nbn = (N + BN - 1) / BN, pid = (int)work_group();                       // < 2^30 + 2^21
    if (pid >= nbm * nbn) return;
    tile_of_pid(pid, nbm, nbn, bm, bn);
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
        const f32x4_t old = fp8_old4<EPI>(ep, m0 + r, n0 + c);
#pragma unroll
        for (int w = 0; w < NW; ++w) v += *reinterpret_cast<const f32x4_t *>(part + w * (WAVE / 4) + r * RS + c);
        fp8_store4<EPI>(ep, m0 + r, n0 + c, v, old);
    }
}

// ------------------------------------------------------------------ large products with a bf16 output
// A 256 x 256 tile by eight wavefronts (2 x 4, 128 x 64 each, v_mfma_scale_f32_32x32x64_f8f6f4), persistent: one work-group per CU walks
// its tiles, and the LDS ring runs from one tile into the next.  The bytes move as in gemm_bf16_persist_kernel (gemm_persist.hpp): LDS is a
// ring of five units of 32 KB, each 256 rows x 128 bytes of A or W in the swizzled layout; block T has A in unit 2T mod 5 and W in unit
// 2T + 1 mod 5:
//     half 0 of T: products of its first 64 k | operands of its second half | loads of A of T+2 (unit 2T+4: W of T-1 is done)
//     half 1 of T, its first two products; barrier: T+1 has landed, T has been read by all
//     the others of the second 64 k | operands of T+1's first half | loads of W of T+2 (unit 2T: A of T is done)
// An operand of A is read for the next half behind the two products that use it in this one, into the same registers.  The ring is all of
// the LDS, so the scales are in registers: the words of four blocks for this lane's rows, the lowest byte in use, and those of the next
// four, requested when the last ones begin to be used.
// 8192^3: 408 .. 432 us (2.5 .. 2.7 PFLOP/s, the matrix pipes busy for 72% of the clocks at a sustained 1.7 GHz, where a bare loop of the
// instruction reaches 3.9 PFLOP/s), 418 with a wait for the stores of a tile in front of the next one's loads; 16384 x 1024 x 4096, one tile
// a CU, 59 .. 65 us (2.1 .. 2.3 PFLOP/s): the first loads and the last stores have nothing to hide behind.
constexpr int kFp8PersistLds = 160 * 1024;
template <int EPI>
__global__ void __launch_bounds__(512)
gemm_fp8_persist_kernel(const unsigned char *__restrict__ A, const uint32_t *__restrict__ sa, const unsigned char *__restrict__ W,
                        const uint32_t *__restrict__ sw, int64_t M, int N, int Kp, Fp8Epi ep)
{
    static_assert(!kFp8Exact<EPI>, "bf16 outputs");
    constexpr int BM = 256, BN = 256, WN = 4, WTM = 128, WTN = 64, TM = 4, TN = 2;
    constexpr int UNITS = 5, UNIT = 256 * 128, LD_IT = UNIT / 16 / 512;
    static_assert(UNITS * UNIT <= kFp8PersistLds, "the ring is the LDS");
    extern __shared__ __align__(16) unsigned char fp8_smem[];
    const unsigned ring = fp8_lds_address(fp8_smem);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN, l32 = lane & 31, lq = lane >> 5;
    const int nbm = (int)((M + BM - 1) / BM), nbn = (N + BN - 1) / BN, nblk = nbm * nbn;
    const int KT = Kp / 128, KG = (KT + 3) / 4;      // KT >= 2 (the launcher checks)

    // one wavefront's load: 8 rows x 128 bytes, lane (r = l >> 3, slot = l & 7) fetches chunk slot ^ swz(r) of its row.  The row is in the
    // lanes' offset, which the descriptor's size bounds by itself; the common one stays within a row, and is 0 for a tile that does not exist.
    const int ld_r = tid >> 3;
    int ld_voff[LD_IT];
#pragma unroll
    for (int i = 0; i < LD_IT; ++i) ld_voff[i] = (i * 64 + ld_r) * Kp + (((tid & 7) ^ swz_of_row(ld_r)) << 4);
    auto dma_one = [&](int i, const u32x4_t &rs, int kt, unsigned unit) {
        fp8_dma16(ring + unit + (i * 64 + wave * 8) * 128, rs, ld_voff[i], kt * 128);
    };
    struct Tile {
        int64_t m0;
        int n0;
        u32x4_t ra, rw;
    };
    auto tile_at = [&](int v) {
        Tile t;
        const bool exists = v < nblk;
        int bm, bn;
        tile_of_pid(exists ? v : 0, nbm, nbn, bm, bn);
        t.m0 = (int64_t)bm * BM;
        t.n0 = bn * BN;
        t.ra = fp8_descriptor(A + t.m0 * Kp, exists ? (int)min((int64_t)BM, M - t.m0) * Kp : 0);
        t.rw = fp8_descriptor(W + (int64_t)t.n0 * Kp, exists ? min(BN, N - t.n0) * Kp : 0);
        return t;
    };
#define FP8_WAIT_VM(n) __builtin_amdgcn_s_waitcnt(0x0F70 | ((n) & 15) | (((n) >> 4) << 14))
    auto lds_barrier = [] {                          // orders LDS accesses only
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
        __builtin_amdgcn_s_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    };
    // the scales of group g: rows that do not exist take those of the last one (their results are not stored)
    uint32_t ca[TM], cw[TN], na[TM], nw[TN];
    auto request_scales = [&](const Tile &t, int g) {
        const uint32_t *pa = sa + (int64_t)g * M, *pw = sw + (int64_t)g * N;
#pragma unroll
        for (int i = 0; i < TM; ++i) na[i] = pa[min(t.m0 + wm * WTM + i * 32 + l32, M - 1)];
#pragma unroll
        for (int j = 0; j < TN; ++j) nw[j] = pw[min(t.n0 + wn * WTN + j * 32 + l32, N - 1)];
    };
    auto take_scales = [&] {
#pragma unroll
        for (int i = 0; i < TM; ++i) ca[i] = na[i];
#pragma unroll
        for (int j = 0; j < TN; ++j) cw[j] = nw[j];
    };

    // LDS byte offsets of this lane's first chunk of half 0; its second lies at ^ 16, those of half 1 at ^ 64
    typedef const __attribute__((address_space(3))) u32x4_t lds_frag;
    const unsigned a_lds = ring + (wm * WTM + l32) * 128 + (((2 * lq) ^ swz_of_row(l32)) << 4);
    const unsigned w_lds = ring + (wn * WTN + l32) * 128 + (((2 * lq) ^ swz_of_row(l32)) << 4);
    i32x8_t fa[TM], fw[2][TN];
    f32x16_t acc[TM][TN];
    auto fragment = [](unsigned at) {
        const u32x4_t x = *(lds_frag *)(unsigned long long)at, y = *(lds_frag *)(unsigned long long)(at ^ 16);
        return i32x8_t{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
    };
    auto read_a = [&](int i, int h, unsigned ua) { fa[i] = fragment((a_lds ^ (h * 64)) + ua + i * (32 * 128)); };
    auto read_w = [&](int j, int h, unsigned uw) { fw[h][j] = fragment((w_lds ^ (h * 64)) + uw + j * (32 * 128)); };
    // products of half h; behind them the operands of the other half from units ua, uw, and a unit's loads
    auto half = [&](auto h_, auto &&before_reads, unsigned ua, unsigned uw, const u32x4_t &rs, int kt, unsigned unit) {
        constexpr int h = decltype(h_)::value;
        static_for<0, TM>([&](auto i_) {
            constexpr int i = decltype(i_)::value;
            static_for<0, TN>([&](auto j_) {
                constexpr int j = decltype(j_)::value;
                acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fw[h][j], fa[i], acc[i][j], 0, 0, 0, (int)cw[j], 0, (int)ca[i]);
            });
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (i == 0) before_reads();
            read_a(i, 1 - h, ua);
            if constexpr (i < TN) read_w(i, 1 - h, uw);
            dma_one(i, rs, kt, unit);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    static_assert(LD_IT == TM, "a load behind the products of each operand");
    constexpr std::integral_constant<int, 0> h0{};
    constexpr std::integral_constant<int, 1> h1{};

    int v = blockIdx.x;                              // gridDim.x <= nblk: every work-group has a first tile
    Tile cur = tile_at(v);
    request_scales(cur, 0);
    __builtin_amdgcn_sched_barrier(0);
    static_for<0, LD_IT>([&](auto i_) { dma_one(decltype(i_)::value, cur.ra, 0, 0); });
    static_for<0, LD_IT>([&](auto i_) { dma_one(decltype(i_)::value, cur.rw, 0, UNIT); });
    static_for<0, LD_IT>([&](auto i_) { dma_one(decltype(i_)::value, cur.ra, 1, 2 * UNIT); });
    static_for<0, LD_IT>([&](auto i_) { dma_one(decltype(i_)::value, cur.rw, 1, 3 * UNIT); });
    FP8_WAIT_VM(0);                                  // the scales and blocks 0 and 1 are there
    lds_barrier();
    take_scales();
    unsigned u = 0;                                  // unit of A of this block; the five units from there on:
    auto at = [&](unsigned k) { const unsigned x = u + k; return (x >= UNITS ? x - UNITS : x) * UNIT; };
    for (;;) {
        const int vn = v + (int)gridDim.x;
        const Tile nxt = tile_at(vn);                // of zero size behind the last tile
        // (the last block's half 1 has read these too, but they are not held across the epilogue, which has no registers for them)
#pragma unroll
        for (int j = 0; j < TN; ++j) read_w(j, 0, at(1));
#pragma unroll
        for (int i = 0; i < TM; ++i) read_a(i, 0, at(0));
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int k = 0; k < 16; ++k) acc[i][j][k] = 0.0f;
        for (int kt = 0; kt < KT; ++kt) {
            if ((kt & 3) == 0) {
                if (kt) {                            // the next scales have landed (and what else is on its way, requested most of a half ago)
                    FP8_WAIT_VM(0);
                    take_scales();
                }
                __builtin_amdgcn_sched_barrier(0);
                const bool last = kt + 4 >= KT;
                request_scales(last ? nxt : cur, last ? 0 : (kt >> 2) + 1);
                __builtin_amdgcn_sched_barrier(0);
            }
            const bool ahead = kt + 2 >= KT;
            const u32x4_t ra = ahead ? nxt.ra : cur.ra, rw = ahead ? nxt.rw : cur.rw;
            const int kq = ahead ? (vn < nblk ? kt + 2 - KT : 0) : kt + 2;
            half(h0, [] {}, at(0), at(1), ra, kq, at(4));
            half(h1, [&] {
                if (kt) FP8_WAIT_VM(LD_IT);          // block T+1 has landed
                lds_barrier();                       // ... for everyone, and T's units are free
            }, at(2), at(3), rw, kq, at(0));
            u = u + 2 >= UNITS ? u + 2 - UNITS : u + 2;
#pragma unroll
            for (int i = 0; i < TM; ++i) ca[i] >>= 8;
#pragma unroll
            for (int j = 0; j < TN; ++j) cw[j] >>= 8;
        }
        // The next tile's first scales and its blocks 0 and 1, waited for in front of the stores: stores count as loads do, and a wait
        // behind them would be one for them.
        FP8_WAIT_VM(0);
        take_scales();
        // The epilogue: acc[i][j][4 g + k] of lane (lq, l32) is row 32 i + l32, column 32 j + 8 g + 4 lq + k of the wave tile.  32 rows at a
        // time pass through a wave-private stage of 32 x 64 bf16 in the unit of the last block's W, free since that block's barrier: 16-byte
        // chunk c of row r at chunk c ^ (r & 7).
        int tid_e = threadIdx.x;                     // (an opaque copy: addresses formed here are not held across the k loop)
        asm volatile("" : "+v"(tid_e));
        const int le = tid_e & 63, row_e = le & 31, half_e = le >> 5, n_wave = cur.n0 + wn * WTN;
        unsigned char *stage = fp8_smem + at(4) + wave * 4096;
#pragma unroll
        for (int i = 0; i < TM; ++i) {
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    f32x4_t x = {acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
                    if (ep.bias) x += fp8_bias4(ep, n_wave + 32 * j + 8 * g + 4 * half_e);
                    if constexpr (EPI == EPI_GELU) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) x[k] = gelu_bf16out(x[k]);
                    }
                    const bf16x4_t o = {(bf16)x[0], (bf16)x[1], (bf16)x[2], (bf16)x[3]};
                    *reinterpret_cast<bf16x4_t *>(stage + row_e * 128 + (((4 * j + g) ^ (row_e & 7)) << 4) + half_e * 8) = o;
                }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const int r = it * 8 + (le >> 3), c = le & 7, col = n_wave + c * 8;
                const bf16x8_t o = *reinterpret_cast<const bf16x8_t *>(stage + r * 128 + ((c ^ (r & 7)) << 4));
                const int64_t row = cur.m0 + wm * WTM + i * 32 + r;
                if (row >= M || col >= N) continue;
                bf16 *to = static_cast<bf16 *>(ep.out) + row * N + col;
                if (col + 8 <= N) {
                    __builtin_memcpy(to, &o, 16);
                } else {
                    const bf16 *from = reinterpret_cast<const bf16 *>(stage + r * 128 + ((c ^ (r & 7)) << 4));
#pragma unroll 1
                    for (int k = 0; col + k < N; ++k) to[k] = from[k];
                }
            }
            __builtin_amdgcn_wave_barrier();
        }
        if (vn >= nblk) break;                       // (block-uniform)
        v = vn;
        cur = nxt;
        lds_barrier();                               // every wave has read its stage back: the unit can be filled
    }
    FP8_WAIT_VM(0);                                  // (the loads behind the last tile, of zero size)
#undef FP8_WAIT_VM
}
