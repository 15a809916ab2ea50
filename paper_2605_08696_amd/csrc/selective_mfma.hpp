// The selective recurrence of bf16 operands on the matrix cores, sixty-four tokens of one head at a time.
//
// With e_t the decay exponents' running sum from the block's first token to token t, S the state in front of it:
//   y_t = 2^e_t S C_t + sum_{s <= t} M_ts x_s      M_ts = (C_t . B_s) 2^(e_t - e_s) dt_s
//   S' = 2^e_63 S + sum_s (2^(e_63 - e_s) dt_s x_s) B_s^T
// that is four products with 64 tokens as one side.  The running sum is formed in 64 bits, so that the exponents of S', which are small where
// the weights are not, and of M lose nothing to what came before them.
//
// Roundings.  The state stays in fp32 in the accumulators of its own product.  What is rounded to bf16 is, for y alone, M and the copy of S
// that meets C (2^-9 each, as much as y itself when it is stored).  x times its weight for S' is not rounded: it is cut into three bf16
// numbers that add up to it, each of which is multiplied; with two the state would be 3e-6 off.
//
// Layout.  Four wavefronts with sixteen rows p of the head each.  A product's result D[i][j] lies as column j in lane j % 16, rows
// 4 (lane / 16) .. + 3; an operand as row or column lane % 16, eight k from 8 (lane / 16) on.  S is formed as S^T (rows n), its rows n in
// such an order that a lane's two tiles hold eight consecutive n: converted, they are the operand that meets C, without a way through LDS.
// y is formed as y^T (rows p), four consecutive p of a token in a lane.  B^T and x^T come from LDS by the transposing reads.  M goes through
// LDS, since the wavefronts share it: its ten tiles of sixteen by sixteen tokens are dealt to them.
#pragma once
#include "selective.hpp"
#include "tile.hpp"

typedef __attribute__((ext_vector_type(4))) short i16x4_t;
typedef __attribute__((ext_vector_type(8))) short i16x8_t;

#define SCAN_INLINE __attribute__((always_inline))
constexpr int kScanBlock = 64;                       // tokens of a block, rows of P of a work-group

// LDS rows of CH chunks of sixteen bytes: chunk c of row r lies at c ^ f(r).  Sixteen rows' chunks c then lie on all banks, and so do the
// sixteen chunks or halves of chunks that a transposing read takes from four rows.
template <int CH>
__device__ __forceinline__ int scan_chunk(int r, int c)
{
    const int f = CH == 4 ? (r >> 2) & 3 : CH == 8 ? (r << 1 & 4) | (r >> 2 & 3) : (r << 2 & 12) | (r >> 2 & 3);
    return (r * CH + (c ^ f)) * 8;
}
template <int CH>
__device__ __forceinline__ bf16x8_t scan_row8(const bf16 *lds, int r, int c)
{
    return *reinterpret_cast<const bf16x8_t *>(lds + scan_chunk<CH>(r, c));
}
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;
__device__ __forceinline__ i16x4_t scan_transposed(const bf16 *p) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4 *)p); }
__device__ __forceinline__ bf16x8_t scan_pair(i16x4_t a, i16x4_t b)
{
    return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Running sum over the wavefront's lanes, this one's included.
__device__ __forceinline__ double wave_scan(double v)
{
    auto moved = [](double x, auto ctrl, auto rows) {
        const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
        const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
        const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), decltype(ctrl)::value, decltype(rows)::value, 0xF, false);
        return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
    };
    using std::integral_constant;
    v += moved(v, integral_constant<int, 0x111>{}, integral_constant<int, 0xF>{});     // row_shr:1, 2, 4, 8
    v += moved(v, integral_constant<int, 0x112>{}, integral_constant<int, 0xF>{});
    v += moved(v, integral_constant<int, 0x114>{}, integral_constant<int, 0xF>{});
    v += moved(v, integral_constant<int, 0x118>{}, integral_constant<int, 0xF>{});
    v += moved(v, integral_constant<int, 0x142>{}, integral_constant<int, 0xA>{});     // row_bcast:15 into rows 1 and 3
    v += moved(v, integral_constant<int, 0x143>{}, integral_constant<int, 0xC>{});     // row_bcast:31 into rows 2 and 3
    return v;
}

struct ScanBlockSizes {                              // of a block's tokens: running exponent, dt, weight in S', 2^exponent
    float e[kScanBlock], dt[kScanBlock], w[kScanBlock], f[kScanBlock];
    float total, factor;                             // the block's exponent and 2^it
};

// WHOLE: rows in whole chunks of eight elements, all at multiples of four bytes, row strides of less than 2^23.
template <int NP, int MODE, bool WHOLE>
__global__ void __launch_bounds__(256, 2)
selective_scan_mfma_kernel(const bf16 *__restrict__ xbc, bf16 *__restrict__ out, ScanCall c)
{
    constexpr int CH = NP / 8, NJ = NP / 32, Q = kScanBlock, BC = Q * CH / 256;      // chunks of a thread of B or C
    constexpr bool Y = MODE != SCAN_CARRY;
    __shared__ __align__(16) bf16 sb[Q * NP], sc[Y ? Q * NP : 8], sx[Q * 64], sm[Y ? Q * Q : 8];
    __shared__ __align__(16) ScanBlockSizes sizes[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int64_t id = work_group();
    const int per = c.H * c.parts;
    const int64_t work = id / per;
    const int h = (int)(id % per) / c.parts, p0 = (int)(id % per) % c.parts * 64, g = h / (c.H / c.G);
    const int P = c.P, N = c.N, np = min(64, P - p0);
    const int segments = (c.seqs.hi - c.seqs.lo + c.seg - 1) / c.seg;
    if (MODE == SCAN_WHOLE ? work >= c.seqs.n : work >= segments) return;
    const float a = c.a[h], skip = c.skip ? c.skip[h] : 0.0f, bias = c.dt.bias ? c.dt.bias[h] : 0.0f;
    const int64_t head_at = ((int64_t)h * P + p0) * N;
    const int64_t x_at = (int64_t)h * P + p0, b_at = (int64_t)c.H * P + (int64_t)g * N, c_at = b_at + (int64_t)c.G * N;

    f32x4_t S[2 * NJ];                               // S^T: tile 2 j + e, row 4 g4 + i is n = 32 j + 8 g4 + 4 e + i; column p = 16 wave + l16
    const int my_p = wave * 16 + l16;
    auto clear = [&]() SCAN_INLINE {
#pragma unroll
        for (int j = 0; j < 2 * NJ; ++j) S[j] = f32x4_t{0, 0, 0, 0};
    };
    auto each = [&](auto &&fn) SCAN_INLINE {                     // fn(four elements, offset from the head's first, how many of them exist)
        if (my_p < np) {
            static_for<0, 2 * NJ>([&](auto j_) SCAN_INLINE {
                constexpr int j = decltype(j_)::value;
                const int n = 32 * (j >> 1) + 8 * g4 + 4 * (j & 1);
                if (n < N) fn(S[j], (int64_t)my_p * N + n, min(4, N - n));
            });
        }
    };
    auto four = [&](const float *from, int many) SCAN_INLINE {
        if (many == 4) return (f32x4_t)*reinterpret_cast<const f32x4_any *>(from);
        f32x4_t v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < many) v[i] = from[i];
        return v;
    };
    auto load = [&](const float *from) SCAN_INLINE { each([&](f32x4_t &v, int64_t at, int many) SCAN_INLINE { v = four(from + at, many); }); };
    auto add = [&](const float *from, float scale) SCAN_INLINE {
        each([&](f32x4_t &v, int64_t at, int many) SCAN_INLINE {
            const f32x4_t w = four(from + at, many);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = fmaf(scale, w[i], v[i]);
        });
    };
    auto store = [&](float *to) SCAN_INLINE {
        each([&](f32x4_t &v, int64_t at, int many) SCAN_INLINE {
            if (many == 4) *reinterpret_cast<f32x4_any *>(to + at) = v;
            else
#pragma unroll
                for (int i = 0; i < 3; ++i)
                    if (i < many) to[at + i] = v[i];
        });
    };
    auto zeros = [&](int t0, int t1) SCAN_INLINE {
        for (int t = t0 + wave; t < t1; t += 4)
            if (lane < np) out[(int64_t)t * c.ld_out + x_at + lane] = (bf16)0.0f;
    };

    // The next block's rows travel in registers, sixteen bytes at a time, by loads that bring zeros from behind the sequence's last row and
    // for chunks behind a row's part.  Where the operands do not lie in whole chunks and words, the rows come one element at a time, when
    // they are put to LDS.
    bf16x8_t rb[BC], rc[Y ? BC : 1], rx[2];
    constexpr uint32_t kNone = 0x80000000u;          // behind every row
    const uint32_t row_bytes = (uint32_t)c.ld * 2;
    const int b_ch = (tid % CH), x_ch = tid & 7;
    const uint32_t b_off = b_ch * 8 < N ? (uint32_t)(tid / CH) * row_bytes + (uint32_t)b_at * 2 + b_ch * 16 : kNone;
    const uint32_t x_off = x_ch * 8 < np ? (uint32_t)(tid >> 3) * row_bytes + (uint32_t)x_at * 2 + x_ch * 16 : kNone;
    const uint32_t y_col = wave * 16 + 4 * g4 < np ? (wave * 16 + 4 * g4) * 2 : kNone;
    auto rows_of = [&](const void *base, int64_t ld, int64_t at, int rows, int row) SCAN_INLINE {
        return __builtin_amdgcn_make_buffer_rsrc(const_cast<bf16 *>(static_cast<const bf16 *>(base) + at), 0,
                                                 (uint32_t)(rows - 1) * (uint32_t)ld * 2 + (uint32_t)row * 2, 0x27000);
    };
    auto fetch_block = [&](int t, int t1) SCAN_INLINE {
        if constexpr (!WHOLE) return;
        const auto rs = rows_of(xbc, c.ld, (int64_t)t * c.ld, min(Q, t1 - t), c.H * P + 2 * c.G * N);
        static_for<0, BC>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            const uint32_t off = b_off + i * (256 / CH) * row_bytes;
            rb[i] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, 0, 0));
            if constexpr (Y) rc[i] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)off, c.G * N * 2, 0));
        });
        static_for<0, 2>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            rx[i] = __builtin_bit_cast(bf16x8_t, __builtin_amdgcn_raw_buffer_load_b128(rs, (int)(x_off + i * 32 * row_bytes), 0, 0));
        });
    };
    auto put_block = [&](int t, int t1) SCAN_INLINE {
        if constexpr (!WHOLE) {
            for (int e = tid; e < Q * NP; e += 256) {
                const int r = e / NP, n = e % NP;
                const bool there = t + r < t1 && n < N;
                const bf16 *row = xbc + (int64_t)(t + r) * c.ld + n;
                sb[scan_chunk<CH>(r, n >> 3) + (n & 7)] = there ? row[b_at] : (bf16)0.0f;
                if constexpr (Y) sc[scan_chunk<CH>(r, n >> 3) + (n & 7)] = there ? row[c_at] : (bf16)0.0f;
            }
            for (int e = tid; e < Q * 64; e += 256) {
                const int r = e >> 6, p = e & 63;
                sx[scan_chunk<8>(r, p >> 3) + (p & 7)] = t + r < t1 && p < np ? xbc[(int64_t)(t + r) * c.ld + x_at + p] : (bf16)0.0f;
            }
            return;
        }
        static_for<0, BC>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            const int at = scan_chunk<CH>(tid / CH + i * (256 / CH), b_ch);
            *reinterpret_cast<bf16x8_t *>(sb + at) = rb[i];
            if constexpr (Y) *reinterpret_cast<bf16x8_t *>(sc + at) = rc[i];
        });
        static_for<0, 2>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            *reinterpret_cast<bf16x8_t *>(sx + scan_chunk<8>((tid >> 3) + 32 * i, x_ch)) = rx[i];
        });
    };
    // A block's sizes, by one wavefront, a token in each lane.
    auto put_sizes = [&](ScanBlockSizes &to, float raw, bool there) SCAN_INLINE {
        float dt = dt_of(c.dt, raw, bias);
        dt = there ? dt : 0.0f;
        const double upto = wave_scan(there ? (double)decay_exponent(dt, a) : 0.0);
        const unsigned long long u = __builtin_bit_cast(unsigned long long, upto);
        const double total = __builtin_bit_cast(double, (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 63) << 32 |
                                                            (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63));
        to.e[lane] = (float)upto;
        to.dt[lane] = dt;
        to.w[lane] = __builtin_amdgcn_exp2f((float)(total - upto)) * dt;
        to.f[lane] = __builtin_amdgcn_exp2f((float)upto);
        if (lane == 0) {
            to.total = (float)total;
            to.factor = __builtin_amdgcn_exp2f((float)total);
        }
    };

    // Tokens [t0, t1) of one sequence.
    auto run = [&](int t0, int t1, float &sum) SCAN_INLINE {
        fetch_block(t0, t1);
        __syncthreads();                             // (nobody reads what an earlier call has left)
        if (wave == 0) put_sizes(sizes[0], dt_raw(c.dt, min(t0 + lane, t1 - 1), h), t0 + lane < t1);
        put_block(t0, t1);
        if constexpr (Y) {                           // the tiles above the diagonal that a step of k = 32 takes along
            for (int e = tid; e < 2 * 16 * 2; e += 256) {
                const int r = (e >> 5) * 32 + (e >> 1 & 15), ch = (e >> 5) * 4 + 2 + (e & 1);
                *reinterpret_cast<bf16x8_t *>(sm + scan_chunk<8>(r, ch)) = bf16x8_t{};
            }
        }
        __syncthreads();
        int now = 0;
        for (int t = t0; t < t1; t += Q, now ^= 1) {
            const ScanBlockSizes &z = sizes[now];
            const bool more = t + Q < t1, sizer = more && wave == (now ? 1 : 3);
            bf16x4_t gate[Y ? 4 : 1];                // z, as the lane's four tiles of y^T lie
            if constexpr (Y)
                if (WHOLE && c.z) {
                    const auto rs = rows_of(c.z, c.ld_z, (int64_t)t * c.ld_z + x_at, min(Q, t1 - t), np);
                    static_for<0, 4>([&](auto i_) SCAN_INLINE {
                        constexpr int i = decltype(i_)::value;
                        gate[i] = __builtin_bit_cast(bf16x4_t, __builtin_amdgcn_raw_buffer_load_b64(rs, (int)(y_col + (16 * i + l16) * (uint32_t)c.ld_z * 2), 0, 0));
                    });
                }
            float raw = 0.0f;
            if (sizer) raw = dt_raw(c.dt, min(t + Q + lane, t1 - 1), h);
            if (more) fetch_block(t + Q, t1);
            sum += z.total;
            f32x4_t acc[4];
            if constexpr (Y) {
                // M, its tiles (token tile tt, earlier tokens ss) in turn.  (The compiler must not know that their addresses are the same in
                // every block: it would keep some forty of them in registers.)
                int first = wave;
                asm volatile("" : "+s"(first));
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                    const int tile = first + 4 * k;
                    if (tile >= 10) break;
                    const int tt = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, ss = tile - tt * (tt + 1) / 2;
                    f32x4_t m = {0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        m = __builtin_amdgcn_mfma_f32_16x16x32_bf16(scan_row8<CH>(sb, ss * 16 + l16, 4 * j + g4), scan_row8<CH>(sc, tt * 16 + l16, 4 * j + g4), m, 0, 0, 0);
                    const int row = tt * 16 + l16, s0 = ss * 16 + 4 * g4;
                    const float e = z.e[row];
                    const f32x4_t es = *reinterpret_cast<const f32x4_t *>(z.e + s0), ds = *reinterpret_cast<const f32x4_t *>(z.dt + s0);
                    bf16x4_t q;
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float v = m[i] * (__builtin_amdgcn_exp2f(e - es[i]) * ds[i]);
                        q[i] = (bf16)(s0 + i <= row ? v : 0.0f);
                    }
                    *reinterpret_cast<bf16x4_t *>(sm + scan_chunk<8>(row, s0 >> 3) + (s0 & 4)) = q;
                }
                // what the state in front of the block brings
                bf16x8_t sf[NJ];
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) sf[j][i] = (bf16)S[2 * j + (i >> 2)][i & 3];
#pragma unroll
                for (int tt = 0; tt < 4; ++tt) {
                    acc[tt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
                    for (int j = 0; j < NJ; ++j)
                        acc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sf[j], scan_row8<CH>(sc, tt * 16 + l16, 4 * j + g4), acc[tt], 0, 0, 0);
                    const float f = z.f[tt * 16 + l16];
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[tt][i] *= f;
                }
            }
            // x^T: row p, eight tokens from 32 k + 8 g4 on
            bf16x8_t xf[2];
            const int q4 = l16 >> 2, c4 = l16 & 3;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int r = 32 * k + 8 * g4 + q4, ch = 2 * wave + (c4 >> 1), half = (c4 & 1) * 4;
                xf[k] = scan_pair(scan_transposed(sx + scan_chunk<8>(r, ch) + half), scan_transposed(sx + scan_chunk<8>(r + 4, ch) + half));
            }
            if constexpr (Y) {
                __syncthreads();
                // An x that is not finite would make NaN of the tokens in front of it too (0 times it): such are left out here and added
                // where they belong, one by one.
                uint32_t odd = 0;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const u32x4_t u = __builtin_bit_cast(u32x4_t, xf[k]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) odd |= (u[i] & 0x7f807f80u) + 0x00800080u;
                }
                const bool any = __ballot((odd & 0x80008000u) != 0) != 0;
                bf16x8_t xg[2] = {xf[0], xf[1]};
                if (any) {
#pragma unroll
                    for (int k = 0; k < 2; ++k)
#pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const float v = (float)xg[k][i];
                            if (!(fabsf(v) < INFINITY)) xg[k][i] = (bf16)0.0f;
                        }
                }
#pragma unroll
                for (int tt = 0; tt < 4; ++tt)
#pragma unroll
                    for (int k = 0; k <= tt >> 1; ++k)
                        acc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xg[k], scan_row8<8>(sm, tt * 16 + l16, 4 * k + g4), acc[tt], 0, 0, 0);
                if (any) {
                    int column = l16;
                    asm volatile("" : "+v"(column)); // (nor of these)
                    for (int s = 0; s < Q; ++s) {
                        const bf16x4_t v = *reinterpret_cast<const bf16x4_t *>(sx + scan_chunk<8>(s, 2 * wave + (g4 >> 1)) + (g4 & 1) * 4);
#pragma unroll
                        for (int tt = 0; tt < 4; ++tt) {
                            const int row = tt * 16 + column;
                            if (row < s) continue;
                            const float m = (float)sm[scan_chunk<8>(row, s >> 3) + (s & 7)];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (!(fabsf((float)v[i]) < INFINITY)) acc[tt][i] = fmaf(m, (float)v[i], acc[tt][i]);
                        }
                    }
                }
            }
            // S'
            const float factor = z.factor;
#pragma unroll
            for (int j = 0; j < 2 * NJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) S[j][i] *= factor;
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const f32x4_t w0 = *reinterpret_cast<const f32x4_t *>(z.w + 32 * k + 8 * g4), w1 = *reinterpret_cast<const f32x4_t *>(z.w + 32 * k + 8 * g4 + 4);
                uint32_t part[3][8];                 // the upper halves of three numbers that add up to x times its weight
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = (float)xf[k][i] * (i < 4 ? w0[i & 3] : w1[i & 3]);
                    part[0][i] = __float_as_uint(v);
                    const float r = v - __uint_as_float(part[0][i] & 0xffff0000u);
                    part[1][i] = __float_as_uint(r);
                    part[2][i] = __float_as_uint(r - __uint_as_float(part[1][i] & 0xffff0000u));
                }
                bf16x8_t xw[3];
#pragma unroll
                for (int q = 0; q < 3; ++q) {
                    u32x4_t u;
#pragma unroll
                    for (int i = 0; i < 4; ++i) u[i] = __builtin_amdgcn_perm(part[q][2 * i + 1], part[q][2 * i], 0x07060302u);
                    xw[q] = __builtin_bit_cast(bf16x8_t, u);
                }
#pragma unroll
                for (int j = 0; j < 2 * NJ; ++j) {
                    const int r = 32 * k + 8 * g4 + q4, ch = 4 * (j >> 1) + c4, half = (j & 1) * 4;
                    const bf16x8_t bt = scan_pair(scan_transposed(sb + scan_chunk<CH>(r, ch) + half), scan_transposed(sb + scan_chunk<CH>(r + 4, ch) + half));
#pragma unroll
                    for (int q = 0; q < 3; ++q) S[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bt, xw[q], S[j], 0, 0, 0);
                }
            }
            if (sizer) put_sizes(sizes[now ^ 1], raw, t + Q + lane < t1);
            if constexpr (Y) {
                const int p = wave * 16 + 4 * g4;
                const auto rs = rows_of(out, c.ld_out, (int64_t)t * c.ld_out + x_at, min(Q, t1 - t), np);
                static_for<0, 4>([&](auto tt_) SCAN_INLINE {
                    constexpr int tt = decltype(tt_)::value;
                    const int r = tt * 16 + l16;
                    const bf16x4_t x = *reinterpret_cast<const bf16x4_t *>(sx + scan_chunk<8>(r, p >> 3) + (p & 4));
                    float y[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[i] = fmaf(skip, (float)x[i], acc[tt][i]);
                    if constexpr (WHOLE) {
                        bf16x4_t q;
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if (c.z) y[i] *= silu((float)gate[tt][i]);
                            q[i] = (bf16)y[i];
                        }
                        typedef __attribute__((ext_vector_type(2))) uint32_t u32x2_t;
                        __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2_t, q), rs, (int)(y_col + r * (uint32_t)c.ld_out * 2), 0, 0);
                    } else if (t + r < t1) {
                        for (int i = 0; i < 4; ++i)
                            if (p + i < np) {
                                const float v = i == 0 ? y[0] : i == 1 ? y[1] : i == 2 ? y[2] : y[3];
                                const int64_t col = x_at + p + i;
                                const float u = c.z ? v * silu((float)static_cast<const bf16 *>(c.z)[(int64_t)(t + r) * c.ld_z + col]) : v;
                                out[(int64_t)(t + r) * c.ld_out + col] = (bf16)u;
                            }
                    }
                });
            }
            __syncthreads();
            if (more) {
                put_block(t + Q, t1);
                __syncthreads();
            }
        }
    };
    scan_drive<MODE>(c, work, h, p0, head_at, lane, clear, load, store, add, run, zeros);
}
