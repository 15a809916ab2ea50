// The selective recurrence of bf16 operands on the matrix cores, thirty-two tokens of one head at a time.
//
// With e_t the decay exponents' running sum from the block's first token to token t, S the state in front of it:
//   y_t = 2^e_t S C_t + sum_{s <= t} M_ts x_s      M_ts = (C_t . B_s) 2^(e_t - e_s) dt_s
//   S' = 2^e_31 S + sum_s (2^(e_31 - e_s) dt_s x_s) B_s^T
// that is four products with 32 tokens as one side.  The running sum is formed in 64 bits and kept in two parts, so that the exponents of S' and
// of M, which are small where the weights are not, lose nothing to what came before them.
//
// Roundings.  The state stays in fp32 in the accumulators of its own product.  M and the copy of S that meets C are cut into two bf16 numbers
// each, which leave 2^-15 of a value at most (a hundredth of what y may lose when it is stored), and both are multiplied.  x times its
// weight for S' is cut into three bf16 numbers that add up to it; with two the state would be 3e-6 off.
//
// Layout.  Four wavefronts with sixteen rows p of the head each.  A product's result D[i][j] lies as column j in lane j % 16, rows
// 4 (lane / 16) .. + 3; an operand as row or column lane % 16, eight k from 8 (lane / 16) on.  S is formed as S^T (rows n), its rows n in
// such an order that a lane's two tiles hold eight consecutive n: converted, they are the operand that meets C, without a way through LDS.
// y is formed as y^T (rows p), four consecutive p of a token in a lane.  B^T and x^T come from LDS by the transposing reads.  M goes through
// LDS, since the wavefronts share it: three of them form one of its tiles of sixteen by sixteen tokens each.  The tile of the later sixteen tokens
// with themselves, the one with the sixteen in front and their remainders make two operands of 32 tokens; the first sixteen's own tile and
// its remainder are one, against those tokens of x twice.
#pragma once
#include "selective.hpp"

typedef __attribute__((ext_vector_type(4))) short i16x4_t;
typedef __attribute__((ext_vector_type(8))) short i16x8_t;

constexpr int kScanBlock = 32, kScanRows = 64;       // tokens of a block, rows of P of a work-group
constexpr int kScanAhead = 3;                        // blocks whose sizes are formed together, one by a wavefront (a fourth's have no room in LDS)

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

// Two values as pairs of bf16: their upper halves, and what these leave (less than 2^-7 of a value), rounded.
struct ScanHalves {
    uint32_t high, low;
};
__device__ __forceinline__ ScanHalves scan_halves(float a, float b)
{
    const uint32_t u = __float_as_uint(a), v = __float_as_uint(b);
    const f32x2_t left = {a - __uint_as_float(u & 0xffff0000u), b - __uint_as_float(v & 0xffff0000u)};
    return {__builtin_amdgcn_perm(v, u, 0x07060302u), __builtin_bit_cast(uint32_t, __builtin_convertvector(left, bf16x2_t))};
}

// Running sum over each half of the wavefront's lanes, this one's included.
__device__ __forceinline__ double half_scan(double v)
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
    return v;
}

struct ScanBlockSizes {                              // of a block's tokens: running exponent (the last one's is the block's), dt, weight in S'
    float e[kScanBlock], low[kScanBlock], dt[kScanBlock], w[kScanBlock];
};

// Loads from memory to LDS are issued from asm statements: for one that it knows the compiler would wait in front of the next LDS read that
// it cannot prove disjoint.  16 bytes of every lane to 1024 bytes at LDS address `dst`, in the lanes' order; zeros from behind the operand.
__device__ __forceinline__ u32x4_t scan_rows_at(const void *base, uint32_t bytes)
{
    u32x4_t rs;
    const unsigned long long a = reinterpret_cast<unsigned long long>(base);
    rs[0] = __builtin_amdgcn_readfirstlane((unsigned)a);
    rs[1] = __builtin_amdgcn_readfirstlane((unsigned)(a >> 32));                 // stride 0: raw buffer
    rs[2] = __builtin_amdgcn_readfirstlane(bytes);
    rs[3] = 0x00020000u;
    return rs;
}
__device__ __forceinline__ void scan_dma16(unsigned dst, const u32x4_t &rs, uint32_t voff, int soff)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds" : : "s"(dst), "v"(voff), "s"(rs), "s"(soff) : "memory");
}
__device__ __forceinline__ unsigned scan_lds_address(const void *p)
{
    typedef __attribute__((address_space(3))) const unsigned char lds_byte;
    return __builtin_amdgcn_readfirstlane((unsigned)reinterpret_cast<unsigned long long>((lds_byte *)p));
}
// all but this wavefront's youngest N requests to memory have come back, its LDS writes are done, and so are the other wavefronts'
template <int N>
__device__ __forceinline__ void scan_barrier() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "i"(N) : "memory"); }
__device__ __forceinline__ void scan_barrier_lds() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// WHOLE: rows in whole chunks of eight elements, all at multiples of sixteen bytes, row strides of less than 2^23.
//
// A block's rows come to one of two LDS buffers while the block in front of it is worked on in the other, straight from memory (WHOLE), or by
// way of registers where rows in whole chunks lie at any element, or one element at a time.  Two barriers a block: its rows are there; M is
// there.  y takes x's place in LDS, and leaves from there in whole rows behind the next barrier.
//
// What bounds it: 32768 tokens in eight prompts of 64 heads of 64 x 128 take 357 us, 940 MB at 2.6 TB/s.  Two work-groups on a CU; their
// wavefronts issue vector instructions for two thirds of the time, 359 a block beside 46 products of 16 clocks, and wait for each other, for LDS
// and for products for a third.  What the precision of y costs, measured in turn: exponents in one part of fp32 (and the sizes of four blocks
// together) 346, M and S's copy rounded to one bf16 number each besides 306.  Remainders of S from pairs rounded by one conversion +0, each value
// rounded once more for its remainder +6 %; four blocks' sizes, two work-groups on a CU instead of three, 16384 tokens in one prompt 144 | 128.
// Of the 306: without the two smaller parts of x 274, without M 284, without the gate's exponentials 289; without any of these and the other
// products 242, which is what the trips through memory take.  Not kept there: three buffers (two work-groups on a CU): 331, 8192 tokens in eight
// prompts of 32 heads 62 | 60 with two, states of 256 99 | 91; loads and stores that bypass the caches +-2%.
// On the way: blocks of 64 tokens with rows through registers 394 (228 registers), each block's decays formed by one wavefront in front of a
// barrier 394, by all for four blocks 354, y stored and z read by each wavefront in 32 bytes of a row 332.
template <int NP, int MODE, bool WHOLE>
__global__ void __launch_bounds__(256, NP > 128 && MODE != SCAN_CARRY ? 1 : WHOLE || NP <= 64 ? 3 : 2)
selective_scan_mfma_kernel(const bf16 *__restrict__ xbc, bf16 *__restrict__ out, ScanCall c)
{
    constexpr int CH = NP / 8, NJ = NP / 32, Q = kScanBlock, SLOTS = Q * CH / 64;    // loads of 64 chunks that B or C of a block takes
    constexpr bool Y = MODE != SCAN_CARRY;
    __shared__ __align__(16) bf16 sb[2][Q * NP], sc[Y ? 2 : 1][Y ? Q * NP : 8], sx[2][Q * 64], sg[Y ? 2 : 1][Y ? Q * 64 : 8],
        sm[Y ? 48 * Q : 8];
    __shared__ __align__(16) ScanBlockSizes sizes[kScanAhead];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l16 = lane & 15, g4 = lane >> 4;
    const int64_t id = scan_unit();
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
    auto clear = [&]() SCAN_INLINE { static_for<0, 2 * NJ>([&](auto j_) SCAN_INLINE { S[decltype(j_)::value] = f32x4_t{0, 0, 0, 0}; }); };
    auto each = [&](auto &&fn) SCAN_INLINE {         // fn(four elements, offset from the head's first, how many of them exist)
        if (my_p < np)
            static_for<0, 2 * NJ>([&](auto j_) SCAN_INLINE {
                constexpr int j = decltype(j_)::value;
                const int n = 32 * (j >> 1) + 8 * g4 + 4 * (j & 1);
                if (n < N) fn(S[j], (int64_t)my_p * N + n, min(4, N - n));
            });
    };
    auto four = [&](const float *from, int many) SCAN_INLINE {
        if (WHOLE || many == 4) return (f32x4_t)*reinterpret_cast<const f32x4_any *>(from);
        f32x4_t v = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < many) v[i] = from[i];
        return v;
    };
    auto load = [&](const float *from) SCAN_INLINE { each([&](f32x4_t &v, int64_t at, int many) SCAN_INLINE { v = four(from + at, many); }); };
    auto store = [&](float *to) SCAN_INLINE {
        each([&](f32x4_t &v, int64_t at, int many) SCAN_INLINE {
            if (WHOLE || many == 4) *reinterpret_cast<f32x4_any *>(to + at) = v;
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

    // This lane's chunk of each load: LDS slot s holds chunk (s % CH) ^ f(r) of row r = s / CH.
    constexpr uint32_t kNone = 0x80000000u;          // behind every operand
    const uint32_t row_bytes = (uint32_t)c.ld * 2;
    constexpr int LOADS = SLOTS >= 4 ? SLOTS / 4 : 1;                   // of a wavefront (with two slots: wavefronts 0, 1 B, 2, 3 C)
    uint32_t b_off[LOADS], x_off, z_off, y_off;
    unsigned lds_b = 0, lds_c = 0, lds_x = 0, lds_z = 0;
    if constexpr (WHOLE) {
        static_for<0, LOADS>([&](auto i_) SCAN_INLINE {
            constexpr int i = decltype(i_)::value;
            const int s = ((SLOTS >= 4 ? wave + 4 * i : wave & 1) * 64) + lane, r = s / CH, ch = scan_chunk<CH>(r, s % CH) / 8 % CH;
            b_off[i] = ch * 8 < N ? (uint32_t)r * row_bytes + (uint32_t)b_at * 2 + ch * 16 : kNone;
        });
        const int r = tid >> 3, ch = scan_chunk<8>(r, tid & 7) / 8 % 8;
        x_off = ch * 8 < np ? (uint32_t)r * row_bytes + (uint32_t)x_at * 2 + ch * 16 : kNone;
        z_off = ch * 8 < np ? (uint32_t)r * (uint32_t)c.ld_z * 2 + ch * 16 : kNone;
        y_off = ch * 8 < np ? (uint32_t)r * (uint32_t)c.ld_out * 2 + ch * 16 : kNone;
        lds_b = scan_lds_address(sb), lds_c = scan_lds_address(sc), lds_x = scan_lds_address(sx), lds_z = scan_lds_address(sg);
    }
    typedef u32x4_t __attribute__((aligned(2))) u32x4_any;
    constexpr int BC = (Q * CH + 255) / 256;
    u32x4_t rb[WHOLE ? 1 : BC], rc[WHOLE || !Y ? 1 : BC], rx[2];
    // Rows [t, t + Q) up to t1 on their way to buffer `to`.
    auto bring = [&](int t, int t1, auto to_) SCAN_INLINE {
        constexpr int to = decltype(to_)::value;
        if constexpr (WHOLE) {
            const u32x4_t rs = scan_rows_at(xbc + (int64_t)t * c.ld, (uint32_t)(min(Q, t1 - t) - 1) * row_bytes + (uint32_t)(c.H * P + 2 * c.G * N) * 2);
            const int to_c = c.G * N * 2;
            if constexpr (SLOTS >= 4) {
                static_for<0, LOADS>([&](auto i_) SCAN_INLINE {
                    constexpr int i = decltype(i_)::value;
                    scan_dma16(lds_b + to * Q * NP * 2 + (wave + 4 * i) * 1024, rs, b_off[i], 0);
                    if constexpr (Y) scan_dma16(lds_c + to * Q * NP * 2 + (wave + 4 * i) * 1024, rs, b_off[i], to_c);
                });
            } else {
                if (wave < 2) scan_dma16(lds_b + to * Q * NP * 2 + (wave & 1) * 1024, rs, b_off[0], 0);
                else if (Y) scan_dma16(lds_c + to * Q * NP * 2 + (wave & 1) * 1024, rs, b_off[0], to_c);
            }
            scan_dma16(lds_x + to * Q * 64 * 2 + wave * 1024, rs, x_off, 0);
            if (Y && c.z)
                scan_dma16(lds_z + to * Q * 64 * 2 + wave * 1024,
                           scan_rows_at(static_cast<const bf16 *>(c.z) + (int64_t)t * c.ld_z + x_at, (uint32_t)(min(Q, t1 - t) - 1) * (uint32_t)c.ld_z * 2 + np * 2), z_off, 0);
        } else {
            if (c.chunks) {
                static_for<0, BC>([&](auto i_) SCAN_INLINE {
                    constexpr int i = decltype(i_)::value;
                    const int e = min(tid + 256 * i, Q * CH - 1), r = e / CH, ch = scan_chunk<CH>(r, e % CH) / 8 % CH;
                    const bf16 *row = xbc + (int64_t)min(t + r, t1 - 1) * c.ld + min(ch * 8, N - 8);
                    rb[i] = *reinterpret_cast<const u32x4_any *>(row + b_at);
                    if constexpr (Y) rc[i] = *reinterpret_cast<const u32x4_any *>(row + c_at);
                });
                const int64_t row = min(t + (tid >> 3), t1 - 1);
                const int col = min(scan_chunk<8>(tid >> 3, tid & 7) / 8 % 8 * 8, np - 8);
                rx[0] = *reinterpret_cast<const u32x4_any *>(xbc + row * c.ld + x_at + col);
                if (Y && c.z) rx[1] = *reinterpret_cast<const u32x4_any *>(static_cast<const bf16 *>(c.z) + row * c.ld_z + x_at + col);
                return;
            }
            for (int e = tid; e < Q * NP; e += 256) {
                const int r = e / NP, n = e % NP;
                const bool there = t + r < t1 && n < N;
                const bf16 *row = xbc + (int64_t)(t + r) * c.ld + n;
                sb[to][scan_chunk<CH>(r, n >> 3) + (n & 7)] = there ? row[b_at] : (bf16)0.0f;
                if constexpr (Y) sc[to][scan_chunk<CH>(r, n >> 3) + (n & 7)] = there ? row[c_at] : (bf16)0.0f;
            }
            for (int k = 0; k < 8; ++k) {            // (the rows whose y this wavefront has taken from there)
                const int r = wave * 8 + k, p = lane;
                const bool there = t + r < t1 && p < np;
                sx[to][scan_chunk<8>(r, p >> 3) + (p & 7)] = there ? xbc[(int64_t)(t + r) * c.ld + x_at + p] : (bf16)0.0f;
                if (Y && c.z) sg[to][scan_chunk<8>(r, p >> 3) + (p & 7)] = there ? static_cast<const bf16 *>(c.z)[(int64_t)(t + r) * c.ld_z + x_at + p] : (bf16)0.0f;
            }
        }
    };
    // ... and from registers, where they came that way.
    auto put = [&](int t, int t1, auto to_) SCAN_INLINE {
        constexpr int to = decltype(to_)::value;
        if constexpr (!WHOLE) {
            if (!c.chunks) return;
            const u32x4_t zero = {0, 0, 0, 0};
            static_for<0, BC>([&](auto i_) SCAN_INLINE {
                constexpr int i = decltype(i_)::value;
                const int e = tid + 256 * i, r = e / CH, ch = scan_chunk<CH>(r, e % CH) / 8 % CH;
                if (e >= Q * CH) return;
                const bool there = t + r < t1 && ch * 8 < N;
                *reinterpret_cast<u32x4_t *>(sb[to] + e * 8) = there ? rb[i] : zero;
                if constexpr (Y) *reinterpret_cast<u32x4_t *>(sc[to] + e * 8) = there ? rc[i] : zero;
            });
            const bool there = t + (tid >> 3) < t1 && scan_chunk<8>(tid >> 3, tid & 7) / 8 % 8 * 8 < np;
            *reinterpret_cast<u32x4_t *>(sx[to] + tid * 8) = there ? rx[0] : zero;
            if (Y && c.z) *reinterpret_cast<u32x4_t *>(sg[to] + tid * 8) = there ? rx[1] : zero;
        }
    };
    // y of rows [t, t + Q) up to t1 from buffer `from`: this lane's chunk of the rows that this wavefront's loads bring to the same place next.
    auto leave = [&](int t, int t1, auto from_) SCAN_INLINE {
        constexpr int from = decltype(from_)::value;
        if constexpr (Y) {
            if constexpr (WHOLE) {
                const u32x4_t v = *reinterpret_cast<const u32x4_t *>(sx[from] + tid * 8);
                const auto rs = __builtin_amdgcn_make_buffer_rsrc(out + (int64_t)t * c.ld_out + x_at, 0,
                                                                  (uint32_t)(min(Q, t1 - t) - 1) * (uint32_t)c.ld_out * 2 + (uint32_t)np * 2, 0x00020000);
                __builtin_amdgcn_raw_buffer_store_b128(v, rs, (int)y_off, 0, 0);
            } else {
                const bf16x8_t v = *reinterpret_cast<const bf16x8_t *>(sx[from] + tid * 8);
                const int r = tid >> 3, col = scan_chunk<8>(r, tid & 7) / 8 % 8 * 8;
                bf16 *o = out + (int64_t)(t + r) * c.ld_out + x_at + col;
                if (t + r < t1 && col + 8 <= np) *reinterpret_cast<u32x4_any *>(o) = __builtin_bit_cast(u32x4_t, v);
                else if (t + r < t1)
#pragma unroll
                    for (int i = 0; i < 7; ++i)
                        if (col + i < np) o[i] = v[i];
            }
        }
    };
    // The sizes of the kScanAhead blocks from t on: a token in each lane of a wavefront's halves.
    auto raw_of = [&](int t, int t1) SCAN_INLINE { return dt_raw(c.dt, min(t + wave * Q + (lane & 31), t1 - 1), h); };
    auto put_sizes = [&](float raw, int t, int t1) SCAN_INLINE {
        const bool there = t + wave * Q + (lane & 31) < t1;
        float dt = dt_of(c.dt, raw, bias);
        dt = there ? dt : 0.0f;
        const double upto = half_scan(there ? decay_exponent(dt, a) : 0.0);
        const unsigned long long u = __builtin_bit_cast(unsigned long long, upto);
        const double total = __builtin_bit_cast(double, (unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(u >> 32), 31) << 32 |
                                                            (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 31));
        ScanBlockSizes &to = sizes[wave];
        const int at = lane & 31;                    // (the halves of the wavefront write the same)
        to.e[at] = (float)upto;
        const float low = (float)(upto - (float)upto);
        to.low[at] = low;
        to.dt[at] = fmaf(dt, low * -0.69314718f, dt);
        to.w[at] = exp2_of(total - upto) * dt;
    };

    float raw = 0.0f;                                // dt_raw of the next blocks whose sizes are formed
    double sum_of = 0.0;
    // Block [t, t + Q) up to t1, number n of its sequence, which lies in buffer `now`.
    auto block = [&](int t, int t1, int n, auto now_) SCAN_INLINE {
        constexpr int now = decltype(now_)::value;
        constexpr int then = 1 - now;                // the buffer of the blocks before and behind
        if constexpr (WHOLE) scan_barrier<0>();
        else scan_barrier_lds();
        // (dt has come with some block's rows; the compiler, which does not count those, must not wait for it behind further ones)
        asm volatile("" : "+v"(raw));
        if (n > 0) leave(t - Q, t1, std::integral_constant<int, then>{});
        if (t + Q < t1) {
            asm volatile("s_waitcnt lgkmcnt(0)" : : : "memory");               // (y has been read)
            bring(t + Q, t1, std::integral_constant<int, then>{});
        }
        if (n % kScanAhead == 0) {
            if (wave < kScanAhead) put_sizes(raw, t, t1);
            if (t + kScanAhead * Q < t1) raw = raw_of(t + kScanAhead * Q, t1);
            scan_barrier_lds();
        }
        const ScanBlockSizes &sz = sizes[n % kScanAhead];
        bf16 *const xs = sx[now];
        const bf16 *const bs = sb[now], *const cs = sc[Y ? now : 0];
        const float factor = exp2_of(sz.e[Q - 1], sz.low[Q - 1]);       // (tokens behind the last add nothing)
        if (MODE == SCAN_CARRY) sum_of += (double)sz.e[Q - 1] + (double)sz.low[Q - 1];
        const int q4 = l16 >> 2, c4 = l16 & 3;
        f32x4_t acc[2];
        if constexpr (Y) {
            // M: three of the wavefronts take a tile each (tokens tt, earlier tokens ss)
            if (wave < 3) {
                const int tt = wave > 0, ss = wave == 2;
                f32x4_t m = {0, 0, 0, 0};
                static_for<0, NJ>([&](auto j_) SCAN_INLINE {
                    constexpr int j = decltype(j_)::value;
                    m = __builtin_amdgcn_mfma_f32_16x16x32_bf16(scan_row8<CH>(bs, ss * 16 + l16, 4 * j + g4), scan_row8<CH>(cs, tt * 16 + l16, 4 * j + g4), m, 0, 0, 0);
                });
                const int row = tt * 16 + l16, s0 = ss * 16 + 4 * g4;
                const float e = sz.e[row], low = sz.low[row];
                const f32x4_t es = *reinterpret_cast<const f32x4_t *>(sz.e + s0), ds = *reinterpret_cast<const f32x4_t *>(sz.dt + s0);
                float v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = m[i] * (__builtin_amdgcn_exp2f(e - es[i] + low) * ds[i]);
                    v[i] = s0 + i <= row ? v[i] : 0.0f;
                }
                const ScanHalves a = scan_halves(v[0], v[1]), b = scan_halves(v[2], v[3]);
                *reinterpret_cast<uint2 *>(sm + scan_chunk<4>(row, s0 >> 3) + (s0 & 4)) = make_uint2(a.high, b.high);
                *reinterpret_cast<uint2 *>(sm + scan_chunk<4>(row + 16 * tt, (s0 >> 3) + (tt ? 0 : 2)) + (s0 & 4)) = make_uint2(a.low, b.low);
            }
            // what the state in front of the block brings
            acc[0] = acc[1] = f32x4_t{0, 0, 0, 0};
            static_for<0, NJ>([&](auto j_) SCAN_INLINE {
                constexpr int j = decltype(j_)::value;
                u32x4_t high, low;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const ScanHalves q = scan_halves(S[2 * j + (i >> 1)][2 * (i & 1)], S[2 * j + (i >> 1)][2 * (i & 1) + 1]);
                    high[i] = q.high;
                    low[i] = q.low;
                }
                const bf16x8_t s = __builtin_bit_cast(bf16x8_t, high), left = __builtin_bit_cast(bf16x8_t, low);
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
                    const bf16x8_t row = scan_row8<CH>(cs, tt * 16 + l16, 4 * j + g4);
                    acc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(left, row, acc[tt], 0, 0, 0);
                    acc[tt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(s, row, acc[tt], 0, 0, 0);
                }
            });
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const float f = __builtin_amdgcn_exp2f(sz.e[tt * 16 + l16]);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[tt][i] *= f;
            }
        }
        // x^T: row p, eight tokens from 8 g4 on
        bf16x8_t xf;
        {
            const int r = 8 * g4 + q4, ch = 2 * wave + (c4 >> 1), half = (c4 & 1) * 4;
            xf = scan_pair(scan_transposed(xs + scan_chunk<8>(r, ch) + half), scan_transposed(xs + scan_chunk<8>(r + 4, ch) + half));
        }
        // S'
        const f32x4_t w0 = *reinterpret_cast<const f32x4_t *>(sz.w + 8 * g4), w1 = *reinterpret_cast<const f32x4_t *>(sz.w + 8 * g4 + 4);
        uint32_t part[3][8];                         // the upper halves of three numbers that add up to x times its weight
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = (float)xf[i] * (i < 4 ? w0[i & 3] : w1[i & 3]);
            part[0][i] = __float_as_uint(v);
            const float r = v - __uint_as_float(part[0][i] & 0xffff0000u);
            part[1][i] = __float_as_uint(r);
            part[2][i] = __float_as_uint(r - __uint_as_float(part[1][i] & 0xffff0000u));
        }
        bf16x8_t xw[3];
#pragma unroll
        for (int q = 0; q < 3; ++q) {
            u32x4_t v;
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __builtin_amdgcn_perm(part[q][2 * i + 1], part[q][2 * i], 0x07060302u);
            xw[q] = __builtin_bit_cast(bf16x8_t, v);
        }
        static_for<0, 2 * NJ>([&](auto j_) SCAN_INLINE {
            constexpr int j = decltype(j_)::value;
            const int r = 8 * g4 + q4, ch = 4 * (j >> 1) + c4, half = (j & 1) * 4;
            const bf16x8_t bt = scan_pair(scan_transposed(bs + scan_chunk<CH>(r, ch) + half), scan_transposed(bs + scan_chunk<CH>(r + 4, ch) + half));
#pragma unroll
            for (int i = 0; i < 4; ++i) S[j][i] *= factor;
#pragma unroll
            for (int q = 0; q < 3; ++q) S[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(bt, xw[q], S[j], 0, 0, 0);
        });
        if constexpr (Y) {
            scan_barrier_lds();
            // An x that is not finite would make NaN of the tokens in front of it too (0 times it): such are left out here and added
            // where they belong, one by one.  One of this lane's column has made a NaN of all of the column's state.
            const bool any = __ballot(!(fabsf(S[0][0]) < INFINITY)) != 0;
            bf16x8_t xg = xf;
            if (any) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float v = (float)xg[i];
                    if (!(fabsf(v) < INFINITY)) xg[i] = (bf16)0.0f;
                }
            }
            u32x4_t twice = __builtin_bit_cast(u32x4_t, xg);       // the first sixteen tokens, in both halves of the wavefront
#pragma unroll
            for (int i = 0; i < 4; ++i) twice[i] = __builtin_amdgcn_permlane32_swap(twice[i], twice[i], false, false)[0];
            acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, twice), scan_row8<4>(sm, l16, g4), acc[0], 0, 0, 0);
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xg, scan_row8<4>(sm, 32 + l16, g4), acc[1], 0, 0, 0);
            acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(xg, scan_row8<4>(sm, 16 + l16, g4), acc[1], 0, 0, 0);
            if (any) {
                int column = l16;
                asm volatile("" : "+v"(column));     // (addresses of this path are not kept in registers for all blocks)
                for (int s = 0; s < Q; ++s) {
                    const bf16x4_t v = *reinterpret_cast<const bf16x4_t *>(xs + scan_chunk<8>(s, 2 * wave + (g4 >> 1)) + (g4 & 1) * 4);
#pragma unroll
                    for (int tt = 0; tt < 2; ++tt) {
                        const int row = tt * 16 + column;
                        if (row < s) continue;
                        const float m = (float)sm[scan_chunk<4>(row, s >> 3) + (s & 7)] + (float)sm[scan_chunk<4>(row + 16 * tt, (s >> 3) + (tt ? 0 : 2)) + (s & 7)];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (!(fabsf((float)v[i]) < INFINITY)) acc[tt][i] = fmaf(m, (float)v[i], acc[tt][i]);
                    }
                }
            }
        }
        if constexpr (Y) {
            const int p = wave * 16 + 4 * g4;
            float y[2][4];
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const bf16x4_t x = *reinterpret_cast<const bf16x4_t *>(xs + scan_chunk<8>(tt * 16 + l16, p >> 3) + (p & 4));
#pragma unroll
                for (int i = 0; i < 4; ++i) y[tt][i] = c.skip ? fmaf(skip, (float)x[i], acc[tt][i]) : acc[tt][i];
            }
            if (c.z)
#pragma unroll
                for (int tt = 0; tt < 2; ++tt) {
                    const bf16x4_t z = *reinterpret_cast<const bf16x4_t *>(sg[now] + scan_chunk<8>(tt * 16 + l16, p >> 3) + (p & 4));
#pragma unroll
                    for (int i = 0; i < 4; ++i) y[tt][i] *= silu<bf16>((float)z[i]);
                }
#pragma unroll
            for (int tt = 0; tt < 2; ++tt) {
                const bf16x2_t lo = __builtin_convertvector(f32x2_t{y[tt][0], y[tt][1]}, bf16x2_t), hi = __builtin_convertvector(f32x2_t{y[tt][2], y[tt][3]}, bf16x2_t);
                *reinterpret_cast<bf16x4_t *>(xs + scan_chunk<8>(tt * 16 + l16, p >> 3) + (p & 4)) = __builtin_shufflevector(lo, hi, 0, 1, 2, 3);
            }
        }
        if (t + Q < t1) put(t + Q, t1, std::integral_constant<int, then>{});
    };

    // Tokens [t0, t1) of one sequence.
    auto run = [&](int t0, int t1, double &sum) SCAN_INLINE {
        __syncthreads();                             // (nobody reads what an earlier call has left)
        raw = raw_of(t0, t1);
        bring(t0, t1, std::integral_constant<int, 0>{});
        put(t0, t1, std::integral_constant<int, 0>{});
        asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
        sum_of = 0.0;
        for (int t = t0, n = 0; t < t1;)
            static_for<0, 2>([&](auto now_) SCAN_INLINE {
                if (t >= t1) return;
                block(t, t1, n++, now_);
                t += Q;
                if (t >= t1) {
                    scan_barrier_lds();
                    leave(t - Q, t1, now_);
                }
            });
        sum += sum_of;
    };
    scan_drive<MODE>(c, work, h, p0, head_at, lane, clear, load, store, run, zeros);
}
