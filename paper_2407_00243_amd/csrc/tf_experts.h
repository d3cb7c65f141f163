// Products of a few rows with the weights of the experts that name them (or with one 4-bit matrix).
#pragma once
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "tf_moe_device.h"

namespace tf {
namespace {

// Waves of a workgroup by the blocks of rows that each multiplies.
constexpr int expert_waves(int nf) { return nf == 1 ? 8 : 4; }
constexpr int kNearRows = 256;        // row pointers that are held in LDS
constexpr int kNearEntries = 256;     // entries whose sum finds columns and values in LDS
// The most tokens whose entries the last workgroups add up: one bf16 token through two experts of 4096 x 8192 85.4 us, with a launch of
// its own 86.7 (calls of small layers 0.5 us); but 32 tokens through 64 experts of 2048 x 1024 158 us, with that launch 141.
constexpr int kJoinTokens = 16;

// Hidden rows of TF_F16 are held in two parts, high * 2^12 + low: fp16 alone ends at 65504, which a gate times
// what it gates passes easily.  Two parts in fp16, since that is what the instructions multiply beside fp16 weights: up to 2^28, off by 2^-22
// of a number and, where the low part is subnormal, by 2^-25, which is what fp16 itself holds of numbers below 2^-14.
constexpr float kHalfHigh = 4096.0f;

__device__ __forceinline__ Float4 mfma_bf16(const Words4 &a, const Words4 &b, Float4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(Bf8, a), __builtin_bit_cast(Bf8, b), c, 0, 0, 0);
}
__device__ __forceinline__ Float4 mfma_f16(const Words4 &a, const Words4 &b, Float4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(Half8, a), __builtin_bit_cast(Half8, b), c, 0, 0, 0);
}
__device__ __forceinline__ Float4 mfma_f32(float a, float b, Float4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}

// 4-bit weights meet bf16 and fp32 rows of X as 2^-10 of their codes' values, and results are multiplied by 2^10 at the very end:
// a group's sum is taken before its scale, and 128 codes of 7 times the largest X would pass 2^128 where the result does not.
// What is below 2^-126 is subnormal, so a group's sum is good to 2^-139 at the best.  (fp16 rows are far from either end.)
constexpr float kCodeDown = 0x1p-10f, kCodeUp = 0x1p10f;

// Eight weights of a word of codes, as numbers of sixteen bits (bf16 where X is fp32).  INT: sign and magnitude m
// sit where an e4m3 number has its sign and its lowest bits; without exponent bits that is m 2^-9.
template <int EL, int KIND> __device__ __forceinline__ Words4 q4_decode(uint32_t w) {
    constexpr float e2m1_down = kCodeDown, int_down = 512.0f * kCodeDown;
    Words4 y;
    if constexpr (KIND == TF_Q4_E2M1) {
        if constexpr (EL == TF_F16) {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
        } else {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, e2m1_down, 0));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, e2m1_down, 1));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, e2m1_down, 2));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, e2m1_down, 3));
        }
    } else {
        const uint32_t lo = w & 0x87878787u, hi = __builtin_amdgcn_alignbit(w, w, 4) & 0x87878787u;
        if constexpr (EL == TF_F16) {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true));
        } else {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, int_down, false));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, int_down, true));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, int_down, false));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, int_down, true));
        }
    }
    return y;
}

// Two fp32 numbers in three bf16 parts each: h + 2^-8 (m + l) (cut off, not rounded: the parts of a number have its sign, and no
// part of a finite number is infinite).  They add up to it exactly from 2^-118 on; parts below 2^-133 are subnormal,
// and without the factor that would begin at 2^-110.  An infinity is its first part alone.
constexpr float kRestUp = 256.0f;
__device__ __forceinline__ void cut_pair(uint32_t &h, uint32_t &m, uint32_t &l, float a, float b) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    h = (ua >> 16) | (ub & 0xffff0000u);
    float ra = kRestUp * (a - __uint_as_float(ua & 0xffff0000u)), rb = kRestUp * (b - __uint_as_float(ub & 0xffff0000u));
    ra = __builtin_isinf(a) ? 0.0f : ra;
    rb = __builtin_isinf(b) ? 0.0f : rb;
    const uint32_t va = __float_as_uint(ra), vb = __float_as_uint(rb);
    m = (va >> 16) | (vb & 0xffff0000u);
    const uint32_t wa = __float_as_uint(ra - __uint_as_float(va & 0xffff0000u));
    const uint32_t wb = __float_as_uint(rb - __uint_as_float(vb & 0xffff0000u));
    l = (wa >> 16) | (wb & 0xffff0000u);
}

// (in forms that keep their relative precision where they come close to zero: no 1 - 1, no exp that overflows)
__device__ __forceinline__ float activate(int act, float x) {
    switch (act) {
        case TF_ACT_RELU: return x < 0.0f ? 0.0f : x;       // (a NaN stays one)
        case TF_ACT_SILU: {
            const float e = expf(-fabsf(x));
            return (x < 0.0f ? x * e : x) / (1.0f + e);
        }
        case TF_ACT_GELU: return 0.5f * x * erfcf(x * -0.70710678118654752f);
        default: return x;
    }
}

// Row of A that entry q belongs to: where all rows have the same number of entries, as a router leaves them, the first
// guess is right.
__device__ __forceinline__ int row_of_entry(const int32_t *rowptr, int n_rows, int nnz, int q) {
    const int guess = (int)((int64_t)q * n_rows / nnz);
    if (rowptr[guess] <= q && q < rowptr[guess + 1]) return guess;
    int lo = 0, hi = n_rows;              // the first row that ends beyond q
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (rowptr[mid + 1] > q) hi = mid;
        else lo = mid + 1;
    }
    return min(lo, n_rows - 1);
}

// Sixteen bytes of a row that ends at column n were loaded at min(k, n - piece) instead of column k: moved to their places,
// zeros from the end of the row on.
template <typename T> __device__ __forceinline__ Words4 set_right(Words4 x, int k, int n) {
    constexpr int piece = 16 / (int)sizeof(T);
    const int bits = min(max(k + piece - n, 0), piece) * 8 * (int)sizeof(T);
    if constexpr (sizeof(T) == 2) {
        const bool half = bits & 16;
        x = Words4{half ? x[0] >> 16 | x[1] << 16 : x[0], half ? x[1] >> 16 | x[2] << 16 : x[1], half ? x[2] >> 16 | x[3] << 16 : x[2],
                   half ? x[3] >> 16 : x[3]};
    }
    x = bits & 32 ? Words4{x[1], x[2], x[3], 0} : x;
    x = bits & 64 ? Words4{x[2], x[3], 0, 0} : x;
    return bits & 128 ? Words4{0, 0, 0, 0} : x;
}
// The same for a row of fewer than sixteen bytes, loaded element by element.
template <typename T> __device__ __forceinline__ Words4 load_short(const char *p, int k, int n) {
    Words4 y = {0, 0, 0, 0};
#pragma unroll 1
    for (int i = 0; i < 16 / (int)sizeof(T); ++i) {
        const uint32_t e = k + i < n ? reinterpret_cast<const T *>(p)[k + i] : T(0);
        if constexpr (sizeof(T) == 4) y = Words4{y[1], y[2], y[3], e};
        else y = Words4{y[0] >> 16 | y[1] << 16, y[1] >> 16 | y[2] << 16, y[2] >> 16 | y[3] << 16, y[3] >> 16 | e << 16};
    }
    return y;
}

// EL: element type; KIND: 4-bit kind or -1; G: groups in 128 columns; HID: X are hidden rows; in their methods NT: blocks of
// sixteen entries that are multiplied at a time.
//
// A wave multiplies NF blocks of sixteen rows of one expert's weights (with a gate: sixteen of the gate and the sixteen
// that it multiplies) with the rows of X of the entries that name the expert.  a.k_waves waves of the workgroup share the
// columns of the same rows, a step in turn, and their sums are added up through LDS, wave after wave.  Weights are an operand of
// the matrix instructions straight from memory: whatever the number of entries up to sixteen, what one instruction
// multiplies was loaded by one instruction.  X is the other operand and passes through LDS, chunk by chunk, in operand order,
// where all waves read it.  X is the first of the two: a lane then holds sums of four entries and one row of weights, whose
// group has one scale (with the weights first it took four scales a group and 128-column steps of twice the registers).
//
// Bound by memory where entries of an expert are few: 32 bf16 tokens through 64 experts of 2048 x 1024 (0.77 GB) 145 us, 5.3 TB/s;
// one through two of 4096 x 8192 85 us, 4.7; an fp16 row times a 4-bit matrix of 32768 x 8192 29.6 us, 5.1; and by the instructions of
// products and staging where they are many: 128 fp16 tokens through 16 4-bit experts of 4096 x 8192 305 us, 3.0 TB/s, vector
// instructions 28 to 31 % of the waves' cycles, waits 36 to 39, at the two waves a SIMD that 256 registers leave (three or four with
// spilled registers were slower).  (Medians of passes in a graph over two sets of inputs in turn.)
//
// X in registers, straight from memory into the operand, took 983 us there, and 247 for the 32 tokens.  It was ahead where little
// is multiplied with an X that is staged: a bf16 row times 4-bit 4096 x 4096 6.4 us (now 6.9), 13 fp32 rows times 5003 x 2891
// 9.5 (13.4), 64 bf16 rows times 8192 x 8192 36.7 (37.1), 11 fp16 tokens through 10 experts of 1037 x 515 20 (26).
//
// Dense weights are loaded by whole lines of 128 bytes: an instruction takes eight rows x 128 bytes, and two of them are
// put in operand order (sixteen rows x 64 bytes) by exchanging halves of sixteen lanes (a read of 512 MiB by itself, rows of
// 4 / 8 / 16 KiB: sixteen rows x 64 bytes 4.9 / 6.0 / 5.2 TB/s, eight rows x 128 bytes 6.2 / 6.4 / 5.8).
template <int EL, int KIND, int G, bool HID, int NF> struct Expert {
    typedef typename El<EL>::T T;
    typedef std::conditional_t<EL == TF_F32, uint32_t, uint16_t> Bits;
    static constexpr int WAVES = expert_waves(NF), THREADS = 64 * WAVES;
    static constexpr int CHUNK = WAVES * (8 << 10);                  // LDS of a chunk of X, of which there are two
    static constexpr int MOST = KIND < 0 || NF == 1 ? 4 : 2;           // blocks of sixteen entries that are multiplied at a time
    static constexpr bool DENSE = KIND < 0, WIDE = EL == TF_F32;
    static constexpr int PIECE = 16 / (int)sizeof(T);                // elements of sixteen bytes
    static constexpr int STEP = DENSE ? 8 * PIECE : kQ4Block;        // columns of a step
    static constexpr int SUB = DENSE ? 2 : 4;                        // operands of X in a step
    static constexpr int XP = !DENSE && WIDE ? 3 : HID && !WIDE ? 2 : 1;   // parts of X
    static constexpr int SETS = !DENSE && WIDE ? 2 : HID && EL == TF_F16 ? 2 : 1;   // sums of high and of low parts
    static constexpr int WL = DENSE ? 2 : 1;                         // pieces of weights that a lane holds of a step and block
    static constexpr int SW = G == 4 ? 2 : 1;                        // words of scales
    static constexpr int AHEAD = 1, RING = AHEAD + 1;                // steps whose weights are on their way, and the one multiplied
    static constexpr int XE = DENSE && WIDE ? 4 : 8;                 // columns of X that a lane holds of an operand
    static constexpr int XR = !DENSE && WIDE ? 2 : XP;               // sixteen-byte pieces that a lane loads of an operand

    // Chunks of X for NT blocks of TOK entries (of fewer than sixteen only these are held; an operand is 4 TOK pieces then).
    template <int NT, int TOK> struct Chunk {
        static constexpr int LANES = 4 * TOK;
        static constexpr int FIT = CHUNK / (SUB * NT * XP * LANES * 16);
        static constexpr int STEPS = FIT >= 32 ? 32 : FIT >= 16 ? 16 : FIT >= 8 ? 8 : FIT >= 4 ? 4 : FIT >= 2 ? 2 : 1;
        static constexpr int SLOTS = STEPS * SUB * NT;
        static constexpr int MINE = (SLOTS * LANES + THREADS - 1) / THREADS;
        static constexpr int PIECES = SLOTS * XP * LANES;            // of a buffer
        const char *row[MINE];                                       // where the thread's pieces begin
        Words4 x[MINE][XR];
    };

    // LDS of a workgroup: two chunks of X, or one if that is all there is; the waves' sums in their place.
    template <int NT, int TOK> static int bytes(int steps) {
        typedef Chunk<NT, TOK> C;
        const int x = steps > C::STEPS ? 2 * C::PIECES : steps * SUB * NT * C::LANES * XP;
        return std::max(x * 16, WAVES * NF * NT * 1024);
    }

    // Entries that a pass multiplies at the most, in the case of run() that holds `entries` of them: what a launch's LDS and the waves
    // that share columns are chosen for.  Entries beyond it are another pass.
    static int pass_of(int entries) { return entries <= 4 ? 4 : entries <= 16 ? 16 : entries <= 32 || MOST == 2 ? 32 : 16 * MOST; }
    static int pass_steps(int pass) {          // steps of its chunks (fewer in the larger cases, so each is enough for the smaller ones)
        static_assert(Chunk<1, 4>::STEPS >= Chunk<1, 16>::STEPS && Chunk<1, 16>::STEPS >= Chunk<2, 16>::STEPS &&
                      Chunk<2, 16>::STEPS >= Chunk<MOST, 16>::STEPS, "");
        return pass == 4 ? Chunk<1, 4>::STEPS : pass == 16 ? Chunk<1, 16>::STEPS : pass == 32 ? Chunk<2, 16>::STEPS : Chunk<MOST, 16>::STEPS;
    }
    static int pass_bytes(int pass, int steps) {
        int b = bytes<1, 4>(steps);
        if (pass >= 16) b = std::max(b, bytes<1, 16>(steps));
        if (pass >= 32) b = std::max(b, bytes<2, 16>(steps));
        if (pass > 32) b = std::max(b, bytes<MOST, 16>(steps));
        return b;
    }

    struct Weights {
        Words4 w[NF][WL];
        uint32_t s[DENSE ? 1 : NF][SW];
    };

    // Places of a wave's weights: of a block of sixteen rows one that is the same for all lanes, and a lane's offset from it
    // (below 2^31: columns are limited, kMaxColumns).
    const char *wb[NF], *sb[NF];
    uint32_t w_at[WL], w_up, s_at, s_up;      // (4 bits: those of the rows behind a gate's begin anywhere in the layout's blocks)
    int n_cols, g, r, wave, lane, tid;

    // row0: row of the first block of outputs
    __device__ __forceinline__ void set(const ExpertLaunch &a, int expert, int row0) {
        tid = threadIdx.x;
        lane = tid & 63;
        wave = __builtin_amdgcn_readfirstlane(tid >> 6);
        g = lane >> 4;
        r = lane & 15;
        n_cols = a.n_cols;
        const int out_blocks = a.gated ? NF / 2 : NF;
        const int64_t blocks = (n_cols + kQ4Block - 1) / kQ4Block;
        const char *w = static_cast<const char *>(a.W) + expert * a.w_mat;
        const char *sc = static_cast<const char *>(a.scales) + expert * a.s_mat;
        w_up = s_up = s_at = 0;
#pragma unroll
        for (int f = 0; f < NF; ++f) {
            const int up = f >= out_blocks;
            const int first = block_row(a, row0, f - up * out_blocks) + up * a.n_rows;
            if constexpr (DENSE) {
                wb[f] = w + (int64_t)first * n_cols * (int)sizeof(T);
                sb[f] = nullptr;
            } else {
                wb[f] = w + (first >> 4) * blocks * 1024;
                sb[f] = sc + (first >> 4) * blocks * (32 * G);
            }
        }
        if constexpr (DENSE) {
            const int rows = min(a.n_rows, 16);       // (of a matrix with fewer rows than a block the last one is read again)
#pragma unroll
            for (int i = 0; i < 2; ++i) w_at[i] = (uint32_t)min(8 * i + (r & 7), rows - 1) * (uint32_t)n_cols * (uint32_t)sizeof(T);
        } else {
            w_at[0] = lane * 16;
            s_at = r * (2 * G);
            // rows behind a gate's: the first of a block is row o of a block of the layout, whose next one exists where rows of it
            // are used (rows beyond the matrix: others are read)
            const int row = (a.n_rows & 15) + r;
            const bool next = row > 15 && (a.n_rows + block_row(a, row0, 0)) >> 4 < (2 * a.n_rows - 1) >> 4;
            w_up = (next ? (uint32_t)blocks * 1024 : 0) + (16 * g + (row & 15)) * 16;
            s_up = (next ? (uint32_t)blocks * (32 * G) : 0) + (row & 15) * (2 * G);
        }
    }
    // First row of a block of outputs: the last block of dense weights ends with the matrix (rows that two blocks hold are stored
    // twice, the same), blocks beyond the matrix are its last one.
    static __device__ __forceinline__ int block_row(const ExpertLaunch &a, int row0, int f) {
        return max(0, min(row0 + 16 * f, DENSE ? a.n_rows - 16 : (a.n_rows - 1) & ~15));
    }
    __device__ __forceinline__ int dense_column(int step) const { return step * STEP + PIECE * (g + 4 * (r >> 3)); }
    __device__ __forceinline__ void load(Weights &x, int step, const ExpertLaunch &a) const {
        if constexpr (DENSE) {
            const uint32_t k = (uint32_t)min(dense_column(step), n_cols - PIECE) * (uint32_t)sizeof(T);
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int i = 0; i < 2; ++i) x.w[f][i] = __builtin_nontemporal_load(reinterpret_cast<const AnyWords4 *>(wb[f] + (w_at[i] + k)));
        } else {
            const int out_blocks = a.gated ? NF / 2 : NF;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                x.w[f][0] = __builtin_nontemporal_load(
                    reinterpret_cast<const Words4 *>(wb[f] + (int64_t)step * 1024 + (f >= out_blocks ? w_up : w_at[0])));
                const char *p = sb[f] + (int64_t)step * (32 * G) + (f >= out_blocks ? s_up : s_at);
                if constexpr (G == 1) {
                    x.s[f][0] = *reinterpret_cast<const uint16_t *>(p);
                } else {
#pragma unroll
                    for (int i = 0; i < SW; ++i) x.s[f][i] = reinterpret_cast<const uint32_t *>(p)[i];
                }
            }
        }
    }
    // Operand j of the step, in the order of the instructions.
    static __device__ __forceinline__ Words4 operand(const Weights &x, int f, int j) {
        if constexpr (DENSE) {
            constexpr int ror8 = 0x128;
            Words4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                y[i] = j == 0 ? (uint32_t)__builtin_amdgcn_update_dpp((int)x.w[f][0][i], (int)x.w[f][WL - 1][i], ror8, 0xf, 0xc, false)
                              : (uint32_t)__builtin_amdgcn_update_dpp((int)x.w[f][WL - 1][i], (int)x.w[f][0][i], ror8, 0xf, 0x3, false);
            return y;
        } else {
            return q4_decode<EL, KIND>(x.w[f][0][j]);
        }
    }

    // Dense weights: sums of high and of low parts; 4 bits: sums that the scales are in (DOWN: 2^-10 of them).
    static constexpr bool DOWN = !DENSE && EL != TF_F16;
    template <int NT> struct Sums {
        Float4 v[DENSE ? SETS : 1][NF][NT];
    };
    // xs: operands of X in LDS, the step's from j0 on.
    template <int NT, int TOK> __device__ __forceinline__ void multiply(Sums<NT> &c, const Weights &x, const Words4 *xs, int j0) const {
        if constexpr (DENSE) {
#pragma unroll
            for (int j = 0; j < SUB; ++j) multiply_operand<NT, TOK>(c.v, x, xs, j0, j);
        } else {
            // a group's sums are multiplied by its scales when the instructions of the next group are on their way
            constexpr int per = 4 / G;
            Float4 acc[2][SETS][NF][NT];
#pragma unroll
            for (int q = 0; q <= G; ++q) {
                if (q < G) {
#pragma unroll
                    for (int h = 0; h < SETS; ++h)
#pragma unroll
                        for (int f = 0; f < NF; ++f)
#pragma unroll
                            for (int n = 0; n < NT; ++n) acc[q & 1][h][f][n] = Float4{0, 0, 0, 0};
#pragma unroll
                    for (int j = q * per; j < (q + 1) * per; ++j) multiply_operand<NT, TOK>(acc[q & 1], x, xs, j0, j);
                }
                if (q > 0) {
                    const int p = q - 1;
#pragma unroll
                    for (int f = 0; f < NF; ++f) {
                        const float s = p & 1 ? bf16_high(x.s[f][p / 2]) : bf16_low(x.s[f][p / 2]);
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int v = 0; v < 4; ++v) {
                                float d = acc[p & 1][0][f][n][v];
                                if constexpr (SETS > 1)
                                    d = EL == TF_F16 ? fmaf(d, kHalfHigh, acc[p & 1][SETS - 1][f][n][v])
                                                     : fmaf(acc[p & 1][SETS - 1][f][n][v], 1.0f / kRestUp, d);
                                c.v[0][f][n][v] = fmaf(s, d, c.v[0][f][n][v]);
                            }
                    }
                }
            }
        }
    }
    template <int NT, int TOK, int S>
    __device__ __forceinline__ void multiply_operand(Float4 (&acc)[S][NF][NT], const Weights &x, const Words4 *xs, int j0, int j) const {
        xs += (j0 + j) * (NT * XP * 4 * TOK) + place<NT, TOK>(j0 + j, g, r % TOK);
        Words4 w[NF];
#pragma unroll
        for (int f = 0; f < NF; ++f) w[f] = operand(x, f, j);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            Words4 y[XP];
#pragma unroll
            for (int h = 0; h < XP; ++h) y[h] = xs[(n * XP + h) * (4 * TOK)];
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                if constexpr (DENSE && WIDE) {
                    const Float4 v = __builtin_bit_cast(Float4, w[f]), b = __builtin_bit_cast(Float4, y[0]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[0][f][n] = mfma_f32(b[i], v[i], acc[0][f][n]);
                } else {
#pragma unroll
                    for (int h = 0; h < XP; ++h) {
                        Float4 &d = acc[h < SETS ? h : SETS - 1][f][n];
                        d = EL == TF_F16 ? mfma_f16(y[h], w[f], d) : mfma_bf16(y[h], w[f], d);
                    }
                }
            }
        }
    }
    // What the sum of an entry and a row is for.  up: the sum that the gate multiplies.
    static __device__ __forceinline__ void store(const ExpertLaunch &a, int entry, int row, float y, float up) {
        const int64_t at = (int64_t)entry * a.ldo + row;
        if constexpr (HID) {
            // (read by another workgroup of the launch: past the caches that it does not share)
            __hip_atomic_store(static_cast<float *>(a.out) + at, y, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        } else if (a.out_kind == kOutRows) {
            static_cast<T *>(a.out)[at] = El<EL>::put(y);
        } else {
            const float h = activate(a.activation, y) * up;
            T *hi = static_cast<T *>(a.out);
            T *lo = reinterpret_cast<T *>(static_cast<char *>(a.out) + a.out_part);
            if constexpr (EL == TF_F32) {
                hi[at] = h;
            } else if constexpr (EL == TF_BF16) {
                // (numbers that round to infinity take the largest bf16 number as their high part)
                const uint16_t near = El<EL>::put(h);
                const uint16_t top = near - (__builtin_isinf(El<EL>::get(near)) && !__builtin_isinf(h));
                const float rest = h - El<EL>::get(top);
                hi[at] = top;
                lo[at] = __builtin_isinf(El<EL>::get(top)) ? 0 : El<EL>::put(rest);
            } else {
                const uint16_t top = El<EL>::put(h * (1.0f / kHalfHigh));
                const float rest = fmaf(-kHalfHigh, El<EL>::get(top), h);
                hi[at] = top;
                lo[at] = __builtin_isinf(El<EL>::get(top)) ? 0 : El<EL>::put(fminf(fmaxf(rest, -65504.0f), 65504.0f));
            }
        }
    }

    // This thread's pieces of a chunk of X: from memory, and into LDS when they have arrived.
    // Pieces are dealt to the threads row by row: a wave loads a contiguous part of a row, and rows of no entry are not loaded at
    // all.  A piece's place among those of its operand is rotated with its column: without that the 64 pieces of a row that a wave
    // writes would all be in the same four banks (of the LDS cycles of 128 fp16 tokens through 4-bit experts 40 % are
    // still conflicts; with pieces dealt operand by operand, sixteen rows x 64 bytes a load, none are, but 64 bf16 rows times a 4-bit
    // 8192 x 8192 matrix took 66 us where this took 59, both with two blocks of rows a wave).
    template <int NT, int TOK> struct Piece {
        static constexpr int ROW = Chunk<NT, TOK>::STEPS * SUB * 4;       // pieces of a row in a chunk
        int e, c;                                                        // entry, piece of its row
        __device__ __forceinline__ Piece(int m, int tid) : e((m * THREADS + tid) / ROW), c((m * THREADS + tid) % ROW) {}
    };
    template <int NT, int TOK> static __device__ __forceinline__ int place(int j, int g, int r) {       // operand j of the chunk
        return TOK == 16 ? g * 16 + ((r + g + 4 * j) & 15) : (g * TOK + r + j) & (4 * TOK - 1);
    }
    template <int NT, int TOK> __device__ __forceinline__ int chunk_pieces(int chunk) const {          // of a row, as far as it goes
        return min(Chunk<NT, TOK>::STEPS, steps() - chunk * Chunk<NT, TOK>::STEPS) * (SUB * 4);
    }
    template <int NT, int TOK>
    __device__ __forceinline__ void find_rows(Chunk<NT, TOK> &y, const ExpertLaunch &a, const int *s_row, int count) const {
#pragma unroll
        for (int m = 0; m < Chunk<NT, TOK>::MINE; ++m) {
            int at = s_row[min(Piece<NT, TOK>(m, tid).e, count - 1)];
            if constexpr (Piece<NT, TOK>::ROW % 64 == 0) at = __builtin_amdgcn_readfirstlane(at);
            y.row[m] = static_cast<const char *>(a.X) + at * a.ldx * (int64_t)sizeof(T);
        }
    }
    template <int NT, int TOK>
    __device__ __forceinline__ void fetch(Chunk<NT, TOK> &y, const ExpertLaunch &a, int count, int chunk) const {
        typedef Chunk<NT, TOK> C;
        const int limit = chunk_pieces<NT, TOK>(chunk);
        const bool cut = (chunk + 1) * (C::STEPS * STEP) > n_cols;
#pragma unroll
        for (int m = 0; m < C::MINE; ++m) {
            if (m * THREADS / Piece<NT, TOK>::ROW >= count) break;
            const Piece<NT, TOK> p(m, tid);
            if (p.e >= count || p.c >= limit) continue;
            const int k0 = chunk * (C::STEPS * STEP) + XE * p.c;
#pragma unroll
            for (int h = 0; h < XR; ++h) {
                const char *q = HID && !WIDE && h ? y.row[m] + a.x_part : y.row[m];
                int k = k0 + (WIDE && h ? 4 : 0);
                if (cut && n_cols < PIECE) {
                    y.x[m][h] = load_short<Bits>(q, k, n_cols);
                    continue;
                }
                if (cut) k = min(k, n_cols - PIECE);
                y.x[m][h] = *reinterpret_cast<const AnyWords4 *>(q + (uint32_t)k * (uint32_t)sizeof(T));
            }
        }
    }
    template <int NT, int TOK> __device__ __forceinline__ void put(Chunk<NT, TOK> &y, int count, int chunk, Words4 *xs) const {
        typedef Chunk<NT, TOK> C;
        const int limit = chunk_pieces<NT, TOK>(chunk);
        const bool move = (chunk + 1) * (C::STEPS * STEP) > n_cols && n_cols >= PIECE;
#pragma unroll
        for (int m = 0; m < C::MINE; ++m) {
            if (m * THREADS / Piece<NT, TOK>::ROW >= count) break;
            const Piece<NT, TOK> p(m, tid);
            if (p.e >= count || p.c >= limit) continue;
            Words4 *to = xs + (p.c / 4 * NT + p.e / 16) * (XP * C::LANES) + place<NT, TOK>(p.c / 4, p.c % 4, p.e % 16);
            if (move) {
                const int k = chunk * (C::STEPS * STEP) + XE * p.c;
#pragma unroll
                for (int h = 0; h < XR; ++h) y.x[m][h] = set_right<Bits>(y.x[m][h], k + (WIDE && h ? 4 : 0), n_cols);
            }
            if constexpr (!DENSE && WIDE) {
                Words4 part[3];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t h, m1, l;
                    cut_pair(h, m1, l, __uint_as_float(y.x[m][i / 2][2 * (i & 1)]), __uint_as_float(y.x[m][i / 2][2 * (i & 1) + 1]));
                    part[0][i] = h;
                    part[1][i] = m1;
                    part[2][i] = l;
                }
#pragma unroll
                for (int h = 0; h < 3; ++h) to[h * C::LANES] = part[h];
            } else {
#pragma unroll
                for (int h = 0; h < XP; ++h) to[h * C::LANES] = y.x[m][h];
            }
        }
    }

    __device__ __forceinline__ int steps() const { return (n_cols + STEP - 1) / STEP; }
    // The first weights are on their way.
    __device__ __forceinline__ void start(Weights (&w)[RING], const ExpertLaunch &a, int k_wave) const {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) load(w[i], min(k_wave + i * a.k_waves, steps() - 1), a);
    }

    // The `count` entries (at most NT blocks of sixteen; TOK < 16: at most TOK) in s_entry, their rows of X in s_row.  row0: the
    // wave's first row.  smem: LDS of bytes().
    template <int NT, int TOK>
    __device__ __forceinline__ void run(const ExpertLaunch &a, Weights (&w)[RING], int k_wave, int row0, int count, const int *s_entry,
                                        const int *s_row, unsigned char *smem) {
        typedef Chunk<NT, TOK> C;
        asm volatile("" : "+v"(tid));          // (what follows from it is worked out here, not before all cases and kept)
        Words4 *const xs = reinterpret_cast<Words4 *>(smem);
        C y;
        find_rows<NT, TOK>(y, a, s_row, count);
        fetch<NT, TOK>(y, a, count, 0);
        Sums<NT> c;
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int h = 0; h < (DENSE ? SETS : 1); ++h) c.v[h][f][n] = Float4{0, 0, 0, 0};
        const int last = steps() - 1, turns = last / a.k_waves + 1, chunk_turns = C::STEPS / a.k_waves;
        const int mine = row0 < a.n_rows ? last - k_wave : -1;       // (steps of this wave: those up to k_wave + mine)
        for (int t0 = 0; t0 < turns; t0 += RING) {
#pragma unroll
            for (int i = 0; i < RING; ++i) {
                const int t = t0 + i;
                if (t >= turns) break;
                const int chunk = t / chunk_turns;
                Words4 *const x = xs + (chunk & 1) * C::PIECES;
                if (t % chunk_turns == 0) {
                    put<NT, TOK>(y, count, chunk, x);
                    __syncthreads();
                    if (t + chunk_turns < turns) fetch<NT, TOK>(y, a, count, chunk + 1);
                }
                const int s = k_wave + t * a.k_waves;
                load(w[(i + AHEAD) % RING], min(s + AHEAD * a.k_waves, last), a);
                if (t * a.k_waves > mine) continue;
                if constexpr (DENSE) {
                    if ((s + 1) * STEP > n_cols) {
#pragma unroll
                        for (int f = 0; f < NF; ++f)
#pragma unroll
                            for (int q = 0; q < WL; ++q) w[i].w[f][q] = set_right<Bits>(w[i].w[f][q], dense_column(s), n_cols);
                    }
                }
                multiply<NT, TOK>(c, w[i], x, s % C::STEPS * SUB);
            }
        }
        __syncthreads();
        if constexpr (DENSE && SETS > 1) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int v = 0; v < 4; ++v) c.v[0][f][n][v] = fmaf(c.v[0][f][n][v], kHalfHigh, c.v[SETS - 1][f][n][v]);
        }

        const int out_blocks = a.gated ? NF / 2 : NF;
        // sums of the waves that share rows, in their order (in the place of X, which all waves are done with)
        Float4 *const red = reinterpret_cast<Float4 *>(smem);
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int n = 0; n < NT; ++n) red[((wave * NF + f) * NT + n) * 64 + lane] = c.v[0][f][n];
        __syncthreads();
        const int row_groups = WAVES / a.k_waves, per_group = out_blocks * NT * 64;
        for (int item = threadIdx.x; item < row_groups * per_group; item += THREADS) {
            const int rg = item / per_group, in = item % per_group;        // (in: block, sixteen entries, lane)
            const Float4 *p = red + rg * a.k_waves * (NF * NT * 64) + in;
            Float4 y = p[0];
            for (int w = 1; w < a.k_waves; ++w) y += p[w * (NF * NT * 64)];
            Float4 up = Float4{1, 1, 1, 1};
            if (a.gated) {
                p += NF / 2 * NT * 64;
                up = p[0];
                for (int w = 1; w < a.k_waves; ++w) up += p[w * (NF * NT * 64)];
            }
            if constexpr (DOWN) {
                y *= kCodeUp;
                if (a.gated) up *= kCodeUp;
            }
            const int f = in / (NT * 64), n = in / 64 % NT, il = in & 63;
            const int slot = 16 * n + 4 * (il >> 4);
            // (row0 is that of this wave's group)
            const int first = row0 + (rg - wave / a.k_waves) * (16 * out_blocks);
            const int row = block_row(a, first, f) + (il & 15);
            if (first + 16 * f >= a.n_rows || row >= a.n_rows) continue;
#pragma unroll
            for (int v = 0; v < 4; ++v)
                if (slot + v < count) store(a, s_entry[slot + v], row, y[v], up[v]);
        }
    }
};

// One element of D: the sum of value times result over the entries q0 .. q1 - 1 of a token, in their order.  SHARED: results that
// workgroups of this launch have stored.
template <bool SHARED>
__device__ __forceinline__ float combine_entries(int q0, int q1, const int32_t *colidx, const float *vals, const float *Y, int64_t ldy,
                                                 int n_experts, int c) {
    constexpr int batch = 4;          // entries whose loads go out together
    float d = 0.0f;
    for (int q = q0; q < q1; q += batch) {
        float v[batch], y[batch];
        bool in[batch];
#pragma unroll
        for (int i = 0; i < batch; ++i) {
            const int e = min(q + i, q1 - 1);
            in[i] = q + i < q1 && (uint32_t)colidx[e] < (uint32_t)n_experts;
            v[i] = vals[e];
            const float *p = Y + (int64_t)e * ldy + c;
            y[i] = SHARED ? __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : *p;
        }
#pragma unroll
        for (int i = 0; i < batch; ++i)
            if (in[i]) d = fmaf(v[i], y[i], d);
    }
    return d;
}

template <int EL, int KIND, int G, bool HID, int NF>
__global__ __launch_bounds__(64 * expert_waves(NF), 2) void k_experts(const ExpertLaunch a) {
    typedef Expert<EL, KIND, G, HID, NF> Ex;
    const int most = a.pass_entries;
    __shared__ int s_count[Ex::WAVES], s_entry[16 * Ex::MOST], s_row[16 * Ex::MOST], s_rowptr[HID ? kJoinTokens + 1 : kNearRows], s_last;
    __shared__ int s_col[HID ? kNearEntries : 1];
    __shared__ float s_val[HID ? kNearEntries : 1];
    extern __shared__ __align__(16) unsigned char smem[];

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wave_rows = 16 * (a.gated ? NF / 2 : NF), rows_per = Ex::WAVES / a.k_waves * wave_rows;
    const int tiles = (a.n_rows + rows_per - 1) / rows_per;
    const int tile = blockIdx.x % tiles, unit = blockIdx.x / tiles;
    const int row0 = tile * rows_per + wave / a.k_waves * wave_rows, k_wave = wave % a.k_waves;

    const bool by_entry = a.rowptr && a.n_entries <= a.n_experts;
    int expert = 0;
    if (a.rowptr) expert = !by_entry ? unit : unit < a.n_entries ? a.colidx[unit] : -1;
    const bool named = expert >= 0 && expert < a.n_experts;
    // what the sum over the entries needs of A (its loads are ahead of those of the weights: what is loaded first is waited for first)
    const bool join = HID && a.arrived, near_entries = join && a.n_entries <= kNearEntries;
    int32_t col = -1, end = 0;
    float val = 0.0f;
    if (near_entries && (int)threadIdx.x < a.n_entries) {
        col = a.colidx[threadIdx.x];
        val = a.vals[threadIdx.x];
    }
    if (join && (int)threadIdx.x <= a.n_tokens) end = min(max(a.rowptr[threadIdx.x], 0), a.n_entries);
    // few entries: every wave looks for those of its expert by itself
    const bool few = a.rowptr && a.n_entries <= 64 && a.n_tokens <= kJoinTokens;
    int here = -1, here_row = 0;
    if (few) {
        if (lane < a.n_entries) here = a.colidx[lane];
        if (!HID)
            for (int t = 1; t < a.n_tokens; ++t) here_row += a.rowptr[t] <= lane;
    }
    Ex x;
    typename Ex::Weights w[Ex::RING];
    if (named) {
        x.set(a, expert, row0);
        x.start(w, a, k_wave);        // (before the entries are looked for: nearly always there are some)
    }
    if (near_entries && threadIdx.x < kNearEntries) {
        s_col[threadIdx.x] = col;
        s_val[threadIdx.x] = val;
    }
    if (join && threadIdx.x <= kJoinTokens) s_rowptr[threadIdx.x] = end;
    // row pointers are looked at in LDS, as far as they fit
    const bool near = !HID && !few && a.rowptr && a.n_tokens < kNearRows;
    if (near && named)
        for (int i = threadIdx.x; i <= a.n_tokens; i += Ex::THREADS) s_rowptr[i] = a.rowptr[i];
    for (int first = 0; named; first += most) {
        // the entries first .. first + most - 1 of those that name the expert
        int total = a.n_entries, leader = unit;
        if (few) {
            const uint64_t m = __builtin_amdgcn_ballot_w64(here == expert);
            total = __popcll(m);
            leader = __ffsll((unsigned long long)m) - 1;
            const int rank = __popcll(m & ((1ull << lane) - 1)) - first;
            if (here == expert && rank >= 0 && rank < most) {       // (all waves write the same)
                s_entry[rank] = lane;
                s_row[rank] = HID ? lane : here_row;
            }
        } else if (a.rowptr) {
            total = 0;
            for (int i0 = 0; i0 < a.n_entries; i0 += Ex::THREADS) {
                const int i = i0 + (int)threadIdx.x;
                const bool hit = i < a.n_entries && a.colidx[i] == expert;
                const uint64_t m = __builtin_amdgcn_ballot_w64(hit);
                if (lane == 0) s_count[wave] = __popcll(m);
                __syncthreads();
                int before = total;
#pragma unroll
                for (int w = 0; w < Ex::WAVES; ++w) {
                    if (w < wave) before += s_count[w];
                    total += s_count[w];
                }
                const int rank = before + __popcll(m & ((1ull << lane) - 1)) - first;
                if (hit && rank >= 0 && rank < most) {
                    s_entry[rank] = i;
                    if (HID) s_row[rank] = i;
                    else if (near) s_row[rank] = row_of_entry(s_rowptr, a.n_tokens, a.n_entries, i);
                    else s_row[rank] = row_of_entry(a.rowptr, a.n_tokens, a.n_entries, i);
                }
                __syncthreads();
            }
            if (first == 0 && total > 0) leader = s_entry[0];
        }
        total = __builtin_amdgcn_readfirstlane(total);
        if (total <= first) break;
        // (by entry: the first that names the expert does the work of all)
        if (by_entry && first == 0 && __builtin_amdgcn_readfirstlane(leader) != unit) break;
        const int count = min(total - first, most);
        if (first > 0) x.start(w, a, k_wave);
        if (!a.rowptr) {
            if ((int)threadIdx.x < count) s_entry[threadIdx.x] = s_row[threadIdx.x] = first + (int)threadIdx.x;
            __syncthreads();
        }
        if (count <= 4) x.template run<1, 4>(a, w, k_wave, row0, count, s_entry, s_row, smem);
        else if (count <= 16) x.template run<1, 16>(a, w, k_wave, row0, count, s_entry, s_row, smem);
        else if (Ex::MOST == 2 || count <= 32) x.template run<2, 16>(a, w, k_wave, row0, count, s_entry, s_row, smem);
        else x.template run<Ex::MOST, 16>(a, w, k_wave, row0, count, s_entry, s_row, smem);
        if (last_pass(first, total, most)) break;
        __syncthreads();
    }
    if constexpr (HID) {
        if (!join) return;
        // This workgroup's sums are where all others see them, then it counts itself in; the last one for a block of columns
        // adds up the entries of each token.  The sums are stored and loaded by relaxed atomics of agent scope, which pass the caches that
        // workgroups do not share, so it is enough that a thread's stores are complete (the wait for all of them) before its workgroup's
        // count; the fences only keep the compiler from moving accesses.  A release of agent scope would write back the whole L2.
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
        __builtin_amdgcn_s_waitcnt(0);
        __syncthreads();
        if (threadIdx.x == 0) s_last = atomicInc(a.arrived + tile, (unsigned)(gridDim.x / tiles - 1)) == gridDim.x / tiles - 1;
        __syncthreads();
        if (!s_last) return;
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
        const int cols = min(rows_per, a.n_rows - tile * rows_per);
        for (int i = threadIdx.x; i < a.n_tokens * cols; i += Ex::THREADS) {
            const int t = i / cols, c = tile * rows_per + i % cols;
            const float *Y = static_cast<const float *>(a.out);
            const float d = near_entries ? combine_entries<true>(s_rowptr[t], s_rowptr[t + 1], s_col, s_val, Y, a.ldo, a.n_experts, c)
                                         : combine_entries<true>(s_rowptr[t], s_rowptr[t + 1], a.colidx, a.vals, Y, a.ldo, a.n_experts, c);
            static_cast<typename El<EL>::T *>(a.D)[(int64_t)t * a.ldd + c] = El<EL>::put(d);
        }
    }
}

template <int EL> __global__ __launch_bounds__(256) void k_combine(const ExpertLaunch a, int col_blocks) {
    const int t = a.first_token + (int)(blockIdx.x / col_blocks), c = blockIdx.x % col_blocks * 256 + threadIdx.x;
    if (c >= a.n_rows) return;
    static_cast<typename El<EL>::T *>(a.D)[(int64_t)t * a.ldd + c] =
        El<EL>::put(combine_entries<false>(max(a.rowptr[t], 0), min(a.rowptr[t + 1], a.n_entries), a.colidx, a.vals, static_cast<const float *>(a.out), a.ldo, a.n_experts, c));
}

// Entries of an expert that a launch is made for: one a token, as a router leaves them.  (Rows may name an expert more than once:
// what is more takes further passes.)
inline int usual_entries(const ExpertLaunch &a) { return a.rowptr ? a.n_tokens : a.n_entries; }

template <int EL, int KIND, int G, bool HID, int NF> int launch_experts_nf(ExpertLaunch a, int64_t units, int k_waves, hipStream_t st) {
    typedef Expert<EL, KIND, G, HID, NF> Ex;
    a.pass_entries = Ex::pass_of(usual_entries(a));
    const int lds = Ex::pass_bytes(a.pass_entries, (a.n_cols + Ex::STEP - 1) / Ex::STEP);
    const int rows_per = Ex::WAVES / k_waves * 16 * (a.gated ? NF / 2 : NF);
    const int64_t tiles = (a.n_rows + rows_per - 1) / rows_per;
    a.k_waves = k_waves;
    // (more LDS than a launch may ask for by default; a limit of the kernel on one device)
    static DoneOnDevices raised;
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e == hipSuccess && !raised.has(device)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_experts<EL, KIND, G, HID, NF>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, 144 << 10);
        if (e == hipSuccess) raised.add(device);
    }
    if (e != hipSuccess) return (int)e;
    hipLaunchKernelGGL((k_experts<EL, KIND, G, HID, NF>), dim3((unsigned)(tiles * units)), dim3(Ex::THREADS), lds, st, a);
    return (int)hipGetLastError();
}
// The most waves of a workgroup that may share columns: each has a step of every chunk.
template <typename Ex> int most_k_waves(int most) {
    return std::min(Ex::WAVES, Ex::pass_steps(Ex::pass_of(most)));
}
// How a launch is cut: k_waves and an estimate of its time, in steps of a wave that multiplies two blocks of rows.
struct ExpertCut {
    int k_waves;
    double cost;
};
// Workgroups run in rounds of as many as the card holds (two of four waves a compute unit, or one of eight), each as long
// as its waves' steps and some four more for what comes before and after them.  A step of one block of rows takes 0.6 of one of
// two.  More waves on the same columns make shorter workgroups, and more of them.  (64 bf16 rows times 4-bit 8192 x 8192: one block
// of rows and four waves on the same columns 37 us, two blocks 58 to 109; fp16 row times 32768 x 8192: two blocks and two waves 29.7,
// four 32.5, one 37, one block 38 to 64.)
// units: experts that have work, in the mean; launched: those that workgroups are launched for.  k_waves is 0 if no cut fits a launch.
template <typename Ex, int NF> ExpertCut cut_experts(const ExpertLaunch &a, int most, double units, int64_t launched) {
    const int steps = (a.n_cols + Ex::STEP - 1) / Ex::STEP;
    const double slots = NF == 1 ? 256.0 : 512.0, step = NF == 1 ? 0.6 : 1.0;
    const double passes = a.rowptr ? 1.0 : (double)ceil_div(most, 16 * Ex::MOST);
    ExpertCut best{0, 0.0};
    for (int k = most_k_waves<Ex>(most); k >= 1; k /= 2) {
        const int rows = Ex::WAVES / k * 16 * (a.gated ? NF / 2 : NF);
        const int64_t tiles = ceil_div(a.n_rows, rows);
        if (tiles * launched > most_workgroups(Ex::THREADS)) continue;
        const double rounds = std::ceil(tiles * units / slots);
        const double cost = rounds * passes * (step * ((steps + k - 1) / k) + 4.0);
        if (!best.k_waves || cost < best.cost) best = ExpertCut{k, cost};
    }
    return best;
}
template <int EL, int KIND, int G, bool HID> int launch_experts_hid(ExpertLaunch a, hipStream_t st) {
    const int most = usual_entries(a);
    const int64_t units = !a.rowptr ? 1 : a.n_entries < 1 ? 1 : a.n_entries <= a.n_experts ? a.n_entries : a.n_experts;
    if (HID && a.n_tokens > kJoinTokens) a.arrived = nullptr;
    // experts that entries name, if any is as likely as the other
    const double named = !a.rowptr ? 1.0 : std::max(1.0, a.n_experts * -std::expm1(a.n_entries * std::log1p(-1.0 / (a.n_experts + 1.0))));
    // Two blocks of rows a wave, so that what is read of X from LDS is used twice; one where workgroups would be too few otherwise.
    const ExpertCut two = cut_experts<Expert<EL, KIND, G, HID, 2>, 2>(a, most, named, units);
    const ExpertCut one = a.gated ? ExpertCut{0, 0.0} : cut_experts<Expert<EL, KIND, G, HID, 1>, 1>(a, most, named, units);
    if (!one.k_waves && !two.k_waves) return (int)hipErrorInvalidConfiguration;
    const int e = one.k_waves && (!two.k_waves || one.cost < two.cost) ? launch_experts_nf<EL, KIND, G, HID, 1>(a, units, one.k_waves, st)
                                                                         : launch_experts_nf<EL, KIND, G, HID, 2>(a, units, two.k_waves, st);
    if (e || !HID || a.arrived) return e;
    const int col_blocks = (a.n_rows + 255) / 256;
    const int64_t most_tokens = most_workgroups(256) / col_blocks;
    for (int64_t first = 0; first < a.n_tokens; first += most_tokens) {
        a.first_token = (int32_t)first;
        hipLaunchKernelGGL((k_combine<EL>), dim3((unsigned)(col_blocks * std::min(most_tokens, a.n_tokens - first))), dim3(256), 0, st, a, col_blocks);
        const hipError_t error = hipGetLastError();
        if (error != hipSuccess) return (int)error;
    }
    return 0;
}
template <int EL, int KIND, int G> int launch_experts_g(const ExpertLaunch &a, hipStream_t st) {
    return a.x_hidden ? launch_experts_hid<EL, KIND, G, true>(a, st) : launch_experts_hid<EL, KIND, G, false>(a, st);
}
template <int EL, int KIND> int launch_experts_kind(const ExpertLaunch &a, hipStream_t st) {
    return a.group == 128 ? launch_experts_g<EL, KIND, 1>(a, st)
                          : a.group == 64 ? launch_experts_g<EL, KIND, 2>(a, st) : launch_experts_g<EL, KIND, 4>(a, st);
}
template <int EL> int launch_experts_el(const ExpertLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.kind < 0) return launch_experts_g<EL, -1, 1>(a, st);
    return a.kind == TF_Q4_INT ? launch_experts_kind<EL, TF_Q4_INT>(a, st) : launch_experts_kind<EL, TF_Q4_E2M1>(a, st);
}

}  // namespace
}  // namespace tf
