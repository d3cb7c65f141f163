// Products of the cross entropy: C = M N^T, a tile of C by each workgroup, 16-bit operands (fp32 ones as they are or in three parts), sums in 32 bits.
//   logits  l = W X^T      ended by their largest, the sum of exponentials and the label's (loss), or by g = dloss (exp(l - lse) - [label]) (gradient)
//   dX^T    = W^T G^T      W by columns
//   dW^T    = X^T G        both by columns, K goes over the rows that count
// Bound by the matrix cores where there are many rows: 8192 rows, 4096 -> 32768 classes, bf16, tiles of 256 x 256: logits to sums 1.63 ms (1.35 PFLOP/s), to G
// 1.71, dX 1.58, dW 1.54.  A wave's 128 x 128 sums fill the accumulation registers, so 64 products follow 16 reads of LDS and one workgroup a compute unit
// suffices.  Instructions of 32 x 32 x 16 took 1.39 ms on zeros (these 1.41) but 1.79 on normal
// numbers, where the card's clock gives way.  With few rows bound by reading W: 1 row of 4096 -> 65536, tiles of 64 x 16: 99 us, 5.4 TB/s.
#pragma once
#include <algorithm>
#include <type_traits>

#include "tf_loss_device.h"
#include "tf_moe_device.h"

namespace tf {
namespace {

// Matrix instructions by the type of the elements: D (16 x 16) += M (16 x K) N^T, K 32 or (fp32) four times 4.  A lane holds eight (four) columns of K.
template <int EL> struct Mfma;
template <> struct Mfma<TF_F32> {
    typedef Float4 V;
    static __device__ __forceinline__ Float4 mul(V a, V b, Float4 c) {
#pragma unroll
        for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    }
};
template <> struct Mfma<TF_BF16> {
    typedef Bf8 V;
    static __device__ __forceinline__ Float4 mul(V a, V b, Float4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ void add(Float4 &c, V a, V b) { asm volatile("v_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};
template <> struct Mfma<TF_F16> {
    typedef Half8 V;
    static __device__ __forceinline__ Float4 mul(V a, V b, Float4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ void add(Float4 &c, V a, V b) { asm volatile("v_mfma_f32_16x16x32_f16 %0, %1, %2, %0" : "+a"(c) : "v"(a), "v"(b)); }
};

typedef __attribute__((address_space(3))) void *LdsPtr;
typedef short Short4 __attribute__((ext_vector_type(4)));
typedef short Short8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) Short4 *LdsShort4;

// A step of K: 128 bytes of a row, whose pieces of sixteen bytes are the units of all that follows.
template <int EL> struct Size {
    static constexpr int BYTES = EL == TF_F32 ? 4 : 2, PIECE = 16 / BYTES, STEP = 128 / BYTES;
};

// Sixteen bytes a lane from a buffer to LDS, lane by lane from `to` + AT on (bytes).  In assembly, because the compiler would have every read of
// LDS that transposes wait for all loads before it.  It writes no vector register; what it writes in LDS is waited for in arrive().  (Nothing
// else here uses m0, which cannot be named as clobbered.)
template <int AT> __device__ __forceinline__ void load_to_lds(const Words4 &from, uint32_t offset, uint32_t to) {
    asm volatile("s_add_u32 m0, %2, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, 0 offen lds" ::"v"(offset), "s"(from), "s"(to), "i"(AT) : "scc");
}

// A step of an operand in LDS: W rows (of M or N) x 64 columns (K; 32 of fp32) if it lies in memory that way, else 64 rows (K) x W columns
// (TR).  It comes sixteen bytes a lane straight from memory, 1 KiB an instruction, and LDS gets them in the order of the lanes; so
// that sixteen lanes that read an operand of an instruction meet different banks, the pieces of a row are permuted on the way
// by which lane asks for which: piece p of row r is at p ^ (r & 7); with TR piece p of row k at p ^ swap(k): a unit of
// sixteen columns stays one.
template <int EL> __device__ __forceinline__ int swap(int k) { return EL == TF_F32 ? ((k >> 2) & 3) << 2 : ((k & 3) | ((k >> 3) & 1) << 2) << 1; }
template <int EL, int W, bool TR, int WAVES> struct Loader {
    static constexpr int BYTES = Size<EL>::BYTES, PIECE = Size<EL>::PIECE, STEP = Size<EL>::STEP;
    static constexpr int INSTR = W / 8, PER = (INSTR + WAVES - 1) / WAVES, PER_LEAST = INSTR / WAVES, CPR = TR ? W / PIECE : 8;
    static_assert(!TR || W >= 64, "rows of a transposed operand");
    uint32_t off[PER];             // of each instruction's sixteen bytes, from the step's first ones on
    uint64_t base, at;             // of the tile in a part's first step; of the step that comes next
    uint32_t row, stride;          // bytes from row to row, from step to step
    uint32_t records, tail;        // bytes of a whole step, of a row of it (TR)
    int32_t left, left0;           // of K: from the next step on, in all

    static __device__ __forceinline__ int row_of(int j, int lane) { return j * (64 / CPR) + lane / CPR; }
    static __device__ __forceinline__ int chunk_of(int j, int lane) {
        const int r = row_of(j, lane), s = lane % CPR;
        return TR ? s ^ (swap<EL>(r) & (CPR - 1)) : s ^ (r & 7);
    }
    // first: the tile's first row of M or N; k: the first column (row with TR) of K.
    __device__ __forceinline__ void begin(const Side &s, int64_t first, int64_t k, int part, int wave, int lane) {
        row = (uint32_t)(s.ld * BYTES);
        const int64_t there = (TR ? s.cols : s.rows) - first;      // of M or N
        const uint32_t some = (uint32_t)(there < 0 ? 0 : there < W ? there : W);
        tail = some * BYTES;
        base = (uint64_t)s.p + (uint64_t)((TR ? k * s.ld + first : first * s.ld + k) * BYTES);
        stride = TR ? STEP * row : 128;
        records = TR ? (STEP - 1) * row + tail : some ? (some - 1) * row + 128 : 0;
        left0 = (int32_t)((TR ? s.rows : s.cols) - k);
        go_to(s, part);
#pragma unroll
        for (int c = 0; c < PER; ++c) {
            const int j = wave + WAVES * c;
            const uint32_t o = (uint32_t)row_of(j, lane) * row + chunk_of(j, lane) * 16;
            off[c] = (uint32_t)(TR ? chunk_of(j, lane) * PIECE : row_of(j, lane)) < some ? o : ~0u;
        }
    }
    __device__ __forceinline__ void go_to(const Side &s, int part) {
        at = base + (uint64_t)(part * s.plane * BYTES);
        left = left0;
    }
    // Where the next step lies, what lies behind its end counting as zeros; goes on to the one after it.
    __device__ __forceinline__ Words4 next(int lane) {
        const uint32_t n = !TR || left >= STEP ? records : left <= 0 ? 0u : (uint32_t)(left - 1) * row + tail;
        // (the same for all lanes, which the compiler does not always see)
        const auto one = [](uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); };
        const Words4 w{one((uint32_t)at), one((uint32_t)(at >> 32)), one(n), 0x00020000u};
        if (!TR && left < STEP) {
            // The last step, which ends inside of its columns.  (A lane's columns are the same ones in every instruction; numbers in parts have
            // whole steps, so that this is the end of all steps.)
            if (chunk_of(0, lane) * PIECE >= left)
#pragma unroll
                for (int c = 0; c < PER; ++c) off[c] = ~0u;
        }
        at += stride;
        left -= STEP;
        return w;
    }
    // Instruction C of those that load a step into LDS from lds + AT on; lds: of this wave's first instruction.
    template <int C, int AT> __device__ __forceinline__ void load(const Words4 &from, uint32_t lds, bool, int wave, int) const {
        if (INSTR % WAVES == 0 || wave + WAVES * C < INSTR) load_to_lds<AT + WAVES * C * 1024>(from, off[C], lds);
    }
    __device__ __forceinline__ void put(char *, int, int) const {}
};

// The same for rows that begin at any element: through registers.  A step is fetched where the other loader's loads go out, and put into LDS before the
// barrier that they are waited for at.
template <int EL, int W, bool TR, int WAVES> struct AnyLoader {
    typedef Loader<EL, W, TR, WAVES> Way;
    static constexpr int BYTES = Way::BYTES, PIECE = Way::PIECE, STEP = Way::STEP;
    static constexpr int INSTR = Way::INSTR, PER = Way::PER, PER_LEAST = 0;      // (no load of it is waited for by counting)
    const char *at;                // the next step's first row and column
    int64_t row, stride;           // bytes from row to row, from step to step
    int32_t some, left;            // of M or N in the tile; of K from the next step on
    bool wide;                     // rows have a piece or more
    Words4 r[PER];

    __device__ __forceinline__ void begin(const Side &s, int64_t first, int64_t k, int, int, int) {
        row = s.ld * BYTES;
        const int64_t there = (TR ? s.cols : s.rows) - first;
        some = (int32_t)(there < 0 ? 0 : there < W ? there : W);
        left = (int32_t)((TR ? s.rows : s.cols) - k);
        wide = s.cols >= PIECE;
        at = static_cast<const char *>(s.p) + (TR ? k * s.ld + first : first * s.ld + k) * BYTES;
        stride = TR ? STEP * row : 128;
    }
    __device__ __forceinline__ void go_to(const Side &, int) {}
    __device__ __forceinline__ Words4 next(int) { return Words4{0, 0, 1, 0}; }
    // (is: there is such a step)
    template <int C, int AT> __device__ __forceinline__ void load(const Words4 &, uint32_t, bool is, int wave, int lane) {
        const int j = wave + WAVES * C;
        if (INSTR % WAVES != 0 && j >= INSTR) return;
        const int o = Way::row_of(j, lane), c = Way::chunk_of(j, lane) * PIECE, n = (TR ? some : left) - c;
        const char *p = at + o * row + c * BYTES;
        Words4 w{0, 0, 0, 0};
        if (is && o < (TR ? left : some)) {
            if (n >= PIECE) {
                w = *reinterpret_cast<const AnyWords4 *>(p);
            } else if (n > 0 && wide) {
                // the row's last piece, whose first elements go
                const AnyWords4 x = *reinterpret_cast<const AnyWords4 *>(p - (PIECE - n) * BYTES);
                const uint64_t lo = x[0] | (uint64_t)x[1] << 32, hi = x[2] | (uint64_t)x[3] << 32;
                const int off = 8 * BYTES * (PIECE - n);        // 16 .. 112 bits
                const uint64_t l = off < 64 ? lo >> off | hi << (64 - off) : hi >> (off - 64), h = off < 64 ? hi >> off : 0;
                w = Words4{(uint32_t)l, (uint32_t)(l >> 32), (uint32_t)h, (uint32_t)(h >> 32)};
            } else if (n > 0) {
                for (int i = 0; i < n; ++i) {
                    if constexpr (BYTES == 4) {
                        w[i] = reinterpret_cast<const uint32_t *>(p)[i];
                    } else {
                        const uint32_t x = reinterpret_cast<const uint16_t *>(p)[i];
                        w[i / 2] |= x << (16 * (i & 1));
                    }
                }
            }
        }
        r[C] = w;
    }
    __device__ __forceinline__ void put(char *lds, int wave, int lane) {
#pragma unroll
        for (int c = 0; c < PER; ++c)
            if (INSTR % WAVES == 0 || wave + WAVES * c < INSTR) *reinterpret_cast<Words4 *>(lds + (wave + WAVES * c) * 1024 + lane * 16) = r[c];
        at += stride;
        left -= STEP;
    }
};

// T operands of 16 rows x half a step, from row `first` of the step on: lane l has row l % 16 and a piece of K, number l / 16 of the half's four.
template <int EL, int W, bool TR, int T> struct Reader {
    static constexpr int BYTES = Size<EL>::BYTES, PIECE = Size<EL>::PIECE, HALF = Size<EL>::STEP / 2;
    typedef typename Mfma<EL>::V V;
    uint32_t at[TR ? T : 2];
    __device__ __forceinline__ void begin(int first, int lane) {
        if constexpr (TR && BYTES == 4) {
            const int k = 4 * (lane / 16), m = lane % 16;
#pragma unroll
            for (int i = 0; i < T; ++i) at[i] = k * (W * 4) + (((first + 16 * i + m) / 4) ^ (swap<EL>(k) & (W / 4 - 1))) * 16 + m % 4 * 4;
        } else if constexpr (TR) {
            const int k = 8 * (lane / 16) + lane % 16 / 4;
#pragma unroll
            for (int i = 0; i < T; ++i) at[i] = k * (W * 2) + (((first + 16 * i) / 8 + lane % 4 / 2) ^ (swap<EL>(k) & (W / 8 - 1))) * 16 + lane % 2 * 8;
        } else {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = (first + lane % 16) * 128 + (((kk * 4 + lane / 16) ^ (lane & 7)) * 16);
        }
    }
    // Operand i of half kk of a step that lies at lds.
    __device__ __forceinline__ V read(const char *lds, int kk, int i) const {
        if constexpr (TR && BYTES == 4) {
            const char *p = lds + at[i] + kk * HALF * W * 4;
            return V{*reinterpret_cast<const float *>(p), *reinterpret_cast<const float *>(p + W * 4), *reinterpret_cast<const float *>(p + W * 8),
                     *reinterpret_cast<const float *>(p + W * 12)};
        } else if constexpr (TR) {
            const Short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)(lds + at[i] + kk * HALF * W * 2));
            const Short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)(lds + at[i] + kk * HALF * W * 2 + 4 * W * 2));
            return __builtin_bit_cast(V, (Short8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
        } else {
            return *reinterpret_cast<const V *>(lds + at[kk] + i * 2048);
        }
    }
};

// Waits for this wave's reads and for its loads but the last LATER ones, then for all waves.
template <int LATER> __device__ __forceinline__ void arrive() { asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"i"(LATER) : "memory"); }

// The parts of M and N whose products are summed, small products first.
__device__ __forceinline__ int part_m(int pair) { return (0x001102 >> (4 * pair)) & 15; }
__device__ __forceinline__ int part_n(int pair) { return (0x010120 >> (4 * pair)) & 15; }

template <int EL> __device__ __forceinline__ void split3(float x, uint16_t (&p)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        p[i] = El<EL>::put(x);
        x -= El<EL>::get(p[i]);
    }
}

// Numbers that another workgroup of the launch may read: past the caches that it does not share.
__device__ __forceinline__ void store_past(float *to, float x) { __hip_atomic_store(to, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void store_past(Float2 *to, Float2 x) {
    __hip_atomic_store(reinterpret_cast<uint64_t *>(to), __builtin_bit_cast(uint64_t, x), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ Float2 load_past(const Float2 *from) {
    return __builtin_bit_cast(Float2, __hip_atomic_load(reinterpret_cast<const uint64_t *>(from), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
}

// The last workgroup of the `blocks` sums of rows first .. first + n adds them up in an order of its own and writes the losses: where there are few sums
// that is sooner done than another launch.  A thread's stores are complete (the wait for all of them) before its workgroup's count; stores and loads pass
// the caches that workgroups do not share, and the fences only keep the compiler from moving them.
template <int THREADS> __device__ __forceinline__ void join_sums(const ProductLaunch &a, char *lds, int tile, int64_t first, int n, int blocks) {
    int *flag = reinterpret_cast<int *>(lds + THREADS * sizeof(Float2));
    Float2 *sums = reinterpret_cast<Float2 *>(lds);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup");
    __builtin_amdgcn_s_waitcnt(0);
    __syncthreads();
    if (a.m_tiles > 1) {
        if (threadIdx.x == 0) *flag = atomicInc(a.arrived + tile * kJoinApart, (unsigned)a.m_tiles - 1) == (unsigned)a.m_tiles - 1;
        __syncthreads();
        if (!*flag) return;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup");
    const int rows = n <= 1 ? 1 : 1 << (32 - __builtin_clz((unsigned)n - 1)), r = threadIdx.x & (rows - 1), slices = THREADS / rows;
    Float2 x{-__builtin_inff(), 0.0f};
    if (r < n) {
        const Float2 *p = a.part + first + r;
        for (int b0 = threadIdx.x / rows; b0 < blocks; b0 += 8 * slices) {
            Float2 y[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = load_past(p + (int64_t)min(b0 + i * slices, blocks - 1) * a.part_ld);
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (b0 + i * slices < blocks) x = add_sums(x, y[i]);
        }
    }
    for (int d = rows; d < 64; d <<= 1) x = add_sums(x, Float2{__shfl_xor(x[0], d, 64), __shfl_xor(x[1], d, 64)});
    sums[threadIdx.x] = x;
    __syncthreads();
    if ((int)threadIdx.x >= n) return;
    for (int s = max(rows, 64); s < THREADS; s += max(rows, 64)) x = add_sums(x, sums[s + threadIdx.x]);
    const int64_t to = a.out_row[first + threadIdx.x];
    write_loss(x, __hip_atomic_load(a.hit + first + threadIdx.x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), a.loss + to, a.lse_out + to);
}

// Four 16-bit numbers.
typedef uint32_t Words2 __attribute__((ext_vector_type(2), aligned(2)));
template <int EL> __device__ __forceinline__ Words2 pack4(float a, float b, float c, float d) {
    return Words2{El<EL>::put(a) | (uint32_t)El<EL>::put(b) << 16, El<EL>::put(c) | (uint32_t)El<EL>::put(d) << 16};
}
// Two neighbouring tiles of results lie in a lane as four columns of each; exchanged between rows of sixteen lanes, as eight columns of one (those that
// columns_of(number of the first tile, lane / 16) tells): stores of 16 bytes, 64 in a line.  dW of 128 rows, 4096 -> 20000, 62 us; with stores of 8 bytes,
// 32 in a line, 73.
__device__ __forceinline__ int columns_of(int x, int g) { return 16 * (x + (g & 1)) + 8 * (g >> 1); }
__device__ __forceinline__ AnyWords4 eight_columns(Words2 a, Words2 b) {
    const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false), hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    return AnyWords4{(uint32_t)lo[0], (uint32_t)hi[0], (uint32_t)lo[1], (uint32_t)hi[1]};
}
// N of them to columns c, c + 1, ... of a row, those behind its last one left out.
template <int N> __device__ __forceinline__ void put_columns(uint16_t *row, int64_t c, int64_t columns, AnyWords4 w) {
    if (c + N <= columns) {
        if constexpr (N == 8) *reinterpret_cast<AnyWords4 *>(row + c) = w;
        else *reinterpret_cast<Words2 *>(row + c) = Words2{w[0], w[1]};
    } else {
#pragma unroll
        for (int v = 0; v < N; ++v)
            if (c + v < columns) row[c + v] = (uint16_t)(w[v / 2] >> (16 * (v & 1)));
    }
}

// f(0), f(1), ... f(N - 1), the number known when the code is made.
template <int N, int I = 0, typename F> __device__ __forceinline__ void each(F &&f) {
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        each<N, I + 1>(f);
    }
}

template <int EL, int WM, int WN, int TM, int TN, int PLACES, bool ANY, bool MTR, bool NTR, int END>
__global__ __launch_bounds__(WM * WN * 64, TM * TN > 32 ? 1 : 2) void k_product(const ProductLaunch a) {
    constexpr int WAVES = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16;
    constexpr int STEP = Size<EL>::STEP;
    constexpr bool BIG = TM * TN > 32;      // sums fill the accumulation registers: left alone, the compiler moves them about in every step
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const int kept = *a.n;
    // Tiles: a contiguous share for each XCD, in bands of eight rows of tiles, so that the 32 workgroups that an XCD runs at a time are eight by four
    // tiles and its L2 is asked for twelve pieces of operands a step, not 33.
    // (Only as many as there are kept rows for; a share of K that would have too few steps is not made.)
    int steps = a.k_rows ? (kept + STEP - 1) / STEP : a.k_steps;
    const int n_tiles = a.n_rows ? (kept + BN - 1) / BN : a.n_tiles, splits = shares_of(a.splits, steps, a.parts);
    const int tiles = a.m_tiles * n_tiles, all = tiles * splits;
    int b = blockIdx.x;
    if (b >= all) return;
    {
        const int xcd = b & 7, at = b >> 3, each = all >> 3, more = all & 7;
        b = xcd * each + min(xcd, more) + at;
    }
    const int split = b / tiles, tile = b % tiles;
    const int band = tile / (8 * n_tiles), high = min(8, a.m_tiles - 8 * band), in_band = tile - band * 8 * n_tiles;
    const int mt = 8 * band + in_band % high, nt = in_band / high;
    const int64_t m0 = (int64_t)mt * BM, n0 = (int64_t)nt * BN;
    Side M = a.M, N = a.N;
    if (a.k_rows) {
        M.rows = N.rows = kept;
        if (EL == TF_F16 && !*a.same) N.p = static_cast<const uint16_t *>(N.p) + a.g_plane;
    }
    const int s0 = (int)((int64_t)steps * split / splits), s1 = (int)((int64_t)steps * (split + 1) / splits);
    const int pairs = a.parts == 3 ? 6 : 1, total = pairs * (s1 - s0);
    int pair = a.parts == 3 ? 0 : 5, in_pair = s1 - s0, to_load = total;
    typedef std::conditional_t<ANY, AnyLoader<EL, BM, MTR, WAVES>, Loader<EL, BM, MTR, WAVES>> LM;
    typedef Loader<EL, BN, NTR, WAVES> LN;
    LM lm;
    LN ln;
    lm.begin(M, m0, (int64_t)s0 * STEP, part_m(pair), wave, lane);
    ln.begin(N, n0, (int64_t)s0 * STEP, part_n(pair), wave, lane);
    Reader<EL, BM, MTR, TM> rm;
    Reader<EL, BN, NTR, TN> rn;
    rm.begin(wm * TM * 16, lane);
    rn.begin(wn * TN * 16, lane);
    Float4 acc[TM][TN] = {};
    Words4 from_m, from_n;
    auto next = [&]() {           // sets up the loads of the next step
        from_m = lm.next(lane);
        from_n = ln.next(lane);
        if (--to_load < 0) from_m[2] = from_n[2] = 0;
        if (--in_pair == 0 && to_load > 0) {
            in_pair = s1 - s0;
            ++pair;
            lm.go_to(M, part_m(pair));
            ln.go_to(N, part_n(pair));
        }
    };
    constexpr int LOADS = LM::PER + LN::PER, READS = TM + TN, PRODUCTS = TM * TN;
    // LDS has places for PLACES steps, first M's, then N's.  A step's place is known when the code is made: then all addresses are registers that stay and
    // a constant.  A wave waits until all but the loads of the steps behind the next one have arrived.
    constexpr int AT_N = PLACES * BM * 128, LEAST = LM::PER_LEAST + LN::PER_LEAST;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(LdsPtr)lds + wave * 1024;
    auto load = [&](auto c, auto to) {
        constexpr int C = decltype(c)::value, TO = decltype(to)::value;
        if constexpr (C < LM::PER) lm.template load<C, TO * BM * 128>(from_m, lds0, to_load >= 0, wave, lane);
        else if constexpr (C < LOADS) ln.template load<C - LM::PER, AT_N + TO * BN * 128>(from_n, lds0, true, wave, lane);
    };
    auto put = [&](auto to) { lm.put(lds + decltype(to)::value * BM * 128, wave, lane); };
    typename Mfma<EL>::V vm[2][TM], vn[2][TN];
    auto read = [&](int r, int half, int from) {
        if (r < TM) vm[half][r] = rm.read(lds + from * BM * 128, half, r);
        else if (r < READS) vn[half][r - TM] = rn.read(lds + AT_N + from * BN * 128, half, r - TM);
    };
    // Multiplies one half of a step.  Meanwhile the other half's operands come from LDS (`reads`: of the step at place `from`), the loads of a step go
    // out (`loads`: to place `to`), or are set up.  An instruction of the matrix cores takes the time of four others: these are spread, a few
    // behind each product.
    auto multiply = [&](auto half, auto reads, auto from, auto loads, auto to, auto sets_up) {
        constexpr int HALF = decltype(half)::value, SLOTS = PRODUCTS > 1 ? PRODUCTS / 2 : 1;
        each<PRODUCTS>([&](auto slot) {
            constexpr int P = decltype(slot)::value;
            if constexpr (decltype(loads)::value && P < SLOTS)
                each<LOADS * (P + 1) / SLOTS - LOADS * P / SLOTS>([&](auto c) { load(std::integral_constant<int, LOADS * P / SLOTS + decltype(c)::value>{}, to); });
            if constexpr (decltype(reads)::value && P < SLOTS) {
                // (half a turn later than the loads)
                constexpr int lo = P ? (READS * (2 * P + 1) / 2) / SLOTS : 0, hi = P + 1 < SLOTS ? (READS * (2 * P + 3) / 2) / SLOTS : READS;
                each<hi - lo>([&](auto r) { read(lo + decltype(r)::value, 1 - HALF, decltype(from)::value); });
            }
            if constexpr (decltype(sets_up)::value && P == (SLOTS < PRODUCTS ? SLOTS : PRODUCTS - 1)) next();
            constexpr int x = P / TN, y = P % TN;
            if constexpr (BIG) Mfma<EL>::add(acc[x][y], vm[HALF][x], vn[HALF][y]);
            else acc[x][y] = Mfma<EL>::mul(vm[HALF][x], vn[HALF][y], acc[x][y]);
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    constexpr std::integral_constant<int, 0> zero{};
    constexpr std::integral_constant<int, 1> one{};
    constexpr std::true_type yes{};
    constexpr std::false_type no{};
    // The barrier lies between a step's halves: behind it the next step is in LDS, and nobody reads this one any more.
    auto step = [&](auto place, auto other) {
        multiply(zero, yes, place, no, zero, yes);
        // (what is fetched is the step that the place before this one is for)
        put(std::integral_constant<int, (decltype(place)::value + PLACES - 1) % PLACES>{});
        arrive<(PLACES - 2) * LEAST>();
        multiply(one, yes, other, yes, place, no);
    };
    each<PLACES>([&](auto place) {
        next();
        each<LOADS>([&](auto c) { load(c, place); });
        if constexpr (decltype(place)::value + 1 < PLACES) put(place);
    });
    arrive<(PLACES - 1) * LEAST>();
#pragma unroll
    for (int r = 0; r < READS; ++r) read(r, 0, 0);
    // A round of steps, as addresses are made for; steps behind the last one are zeros, which come from no memory.
    for (int i = 0; i < total; i += PLACES)
        each<PLACES>([&](auto place) { step(place, std::integral_constant<int, (decltype(place)::value + 1) % PLACES>{}); });
    arrive<0>();        // (loads that nobody reads: LDS is given away when the workgroup ends)
    if constexpr (BIG) {
        // (the compiler does not know what the last instructions write, nor when)
        asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }
    auto value = [&](int x, int y, int v) {
        if constexpr (BIG) {
            float f;
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(f) : "a"(acc[x][y][v]));
            return f;
        } else {
            return acc[x][y][v];
        }
    };
    // Lane 16 g + r holds, of acc[x][y], rows 16 x + 4 g .. + 3 of M (from `mw` on) and row 16 y + r of N.
    const int g = lane / 16;
    const int64_t mw = m0 + wm * TM * 16, nw = n0 + wn * TN * 16 + lane % 16;
    if constexpr (END == kEndSums || END == kEndGradient) {
        // Exponentials are powers of two of l log2(e) - c: one multiplication and addition and one instruction of a quarter of the others' rate for each
        // logit, 256 of them a lane.  What c = fl(top log2(e)) is off by scales all terms alike, by less than 2^-24 |top|.
        constexpr float LOG2E = 1.44269504088896340736f;
        const bool whole = mw + TM * 16 <= a.m_count;
        const bool same = EL == TF_F16 && END == kEndGradient && *a.same, first_plane = a.for_dx || same, second_plane = a.for_dw && !same;
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int64_t row = nw + 16 * y;
            const bool is = row < kept;
            const int label = is ? a.label[row] - a.first_class : -1;
            const int64_t at = (int64_t)label - mw - 4 * g;      // 16 x + v where the label's logit is in this lane
            const bool any = __ballot(at >= 0 && at < 16 * TM && (at & 15) < 4) != 0;      // (in this wave: seldom)
            if constexpr (END == kEndSums) {
                float top = -__builtin_inff(), sum = 0.0f, l[TM][4];
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) l[x][v] = value(x, y, v);
                if (!whole)
#pragma unroll
                    for (int x = 0; x < TM; ++x)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (mw + 16 * x + 4 * g + v >= a.m_count) l[x][v] = -__builtin_inff();
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) top = fmaxf(top, l[x][v]);
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                if (any)        // the label's own is added to the sum at the end
#pragma unroll
                    for (int x = 0; x < TM; ++x)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (at == 16 * x + v) {
                                store_past(a.hit + row, l[x][v]);
                                l[x][v] = -__builtin_inff();
                            }
                const float from = top == -__builtin_inff() ? 0.0f : top * LOG2E;
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) sum += __builtin_amdgcn_exp2f(fmaf(l[x][v], LOG2E, -from));
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                if constexpr (WN > 1) {
                    if (is && g == 0) store_past(a.part + ((int64_t)mt * WM + wm) * a.part_ld + row, Float2{top, sum});
                } else {        // few rows: the waves' sums are put together first
                    Float2 *all = reinterpret_cast<Float2 *>(lds);
                    if (g == 0) all[(wm * TN + y) * 16 + lane] = Float2{top, sum};
                    if (y == TN - 1) {
                        __syncthreads();
                        for (int i = threadIdx.x; i < 16 * TN; i += 64 * WM) {
                            const int64_t to = n0 + i;
                            Float2 x = all[i];
                            for (int w = 1; w < WM; ++w) x = add_sums(x, all[w * TN * 16 + i]);
                            if (to < kept) store_past(a.part + (int64_t)mt * a.part_ld + to, x);
                        }
                    }
                }
            } else if (is) {
                // The label's is exp(l - lse) - 1, which for rows that are nearly certain of it cancels to 2^-24 of lse; exp(-loss) - 1 does not.
                const float from = a.lse[row] * LOG2E, scale = a.g[row], own = any && a.hit ? expm1f(a.hit[row]) : -1.0f, times = a.hit ? 0.0f : 1.0f;
                typedef typename El<EL>::T T;
                T *row_of_G = static_cast<T *>(a.G) + row * a.g_ld + mw, *out = row_of_G + 4 * g;
                typedef uint16_t U4 __attribute__((ext_vector_type(4)));
                Words2 before[2];
                // four columns, times `by`, to one of the planes
                auto put = [&](const float (&d)[4], float by, T *plane, int x, Words2 &before) __attribute__((always_inline)) {
                    if constexpr (EL != TF_F32) {
                        const Words2 w = pack4<EL>(d[0] * by, d[1] * by, d[2] * by, d[3] * by);
                        if constexpr (TM % 2 == 0) {
                            if (x % 2) *reinterpret_cast<AnyWords4 *>(plane + columns_of(x - 1, g)) = eight_columns(before, w);
                            else before = w;
                        } else {
                            *reinterpret_cast<Words2 *>(plane + 16 * x + 4 * g) = w;
                        }
                    }
                };
#pragma unroll
                for (int x = 0; x < TM; ++x) {
                    float d[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) d[v] = __builtin_amdgcn_exp2f(fmaf(value(x, y, v), LOG2E, -from));
                    if (any)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (at == 16 * x + v) d[v] = fmaf(d[v], times, own);
                    if constexpr (EL != TF_F16)
#pragma unroll
                        for (int v = 0; v < 4; ++v) d[v] *= scale;
                    if (!whole)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (mw + 16 * x + 4 * g + v >= a.m_count) d[v] = 0.0f;
                    if constexpr (EL == TF_F32) {
                        *reinterpret_cast<Float4 *>(out + 16 * x) = Float4{d[0], d[1], d[2], d[3]};
                    } else if (EL == TF_BF16 && a.parts == 3) {
                        uint16_t p[4][3];
#pragma unroll
                        for (int v = 0; v < 4; ++v) split3<EL>(d[v], p[v]);
#pragma unroll
                        for (int i = 0; i < 3; ++i) *reinterpret_cast<U4 *>(out + i * a.g_plane + 16 * x) = U4{p[0][i], p[1][i], p[2][i], p[3][i]};
                    } else if constexpr (EL == TF_F16) {
                        if (first_plane) put(d, 1.0f / kRowUnit, row_of_G, x, before[0]);
                        if (second_plane) put(d, scale, row_of_G + a.g_plane, x, before[1]);
                    } else {
                        put(d, 1.0f, row_of_G, x, before[0]);
                    }
                }
            }
        }
        if constexpr (END == kEndSums)
            if (a.join) join_sums<WM * WN * 64>(a, lds, nt, n0, (int)min((int64_t)BN, kept - n0), a.m_tiles * (WN > 1 ? WM : 1));
    } else if constexpr (END == kEndSlab) {
        const int64_t rows = a.n_rows ? kept : a.n_count;
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int64_t row = nw + 16 * y;
            if (row < rows) {
                float *out = a.slab + split * a.slab_size + row * a.slab_ld + mw + 4 * g;
#pragma unroll
                for (int x = 0; x < TM; ++x) {
                    Float4 *to = reinterpret_cast<Float4 *>(out + 16 * x);
                    const Float4 d = {value(x, y, 0), value(x, y, 1), value(x, y, 2), value(x, y, 3)};
                    *to = a.add ? *to + d : d;
                }
            }
        }
    } else {
        const float unit = *a.unit;
        const int64_t rows = a.n_rows ? kept : a.n_count;
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            int64_t row = nw + 16 * y;
            if (row >= rows) continue;
            const float times = EL == TF_F16 && a.row_unit ? a.row_unit[row] * kRowUnit : unit;
            if (a.out_row) row = a.out_row[row];
            Words2 before;
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                const int64_t m = mw + 16 * x + 4 * g;
                Float4 f;
#pragma unroll
                for (int v = 0; v < 4; ++v) f[v] = value(x, y, v) * times;
                if (EL == TF_F32 || a.out_dtype == TF_F32) {
                    float *to = static_cast<float *>(a.out) + row * a.ldo + m;
                    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
                    if (m + 4 <= a.m_count) *reinterpret_cast<F4 *>(to) = f;
                    else
                        for (int v = 0; v < 4; ++v)
                            if (m + v < a.m_count) to[v] = f[v];
                } else if constexpr (EL != TF_F32) {
                    uint16_t *to = static_cast<uint16_t *>(a.out) + row * a.ldo;
                    const Words2 w = pack4<EL>(f[0], f[1], f[2], f[3]);
                    if constexpr (TM % 2 == 0) {
                        const int64_t c = mw + columns_of(x - 1, g);
                        if (x % 2) put_columns<8>(to, c, a.m_count, eight_columns(before, w));
                        else before = w;
                    } else {
                        put_columns<4>(to, m, a.m_count, Words4{w[0], w[1], 0, 0});
                    }
                }
            }
        }
    }
}

template <int EL, int WM, int WN, int TM, int TN, int PLACES, bool ANY, bool MTR, bool NTR, int END> int product_with(ProductLaunch a, hipStream_t st) {
    constexpr int BM = WM * TM * 16, BN = WN * TN * 16, LDS = PLACES * (BM + BN) * 128;
    static DoneOnDevices done;
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return (int)e;
    if (!done.has(device)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(k_product<EL, WM, WN, TM, TN, PLACES, ANY, MTR, NTR, END>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return (int)e;
        done.add(device);
    }
    a.m_tiles = (int32_t)ceil_div(a.m_count, BM);
    a.n_tiles = (int32_t)ceil_div(a.n_count, BN);
    const int64_t groups = (int64_t)a.m_tiles * a.n_tiles * a.splits;
    if (groups == 0) return 0;
    if (groups > most_workgroups(WM * WN * 64)) return (int)hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_product<EL, WM, WN, TM, TN, PLACES, ANY, MTR, NTR, END>), dim3((unsigned)groups), dim3(WM * WN * 64), LDS, st, a);
    return (int)hipGetLastError();
}

template <int EL, bool ANY, bool MTR, bool NTR, int END> int product_tile(const ProductLaunch &a, hipStream_t st) {
    if constexpr (!NTR) {
        if (a.tile == kTile64) return product_with<EL, 4, 1, 2, 4, 3, ANY, MTR, NTR, END>(a, st);
        if (a.tile == kTile16) return product_with<EL, 4, 1, 1, 1, 4, ANY, MTR, NTR, END>(a, st);
    }
    if constexpr (ANY && END != kEndSums && EL != TF_F32) {
        return (int)hipErrorInvalidValue;       // (gradients of few rows only)
    } else {
        if constexpr (EL != TF_F32)
            if (a.tile == kTile256) return product_with<EL, 2, 2, 8, 8, 2, ANY, MTR, NTR, END>(a, st);
        return product_with<EL, 2, 2, 4, 4, 2, ANY, MTR, NTR, END>(a, st);
    }
}
template <int EL, bool MTR, int END> int product_any(const ProductLaunch &a, hipStream_t st) {
    return a.any ? product_tile<EL, true, MTR, false, END>(a, st) : product_tile<EL, false, MTR, false, END>(a, st);
}

// The four products: logits (their sums, or the gradient), dX (W by columns), dW (both operands by columns).
template <int EL> int product(const ProductLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.end == kEndSums) return product_any<EL, false, kEndSums>(a, st);
    if (a.end == kEndGradient) return product_any<EL, false, kEndGradient>(a, st);
    if (!a.k_rows) return a.end == kEndSlab ? product_any<EL, true, kEndSlab>(a, st) : product_any<EL, true, kEndOut>(a, st);
    return a.end == kEndSlab ? product_tile<EL, false, true, true, kEndSlab>(a, st) : product_tile<EL, false, true, true, kEndOut>(a, st);
}

}  // namespace
}  // namespace tf
