// Products of the cross entropy: C = M N^T, a tile of C by each workgroup, 16-bit operands, sums in 32 bits.
#pragma once
#include <algorithm>

#include "tf_loss.h"
#include "tf_moe_device.h"

namespace tf {
namespace {

template <int EL> struct Mfma;
template <> struct Mfma<TF_BF16> {
    typedef Bf8 V;
    static __device__ __forceinline__ Float4 mul(V a, V b, Float4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma<TF_F16> {
    typedef Half8 V;
    static __device__ __forceinline__ Float4 mul(V a, V b, Float4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

typedef __attribute__((address_space(3))) void *LdsPtr;
typedef short Short4 __attribute__((ext_vector_type(4)));
typedef short Short8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) Short4 *LdsShort4;

constexpr int kStep = 64;      // of K

// A step of an operand in LDS: W rows (of M or N) x 64 columns (K) if it lies in memory that way, else 64 rows (K) x W columns
// (TR).  It comes sixteen bytes a lane straight from memory, 1 KiB an instruction, and LDS gets them in the order of the lanes; so
// that sixteen lanes that read an operand of an instruction meet different banks, the pieces of a row are permuted on the way
// by which lane asks for which: piece p of row r is at p ^ (r & 7); with TR 32-byte units u of row k at u ^ (k & 3 | k / 8 % 2 * 4).
template <int W, bool TR, int WAVES> struct Loader {
    static constexpr int INSTR = W / 8, PER = (INSTR + WAVES - 1) / WAVES, CPR = TR ? W / 8 : 8;
    static_assert(!TR || W >= 64, "rows of a transposed operand");
    uint32_t off[PER];
    int chunk;                     // of the first one
    const char *base;
    int64_t left;                  // rows (TR) or columns of K from the base on
    int64_t ld2;                   // bytes

    static __device__ __forceinline__ int row_of(int j, int lane) { return j * (64 / CPR) + lane / CPR; }
    static __device__ __forceinline__ int chunk_of(int j, int lane) {
        const int r = row_of(j, lane), s = lane % CPR;
        return TR ? s ^ ((((r & 3) | ((r >> 3) & 1) << 2) << 1) & (CPR - 1)) : s ^ (r & 7);
    }
    int64_t outer, inner;          // of the tile, what there is

    // first: the tile's first row of M or N.
    __device__ __forceinline__ void begin(const Side &s, int64_t first, int wave, int lane) {
        ld2 = s.ld * 2;
        outer = TR ? s.cols - first : s.rows - first;
#pragma unroll
        for (int c = 0; c < PER; ++c) {
            const int j = wave + WAVES * c;
            const uint32_t o = (uint32_t)(row_of(j, lane) * (uint32_t)ld2 + chunk_of(j, lane) * 16);
            off[c] = (TR ? chunk_of(j, lane) * 8 < outer : row_of(j, lane) < outer) ? o : ~0u;
        }
    }
    // Loads the step that begins at column (row with TR) k of a part into `lds`.
    __device__ __forceinline__ void load(const Side &s, int64_t first, int64_t k, int part, char *lds, int wave, int lane) const {
        const char *p = static_cast<const char *>(s.p) + (part * s.plane + (TR ? k * s.ld + first : first * s.ld + k)) * 2;
        // bytes up to the end of the last row
        int64_t n = TR ? ((s.rows - k - 1) * ld2 + outer * 2) : ((outer - 1) * ld2 + (s.cols - k) * 2);
        if ((TR ? s.rows - k : outer) <= 0) n = 0;
        const auto r = __builtin_amdgcn_make_buffer_rsrc(const_cast<char *>(p), 0, (int)(uint32_t)(n < 0xffffffe0ll ? n : 0xffffffe0ll), 0x00020000);
#pragma unroll
        for (int c = 0; c < PER; ++c) {
            const int j = wave + WAVES * c;
            if (INSTR % WAVES == 0 || j < INSTR) {
                uint32_t o = off[c];
                if (!TR && k + kStep > s.cols && k + chunk_of(j, lane) * 8 >= s.cols) o = ~0u;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsPtr)(lds + j * 1024), 16, (int)o, 0, 0, 0);
            }
        }
    }
};

// T operands of 16 rows x 32 of K, from row `first` of the step on.
template <int W, bool TR, int T> struct Reader {
    uint32_t at[TR ? T : 2];
    __device__ __forceinline__ void begin(int first, int lane) {
        if constexpr (TR) {
            const int k = 8 * (lane / 16) + lane % 16 / 4, swap = (k & 3) | ((k >> 3) & 1) << 2;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                const int unit = (first / 16 + i) ^ (swap & (W / 16 - 1));
                at[i] = k * (W * 2) + unit * 32 + (lane % 4) * 8;
            }
        } else {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = (first + lane % 16) * 128 + (((kk * 4 + lane / 16) ^ (lane & 7)) * 16);
        }
    }
    template <int EL> __device__ __forceinline__ void read(typename Mfma<EL>::V (&v)[T], const char *lds, int kk) const {
#pragma unroll
        for (int i = 0; i < T; ++i) {
            if constexpr (TR) {
                const Short4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)(lds + at[i] + kk * 32 * W * 2));
                const Short4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsShort4)(lds + at[i] + kk * 32 * W * 2 + 4 * W * 2));
                v[i] = __builtin_bit_cast(typename Mfma<EL>::V, (Short8){lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]});
            } else {
                v[i] = *reinterpret_cast<const typename Mfma<EL>::V *>(lds + at[kk] + i * 2048);
            }
        }
    }
};

// Waits for this wave's loads, then for all waves.  (Neither builtin orders memory accesses for the compiler.)
__device__ __forceinline__ void arrive() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);      // vmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

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

template <int EL, int WM, int WN, int TM, int TN, bool MTR, bool NTR, int END>
__global__ __launch_bounds__(WM * WN * 64, 2) void k_product(const ProductLaunch a) {
    constexpr int WAVES = WM * WN, BM = WM * TM * 16, BN = WN * TN * 16, STAGE = (BM + BN) * 128;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    const int kept = a.n ? *a.n : 0;
    // tiles: a contiguous share for each XCD, whose L2 then meets few rows of M
    const int tiles = a.m_tiles * a.n_tiles, all = tiles * a.splits;
    int b = blockIdx.x;
    {
        const int xcd = b & 7, at = b >> 3, each = all >> 3, more = all & 7;
        b = xcd * each + min(xcd, more) + at;
    }
    const int split = b / tiles, tile = b % tiles;
    const int mt = tile / a.n_tiles, nt = tile % a.n_tiles;
    const int64_t m0 = (int64_t)mt * BM, n0 = (int64_t)nt * BN;
    if (a.n_rows && n0 >= kept) return;
    Side M = a.M, N = a.N;
    int steps = a.k_steps;
    if (a.k_rows) {
        steps = (kept + kStep - 1) / kStep;
        M.rows = N.rows = kept;
    }
    int s0 = 0, s1 = steps;
    if (a.splits > 1) {
        s0 = (int)((int64_t)steps * split / a.splits);
        s1 = (int)((int64_t)steps * (split + 1) / a.splits);
    }
    Loader<BM, MTR, WAVES> lm;
    Loader<BN, NTR, WAVES> ln;
    lm.begin(M, m0, wave, lane);
    ln.begin(N, n0, wave, lane);
    Reader<BM, MTR, TM> rm;
    Reader<BN, NTR, TN> rn;
    rm.begin(wm * TM * 16, lane);
    rn.begin(wn * TN * 16, lane);
    Float4 acc[TM][TN] = {};
    const int pairs = a.parts == 3 ? 6 : 1, total = pairs * (s1 - s0);
    int pair = a.parts == 3 ? 0 : 5, step = s0;
    char *cur = lds, *other = lds + STAGE;
    auto load = [&](char *to) {
        lm.load(M, m0, (int64_t)step * kStep, part_m(pair), to, wave, lane);
        ln.load(N, n0, (int64_t)step * kStep, part_n(pair), to + BM * 128, wave, lane);
        if (++step == s1) {
            step = s0;
            ++pair;
        }
    };
    if (total > 0) load(cur);
    for (int i = 0; i < total; ++i) {
        arrive();
        if (i + 1 < total) load(other);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            typename Mfma<EL>::V vm[TM], vn[TN];
            rm.template read<EL>(vm, cur, kk);
            rn.template read<EL>(vn, cur + BM * 128, kk);
#pragma unroll
            for (int x = 0; x < TM; ++x)
#pragma unroll
                for (int y = 0; y < TN; ++y) acc[x][y] = Mfma<EL>::mul(vm[x], vn[y], acc[x][y]);
        }
        char *t = cur;
        cur = other;
        other = t;
    }
    // Lane 16 g + r holds, of acc[x][y], rows 16 x + 4 g .. + 3 of M (from `mw` on) and row 16 y + r of N.
    const int g = lane / 16;
    const int64_t mw = m0 + wm * TM * 16, nw = n0 + wn * TN * 16 + lane % 16;
    if constexpr (END == kEndSums || END == kEndGradient) {
        const bool whole = mw + TM * 16 <= a.m_count;
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int64_t row = nw + 16 * y;
            const bool is = row < kept;
            const int label = is ? a.label[row] - a.first_class : -1;
            const int64_t at = (int64_t)label - mw - 4 * g;      // 16 x + v where the label's logit is in this lane
            if constexpr (END == kEndSums) {
                float top = -__builtin_inff(), sum = 0.0f;
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        if (!whole && mw + 16 * x + 4 * g + v >= a.m_count) acc[x][y][v] = -__builtin_inff();
                        top = fmaxf(top, acc[x][y][v]);
                        if (at == 16 * x + v) a.hit[row] = acc[x][y][v];
                    }
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
                for (int x = 0; x < TM; ++x)
#pragma unroll
                    for (int v = 0; v < 4; ++v) sum += at == 16 * x + v ? 0.0f : expf(acc[x][y][v] - from);      // (the label's is added at the end)
                sum += __shfl_xor(sum, 16, 64);
                sum += __shfl_xor(sum, 32, 64);
                if (is && g == 0) {
                    const int64_t to = ((int64_t)mt * WM + wm) * a.part_ld + row;
                    a.part_top[to] = top;
                    a.part_sum[to] = sum;
                }
            } else if (is) {
                const float lse = a.lse[row], scale = a.g[row];
                uint16_t *out = static_cast<uint16_t *>(a.G) + row * a.g_ld + mw + 4 * g;
#pragma unroll
                for (int x = 0; x < TM; ++x) {
                    uint16_t p[4][3];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        float d = (expf(acc[x][y][v] - lse) - (at == 16 * x + v ? 1.0f : 0.0f)) * scale;
                        if (!whole && mw + 16 * x + 4 * g + v >= a.m_count) d = 0.0f;
                        split3<EL>(d, p[v]);
                    }
                    typedef uint16_t U4 __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<U4 *>(out + 16 * x) = U4{p[0][0], p[1][0], p[2][0], p[3][0]};
                    if (a.parts == 3) {
                        *reinterpret_cast<U4 *>(out + a.g_plane + 16 * x) = U4{p[0][1], p[1][1], p[2][1], p[3][1]};
                        *reinterpret_cast<U4 *>(out + 2 * a.g_plane + 16 * x) = U4{p[0][2], p[1][2], p[2][2], p[3][2]};
                    }
                }
            }
        }
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
                    *to = a.add ? *to + acc[x][y] : acc[x][y];
                }
            }
        }
    } else {
        const float unit = *a.unit;
#pragma unroll
        for (int y = 0; y < TN; ++y) {
            const int64_t row = nw + 16 * y;
            if (row >= a.n_count) continue;
#pragma unroll
            for (int x = 0; x < TM; ++x) {
                const int64_t m = mw + 16 * x + 4 * g;
                if (a.out_dtype == TF_F32) {
                    float *to = static_cast<float *>(a.out) + row * a.ldo + m;
                    typedef float F4 __attribute__((ext_vector_type(4), aligned(4)));
                    const Float4 d = acc[x][y] * unit;
                    if (m + 4 <= a.m_count) *reinterpret_cast<F4 *>(to) = d;
                    else
                        for (int v = 0; v < 4; ++v)
                            if (m + v < a.m_count) to[v] = d[v];
                } else {
                    uint16_t *to = static_cast<uint16_t *>(a.out) + row * a.ldo + m;
                    typedef uint16_t U4 __attribute__((ext_vector_type(4), aligned(2)));
                    U4 d;
#pragma unroll
                    for (int v = 0; v < 4; ++v) d[v] = El<EL>::put(acc[x][y][v] * unit);
                    if (m + 4 <= a.m_count) *reinterpret_cast<U4 *>(to) = d;
                    else
                        for (int v = 0; v < 4; ++v)
                            if (m + v < a.m_count) to[v] = d[v];
                }
            }
        }
    }
}

template <int EL, int WM, int WN, int TM, int TN, bool MTR, bool NTR, int END> int product_with(ProductLaunch a, hipStream_t st) {
    constexpr int BM = WM * TM * 16, BN = WN * TN * 16, LDS = 2 * (BM + BN) * 128;
    static DoneOnDevices done;
    int device = 0;
    hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return (int)e;
    if (!done.has(device)) {
        e = hipFuncSetAttribute(reinterpret_cast<const void *>(k_product<EL, WM, WN, TM, TN, MTR, NTR, END>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, LDS);
        if (e != hipSuccess) return (int)e;
        done.add(device);
    }
    a.m_tiles = (int32_t)ceil_div(a.m_count, BM);
    a.n_tiles = (int32_t)ceil_div(a.n_count, BN);
    const int64_t groups = (int64_t)a.m_tiles * a.n_tiles * a.splits;
    if (groups == 0) return 0;
    if (groups > most_workgroups(WM * WN * 64)) return (int)hipErrorInvalidConfiguration;
    hipLaunchKernelGGL((k_product<EL, WM, WN, TM, TN, MTR, NTR, END>), dim3((unsigned)groups), dim3(WM * WN * 64), LDS, st, a);
    return (int)hipGetLastError();
}

template <int EL, bool MTR, bool NTR, int END> int product_tile(const ProductLaunch &a, hipStream_t st) {
    if (a.tile == kTile256) return product_with<EL, 2, 4, 8, 4, MTR, NTR, END>(a, st);
    if constexpr (!NTR) {
        if (a.tile == kTile64) return product_with<EL, 4, 1, 2, 4, MTR, NTR, END>(a, st);
        if (a.tile == kTile16) return product_with<EL, 4, 1, 2, 1, MTR, NTR, END>(a, st);
    }
    return product_with<EL, 2, 2, 4, 4, MTR, NTR, END>(a, st);
}

// The four products: logits (their sums, or the gradient), dX (W by columns), dW (both operands by columns).
template <int EL> int product(const ProductLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.end == kEndSums) return product_tile<EL, false, false, kEndSums>(a, st);
    if (a.end == kEndGradient) return product_tile<EL, false, false, kEndGradient>(a, st);
    if (a.end == kEndSlab && !a.k_rows) return product_tile<EL, true, false, kEndSlab>(a, st);
    if (a.end == kEndSlab) return product_tile<EL, true, true, kEndSlab>(a, st);
    return product_tile<EL, true, true, kEndOut>(a, st);
}

}  // namespace
}  // namespace tf
