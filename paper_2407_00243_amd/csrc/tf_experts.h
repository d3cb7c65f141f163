// Products of a few rows with the weights of the experts that name them (or with one 4-bit matrix).
#pragma once
#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr int kExpertWaves = 8, kExpertThreads = 64 * kExpertWaves;
constexpr int kExpertFrags = 2;       // blocks of sixteen rows of weights per workgroup

// Hidden rows of TF_F16 are held in two parts, high * 2^12 + low: fp16 alone ends at 65504, which a gate times
// what it gates passes easily.
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

// Eight weights of a word of codes, as numbers of sixteen bits (bf16 where X is fp32).  INT: sign and magnitude m
// sit where an e4m3 number has its sign and its lowest bits; without exponent bits that is m 2^-9.
template <int EL, int KIND> __device__ __forceinline__ Words4 q4_decode(uint32_t w) {
    Words4 y;
    if constexpr (KIND == TF_Q4_E2M1) {
        if constexpr (EL == TF_F16) {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 0));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 1));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 2));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, 1.0f, 3));
        } else {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 0));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 1));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 2));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, 1.0f, 3));
        }
    } else {
        const uint32_t lo = w & 0x87878787u, hi = __builtin_amdgcn_alignbit(w, w, 4) & 0x87878787u;
        if constexpr (EL == TF_F16) {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, false));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 512.0f, true));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, false));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 512.0f, true));
        } else {
            y[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, false));
            y[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.0f, true));
            y[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, false));
            y[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.0f, true));
        }
    }
    return y;
}

// Two fp32 numbers in three bf16 parts each (cut off, not rounded: the parts of a number have its sign and add up to it
// exactly, and no part of a finite number is infinite).  An infinity is its first part alone.
__device__ __forceinline__ void cut_pair(uint32_t &h, uint32_t &m, uint32_t &l, float a, float b) {
    const uint32_t ua = __float_as_uint(a), ub = __float_as_uint(b);
    h = (ua >> 16) | (ub & 0xffff0000u);
    float ra = a - __uint_as_float(ua & 0xffff0000u), rb = b - __uint_as_float(ub & 0xffff0000u);
    ra = __builtin_isinf(a) ? 0.0f : ra;
    rb = __builtin_isinf(b) ? 0.0f : rb;
    const uint32_t va = __float_as_uint(ra), vb = __float_as_uint(rb);
    m = (va >> 16) | (vb & 0xffff0000u);
    const uint32_t wa = __float_as_uint(ra - __uint_as_float(va & 0xffff0000u));
    const uint32_t wb = __float_as_uint(rb - __uint_as_float(vb & 0xffff0000u));
    l = (wa >> 16) | (wb & 0xffff0000u);
}

__device__ __forceinline__ float activate(int act, float x) {
    switch (act) {
        case TF_ACT_RELU: return x < 0.0f ? 0.0f : x;       // (a NaN stays one)
        case TF_ACT_SILU: return x / (1.0f + expf(-x));
        case TF_ACT_GELU: return 0.5f * x * (1.0f + erff(x * 0.70710678118654752f));
        default: return x;
    }
}

// Row of A that entry q belongs to.  Where all rows have the same number of entries, as a router leaves them, the first
// guess is right.
__device__ __forceinline__ int row_of_entry(const int32_t *__restrict__ rowptr, int n_rows, int nnz, int q) {
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

// EL: element type; KIND: 4-bit kind or -1; G: groups in 128 columns; HID: X are hidden rows; NT: blocks of sixteen
// entries that are multiplied at a time.
//
// A workgroup multiplies kExpertFrags blocks of sixteen rows of one expert's weights (with a gate: sixteen of the gate and
// the sixteen that it multiplies) with the rows of X of the entries that name the expert; its waves share the columns,
// a group of steps in turn, and their sums are added up through LDS, wave after wave.  Weights are the first operand of the
// matrix instructions, straight from memory: whatever the number of entries up to sixteen, what one instruction
// multiplies was loaded by one instruction.
template <int EL, int KIND, int G, bool HID, int NT>
__global__ __launch_bounds__(kExpertThreads) void k_experts(const ExpertLaunch a) {
    typedef typename El<EL>::T T;
    constexpr int NF = kExpertFrags;
    constexpr bool DENSE = KIND < 0, WIDE = EL == TF_F32;
    constexpr int STEP = DENSE ? (WIDE ? 16 : 32) : kQ4Block;     // columns of a step
    constexpr int SUB = DENSE ? 1 : 4;                            // operands of X in a step
    constexpr int XE = DENSE && WIDE ? 4 : 8;                     // columns of X that a lane holds of an operand
    constexpr int XR = !DENSE && WIDE ? 2 : HID && !WIDE ? 2 : 1; // sixteen-byte pieces of it
    constexpr int U = DENSE ? (NT > 1 ? 2 : 4) : (NT > 1 ? 1 : 2);
    constexpr int SETS = !DENSE && WIDE ? 2 : HID && EL == TF_F16 ? 2 : 1;   // sums of high and of low parts

    __shared__ int s_count[kExpertWaves], s_entry[16 * NT];
    extern __shared__ __align__(16) unsigned char smem[];
    Float4 *red = reinterpret_cast<Float4 *>(smem);

    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4, r = lane & 15;
    const int rows_per = a.gated ? 16 : 16 * NF;
    const int tiles = (a.n_rows + rows_per - 1) / rows_per;
    const int tile = blockIdx.x % tiles, unit = blockIdx.x / tiles;

    int expert = 0;
    const bool by_entry = a.rowptr && a.n_entries <= a.n_experts;
    if (a.rowptr) {
        expert = by_entry ? a.colidx[unit] : unit;
        if (expert < 0 || expert >= a.n_experts) return;
    }

    // weights
    const char *wp[NF];
    const char *sp[NF];
    const int blocks = (a.n_cols + kQ4Block - 1) / kQ4Block;
#pragma unroll
    for (int f = 0; f < NF; ++f) {
        // (a block beyond the matrix reads its last row again; what comes of it is not stored)
        const char *base = static_cast<const char *>(a.W) + expert * a.w_mat;
        if constexpr (DENSE) {
            int row = a.gated ? min(tile * 16 + r, a.n_rows - 1) + f * a.n_rows : min((tile * NF + f) * 16 + r, a.n_rows - 1);
            wp[f] = base + ((int64_t)row * a.n_cols + XE * g) * (int)sizeof(T);
            sp[f] = nullptr;
        } else {
            // with a gate n_rows is a multiple of sixteen or the second half begins inside a block: rows are looked up one by one
            int row = a.gated ? min(tile * 16 + r, a.n_rows - 1) + f * a.n_rows : min((tile * NF + f) * 16 + r, a.n_rows - 1);
            wp[f] = base + (int64_t)(row >> 4) * blocks * 1024 + (16 * g + (row & 15)) * 16;
            sp[f] = static_cast<const char *>(a.scales) + expert * a.s_mat;
        }
    }
    (void)sp;

    for (int first = 0;; first += 16 * NT) {
        // the entries first .. first + 16 NT - 1 of those that name the expert
        int total = a.n_entries;
        if (a.rowptr) {
            total = 0;
            for (int i0 = 0; i0 < a.n_entries; i0 += kExpertThreads) {
                const int i = i0 + (int)threadIdx.x;
                const bool hit = i < a.n_entries && a.colidx[i] == expert;
                const uint64_t m = __builtin_amdgcn_ballot_w64(hit);
                if (lane == 0) s_count[wave] = __popcll(m);
                __syncthreads();
                int before = total;
#pragma unroll
                for (int w = 0; w < kExpertWaves; ++w) {
                    if (w < wave) before += s_count[w];
                    total += s_count[w];
                }
                const int rank = before + __popcll(m & ((1ull << lane) - 1)) - first;
                if (hit && rank >= 0 && rank < 16 * NT) s_entry[rank] = i;
                __syncthreads();
            }
        }
        if (total <= first) return;
        // (by entry: the first that names the expert does the work of all)
        if (by_entry && first == 0 && s_entry[0] != unit) return;
        const int count = min(total - first, 16 * NT);

        const char *xp[NT];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            // (beyond the last entry: the first one again; what comes of it is not stored)
            const int at = 16 * n + r < count ? 16 * n + r : 0;
            int row = a.rowptr ? s_entry[at] : first + at;
            if (a.rowptr && !HID) row = row_of_entry(a.rowptr, a.n_tokens, a.n_entries, row);
            xp[n] = static_cast<const char *>(a.X) + (row * a.ldx + XE * g) * (int64_t)sizeof(T);
        }

        Float4 sum[NF][NT], acc[SETS][NF][NT];
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                sum[f][n] = Float4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < SETS; ++s) acc[s][f][n] = Float4{0, 0, 0, 0};
            }

        struct Step {
            Words4 w[NF];
            float scale[DENSE ? 1 : NF][DENSE ? 1 : G][DENSE ? 1 : 4];
            Words4 x[SUB][NT][XR];
        };
        auto load = [&](Step &s, int step, bool whole) __attribute__((always_inline)) {
            const int k0 = step * STEP;
#pragma unroll
            for (int f = 0; f < NF; ++f) {
                if constexpr (DENSE) {
                    const char *p = wp[f] + (int64_t)k0 * (int)sizeof(T);
                    if (whole) {
                        s.w[f] = __builtin_nontemporal_load(reinterpret_cast<const AnyWords4 *>(p));
                    } else {
                        T e[XE];
#pragma unroll
                        for (int i = 0; i < XE; ++i) e[i] = k0 + XE * g + i < a.n_cols ? reinterpret_cast<const T *>(p)[i] : T(0);
                        s.w[f] = __builtin_bit_cast(Words4, e);
                    }
                } else {
                    s.w[f] = __builtin_nontemporal_load(reinterpret_cast<const Words4 *>(wp[f] + (int64_t)step * 1024));
#pragma unroll
                    for (int q = 0; q < G; ++q)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int out = a.gated ? min(tile * 16 + 4 * g + v, a.n_rows - 1) + f * a.n_rows
                                                    : min((tile * NF + f) * 16 + 4 * g + v, a.n_rows - 1);
                            const int64_t at = ((int64_t)(out >> 4) * blocks + step) * (16 * G) + ((out & 15) >> 2) * (4 * G) + 4 * q + (out & 3);
                            s.scale[f][q][v] = El<TF_BF16>::get(reinterpret_cast<const uint16_t *>(sp[f])[at]);
                        }
                }
            }
#pragma unroll
            for (int j = 0; j < SUB; ++j)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < XR; ++h) {
                        constexpr int per = 16 / (int)sizeof(T);        // elements of a piece
                        const int k = k0 + 32 * j + (WIDE && h ? 4 : 0);
                        const char *p = xp[n] + (int64_t)k * (int)sizeof(T) + (HID && !WIDE && h ? a.x_part : 0);
                        if (whole) {
                            s.x[j][n][h] = *reinterpret_cast<const AnyWords4 *>(p);
                        } else {
                            T e[per];
#pragma unroll
                            for (int i = 0; i < per; ++i) e[i] = k + XE * g + i < a.n_cols ? reinterpret_cast<const T *>(p)[i] : T(0);
                            s.x[j][n][h] = __builtin_bit_cast(Words4, e);
                        }
                    }
        };
        auto multiply = [&](const Step &s) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < SUB; ++j) {
                Words4 w[NF];
#pragma unroll
                for (int f = 0; f < NF; ++f)
                    if constexpr (DENSE) w[f] = s.w[f];
                    else w[f] = q4_decode<EL, KIND>(s.w[f][j]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if constexpr (DENSE && WIDE) {
                        const Float4 x = __builtin_bit_cast(Float4, s.x[j][n][0]);
#pragma unroll
                        for (int f = 0; f < NF; ++f) {
                            const Float4 y = __builtin_bit_cast(Float4, w[f]);
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[0][f][n] = mfma_f32(y[i], x[i], acc[0][f][n]);
                        }
                    } else if constexpr (WIDE) {
                        Words4 part[3];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t h, m, l;
                            cut_pair(h, m, l, __uint_as_float(s.x[j][n][i / 2][2 * (i & 1)]), __uint_as_float(s.x[j][n][i / 2][2 * (i & 1) + 1]));
                            part[0][i] = h;
                            part[1][i] = m;
                            part[2][i] = l;
                        }
#pragma unroll
                        for (int f = 0; f < NF; ++f) {
                            acc[0][f][n] = mfma_bf16(w[f], part[0], acc[0][f][n]);
                            acc[1][f][n] = mfma_bf16(w[f], part[1], acc[1][f][n]);
                            acc[1][f][n] = mfma_bf16(w[f], part[2], acc[1][f][n]);
                        }
                    } else {
#pragma unroll
                        for (int f = 0; f < NF; ++f)
#pragma unroll
                            for (int h = 0; h < XR; ++h) {
                                Float4 &c = acc[SETS > 1 ? h : 0][f][n];
                                c = EL == TF_F16 ? mfma_f16(w[f], s.x[j][n][h], c) : mfma_bf16(w[f], s.x[j][n][h], c);
                            }
                    }
                }
                if constexpr (!DENSE) {
                    if ((j + 1) % (4 / G) == 0) {
#pragma unroll
                        for (int f = 0; f < NF; ++f)
#pragma unroll
                            for (int n = 0; n < NT; ++n)
#pragma unroll
                                for (int v = 0; v < 4; ++v) {
                                    float c = acc[0][f][n][v];
                                    acc[0][f][n][v] = 0.0f;
                                    if constexpr (SETS > 1) {
                                        c = EL == TF_F16 ? fmaf(c, kHalfHigh, acc[1][f][n][v]) : c + acc[1][f][n][v];
                                        acc[1][f][n][v] = 0.0f;
                                    }
                                    sum[f][n][v] = fmaf(s.scale[f][j / (4 / G)][v], c, sum[f][n][v]);
                                }
                    }
                }
            }
        };

        const int whole_steps = a.n_cols / STEP, steps = (a.n_cols + STEP - 1) / STEP;
        for (int s0 = wave * U; s0 < steps; s0 += kExpertWaves * U) {
            if (s0 + U <= whole_steps) {
                Step s[U];
#pragma unroll
                for (int u = 0; u < U; ++u) load(s[u], s0 + u, true);
#pragma unroll
                for (int u = 0; u < U; ++u) multiply(s[u]);
            } else {
                for (int u = s0; u < min(s0 + U, steps); ++u) {
                    Step s;
                    load(s, u, false);
                    multiply(s);
                }
            }
        }
        if constexpr (DENSE) {
#pragma unroll
            for (int f = 0; f < NF; ++f)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int v = 0; v < 4; ++v)
                        sum[f][n][v] = SETS > 1 ? fmaf(acc[0][f][n][v], kHalfHigh, acc[SETS - 1][f][n][v]) : acc[0][f][n][v];
        }

        // sums of the waves, in their order
#pragma unroll
        for (int f = 0; f < NF; ++f)
#pragma unroll
            for (int n = 0; n < NT; ++n) red[((wave * NF + f) * NT + n) * 64 + lane] = sum[f][n];
        __syncthreads();
        const int items = (a.gated ? 1 : NF) * NT * 64;
        for (int item = threadIdx.x; item < items; item += kExpertThreads) {
            Float4 y = red[item];
            for (int w = 1; w < kExpertWaves; ++w) y += red[w * (NF * NT * 64) + item];
            Float4 up = Float4{1, 1, 1, 1};
            if (a.gated) {
                up = red[NT * 64 + item];
                for (int w = 1; w < kExpertWaves; ++w) up += red[(w * NF + 1) * (NT * 64) + item];
            }
            const int f = item / (NT * 64), n = item / 64 % NT, il = item & 63;
            const int slot = 16 * n + (il & 15);
            const int row0 = (a.gated ? tile : tile * NF + f) * 16 + 4 * (il >> 4);
            if (slot < count) {
                const int entry = a.rowptr ? s_entry[slot] : first + slot;
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    if (row0 + v >= a.n_rows) continue;
                    const int64_t at = (int64_t)entry * a.ldo + row0 + v;
                    if (a.out_kind == kOutSums) {
                        static_cast<float *>(a.out)[at] = y[v];
                    } else if (a.out_kind == kOutRows) {
                        static_cast<T *>(a.out)[at] = El<EL>::put(y[v]);
                    } else {
                        const float h = activate(a.activation, y[v]) * up[v];
                        T *hi = static_cast<T *>(a.out);
                        T *lo = reinterpret_cast<T *>(static_cast<char *>(a.out) + a.out_part);
                        if constexpr (EL == TF_F32) {
                            hi[at] = h;
                        } else if constexpr (EL == TF_BF16) {
                            const uint16_t top = El<EL>::put(h);
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
            }
        }
        if (first + 16 * NT >= total) return;
        __syncthreads();
    }
}

template <int EL, int KIND, int G, bool HID, int NT> int launch_experts_nt(const ExpertLaunch &a, hipStream_t st) {
    const int rows_per = a.gated ? 16 : 16 * kExpertFrags;
    const int64_t tiles = (a.n_rows + rows_per - 1) / rows_per;
    const int64_t units = !a.rowptr ? 1 : a.n_entries <= a.n_experts ? a.n_entries : a.n_experts;
    const size_t lds = (size_t)kExpertWaves * kExpertFrags * NT * 64 * sizeof(Float4);
    if (lds >= (64 << 10) - 1024) {          // (more than a launch may ask for by default, with the static LDS)
        static const int raised = (int)hipFuncSetAttribute(reinterpret_cast<const void *>(&k_experts<EL, KIND, G, HID, NT>),
                                                           hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
        if (raised) return raised;
    }
    hipLaunchKernelGGL((k_experts<EL, KIND, G, HID, NT>), dim3((unsigned)(tiles * units)), dim3(kExpertThreads), lds, st, a);
    return (int)hipGetLastError();
}
template <int EL, int KIND, int G, bool HID> int launch_experts_hid(const ExpertLaunch &a, hipStream_t st) {
    const int most = a.rowptr ? a.n_tokens : a.n_entries;      // entries of an expert, one a token
    return most <= 16 ? launch_experts_nt<EL, KIND, G, HID, 1>(a, st) : launch_experts_nt<EL, KIND, G, HID, 4>(a, st);
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
