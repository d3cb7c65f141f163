// Cross entropy of a product: the rows that count, operands, merging of sums, and the launches of a call.
#include <algorithm>
#include <type_traits>

#include "tf_loss_device.h"
#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr float kLow = -__builtin_inff();

// -------------------------------------------------------------------------------------- operands

// Eight columns of a row, from column k on, in 32 bits; zeros behind the last one.
template <int EL> __device__ __forceinline__ void read8(float (&x)[8], const void *row, int64_t k, int64_t n) {
    typedef typename El<EL>::T T;
    const T *p = static_cast<const T *>(row) + k;
    if (k + 8 <= n) {
        if constexpr (EL == TF_F32) {
            const AnyWords4 lo = *reinterpret_cast<const AnyWords4 *>(p), hi = *reinterpret_cast<const AnyWords4 *>(p + 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[i] = __uint_as_float(lo[i]);
                x[4 + i] = __uint_as_float(hi[i]);
            }
        } else {
            const AnyWords4 w = *reinterpret_cast<const AnyWords4 *>(p);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = El<EL>::get((uint16_t)(w[i / 2] >> (16 * (i & 1))));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = k + i < n ? El<EL>::get(p[i]) : 0.0f;
    }
}
template <int EL> __device__ __forceinline__ void write8(const float (&x)[8], void *row, int64_t k, int64_t n) {
    typedef typename El<EL>::T T;
    T *p = static_cast<T *>(row) + k;
    if (k + 8 <= n) {
        AnyWords4 lo, hi;
        if constexpr (EL == TF_F32) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lo[i] = __float_as_uint(x[i]);
                hi[i] = __float_as_uint(x[4 + i]);
            }
            *reinterpret_cast<AnyWords4 *>(p + 4) = hi;
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) lo[i] = El<EL>::put(x[2 * i]) | (uint32_t)El<EL>::put(x[2 * i + 1]) << 16;
        }
        *reinterpret_cast<AnyWords4 *>(p) = lo;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < n) p[i] = El<EL>::put(x[i]);
    }
}

// The first part of a finite number is finite: beside the largest ones rounding would give infinity, and NaN in the parts behind it.
__device__ __forceinline__ uint16_t first_part(float x) {
    constexpr float MOST = 0x1.fep127f;        // of bf16
    const float size = fabsf(x);
    return El<TF_BF16>::put(size > MOST && size < __builtin_inff() ? copysignf(MOST, x) : x);
}

// Eight columns as an operand of the products: 16-bit numbers as they are, fp32 ones as three bf16 numbers that add up to them.
template <int EL> __device__ __forceinline__ void put8(const float (&x)[8], void *to_row, int64_t k, int64_t plane) {
    uint16_t *to = static_cast<uint16_t *>(to_row) + k;
    Words4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (EL == TF_F32) {
            float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const uint16_t ha = p ? El<TF_BF16>::put(a) : first_part(a), hb = p ? El<TF_BF16>::put(b) : first_part(b);
                w[p][i] = ha | (uint32_t)hb << 16;
                a -= El<TF_BF16>::get(ha);
                b -= El<TF_BF16>::get(hb);
            }
        } else {
            w[0][i] = El<EL>::put(x[2 * i]) | (uint32_t)El<EL>::put(x[2 * i + 1]) << 16;
        }
    }
#pragma unroll
    for (int p = 0; p < (EL == TF_F32 ? 3 : 1); ++p) *reinterpret_cast<Words4 *>(to + p * plane) = w[p];
}

// How many threads take a row of `columns`, eight columns each: a power of two, 256 at most.
__device__ __forceinline__ int threads_of_row(int64_t columns) {
    const int n = (int)min(ceil_div(columns, 8), (int64_t)256);
    return n <= 1 ? 1 : 1 << (32 - __builtin_clz((unsigned)n - 1));
}

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}

// dloss of the rows that have a label: the largest finite size, and (fp16) the smallest and the largest number, +-infinity where one is not finite.
template <bool BOTH> struct Gradients {
    float top, low, high;
    static __device__ __forceinline__ Gradients none() { return Gradients{0.0f, __builtin_inff(), kLow}; }
    __device__ __forceinline__ void add(float g) {
        const float size = fabsf(g);
        const bool finite = size < __builtin_inff();
        if (finite) top = fmaxf(top, size);
        if constexpr (BOTH) {
            low = fminf(low, finite ? g : kLow);
            high = fmaxf(high, finite ? g : __builtin_inff());
        }
    }
    __device__ __forceinline__ void add(Gradients x) {
        top = fmaxf(top, x.top);
        if constexpr (BOTH) {
            low = fminf(low, x.low);
            high = fmaxf(high, x.high);
        }
    }
    __device__ __forceinline__ void over_wave() {
        top = wave_max(top);
        if constexpr (BOTH) {
            low = -wave_max(-low);
            high = wave_max(high);
        }
    }
};
// Whether a row has a label.
__device__ __forceinline__ bool counts(const XentLaunch &a, int64_t row) {
    const int y = a.labels[row];
    return y >= 0 && y < a.n_classes;
}
// The same, and what it adds to the gradients.
template <bool BOTH> __device__ __forceinline__ bool counts(const XentLaunch &a, int64_t row, Gradients<BOTH> &g) {
    const bool keep = counts(a, row);
    if (keep && a.dloss) g.add(a.dloss[row]);
    return keep;
}

// Count and largest gradient of a block of rows a workgroup.
template <bool BOTH> __global__ __launch_bounds__(256) void k_count_rows(const XentLaunch a, const int block) {
    __shared__ int n_of[4];
    __shared__ Gradients<BOTH> g_of[4];
    const int tid = threadIdx.x;
    const int64_t first = (int64_t)blockIdx.x * block, end = min(first + block, (int64_t)a.n_rows);
    int n = 0;
    Gradients<BOTH> g = Gradients<BOTH>::none();
    for (int64_t r = first + tid; r < end; r += 256) n += counts(a, r, g);
    n = wave_sum(n);
    g.over_wave();
    if ((tid & 63) == 0) {
        n_of[tid >> 6] = n;
        g_of[tid >> 6] = g;
    }
    __syncthreads();
    if (tid == 0) {
        for (int w = 1; w < 4; ++w) g.add(g_of[w]);
        a.s.block_rows[blockIdx.x] = n_of[0] + n_of[1] + n_of[2] + n_of[3];
        a.s.block_top[blockIdx.x] = g.top;
        if constexpr (BOTH) {
            a.s.block_low[blockIdx.x] = g.low;
            a.s.block_high[blockIdx.x] = g.high;
        }
    }
}

// w: rows first .. first + count of W, columns as above; `group` of `groups` workgroups.
template <int EL> __device__ __forceinline__ void pack_classes(const XentLaunch &a, int64_t first, int64_t count, int64_t group, int64_t groups) {
    const int64_t columns = round_up(a.n_in, 64);
    const int per_row = threads_of_row(columns), at_once = 256 / per_row;
    for (int64_t i = group * at_once + threadIdx.x / per_row; i < count; i += groups * at_once)
        for (int64_t k = threadIdx.x % per_row * 8; k < columns; k += per_row * 8) {
            float x[8];
            read8<EL>(x, static_cast<const typename El<EL>::T *>(a.W) + (first + i) * a.ldw, k, a.n_in);
            put8<EL>(x, static_cast<uint16_t *>(a.s.w) + i * a.s.ld, k, a.s.w_cap);
        }
}
template <int EL> __global__ __launch_bounds__(256) void k_pack_classes(const XentLaunch a, const int64_t first, const int64_t count) {
    pack_classes<EL>(a, first, count, blockIdx.x, gridDim.x);
}

// Numbers the rows that have a label in their order and copies them, one after the other, to x, where columns up to a multiple of 64 are zeros behind
// the last one; rows without a label get their zeros.  A block of rows a workgroup, which sums up the counts of the blocks before
// it; where there are few rows (`counted` 0) it counts them itself, which saves a launch.  Workgroups behind the `blocks` first ones pack W's first rows.
// 8192 rows of 4096 bf16 numbers 38 us, 3.5 TB/s; one row 4.7 us, a chain of three loads.
template <int EL> __global__ __launch_bounds__(256) void k_pack_rows(const XentLaunch a, const int block, const int blocks, const int counted, const int64_t classes) {
    typedef Gradients<EL == TF_F16> Of;
    __shared__ int n_of[4], rows[256], ats[256];
    __shared__ Of g_of[4];
    if ((int)blockIdx.x >= blocks) return pack_classes<EL>(a, 0, classes, blockIdx.x - blocks, gridDim.x - blocks);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t first = (int64_t)blockIdx.x * block, end = min(first + block, (int64_t)a.n_rows);
    int n = 0;
    Of g = Of::none();
    if (counted) {
        for (int b = tid; b < blocks; b += 256) {
            if (b < (int)blockIdx.x) n += a.s.block_rows[b];
            if (a.dloss) g.add(EL == TF_F16 ? Of{a.s.block_top[b], a.s.block_low[b], a.s.block_high[b]} : Of{a.s.block_top[b], 0.0f, 0.0f});
        }
    } else {
        for (int64_t r = tid; r < (a.dloss ? (int64_t)a.n_rows : first); r += 256) {
            const bool keep = counts(a, r, g);
            n += keep && r < first;
        }
    }
    n = wave_sum(n);
    if (a.dloss) g.over_wave();
    if (lane == 0) {
        n_of[wave] = n;
        g_of[wave] = g;
    }
    __syncthreads();
    n = n_of[0] + n_of[1] + n_of[2] + n_of[3];
    for (int w = 0; w < 4; ++w) g.add(g_of[w]);
    float top = g.top;
    // fp16: gradients are divided by the largest one, so that what dW, their sum, can hold is not lost in 16 bits.  The other types' range is that of the
    // results: only gradients that are all very small, or one as large as the type, are divided (others would pass the range that their sums stay in).
    const float scale = a.dtype == TF_F16 ? 32768.0f : 1.0f;
    if (top == 0.0f || (a.dtype != TF_F16 && top > 0x1p-64f && top < 0x1p126f)) top = 1.0f;
    if (!a.loss && blockIdx.x == 0 && tid == 0) {        // (without rows there is no dloss)
        const bool same = EL == TF_F16 && g.low == g.high;
        if (EL == TF_F16) *a.s.same = same;
        *a.s.unit = (same ? g.high : top) / scale;
    }
    const int64_t columns = round_up(a.n_in, 64);
    const int per_row = threads_of_row(columns), at_once = 256 / per_row;
    for (int64_t r0 = first; r0 < end; r0 += 256) {
        const int64_t r = r0 + tid;
        const bool keep = r < end && counts(a, r);
        const uint64_t kept = __ballot(keep);
        __syncthreads();        // (the last round's lists have been read)
        if (lane == 0) n_of[wave] = __popcll(kept);
        __syncthreads();
        int at = __popcll(kept & (((uint64_t)1 << lane) - 1)), here = 0;
        for (int w = 0; w < 4; ++w) {
            if (w < wave) at += n_of[w];
            here += n_of[w];
        }
        if (r < end) {
            a.s.pos[r] = keep ? n + at : -1;
            if (keep) {
                rows[at] = (int)r;
                a.s.list[n + at] = (int)r;
                a.s.label[n + at] = a.labels[r];
                if (a.dloss) {
                    a.s.lse[n + at] = a.lse_in[r];
                    a.s.g[n + at] = a.dloss[r] / top * scale;
                    if (EL == TF_F16) a.s.dloss[n + at] = a.dloss[r];
                    if (a.loss_in) a.s.hit[n + at] = -a.loss_in[r];
                }
            } else if (a.loss) {
                a.loss[r] = a.lse[r] = 0.0f;
            }
            ats[tid] = keep;
        }
        __syncthreads();
        for (int i = tid / per_row; i < here; i += at_once)
            for (int64_t k = tid % per_row * 8; k < columns; k += per_row * 8) {
                float x[8];
                read8<EL>(x, static_cast<const typename El<EL>::T *>(a.X) + rows[i] * a.ldx, k, a.n_in);
                if (EL == TF_F32 && a.native) write8<TF_F32>(x, static_cast<float *>(a.s.x) + (n + i) * a.s.ld, k, columns);
                else put8<EL>(x, static_cast<uint16_t *>(a.s.x) + (n + i) * a.s.ld, k, a.s.x_plane);
            }
        if (a.dX && a.direct_dx)
            for (int i = tid / per_row; i < (int)min(end - r0, (int64_t)256); i += at_once)
                if (!ats[i])
                    for (int64_t k = tid % per_row * 8; k < a.n_in; k += per_row * 8) {
                        const float x[8] = {};
                        write8<EL>(x, static_cast<typename El<EL>::T *>(a.dX) + (r0 + i) * a.lddx, k, a.n_in);
                    }
        n += here;
    }
    if ((int)blockIdx.x == blocks - 1 && tid == 0) *a.s.n = n;
    if (blockIdx.x == 0)
        for (int i = tid; i < kMostJoins; i += 256) a.s.arrived[i * kJoinApart] = 0;
}
// ------------------------------------------------------------------------------------------- ends

// Adds the sums of `blocks` blocks of classes to those of the classes before them (unless `first`).  ROWS rows a workgroup: 64 / ROWS lanes of each of
// its 16 waves take a row, and all of them every block once.  The last call writes the results.  Bound by reading: 8192 rows with 2048 sums each 26 us, 5.1 TB/s; one
// row with 1024 sums 6 us, latency.
template <int ROWS> __global__ __launch_bounds__(1024) void k_merge(const XentLaunch a, const int64_t blocks, const int64_t ld, const int first, const int last) {
    __shared__ Float2 of_wave[16][ROWS];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * ROWS + lane % ROWS;
    const int n = *a.s.n;
    if ((int64_t)blockIdx.x * ROWS >= n) return;
    Float2 x{kLow, 0.0f};
    if (row < n)
#pragma unroll 4
        for (int64_t b = wave * (64 / ROWS) + lane / ROWS; b < blocks; b += 16 * (64 / ROWS)) x = add_sums(x, a.s.part[b * ld + row]);
#pragma unroll
    for (int d = ROWS; d < 64; d <<= 1) x = add_sums(x, Float2{__shfl_xor(x[0], d, 64), __shfl_xor(x[1], d, 64)});
    if (lane < ROWS) of_wave[wave][lane] = x;
    __syncthreads();
    if (wave) return;
    x = !first && row < n && lane < ROWS ? Float2{a.s.top[row], a.s.sum[row]} : Float2{kLow, 0.0f};
    for (int w = lane / ROWS; w < 16; w += 64 / ROWS) x = add_sums(x, of_wave[w][lane % ROWS]);
#pragma unroll
    for (int d = ROWS; d < 64; d <<= 1) x = add_sums(x, Float2{__shfl_xor(x[0], d, 64), __shfl_xor(x[1], d, 64)});
    if (row >= n || lane >= ROWS) return;
    if (!last) {
        a.s.top[row] = x[0];
        a.s.sum[row] = x[1];
        return;
    }
    const int64_t to = a.s.list[row];
    write_loss(x, a.s.hit[row], a.loss + to, a.lse + to);
}

// Rows `row` of an output from the sums of `splits` slabs, `none` for zeros.  A row's columns lie in `per_row` threads; the others of a workgroup take
// other rows, or, where there are many slabs, other slabs (`by_slab`), added up in their order.  Bound by reading: one slab of 8192 x 4096 to bf16 39 us, 5.1 TB/s.
template <int EL> __device__ __forceinline__ void finish_row(const float *slab, int64_t size, int splits, void *out, int64_t n_in, bool none, float unit,
                                                             int per_row, bool by_slab, bool is) {
    __shared__ float part[256][9];
    const int tid = threadIdx.x, slices = by_slab ? 256 / per_row : 1, slice = by_slab ? tid / per_row : 0;
    for (int64_t k0 = (int64_t)blockIdx.y * per_row * 8; k0 < n_in; k0 += (int64_t)gridDim.y * per_row * 8) {
        const int64_t k = k0 + tid % per_row * 8;
        float x[8] = {};
        if (is && !none && k < n_in)
            for (int z0 = slice; z0 < splits; z0 += 4 * slices) {
                Float4 lo[4], hi[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int z = min(z0 + i * slices, splits - 1);
                    const Float4 *p = reinterpret_cast<const Float4 *>(slab + z * size + k);
                    lo[i] = p[0];
                    hi[i] = p[1];
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (z0 + i * slices < splits)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            x[j] += lo[i][j];
                            x[4 + j] += hi[i][j];
                        }
            }
        if (by_slab) {
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) part[tid][j] = x[j];
            __syncthreads();
            if (slice == 0)
                for (int s = 1; s < slices; ++s)
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] += part[s * per_row + tid][j];
        }
        if (is && slice == 0 && k < n_in) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= unit;
            write8<EL>(x, out, k, n_in);
        }
    }
}
constexpr int kManySlabs = 8;
// Columns of a step of the products.
__host__ __device__ constexpr int step_of(const XentLaunch &a) { return a.native ? 32 : 64; }
// Parts of a number.
__host__ __device__ constexpr int parts_of(const XentLaunch &a) { return a.dtype == TF_F32 && !a.native ? 3 : 1; }

// dX: the shares' sums of each row that counts, zeros in the others.
template <int EL> __global__ __launch_bounds__(256) void k_finish_rows(const XentLaunch a, const int splits, const int64_t size) {      // (the same for every piece)
    const float all = *a.s.unit;
    const bool by_slab = splits >= kManySlabs;
    const int per_row = min(threads_of_row(a.n_in), by_slab ? 32 : 256);
    const int at_once = by_slab ? 1 : 256 / per_row;
    for (int64_t t0 = (int64_t)blockIdx.x * at_once; t0 < a.n_rows; t0 += (int64_t)gridDim.x * at_once) {
        const int64_t t = t0 + (by_slab ? 0 : threadIdx.x / per_row);
        const bool is = t < a.n_rows;
        const int64_t i = is ? a.s.pos[t] : -1;
        const float unit = EL == TF_F16 && i >= 0 ? a.s.dloss[i] * kRowUnit : all;
        finish_row<EL>(a.s.dx + i * a.s.slab_ld, size, splits, static_cast<typename El<EL>::T *>(a.dX) + t * a.lddx, a.n_in, i < 0, unit, per_row, by_slab, is);
    }
}
// Rows first .. first + count of dW.
template <int EL> __global__ __launch_bounds__(256) void k_finish_classes(const XentLaunch a, const int64_t first, const int64_t count, const int most, const int64_t size) {
    const int splits = shares_of(most, (int)ceil_div(*a.s.n, step_of(a)), parts_of(a));
    const float unit = *a.s.unit;
    const bool by_slab = splits >= kManySlabs;
    const int per_row = min(threads_of_row(a.n_in), by_slab ? 32 : 256);
    const int at_once = by_slab ? 1 : 256 / per_row;
    for (int64_t i0 = (int64_t)blockIdx.x * at_once; i0 < count; i0 += (int64_t)gridDim.x * at_once) {
        const int64_t i = i0 + (by_slab ? 0 : threadIdx.x / per_row);
        finish_row<EL>(a.s.dw + i * a.s.slab_ld, size, splits, static_cast<typename El<EL>::T *>(a.dW) + (first + i) * a.lddw, a.n_in, false, unit, per_row, by_slab,
                       i < count);
    }
}

// dW of few rows, 32 KH at most: dW = G^T X has as little as one step of K then, and is bound by writing it.  A wave holds its 64 columns of X as
// operands and goes over classes, 64 at a time, the next ones' G on its way.  Which rows of an operand are which columns and classes is free: with
// those below a lane reads four classes of G at once and writes eight columns of dW.  4096 -> 65536 classes, bf16, one row 96 us, 5.6 TB/s; 64 rows of
// 4096 -> 20000 51 us, 3.2 TB/s (registers for three waves a SIMD).
template <int EL, int KH> __global__ __launch_bounds__(256, KH > 1 ? 3 : 4) void k_few_rows(const XentLaunch a, const int64_t first, const int64_t count, const int64_t g_ld,
                                                                                            const int64_t each) {
    typedef typename El<EL>::T T;
    typedef std::conditional_t<EL == TF_BF16, Bf8, Half8> V;
    typedef uint16_t U4 __attribute__((ext_vector_type(4)));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane % 16, g = lane / 16, kept = *a.s.n;
    const int64_t c0 = (int64_t)blockIdx.x * 256 + wave * 64, v_end = min(count, ((int64_t)blockIdx.y + 1) * each);
    if (c0 >= a.n_in) return;
    const float unit = *a.s.unit;
    const uint16_t *G = static_cast<const uint16_t *>(a.s.G) + (EL == TF_F16 && !*a.s.same ? a.s.g_cap : 0);
    V x[4][KH];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t c = c0 + 32 * (i / 2) + 8 * (r / 4) + 4 * (i % 2) + r % 4;
#pragma unroll
        for (int h = 0; h < KH; ++h) {
            Words4 w;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t t = 32 * h + 8 * g + k;
                const uint32_t e = t < kept && c < a.n_in ? (uint32_t)static_cast<const uint16_t *>(a.s.x)[t * a.s.ld + c] : 0u;
                w[k / 2] = k & 1 ? w[k / 2] | e << 16 : e;
            }
            x[i][h] = __builtin_bit_cast(V, w);
        }
    }
    U4 next[KH][8];
    auto load = [&](int64_t v) {
#pragma unroll
        for (int h = 0; h < KH; ++h)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int64_t t = 32 * h + 8 * g + k;
                next[h][k] = U4{0, 0, 0, 0};
                if (t < kept) next[h][k] = *reinterpret_cast<const U4 *>(G + t * g_ld + v + 4 * r);
            }
    };
    int64_t v0 = blockIdx.y * each;
    if (v0 < v_end) load(v0);
    for (; v0 < v_end; v0 += 64) {
        V y[4][KH];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int h = 0; h < KH; ++h) {
                Words4 w;
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = next[h][2 * k][j] | (uint32_t)next[h][2 * k + 1][j] << 16;
                y[j][h] = __builtin_bit_cast(V, w);
            }
        if (v0 + 64 < v_end) load(v0 + 64);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int64_t v = v0 + 4 * r + j;
            T *row = static_cast<T *>(a.dW) + (first + v) * a.lddw + c0;
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                float d[8];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    Float4 sum = {};
#pragma unroll
                    for (int h = 0; h < KH; ++h) {
                        if constexpr (EL == TF_BF16) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x[2 * p + i][h], y[j][h], sum, 0, 0, 0);
                        else sum = __builtin_amdgcn_mfma_f32_16x16x32_f16(x[2 * p + i][h], y[j][h], sum, 0, 0, 0);
                    }
#pragma unroll
                    for (int k = 0; k < 4; ++k) d[4 * i + k] = sum[k] * unit;
                }
                if (v < v_end) write8<EL>(d, row, 32 * p + 8 * g, a.n_in - c0);
            }
        }
    }
}

// --------------------------------------------------------------------------------------- launches

// Workgroups for `rows` rows of `columns`, 2048 columns at a time.
dim3 row_grid(int64_t rows, int64_t columns) {
    const int64_t per_row = std::min<int64_t>(256, ceil_div(columns, 8));
    return dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows * per_row, 256), 8192)));
}
// The same for rows that are summed from slabs; of many slabs 256 columns a workgroup.
dim3 slab_grid(int64_t rows, int64_t columns, int64_t splits) {
    return splits >= kManySlabs ? dim3((unsigned)std::min<int64_t>(rows, 8192), (unsigned)std::min<int64_t>(ceil_div(columns, 256), 64)) : row_grid(rows, columns);
}
#define TF_BY_TYPE(dtype, kernel, grid, ...)                                                                           \
    do {                                                                                                               \
        if (dtype == TF_BF16) hipLaunchKernelGGL((kernel<TF_BF16>), grid, dim3(256), 0, st, __VA_ARGS__);              \
        else if (dtype == TF_F16) hipLaunchKernelGGL((kernel<TF_F16>), grid, dim3(256), 0, st, __VA_ARGS__);           \
        else hipLaunchKernelGGL((kernel<TF_F32>), grid, dim3(256), 0, st, __VA_ARGS__);                                \
    } while (0)

int launch_product(const ProductLaunch &p, const XentLaunch &a, void *stream) {
    return a.dtype == TF_F16 ? launch_product_f16(p, stream) : a.native ? launch_product_f32(p, stream) : launch_product_bf16(p, stream);
}

// Few fp32 rows are multiplied by the fp32 instructions, W where it lies: as parts its numbers would be written and read again several times.  How many are
// few depends on the sizes; up to kNativeRows the instructions are ahead at all that were tried but 192 rows of 47 classes.  fp32 instructions / parts, us,
// loss of 448, 600, 1024 rows: 4096 -> 100000 2675 / 3563, 3729 / 3862, 5862 / 6232; 2048 -> 20000 326 / 394, 451 / 362, 600 / 554; 1000 -> 5000
// 60 / 73, 78 / 76, 111 / 89.  Gradients of 192, 256, 448 rows: 3709 / 4749, 4784 / 5831, 8391 / 8286; 404 / 482, 534 / 517, 913 / 870; 86 / 89, 108 / 97, 163 / 150.
bool is_native(const XentLaunch &a) { return a.dtype == TF_F32 && a.n_rows <= kNativeRows[a.loss ? 0 : 1]; }

// Whether W's rows are whole 16-byte pieces, as the products load them.
bool whole_pieces(const XentLaunch &a) {
    const int64_t piece = a.dtype == TF_F32 ? 4 : 8;
    return a.n_in % piece == 0 && (a.ldw % piece == 0 || a.n_classes == 1) && reinterpret_cast<uintptr_t>(a.W) % 16 == 0 && a.ldw <= kXentMaxColumns;
}
// Otherwise they go through registers while there are few rows, and are copied first where the products take long enough to pay for that.
// 1023 -> 40000 classes, bf16, through registers / copied, us: loss of 64 rows 37 / 60, 300 64 / 78, 1024 135 / 133; gradients of 64 126 / 140, 300 226 / 201.
// fp32 numbers that are multiplied in parts are always packed.
bool through_registers(const XentLaunch &a) { return !whole_pieces(a) && (a.dtype == TF_F32 ? a.native : a.n_rows <= kRegisterRows[a.loss ? 0 : 1]); }
bool in_place(const XentLaunch &a) { return a.dtype == TF_F32 ? a.native : whole_pieces(a) || through_registers(a); }

// Numbers and copies the rows that count.  (Also without rows: it sets the unit.)  Up to 8192 rows every block counts the rows before it.  Packs the
// first `classes` of W as well, where it has to be.
int begin(const XentLaunch &a, int64_t classes, hipStream_t st) {
    const int counted = a.n_rows > 8192;
    const int64_t block = std::max<int64_t>(1, ceil_div(a.n_rows, kMostBlocks)), blocks = std::max<int64_t>(1, ceil_div(a.n_rows, block));
    if (counted && a.dtype == TF_F16) hipLaunchKernelGGL(k_count_rows<true>, dim3((unsigned)blocks), dim3(256), 0, st, a, (int)block);
    else if (counted) hipLaunchKernelGGL(k_count_rows<false>, dim3((unsigned)blocks), dim3(256), 0, st, a, (int)block);
    const int64_t others = a.n_rows && !in_place(a) ? row_grid(classes, round_up(a.n_in, 64)).x : 0;
    TF_BY_TYPE(a.dtype, k_pack_rows, dim3((unsigned)(blocks + others)), a, (int)block, (int)blocks, counted, classes);
    return (int)hipGetLastError();
}

// W's rows as an operand, packed where they cannot be read in place (the first ones have been).
Side classes(const XentLaunch &a, int64_t first, int64_t count, hipStream_t st) {
    if (in_place(a)) return Side{static_cast<const char *>(a.W) + first * a.ldw * (a.dtype == TF_F32 ? 4 : 2), a.ldw, 0, count, a.n_in};
    if (first) TF_BY_TYPE(a.dtype, k_pack_classes, row_grid(count, round_up(a.n_in, 64)), a, first, count);
    return Side{a.s.w, a.s.ld, a.s.w_cap, count, round_up(a.n_in, 64)};
}

ProductLaunch logits(const XentLaunch &a, const Side &W, int64_t first, int64_t count) {
    ProductLaunch p{};
    p.M = W;
    p.N = Side{a.s.x, a.s.ld, a.s.x_plane, round_up(a.n_rows, 256), round_up(a.n_in, 64)};
    p.any = through_registers(a);
    p.parts = parts_of(a);
    p.k_steps = (int32_t)ceil_div(a.n_in, step_of(a));
    p.n = a.s.n;
    p.n_rows = 1;
    p.splits = 1;
    p.m_count = (int32_t)count;
    p.n_count = a.n_rows;
    p.first_class = (int32_t)first;
    p.label = a.s.label;
    return p;
}

int64_t m_side(ProductTile t) { return t == kTile256 ? 256 : t == kTile16 ? 64 : 128; }
int64_t n_side(ProductTile t) { return t == kTile256 ? 256 : t == kTile16 ? 16 : t == kTile64 ? 64 : 128; }
// Sums that a tile of logits leaves of each row.
int64_t sums_of(ProductTile t) { return t == kTile256 || t == kTile128 ? 2 : 1; }
// How a product of m x n, `steps` steps long (each made of `pairs` pairs of parts), is launched: its tile, and the shares of its contraction (`most`
// of them at most; 0: it cannot be cut).  16 rows or fewer are one tile: the launch is bound by reading the other operand.  Otherwise whichever tile is expected
// to take the least time: tenths of a microsecond a step and a tile, fitted to sizes from 100 x 300 x 4096 to 8192 x 32768 x 4096 in bf16 (which
// they meet within a fifth; `slow`: operands through registers or transposed; fp32 is bound by its instructions).  Measured, us, tiles of 64 x 16, 128 x 64, 128 x 128,
// 256 x 256: logits of 100 x 300 x 4096 13, 23, 39; 300 x 2000 x 4096 23, 24, 43; 2000 x 1000 x 2000 38, 19, 28; 500 x 10000 x 2048 74, 38, 32;
// 1024 x 40960 x 1024 91 and 105 with the last two, 8192 x 32768 x 4096 1770 and 1610.
struct Cut {
    ProductTile tile;
    int64_t shares;
};
double tenths(ProductTile t, int64_t tiles, double steps, bool native, bool slow) {
    const double rounds = (double)ceil_div(tiles, 256);
    switch (t) {
        case kTile16: return (native ? 1.6 : slow ? 1.8 : 1.2) * rounds * steps + 2 * rounds + 47;
        case kTile64: return (native ? 8.5 : 2.8) * rounds * steps + 22 * rounds + 50;
        case kTile128: return (native ? 17 * rounds : std::max(4 * rounds, 6.0)) * steps + 18 * rounds + 80;
        default: return 14 * rounds * steps + 130 * rounds;
    }
}
Cut cut_product(int64_t m, int64_t n, int64_t steps, int pairs, bool native, bool slow, bool rows, int64_t most) {
    most = std::max<int64_t>(1, std::min<int64_t>(most, steps / least_share(pairs == 6 ? 3 : 1)));
    n = std::max<int64_t>(n, 1);
    if (rows && n <= 16) return Cut{kTile16, std::max<int64_t>(1, std::min(1024 / ceil_div(m, m_side(kTile16)), most))};
    const bool few = rows && (n <= 64 || m <= 128);
    Cut best{few ? kTile64 : kTile128, 1};
    double least = 0;
    for (const ProductTile t : {kTile64, kTile16, kTile128, kTile256}) {
        const bool small = t == kTile64 || t == kTile16;
        if (small ? !rows : few || (native && t == kTile256)) continue;
        for (int64_t s = 1; s <= std::min<int64_t>(most, 512); s = s < 8 ? s + 1 : s * 5 / 4) {
            const double time = tenths(t, ceil_div(m, m_side(t)) * ceil_div(n, n_side(t)) * s, (double)steps * pairs / s, native, slow) + (s > 1 ? 40 + (double)s * m * n / 50000 : 0.0);
            if (least == 0 || time < least) {
                best = Cut{t, s};
                least = time;
            }
        }
    }
    return best;
}

// Up to 32 rows, and up to 64 where that fills the card.  Columns -> classes, us, and as a product of tiles of 128 x 128: 4096 -> 65536 1 row 96 / 180,
// 16 rows 125 / 199; 4096 -> 20000 32 rows 36 / 60, 64 rows 51 / 60; 777 -> 50000 20 rows 35 / 42; 512 -> 1000 64 rows 10.4 / 5.7.
bool few_rows(const XentLaunch &a, int64_t count) {
    return a.dtype != TF_F32 && (a.n_rows <= 32 || (a.n_rows <= 64 && count * a.n_in >= (int64_t)1 << 23));
}
template <int EL> void launch_few_rows(const XentLaunch &a, int64_t first, int64_t count, int64_t g_ld, hipStream_t st) {
    const int64_t columns = ceil_div(a.n_in, 256), each = round_up(std::max<int64_t>(64, count * columns / 2048), 64);
    const dim3 grid((unsigned)columns, (unsigned)ceil_div(count, each));
    if (a.n_rows <= 32) hipLaunchKernelGGL((k_few_rows<EL, 1>), grid, dim3(256), 0, st, a, first, count, g_ld, each);
    else hipLaunchKernelGGL((k_few_rows<EL, 2>), grid, dim3(256), 0, st, a, first, count, g_ld, each);
}

// Whether the last workgroup of a block of rows adds up its `sums` sums: the workgroups count themselves in one after the other, 20 ns each, which
// is lost where many end at the same time.  Calls of one bf16 row, us, joined / by another launch: 8000 x 512 (125 workgroups) 13.6 / 14.2, 20000 x 1024
// (313) 19.0 / 18.7, 65000 x 256 (1016) 24.3 / 16.8, 65536 x 4096 (1024) 110.8 / 112.4; 300 rows of 2000 x 1000 18.5 / 19.7.
bool joins(int64_t m_tiles, int64_t n_tiles, int64_t sums) { return m_tiles == 1 || (m_tiles <= 256 && n_tiles <= kMostJoins && sums <= 8192); }

}  // namespace

int launch_xent(const XentLaunch &call, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    XentLaunch a = call;
    a.native = is_native(a);
    const int64_t ld = round_up(a.n_rows, 16);
    int64_t piece = a.s.part_cap / ld * 64 / 256 * 256;       // (a sum of every 64 classes at the most)
    if (!in_place(a)) piece = std::min(piece, a.s.w_cap / a.s.ld);
    int e = begin(a, std::min<int64_t>(piece, a.n_classes), st);
    if (e) return e;
    for (int64_t first = 0; first < a.n_classes; first += piece) {
        const int64_t count = std::min<int64_t>(piece, a.n_classes - first);
        ProductLaunch p = logits(a, classes(a, first, count, st), first, count);
        p.tile = cut_product(count, a.n_rows, p.k_steps, p.parts == 3 ? 6 : 1, a.native, p.any, true, 0).tile;
        p.end = kEndSums;
        p.hit = a.s.hit;
        p.part = a.s.part;
        p.part_ld = ld;
        const int64_t blocks = ceil_div(count, m_side(p.tile)) * sums_of(p.tile);
        p.join = count == a.n_classes && joins(ceil_div(count, m_side(p.tile)), ceil_div(a.n_rows, n_side(p.tile)), blocks * std::min<int64_t>(std::max(a.n_rows, 1), n_side(p.tile)));
        p.arrived = a.s.arrived;
        p.out_row = a.s.list;
        p.loss = a.loss;
        p.lse_out = a.lse;
        e = launch_product(p, a, stream);
        if (e) return e;
        if (p.join) return 0;
        const int is_first = first == 0, is_last = first + count == a.n_classes;
        if (a.n_rows <= 256) hipLaunchKernelGGL(k_merge<1>, dim3((unsigned)a.n_rows), dim3(1024), 0, st, a, blocks, ld, is_first, is_last);
        else if (a.n_rows <= 4096) hipLaunchKernelGGL(k_merge<8>, dim3((unsigned)ceil_div(a.n_rows, 8)), dim3(1024), 0, st, a, blocks, ld, is_first, is_last);
        else hipLaunchKernelGGL(k_merge<64>, dim3((unsigned)ceil_div(a.n_rows, 64)), dim3(1024), 0, st, a, blocks, ld, is_first, is_last);
        e = (int)hipGetLastError();
        if (e) return e;
    }
    return 0;
}

int launch_xent_grad(const XentLaunch &call, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    XentLaunch a = call;
    a.native = is_native(a);
    const int64_t rows = round_up(std::max(a.n_rows, 1), 256);
    int64_t piece = std::min({round_up(a.n_classes, 256), (a.s.g_cap / rows - kRowPad) / 256 * 256, kMostColumnsOfG});
    if (!in_place(a)) piece = std::min(piece, a.s.w_cap / a.s.ld);
    const int64_t g_ld = piece + kRowPad;
    const int parts = parts_of(a), pairs = parts == 3 ? 6 : 1, step = step_of(a);
    const int64_t dx_size = rows * a.s.slab_ld;
    // (the same shares for every piece: the slabs are added to)
    const Cut dx = cut_product(a.n_in, a.n_rows, ceil_div(std::min<int64_t>(piece, a.n_classes), step), pairs, a.native, true, true, a.s.dx_cap / dx_size);
    a.direct_dx = piece >= a.n_classes && dx.shares == 1;
    int e = begin(a, std::min<int64_t>(piece, a.n_classes), st);
    if (e) return e;
    for (int64_t first = 0; first < a.n_classes; first += piece) {
        const int64_t count = std::min<int64_t>(piece, a.n_classes - first);
        if (a.n_rows) {
            const Side W = classes(a, first, count, st);
            ProductLaunch p = logits(a, W, first, count);
            p.tile = cut_product(count, a.n_rows, p.k_steps, p.parts == 3 ? 6 : 1, a.native, p.any, true, 0).tile;
            p.end = kEndGradient;
            p.lse = a.s.lse;
            p.g = a.s.g;
            p.hit = a.loss_in ? a.s.hit : nullptr;
            p.G = a.s.G;
            p.g_ld = g_ld;
            p.g_plane = a.s.g_cap;
            p.for_dx = a.dX != nullptr;
            p.for_dw = a.dW != nullptr;
            p.same = a.s.same;
            e = launch_product(p, a, stream);
            if (e) return e;
            if (a.dX) {
                ProductLaunch q{};
                q.M = W;
                q.any = through_registers(a);
                q.N = Side{a.s.G, g_ld, a.s.g_cap, rows, round_up(count, 64)};
                q.parts = parts;
                q.k_steps = (int32_t)ceil_div(count, step);
                q.n = a.s.n;
                q.n_rows = 1;
                q.m_count = a.n_in;
                q.n_count = a.n_rows;
                q.end = a.direct_dx ? kEndOut : kEndSlab;
                q.unit = a.s.unit;
                q.row_unit = a.dtype == TF_F16 ? a.s.dloss : nullptr;
                q.out = a.dX;
                q.ldo = a.lddx;
                q.out_row = a.s.list;
                q.out_dtype = a.dtype;
                q.tile = dx.tile;
                q.splits = (int32_t)dx.shares;
                q.slab = a.s.dx;
                q.slab_ld = a.s.slab_ld;
                q.slab_size = dx_size;
                q.add = first != 0;
                e = launch_product(q, a, stream);
                if (e) return e;
            }
        }
        if (a.dW && few_rows(a, count)) {
            if (a.dtype == TF_BF16) launch_few_rows<TF_BF16>(a, first, count, g_ld, st);
            else launch_few_rows<TF_F16>(a, first, count, g_ld, st);
            e = (int)hipGetLastError();
            if (e) return e;
        } else if (a.dW) {
            ProductLaunch q{};
            q.M = Side{a.s.x, a.s.ld, a.s.x_plane, 0, a.s.ld};
            q.N = Side{a.s.G, g_ld, a.s.g_cap, 0, piece};
            q.g_plane = a.s.g_cap;
            q.same = a.s.same;
            q.parts = parts;
            q.n = a.s.n;
            q.k_rows = 1;
            q.m_count = a.n_in;
            q.n_count = (int32_t)count;
            const int64_t size = round_up(count, 256) * a.s.slab_ld;
            const Cut dw = cut_product(a.n_in, count, ceil_div(a.n_rows, step), pairs, a.native, false, false, a.s.dw_cap / size);
            q.tile = dw.tile;
            q.splits = (int32_t)dw.shares;
            q.unit = a.s.unit;
            q.out = static_cast<char *>(a.dW) + first * a.lddw * (a.dtype == TF_F32 ? 4 : 2);
            q.ldo = a.lddw;
            q.out_dtype = a.dtype;
            q.slab = a.s.dw;
            q.slab_ld = a.s.slab_ld;
            q.slab_size = size;
            q.end = q.splits > 1 ? kEndSlab : kEndOut;
            e = launch_product(q, a, stream);
            if (e) return e;
            if (q.splits > 1) TF_BY_TYPE(a.dtype, k_finish_classes, slab_grid(count, a.n_in, q.splits), a, first, count, q.splits, size);
        }
    }
    if (a.dX && a.n_rows && !a.direct_dx) TF_BY_TYPE(a.dtype, k_finish_rows, slab_grid(a.n_rows, a.n_in, dx.shares), a, (int)dx.shares, dx_size);
    return (int)hipGetLastError();
}

}  // namespace tf
