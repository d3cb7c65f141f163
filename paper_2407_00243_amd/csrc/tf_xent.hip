// Cross entropy of a product: the rows that count, operands, merging of sums, and the launches of a call.
#include <algorithm>

#include "tf_loss.h"
#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr float kLow = -__builtin_inff();

// ------------------------------------------------------------------------------ rows with a label

// Numbers the rows that have a label in their order.  A block of 4096 rows a workgroup: with `sums` 1 it only counts, with 0 it takes the
// counts of the blocks before it and writes.
__global__ __launch_bounds__(1024) void k_rows(const XentLaunch a, const int only_count) {
    __shared__ int of_wave[16], before[16];
    __shared__ float top_of_wave[16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t r0 = (int64_t)blockIdx.x * kRowBlock + tid * 4;
    int mine = 0;
    float top = 0.0f;
    bool keep[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        keep[i] = false;
        if (r0 + i < a.n_rows) {
            const int y = a.labels[r0 + i];
            keep[i] = y >= 0 && y < a.n_classes;
            if (keep[i] && a.dloss) {
                const float g = fabsf(a.dloss[r0 + i]);
                if (g < __builtin_inff()) top = fmaxf(top, g);
            }
        }
        mine += keep[i];
    }
    int upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(upto, d, 64);
        if (lane >= d) upto += x;
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d, 64));
    int earlier = 0;
    if (!only_count)
        for (int b = tid; b < (int)blockIdx.x; b += 1024) earlier += a.s.block_rows[b];
#pragma unroll
    for (int d = 32; d; d >>= 1) earlier += __shfl_xor(earlier, d, 64);
    if (lane == 63) of_wave[wave] = upto;
    if (lane == 0) {
        top_of_wave[wave] = top;
        before[wave] = earlier;
    }
    __syncthreads();
    int at = upto - mine, all = 0;
    top = 0.0f;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) at += of_wave[w];
        all += of_wave[w];
        top = fmaxf(top, top_of_wave[w]);
        if (!only_count) at += before[w];
    }
    if (tid == 0 && (only_count || gridDim.x == 1)) {
        a.s.block_rows[blockIdx.x] = all;
        a.s.block_top[blockIdx.x] = top;
    }
    if (only_count) return;
    if (tid == 1023 && blockIdx.x == gridDim.x - 1) *a.s.n = at + mine;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (r0 + i < a.n_rows) {
            a.s.pos[r0 + i] = keep[i] ? at : -1;
            if (keep[i]) a.s.list[at++] = (int)(r0 + i);
            else if (a.loss) a.loss[r0 + i] = a.lse[r0 + i] = 0.0f;
        }
}

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

// Eight columns as an operand of the products: 16-bit numbers as they are, fp32 ones as three bf16 numbers that add up to them.
template <int EL> __device__ __forceinline__ void put8(const float (&x)[8], uint16_t *to, int64_t plane) {
    Words4 w[3];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (EL == TF_F32) {
            float a = x[2 * i], b = x[2 * i + 1];
#pragma unroll
            for (int p = 0; p < 3; ++p) {
                const uint16_t ha = El<TF_BF16>::put(a), hb = El<TF_BF16>::put(b);
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

// x: the rows that count, one after the other; columns up to a multiple of 64 are zeros behind the last one.
template <int EL> __global__ __launch_bounds__(256) void k_pack_rows(const XentLaunch a) {
    const int n = *a.s.n;
    const int64_t k = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
    float top = 0.0f;
    if (a.dloss && blockIdx.y == 0)
        for (int b = 0; b < (int)ceil_div(a.n_rows, kRowBlock); ++b) top = fmaxf(top, a.s.block_top[b]);
    const float scale = a.dtype == TF_F16 ? 32768.0f : 1.0f;
    if (top == 0.0f) top = 1.0f;
    if (a.dloss && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *a.s.unit = top / scale;
    for (int64_t i = blockIdx.x; i < n; i += gridDim.x) {
        const int64_t row = a.s.list[i];
        if (blockIdx.y == 0 && threadIdx.x == 0) {
            a.s.label[i] = a.labels[row];
            if (a.dloss) {
                a.s.lse[i] = a.lse_in[row];
                a.s.g[i] = a.dloss[row] / top * scale;
            }
        }
        if (k >= round_up(a.n_in, 64)) continue;
        float x[8];
        read8<EL>(x, static_cast<const typename El<EL>::T *>(a.X) + row * a.ldx, k, a.n_in);
        put8<EL>(x, static_cast<uint16_t *>(a.s.x) + i * a.s.ld + k, a.s.x_plane);
    }
}
// w: rows first .. first + count of W likewise.
template <int EL> __global__ __launch_bounds__(256) void k_pack_classes(const XentLaunch a, const int64_t first, const int64_t count, const int64_t plane) {
    const int64_t k = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
    if (k >= round_up(a.n_in, 64)) return;
    for (int64_t i = blockIdx.x; i < count; i += gridDim.x) {
        float x[8];
        read8<EL>(x, static_cast<const typename El<EL>::T *>(a.W) + (first + i) * a.ldw, k, a.n_in);
        put8<EL>(x, static_cast<uint16_t *>(a.s.w) + i * a.s.ld + k, plane);
    }
}

// ------------------------------------------------------------------------------------------- ends

// Adds the sums of `blocks` blocks of classes to those of the classes before them (unless `first`): 64 rows a workgroup, whose 16 waves take
// every sixteenth block each.  The last call writes the results.
__global__ __launch_bounds__(1024) void k_merge(const XentLaunch a, const int64_t blocks, const int64_t ld, const int first, const int last) {
    __shared__ float tops[16][64], sums[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 64 + lane;
    const int n = *a.s.n;
    if ((int64_t)blockIdx.x * 64 >= n) return;
    float top = kLow, sum = 0.0f;
    if (row < n)
#pragma unroll 4
        for (int64_t b = wave; b < blocks; b += 16) {
            const float t = a.s.part_top[b * ld + row], s = a.s.part_sum[b * ld + row], m = fmaxf(top, t);
            sum = (top == kLow ? sum : sum * expf(top - m)) + (t == kLow ? s : s * expf(t - m));
            top = m;
        }
    tops[wave][lane] = top;
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave || row >= n) return;
    if (!first) {
        top = a.s.top[row];
        sum = a.s.sum[row];
    }
    for (int w = first ? 1 : 0; w < 16; ++w) {
        const float t = tops[w][lane], s = sums[w][lane], m = fmaxf(top, t);
        sum = (top == kLow ? sum : sum * expf(top - m)) + (t == kLow ? s : s * expf(t - m));
        top = m;
    }
    if (!last) {
        a.s.top[row] = top;
        a.s.sum[row] = sum;
        return;
    }
    // `sum` is that of the other classes: a small loss keeps its precision as log(1 + sum / exp(label's logit))
    const float hit = a.s.hit[row], lse = top + logf(sum + expf(hit - top));
    const int64_t to = a.s.list[row];
    a.lse[to] = lse;
    a.loss[to] = top - hit < 40.0f ? log1pf(sum * expf(top - hit)) : lse - hit;
}

// dX: the shares' sums of each row that counts, zeros in the others.
template <int EL> __global__ __launch_bounds__(256) void k_finish_rows(const XentLaunch a, const int splits, const int64_t size) {
    const int64_t k = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
    if (k >= a.n_in) return;
    const float unit = *a.s.unit;
    for (int64_t t = blockIdx.x; t < a.n_rows; t += gridDim.x) {
        const int64_t i = a.s.pos[t];
        float x[8] = {};
        if (i >= 0) {
            for (int z = 0; z < splits; ++z) {
                const Float4 *p = reinterpret_cast<const Float4 *>(a.s.dx + z * size + i * a.s.ld + k);
                const Float4 lo = p[0], hi = p[1];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[j] += lo[j];
                    x[4 + j] += hi[j];
                }
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] *= unit;
        }
        write8<EL>(x, static_cast<typename El<EL>::T *>(a.dX) + t * a.lddx, k, a.n_in);
    }
}
// Rows first .. first + count of dW.
template <int EL> __global__ __launch_bounds__(256) void k_finish_classes(const XentLaunch a, const int64_t first, const int64_t count, const int splits, const int64_t size) {
    const int64_t k = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 8;
    if (k >= a.n_in) return;
    const float unit = *a.s.unit;
    for (int64_t i = blockIdx.x; i < count; i += gridDim.x) {
        float x[8] = {};
        for (int z = 0; z < splits; ++z) {
            const Float4 *p = reinterpret_cast<const Float4 *>(a.s.dw + z * size + i * a.s.ld + k);
            const Float4 lo = p[0], hi = p[1];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[j] += lo[j];
                x[4 + j] += hi[j];
            }
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= unit;
        write8<EL>(x, static_cast<typename El<EL>::T *>(a.dW) + (first + i) * a.lddw, k, a.n_in);
    }
}

// --------------------------------------------------------------------------------------- launches

// Rows of a launch (each workgroup goes on by this many) x blocks of 2048 columns.
dim3 row_grid(int64_t rows, int64_t columns) {
    return dim3((unsigned)std::min<int64_t>(rows, 8192), (unsigned)ceil_div(columns, 2048));
}
#define TF_BY_TYPE(dtype, kernel, grid, ...)                                                                           \
    do {                                                                                                               \
        if (dtype == TF_BF16) hipLaunchKernelGGL((kernel<TF_BF16>), grid, dim3(256), 0, st, __VA_ARGS__);              \
        else if (dtype == TF_F16) hipLaunchKernelGGL((kernel<TF_F16>), grid, dim3(256), 0, st, __VA_ARGS__);           \
        else hipLaunchKernelGGL((kernel<TF_F32>), grid, dim3(256), 0, st, __VA_ARGS__);                                \
    } while (0)

int launch_product(const ProductLaunch &p, int dtype, void *stream) {
    return dtype == TF_F16 ? launch_product_f16(p, stream) : launch_product_bf16(p, stream);
}

// Whether W can be read where it lies: 16-bit rows of whole 16-byte pieces.
bool in_place(const XentLaunch &a) {
    return a.dtype != TF_F32 && a.n_in % 8 == 0 && (a.ldw % 8 == 0 || a.n_classes == 1) && reinterpret_cast<uintptr_t>(a.W) % 16 == 0 &&
           a.ldw <= kXentMaxColumns;
}

int begin(const XentLaunch &a, hipStream_t st) {
    const unsigned blocks = (unsigned)std::max<int64_t>(1, ceil_div(a.n_rows, kRowBlock));
    if (blocks > 1) hipLaunchKernelGGL(k_rows, dim3(blocks), dim3(1024), 0, st, a, 1);
    hipLaunchKernelGGL(k_rows, dim3(blocks), dim3(1024), 0, st, a, 0);
    // (also without rows: it sets the unit)
    TF_BY_TYPE(a.dtype, k_pack_rows, row_grid(std::max(a.n_rows, 1), round_up(a.n_in, 64)), a);
    return (int)hipGetLastError();
}

// W's rows as an operand, packed first where they cannot be read in place.
Side classes(const XentLaunch &a, int64_t first, int64_t count, hipStream_t st) {
    if (in_place(a)) return Side{static_cast<const uint16_t *>(a.W) + first * a.ldw, a.ldw, 0, count, a.n_in};
    const int64_t plane = a.s.w_cap;
    TF_BY_TYPE(a.dtype, k_pack_classes, row_grid(count, round_up(a.n_in, 64)), a, first, count, plane);
    return Side{a.s.w, a.s.ld, plane, count, round_up(a.n_in, 64)};
}

ProductLaunch logits(const XentLaunch &a, const Side &W, int64_t first, int64_t count) {
    ProductLaunch p{};
    p.M = W;
    p.N = Side{a.s.x, a.s.ld, a.s.x_plane, round_up(a.n_rows, 256), round_up(a.n_in, 64)};
    p.parts = a.dtype == TF_F32 ? 3 : 1;
    p.k_steps = (int32_t)ceil_div(a.n_in, 64);
    p.n = a.s.n;
    p.n_rows = 1;
    p.splits = 1;
    p.m_count = (int32_t)count;
    p.n_count = a.n_rows;
    p.first_class = (int32_t)first;
    p.label = a.s.label;
    return p;
}

// A tile of 256 x 256 where there are enough of them for the compute units, else smaller ones; few rows: all of them in one.
ProductTile tile_for(int64_t m, int64_t n, bool rows) {
    if (rows && n <= 16) return kTile16;
    if (rows && n <= 64) return kTile64;
    return ceil_div(m, 256) * ceil_div(n, 256) >= 192 ? kTile256 : kTile128;
}
int64_t side_of(ProductTile t) { return t == kTile256 ? 256 : 128; }
// Shares of a contraction of `steps`, so that the launch has enough workgroups; each has four steps at least.
int64_t shares(ProductTile t, int64_t m, int64_t n, int64_t steps, int64_t most) {
    const int64_t across = t == kTile16 ? 16 : t == kTile64 ? 64 : side_of(t);
    const int64_t groups = ceil_div(m, side_of(t)) * ceil_div(n, across), want = t == kTile256 ? 256 : 512;
    return std::max<int64_t>(1, std::min({want / groups, steps / 4, most}));
}

}  // namespace

int launch_xent(const XentLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    int e = begin(a, st);
    if (e || a.n_rows == 0) return e;
    const int64_t ld = round_up(a.n_rows, 256);
    const int64_t per_tile = a.n_rows <= 64 ? 4 : 2;          // blocks of classes in a tile
    int64_t piece = a.s.part_cap / (ld * per_tile) * 128 / 256 * 256;
    if (!in_place(a)) piece = std::min(piece, a.s.w_cap / a.s.ld);
    for (int64_t first = 0; first < a.n_classes; first += piece) {
        const int64_t count = std::min<int64_t>(piece, a.n_classes - first);
        ProductLaunch p = logits(a, classes(a, first, count, st), first, count);
        p.tile = tile_for(count, a.n_rows, true);
        p.end = kEndSums;
        p.hit = a.s.hit;
        p.part_top = a.s.part_top;
        p.part_sum = a.s.part_sum;
        p.part_ld = ld;
        e = launch_product(p, a.dtype, stream);
        if (e) return e;
        const int64_t blocks = ceil_div(count, side_of(p.tile)) * per_tile;
        hipLaunchKernelGGL(k_merge, dim3((unsigned)ceil_div(a.n_rows, 64)), dim3(1024), 0, st, a, blocks, ld, first == 0, first + count == a.n_classes);
        e = (int)hipGetLastError();
        if (e) return e;
    }
    return 0;
}

int launch_xent_grad(const XentLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    int e = begin(a, st);
    if (e) return e;
    const int64_t rows = round_up(std::max(a.n_rows, 1), 256);
    int64_t piece = std::min(round_up(a.n_classes, 256), (a.s.g_cap / rows - kRowPad) / 256 * 256);
    if (!in_place(a)) piece = std::min(piece, a.s.w_cap / a.s.ld);
    const int64_t g_ld = piece + kRowPad;
    const int parts = a.dtype == TF_F32 ? 3 : 1;
    const int64_t dx_size = rows * a.s.ld;
    // (the same shares for every piece: the slabs are added to)
    const ProductTile dx_tile = tile_for(a.n_in, a.n_rows, true);
    const int64_t dx_shares = a.dX && a.n_rows ? shares(dx_tile, a.n_in, a.n_rows, ceil_div(std::min<int64_t>(piece, a.n_classes), 64), a.s.dx_cap / dx_size) : 1;
    for (int64_t first = 0; first < a.n_classes; first += piece) {
        const int64_t count = std::min<int64_t>(piece, a.n_classes - first);
        if (a.n_rows) {
            const Side W = classes(a, first, count, st);
            ProductLaunch p = logits(a, W, first, count);
            p.tile = tile_for(count, a.n_rows, true);
            p.end = kEndGradient;
            p.lse = a.s.lse;
            p.g = a.s.g;
            p.G = a.s.G;
            p.g_ld = g_ld;
            p.g_plane = a.s.g_cap;
            e = launch_product(p, a.dtype, stream);
            if (e) return e;
            if (a.dX) {
                ProductLaunch q{};
                q.M = W;
                q.N = Side{a.s.G, g_ld, a.s.g_cap, rows, round_up(count, 64)};
                q.parts = parts;
                q.k_steps = (int32_t)ceil_div(count, 64);
                q.n = a.s.n;
                q.n_rows = 1;
                q.m_count = a.n_in;
                q.n_count = a.n_rows;
                q.end = kEndSlab;
                q.tile = dx_tile;
                q.splits = (int32_t)dx_shares;
                q.slab = a.s.dx;
                q.slab_ld = a.s.ld;
                q.slab_size = dx_size;
                q.add = first != 0;
                e = launch_product(q, a.dtype, stream);
                if (e) return e;
            }
        }
        if (a.dW) {
            ProductLaunch q{};
            q.M = Side{a.s.x, a.s.ld, a.s.x_plane, 0, a.s.ld};
            q.N = Side{a.s.G, g_ld, a.s.g_cap, 0, piece};
            q.parts = parts;
            q.n = a.s.n;
            q.k_rows = 1;
            q.m_count = a.n_in;
            q.n_count = (int32_t)count;
            q.tile = tile_for(a.n_in, count, false);
            const int64_t size = round_up(count, 256) * a.s.ld;
            q.splits = (int32_t)shares(q.tile, a.n_in, count, ceil_div(a.n_rows, 64), a.s.dw_cap / size);
            q.unit = a.s.unit;
            q.out = static_cast<char *>(a.dW) + first * a.lddw * (a.dtype == TF_F32 ? 4 : 2);
            q.ldo = a.lddw;
            q.out_dtype = a.dtype;
            q.slab = a.s.dw;
            q.slab_ld = a.s.ld;
            q.slab_size = size;
            q.end = q.splits > 1 ? kEndSlab : kEndOut;
            e = launch_product(q, a.dtype, stream);
            if (e) return e;
            if (q.splits > 1) TF_BY_TYPE(a.dtype, k_finish_classes, row_grid(count, a.n_in), a, first, count, q.splits, size);
        }
    }
    if (a.dX && a.n_rows) TF_BY_TYPE(a.dtype, k_finish_rows, row_grid(a.n_rows, a.n_in), a, (int)dx_shares, dx_size);
    return (int)hipGetLastError();
}

}  // namespace tf
