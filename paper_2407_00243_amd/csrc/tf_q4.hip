// Weights of 4 bits: into and out of the library's layout (tf_moe.h).  One pass over memory each, run when weights are loaded, and
// written for that: elements are read and written one by one, at an eighth to a fifth of a copy's rate.  8192 x 8192, E2M1 with groups
// of 32: pack 175 us (with its check, 0.6 TB/s), quantize from bf16 200 (0.84), unpack to bf16 294 (0.57).
#include <algorithm>

#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr int kThreads = 256;

// Where word `w` of a stack of matrices sits: its matrix, row and first column.
struct Place {
    int64_t mat, row, col;
};
__device__ __forceinline__ Place place_of_word(int64_t w, int64_t tiles, int64_t blocks) {
    const int j = w & 3, lane = (w >> 2) & 63;
    const int64_t block = w >> 8, kb = block % blocks, t = block / blocks;
    return Place{t / tiles, (t % tiles) * 16 + (lane & 15), kb * kQ4Block + 32 * j + 8 * (lane >> 4)};
}
// Place of the scale of (row, group q of block kb) of a matrix, in elements from the matrix's first.
__device__ __forceinline__ int64_t scale_at(int64_t row, int64_t kb, int q, int64_t blocks, int per_block) {
    return ((row >> 4) * blocks + kb) * (16 * per_block) + (row & 15) * per_block + q;
}

template <int KIND> __global__ __launch_bounds__(kThreads) void k_q4_pack(const Q4Launch a, int64_t tiles, int64_t blocks) {
    const int64_t words = a.n_mats * tiles * blocks * 256;
    bool bad = false;
    for (int64_t w = (int64_t)blockIdx.x * kThreads + threadIdx.x; w < words; w += (int64_t)gridDim.x * kThreads) {
        const Place at = place_of_word(w, tiles, blocks);
        uint32_t word = 0;
        if (at.row < a.n_rows) {
            const int8_t *src = a.src_codes + (at.mat * a.n_rows + at.row) * a.n_cols + at.col;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (at.col + i >= a.n_cols) break;
                const int c = src[i];
                if constexpr (KIND == TF_Q4_E2M1) {
                    bad |= c < 0 || c > 15;
                    word |= (uint32_t)(c & 7) << q4_low_bit(KIND, i) | (uint32_t)((c >> 3) & 1) << q4_sign_bit(KIND, i);
                } else {
                    bad |= c < -7 || c > 7;
                    word |= (uint32_t)((c < 0 ? -c : c) & 7) << q4_low_bit(KIND, i) | (uint32_t)(c < 0) << q4_sign_bit(KIND, i);
                }
            }
        }
        static_cast<uint32_t *>(a.codes)[w] = word;
    }
    if (bad) *a.bad = 1;         // (every writer writes the same)
}

__global__ __launch_bounds__(kThreads) void k_q4_pack_scales(const Q4Launch a, int64_t tiles, int64_t blocks) {
    const int per_block = kQ4Block / a.group;
    const int64_t groups = (a.n_cols + a.group - 1) / a.group, n = a.n_mats * tiles * 16 * blocks * per_block;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) {
        const int64_t q = i % (blocks * per_block), row = i / (blocks * per_block) % (tiles * 16), mat = i / (blocks * per_block) / (tiles * 16);
        uint16_t s = 0;
        if (row < a.n_rows && q < groups) s = static_cast<const uint16_t *>(a.src_scales)[(mat * a.n_rows + row) * groups + q];
        static_cast<uint16_t *>(a.scales)[mat * tiles * blocks * 16 * per_block + scale_at(row, q / per_block, (int)(q % per_block), blocks, per_block)] = s;
    }
}

__device__ __forceinline__ uint32_t quantize_one(int kind, float w, float s) {
    const float q = fabsf(w) / s;
    // (scale 0: the group holds nothing else; an infinite or NaN scale makes NaN of any code)
    if (!(s > 0.0f) || !(q >= 0.0f)) return 0;
    if (kind == TF_Q4_INT) return (uint32_t)fminf(rintf(q), 7.0f);
    return (q > 0.25f) + (q >= 0.75f) + (q > 1.25f) + (q >= 1.75f) + (q > 2.5f) + (q >= 3.5f) + (q > 5.0f);
}

// A wave takes the 128 columns of a block of one row, two columns a lane.
template <int EL> __global__ __launch_bounds__(kThreads) void k_q4_quantize(const Q4Launch a, int64_t tiles, int64_t blocks) {
    typedef typename El<EL>::T T;
    const int lane = threadIdx.x & 63, per_block = kQ4Block / a.group;
    const int64_t n = a.n_mats * tiles * 16 * blocks;
    for (int64_t i = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); i < n; i += (int64_t)gridDim.x * (kThreads / 64)) {
        const int64_t kb = i % blocks, row = i / blocks % (tiles * 16), mat = i / blocks / (tiles * 16);
        float w[2] = {0.0f, 0.0f};
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int64_t col = kb * kQ4Block + 2 * lane + c;
            if (row < a.n_rows && col < a.n_cols) w[c] = El<EL>::get(static_cast<const T *>(a.weights)[(mat * a.n_rows + row) * a.n_cols + col]);
        }
        // largest magnitude of the group, as bits: a NaN counts as more than infinity
        uint32_t most = max(__float_as_uint(w[0]) & 0x7fffffffu, __float_as_uint(w[1]) & 0x7fffffffu);
        for (int d = 1; d < a.group / 2; d <<= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d, 64));
        const uint16_t scale = El<TF_BF16>::put(__uint_as_float(most) / (a.kind == TF_Q4_INT ? 7.0f : 6.0f));
        const float s = El<TF_BF16>::get(scale);
        uint32_t word = 0;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int at = 2 * (lane & 3) + c;
            const uint32_t code = quantize_one(a.kind, w[c], s);
            word |= code << q4_low_bit(a.kind, at) | (uint32_t)(code != 0 && w[c] < 0.0f) << q4_sign_bit(a.kind, at);
        }
        word |= (uint32_t)__shfl_xor((int)word, 1, 64);
        word |= (uint32_t)__shfl_xor((int)word, 2, 64);
        const int64_t block = (mat * tiles + (row >> 4)) * blocks + kb;
        const int c8 = lane >> 2;                // columns 8 c8 .. 8 c8 + 7 of the block
        if ((lane & 3) == 0) static_cast<uint32_t *>(a.codes)[block * 256 + (16 * (c8 & 3) + (row & 15)) * 4 + (c8 >> 2)] = word;
        if (2 * lane % a.group == 0)
            static_cast<uint16_t *>(a.scales)[mat * tiles * blocks * 16 * per_block + scale_at(row, kb, 2 * lane / a.group, blocks, per_block)] = scale;
    }
}

template <int EL> __global__ __launch_bounds__(kThreads) void k_q4_unpack(const Q4Launch a, int64_t tiles, int64_t blocks) {
    typedef typename El<EL>::T T;
    const int per_block = kQ4Block / a.group;
    const int64_t words = a.n_mats * tiles * blocks * 256;
    for (int64_t w = (int64_t)blockIdx.x * kThreads + threadIdx.x; w < words; w += (int64_t)gridDim.x * kThreads) {
        const Place at = place_of_word(w, tiles, blocks);
        if (at.row >= a.n_rows) continue;
        const uint32_t word = static_cast<const uint32_t *>(a.codes)[w];
        const int64_t kb = at.col / kQ4Block;
        const int q = (int)(at.col % kQ4Block) / a.group;
        const float s = El<TF_BF16>::get(static_cast<const uint16_t *>(
            a.scales)[at.mat * tiles * blocks * 16 * per_block + scale_at(at.row, kb, q, blocks, per_block)]);
        T *dst = static_cast<T *>(a.weights) + (at.mat * a.n_rows + at.row) * a.n_cols + at.col;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (at.col + i >= a.n_cols) break;
            const uint32_t m = (word >> q4_low_bit(a.kind, i)) & 7;
            float v = (float)m;
            if (a.kind == TF_Q4_E2M1) v = m < 2 ? 0.5f * m : (1.0f + 0.5f * (m & 1)) * (float)(1u << ((m >> 1) - 1));
            if ((word >> q4_sign_bit(a.kind, i)) & 1) v = -v;
            dst[i] = El<EL>::put(v * s);
        }
    }
}

unsigned grid_of(int64_t items, int per_block) { return (unsigned)std::max<int64_t>(1, std::min<int64_t>((items + per_block - 1) / per_block, 1 << 16)); }

}  // namespace

int launch_q4_pack(const Q4Launch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t tiles = q4_tiles(a.n_rows), blocks = q4_blocks(a.n_cols), words = a.n_mats * tiles * blocks * 256;
    if (a.kind == TF_Q4_INT)
        hipLaunchKernelGGL(k_q4_pack<TF_Q4_INT>, dim3(grid_of(words, kThreads)), dim3(kThreads), 0, st, a, tiles, blocks);
    else
        hipLaunchKernelGGL(k_q4_pack<TF_Q4_E2M1>, dim3(grid_of(words, kThreads)), dim3(kThreads), 0, st, a, tiles, blocks);
    hipLaunchKernelGGL(k_q4_pack_scales, dim3(grid_of(words, kThreads)), dim3(kThreads), 0, st, a, tiles, blocks);
    return (int)hipGetLastError();
}

int launch_q4_quantize(const Q4Launch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t tiles = q4_tiles(a.n_rows), blocks = q4_blocks(a.n_cols);
    const dim3 grid(grid_of(a.n_mats * tiles * 16 * blocks, kThreads / 64));
    if (a.dtype == TF_BF16) hipLaunchKernelGGL(k_q4_quantize<TF_BF16>, grid, dim3(kThreads), 0, st, a, tiles, blocks);
    else if (a.dtype == TF_F16) hipLaunchKernelGGL(k_q4_quantize<TF_F16>, grid, dim3(kThreads), 0, st, a, tiles, blocks);
    else hipLaunchKernelGGL(k_q4_quantize<TF_F32>, grid, dim3(kThreads), 0, st, a, tiles, blocks);
    return (int)hipGetLastError();
}

int launch_q4_unpack(const Q4Launch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const int64_t tiles = q4_tiles(a.n_rows), blocks = q4_blocks(a.n_cols);
    const dim3 grid(grid_of(a.n_mats * tiles * blocks * 256, kThreads));
    if (a.dtype == TF_BF16) hipLaunchKernelGGL(k_q4_unpack<TF_BF16>, grid, dim3(kThreads), 0, st, a, tiles, blocks);
    else if (a.dtype == TF_F16) hipLaunchKernelGGL(k_q4_unpack<TF_F16>, grid, dim3(kThreads), 0, st, a, tiles, blocks);
    else hipLaunchKernelGGL(k_q4_unpack<TF_F32>, grid, dim3(kThreads), 0, st, a, tiles, blocks);
    return (int)hipGetLastError();
}

}  // namespace tf
