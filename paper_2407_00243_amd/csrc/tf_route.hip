// Router: the largest scores of each token and their weights.
#include <algorithm>

#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves;

__device__ __forceinline__ float wave_sum(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ __forceinline__ float wave_max(float x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
    return x;
}

// One wave per token; lane l holds the scores of experts l, l + 64, ..., V of them.  k times the largest of those left: k exchanges
// over the wave, all in registers, no LDS and no barrier.  Bound by launch and latency: 1 token, 64 experts, k = 6 5.5 us in a graph; 2048
// tokens, 160 experts, k = 8 (0.8 MB) 8.9 us.
template <int EL, int V> __global__ __launch_bounds__(kThreads) void k_route(const RouteLaunch a) {
    typedef typename El<EL>::T T;
    const int lane = threadIdx.x & 63;
    const int t = a.first + (int)(blockIdx.x * kWaves + (threadIdx.x >> 6));      // (below 2^31: a launch's first is a multiple of kWaves)
    if (t >= a.n_tokens) return;
    const T *row = static_cast<const T *>(a.scores) + (int64_t)t * a.ld;
    const float low = -__builtin_inff();
    float l[V], key[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const int e = lane + 64 * v;
        l[v] = low;
        key[v] = low;
        if (e < a.n_experts) {
            const float x = El<EL>::get(row[e]);
            l[v] = __builtin_isnan(x) ? low : x;
            const float y = a.bias ? l[v] + a.bias[e] : l[v];
            key[v] = __builtin_isnan(y) ? low : y;
        }
    }
    int mine = -1;             // the expert that this lane's rank selects, and its score
    float score = low;
    for (int i = 0; i < a.k; ++i) {
        float best = low, best_l = low;
        int at = 0x7fffffff;
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (key[v] > best) {
                best = key[v];
                best_l = l[v];
                at = lane + 64 * v;
            }
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const float ob = __shfl_xor(best, d, 64), ol = __shfl_xor(best_l, d, 64);
            const int oa = __shfl_xor(at, d, 64);
            if (ob > best || (ob == best && oa < at)) {
                best = ob;
                best_l = ol;
                at = oa;
            }
        }
        if (!(best > low)) break;
        if (lane == i) {
            mine = at;
            score = best_l;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
            if (at == lane + 64 * v) key[v] = low;
    }
    float w;
    if (a.scoring == TF_ROUTE_SOFTMAX || a.scoring == TF_ROUTE_SOFTMAX_TOP) {
        float top = score, sum = 0.0f;
        if (a.scoring == TF_ROUTE_SOFTMAX) {
#pragma unroll
            for (int v = 0; v < V; ++v) top = fmaxf(top, l[v]);
            top = wave_max(top);
#pragma unroll
            for (int v = 0; v < V; ++v) sum += l[v] > low ? expf(l[v] - top) : 0.0f;
        } else {
            top = wave_max(top);
            sum = mine >= 0 ? expf(score - top) : 0.0f;
        }
        w = expf(score - top) / wave_sum(sum);
    } else {
        // 1 / (1 + exp(-l)) = exp(min(l, 0)) / (1 + exp(-|l|)), where nothing overflows.  Shares are taken of numerators over the largest
        // one, so that their sum is 1/2 or more however small the sigmoids are.
        const float below = fminf(score, 0.0f);
        const float top = a.scoring == TF_ROUTE_SIGMOID_TOP ? wave_max(mine >= 0 ? below : low) : 0.0f;
        w = expf(below - top) / (1.0f + expf(-fabsf(score)));
        if (a.scoring == TF_ROUTE_SIGMOID_TOP) w /= wave_sum(mine >= 0 ? w : 0.0f);
    }
    if (lane < a.k) {
        a.colidx[(int64_t)t * a.k + lane] = mine;
        a.vals[(int64_t)t * a.k + lane] = mine >= 0 ? w * a.scale : 0.0f;
    }
    if (lane == 0) {
        a.rowptr[t] = t * a.k;
        if (t == a.n_tokens - 1) a.rowptr[t + 1] = (t + 1) * a.k;
    }
}

template <int EL> void route_el(const RouteLaunch &a, hipStream_t st) {
    const dim3 grid((unsigned)std::min(ceil_div((int64_t)a.n_tokens - a.first, kWaves), most_workgroups(kThreads))), block(kThreads);
    if (a.n_experts <= 64) hipLaunchKernelGGL((k_route<EL, 1>), grid, block, 0, st, a);
    else if (a.n_experts <= 128) hipLaunchKernelGGL((k_route<EL, 2>), grid, block, 0, st, a);
    else if (a.n_experts <= 256) hipLaunchKernelGGL((k_route<EL, 4>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_route<EL, 16>), grid, block, 0, st, a);
}

}  // namespace

int launch_route(const RouteLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    RouteLaunch b = a;
    for (int64_t first = 0; first < a.n_tokens; first += most_workgroups(kThreads) * kWaves) {
        b.first = (int32_t)first;
        if (a.dtype == TF_BF16) route_el<TF_BF16>(b, st);
        else if (a.dtype == TF_F16) route_el<TF_F16>(b, st);
        else route_el<TF_F32>(b, st);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return (int)e;
    }
    return 0;
}

}  // namespace tf
