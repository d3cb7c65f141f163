// Router: counts and mass of the experts, the balance loss, and the gradient of the scores.
#include <algorithm>

#include "tf_loss.h"
#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr float kLow = -__builtin_inff();

// A row of scores lies in L lanes; lane i of them holds NV chunks of sixteen bytes, chunk i + L c: VEC consecutive experts each.
template <int EL, int L, int NV> struct Row {
    static constexpr int VEC = EL == TF_F32 ? 4 : 8, N = VEC * NV, ROWS = 64 / L;
    typedef typename El<EL>::T T;

    static __device__ __forceinline__ int expert(int lane, int i) { return ((lane & (L - 1)) + L * (i / VEC)) * VEC + i % VEC; }

    // The chunks as they lie in memory.  (Rows may begin at any element; what lies behind the last expert is not read.)
    struct Raw {
        AnyWords4 c[NV];
    };
    static __device__ __forceinline__ void load(Raw &r, const T *row, int lane, int n_experts) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int e = expert(lane, c * VEC);
            r.c[c] = AnyWords4{0, 0, 0, 0};
            if (e + VEC <= n_experts) {
                r.c[c] = *reinterpret_cast<const AnyWords4 *>(row + e);
            } else if (e < n_experts) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (e + j < n_experts) put(r.c[c], j, row[e + j]);
            }
        }
    }
    static __device__ __forceinline__ void put(AnyWords4 &w, int j, T x) {
        if constexpr (EL == TF_F32) w[j] = __float_as_uint(x);
        else w[j / 2] |= (uint32_t)x << (16 * (j & 1));
    }
    // Scores in 32 bits; -inf where there is no expert or the score is NaN.
    static __device__ __forceinline__ void unpack(float (&l)[N], const Raw &r, int lane, int n_experts) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float x;
            if constexpr (EL == TF_F32) x = __uint_as_float(r.c[i / VEC][i % VEC]);
            else x = El<EL>::get((uint16_t)(r.c[i / VEC][i % VEC / 2] >> (16 * (i & 1))));
            l[i] = expert(lane, i) < n_experts && !__builtin_isnan(x) ? x : kLow;
        }
    }
    static __device__ __forceinline__ void store(T *row, const float (&d)[N], int lane, int n_experts) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const int e = expert(lane, c * VEC);
            AnyWords4 w{0, 0, 0, 0};
#pragma unroll
            for (int j = 0; j < VEC; ++j) put(w, j, El<EL>::put(d[c * VEC + j]));
            if (e + VEC <= n_experts) {
                *reinterpret_cast<AnyWords4 *>(row + e) = w;
            } else if (e < n_experts) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    if (e + j < n_experts) row[e + j] = El<EL>::put(d[c * VEC + j]);
            }
        }
    }
    static __device__ __forceinline__ float sum(float x) {
#pragma unroll
        for (int d = L / 2; d; d >>= 1) x += __shfl_xor(x, d, 64);
        return x;
    }
    static __device__ __forceinline__ float max(float x) {
#pragma unroll
        for (int d = L / 2; d; d >>= 1) x = fmaxf(x, __shfl_xor(x, d, 64));
        return x;
    }
    // Whether it is true in any of the row's lanes.
    static __device__ __forceinline__ bool any(bool x) {
        const uint64_t b = __ballot(x) >> (threadIdx.x & 63 & ~(L - 1));
        return L == 64 ? b != 0 : (b & (((uint64_t)1 << (L & 63)) - 1)) != 0;
    }
};

// What sigmoids need of a score: sigma = 1 / (1 + exp(-l)) and 1 - sigma, neither of which overflows or cancels.  (The reciprocal is
// good to a unit of 2^-23.)
__device__ __forceinline__ void sigmoid(float l, float &s, float &rest) {
    const float t = expf(-fabsf(l)), r = __builtin_amdgcn_rcpf(1.0f + t);
    s = l >= 0.0f ? r : t * r;
    rest = l >= 0.0f ? t * r : r;
}

// Numerators n_e of the shares n_e / sum n: exp(l_e - top) or sigma(l_e), the latter over exp(top) where all of them are small.  `top` is
// the largest score that counts (min(l, 0) for sigmoids), which is what keeps a sum from being 0; `rest` = 1 - sigma.
template <int N> __device__ __forceinline__ void numerators(float (&n)[N], const float (&l)[N], const float (&s)[N], bool sigmoids, float top) {
    if (sigmoids) {
        const bool small = top < -40.0f;
#pragma unroll
        for (int i = 0; i < N; ++i) n[i] = s[i];
        if (__ballot(small)) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (small) n[i] = l[i] > kLow ? expf(fminf(l[i], 0.0f) - top) * __builtin_amdgcn_rcpf(1.0f + expf(-fabsf(l[i]))) : 0.0f;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) n[i] = l[i] > kLow ? expf(l[i] - top) : 0.0f;
    }
}

__device__ __forceinline__ float over(float x, float total) { return total == 0.0f ? 0.0f : x / total; }

// ---------------------------------------------------------------------------------------- balance

// loss = E sum_e f_e mass_e from the sums of `groups` workgroups, added up in their order: 1024 threads, each an expert and every
// (1024 / experts)-th workgroup.
struct Finish {
    float mass[1024];
    int count[1024];
    float part[16];
    int named[16], rows[16];
};
__device__ void finish(const RouterLaunch &a, int groups, Finish &sh) {
    const int E = a.n_experts, tid = threadIdx.x, threads = blockDim.x;
    const float *mass = static_cast<const float *>(a.workspace);
    const int *count = reinterpret_cast<const int *>(mass + (int64_t)kBalanceGroups * E);
    const int *rows = count + (int64_t)kBalanceGroups * E;
    const int slices = threads / E;
    float m = 0.0f;
    int c = 0, r = 0;
    if (tid < slices * E) {
        const int e = tid % E;
#pragma unroll 8
        for (int g = tid / E; g < groups; g += slices) {
            m += mass[g * E + e];
            c += count[g * E + e];
        }
    }
    for (int g = tid; g < groups; g += threads) r += rows[g];
    sh.mass[tid] = m;
    sh.count[tid] = c;
    __syncthreads();
    m = 0.0f, c = 0;
    if (tid < E)
        for (int s = 0; s < slices; ++s) {
            m += sh.mass[s * E + tid];
            c += sh.count[s * E + tid];
        }
    float x = m * (float)c;
    int named = c;
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        x += __shfl_xor(x, d, 64);
        named += __shfl_xor(named, d, 64);
        r += __shfl_xor(r, d, 64);
    }
    if ((tid & 63) == 0) {
        sh.part[tid >> 6] = x;
        sh.named[tid >> 6] = named;
        sh.rows[tid >> 6] = r;
    }
    __syncthreads();
    x = 0.0f, named = 0, r = 0;
    for (int w = 0; w < threads / 64; ++w) {
        x += sh.part[w];
        named += sh.named[w];
        r += sh.rows[w];
    }
    if (tid < E) {
        a.counts[tid] = c;
        a.mass[tid] = r ? m / (float)r : 0.0f;
    }
    if (tid == 0) {
        a.counts[E] = r;
        a.loss[0] = r ? (float)E * x / ((float)named * (float)r) : 0.0f;
    }
}

__global__ __launch_bounds__(1024) void k_balance_finish(const RouterLaunch a, const int groups) {
    __shared__ Finish sh;
    finish(a, groups, sh);
}

// Every wave takes ROWS tokens at a time and adds up their shares in registers; entries are counted in LDS (whole numbers: their order
// does not matter).
template <int EL, int L, int NV> __global__ __launch_bounds__(1024) void k_balance(const RouterLaunch a) {
    typedef Row<EL, L, NV> R;
    __shared__ union {
        struct {
            float mass[1024];
            int count[1024];
            int rows;
        } own;
        Finish fin;
    } sh;
    const int E = a.n_experts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int sub = lane / L, at = lane & (L - 1);
    const bool sigmoids = a.scoring == TF_ROUTE_SIGMOID || a.scoring == TF_ROUTE_SIGMOID_TOP;
    for (int e = threadIdx.x; e < 1024; e += blockDim.x) sh.own.count[e] = 0;
    __syncthreads();
    float mass[R::N] = {};
    int rows = 0;
    const int64_t step = (int64_t)gridDim.x * waves * R::ROWS;
    typename R::Raw raw{}, next{};
    int64_t t = ((int64_t)blockIdx.x * waves + wave) * R::ROWS + sub;
    const typename R::T *scores = static_cast<const typename R::T *>(a.scores);
    if (t < a.n_tokens) R::load(next, scores + t * a.ld, lane, E);
    for (int64_t base = t - sub; base < a.n_tokens; base += step, t += step) {
        raw = next;
        if (t + step < a.n_tokens) R::load(next, scores + (t + step) * a.ld, lane, E);
        bool named = false;
        if (t < a.n_tokens)
            for (int i = at; i < a.k; i += L) {
                const int c = a.colidx[t * a.k + i];
                if (c >= 0 && c < E) {
                    named = true;
                    atomicAdd(&sh.own.count[c], 1);
                }
            }
        named = R::any(named);
        rows += named;
        float l[R::N], s[R::N], n[R::N], rest, top = kLow, total = 0.0f;
        R::unpack(l, raw, lane, E);
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            if (sigmoids) sigmoid(l[i], s[i], rest);
            top = fmaxf(top, sigmoids ? fminf(l[i], 0.0f) : l[i]);
        }
        numerators(n, l, s, sigmoids, R::max(top));
#pragma unroll
        for (int i = 0; i < R::N; ++i) total += n[i];
        total = R::sum(total);
        const float each = named ? over(1.0f, total) : 0.0f;
        if (named)
#pragma unroll
            for (int i = 0; i < R::N; ++i) mass[i] += n[i] * each;
    }
    // rows of a wave, then waves in their order
#pragma unroll
    for (int d = L; d < 64; d <<= 1) {
#pragma unroll
        for (int i = 0; i < R::N; ++i) mass[i] += __shfl_xor(mass[i], d, 64);
        rows += __shfl_xor(rows, d, 64);
    }
    for (int w = 0; w < waves; ++w) {
        if (w == wave && sub == 0) {
#pragma unroll
            for (int i = 0; i < R::N; ++i) {
                const int e = R::expert(lane, i);
                if (e < E) sh.own.mass[e] = w ? sh.own.mass[e] + mass[i] : mass[i];
            }
            if (at == 0) sh.own.rows = w ? sh.own.rows + rows : rows;
        }
        __syncthreads();
    }
    float *out = static_cast<float *>(a.workspace);
    int *count = reinterpret_cast<int *>(out + (int64_t)kBalanceGroups * E);
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        out[blockIdx.x * E + e] = sh.own.mass[e];
        count[blockIdx.x * E + e] = sh.own.count[e];
    }
    if (threadIdx.x == 0) count[(int64_t)kBalanceGroups * E + blockIdx.x] = sh.own.rows;
    if (gridDim.x == 1) {        // few tokens: one launch
        __syncthreads();
        finish(a, 1, sh.fin);
    }
}

// --------------------------------------------------------------------------------------- gradient

template <int EL, int L, int NV> __global__ __launch_bounds__(256) void k_route_grad(const RouterLaunch a) {
    typedef Row<EL, L, NV> R;
    const int E = a.n_experts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sub = lane / L, at = lane & (L - 1);
    const bool sigmoids = a.scoring == TF_ROUTE_SIGMOID || a.scoring == TF_ROUTE_SIGMOID_TOP;
    const bool over_all = a.dloss || a.scoring == TF_ROUTE_SOFTMAX;
    // shares of the entries that name an expert, and what a share's gradient is multiplied by
    float f[R::N], factor = 0.0f;
    if (a.dloss) {
        float named = 0.0f;
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            const int e = R::expert(lane, i);
            f[i] = e < E ? (float)a.counts[e] : 0.0f;
            named += f[i];
        }
        named = R::sum(named);
#pragma unroll
        for (int i = 0; i < R::N; ++i) f[i] = over(f[i], named);
        factor = over(a.dloss[0] * (float)E, (float)a.counts[E]);
    }
    const int64_t step = (int64_t)gridDim.x * 4 * R::ROWS;
    int64_t t = ((int64_t)blockIdx.x * 4 + wave) * R::ROWS + sub;
    const typename R::T *scores = static_cast<const typename R::T *>(a.scores);
    typename R::T *out = static_cast<typename R::T *>(a.dscores);
    typename R::Raw raw{}, next{};
    if (t < a.n_tokens) R::load(next, scores + t * a.ld, lane, E);
    for (int64_t base = t - sub; base < a.n_tokens; base += step, t += step) {
        raw = next;
        if (t + step < a.n_tokens) R::load(next, scores + (t + step) * a.ld, lane, E);
        float l[R::N], s[R::N], rest[R::N], n[R::N], d[R::N], g[R::N], m[R::N];
        R::unpack(l, raw, lane, E);
        float top = kLow, top_of_named = kLow;
        // entries: how often each expert is named, and the sum of its entries' gradients
#pragma unroll
        for (int i = 0; i < R::N; ++i) g[i] = m[i] = 0.0f;
        bool named = false;
        for (int first = 0; first < a.k; first += L) {
            int c = -1;
            float x = 0.0f;
            if (t < a.n_tokens && first + at < a.k) {
                c = a.colidx[t * a.k + first + at];
                if (c >= E) c = -1;
                if (a.dvals) x = a.dvals[t * a.k + first + at] * a.scale;
            }
            named |= c >= 0;
            const int here = min(L, a.k - first);
            for (int i = 0; i < here; ++i) {
                const int ci = __shfl(c, i, L);
                const float xi = __shfl(x, i, L);
#pragma unroll
                for (int j = 0; j < R::N; ++j)
                    if (R::expert(lane, j) == ci) {
                        g[j] += xi;
                        m[j] += 1.0f;
                    }
            }
        }
        named = R::any(named);
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            rest[i] = 1.0f;
            if (sigmoids) sigmoid(l[i], s[i], rest[i]);
            const float x = sigmoids ? fminf(l[i], 0.0f) : l[i];
            top = fmaxf(top, x);
            if (m[i] > 0.0f) top_of_named = fmaxf(top_of_named, x);
            d[i] = 0.0f;
        }
        top = R::max(top);
        numerators(n, l, s, sigmoids, top);
        if (over_all) {
            float total = 0.0f, fs = 0.0f, gs = 0.0f;
#pragma unroll
            for (int i = 0; i < R::N; ++i) {
                total += n[i];
                if (a.dloss) fs += n[i] * f[i];
                gs += n[i] * g[i];
            }
            total = R::sum(total);
            const float each = over(1.0f, total);
            if (a.dloss && named) {
                fs = R::sum(fs) * each;
#pragma unroll
                for (int i = 0; i < R::N; ++i) d[i] += factor * (n[i] * each) * rest[i] * (f[i] - fs);
            }
            if (a.dvals && named && a.scoring == TF_ROUTE_SOFTMAX) {
                gs = R::sum(gs) * each;
#pragma unroll
                for (int i = 0; i < R::N; ++i) d[i] += n[i] * each * (g[i] - gs);
            }
        }
        if (a.dvals && named && a.scoring == TF_ROUTE_SIGMOID) {
#pragma unroll
            for (int i = 0; i < R::N; ++i)
                if (m[i] > 0.0f) d[i] += s[i] * rest[i] * g[i];
        }
        if (a.dvals && (a.scoring == TF_ROUTE_SOFTMAX_TOP || a.scoring == TF_ROUTE_SIGMOID_TOP)) {
            // a bias may have selected experts far below the largest score: their shares are taken of the largest selected one
            top_of_named = R::max(top_of_named);
            if (__ballot(top_of_named < top - 40.0f)) numerators(n, l, s, sigmoids, top_of_named);
            float total = 0.0f, gs = 0.0f;
#pragma unroll
            for (int i = 0; i < R::N; ++i)
                if (m[i] > 0.0f) {
                    total += m[i] * n[i];
                    gs += n[i] * g[i];
                }
            total = R::sum(total);
            gs = over(R::sum(gs), total);
#pragma unroll
            for (int i = 0; i < R::N; ++i)
                if (m[i] > 0.0f) d[i] += over(n[i], total) * rest[i] * (g[i] - m[i] * gs);
        }
        if (t < a.n_tokens) R::store(out + t * a.ldg, d, lane, E);
    }
}

template <int EL, int L, int NV> void balance_with(const RouterLaunch &a, hipStream_t st) {
    // a workgroup for every 16 waves with two rounds of tokens
    const int64_t groups = std::max<int64_t>(1, std::min<int64_t>(kBalanceGroups, ceil_div(a.n_tokens, 2 * 16 * (64 / L))));
    hipLaunchKernelGGL((k_balance<EL, L, NV>), dim3((unsigned)groups), dim3(1024), 0, st, a);
    if (groups > 1) hipLaunchKernelGGL(k_balance_finish, dim3(1), dim3(1024), 0, st, a, (int)groups);
}
template <int EL, int L, int NV> void grad_with(const RouterLaunch &a, hipStream_t st) {
    const int64_t groups = std::min<int64_t>(2048, ceil_div(a.n_tokens, 4 * (64 / L)));
    hipLaunchKernelGGL((k_route_grad<EL, L, NV>), dim3((unsigned)groups), dim3(256), 0, st, a);
}
template <int EL, bool GRAD> void router_el(const RouterLaunch &a, hipStream_t st) {
    const int chunks = (int)ceil_div(a.n_experts, EL == TF_F32 ? 4 : 8);
#define TF_ROW(L, NV) return GRAD ? grad_with<EL, L, NV>(a, st) : balance_with<EL, L, NV>(a, st)
    if (chunks <= 8) TF_ROW(8, 1);
    if (chunks <= 16) TF_ROW(16, 1);
    if (chunks <= 32) TF_ROW(32, 1);
    if (chunks <= 64) TF_ROW(64, 1);
    if constexpr (EL == TF_F32) {
        if (chunks <= 128) TF_ROW(64, 2);
        TF_ROW(64, 4);
    } else {
        TF_ROW(64, 2);
    }
#undef TF_ROW
}
template <bool GRAD> int router(const RouterLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.dtype == TF_BF16) router_el<TF_BF16, GRAD>(a, st);
    else if (a.dtype == TF_F16) router_el<TF_F16, GRAD>(a, st);
    else router_el<TF_F32, GRAD>(a, st);
    return (int)hipGetLastError();
}

}  // namespace

int launch_balance(const RouterLaunch &a, void *stream) { return router<false>(a, stream); }
int launch_route_grad(const RouterLaunch &a, void *stream) { return router<true>(a, stream); }

}  // namespace tf
