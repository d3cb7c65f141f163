// Router: counts and mass of the experts, the balance loss, and the gradient of the scores.
#include <algorithm>

#include "tf_loss.h"
#include "tf_moe_device.h"

namespace tf {
namespace {

constexpr float kLow = -__builtin_inff();
typedef int Int4 __attribute__((ext_vector_type(4)));
typedef double Double4 __attribute__((ext_vector_type(4)));

// Sums and maxima over 2, 4, 8 or 16 neighbouring lanes take one instruction for each doubling (the neighbours' values come with it: lane ^ 1,
// lane ^ 2, then mirror images of eight and sixteen lanes); 32 and 64 lanes exchange rows of sixteen and halves.
template <int CONTROL> __device__ __forceinline__ float from_lane(float x) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), CONTROL, 0xf, 0xf, true));
}
struct Plus {
    static __device__ __forceinline__ float of(float x, float y) { return x + y; }
};
struct Larger {
    static __device__ __forceinline__ float of(float x, float y) { return fmaxf(x, y); }
};
template <int L, typename F> __device__ __forceinline__ float over_lanes(float x) {
    if constexpr (L >= 2) x = F::of(x, from_lane<0xb1>(x));
    if constexpr (L >= 4) x = F::of(x, from_lane<0x4e>(x));
    if constexpr (L >= 8) x = F::of(x, from_lane<0x141>(x));
    if constexpr (L >= 16) x = F::of(x, from_lane<0x140>(x));
    if constexpr (L >= 32) {
        const uint32_t u = __float_as_uint(x);
        const auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = F::of(__uint_as_float(y[0]), __uint_as_float(y[1]));
    }
    if constexpr (L >= 64) {
        const uint32_t u = __float_as_uint(x);
        const auto y = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = F::of(__uint_as_float(y[0]), __uint_as_float(y[1]));
    }
    return x;
}

// The sum over the lanes that are a multiple of L apart: rotations of sixteen lanes, then rows and halves as above.
template <int L> __device__ __forceinline__ float over_groups(float x) {
    if constexpr (L <= 8) x += from_lane<0x128>(x);
    if constexpr (L <= 4) x += from_lane<0x124>(x);
    if constexpr (L <= 2) x += from_lane<0x122>(x);
    if constexpr (L <= 1) x += from_lane<0x121>(x);
    if constexpr (L <= 16) {
        const uint32_t u = __float_as_uint(x);
        const auto y = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    if constexpr (L <= 32) {
        const uint32_t u = __float_as_uint(x);
        const auto y = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        x = __uint_as_float(y[0]) + __uint_as_float(y[1]);
    }
    return x;
}

// A row of scores lies in L lanes; lane i of them holds NV chunks of sixteen bytes, chunk i + L c: VEC consecutive experts each.
template <int EL, int L, int NV> struct Row {
    static constexpr int VEC = EL == TF_F32 ? 4 : 8, N = VEC * NV, LANES = L, ROWS = 64 / L;
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
            else if constexpr (EL == TF_BF16) x = i & 1 ? bf16_high(r.c[i / VEC][i % VEC / 2]) : bf16_low(r.c[i / VEC][i % VEC / 2]);
            else x = El<EL>::get((uint16_t)(r.c[i / VEC][i % VEC / 2] >> (16 * (i & 1))));
            l[i] = __builtin_isnan(x) ? kLow : x;
        }
        if (n_experts < L * N)
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (expert(lane, i) >= n_experts) l[i] = kLow;
    }
    static __device__ __forceinline__ void store_chunk(T *row, const float (&d)[VEC], int c, int lane, int n_experts) {
        const int e = expert(lane, c * VEC);
        AnyWords4 w{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < VEC; ++j) put(w, j, El<EL>::put(d[j]));
        if (e + VEC <= n_experts) {
            *reinterpret_cast<AnyWords4 *>(row + e) = w;
        } else if (e < n_experts) {
#pragma unroll
            for (int j = 0; j < VEC; ++j)
                if (e + j < n_experts) row[e + j] = El<EL>::put(d[j]);
        }
    }
    static __device__ __forceinline__ float sum(float x) { return over_lanes<L, Plus>(x); }
    static __device__ __forceinline__ float max(float x) { return over_lanes<L, Larger>(x); }
    // Whether it is true in any of the row's lanes.
    static __device__ __forceinline__ bool any(bool x) {
        const uint64_t b = __ballot(x) >> (threadIdx.x & 63 & ~(L - 1));
        return L == 64 ? b != 0 : (b & (((uint64_t)1 << (L & 63)) - 1)) != 0;
    }
};

// Exponentials are powers of two: exp(x) = 2^(x log2(e)), one instruction after a multiplication that is off by 2^-24 of x.
constexpr float kLog2E = 1.44269504088896340736f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2E); }

// What sigmoids need of a score: sigma = 1 / (1 + exp(-l)) and sigma (1 - sigma), neither of which overflows or cancels.  (The reciprocal is
// good to a unit of 2^-23.)
__device__ __forceinline__ void sigmoid(float l, float &s, float &slope) {
    const float t = exp_of(-fabsf(l)), r = __builtin_amdgcn_rcpf(1.0f + t), tr = t * r;
    s = l >= 0.0f ? r : tr;
    slope = r * tr;
}

// Shares are n_e / sum n with numerators n_e = exp(l_e - top), top the row's largest score, or sigma(l_e).  Where the latter are all so small that their
// sum says little (scores below -40), and where a bias has selected experts whose numerators are that small, they are taken again over the
// exponential of the largest score that counts: exp(min(l, 0) - top) / (1 + exp(-|l|)), and `slope`, sigma (1 - sigma), likewise.
constexpr float kSmall = 1e-17f;
template <bool SIGMOIDS> __device__ __forceinline__ float bounded(float l) { return SIGMOIDS ? fminf(l, 0.0f) : l; }
template <bool SIGMOIDS> __device__ __forceinline__ void numerator_over(float l, float top, float &n, float &slope) {
    const float r = SIGMOIDS ? __builtin_amdgcn_rcpf(1.0f + exp_of(-fabsf(l))) : 1.0f;
    n = l > kLow ? exp_of(bounded<SIGMOIDS>(l) - top) * r : 0.0f;
    slope = SIGMOIDS ? n * exp_of(fminf(-l, 0.0f)) * r : n;
}
// Numerators of all of a row's scores, their slopes, their sum, and whether they are over an exponential.  (The scores are taken from their chunks again where they are needed again:
// registers are what limits the number of waves.)
template <typename R, bool SIGMOIDS>
__device__ __forceinline__ float numerators(float (&n)[R::N], float (&slope)[R::N], const typename R::Raw &raw, int lane, int n_experts, bool &scaled) {
    float total = 0.0f, l[R::N];
    scaled = false;
    R::unpack(l, raw, lane, n_experts);
    if constexpr (SIGMOIDS) {
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            sigmoid(l[i], n[i], slope[i]);
            total += n[i];
        }
        total = R::sum(total);
        scaled = total < kSmall;
        if (__ballot(scaled)) {
            float top = kLow;
            R::unpack(l, raw, lane, n_experts);
#pragma unroll
            for (int i = 0; i < R::N; ++i) top = fmaxf(top, fminf(l[i], 0.0f));
            top = R::max(top);
            float again = 0.0f;
#pragma unroll
            for (int i = 0; i < R::N; ++i) {
                float x, y;
                numerator_over<true>(l[i], top, x, y);
                again += x;
                n[i] = scaled ? x : n[i];
                slope[i] = scaled ? y : slope[i];
            }
            again = R::sum(again);
            total = scaled ? again : total;
        }
    } else {
        float top = kLow;
#pragma unroll
        for (int i = 0; i < R::N; ++i) top = fmaxf(top, l[i]);
        top = R::max(top);
        const float from = top > kLow ? top : 0.0f;
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            n[i] = slope[i] = exp_of(l[i] - from);
            total += n[i];
        }
        total = R::sum(total);
    }
    return total;
}

__device__ __forceinline__ float over(float x, float total) { return total == 0.0f ? 0.0f : x / total; }
// 1 / total, good to a unit of 2^-23: a division is a dozen instructions, of which a row of gradients takes two.
__device__ __forceinline__ float inverse(float total) { return total == 0.0f ? 0.0f : __builtin_amdgcn_rcpf(total); }

// ---------------------------------------------------------------------------------------- balance

// The end of it: thread e has the sum of expert e's shares and its count, `rows` are the rows of this thread's.  loss = E sum_e f_e mass_e.
template <typename T> __device__ __forceinline__ T wave_total(T x) {
#pragma unroll
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d, 64);
    return x;
}
__device__ void write_balance(const RouterLaunch &a, double m, int c, int rows) {
    __shared__ double part[16];
    __shared__ int named_of[16], rows_of[16];
    const int E = a.n_experts, tid = threadIdx.x;
    const double x = wave_total(m * c);
    const int named = wave_total(c), r = wave_total(rows);
    if ((tid & 63) == 0) {
        part[tid >> 6] = x;
        named_of[tid >> 6] = named;
        rows_of[tid >> 6] = r;
    }
    __syncthreads();
    double sum = 0.0;
    int n = 0, all = 0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) {
        sum += part[w];
        all += named_of[w];
        n += rows_of[w];
    }
    if (tid < E) {
        a.counts[tid] = c;
        a.mass[tid] = n ? (float)(m / n) : 0.0f;
    }
    if (tid == 0) {
        a.counts[E] = n;
        a.loss[0] = n ? (float)(E * sum / ((double)all * n)) : 0.0f;
    }
}

// Adds up the sums of `groups` workgroups in a fixed order: 1024 threads, each four experts and every (1024 / (experts / 4))-th workgroup.  256 of 256 experts: 9 us,
// a launch and three trips to memory.  (A last workgroup of the launch before would need a counter that somebody clears, and the workspace is the caller's.)
__global__ __launch_bounds__(1024) void k_balance_finish(const RouterLaunch a, const int groups) {
    __shared__ Double4 masses[1024];
    __shared__ Int4 counts[1024];
    const int tid = threadIdx.x, fours = balance_row(a.n_experts) / 4, slices = min(1024 / fours, 16);
    const Float4 *mass = static_cast<const Float4 *>(a.workspace);
    const Int4 *count = reinterpret_cast<const Int4 *>(mass + (int64_t)kBalanceGroups * fours);
    const int *rows = reinterpret_cast<const int *>(count + (int64_t)kBalanceGroups * fours);
    Double4 m = {0, 0, 0, 0};
    Int4 c = {0, 0, 0, 0};
    if (tid < slices * fours) {
        const int e = tid % fours;
#pragma unroll 8
        for (int g = tid / fours; g < groups; g += slices) {
            m += __builtin_convertvector(mass[g * fours + e], Double4);
            c += count[g * fours + e];
        }
    }
    const int r = tid < groups ? rows[tid] : 0;
    masses[tid] = m;
    counts[tid] = c;
    __syncthreads();
    double me = 0.0;
    int ce = 0;
    if (tid < a.n_experts)
        for (int s = 0; s < slices; ++s) {
            me += masses[s * fours + tid / 4][tid % 4];
            ce += counts[s * fours + tid / 4][tid % 4];
        }
    write_balance(a, me, ce, r);
}

// What a row needs from memory: its scores, and of its entries first, first + L, ... (kEntries of them at a time) the columns and, with GRADIENTS, the
// gradients of their values.
constexpr int kEntries = 4;
template <typename R, bool GRADIENTS> struct Input {
    typename R::Raw raw;
    int c[kEntries];
    float x[kEntries];
    __device__ __forceinline__ void entries(const RouterLaunch &a, int64_t t, int first, int at) {
#pragma unroll
        for (int j = 0; j < kEntries; ++j) {
            c[j] = -1;
            if (first + j * R::LANES >= a.k) break;        // (the same for all lanes)
            const int i = first + j * R::LANES + at;
            if (t < a.n_tokens && i < a.k) {
                c[j] = a.colidx[t * a.k + i];
                if (GRADIENTS && a.dvals) x[j] = a.dvals[t * a.k + i];
            }
        }
    }
    __device__ __forceinline__ void load(const RouterLaunch &a, int64_t t, int lane) {
        if (t < a.n_tokens) R::load(raw, static_cast<const typename R::T *>(a.scores) + t * a.ld, lane, a.n_experts);
        entries(a, t, 0, lane & (R::LANES - 1));
    }
    __device__ __forceinline__ bool is(const RouterLaunch &a, int j) const { return c[j] >= 0 && c[j] < a.n_experts; }
};

// mass_e = sum over rows of n_te / sum_j n_tj.  Every wave takes ROWS tokens at a time and adds up their shares in registers; entries are counted in LDS
// (whole numbers: their order does not matter).  In 32 bits a lane adds up kSteps rows at most, in 64 what those come to; its own sum and a workgroup's
// are rounded once, so that what mass is off by does not grow with the number of rows.  LDS holds the counts, the lanes' sums in 64 bits (registers have
// no room for them) and at the end, in their place, a line of sums for each wave.  Two sets of rows are on their way from memory while a third is
// worked on.  131072 rows of 256 bf16 experts, 8 entries each: 20 us, 3.6 TB/s (the launch after it 9); sigmoids 25.  Of 1 Mi rows 120 to 125 us,
// 4.6 TB/s: bound by its instructions, an exponential and about ten others a score.
constexpr int kSteps = 8;
template <int EL, int L, int NV, bool SIGMOIDS> __global__ __launch_bounds__(1024) void k_balance(const RouterLaunch a) {
    typedef Row<EL, L, NV> R;
    extern __shared__ __attribute__((aligned(16))) int shared[];
    const int E = a.n_experts, line = balance_row(E), lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    int *counted = shared, *rows_of = shared + line;
    float *masses = reinterpret_cast<float *>(shared + line + 16);
    const int sub = lane / L, at = lane & (L - 1);
    for (int e = threadIdx.x; e < line; e += blockDim.x) counted[e] = 0;
    __syncthreads();
    double *before = reinterpret_cast<double *>(masses) + threadIdx.x;       // blockDim.x apart
    float mass[R::N] = {};
    int rows = 0;
    const int64_t step = (int64_t)gridDim.x * waves * R::ROWS;
    int64_t t = ((int64_t)blockIdx.x * waves + wave) * R::ROWS + sub;
    Input<R, false> in[2];
    in[0].load(a, t, lane);
    in[1].load(a, t + step, lane);
    auto row = [&](Input<R, false> &in) {
        const typename R::Raw raw = in.raw;
        bool named = false;
        for (int first = 0;;) {
#pragma unroll
            for (int j = 0; j < kEntries; ++j) {
                if (first + j * L >= a.k) break;
                if (in.is(a, j)) {
                    named = true;
                    atomicAdd(counted + in.c[j], 1);
                }
            }
            first += kEntries * L;
            if (first >= a.k) break;
            in.entries(a, t, first, at);
        }
        in.load(a, t + 2 * step, lane);
        named = R::any(named);
        rows += named;
        float n[R::N], slope[R::N];
        bool scaled;
        const float total = numerators<R, SIGMOIDS>(n, slope, raw, lane, E, scaled);
        const float each = named ? inverse(total) : 0.0f;
        if (named)
#pragma unroll
            for (int i = 0; i < R::N; ++i) mass[i] += n[i] * each;
    };
    int steps = 0;
    bool more = false;
    for (int64_t base = t - sub; base < a.n_tokens; base += 2 * step) {
        row(in[0]);
        t += step;
        if (base + step < a.n_tokens) row(in[1]);
        t += step;
        if ((steps += 2) == kSteps && base + 2 * step < a.n_tokens) {
#pragma unroll
            for (int i = 0; i < R::N; ++i) {
                double *to = before + i * blockDim.x;
                *to = more ? *to + mass[i] : mass[i];
                mass[i] = 0.0f;
            }
            more = true;
            steps = 0;
        }
    }
    // rows of a wave, then waves in their order
#pragma unroll
    for (int i = 0; i < R::N; ++i) mass[i] = over_groups<L>(more ? (float)(before[i * blockDim.x] + mass[i]) : mass[i]);
    rows = wave_total(at == 0 ? rows : 0);
    __syncthreads();
    if (sub == 0) {
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            const int e = R::expert(lane, i);
            if (e < E) masses[wave * line + e] = mass[i];
        }
        if (lane == 0) rows_of[wave] = rows;
    }
    __syncthreads();
    const int e = threadIdx.x;
    double m = 0.0;
    if (e < E)
        for (int w = 0; w < waves; ++w) m += masses[w * line + e];
    const int c = e < E ? counted[e] : 0, r = e < waves ? rows_of[e] : 0;
    if (gridDim.x == 1) return write_balance(a, m, c, r);
    float *out = static_cast<float *>(a.workspace);
    int *count = reinterpret_cast<int *>(out + (int64_t)kBalanceGroups * line);
    if (e < line) {
        out[blockIdx.x * line + e] = (float)m;
        count[blockIdx.x * line + e] = c;
    }
    if (wave == 0) {
        const int all = wave_total(r);
        if (lane == 0) count[(int64_t)kBalanceGroups * line + blockIdx.x] = all;
    }
}

// --------------------------------------------------------------------------------------- gradient

// With q the shares (over all experts, or over the named ones) and n' the slopes of their numerators, every kind of gradient is
//     d_e = n'_e (A (f_e - sum_j p_j f_j) + B (g_e - m_e sum_j q_j g_j)),
// g_e the sum of the gradients of a row's entries that name e, m_e their number; A, B over the sums of the numerators.
// The entries of a row meet its scores in LDS: each puts its gradient and a one where its expert's are, and the lanes that hold the scores find
// them there, or zeros.  (They read them, and f, twice: registers hold two numbers a score and what comes from memory next.)  Where a row names an
// expert more than once one lane adds its entries up instead.  A wave has no barrier: its instructions of LDS are done in their order.
// 131072 rows of 256 bf16 experts, 8 entries each, both parts, sigmoid shares: 50 us, 2.8 TB/s; softmax 48.  Bound by its instructions: one or two of a quarter of
// the others' rate a score, and about twenty others.
__device__ __forceinline__ void in_order() { asm volatile("" ::: "memory"); }

template <int EL, int L, int NV, bool SIGMOIDS> __global__ __launch_bounds__(256, NV * (EL == TF_F32 ? 4 : 8) > 8 ? 2 : 4) void k_route_grad(const RouterLaunch a) {
    typedef Row<EL, L, NV> R;
    constexpr int VEC = R::VEC;
    __shared__ __attribute__((aligned(16))) Float2 places[4][64 * R::N];
    __shared__ __attribute__((aligned(16))) float named_share[L * R::N];
    const int E = a.n_experts, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sub = lane / L, at = lane & (L - 1);
    const bool top_only = a.scoring == TF_ROUTE_SOFTMAX_TOP || a.scoring == TF_ROUTE_SIGMOID_TOP, sigmoid_only = a.scoring == TF_ROUTE_SIGMOID;
    Float2 *own = places[wave] + sub * L * R::N;       // of this lane's row
#pragma unroll
    for (int i = 0; i < R::N; ++i) places[wave][i * 64 + lane] = Float2{0.0f, 0.0f};
    // f: shares of the entries that name an expert; and what a share's gradient is multiplied by
    float factor = 0.0f;
    {
        float f[R::N], named = 0.0f;
#pragma unroll
        for (int i = 0; i < R::N; ++i) {
            const int e = R::expert(lane, i);
            f[i] = a.dloss && e < E ? (float)a.counts[e] : 0.0f;
            named += f[i];
        }
        named = over(1.0f, R::sum(named));
        if (threadIdx.x < L)
#pragma unroll
            for (int i = 0; i < R::N; ++i) named_share[R::expert(lane, i)] = f[i] * named;
        if (a.dloss) factor = over(a.dloss[0] * (float)E, (float)a.counts[E]);
    }
    __syncthreads();
    const int64_t step = (int64_t)gridDim.x * 4 * R::ROWS;
    int64_t t = ((int64_t)blockIdx.x * 4 + wave) * R::ROWS + sub;
    // four consecutive experts' f, g and m
    auto f_of = [&](int i) { return *reinterpret_cast<const Float4 *>(named_share + R::expert(lane, i)); };
    auto gm_of = [&](int i, Float4 &g, Float4 &m) {
        const Float4 *w = reinterpret_cast<const Float4 *>(own + R::expert(lane, i));
        const Float4 x = w[0], y = w[1];
        g = Float4{x[0], x[2], y[0], y[2]};
        m = Float4{x[1], x[3], y[1], y[3]};
    };
    Input<R, true> in[2];
    in[0].load(a, t, lane);
    in[1].load(a, t + step, lane);
    auto row = [&](Input<R, true> &in) {
        typename R::Raw raw = in.raw;
        bool named = false, twice = false;
        for (int first = 0;;) {
#pragma unroll
            for (int j = 0; j < kEntries; ++j) {
                if (first + j * L >= a.k) break;
                const bool is = in.is(a, j);
                named |= is;
                // whoever finds another one's number where it has left its own shares an expert with it
                if (a.dvals && is) {
                    Float2 *place = own + in.c[j];
                    const float number = (float)(first + j * L + at + 1);
                    twice |= (*place)[1] != 0.0f;
                    (*place)[1] = number;
                    in_order();
                    twice |= (*place)[1] != number;
                    in_order();
                    *place = Float2{in.x[j] * a.scale, 1.0f};
                }
            }
            if (first + kEntries * L >= a.k) break;
            first += kEntries * L;
            in.entries(a, t, first, at);
        }
        named = R::any(named);
        // clears the places again, or (`sums`) adds the entries up one after the other
        auto each_entry = [&](bool sums) {
            for (int i = sums ? at ? a.k : 0 : at; i < a.k; i += sums ? 1 : L) {
                const int c = t < a.n_tokens ? a.colidx[t * a.k + i] : -1;
                if (c >= 0 && c < E) own[c] = sums ? own[c] + Float2{a.dvals[t * a.k + i] * a.scale, 1.0f} : Float2{0.0f, 0.0f};
            }
        };
        in_order();
        if (__ballot(twice) && R::any(twice)) {
            each_entry(false);
            in_order();
            each_entry(true);
        }
        in_order();
        // (a row without an entry gets zeros whatever its scores are: a softmax of +inf is NaN, which no factor of zero takes away)
        if (__ballot(!named))
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int w = 0; w < 4; ++w) raw.c[c][w] = named ? raw.c[c][w] : 0u;
        float n[R::N], slope[R::N];
        bool scaled;
        const float total = numerators<R, SIGMOIDS>(n, slope, raw, lane, E, scaled);
        const float over_all = named ? inverse(total) : 0.0f;
        float fs = 0.0f, gs = 0.0f, some = 0.0f;
        if (a.dloss) {
#pragma unroll
            for (int i = 0; i < R::N; i += 4) {
                const Float4 f = f_of(i);
#pragma unroll
                for (int j = 0; j < 4; ++j) fs += n[i + j] * f[j];
            }
            fs = R::sum(fs) * over_all;
        }
        if (a.dvals) {
#pragma unroll
            for (int i = 0; i < R::N; i += 4) {
                Float4 g, m;
                gm_of(i, g, m);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    gs += n[i + j] * g[j];
                    some += n[i + j] * m[j];
                }
            }
            gs = R::sum(gs);
            some = R::sum(some);
        }
        // (`again`: numerators that say little; with plain sigmoids, slopes that are over an exponential)
        const bool again = a.dvals && named && (top_only ? some < kSmall : sigmoid_only && scaled);
        const float A = named ? factor * over_all : 0.0f, B = !a.dvals ? 0.0f : sigmoid_only ? 1.0f : top_only ? inverse(some) : over_all;
        gs *= sigmoid_only ? 0.0f : B;
        // what is taken off: A sum p f, B sum q g for the experts that are named or, with shares over all experts, for all of them
        const float Afs = A * fs, Bgs = B * gs, off = Afs + (top_only ? 0.0f : Bgs), off_named = top_only ? Bgs : 0.0f;
        in_order();
        const bool store = t < a.n_tokens;
        typename R::T *out = static_cast<typename R::T *>(a.dscores) + t * a.ldg;
        const bool any_again = __ballot(again) != 0;
        float top = 0.0f, gs2 = 0.0f, over2 = 1.0f;
        if (any_again) {
            // The second term once more, over the exponential of the largest score that is named, or of nothing.
            float l[R::N], sum2 = 0.0f;
            R::unpack(l, raw, lane, E);
            if (top_only) {
                top = kLow;
#pragma unroll
                for (int i = 0; i < R::N; ++i)
                    if (own[R::expert(lane, i)][1] > 0.0f) top = fmaxf(top, bounded<SIGMOIDS>(l[i]));
                top = R::max(top);
            }
#pragma unroll
            for (int i = 0; i < R::N; ++i) {
                const Float2 w = own[R::expert(lane, i)];
                float x, y;
                numerator_over<SIGMOIDS>(l[i], top, x, y);
                if (w[1] > 0.0f) {
                    sum2 += w[1] * x;
                    gs2 += w[0] * x;
                }
            }
            sum2 = R::sum(sum2);
            gs2 = R::sum(gs2);
            if (top_only) over2 = over(1.0f, sum2);
            gs2 = top_only ? gs2 * over2 : 0.0f;
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            float d[VEC];
#pragma unroll
            for (int i = c * VEC; i < (c + 1) * VEC; i += 4) {
                const Float4 f = f_of(i);
                Float4 g, m;
                gm_of(i, g, m);
#pragma unroll
                for (int j = 0; j < 4; ++j) d[i - c * VEC + j] = slope[i + j] * (A * f[j] + (B * g[j] - (off_named * m[j] + off)));
            }
            if (any_again) {
                float l[R::N];
                R::unpack(l, raw, lane, E);
#pragma unroll
                for (int i = c * VEC; i < (c + 1) * VEC; ++i) {
                    const Float2 w = own[R::expert(lane, i)];
                    float x, y;
                    numerator_over<SIGMOIDS>(l[i], top, x, y);
                    const float z = slope[i] * (A * named_share[R::expert(lane, i)] - Afs) + (w[1] > 0.0f ? y * over2 * (w[0] - w[1] * gs2) : 0.0f);
                    if (again) d[i - c * VEC] = z;
                }
            }
            if (store) R::store_chunk(out, d, c, lane, E);
        }
        in_order();
        if (a.dvals) each_entry(false);
        in_order();
        in.load(a, t + 2 * step, lane);
    };
    for (int64_t base = t - sub; base < a.n_tokens; base += 2 * step) {
        row(in[0]);
        t += step;
        if (base + step < a.n_tokens) row(in[1]);
        t += step;
    }
}

// Few scores: one workgroup, and one launch.  Otherwise workgroups of four waves, one or two steps of tokens each, or of sixteen.  (A thread for each
// expert at the least.)
template <int EL, int L, int NV, bool SIGMOIDS> int balance_of(const RouterLaunch &a, hipStream_t st) {
    const int64_t sets = ceil_div(a.n_tokens, 64 / L);
    const bool few = (int64_t)a.n_tokens * a.n_experts <= 16384;
    const int waves = a.n_experts <= 256 && (few ? sets <= 8 : sets <= 8 * kBalanceGroups) ? 4 : 16;
    const int64_t groups = few ? 1 : std::min<int64_t>(kBalanceGroups, ceil_div(sets, waves));
    const bool many = sets > groups * waves * kSteps;       // of a lane's rows
    const int line = balance_row(a.n_experts), sums = Row<EL, L, NV>::N * waves * 64 * 8;
    const int lds = (line + 16) * 4 + std::max(line * waves * 4, many ? sums : 0);
    if (lds > 65536) {
        static DoneOnDevices done;
        int device = 0;
        hipError_t e = hipGetDevice(&device);
        if (e != hipSuccess) return (int)e;
        if (!done.has(device)) {
            e = hipFuncSetAttribute(reinterpret_cast<const void *>(k_balance<EL, L, NV, SIGMOIDS>), hipFuncAttributeMaxDynamicSharedMemorySize, 4096 + 64 + 16 * 8192);
            if (e != hipSuccess) return (int)e;
            done.add(device);
        }
    }
    hipLaunchKernelGGL((k_balance<EL, L, NV, SIGMOIDS>), dim3((unsigned)groups), dim3(64 * waves), lds, st, a);
    if (groups > 1) hipLaunchKernelGGL(k_balance_finish, dim3(1), dim3(1024), 0, st, a, (int)groups);
    return (int)hipGetLastError();
}
template <int EL, int L, int NV> int balance_with(const RouterLaunch &a, hipStream_t st) {
    return a.scoring >= TF_ROUTE_SIGMOID ? balance_of<EL, L, NV, true>(a, st) : balance_of<EL, L, NV, false>(a, st);
}
template <int EL, int L, int NV> int grad_with(const RouterLaunch &a, hipStream_t st) {
    const dim3 grid((unsigned)std::min<int64_t>(2048, ceil_div(a.n_tokens, 4 * (64 / L)))), block(256);
    if (a.scoring >= TF_ROUTE_SIGMOID) hipLaunchKernelGGL((k_route_grad<EL, L, NV, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_route_grad<EL, L, NV, false>), grid, block, 0, st, a);
    return (int)hipGetLastError();
}
// Sixteen experts a lane (eight for the gradient, which holds more of each, while there are lanes for that), in as few lanes as they need: what goes on
// between lanes is then shared by as many rows as there can be.
// Balance with 16 / 8 a lane, us: 131072 rows of 256 bf16 experts 27.6 / 32.1, 1 Mi rows 128 / 176 (fp32, 131072 rows: 36 / 36).  Gradient with 8 / 16: 32768 rows
// 19.7 / 26.6, 131072 rows 47 / 50, 1 Mi rows 356 / 314 (fp32, 131072 rows: 58 / 58).
template <int EL, bool GRAD> int router_el(const RouterLaunch &a, hipStream_t st) {
    constexpr int NV = (EL == TF_F32 ? 4 : 2) / (GRAD ? 2 : 1);
    const int lanes = (int)ceil_div(a.n_experts, GRAD ? 8 : 16);
#define TF_ROW(L, NV)                                            \
    {                                                            \
        if constexpr (GRAD) return grad_with<EL, L, NV>(a, st);  \
        else return balance_with<EL, L, NV>(a, st);              \
    }
    if (lanes <= 1) TF_ROW(1, NV)
    if (lanes <= 2) TF_ROW(2, NV)
    if (lanes <= 4) TF_ROW(4, NV)
    if (lanes <= 8) TF_ROW(8, NV)
    if (lanes <= 16) TF_ROW(16, NV)
    if (lanes <= 32) TF_ROW(32, NV)
    if (lanes <= 64) TF_ROW(64, NV)
    if constexpr (GRAD) return grad_with<EL, 64, 2 * NV>(a, st);
    else return (int)hipErrorInvalidValue;       // (not reached: 1024 experts at most)
#undef TF_ROW
}
template <bool GRAD> int router(const RouterLaunch &a, void *stream) {
    const hipStream_t st = static_cast<hipStream_t>(stream);
    return a.dtype == TF_BF16 ? router_el<TF_BF16, GRAD>(a, st) : a.dtype == TF_F16 ? router_el<TF_F16, GRAD>(a, st) : router_el<TF_F32, GRAD>(a, st);
}

}  // namespace

int launch_balance(const RouterLaunch &a, void *stream) { return router<false>(a, stream); }
int launch_route_grad(const RouterLaunch &a, void *stream) { return router<true>(a, stream); }

}  // namespace tf
