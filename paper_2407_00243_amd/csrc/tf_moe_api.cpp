// C ABI of the routed operators: argument checks, the plan's workspace, the launches of a call.
#include <hip/hip_runtime.h>

#include <new>

#include "tf_moe.h"

namespace {

using tf::report;
using tf::report_hip;

constexpr int64_t kMaxSize = ((int64_t)1 << 31) - 1;

bool routed_dtype(int32_t d) { return d == TF_F32 || d == TF_BF16 || d == TF_F16; }
int64_t bytes_of(int32_t d) { return d == TF_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }

tf_status check_q4_shape(const tf_q4 *W) {
    if (!W) return report(TF_EINVAL, "null argument");
    if (W->n_mats < 1 || W->n_rows < 1 || W->n_cols < 1) return report(TF_EINVAL, "a 4-bit matrix needs positive sizes");
    if (W->kind != TF_Q4_INT && W->kind != TF_Q4_E2M1) return report(TF_EINVAL, "unknown kind of 4-bit codes");
    if (W->group != 32 && W->group != 64 && W->group != 128) return report(TF_EINVAL, "group must be 32, 64 or 128");
    if (W->n_rows > kMaxSize / 4 || W->n_cols > kMaxSize / 4 || W->n_mats > kMaxSize / 4)
        return report(TF_EUNSUPPORTED, "4-bit matrix is too large");
    // (products of two sizes fit 64 bits; the third factor is checked against the address space)
    if (W->n_mats > ((int64_t)1 << 46) / (tf::q4_tiles(W->n_rows) * tf::q4_blocks(W->n_cols) * 1024 + 1))
        return report(TF_EUNSUPPORTED, "4-bit matrices are too large");
    return TF_OK;
}
tf_status check_q4(const tf_q4 *W) {
    const tf_status st = check_q4_shape(W);
    if (st != TF_OK) return st;
    if (!W->codes || !W->scales) return report(TF_EINVAL, "null argument");
    if (!aligned(W->codes, 16) || !aligned(W->scales, 16)) return report(TF_EINVAL, "codes and scales must be 16-byte aligned");
    return TF_OK;
}
tf::Q4Launch q4_args(const tf_q4 *W) {
    tf::Q4Launch a{};
    a.n_mats = W->n_mats;
    a.n_rows = W->n_rows;
    a.n_cols = W->n_cols;
    a.kind = W->kind;
    a.group = W->group;
    a.codes = W->codes;
    a.scales = W->scales;
    return a;
}
void set_q4(tf::ExpertLaunch &a, const tf_q4 *W) {
    a.W = W->codes;
    a.scales = W->scales;
    a.w_mat = tf::q4_code_bytes(W->n_rows, W->n_cols);
    a.s_mat = tf::q4_scale_bytes(W->n_rows, W->n_cols, W->group);
    a.kind = W->kind;
    a.group = W->group;
}

struct Buffer {
    void *p = nullptr;
    ~Buffer() {
        if (p) (void)hipFree(p);
    }
};

}  // namespace

struct tf_moe {
    tf_moe_desc d{};
    Buffer hidden;            // rows between the products, high parts and behind them the low ones
    Buffer sums;              // results of the second product, entry by entry
    Buffer arrived;           // a count for each block of columns of D
    int64_t hidden_part = 0;
};

namespace {

tf_status run_layer(const tf_moe *p, const tf_csr *A, const void *X, int64_t ldx, tf::ExpertLaunch first, tf::ExpertLaunch second,
                    void *D, int64_t ldd, void *stream) {
    const tf_moe_desc &d = p->d;
    if (A->n_rows == 0) return TF_OK;
    first.n_rows = (int32_t)d.n_hidden;
    first.n_cols = (int32_t)d.n_in;
    first.X = X;
    first.ldx = ldx;
    first.out_kind = tf::kOutHidden;
    first.activation = d.activation;
    first.gated = d.gated;
    first.out = p->hidden.p;
    first.ldo = tf::hidden_ld(d.n_hidden);
    first.out_part = p->hidden_part;
    second.n_rows = (int32_t)d.n_out;
    second.n_cols = (int32_t)d.n_hidden;
    second.X = p->hidden.p;
    second.ldx = tf::hidden_ld(d.n_hidden);
    second.x_hidden = 1;
    second.x_part = p->hidden_part;
    second.out = p->sums.p;
    second.ldo = d.n_out;
    second.vals = static_cast<const float *>(A->vals);
    second.D = D;
    second.ldd = ldd;
    second.arrived = static_cast<uint32_t *>(p->arrived.p);
    for (tf::ExpertLaunch *a : {&first, &second}) {
        a->dtype = d.dtype;
        a->rowptr = A->rowptr;
        a->colidx = A->colidx;
        a->n_tokens = (int32_t)A->n_rows;
        a->n_entries = (int32_t)A->nnz;
        a->n_experts = (int32_t)d.n_experts;
        if (A->nnz == 0 && a == &first) continue;        // (the second launch writes the zeros)
        const int e = tf::launch_experts(*a, stream);
        if (e) return report_hip(e, "launching the experts' products");
    }
    return TF_OK;
}

tf_status check_layer(const tf_moe *p, const tf_csr *A, const void *X, int64_t ldx, const void *W1, const void *W2, void *D, int64_t ldd) {
    if (!p || !A || !X || !W1 || !W2 || !D) return report(TF_EINVAL, "null argument");
    if (!A->rowptr || (A->nnz > 0 && (!A->colidx || !A->vals))) return report(TF_EINVAL, "null argument");
    if (!A->on_device) return report(TF_EINVAL, "A must be on the device");
    if (A->dtype != TF_F32) return report(TF_EMISMATCH, "the values of A must be fp32");
    if (A->n_cols != p->d.n_experts) return report(TF_EMISMATCH, "A does not have a column for each expert");
    if (A->n_rows < 0 || A->nnz < 0) return report(TF_EINVAL, "A has a negative size");
    if (A->n_rows > p->d.max_tokens || A->nnz > p->d.max_entries)
        return report(TF_EMISMATCH, "A has more rows or entries than the plan was made for");
    if (ldx < p->d.n_in || ldd < p->d.n_out) return report(TF_EINVAL, "rows of X or D are closer together than they are wide");
    const int64_t es = bytes_of(p->d.dtype);
    if (!aligned(X, es) || !aligned(D, es)) return report(TF_EINVAL, "X and D must be aligned to their elements");
    return TF_OK;
}

}  // namespace

namespace tf {
int launch_experts(const ExpertLaunch &a, void *stream) {
    return a.dtype == TF_BF16 ? launch_experts_bf16(a, stream)
                              : a.dtype == TF_F16 ? launch_experts_f16(a, stream) : launch_experts_f32(a, stream);
}
}  // namespace tf

extern "C" {

tf_status tf_q4_sizes(const tf_q4 *W, int64_t *codes_bytes, int64_t *scales_bytes) {
    if (!codes_bytes || !scales_bytes) return report(TF_EINVAL, "null argument");
    const tf_status st = check_q4_shape(W);
    if (st != TF_OK) return st;
    *codes_bytes = W->n_mats * tf::q4_code_bytes(W->n_rows, W->n_cols);
    *scales_bytes = W->n_mats * tf::q4_scale_bytes(W->n_rows, W->n_cols, W->group);
    return TF_OK;
}

tf_status tf_q4_pack(const tf_q4 *W, const int8_t *codes, const void *scales, void *stream) {
    const tf_status st = check_q4(W);
    if (st != TF_OK) return st;
    if (!codes || !scales) return report(TF_EINVAL, "null argument");
    if (!aligned(scales, 2)) return report(TF_EINVAL, "scales must be aligned to their elements");
    const hipStream_t s = static_cast<hipStream_t>(stream);
    Buffer bad;
    int32_t flag = 0;
    hipError_t e = hipMalloc(&bad.p, sizeof(flag));
    if (e == hipSuccess) e = hipMemcpyAsync(bad.p, &flag, sizeof(flag), hipMemcpyHostToDevice, s);
    if (e != hipSuccess) return report_hip(e, "setting up the check of the codes");
    tf::Q4Launch a = q4_args(W);
    a.src_codes = codes;
    a.src_scales = scales;
    a.bad = static_cast<int32_t *>(bad.p);
    const int le = tf::launch_q4_pack(a, stream);
    if (le) return report_hip(le, "launching the packing of codes");
    e = hipMemcpyAsync(&flag, bad.p, sizeof(flag), hipMemcpyDeviceToHost, s);
    if (e == hipSuccess) e = hipStreamSynchronize(s);
    if (e != hipSuccess) return report_hip(e, "packing codes");
    return flag ? report(TF_EINVAL, "a code is outside of its kind's range") : TF_OK;
}

tf_status tf_q4_quantize(const tf_q4 *W, const void *weights, int32_t dtype, void *stream) {
    const tf_status st = check_q4(W);
    if (st != TF_OK) return st;
    if (!weights) return report(TF_EINVAL, "null argument");
    if (!routed_dtype(dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (!aligned(weights, bytes_of(dtype))) return report(TF_EINVAL, "weights must be aligned to their elements");
    tf::Q4Launch a = q4_args(W);
    a.weights = const_cast<void *>(weights);
    a.dtype = dtype;
    const int e = tf::launch_q4_quantize(a, stream);
    return e ? report_hip(e, "launching the quantisation") : TF_OK;
}

tf_status tf_q4_unpack(const tf_q4 *W, int32_t dtype, void *weights, void *stream) {
    const tf_status st = check_q4(W);
    if (st != TF_OK) return st;
    if (!weights) return report(TF_EINVAL, "null argument");
    if (!routed_dtype(dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (!aligned(weights, bytes_of(dtype))) return report(TF_EINVAL, "weights must be aligned to their elements");
    tf::Q4Launch a = q4_args(W);
    a.weights = weights;
    a.dtype = dtype;
    const int e = tf::launch_q4_unpack(a, stream);
    return e ? report_hip(e, "launching the unpacking of codes") : TF_OK;
}

tf_status tf_q4_matvec(const tf_q4 *W, const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t m, int32_t dtype, void *stream) {
    const tf_status st = check_q4(W);
    if (st != TF_OK) return st;
    if (W->n_mats != 1) return report(TF_EMISMATCH, "a product takes one 4-bit matrix");
    if (W->n_cols > tf::kMaxColumns) return report(TF_EUNSUPPORTED, "weights have rows of at most 2^24 columns");
    if (!routed_dtype(dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (m < 0 || m > kMaxSize) return report(TF_EINVAL, "number of rows");
    if (m == 0) return TF_OK;
    if (!X || !Y) return report(TF_EINVAL, "null argument");
    if (ldx < W->n_cols || ldy < W->n_rows) return report(TF_EINVAL, "rows of X or Y are closer together than they are wide");
    const int64_t es = bytes_of(dtype);
    if (!aligned(X, es) || !aligned(Y, es)) return report(TF_EINVAL, "X and Y must be aligned to their elements");
    tf::ExpertLaunch a{};
    set_q4(a, W);
    a.n_rows = (int32_t)W->n_rows;
    a.n_cols = (int32_t)W->n_cols;
    a.dtype = dtype;
    a.X = X;
    a.ldx = ldx;
    a.n_tokens = a.n_entries = (int32_t)m;
    a.n_experts = 1;
    a.out_kind = tf::kOutRows;
    a.out = Y;
    a.ldo = ldy;
    const int e = tf::launch_experts(a, stream);
    return e ? report_hip(e, "launching the 4-bit product") : TF_OK;
}

tf_status tf_moe_route(const void *scores, int64_t ld, int32_t dtype, const float *bias, int32_t scoring, float scale, const tf_csr *A,
                       void *stream) {
    if (!A) return report(TF_EINVAL, "null argument");
    if (!A->on_device) return report(TF_EINVAL, "A must be on the device");
    if (!routed_dtype(dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (A->dtype != TF_F32) return report(TF_EMISMATCH, "the values of A must be fp32");
    if (scoring < TF_ROUTE_SOFTMAX || scoring > TF_ROUTE_SIGMOID_TOP) return report(TF_EINVAL, "unknown scoring");
    if (A->n_rows < 0 || A->n_cols < 1 || A->nnz < 0) return report(TF_EINVAL, "A has a size that is not positive");
    if (A->n_rows == 0) return TF_OK;
    if (!scores || !A->rowptr || !A->colidx || !A->vals) return report(TF_EINVAL, "null argument");
    if (A->nnz % A->n_rows || A->nnz < A->n_rows) return report(TF_EINVAL, "A must have the same positive number of entries in each row");
    const int64_t k = A->nnz / A->n_rows;
    if (A->n_cols > tf::kRouteMaxExperts || k > tf::kRouteMaxK) return report(TF_EUNSUPPORTED, "at most 1024 experts and 64 entries in a row");
    if (k > A->n_cols) return report(TF_EINVAL, "more entries in a row than there are experts");
    if (A->nnz > kMaxSize || A->n_rows >= kMaxSize) return report(TF_EUNSUPPORTED, "A has too many entries");
    if (ld < A->n_cols) return report(TF_EINVAL, "rows of the scores are closer together than they are wide");
    if (!aligned(scores, bytes_of(dtype)) || !aligned(bias, 4) || !aligned(A->rowptr, 4) || !aligned(A->colidx, 4) || !aligned(A->vals, 4))
        return report(TF_EINVAL, "arrays must be aligned to their elements");
    tf::RouteLaunch a{};
    a.scores = scores;
    a.ld = ld;
    a.bias = bias;
    a.rowptr = const_cast<int32_t *>(A->rowptr);
    a.colidx = const_cast<int32_t *>(A->colidx);
    a.vals = static_cast<float *>(const_cast<void *>(A->vals));
    a.n_tokens = (int32_t)A->n_rows;
    a.n_experts = (int32_t)A->n_cols;
    a.k = (int32_t)k;
    a.dtype = dtype;
    a.scoring = scoring;
    a.scale = scale;
    const int e = tf::launch_route(a, stream);
    return e ? report_hip(e, "launching the router") : TF_OK;
}

tf_status tf_moe_create(const tf_moe_desc *desc, tf_moe **out) {
    if (!out) return report(TF_EINVAL, "null argument");
    *out = nullptr;
    if (!desc) return report(TF_EINVAL, "null argument");
    const tf_moe_desc &d = *desc;
    if (d.n_experts < 1 || d.n_in < 1 || d.n_hidden < 1 || d.n_out < 1 || d.max_tokens < 1 || d.max_entries < 1)
        return report(TF_EINVAL, "sizes must be positive");
    if (!routed_dtype(d.dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (d.activation < TF_ACT_IDENTITY || d.activation > TF_ACT_GELU) return report(TF_EINVAL, "unknown activation");
    if (d.gated != 0 && d.gated != 1) return report(TF_EINVAL, "gated must be 0 or 1");
    if (d.n_in > tf::kMaxColumns || d.n_hidden > tf::kMaxColumns) return report(TF_EUNSUPPORTED, "weights have rows of at most 2^24 columns");
    const int64_t most = kMaxSize / 4;
    if (d.n_experts > most || d.n_in > most || d.n_hidden > most || d.n_out > most || d.max_tokens > most || d.max_entries > most)
        return report(TF_EUNSUPPORTED, "a size is too large");
    // workgroups of a launch: blocks of rows times experts (or entries, if fewer)
    const int64_t units = d.max_entries < d.n_experts ? d.max_entries : d.n_experts;
    if (units > most / ((d.n_hidden + 15) / 16) || units > most / ((d.n_out + 15) / 16) || d.max_tokens > most / ((d.n_out + 255) / 256))
        return report(TF_EUNSUPPORTED, "a size is too large");
    tf_moe *p = new (std::nothrow) tf_moe;
    if (!p) return report(TF_ENOMEM, "out of host memory");
    p->d = d;
    const int64_t es = bytes_of(d.dtype), ld = tf::hidden_ld(d.n_hidden);
    hipError_t e = hipErrorOutOfMemory;
    if (d.max_entries <= ((int64_t)1 << 50) / (ld + d.n_out)) {
        p->hidden_part = d.max_entries * ld * es;
        const size_t hidden = (size_t)p->hidden_part * (d.dtype == TF_F32 ? 1 : 2);
        e = hipMalloc(&p->hidden.p, hidden);
        if (e == hipSuccess) e = hipMalloc(&p->sums.p, (size_t)(d.max_entries * d.n_out) * 4);
        const size_t counts = (size_t)((d.n_out + 15) / 16) * sizeof(uint32_t);
        if (e == hipSuccess) e = hipMalloc(&p->arrived.p, counts);
        if (e == hipSuccess) e = hipMemset(p->arrived.p, 0, counts);
        if (e == hipSuccess) e = hipDeviceSynchronize();
    }
    if (e != hipSuccess) {
        delete p;
        return report_hip(e, "allocating the workspace");
    }
    *out = p;
    return TF_OK;
}

tf_status tf_moe_destroy(tf_moe *p) {
    delete p;
    return TF_OK;
}

tf_status tf_moe_layer(const tf_moe *p, const tf_csr *A, const void *X, int64_t ldx, const void *W1, const void *W2, void *D, int64_t ldd,
                       void *stream) {
    const tf_status st = check_layer(p, A, X, ldx, W1, W2, D, ldd);
    if (st != TF_OK) return st;
    if (!aligned(W1, 16) || !aligned(W2, 16)) return report(TF_EINVAL, "weights must be 16-byte aligned");
    const tf_moe_desc &d = p->d;
    if (d.n_in * bytes_of(d.dtype) < 16 || d.n_hidden * bytes_of(d.dtype) < 16)
        return report(TF_EUNSUPPORTED, "dense weights must have rows of 16 bytes or more");
    tf::ExpertLaunch first{}, second{};
    first.W = W1;
    first.w_mat = (d.gated ? 2 : 1) * d.n_hidden * d.n_in * bytes_of(d.dtype);
    second.W = W2;
    second.w_mat = d.n_out * d.n_hidden * bytes_of(d.dtype);
    first.kind = second.kind = -1;
    return run_layer(p, A, X, ldx, first, second, D, ldd, stream);
}

tf_status tf_moe_layer_q4(const tf_moe *p, const tf_csr *A, const void *X, int64_t ldx, const tf_q4 *W1, const tf_q4 *W2, void *D,
                          int64_t ldd, void *stream) {
    tf_status st = check_layer(p, A, X, ldx, W1, W2, D, ldd);
    if (st != TF_OK) return st;
    if ((st = check_q4(W1)) != TF_OK || (st = check_q4(W2)) != TF_OK) return st;
    const tf_moe_desc &d = p->d;
    if (W1->n_mats != d.n_experts || W1->n_rows != (d.gated ? 2 : 1) * d.n_hidden || W1->n_cols != d.n_in)
        return report(TF_EMISMATCH, "W1 does not have the plan's shape");
    if (W2->n_mats != d.n_experts || W2->n_rows != d.n_out || W2->n_cols != d.n_hidden)
        return report(TF_EMISMATCH, "W2 does not have the plan's shape");
    tf::ExpertLaunch first{}, second{};
    set_q4(first, W1);
    set_q4(second, W2);
    return run_layer(p, A, X, ldx, first, second, D, ldd, stream);
}

}  // extern "C"
