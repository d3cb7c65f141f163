// C ABI of the losses and their gradients: argument checks, the plan's workspace.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <new>

#include "tf_loss.h"

namespace {

using tf::ceil_div;
using tf::report;
using tf::report_hip;
using tf::round_up;

constexpr int64_t kMaxSize = ((int64_t)1 << 31) - 1;

bool loss_dtype(int32_t d) { return d == TF_F32 || d == TF_BF16 || d == TF_F16; }
int64_t bytes_of(int32_t d) { return d == TF_F32 ? 4 : 2; }
bool aligned(const void *p, int64_t to) { return reinterpret_cast<uintptr_t>(p) % (uintptr_t)to == 0; }

// Scores and routing matrix of the router's calls; the number of entries of a row in *k.
tf_status check_router(const void *scores, int64_t ld, int32_t dtype, int32_t scoring, const tf_csr *A, int64_t *k) {
    if (!A) return report(TF_EINVAL, "null argument");
    if (!A->on_device) return report(TF_EINVAL, "A must be on the device");
    if (!loss_dtype(dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (scoring < TF_ROUTE_SOFTMAX || scoring > TF_ROUTE_SIGMOID_TOP) return report(TF_EINVAL, "unknown scoring");
    if (A->n_rows < 0 || A->n_cols < 1 || A->nnz < 0) return report(TF_EINVAL, "A has a size that is not positive");
    if (A->n_cols > tf::kRouteMaxExperts) return report(TF_EUNSUPPORTED, "at most 1024 experts and 64 entries in a row");
    *k = 0;
    if (A->n_rows == 0) return TF_OK;
    if (!scores || !A->colidx) return report(TF_EINVAL, "null argument");
    if (A->nnz % A->n_rows || A->nnz < A->n_rows) return report(TF_EINVAL, "A must have the same positive number of entries in each row");
    *k = A->nnz / A->n_rows;
    if (*k > tf::kRouteMaxK) return report(TF_EUNSUPPORTED, "at most 1024 experts and 64 entries in a row");
    if (A->nnz > kMaxSize || A->n_rows >= kMaxSize) return report(TF_EUNSUPPORTED, "A has too many entries");
    if (ld < A->n_cols) return report(TF_EINVAL, "rows of the scores are closer together than they are wide");
    if (!aligned(scores, bytes_of(dtype)) || !aligned(A->colidx, 4)) return report(TF_EINVAL, "arrays must be aligned to their elements");
    return TF_OK;
}
tf::RouterLaunch router_args(const void *scores, int64_t ld, int32_t dtype, int32_t scoring, const tf_csr *A, int64_t k) {
    tf::RouterLaunch a{};
    a.scores = scores;
    a.ld = ld;
    a.colidx = A->colidx;
    a.n_tokens = (int32_t)A->n_rows;
    a.n_experts = (int32_t)A->n_cols;
    a.k = (int32_t)k;
    a.dtype = dtype;
    a.scoring = scoring;
    return a;
}

}  // namespace

struct tf_xent {
    tf_xent_desc d{};
    int device = 0;
    tf::XentSpace s{};
    void *memory = nullptr;
    ~tf_xent() {
        if (memory) (void)hipFree(memory);
    }
};

namespace {

// Cuts the workspace out of one allocation; with base 0 it only adds up the bytes.
struct Cut {
    char *base;
    int64_t bytes = 0;
    template <typename T> void take(T *&p, int64_t n) {
        p = reinterpret_cast<T *>(base + bytes);
        bytes += round_up(n * (int64_t)sizeof(T), 256);
    }
};

// Sizes of the workspace.  G (the gradient of the logits) is held for as many classes at a time as 2^29 bytes allow (256 at least), a copy of W for as many
// as 2^28 do, partial sums for as many as leave 2^25 of them, slabs of the shares of dX up to 2^26 numbers, or what one share needs, of dW 2^25; and
// nothing of it for which the plan's sizes leave no use.  fp32 numbers take three planes of 16 bits, in which they also lie as they are; G in fp16 has two.
int64_t lay_out(tf_xent &p, char *base) {
    const tf_xent_desc &d = p.d;
    tf::XentSpace &s = p.s;
    const bool f32 = d.dtype == TF_F32;
    const int64_t rows = round_up(d.max_rows, 256), classes = round_up(d.n_classes, 256);
    const int64_t planes = f32 ? 3 : 1, g_planes = d.dtype == TF_F16 ? 2 : planes;
    s.ld = round_up(d.n_in, 64) + tf::kRowPad;
    s.slab_ld = round_up(d.n_in, 256) + tf::kRowPad;
    s.x_plane = rows * s.ld;
    s.part_cap = std::max(std::min(classes / 64 * rows, (int64_t)1 << 25), 4 * rows);
    const auto piece = [&](int64_t row, int64_t most) { return std::max<int64_t>(256, std::min(classes, most / row / 256 * 256)); };
    // W is copied by calls of more rows than kNativeRows or kRegisterRows only; 16-bit rows of whole pieces of 16 bytes only where they do not begin at
    // such pieces, for which a small piece at a time will do.
    const int64_t least_rows = (f32 ? tf::kNativeRows : tf::kRegisterRows)[d.gradients], w_most = f32 || d.n_in % 8 ? ((int64_t)1 << 27) / planes : (int64_t)1 << 24;
    const int64_t w_piece = piece(s.ld, w_most), g_piece = piece(rows, ((int64_t)1 << 28) / g_planes);
    s.w_cap = d.max_rows > least_rows ? w_piece * s.ld : 0;
    s.g_cap = d.gradients ? (g_piece + tf::kRowPad) * rows : 0;
    // shares that contractions over so many classes or rows can be cut into
    const auto most_shares = [&](int64_t k) {
        const int whole = tf::shares_of(1 << 30, (int)ceil_div(k, 64), (int)planes);
        return (int64_t)(f32 ? std::max(whole, tf::shares_of(1 << 30, (int)ceil_div(k, 32), 1)) : whole);
    };
    const int64_t dx_shares = most_shares(d.n_classes), dw_shares = most_shares(d.max_rows), dx_size = rows * s.slab_ld;
    const bool one_piece = g_piece >= classes && classes <= tf::kMostColumnsOfG && (s.w_cap == 0 || w_piece >= classes);
    s.dx_cap = !d.gradients || (one_piece && dx_shares == 1)
                   ? 0
                   : std::min(dx_shares * dx_size, std::max({dx_size, std::min((int64_t)1 << 26, 4 * dx_size), std::min((int64_t)1 << 24, 512 * 64 * s.slab_ld)}));
    s.dw_cap = !d.gradients || dw_shares == 1 ? 0 : std::min((int64_t)1 << 25, dw_shares * classes * s.slab_ld);
    Cut c{base};
    c.take(s.list, d.max_rows);
    c.take(s.pos, d.max_rows);
    c.take(s.block_rows, tf::kMostBlocks);
    c.take(s.block_top, tf::kMostBlocks);
    c.take(s.block_low, tf::kMostBlocks);
    c.take(s.block_high, tf::kMostBlocks);
    c.take(s.n, 1);
    c.take(s.arrived, tf::kMostJoins * tf::kJoinApart);
    c.take(s.unit, 1);
    c.take(s.same, 1);
    c.take(s.label, d.max_rows);
    c.take(s.lse, d.max_rows);
    c.take(s.g, d.max_rows);
    c.take(s.hit, d.max_rows);
    c.take(s.dloss, d.dtype == TF_F16 ? d.max_rows : 0);
    c.take(s.top, d.max_rows);
    c.take(s.sum, d.max_rows);
    c.take(s.part, s.part_cap);
    uint16_t *x, *w, *G;
    c.take(x, planes * s.x_plane);
    c.take(w, planes * s.w_cap);
    c.take(G, g_planes * s.g_cap);
    s.x = x;
    s.w = w;
    s.G = G;
    c.take(s.dx, s.dx_cap);
    c.take(s.dw, s.dw_cap);
    return c.bytes;
}

tf_status check_desc(const tf_xent_desc *desc) {
    if (!desc) return report(TF_EINVAL, "null argument");
    if (desc->n_classes < 1 || desc->n_in < 1 || desc->max_rows < 1) return report(TF_EINVAL, "sizes must be positive");
    if (!loss_dtype(desc->dtype)) return report(TF_EUNSUPPORTED, "element type must be fp32, bf16 or fp16");
    if (desc->gradients != 0 && desc->gradients != 1) return report(TF_EINVAL, "gradients must be 0 or 1");
    if (desc->n_in > tf::kXentMaxColumns) return report(TF_EUNSUPPORTED, "weights have rows of at most 2^22 columns");
    if (desc->n_classes > tf::kXentMaxClasses || desc->max_rows > tf::kXentMaxRows) return report(TF_EUNSUPPORTED, "a size is too large");
    return TF_OK;
}
tf_status check_xent(const tf_xent *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, int64_t n_rows) {
    if (!p || !W) return report(TF_EINVAL, "null argument");
    if (n_rows < 0) return report(TF_EINVAL, "number of rows");
    if (n_rows > p->d.max_rows) return report(TF_EMISMATCH, "more rows than the plan was made for");
    if (n_rows > 0 && (!X || !labels)) return report(TF_EINVAL, "null argument");
    if (ldx < p->d.n_in || ldw < p->d.n_in) return report(TF_EINVAL, "rows of X or W are closer together than they are wide");
    const int64_t es = bytes_of(p->d.dtype);
    if (!aligned(X, es) || !aligned(W, es) || !aligned(labels, 4)) return report(TF_EINVAL, "arrays must be aligned to their elements");
    int device = 0;
    const hipError_t e = hipGetDevice(&device);
    if (e != hipSuccess) return report_hip(e, "asking for the current device");
    if (device != p->device) return report(TF_EMISMATCH, "the plan was made on another device than the current one");
    return TF_OK;
}
tf::XentLaunch xent_args(const tf_xent *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, int64_t n_rows) {
    tf::XentLaunch a{};
    a.s = p->s;
    a.X = X;
    a.W = W;
    a.ldx = ldx;
    a.ldw = ldw;
    a.labels = labels;
    a.n_rows = (int32_t)n_rows;
    a.n_classes = (int32_t)p->d.n_classes;
    a.n_in = (int32_t)p->d.n_in;
    a.dtype = p->d.dtype;
    return a;
}

}  // namespace

extern "C" {

tf_status tf_moe_balance_size(int64_t n_tokens, int64_t n_experts, int64_t *bytes) {
    if (!bytes) return report(TF_EINVAL, "null argument");
    if (n_tokens < 0 || n_experts < 1) return report(TF_EINVAL, "sizes must be positive");
    if (n_experts > tf::kRouteMaxExperts) return report(TF_EUNSUPPORTED, "at most 1024 experts and 64 entries in a row");
    *bytes = tf::balance_bytes((int)n_experts);
    return TF_OK;
}

tf_status tf_moe_balance(const void *scores, int64_t ld, int32_t dtype, int32_t scoring, const tf_csr *A, int32_t *counts, float *mass,
                         float *loss, void *workspace, void *stream) {
    int64_t k;
    const tf_status st = check_router(scores, ld, dtype, scoring, A, &k);
    if (st != TF_OK) return st;
    if (!counts || !mass || !loss || !workspace) return report(TF_EINVAL, "null argument");
    if (!aligned(counts, 4) || !aligned(mass, 4) || !aligned(loss, 4))
        return report(TF_EINVAL, "arrays must be aligned to their elements");
    if (!aligned(workspace, 16)) return report(TF_EINVAL, "the workspace must be 16-byte aligned");
    tf::RouterLaunch a = router_args(scores, ld, dtype, scoring, A, k);
    a.counts = counts;
    a.mass = mass;
    a.loss = loss;
    a.workspace = workspace;
    const int e = tf::launch_balance(a, stream);
    return e ? report_hip(e, "launching the balance") : TF_OK;
}

tf_status tf_moe_route_grad(const void *scores, int64_t ld, int32_t dtype, int32_t scoring, float scale, const tf_csr *A, const float *dvals,
                            const int32_t *counts, const float *dloss, void *dscores, int64_t ldd, void *stream) {
    int64_t k;
    const tf_status st = check_router(scores, ld, dtype, scoring, A, &k);
    if (st != TF_OK || A->n_rows == 0) return st;
    if (!dscores || !counts != !dloss) return report(TF_EINVAL, "null argument");
    if (!dvals && !dloss) return report(TF_EINVAL, "no gradient is given");
    if (ldd < A->n_cols) return report(TF_EINVAL, "rows of the gradient are closer together than they are wide");
    if (dscores == scores && ldd != ld) return report(TF_EINVAL, "a gradient in the scores' place has their rows");
    if (!aligned(dscores, bytes_of(dtype)) || !aligned(dvals, 4) || !aligned(counts, 4) || !aligned(dloss, 4))
        return report(TF_EINVAL, "arrays must be aligned to their elements");
    tf::RouterLaunch a = router_args(scores, ld, dtype, scoring, A, k);
    a.scale = scale;
    a.dvals = dvals;
    a.counts = const_cast<int32_t *>(counts);
    a.dloss = dloss;
    a.dscores = dscores;
    a.ldg = ldd;
    const int e = tf::launch_route_grad(a, stream);
    return e ? report_hip(e, "launching the router's gradient") : TF_OK;
}

tf_status tf_xent_size(const tf_xent_desc *desc, int64_t *bytes) {
    if (!bytes) return report(TF_EINVAL, "null argument");
    const tf_status st = check_desc(desc);
    if (st != TF_OK) return st;
    tf_xent p;
    p.d = *desc;
    *bytes = lay_out(p, nullptr);
    return TF_OK;
}

tf_status tf_xent_create(const tf_xent_desc *desc, tf_xent **out) {
    if (!out) return report(TF_EINVAL, "null argument");
    *out = nullptr;
    const tf_status st = check_desc(desc);
    if (st != TF_OK) return st;
    tf_xent *p = new (std::nothrow) tf_xent;
    if (!p) return report(TF_ENOMEM, "out of host memory");
    p->d = *desc;
    hipError_t e = hipGetDevice(&p->device);
    const int64_t bytes = lay_out(*p, nullptr);
    if (e == hipSuccess) e = hipMalloc(&p->memory, (size_t)bytes);
    if (e != hipSuccess) {
        p->memory = nullptr;
        delete p;
        return report_hip(e, "allocating the workspace");
    }
    lay_out(*p, static_cast<char *>(p->memory));
    *out = p;
    return TF_OK;
}

tf_status tf_xent_destroy(tf_xent *p) {
    delete p;
    return TF_OK;
}

tf_status tf_xent_loss(const tf_xent *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, int64_t n_rows,
                       float *loss, float *lse, void *stream) {
    const tf_status st = check_xent(p, X, ldx, W, ldw, labels, n_rows);
    if (st != TF_OK || n_rows == 0) return st;
    if (!loss || !lse) return report(TF_EINVAL, "null argument");
    if (!aligned(loss, 4) || !aligned(lse, 4)) return report(TF_EINVAL, "arrays must be aligned to their elements");
    tf::XentLaunch a = xent_args(p, X, ldx, W, ldw, labels, n_rows);
    a.loss = loss;
    a.lse = lse;
    const int e = tf::launch_xent(a, stream);
    return e ? report_hip(e, "launching the cross entropy") : TF_OK;
}

tf_status tf_xent_grad(const tf_xent *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, const float *lse,
                       const float *dloss, int64_t n_rows, void *dX, int64_t lddx, void *dW, int64_t lddw, void *stream) {
    return tf_xent_grad_by_loss(p, X, ldx, W, ldw, labels, nullptr, lse, dloss, n_rows, dX, lddx, dW, lddw, stream);
}

tf_status tf_xent_grad_by_loss(const tf_xent *p, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, const float *loss,
                               const float *lse, const float *dloss, int64_t n_rows, void *dX, int64_t lddx, void *dW, int64_t lddw, void *stream) {
    const tf_status st = check_xent(p, X, ldx, W, ldw, labels, n_rows);
    if (st != TF_OK) return st;
    if (!p->d.gradients) return report(TF_EMISMATCH, "the plan was made without gradients");
    if (!dX && !dW) return report(TF_EINVAL, "no gradient is asked for");
    if (n_rows > 0 && (!lse || !dloss)) return report(TF_EINVAL, "null argument");
    if ((dX && lddx < p->d.n_in) || (dW && lddw < p->d.n_in)) return report(TF_EINVAL, "rows of dX or dW are closer together than they are wide");
    const int64_t es = bytes_of(p->d.dtype);
    if (!aligned(dX, es) || !aligned(dW, es) || !aligned(loss, 4) || !aligned(lse, 4) || !aligned(dloss, 4))
        return report(TF_EINVAL, "arrays must be aligned to their elements");
    if (n_rows == 0 && !dW) return TF_OK;
    tf::XentLaunch a = xent_args(p, X, ldx, W, ldw, labels, n_rows);
    a.lse_in = lse;
    a.dloss = dloss;
    a.loss_in = loss;
    a.dX = dX;
    a.lddx = lddx;
    a.dW = dW;
    a.lddw = lddw;
    const int e = tf::launch_xent_grad(a, stream);
    return e ? report_hip(e, "launching the gradient of the cross entropy") : TF_OK;
}

tf_status tf_xent_device(const tf_xent *p, int32_t *device) {
    if (!p || !device) return report(TF_EINVAL, "null argument");
    *device = p->device;
    return TF_OK;
}

}  // extern "C"
