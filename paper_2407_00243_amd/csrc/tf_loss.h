// Losses of a routed network or a classifier and their gradients: what their sources share.
#pragma once
#include "tf_moe.h"

namespace tf {

// ---------------------------------------------------------------------- router: balance and gradient

// Workgroups of a balance's first launch, each of which leaves its sums in the workspace.
constexpr int kBalanceGroups = 256;
// Bytes of that workspace: for each workgroup a sum and a count for each expert (rounded up to whole fours), and its number of rows.
constexpr int balance_row(int n_experts) { return (n_experts + 3) / 4 * 4; }
inline int64_t balance_bytes(int n_experts) { return (int64_t)kBalanceGroups * (2 * balance_row(n_experts) + 1) * 4; }

struct RouterLaunch {
    const void *scores;
    int64_t ld;
    const int32_t *colidx;
    int32_t n_tokens, n_experts, k, dtype, scoring;
    // balance
    int32_t *counts;              // n_experts, and behind them the rows that have an entry
    float *mass, *loss;
    void *workspace;
    // gradient
    float scale;
    const float *dvals, *dloss;   // NULL: no such part
    void *dscores;
    int64_t ldg;
};
int launch_balance(const RouterLaunch &a, void *stream);
int launch_route_grad(const RouterLaunch &a, void *stream);

// ------------------------------------------------------------------------- cross entropy of a product

constexpr int64_t kXentMaxColumns = (int64_t)1 << 22;      // 256 rows of 16-bit numbers are below 2^32 bytes
constexpr int64_t kXentMaxRows = (int64_t)1 << 28, kXentMaxClasses = (int64_t)1 << 30;
typedef float Float2 __attribute__((ext_vector_type(2)));
constexpr int64_t round_up(int64_t n, int64_t to) { return ceil_div(n, to) * to; }

// A plan's workspace.  Rows that have a label ("kept") are numbered in their order; arrays by row are by that number.
struct XentSpace {
    int32_t *list, *pos;          // row of X of a kept row; number of a row or -1
    int32_t *block_rows;          // kept rows of each block of rows
    float *block_top;             // largest |dloss| there
    float *block_low, *block_high;       // smallest and largest dloss (fp16)
    int32_t *n;                   // kept rows
    unsigned *arrived;            // for blocks of rows: workgroups that have left their sums
    float *unit;                  // what sums of gradients are multiplied by at the end
    int32_t *same;                // 1: all kept rows have the same dloss (fp16)
    int32_t *label;
    float *lse, *g, *hit;         // log of the sum, gradient over the unit, logit of the label (or, where the loss is given, minus that)
    float *dloss;                 // gradient of the row's loss (fp16)
    float *top, *sum;             // running maximum and sum of exponentials
    Float2 *part;                 // both for blocks of classes, block after block
    void *x, *w, *G;              // operands: rows that count, a copy of W where there has to be one, gradient of the logits; planes of 16-bit
                                  // numbers, or (native) fp32.  fp16 has two planes of G: see kRowUnit
    float *dx, *dw;               // sums in 32 bits, one slab for each share of a contraction
    int64_t ld;                   // row length of x and w: n_in rounded up to 64, and kRowPad
    int64_t slab_ld;              // of dx and dw: rounded up to 256
    int64_t x_plane;              // elements
    int64_t part_cap, g_cap, w_cap, dx_cap, dw_cap;     // elements that there is room for (of a plane)
};
constexpr int64_t kMostBlocks = 1024;      // of rows
constexpr int kMostJoins = 1024;           // blocks of rows whose sums the last workgroup adds up
constexpr int kJoinApart = 32;             // their counters: a line of memory each, else all workgroups would count in one
// G in fp16.  Its first plane is what dX is made of: each row is over its own dloss times kRowUnit, so that a row keeps its precision whatever the others'
// dloss is.  The second is what dW, a sum over the rows, is made of: all rows over the largest |dloss| times 2^-15.  Where all rows have the same dloss, as a
// mean's have, the first one serves both.
constexpr float kRowUnit = 1.0f / 32768.0f;
// Elements between the rows of x, w and G: rows a power of two apart would all lie in one channel of an XCD's L2.
constexpr int64_t kRowPad = 64;
// Up to so many rows (of the loss, of its gradients) fp32 numbers are multiplied as they are, and rows of W that begin anywhere go through registers:
// W is not copied.  (Measured where the rules are: tf_xent.hip.)
constexpr int64_t kNativeRows[2] = {448, 192}, kRegisterRows[2] = {1023, 64};
// 256 rows of G stay below 2^32 bytes, as the products' loads count them.  (A plan for very many rows has room for more columns of few.)
constexpr int64_t kMostColumnsOfG = (int64_t)1 << 22;

struct XentLaunch {
    XentSpace s;
    const void *X, *W;
    int64_t ldx, ldw, lddx, lddw;
    const int32_t *labels;
    int32_t n_rows, n_classes, n_in, dtype;
    float *loss, *lse;
    const float *lse_in, *dloss, *loss_in;   // loss_in: NULL or the rows' losses
    void *dX, *dW;
    int32_t native;               // fp32 operands are multiplied as they are, not in parts
    int32_t direct_dx;            // dX is written by its product; rows without a label get their zeros first
};
int launch_xent(const XentLaunch &a, void *stream);
int launch_xent_grad(const XentLaunch &a, void *stream);

// Products of the cross entropy (tf_product.h): C = M N^T summed over K, tiles of C by workgroups.
struct Side {
    const void *p;
    int64_t ld, plane;            // elements: from row to row, from part to part
    int64_t rows, cols;           // what there is of it (cols: whole pieces of 16 bytes, unless `any`); further elements count as zeros
};
// Shares of a contraction: each has four steps at least, or one of numbers in parts, which takes six.
constexpr int least_share(int parts) { return parts == 3 ? 1 : 4; }
constexpr int shares_of(int most, int steps, int parts) {
    const int shares = steps / least_share(parts);
    return most < shares ? most : shares < 1 ? 1 : shares;
}
enum ProductEnd { kEndSums = 0, kEndGradient = 1, kEndSlab = 2, kEndOut = 3 };
enum ProductTile { kTile256 = 0, kTile128 = 1, kTile64 = 2, kTile16 = 3 };
struct ProductLaunch {
    Side M, N;
    int32_t any;                  // 1: rows of M begin at any element (and its columns are any number)
    int32_t parts;                // of a number: 1, or 3 whose six largest products are taken
    int32_t k_steps;              // of 64 columns (fp32: 32)
    const int32_t *n;             // kept rows
    int32_t k_rows;               // 1: K goes over kept rows
    int32_t n_rows;               // 1: N does
    int32_t m_tiles, n_tiles, splits;      // splits: shares of K at most
    ProductEnd end;
    ProductTile tile;
    int32_t m_count, n_count;     // rows of M and N that count
    // ends
    int32_t first_class;
    const int32_t *label;
    const float *lse, *g, *unit;
    const float *row_unit;        // NULL or, for each row of N, what its results are multiplied by besides kRowUnit, in the unit's place
    float *hit;                   // (gradient: NULL or the logarithm of the label's exp(l - lse))
    Float2 *part;                 // largest logit and sum of exponentials over it
    int64_t part_ld;
    int32_t join;                 // 1: the last workgroup of a block of rows adds up its sums and writes
    unsigned *arrived;
    float *loss, *lse_out;        // (at out_row)
    void *G;
    int64_t g_ld, g_plane;
    int32_t for_dx, for_dw;       // fp16: what G is wanted for
    const int32_t *same;          // fp16: which plane is dW's
    float *slab;
    int64_t slab_ld, slab_size;
    int32_t add;                  // to what the slab holds
    void *out;
    int64_t ldo;
    const int32_t *out_row;       // NULL: as they are
    int32_t out_dtype;
};
int launch_product_bf16(const ProductLaunch &a, void *stream);
int launch_product_f16(const ProductLaunch &a, void *stream);
int launch_product_f32(const ProductLaunch &a, void *stream);

}  // namespace tf
