/*
 * tilefusion.h -- C ABI of the tile-fusion library for the matrix chain  D = A (B C)  on gfx950.
 *
 * The operation (paper Section 1, Eq. 1): A is an n x n CSR sparse matrix, B is n x bCol and
 * either dense or CSR sparse, C is a dense bCol x cCol matrix.  Unfused, the chain is
 * D1 = B C followed by D = A D1.  Tile fusion (Section 3) inspects the sparsity pattern of A
 * once, builds a schedule of two wavefronts -- fused tiles that produce a block of D1 rows and
 * at once consume them for the rows of D that depend on nothing else, then the leftover rows
 * of D -- and reuses that schedule for every later execution (Section 3, first paragraph).
 *
 * Conventions for every call
 *   - Dense matrices are row-major and contiguous; B is n x bCol, C is bCol x cCol, D is n x cCol.
 *   - Dense operands and every pointer handed to an execution call are DEVICE pointers, aligned
 *     to 16 bytes.  The element type of B, C, D is the element type of A.
 *   - CSR matrices use int32 row pointers (n_rows + 1 entries, rowptr[0] = 0) and int32 column
 *     indices.  Explicit zeros, duplicate and unsorted column indices are legal; entries are
 *     summed in an unspecified order.
 *   - D is overwritten (the listings of Section 3.2 accumulate into zeroed outputs).
 *   - The caller owns A, B, C and D.  The plan owns a device copy of A (pattern and values), the
 *     schedule and a workspace with one slot for every D1 row that crosses tiles (in the two
 *     wavefronts no other D1 row ever reaches device memory: Section 3.1, one synchronisation).
 *   - Where the tiling was left to the library (see tf_tile_params) the fused calls may run the
 *     chain in another way than the two wavefronts, whichever is expected to be the fastest:
 *     tf_schedule_view.execution tells which.  D agrees to rounding; rows of A without entries
 *     give rows of zeros in every case.  With finite operands the ways differ in nothing else;
 *     D = (A B) C and D = A (B C) may disagree on where infinities and NaN arise.
 *   - Errors are reported by return code; tf_last_error() gives a message for the calling
 *     thread's most recent failure.  No call throws or aborts.
 */
#ifndef TILEFUSION_H
#define TILEFUSION_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    TF_OK = 0,
    TF_EINVAL = 1,        /* null pointer, non-positive size, bad alignment, bad parameter   */
    TF_EBADCSR = 2,       /* malformed CSR: rowptr not monotone, rowptr[n] != nnz, col range  */
    TF_ENOMEM = 3,        /* host or device allocation failed                                 */
    TF_EHIP = 4,          /* a HIP runtime call failed                                        */
    TF_EUNSUPPORTED = 5,  /* shape outside what the kernels cover (see tf_plan_create)        */
    TF_EMISMATCH = 6      /* plan and call disagree (dtype, kind of B, shape of B)            */
} tf_status;

/* The chain D = A (B C) runs in fp32 and fp64, the routed operators (below) in fp32, bf16 and fp16. */
typedef enum { TF_F32 = 0, TF_F64 = 1, TF_BF16 = 2, TF_F16 = 3 } tf_dtype;

/* A CSR matrix.  Caller-owned, read-only.  on_device tells where the three arrays live
 * (all three in the same place). */
typedef struct tf_csr {
    int64_t n_rows;
    int64_t n_cols;
    int64_t nnz;
    const int32_t *rowptr;
    const int32_t *colidx;
    const void *vals;
    int32_t dtype;      /* tf_dtype */
    int32_t on_device;  /* 0 = host pointers, 1 = device pointers */
} tf_csr;

/* Inputs of the scheduler (Algorithm 1) besides the pattern.  Zero selects the default.
 * With ct_size = 0 and p = 0 and neither TF_FLAG_REORDER nor TF_FLAG_NO_SPLIT (in particular with
 * tp = NULL) the tiling is left to the library: ctSize 2048, p = a quarter of the compute units,
 * half of the LDS per tile where two workgroups per compute unit pay (dense B, small bCol x cCol);
 * tiles of consecutive rows as in Algorithm 1 unless they fuse under half of the entries of a
 * matrix whose rows stay near the diagonal and graph-grown tiles spill fewer D1 rows; and where
 * the fused rows that read the fast memory hold under 2 % of the entries (graphs) they are left
 * to the second wavefront, so that the first wavefront needs no tile in fast memory at all.
 * With ct_size or p given, step 1 is Algorithm 1 to the letter. */
typedef struct tf_tile_params {
    int32_t ct_size;         /* coarse tile size ctSize (Section 3.1.1); default 2048           */
    int32_t p;               /* wanted number of tiles per wavefront ("cores"); default 32 when
                                ct_size is given, else a quarter of the compute units            */
    int64_t fast_mem_bytes;  /* fast memory of one tile: the LDS a workgroup may use;
                                default = the device's LDS per workgroup (160 KiB on gfx950)    */
    int32_t col_slice;       /* columns of C/D handled by one workgroup; default = cCol, capped
                                at what the kernels cover; a last narrower slice is allowed     */
    uint32_t flags;          /* TF_FLAG_* */
    int32_t gather_slices;   /* column slices of the D1 workspace, each gathered by its own XCDs
                                in the second wavefront: 1, 2, 4 or 8, slices of a power of two
                                of columns, at least 16 and at least 64 bytes.  Default: 1 for
                                matrices whose rows stay near the diagonal, slices of 128 bytes
                                (any number of them up to 8) or rows padded to that for matrices
                                whose rows reach far (graphs), see tf_schedule_view.d1_slices   */
    int32_t reserved0;
} tf_tile_params;

/* Skip step 2 (tile splitting): tiles that do not fit the fast memory make plan creation fail. */
#define TF_FLAG_NO_SPLIT 1u
/* Build the schedule only: no device is touched and no device memory is allocated, A must be in
 * host memory, fast_mem_bytes is taken as given (default 160 KiB).  The plan serves
 * tf_plan_schedule; execution calls on it fail with TF_EINVAL. */
#define TF_FLAG_SCHEDULE_ONLY 2u
/* Tiles are grown along the dependence graph (breadth first over the column indices of A,
 * starting from the lowest row not yet in a tile) instead of being ranges of consecutive rows, each
 * as large as the fast memory allows and at most t rows.  The paper forms tiles from consecutive
 * iterations (Section 3.1.1) because that is cheap and keeps spatial locality; on matrices whose
 * rows depend on far-away rows (stencils in natural ordering) consecutive tiles small enough
 * for LDS fuse nothing, while graph-grown tiles do. */
#define TF_FLAG_REORDER 4u
/* The chain with the transpose of C (Section 3.2 notes that the fused code also covers it):
 * D = A (B C^T).  The dense-B calls on such a plan take C as a cCol x bCol row-major array, so
 * that element (k, c) of the multiplier is C[c * bCol + k]; everything else is unchanged.  Only
 * plans for a dense B accept the flag (a sparse B gathers whole rows of C; plan creation fails
 * with TF_EUNSUPPORTED). */
#define TF_FLAG_C_TRANSPOSED 8u
/* Rows of D1 = B C that no row of A reads (columns of A without a stored entry) are not computed
 * by the fused calls: they leave the tiles' first lists.  The paper's schedule runs every
 * iteration of both operations exactly once (Section 3.1); this flag gives that up for the first
 * operation, D is unchanged.  The unfused calls still compute all of D1, and after a fused call
 * the workspace rows of skipped D1 rows are not written.  (A plan for a CSR B whose first
 * wavefront streams leaves the rows out one by one instead; the schedule view is the same.) */
#define TF_FLAG_SKIP_UNREAD 16u
/* The plan serves the fused calls only: the packed copy of all rows of A that the unfused
 * baseline runs on is not built (saves its time and device memory); tf_unfused_* then fail with
 * TF_EINVAL.  (A plan whose fused calls themselves run the two operations over all rows,
 * TF_EXECUTE_PLAIN_PAIR, holds that copy all the same; its tf_unfused_* fail likewise.) */
#define TF_FLAG_NO_BASELINE 32u

/* How the fused calls of a plan run the chain (tf_schedule_view.execution).  All but the first are
 * chosen only where no tile parameter, column slice, slice count or fast memory is given. */
#define TF_EXECUTE_WAVEFRONTS 0    /* the schedule: fused tiles, then the leftover rows               */
#define TF_EXECUTE_ONE_PASS 1      /* dense B, rows near the diagonal: D = (A B) C in one launch      */
#define TF_EXECUTE_GATHER_FIRST 2  /* dense B, graph, narrow B: Y = A B for all rows, then D = Y C    */
#define TF_EXECUTE_PLAIN_PAIR 3    /* CSR B, D1 held by the caches: D1 = B C and D = A D1 over all rows */

typedef struct tf_plan tf_plan; /* opaque, library-owned */

/* Host-readable view of a plan's schedule.  All pointers are HOST memory owned by the plan and
 * stay valid until tf_plan_destroy.  A tile v of the first wavefront produces the D1 rows
 *   first_rows[tile_first_ptr[v] .. tile_first_ptr[v+1])      (the tile's "first" list;
 *                                         n_first_rows entries in all: n unless rows are skipped)
 * and then computes the rows of D
 *   second_rows[tile_second_ptr[v] .. tile_second_ptr[v+1])   (the tile's "second" list);
 * unit u of the second wavefront computes the rows wf1_rows[wf1_unit_ptr[u] .. wf1_unit_ptr[u+1]).
 * spill[i] != 0 marks D1 rows that are also stored to device memory because a row of the
 * second wavefront reads them.  Every figure is that of the two wavefronts, whatever `execution`
 * says. */
typedef struct tf_schedule_view {
    int64_t n;
    int64_t nnz;
    int32_t t;                  /* uniform tile size chosen by step 1                          */
    int32_t col_slice;
    int32_t n_slices;
    int32_t dtype;
    int32_t b_is_sparse;
    int32_t execution;          /* TF_EXECUTE_*: what the fused calls of the plan run          */
    int64_t n_coarse_tiles;     /* tiles after step 1                                          */
    int64_t n_tiles;            /* tiles after step 2                                          */
    const int32_t *tile_first_ptr;
    const int32_t *first_rows;
    const int32_t *tile_second_ptr;
    const int32_t *second_rows;
    int64_t n_wf1_units;
    const int32_t *wf1_unit_ptr;
    const int32_t *wf1_rows;
    const uint8_t *spill;
    int64_t n_fused_rows;
    int64_t n_wf1_rows;
    int64_t n_spill_rows;
    int64_t fused_nnz;          /* stored entries of A that belong to fused rows               */
    double fused_ratio_eq3;     /* Eq. 3 literally: fused rows / (|I| + |J|) = / 2n            */
    double fused_ratio_rows;    /* fused rows / n                                              */
    double fused_ratio_nnz;     /* share of the second operation's work done in wavefront 0    */
    int64_t fast_mem_bytes;     /* the budget the tiles were fitted to                         */
    int64_t lds_fixed_bytes;    /* LDS a fused workgroup uses besides its D1 tile              */
    int64_t lds_bytes_per_row;  /* LDS per D1 row of a tile (the row, its id twice, an estimate of
                                   its packed entries); footprint = fixed + rows_pad * this    */
    int32_t lds_row_granule;    /* rows_pad = rows rounded up to a multiple of this            */
    int32_t second_block_in_lds; /* 1: the packed entries of a tile's fused rows are staged in LDS;
                                   0: they did not fit beside the largest tile and are read in place */
    double eq2_cost_max;        /* largest Eq. 2 data-movement cost over the tiles (elements)  */
    double plan_seconds;        /* host time spent building the schedule (without the packed
                                   copy of A that only the unfused baseline uses)              */
    int64_t alg_bytes;          /* algorithmic HBM bytes of the two wavefronts: A, B, C and D once,
                                   every spilled D1 row written once and read once.  A CSR B is
                                   not known to the plan and is NOT included: the caller adds
                                   4 (n + 1) + nnz(B) (4 + element size)                         */
    int64_t alg_bytes_unfused;  /* the same for the unfused two-kernel execution (all of D1
                                   written once and read once)                                   */
    int64_t second_block_bytes; /* largest per-tile block of packed entries (fused rows)       */
    int64_t lds_launch_bytes;   /* LDS one fused workgroup is launched with (0: schedule only) */
    int64_t n_first_rows;       /* D1 rows the first wavefront produces (length of first_rows) */
    const int32_t *spill_slot;  /* n entries: slot of the D1 row in the workspace, -1 = not spilled */
    int64_t n_direct_rows;      /* fused rows of D that are their own D1 row times a single diagonal
                                   entry, or empty: stored from the registers that hold the D1 row
                                   (they are listed in second_rows like every fused row)         */
    int32_t d1_slices;          /* workspace layout: d1_slices column slices of d1_slice_cols     */
    int32_t d1_slice_cols;      /* columns, slice after slice, each d1_rows x d1_slice_cols       */
    int64_t d1_rows;            /* row-major: element (slot, c) is at (c / d1_slice_cols) d1_rows
                                   d1_slice_cols + slot d1_slice_cols + c mod d1_slice_cols; the
                                   slices may hold more than cCol columns, the last of them padding */
    int32_t first_wavefront_streams; /* 1: no fused row reads the LDS tile (all are direct rows), so
                                   the first wavefront runs without tiles in LDS, streaming through
                                   the rows like the plain first operation                        */
    int32_t grown_tiles;        /* 1: tiles were grown along the dependence graph (TF_FLAG_REORDER,
                                   or the library's own choice), 0: ranges of consecutive rows   */
    int64_t n_demoted_rows;     /* rows that their tile could have fused but that the library left
                                   to the second wavefront (only when the tiling was left to the
                                   library, see tf_plan_create); 0 = step 1 is maximal            */
    int32_t far_rows;           /* 1: the rows of A reach far from the diagonal (a graph)         */
    int32_t automatic;          /* 1: the tiling was left to the library                          */
} tf_schedule_view;

/* Inspector: builds the fused schedule for the pattern of A (Algorithm 1: step 1, coarse tile
 * fusion; step 2, tile splitting against the fast-memory size) plus the spill set and the
 * balanced units of the second wavefront.  bCol and cCol are the column counts of B and C;
 * for a sparse B, bCol is the number of columns of B (= rows of C).  b_is_sparse selects which
 * execution call the plan serves.  tp may be NULL for defaults.
 * Validates: A square, 0 <= nnz < 2^31, rowptr monotone with rowptr[0] = 0 and rowptr[n] = nnz,
 * 0 <= col < n, bCol > 0, cCol > 0, one D1 row fits the fast memory.
 * Synchronous; allocates host and device memory owned by the plan.  On failure *out is NULL.
 * Matrices of 2^18 entries or more are inspected by several host threads (as many as the
 * machine reports, at most 16; the environment variable TF_HOST_THREADS=k lowers that to k);
 * the schedule does not depend on their number. */
tf_status tf_plan_create(const tf_csr *A, int64_t bCol, int64_t cCol, int32_t b_is_sparse,
                         const tf_tile_params *tp, tf_plan **out);

/* Frees everything the plan owns.  NULL is accepted. */
tf_status tf_plan_destroy(tf_plan *plan);

/* Fills *out with the plan's schedule (host pointers, see tf_schedule_view). */
tf_status tf_plan_schedule(const tf_plan *plan, tf_schedule_view *out);

/* Fused execution of D = A (B C) with dense B (Section 3.2, fused GeMM-SpMM listing): first
 * wavefront = one launch over the fused tiles, second wavefront = one launch over the leftover
 * rows; stream order is the single barrier between them.  A plan with another `execution` runs one
 * launch (TF_EXECUTE_ONE_PASS: no workspace) or two (TF_EXECUTE_GATHER_FIRST: the plan's workspace
 * holds Y = A B, n x bCol), unless tf_plan_workspace was called.  B, C, D are device pointers.
 * Asynchronous on `hip_stream` (a hipStream_t, NULL = the default stream); allocates nothing,
 * never synchronises.  Two executions of one plan must not overlap (they share the plan's
 * workspace). */
tf_status tf_gemm_spmm(const tf_plan *plan, const void *B, const void *C, void *D,
                       void *hip_stream);

/* tf_gemm_spmm for callers that cannot allocate device memory and do not want a plan-owned
 * workspace to be touched: code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc.  Same arguments and result as tf_gemm_spmm, but what that call keeps in the
 * plan's workspace (the D1 rows that cross tiles; Y = A B of a TF_EXECUTE_GATHER_FIRST plan; nothing
 * of a TF_EXECUTE_ONE_PASS plan) goes to a fixed array of 64 MiB that is part of the library's code
 * object (one copy per GPU, held until the process ends).  (The few sums of rows that are cut over
 * several workgroups go to memory of the plan that its other calls do not use.)  The call allocates
 * nothing.
 * A plan whose workspace (tf_schedule_view: d1_slices x d1_rows x d1_slice_cols elements) exceeds
 * 64 MiB is rejected with TF_EUNSUPPORTED.  All calls on one GPU share that GPU's array, whatever
 * the plan: calls that overlap in time on one GPU race (serialise them on one stream).  The array
 * keeps the last call's contents; nothing in it needs clearing between calls, since every row is
 * written by the first wavefront before the second one reads it. */
tf_status tf_gemm_spmm_static(const tf_plan *plan, const void *B, const void *C, void *D,
                              void *hip_stream);

/* Fused execution with CSR B (Section 3.2, fused SpMM-SpMM listing).  B must be on the device,
 * n x bCol with the plan's bCol and dtype; C is bCol x cCol.  B may alias A's arrays.  A
 * TF_EXECUTE_PLAIN_PAIR plan runs the two operations over all rows instead, with all of D1 in an array
 * of its own (80 MB at most), unless tf_plan_workspace was called.
 * B's arrays live on the device and are NOT validated by the execution calls (only its shape
 * and element type are): a well-formed CSR (monotone rowptr with rowptr[0] = 0, 0 <= column <
 * bCol) is the caller's precondition; tf_csr_validate checks it where that is in doubt. */
tf_status tf_spmm_spmm(const tf_plan *plan, const tf_csr *B, const void *C, void *D,
                       void *hip_stream);

/* The unfused two-kernel baseline on the same plan (Section 4.1: an unfused parallel
 * implementation with the same optimisations): D1 = B C for all rows into a workspace of n rows,
 * then D = A D1 for all rows.  Same argument rules as the fused calls, except that the first
 * unfused call on a plan allocates that workspace (call tf_plan_prepare_unfused beforehand where
 * the call itself must not allocate, e.g. under stream capture). */
tf_status tf_unfused_gemm_spmm(const tf_plan *plan, const void *B, const void *C, void *D,
                               void *hip_stream);
tf_status tf_unfused_spmm_spmm(const tf_plan *plan, const tf_csr *B, const void *C, void *D,
                               void *hip_stream);

/* One wavefront of the fused execution on its own (wavefront 0 = fused tiles, 1 = leftover
 * rows), for per-kernel timing and tests.  Pass the dense B in B_dense or the CSR B in B_csr
 * according to the plan (the other NULL; both may be NULL for wavefront 1, which reads only the
 * plan's workspace).  Wavefront 1 is only meaningful after wavefront 0 of the same inputs.
 * Available whatever the plan's `execution` is. */
tf_status tf_run_wavefront(const tf_plan *plan, int32_t wavefront, const void *B_dense,
                           const tf_csr *B_csr, const void *C, void *D, void *hip_stream);

/* Allocates the workspace of the unfused baseline (all n rows of D1) if it does not exist yet. */
tf_status tf_plan_prepare_unfused(const tf_plan *plan);

/* Device pointer of the plan's D1 workspace: after a fused execution slot spill_slot[i] holds D1
 * row i, in the layout that tf_schedule_view describes (d1_slices, d1_slice_cols, d1_rows).  Only the
 * two wavefronts leave D1 rows there: on a plan with another `execution`, tf_gemm_spmm[_static] and
 * tf_spmm_spmm run the two wavefronts from the first call of this function on (executions before it,
 * and graphs captured before it, leave the workspace untouched or hold Y = A B there).
 * tf_plan_workspace_unfused: the baseline's workspace, same layout with n rows and slot = row
 * (NULL before the first unfused call or tf_plan_prepare_unfused).  For tests. */
tf_status tf_plan_workspace(const tf_plan *plan, void **d1_device);
tf_status tf_plan_workspace_unfused(const tf_plan *plan, void **d1_device);

/* Checks a CSR matrix given with host or device arrays (device arrays are copied to the host):
 * rowptr[0] = 0, rowptr monotone, rowptr[n_rows] = nnz, 0 <= column < n_cols.  TF_OK or
 * TF_EBADCSR.  Synchronous; meant for a CSR B before it is handed to tf_spmm_spmm. */
tf_status tf_csr_validate(const tf_csr *M);

/* ------------------------------------------------------------------------------------------------
 * Routed operators: the chain in which every column of A has dense operands of its own.
 *
 * A is a routing matrix, tokens x experts, in CSR with a few entries in a row; a row of D is
 *     D[t] = sum over the entries q of row t of  A_q f_e(X[t]),   e = column of q,
 *     f_e(x) = ( act(x Wg_e^T) o (x Wu_e^T) ) Wd_e^T      or, without a gate,  act(x Wu_e^T) Wd_e^T
 * (mixture of experts).  The calls are made for the few tokens of a decoding batch, where the weights
 * that the tokens meet have to be read once and this is what takes the time; they are right for any
 * number of tokens, but read an expert's weights again for every 32 or 64 entries that name it (for every 4 or 16
 * of up to 4 or 16 tokens, where rows name an expert more than once).
 *
 * Conventions besides those at the top of this file
 *   - Element types are TF_F32, TF_BF16 and TF_F16.  Products of 16-bit numbers are summed in 32 bits;
 *     results are rounded once, to nearest even.
 *   - X, D, Y and scores may have rows that are further apart than they are wide (ldx, ldd, ...,
 *     in elements).  Their pointers need the alignment of one element; weights and codes 16 bytes.
 *   - A row's values never reach another row: infinities and NaN stay in the rows that hold them.
 *   - Calls are asynchronous on `hip_stream`, allocate nothing and never synchronise, unless their
 *     comment says so; they may be captured into a graph.  Results do not vary from run to run.
 */

/* Stacked matrices with weights of 4 bits: n_mats matrices of n_rows outputs x n_cols inputs.  A weight
 * is the value of its code times the scale of its group, `group` consecutive inputs of one output:
 *   TF_Q4_INT   codes -7 .. 7
 *   TF_Q4_E2M1  0, 0.5, 1, 1.5, 2, 3, 4, 6 (codes 0 .. 7) and their negatives (codes 8 .. 15)
 * Scales are bf16 (powers of two between 2^-126 and 2^127 are exact in it).  codes and scales are device
 * arrays of the caller's, in the library's own order, of the sizes that tf_q4_sizes tells; tf_q4_pack and
 * tf_q4_quantize write them. */
#define TF_Q4_INT 0
#define TF_Q4_E2M1 1
typedef struct tf_q4 {
    int64_t n_mats;
    int64_t n_rows;
    int64_t n_cols;
    void *codes;      /* 16-byte aligned */
    void *scales;     /* 16-byte aligned */
    int32_t kind;     /* TF_Q4_* */
    int32_t group;    /* 32, 64 or 128 */
} tf_q4;

/* Bytes of the two arrays; W->codes and W->scales are not looked at. */
tf_status tf_q4_sizes(const tf_q4 *W, int64_t *codes_bytes, int64_t *scales_bytes);

/* Fills the arrays of *W from codes, one int8 each (n_mats x n_rows x n_cols; E2M1 codes as 0 .. 15), and
 * bf16 scales (n_mats x n_rows x ceil(n_cols / group)); both on the device.  Codes outside of the kind's
 * range make the call fail with TF_EINVAL (the arrays are then not to be used).  Allocates a word for that
 * and waits for the stream: for the time when weights are loaded. */
tf_status tf_q4_pack(const tf_q4 *W, const int8_t *codes, const void *scales_bf16, void *hip_stream);

/* Fills the arrays of *W from weights (n_mats x n_rows x n_cols, `dtype`, on the device): the scale of a group
 * is its largest magnitude over the largest code value (7 or 6) rounded to bf16, a code is the value nearest
 * to weight / scale (halfway cases to the even code) within the kind's range.  A group of zeros has scale 0.
 * Weights are to be finite: a group with an infinity or a NaN comes out as NaN. */
tf_status tf_q4_quantize(const tf_q4 *W, const void *weights, int32_t dtype, void *hip_stream);

/* The weights that *W stands for, rounded to `dtype` (n_mats x n_rows x n_cols, contiguous). */
tf_status tf_q4_unpack(const tf_q4 *W, int32_t dtype, void *weights, void *hip_stream);

/* Y = X W^T for m rows of X (m x n_cols, rows ldx apart) and one matrix (n_mats = 1): Y is m x n_rows, rows ldy
 * apart.  For a few rows: codes are read again for every 32 or 64.  n_cols is at most 2^24. */
tf_status tf_q4_matvec(const tf_q4 *W, const void *X, int64_t ldx, void *Y, int64_t ldy, int64_t m, int32_t dtype,
                       void *hip_stream);

/* Weights of the entries that tf_moe_route makes; all but the first row of the comment are taken of the scores
 * without the bias, for the selected experts only. */
#define TF_ROUTE_SOFTMAX 0      /* exp(l_e) / sum over all experts           */
#define TF_ROUTE_SOFTMAX_TOP 1  /* exp(l_e) / sum over the selected experts  */
#define TF_ROUTE_SIGMOID 2      /* 1 / (1 + exp(-l_e))                       */
#define TF_ROUTE_SIGMOID_TOP 3  /* the same over its sum over the selected   */

/* Router: from scores l (tokens x experts, rows ld apart, `dtype`) to the routing matrix A.  Each token gets the
 * k = A->nnz / A->n_rows experts with the largest l + bias (32-bit sums; bias: n_cols floats on the device or
 * NULL), in falling order, equal ones by their number; their weights (see above) are multiplied by `scale`.
 * Scores of -inf and NaN are never selected (a NaN counts as -inf in every sum): a row with fewer than k others is
 * filled up with entries of column -1 and value 0, which tf_moe_layer passes over.
 * A describes the result: n_rows tokens, n_cols experts (1024 at most), nnz = k n_rows (k 64 at most), device
 * arrays, dtype TF_F32.  The call WRITES its three arrays. */
tf_status tf_moe_route(const void *scores, int64_t ld, int32_t dtype, const float *bias, int32_t scoring, float scale,
                       const tf_csr *A, void *hip_stream);

/* Activations act(x) */
#define TF_ACT_IDENTITY 0
#define TF_ACT_RELU 1
#define TF_ACT_SILU 2           /* x / (1 + exp(-x))           */
#define TF_ACT_GELU 3           /* x (1 + erf(x / sqrt 2)) / 2 */

typedef struct tf_moe_desc {
    int64_t n_experts;
    int64_t n_in;         /* columns of X                                                     */
    int64_t n_hidden;     /* columns between the two products                                 */
    int64_t n_out;        /* columns of D                                                     */
    int64_t max_tokens;   /* largest number of rows of X                                      */
    int64_t max_entries;  /* largest number of stored entries of A                            */
    int32_t dtype;        /* of X, D and dense weights                                        */
    int32_t activation;   /* TF_ACT_*                                                         */
    int32_t gated;        /* 1: W1 holds the n_hidden rows of the gate, then those it multiplies */
    int32_t reserved0;
} tf_moe_desc;

typedef struct tf_moe tf_moe; /* opaque, library-owned: the sizes above and a workspace */

/* Allocates the workspace (max_entries rows between the products).  n_in and n_hidden are at most 2^24.  On failure
 * *out is NULL. */
tf_status tf_moe_create(const tf_moe_desc *desc, tf_moe **out);
/* Frees it.  NULL is accepted. */
tf_status tf_moe_destroy(tf_moe *plan);

/* D = the layer of X (A->n_rows x n_in, rows ldx apart; D: A->n_rows x n_out, rows ldd apart).  W1 is n_experts x
 * (2 n_hidden or n_hidden) x n_in, W2 n_experts x n_out x n_hidden, both contiguous, each row the weights of one
 * output, of 16 bytes or more (TF_EUNSUPPORTED otherwise).  A: device arrays, values TF_F32, at most max_tokens rows and max_entries entries, any number of them
 * in a row; entries whose column is not one of the experts are passed over, whatever their value; a row without
 * entries gives a row of zeros.  A's arrays are not validated (see tf_spmm_spmm).  What lies between the products is
 * off by up to 2^-16 of its size or 2^-134, whichever is more, where X is bf16; by 2^-22 of it or 2^-25 where X is fp16
 * (magnitudes up to 2^28, larger ones become infinite); and held in 32 bits where X is fp32.
 * Two executions of one plan must not overlap (they share its workspace). */
tf_status tf_moe_layer(const tf_moe *plan, const tf_csr *A, const void *X, int64_t ldx, const void *W1, const void *W2,
                       void *D, int64_t ldd, void *hip_stream);
/* The same with weights of 4 bits: W1 and W2 hold n_experts matrices each, of the shapes above. */
tf_status tf_moe_layer_q4(const tf_moe *plan, const tf_csr *A, const void *X, int64_t ldx, const tf_q4 *W1,
                          const tf_q4 *W2, void *D, int64_t ldd, void *hip_stream);

/* ------------------------------------------------------------------------------------------------
 * Losses and their gradients: what trains a router and a classifier (of a graph's nodes, of tokens).  The mixture-of-experts layer has no gradient of its
 * own here: that of A's values (dvals below) is the caller's to make.
 * The conventions of the routed operators hold: fp32, bf16 and fp16, 32-bit sums rounded once, rows that may be further apart
 * than they are wide, calls that allocate nothing and may be captured.
 */

/* Balance of a router.  With p_te the share of expert e in the scores of token t (softmax scorings: exp(l_e) over its sum over all
 * experts; sigmoid scorings: sigma(l_e) over its sum; a score of -inf or NaN has none),
 *     counts[e] = entries of A whose column is e          counts[n_cols] = n = rows of A that have such an entry
 *     mass[e]   = 1/n sum over those rows of p_te         *loss = n_cols sum_e f_e mass[e],   f_e = counts[e] / sum counts
 * which is 1 where experts are met evenly.  All are 0 where n is.  A is a matrix as tf_moe_route makes it: the same number of entries in
 * each row (at most 64, for at most 1024 columns), columns that are not an expert's (-1) are passed over; rowptr and vals are not read.
 * counts (n_cols + 1), mass, loss and the workspace (16-byte aligned) are device arrays; the workspace has the size that tf_moe_balance_size
 * tells (at most 4 MiB) and may be used by one call at a time.  With softmax scorings a score of +inf makes the shares of
 * its row, and so mass and loss, NaN (if the row has an entry); with sigmoid scorings its sigma is 1. */
tf_status tf_moe_balance_size(int64_t n_tokens, int64_t n_experts, int64_t *bytes);
tf_status tf_moe_balance(const void *scores, int64_t ld, int32_t dtype, int32_t scoring, const tf_csr *A, int32_t *counts, float *mass,
                         float *loss, void *workspace, void *hip_stream);

/* Gradient of the scores: dscores (like scores, rows ldd apart) gets the sum of
 *   - the gradient by way of the entries' values that tf_moe_route made with this scoring and scale: dvals (A->nnz floats) is that of
 *     A's values, those of entries that are passed over are not looked at;
 *   - *dloss (a device float) times the gradient of the balance loss, with the counts of tf_moe_balance (held constant; those of
 *     several devices may have been added up).
 * Either dvals, or counts and dloss, may be NULL.  Scores of -inf or NaN get 0, rows without an entry zeros.  An expert that a row names
 * more than once counts as often.  dscores may be the scores' own array (with ldd = ld). */
tf_status tf_moe_route_grad(const void *scores, int64_t ld, int32_t dtype, int32_t scoring, float scale, const tf_csr *A, const float *dvals,
                            const int32_t *counts, const float *dloss, void *dscores, int64_t ldd, void *hip_stream);

/* Softmax cross entropy of a product: the chain whose middle, the logits l = X W^T (rows x classes), is never kept.
 * Row t of X has the class labels[t]; rows whose label is not one of the classes (-1) have no part in anything: they are not read, their loss,
 * lse and rows of dX are 0.
 *     lse[t] = log sum_v exp(l_tv)                                 loss[t] = lse[t] - l_t,labels[t]
 *     g_tv   = dloss[t] (exp(l_tv - lse[t]) - [v = labels[t]])     dX = g W      dW = g^T X
 * A loss below 2^-126 may be 0. The logits are made for a piece of the classes at a time, by both calls; g is held for a piece, rounded to 16 bits
 * (bf16: to bf16; fp16: to fp16, for dX over the row's own dloss, so that rows of every size of it keep their precision, and for dW, a sum over the
 * rows, over the largest |dloss|, both with 2^-40 of it as the smallest number; a caller who needs more bits of it makes a plan for fp32 and converts
 * the operands; fp32: in 32 bits for few rows, else as three bf16 numbers, which hold 24 bits of X, W and g from 2^-110 on, and of smaller numbers
 * those above 2^-126. Infinite fp32 numbers may give NaN where they are held so). */
typedef struct tf_xent_desc {
    int64_t n_classes;    /* rows of W, at most 2^30                                       */
    int64_t n_in;         /* columns of X and W, at most 2^22                              */
    int64_t max_rows;     /* largest number of rows of X, at most 2^28                     */
    int32_t dtype;        /* of X, W, dX and dW                                            */
    int32_t gradients;    /* 1: the workspace also holds what tf_xent_grad needs, 0: it does not */
} tf_xent_desc;

typedef struct tf_xent tf_xent; /* opaque, library-owned: the sizes above and a workspace */

/* Bytes of the workspace that tf_xent_create allocates: a copy of X's rows, at most 2^29 of g (and 256 classes of it at least), 2^28 of W where its rows
 * have to be copied, sums of shares of long contractions. */
tf_status tf_xent_size(const tf_xent_desc *desc, int64_t *bytes);
/* Allocates the workspace on the current device.  On failure *out is NULL. */
tf_status tf_xent_create(const tf_xent_desc *desc, tf_xent **out);
/* Frees it.  NULL is accepted. */
tf_status tf_xent_destroy(tf_xent *plan);
/* The number of the device that the plan was made on, which has to be the current one of every call. */
tf_status tf_xent_device(const tf_xent *plan, int32_t *device);

/* loss and lse (n_rows floats each) of X (n_rows x n_in, rows ldx apart) and W (n_classes x n_in, rows ldw apart).  W is read fastest where its
 * rows begin at multiples of 16 bytes and are whole ones of them; with other rows, calls of many rows make a copy of it, piece by piece, and
 * so do calls of many fp32 rows.
 * Two executions of one plan must not overlap (they share its workspace). */
tf_status tf_xent_loss(const tf_xent *plan, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, int64_t n_rows,
                       float *loss, float *lse, void *hip_stream);
/* dX (n_rows x n_in, rows lddx apart) and dW (n_classes x n_in, rows lddw apart), either of which may be NULL, from the lse that
 * tf_xent_loss made and the gradient of each row's loss.  dX and dW are overwritten; they must not overlap X, W or each other. */
tf_status tf_xent_grad(const tf_xent *plan, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, const float *lse,
                       const float *dloss, int64_t n_rows, void *dX, int64_t lddx, void *dW, int64_t lddw, void *hip_stream);
/* The same from the loss that tf_xent_loss made as well: the label's part of g is then dloss[t] (exp(-loss[t]) - 1), which keeps its precision in rows that
 * are nearly certain of their label.  From lse alone it is off by 2^-24 |lse[t]| of dloss[t], more than itself where the loss is as small as that.
 * loss NULL: tf_xent_grad. */
tf_status tf_xent_grad_by_loss(const tf_xent *plan, const void *X, int64_t ldx, const void *W, int64_t ldw, const int32_t *labels, const float *loss,
                               const float *lse, const float *dloss, int64_t n_rows, void *dX, int64_t lddx, void *dW, int64_t lddw,
                               void *hip_stream);

/* Message for the most recent failure on the calling thread ("" if none). */
const char *tf_last_error(void);

/* Library version, "major.minor". */
const char *tf_version(void);

#ifdef __cplusplus
}
#endif
#endif /* TILEFUSION_H */
