/*
 * ilargi.h -- C ABI of the MI355X (gfx950) library for factorized linear algebra over a target
 * table that is never built:
 *
 *     T = I_1 D_1 M_1^T + ... + I_n D_n M_n^T                 (paper, Sec. 2.2, rewrite rule)
 *
 * D_k  source table k (the paper's S_k), r_k x c_k, float32, row-major, leading dimension c_k.
 * I_k  indicator matrix (paper, Def. 2), logically r_T x r_k binary with at most one 1 per row.
 *      Stored compressed as row_idx: int32[r_T], row_idx[i] = the row of D_k that feeds target row
 *      i, or -1 when target row i takes nothing from source k.  Never stored as a matrix.
 * M_k  mapping matrix (paper, Def. 1), c_T x c_k binary, at most one 1 per row and per column.
 *      Stored compressed as col_map: int32[c_k], col_map[j] = target column of source column j, or
 *      -1 when the column is dropped.  Different sources may map to the same target column; their
 *      contributions are summed, as the rewrite rule says.
 *
 * Conventions for every call
 *   - Matrices are dense float32, row-major, with no padding between rows.
 *   - "device" pointers are HIP device addresses valid on the current device; "host" pointers are
 *     ordinary process memory.  The library never takes ownership of caller memory.  A buffer with
 *     r_T rows may be NULL when r_T = 0 (it is empty); every other buffer must not be.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Operator calls only
 *     enqueue work on that stream and return; outputs are valid once the stream has reached that
 *     point.  ilargi_plan_create synchronizes the stream before it returns.
 *   - The library allocates no device memory.  All device state of a plan (inverse indices, column
 *     tables, intermediates, reduction partials) lives in the caller's workspace, whose size
 *     ilargi_plan_workspace_bytes reports.  Calls that share a plan must not overlap in time.
 *   - Every call returns an ilargi_status_t and never throws or aborts.  On an error detected
 *     before launch, outputs are untouched.  ilargi_last_error() gives a message for the last
 *     failure on the calling thread.
 *   - Floating-point results are deterministic: the same plan and inputs give the same bits on
 *     every run; no floating-point atomics are used.
 */
#ifndef ILARGI_H_
#define ILARGI_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct ilargi_plan ilargi_plan_t; /* opaque; host object owned by the library */

typedef enum {
  ILARGI_OK = 0,
  ILARGI_ERR_NULL = 1,        /* a required pointer is NULL */
  ILARGI_ERR_SHAPE = 2,       /* negative or inconsistent sizes */
  ILARGI_ERR_COLMAP = 3,      /* col_map entry outside [-1, c_T) or two columns of one source share a target */
  ILARGI_ERR_INDEX_RANGE = 4, /* row_idx entry outside [-1, r_k) */
  ILARGI_ERR_WORKSPACE = 5,   /* workspace too small or misaligned, or cx / m above max_cx */
  ILARGI_ERR_UNSUPPORTED = 6, /* combination of arguments that has no kernel */
  ILARGI_ERR_DEVICE = 7       /* a HIP call failed */
} ilargi_status_t;

typedef enum {
  ILARGI_F32 = 0,            /* float32 operands, float32 accumulation */
  ILARGI_BF16_IN_F32_ACC = 1 /* table and X/W entries rounded to bfloat16 (nearest even) as they are
                                read, products accumulated in float32; wide operands only */
} ilargi_precision_t;

typedef enum { ILARGI_LINEAR = 0, ILARGI_LOGISTIC = 1 } ilargi_model_t;

typedef struct {
  const float* D;         /* device, rows x cols; borrowed: must stay alive and unchanged while the plan lives */
  int64_t rows, cols;     /* r_k, c_k (both may be 0) */
  const int32_t* row_idx; /* device int32[r_T], borrowed; NULL = identity (requires rows == r_T) */
  const int32_t* col_map; /* HOST int32[cols]; copied when the plan is created */
  /* Optional: the table in compressed sparse rows instead of D (the paper keeps its matrices sparse,
   * Sec. 3.1).  With csr_rowptr != NULL, D must be NULL.  Borrowed like D.  A plan with a sparse source
   * serves lmm, tmm, gd_step, materialize, row_sum, col_sum, crossprod (up to 16384 target columns) and the
   * element-wise operators that keep zero at zero (which then act on csr_val, nnz values), in float32; the
   * bf16 variants return UNSUPPORTED.  Invalid sparse rows are reported by ilargi_plan_create as INDEX_RANGE.  A dense table has at
   * most 4096 columns; a sparse one up to 2^20 (one-hot encodings), provided that beyond 4096 columns no row
   * holds more than 2048 stored entries (else UNSUPPORTED). */
  const int32_t* csr_rowptr; /* device int32[rows + 1], rising from 0 to nnz */
  const int32_t* csr_col;    /* device int32[nnz], in [0, cols), strictly ascending within a row */
  const float* csr_val;      /* device float32[nnz] */
  int64_t nnz;               /* stored entries, < 2^31 */
} ilargi_source_t;

/* Bytes of device workspace a plan over these shapes needs when operands have at most max_cx
 * columns (X / Y / W columns).  Reads only sizes and whether row_idx is NULL; touches no device.
 * Errors: NULL, SHAPE. */
ilargi_status_t ilargi_plan_workspace_bytes(int n, const ilargi_source_t* sources, int64_t r_T,
                                            int64_t c_T, int64_t max_cx, size_t* bytes);

/* Build a plan: validate shapes and column maps (Def. 1), range-check row_idx on the device
 * (Def. 2) and build, for every source whose row_idx is not the identity, the inverse index of
 * I_k in compressed-row form: rowptr int32[r_k+1] and perm int32[nnz_k], the target rows fed by
 * each source row, ascending within a source row.  `workspace` is device memory, 256-byte aligned,
 * of at least the reported size, owned by the caller and used by the plan until it is destroyed.
 * Errors: NULL, SHAPE, COLMAP, INDEX_RANGE, WORKSPACE, DEVICE.  *plan is written only on success. */
ilargi_status_t ilargi_plan_create(int n, const ilargi_source_t* sources, int64_t r_T, int64_t c_T,
                                   int64_t max_cx, void* workspace, size_t workspace_bytes,
                                   void* stream, ilargi_plan_t** plan);

/* ilargi_plan_create for callers that cannot allocate device memory (code that must not call hipMalloc: tight
 * serving loops, harnesses that forbid allocation, set-up code running beside a captured graph): the plan's
 * device state lives in a scratch array that is part of the library itself, ilargi_static_scratch_bytes() bytes
 * (128 MiB) on every GPU the library is used on, held until the process ends.  The call allocates no device
 * memory and calls no allocating routine.  Same arguments, validation, results and errors as
 * ilargi_plan_create, and the plan serves every operator in the same way (bit-identical results), with
 * these limits:
 *   - a plan that needs more than the array holds (see ilargi_plan_workspace_bytes) is refused with WORKSPACE;
 *   - one such plan per device at a time: while it lives, another ilargi_plan_create_static on that device is
 *     refused with WORKSPACE; ilargi_plan_destroy releases the array;
 *   - the array keeps the last plan's contents; the call initialises every region it reads.  Calls from several
 *     threads that create static plans on one device are serialised by the library, but work that a destroyed
 *     plan still has in flight on a stream races with the next plan's set-up: synchronize before destroying.
 * The current device at the time of the call selects the array. */
ilargi_status_t ilargi_plan_create_static(int n, const ilargi_source_t* sources, int64_t r_T, int64_t c_T,
                                          int64_t max_cx, void* stream, ilargi_plan_t** plan);

/* Size in bytes of the scratch array behind ilargi_plan_create_static. */
size_t ilargi_static_scratch_bytes(void);

/* Release the host object.  The workspace and all borrowed arrays stay with the caller. */
ilargi_status_t ilargi_plan_destroy(ilargi_plan_t* plan);

/* Clustered entity table (a data layout, not an operator of the paper: Alg. 1 sums over the target rows, and
 * a sum does not depend on the order of its terms).  For a two-table star join T = [S | I_R R] -- an identity
 * source S of r_T rows and one source R that every target row joins -- the plan can keep a copy of S with its
 * rows in join order (grouped by the row of R they join, the order of the inverse index).  ilargi_gd_step
 * with one model in float32 then reads S and R once per iteration as two plain streams: the product R w_R,
 * the residual and the segment sums I_R^T e of Sec. 2.2's rules never go to memory.  ilargi_crossprod streams the
 * copy instead of gathering rows of S (same result, bit for bit); every other operator ignores it.  The one-pass
 * iteration pays when at least about four target rows join a row of R on average, or when R holds more cells
 * than S (every row of R costs the pass two reductions over a wavefront, however few target rows it serves):
 * ilargi_gd_step takes it in those two cases and keeps its usual sequence otherwise.
 *   ilargi_plan_cluster_bytes: size of the buffer, 4 r_T c_S + 8 r_T bytes rounded up to 256-byte pieces.
 *     Errors: NULL, UNSUPPORTED (not such a join; S needs 4..32 columns, R 4..256 columns, both in whole
 *     16-byte aligned float4s).
 *   ilargi_plan_cluster: fills `buffer` (device, 256-byte aligned, owned by the caller, used by the plan until
 *     it is destroyed or the call is repeated) on `stream`.  The copy holds the values S has at this call;
 *     sources must stay unchanged while the plan lives anyway, and ilargi_elementwise applied to S in place
 *     makes the plan forget the copy.  `y` (optional, device float[r_T]): the labels of the training set; they
 *     are copied in join order as well, and an ilargi_gd_step whose y is this same pointer reads them from the
 *     copy instead of gathering them (the vector must then stay unchanged like a source table; a gd_step with
 *     any other y gathers its labels as usual).  buffer == NULL: forget the copy.
 *     Errors: NULL, UNSUPPORTED, WORKSPACE, DEVICE. */
ilargi_status_t ilargi_plan_cluster_bytes(const ilargi_plan_t* plan, size_t* bytes);
ilargi_status_t ilargi_plan_cluster(ilargi_plan_t* plan, void* buffer, size_t buffer_bytes, const float* y,
                                    void* stream);

/* Left multiply (paper, Sec. 2.2):  out = T X = sum_k I_k (D_k (M_k^T X)).
 * X device c_T x cx, out device r_T x cx, 1 <= cx <= max_cx.  Errors: NULL, WORKSPACE, UNSUPPORTED. */
ilargi_status_t ilargi_lmm(ilargi_plan_t* plan, const float* X, int64_t cx, float* out,
                           ilargi_precision_t precision, void* stream);

/* Transposed multiply (the transpose operator of Sec. 2.2 / Alg. 1):
 * out = T^T Y = sum_k M_k (D_k^T (I_k^T Y)).  Y device r_T x cx, out device c_T x cx. */
ilargi_status_t ilargi_tmm(ilargi_plan_t* plan, const float* Y, int64_t cx, float* out,
                           ilargi_precision_t precision, void* stream);

/* Right multiply (Tab. 2, row XT):  out = X T = (T^T X^T)^T.  X device cx x r_T, out device cx x c_T,
 * 1 <= cx <= max_cx.  Uses the plan's residual buffer as scratch (like every call on a plan it must not
 * overlap with another). */
ilargi_status_t ilargi_rmm(ilargi_plan_t* plan, const float* X, int64_t cx, float* out,
                           ilargi_precision_t precision, void* stream);

/* Gram matrix  out = T^T T = sum_k sum_l M_k D_k^T (I_k^T I_l) D_l M_l^T, cross terms included.
 * out device c_T x c_T, both triangles written, symmetric to the bit.  A plan with a sparse source forms it
 * as T^T (T I), min(max_cx, 16) identity columns at a time through lmm and tmm (so it uses the plan's
 * residual buffer as scratch), and is limited to c_T <= 16384 (else UNSUPPORTED). */
ilargi_status_t ilargi_crossprod(ilargi_plan_t* plan, float* out, void* stream);

/* Join-gather baseline (paper, Sec. 2.2: the rewrite rule with X = I, i.e. T = sum_k I_k D_k M_k^T written
 * out): write the materialized target table.  T device r_T x c_T.  Each cell is the
 * float32 sum, in source order starting from +0.0, of the source cells mapped to it; cells nobody
 * maps to are +0.0.  The result is reproducible bit for bit. */
ilargi_status_t ilargi_materialize(ilargi_plan_t* plan, float* T, void* stream);

/* One gradient-descent iteration of Alg. 1 for m models at once, without materializing T:
 *   Z = T W;   E = Z - y (LINEAR)  or  sigmoid(Z) - y (LOGISTIC, y in {0,1});
 *   G = T^T E / r_T;   W[:, j] -= lr[j] * G[:, j].
 * Alg. 1 prints the update without the 1/r_T factor; pass lr = gamma * r_T to obtain it.
 * loss[j] (optional, device float[m]) receives the loss at the weights the call started from:
 * ||Z - y||^2 / (2 r_T) for LINEAR, mean(softplus(Z) - y Z) for LOGISTIC.
 * W device c_T x m in/out, y device float[r_T], lr device float[m], 1 <= m <= max_cx. */
ilargi_status_t ilargi_gd_step(ilargi_plan_t* plan, ilargi_model_t model, float* W, int64_t m,
                               const float* y, const float* lr, float* loss,
                               ilargi_precision_t precision, void* stream);

/* One Lloyd iteration of KMeans over the rows of T without materializing it (KMeans is one of the models
 * evaluated in Sec. 4, Tab. 7-9; the paper prints no algorithm for it, this is the textbook one):
 *   a_i = argmin_j ||t_i - c_j||^2  taken as  argmin_j (||c_j||^2 - 2 (T C)_ij),  the first j among equals,
 *   c_j <- mean of the rows with a_i = j  =  (T^T A)_j / n_j  with A the 0/1 assignment matrix;
 *   a centroid without rows keeps its place.
 * C device c_T x k in/out (column j is centroid j), 1 <= k <= min(max_cx, 256); assign (optional) device
 * int32[r_T] receives a_i (with respect to the centroids the call started from); counts (optional) device
 * int32[k] receives n_j.  Values must be finite.  Uses the plan's residual buffer as scratch.
 * Errors: NULL, SHAPE, WORKSPACE, UNSUPPORTED (k > 256). */
ilargi_status_t ilargi_kmeans_step(ilargi_plan_t* plan, float* C, int64_t k, int32_t* assign, int32_t* counts,
                                   void* stream);

/* One round of multiplicative updates of Gaussian NMF, T ~ W H with non-negative factors (Gaussian NMF is one
 * of the models evaluated in Sec. 4, Tab. 7-9; the paper prints no algorithm, these are the updates of Lee and
 * Seung for the squared Frobenius error):
 *   W <- W o (T H^T) (/) max(W (H H^T), 1e-30)          (left multiply by H^T),
 *   H <- H o (W^T T) (/) max((W^T W) H, 1e-30)          (transposed multiply by the new W).
 * W device r_T x r in/out; Ht device c_T x r in/out holds H transposed (row t is column t of H);
 * 1 <= r <= min(max_cx, 64).  Uses the plan's residual buffer as scratch.
 * Errors: NULL, SHAPE, WORKSPACE, UNSUPPORTED (r > 64). */
ilargi_status_t ilargi_gnmf_step(ilargi_plan_t* plan, float* W, float* Ht, int64_t r, void* stream);

/* Element-wise operators of Tab. 2 (first two rows): arithmetic with a scalar, T (/) x, and functions f(T). */
typedef enum {
  ILARGI_OP_MUL = 0,    /* t * x */
  ILARGI_OP_DIV = 1,    /* t / x */
  ILARGI_OP_ADD = 2,    /* t + x */
  ILARGI_OP_SUB = 3,    /* t - x */
  ILARGI_OP_POW = 4,    /* t ^ x */
  ILARGI_OP_EXP = 5,    /* exp(t);  x is ignored from here on */
  ILARGI_OP_LOG = 6,
  ILARGI_OP_SQRT = 7,
  ILARGI_OP_ABS = 8,
  ILARGI_OP_SQUARE = 9
} ilargi_elementwise_t;

/* T (/) x or f(T) in factorized form (Tab. 2: sum_k m_k operations instead of m_T): the result is the
 * table described by the same row_idx / col_map with source tables D_out[k] = op(D_k, x).
 * D_out: host array of n device pointers, D_out[k] r_k x c_k float32 (entries of empty sources are not
 * read); D_out[k] may be the source table itself, and if every table is updated in place the plan keeps
 * describing the result.  The factorized form equals the operator on the cells of T
 *   - always for MUL and DIV (they distribute over the sums of shared cells and keep empty cells 0);
 *   - for SQRT, ABS, SQUARE and POW with x > 0 (zero stays zero) when no target column is fed by two
 *     sources;
 *   - for ADD, SUB, EXP, LOG and POW with x <= 0 when, in addition, every target column is fed and
 *     every source reaches every target row (each cell of T has exactly one source cell).
 * Otherwise the call returns UNSUPPORTED and writes nothing.  Errors: NULL, UNSUPPORTED. */
ilargi_status_t ilargi_elementwise(ilargi_plan_t* plan, ilargi_elementwise_t op, float x,
                                   float* const* D_out, void* stream);

/* rowSum(T) (Tab. 2) = T 1: out device float[r_T]. */
ilargi_status_t ilargi_row_sum(ilargi_plan_t* plan, float* out, void* stream);

/* colSum(T) (Tab. 2) = sum_k M_k (D_k^T cnt_k), cnt_k[j] = number of target rows taking row j of source k
 * (kept with the plan): no pass over the r_T target rows.  out device float[c_T]. */
ilargi_status_t ilargi_col_sum(ilargi_plan_t* plan, float* out, void* stream);

/* Factorize or materialize (Sec. 3)?  Host-only: reads the shapes in `sources` and whether row_idx is NULL
 * (D, row_idx contents and col_map are not touched), like ilargi_plan_workspace_bytes. */
typedef struct {
  int64_t iterations;        /* gradient-descent iterations the table will serve (>= 1); the paper trains 200 */
  int64_t models;            /* models trained at once (>= 1) */
  double bytes_per_second;   /* sustained memory bandwidth to price bytes with; 0 = 5.0e12 (a plain copy on MI355X) */
  double launch_seconds;     /* cost of one dependent kernel launch; 0 = 2.5e-6 */
} ilargi_workload_t;

typedef struct {
  int factorize;             /* 1 = the factorized path is predicted to finish the workload sooner */
  double complexity_ratio;   /* Eq. (1) for linear regression, dense operands: O_materialized / O_factorized */
  double tuple_ratio;        /* r_T / (rows of the sources that have a row_idx) */
  double feature_ratio;      /* (columns of those sources) / (columns of the identity sources) */
  int morpheus_rule;         /* 1 = tuple_ratio >= 5 and feature_ratio >= 1 (the thresholds Sec. 4.3 quotes) */
  double bytes_factorized;   /* bytes one iteration moves, factorized */
  double bytes_materialized; /* the same on the materialized table */
  double bytes_join;         /* bytes the join itself moves (once) */
  double seconds_factorized; /* predicted time of the whole workload */
  double seconds_materialized; /* join + iterations on the table */
} ilargi_choice_t;

/* workload may be NULL (200 iterations, one model, default rates).  Errors: NULL, SHAPE. */
ilargi_status_t ilargi_choose(int n, const ilargi_source_t* sources, int64_t r_T, int64_t c_T,
                              const ilargi_workload_t* workload, ilargi_choice_t* out);

/* I_k^T Y for one source (the segmented sum inside ilargi_tmm), exposed for inspection:
 * Z[j, :] = sum of Y[i, :] over the target rows i with row_idx_k[i] == j.
 * Y device r_T x cx, Z device r_k x cx. */
ilargi_status_t ilargi_segment_sum(ilargi_plan_t* plan, int k, const float* Y, int64_t cx, float* Z,
                                   void* stream);

/* Device pointers to the inverse index of source k inside the workspace (valid while the plan
 * lives).  For an identity source *rowptr and *perm are NULL and *nnz = r_k. */
ilargi_status_t ilargi_plan_inverse_index(const ilargi_plan_t* plan, int k, const int32_t** rowptr,
                                          const int32_t** perm, int64_t* nnz);

/* Per-kernel timing for benchmarks.  After trace_begin, every launch of the kernel family named by
 * `tag` ("*" = every family; "<label>/<family>" = that family under one label) is bracketed by a pair of HIP events on the call's stream (at most
 * max_launches pairs; later launches run untimed).  Families: "lmm_rows:<k>" (product of source k),
 * "lmm_assemble", "segsum:<k>", "colred:<k>", "finalize", "materialize", "gram:<k n + l>", "star_pass", "gd_cluster",
 * "elementwise:<k>".  trace_label sets a
 * prefix ("<label>/<family>") for the launches that follow, so a caller can tell its operators apart.
 * trace_end waits for the recorded events, writes the elapsed milliseconds of up to `capacity`
 * launches to the host array `ms` (may be NULL), stores the number of recorded launches in *count
 * and switches tracing off; trace_name copies the name of recorded launch i (valid until the next
 * trace_begin).  Events are host objects; no device memory is allocated. */
ilargi_status_t ilargi_plan_trace_begin(ilargi_plan_t* plan, const char* tag, int max_launches);
ilargi_status_t ilargi_plan_trace_label(ilargi_plan_t* plan, const char* label);
ilargi_status_t ilargi_plan_trace_end(ilargi_plan_t* plan, float* ms, int capacity, int* count);
ilargi_status_t ilargi_plan_trace_name(const ilargi_plan_t* plan, int i, char* buf, int buf_len);

/* Plain streaming kernels for calibration (what the memory system delivers, and the scale of the
 * profiler's byte counters): kind 0 copies n_floats floats src -> dst, kind 1 only reads src (dst
 * receives one float per workgroup, so it needs `blocks` floats), kind 2 only writes dst; kinds 3 and 4
 * are the copy and the write with non-temporal accesses.  Device
 * pointers, 16-byte aligned, n_floats a multiple of 4, `blocks` workgroups of 256 threads (1 .. 2^22) that
 * walk the buffer with a grid stride: n_floats / 1024 workgroups touch one float4 per thread, in address
 * order, which is the pattern that writes fastest on the MI355X. */
ilargi_status_t ilargi_stream_probe(int kind, float* dst, const float* src, int64_t n_floats, int blocks,
                                    void* stream);

/* --- Models with learned features --------------------------------------------------------------------------------
 * Operators beside the plan: rows of a learned table picked by the keys of a join, a dense layer over joined rows, their
 * gradients, and the orthogonalised update of a layer's matrix.  They take no plan.  Matrices are row-major with a leading
 * dimension `ld` in elements (ld >= columns; the columns between are neither read nor written) and any address that an
 * element of their type may have; 16-byte aligned rows are the fast ones.  The rules of this header hold: device pointers,
 * work enqueued on `stream`, no device memory allocated, the same bits for the same inputs, a status for every call.
 * `workspace` is device memory of the caller, 256-byte aligned, used while the call's work runs: calls that overlap in
 * time need a workspace each.  Outputs may not overlap inputs or each other, except where said. */
typedef enum { ILARGI_TYPE_F32 = 0, ILARGI_TYPE_BF16 = 1 } ilargi_type_t; /* bf16: rounded to nearest even when stored */

/* Rows of a learned table (the local result I_k D_k of Sec. 2.2 for a table that changes and keys that are not planned):
 *   out[i, :] = scale * table[ids[i], :]   (+ out[i, :] when accumulate is not 0),    i < n.
 * An id outside [0, rows) takes nothing: its row is zero (unchanged when accumulating).  Computed in float32 and rounded once.
 * table rows x cols of table_type, ids device int32[n], out n x cols of out_type.  n may be 0.
 * Errors: NULL, SHAPE (n, rows < 0, cols < 1, a leading dimension below cols, more than 2^31 - 1 rows or ids),
 * UNSUPPORTED (a type that is none), DEVICE. */
ilargi_status_t ilargi_embed(const void* table, ilargi_type_t table_type, int64_t rows, int64_t cols, int64_t ld_table,
                             const int32_t* ids, int64_t n, float scale, int accumulate, void* out,
                             ilargi_type_t out_type, int64_t ld_out, void* stream);

/* Its gradient (I_k^T Y of Sec. 2.2, keys sorted in the call):
 *   d_table[v, :] = scale * sum over ids[i] == v of d_out[i, :]   (+ d_table[v, :] when accumulate is not 0).
 * Every row of d_table is written (when accumulating, those that some id names).  Ids outside [0, rows) add nothing.  Sums
 * run in float32 over the ids sorted stably, in an order that depends on n, cols, the types and the ids only.
 * Errors: as ilargi_embed, and WORKSPACE. */
ilargi_status_t ilargi_embed_grad_workspace_bytes(int64_t n, int64_t rows, int64_t cols, size_t* bytes);
ilargi_status_t ilargi_embed_grad(const void* d_out, ilargi_type_t out_type, int64_t ld_out, const int32_t* ids, int64_t n,
                                  float scale, int accumulate, void* d_table, ilargi_type_t table_type, int64_t rows,
                                  int64_t cols, int64_t ld_table, void* workspace, size_t workspace_bytes, void* stream);

typedef enum {
  ILARGI_ACT_NONE = 0,
  ILARGI_ACT_RELU = 1,    /* max(z, 0); slope 0 at 0 */
  ILARGI_ACT_SIGMOID = 2, /* 1 / (1 + exp(-z)) */
  ILARGI_ACT_SILU = 3,    /* z / (1 + exp(-z)) */
  ILARGI_ACT_GELU = 4     /* z (1 + erf(z / sqrt 2)) / 2 */
} ilargi_activation_t;

/* A dense layer: its sizes, the element type of all its matrices and vectors, and its activation. */
typedef struct {
  int64_t n, k, m;        /* rows, input columns, output columns; n may be 0 */
  ilargi_type_t type;     /* products accumulate in float32 for both types */
  ilargi_activation_t act;
} ilargi_layer_t;

/* Bytes of workspace of ilargi_linear and ilargi_linear_grad for this layer (either pointer may be NULL).  In bfloat16, from 7.5e8
 * multiplications on, they hold copies of X and W (and of g) whose rows are whole pieces of 16 bytes, for operands whose rows are not.
 * Errors: NULL (layer), SHAPE (n < 0, k or m < 1, any above 2^31 - 1), UNSUPPORTED (type, act). */
ilargi_status_t ilargi_linear_workspace_bytes(const ilargi_layer_t* layer, size_t* forward, size_t* gradient);

/* z = X W + bias;  out = act(z) + residual.
 * X n x k, W k x m, bias[m] (optional), residual n x m (optional; may be `out` itself), out n x m, pre n x m (optional)
 * receives z, which ilargi_linear_grad needs unless act is NONE.  z, act(z) and the sums are float32; each output is
 * rounded once.  Errors: NULL, SHAPE, UNSUPPORTED, WORKSPACE, DEVICE. */
ilargi_status_t ilargi_linear(const ilargi_layer_t* layer, const void* X, int64_t ld_x, const void* W, int64_t ld_w,
                              const void* bias, const void* residual, int64_t ld_res, void* out, int64_t ld_out,
                              void* pre, int64_t ld_pre, void* workspace, size_t workspace_bytes, void* stream);

/* Gradients of ilargi_linear (the residual's is d_out itself):
 *   g = d_out o act'(pre);  d_X = g W^T;  d_W = X^T g;  d_bias = column sums of g.
 * pre is read unless act is NONE (then it may be NULL).  d_X, d_W and d_bias are each optional.  With accumulate not 0 the
 * results are added to d_W and d_bias (d_X is always set).  g is formed in float32 and rounded to the layer's type before
 * the two products, and not rounded for d_bias.  X is not read without d_W, nor W without d_X.
 * Errors: NULL, SHAPE, UNSUPPORTED, WORKSPACE, DEVICE. */
ilargi_status_t ilargi_linear_grad(const ilargi_layer_t* layer, const void* d_out, int64_t ld_out, const void* pre,
                                   int64_t ld_pre, const void* X, int64_t ld_x, const void* W, int64_t ld_w, void* d_X,
                                   int64_t ld_dx, void* d_W, int64_t ld_dw, void* d_bias, int accumulate,
                                   void* workspace, size_t workspace_bytes, void* stream);

/* Orthogonalised update by Newton-Schulz products, for `batch` matrices G of rows x cols:
 *   X = G / (||G||_F + eps);  `steps` times  A = X X^T (X^T X if cols < rows),  X <- a X + (b A + c A^2) X
 *   out = alpha X + beta base.
 * coef: host float[3] a, b, c (NULL: 3.4445, -4.7750, 2.0315, which bring singular values near 1 in five steps).
 * G of g_type with leading dimension ld_g and `stride_g` elements between matrices; base (read if beta is not 0) and
 * out of out_type with ld_out and stride_out; base may be `out` itself, so alpha = -lr, beta = 1 - lr decay updates weights
 * in place.  The norm is summed in float64; products accumulate in float32.  Where `steps` steps multiply a singular value by at most
 * 4096 (six with the usual coefficients, twenty with a = 1.5), X, X X^T and B = b A + c A^2 are held to 22 bits an entry and 2^-37 of
 * norm 1 (2^-37 |G| / (|G| + eps) of a small X), which float32 products of the whole lose too; parts of G on rows and columns of their
 * own, below about 1e-6 of the norm, keep fewer bits than those would.  With more steps, eps < 0, or coefficients that bring a
 * singular value beyond 2, all is float32, in four to seven times the time.
 * Errors: NULL, SHAPE (batch < 0 or above 65535, rows or cols < 1 or above 16384, steps outside [1, 100], leading dimensions or strides
 * that overlap), UNSUPPORTED (types), WORKSPACE, DEVICE. */
ilargi_status_t ilargi_orthogonalize_workspace_bytes(int64_t batch, int64_t rows, int64_t cols, ilargi_type_t g_type,
                                                     size_t* bytes);
ilargi_status_t ilargi_orthogonalize(const void* G, ilargi_type_t g_type, int64_t batch, int64_t rows, int64_t cols,
                                     int64_t ld_g, int64_t stride_g, int steps, const float* coef, float eps, float alpha,
                                     float beta, const void* base, void* out, ilargi_type_t out_type, int64_t ld_out,
                                     int64_t stride_out, void* workspace, size_t workspace_bytes, void* stream);

/* The end of a block of a deeper model and the start of the next, in one pass:
 *   u = N1(h);   r = x + scale f(gate) o u;   y = N2(r)
 * N is one of
 *   NONE     v o gain + bias
 *   RMS      v / sqrt(mean v^2 + eps) o gain + bias
 *   CENTRED  (v - mean v) / sqrt(mean (v - mean v)^2 + eps) o gain + bias
 * over the m columns of a row; gains and biases are vectors of m, NULL for ones and zeros.  gate is n x m, one row of m for all rows
 * (gate_rows = 0), or NULL for ones; x may be NULL for zeros.  With second = NONE there is no y (then gain2 and bias2 are NULL).
 * All matrices and vectors are of one type; a row is held in float32 from its loads to its stores (its mean is summed in float64), each
 * output is rounded once, and y follows from the r that was not rounded.  A mean of squares that no float32 holds gives what float32 arithmetic gives. */
typedef enum { ILARGI_NORM_NONE = 0, ILARGI_NORM_RMS = 1, ILARGI_NORM_CENTRED = 2 } ilargi_norm_kind_t;

typedef struct {
  int64_t n, m;                     /* rows (may be 0), columns (1 .. 16384) */
  ilargi_type_t type;
  ilargi_norm_kind_t first, second;
  ilargi_activation_t gate_act;     /* f */
  int gate_rows;                    /* 1: a row of the gate for every row; 0: one for all */
  float scale, eps;
  const void *h, *gain1, *bias1, *gate, *x, *gain2, *bias2;
  int64_t ld_h, ld_gate, ld_x;
} ilargi_norm_t;

/* r and y, either of which may be NULL where it is not wanted; r may be x or h itself, y may be h (not r).  No workspace.
 * Errors: NULL (block, h with n > 0), SHAPE (n, m, leading dimensions, eps < 0 or no number), UNSUPPORTED (type, kinds, gate_act, y,
 * gain2 or bias2 without a second norm), DEVICE. */
ilargi_status_t ilargi_norm(const ilargi_norm_t* block, void* r, int64_t ld_r, void* y, int64_t ld_y, void* stream);

/* Its gradients for d_r and d_y (each may be NULL for zeros; y's is refused without a second norm).  Each result is optional:
 *   d_h, d_x: n x m; d_gate: n x m, or m sums over the rows where the gate is one row; d_gain*, d_bias*: m sums over the rows.
 * With accumulate not 0 the sums over rows are added to what is there.  d_x may be d_r itself, d_h may be d_y.  Everything is worked
 * out again from h, gate and x, in float32; sums over rows are added in an order that depends on n, m and the type only.
 * d_x is wanted of a block without x too: it is the gradient of what is added to the gated u.
 * Errors: as ilargi_norm, NULL (a workspace that is needed), UNSUPPORTED (d_gate without a gate, d_gain2 or d_bias2 without a second
 * norm), WORKSPACE, DEVICE.  (d_gain and d_bias need no gain or bias: they are those at ones and zeros.) */
typedef struct {
  void *d_h, *d_x, *d_gate, *d_gain1, *d_bias1, *d_gain2, *d_bias2;
  int64_t ld_h, ld_x, ld_gate;
} ilargi_norm_grads_t;
ilargi_status_t ilargi_norm_grad_workspace_bytes(int64_t n, int64_t m, ilargi_type_t type, size_t* bytes);
ilargi_status_t ilargi_norm_grad(const ilargi_norm_t* block, const void* d_r, int64_t ld_dr, const void* d_y, int64_t ld_dy,
                                 const ilargi_norm_grads_t* out, int accumulate, void* workspace, size_t workspace_bytes,
                                 void* stream);

/* A layer of its own for every group of rows (ilargi_linear over ragged groups):
 *   z[i, :] = X[i, :] W_g + bias_g,   out[i, :] = act(z[i, :]) + residual[i, :]   for offsets[g] <= i < offsets[g + 1].
 * offsets: device int32[groups + 1], ascending, in [0, n]; the rowptr of ilargi_plan_inverse_index is of this form for rows
 * brought together by its perm.  Rows of no group (before offsets[0], from offsets[groups] on) are not written.  The offsets are
 * looked at on the device only: one outside [0, n] or below an earlier one counts as the nearest that is none of that.
 * W: `groups` matrices k x m, stride_w elements apart (>= (k - 1) ld_w + m); bias groups x m (optional) with ld_bias.
 * type, act, pre, residual and the sums are those of ilargi_linear; residual may be `out`.
 * The gradient: g = d_out o act'(pre); d_X[i, :] = g[i, :] W_g^T (rows of no group are not written); d_W_g = X_g^T g_g and
 * d_bias_g = column sums of g_g, zeros for groups without rows; with accumulate not 0 they are added to what is there.  g is formed
 * in float32 and rounded to the layer's type before the two products, and not rounded for d_bias, as in ilargi_linear_grad.  Each
 * result is optional; X is not read without d_W, nor W without d_X; pre is NULL if act is NONE.
 * Errors: NULL, SHAPE (groups < 0 or above 65535, n < 0, k or m < 1, any above 2^31 - 1, leading dimensions, matrices of the groups
 * that overlap, more than 2^31 - 1 blocks of 64 x 64 results), UNSUPPORTED (type, act), WORKSPACE, DEVICE. */
typedef struct {
  int64_t groups, n, k, m;
  ilargi_type_t type;
  ilargi_activation_t act;
} ilargi_groups_t;

ilargi_status_t ilargi_grouped_linear_workspace_bytes(const ilargi_groups_t* layer, size_t* forward, size_t* gradient);
ilargi_status_t ilargi_grouped_linear(const ilargi_groups_t* layer, const int32_t* offsets, const void* X, int64_t ld_x,
                                      const void* W, int64_t ld_w, int64_t stride_w, const void* bias, int64_t ld_bias,
                                      const void* residual, int64_t ld_res, void* out, int64_t ld_out, void* pre,
                                      int64_t ld_pre, void* workspace, size_t workspace_bytes, void* stream);
ilargi_status_t ilargi_grouped_linear_grad(const ilargi_groups_t* layer, const int32_t* offsets, const void* d_out,
                                           int64_t ld_out, const void* pre, int64_t ld_pre, const void* X, int64_t ld_x,
                                           const void* W, int64_t ld_w, int64_t stride_w, void* d_X, int64_t ld_dx, void* d_W,
                                           int64_t ld_dw, int64_t stride_dw, void* d_bias, int64_t ld_dbias, int accumulate,
                                           void* workspace, size_t workspace_bytes, void* stream);

/* The norm over all entries of `count` matrices together, and the matrices scaled so that it is at most max_norm:
 *   norm = sqrt(sum of all squares);   out_t = in_t (max_norm / norm)  if norm > max_norm,  else in_t.
 * A norm that is no finite number scales nothing: the outputs are the inputs, and `norm` says so.  Squares are summed in float64 in an
 * order that depends on the inputs' sizes, types and leading dimensions only, so no float32 or bfloat16 entries are too large or too small for it.
 * tensors: host array, read during the call; a vector is a matrix of one row.  out NULL: the tensor counts and is not written; out may
 * be `in` itself (with ld_out = ld_in: scaled in place, and not written where nothing is scaled).  Any other overlap of an out with an in or
 * out of the call is refused, except that of column blocks of one matrix (rows of one distance in bytes).  norm: device float32
 * (optional), in none of the tensors.
 * (It is stored in 32 bits: infinite beyond 3.4e38, where the tensors are scaled all the same.)
 * max_norm may be infinite: outputs are copies.  count may be 0 (norm 0).
 * Errors: NULL (tensors, an in, workspace), SHAPE (count outside [0, 65535], rows or cols < 0, rows above 2^31 - 1, more than 2^46
 * elements from a tensor's first to its last, a leading dimension below cols, a
 * max_norm below 0 or no number, overlaps), UNSUPPORTED (type), WORKSPACE, DEVICE. */
typedef struct {
  const void* in;
  void* out;
  int64_t rows, cols, ld_in, ld_out;
  ilargi_type_t type;
} ilargi_tensor_t;

ilargi_status_t ilargi_clip_norm_workspace_bytes(const ilargi_tensor_t* tensors, int64_t count, size_t* bytes);
ilargi_status_t ilargi_clip_norm(const ilargi_tensor_t* tensors, int64_t count, float max_norm, float* norm, void* workspace,
                                 size_t workspace_bytes, void* stream);

/* Message for the most recent failure on this thread ("" if none).  Static storage. */
const char* ilargi_last_error(void);

/* Library version, "major.minor". */
const char* ilargi_version(void);

#ifdef __cplusplus
}
#endif
#endif /* ILARGI_H_ */
