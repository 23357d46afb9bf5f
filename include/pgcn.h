/*
 * pgcn.h — C ABI of libpgcn: one partition's PipeGCN training step on
 * AMD Instinct MI355X (gfx950).
 *
 * The operations follow the paper "PipeGCN: Efficient Full-Graph Training of
 * Graph Convolutional Networks with Pipelined Feature Communication"
 * (ICLR 2022):
 *   - Algorithm 1 (per-partition view): set-up of the inner, boundary and
 *     send sets; forward, loss, backward, AllReduce and SGD per iteration;
 *   - Section 3.2: the mean aggregator with one-iteration-stale boundary
 *     features and boundary feature gradients;
 *   - Section 3.4: moving-average smoothing of stale features and gradients;
 *   - Appendix A.1: the layer function Z = P H W, H' = σ(Z) and its two
 *     gradients, with P split into intra- and inter-partition parts.
 *
 * Conventions shared by every call
 * --------------------------------
 * Status:    every int-returning call returns PGCN_OK (0) or a PGCN_E* code;
 *            pgcn_last_error() gives a thread-local message for the last
 *            failure.  No C++ exception crosses this interface.
 * Memory:    the caller owns every activation, weight, gradient and buffer
 *            (device memory, fp32 unless stated).  The library owns only the
 *            partition handle's index arrays.  Scratch memory is passed in as
 *            `workspace` (size from pgcn_workspace_size()).
 * Layout:    dense matrices are row-major with an explicit row stride `ld`
 *            (in elements).  fp32 matrices read by the aggregation kernels
 *            need ld % 4 == 0 and 16-byte aligned bases; bf16 matrices need
 *            ld % 8 == 0.  Columns [f, ld) are padding: never read as data;
 *            the aggregation kernels write zeros there.  Weight matrices W
 *            and weight gradients dW are compact [f_in x f_out].
 * Streams:   compute calls only enqueue work on the given stream; nothing
 *            synchronises the host except pgcn_partition_setup/destroy.
 * Threads:   a partition handle is immutable after set-up; concurrent calls
 *            on different streams with disjoint outputs and workspaces are
 *            safe.
 * Determinism: no floating-point atomics are used; results are bitwise
 *            reproducible for identical inputs and launch configuration.
 */
#ifndef PGCN_H
#define PGCN_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

#define PGCN_VERSION 165

enum pgcn_status {
  PGCN_OK = 0,
  PGCN_EINVAL = 1,        /* null pointer, bad size, bad stride, bad enum       */
  PGCN_ENOMEM = 2,        /* device or host allocation failed during set-up     */
  PGCN_EHIP = 3,          /* a HIP runtime call failed (message has its text)   */
  PGCN_EUNSUPPORTED = 4,  /* device is not gfx950, or an unsupported combination */
  PGCN_EWORKSPACE = 5     /* workspace missing or smaller than required          */
};

/* Arithmetic of the update GEMMs.  PGCN_F32: fp32 operands, fp32 results
 * and fp32 accumulation.  Each product is formed from an exact split of
 * both fp32 operands into three bf16 parts (x = hi + mid + lo), six part
 * products each, on the bf16 matrix cores.  Each part product is exact in
 * fp32, and the three dropped ones are together below 2^-21 (1 + 2^-7) of
 * the product, so results carry fp32 accuracy.  The environment variable
 * PGCN_GEMM_F32=native (read per call) selects the fp32 matrix cores
 * instead.  A non-finite operand gives a non-finite (NaN) result.
 * PGCN_BF16: operands rounded once to bf16 (nearest even), products
 * accumulated in fp32.
 * PGCN_MXFP4 (pgcn_layer_fwd alone, aggregate first): both operands in the
 * 4 bits of PGCN_MX_FP4, quantised along f_in in the call, products
 * accumulated in fp32.  The layer's backward then runs in one of the others,
 * with A as it was before it was quantised. */
enum pgcn_dtype { PGCN_F32 = 0, PGCN_BF16 = 1, PGCN_MXFP4 = 2 };

enum pgcn_setup_flags {
  PGCN_SETUP_HOST_ONLY = 1,     /* build the index structures on the host only: no
                                   device upload; compute calls on such a handle
                                   return PGCN_EINVAL (used to test the builder
                                   without a GPU) */
  PGCN_SETUP_NO_SELF_LOOP = 2,  /* P_i is the mean over N(v) without the self loop
                                   (the GraphSAGE layer's aggregation, Section 2):
                                   entries 1/d_v with d_v = degree; a row without
                                   neighbours is zero.  The sets V_i, B_i, S_{i,j}
                                   are unchanged. */
  PGCN_SETUP_SYMMETRIC = 4      /* P_i is the symmetric normalisation of Appendix
                                   A.1, rows of D̃^{-1/2} (A + I) D̃^{-1/2}: entries
                                   1 / sqrt(d̃_v d̃_u) with d̃ the whole-graph degree + 1
                                   of every inner and boundary node (the boundary
                                   nodes' degrees come from their full rows of the
                                   global CSR).  GCN layers only; not with
                                   PGCN_SETUP_NO_SELF_LOOP. */
};

enum pgcn_pack_kind {
  PGCN_PACK_FEAT = 0,     /* dst[k, :] = src[send_idx[k], :] for k in [0, n_send)       */
  PGCN_ACCUM_GRAD = 1     /* dst[u, :] += sum_{k : send_idx[k] == u} src[k, :], ascending k */
};

enum pgcn_loss_kind { PGCN_SOFTMAX_CE = 0, PGCN_SIGMOID_BCE = 1 };

/* Association in which a GCN layer evaluates its product P H W (Appendix
 * A.1's layer function; the paper fixes none): aggregate first, (P H) W, or
 * transform first, P (H W), which aggregates f_out instead of f_in columns
 * and pays when the layer narrows (f_out < f_in). */
enum pgcn_layer_order { PGCN_ORDER_AGG = 0, PGCN_ORDER_TRANSFORM = 1 };

/* Global graph on the host.  Must be symmetric (u in N(v) <=> v in N(u)).
 * Duplicate entries and self loops are allowed and removed; exactly one
 * self loop per inner row is added (Ã = A + I, Appendix A.1) unless the
 * partition is built with PGCN_SETUP_NO_SELF_LOOP. */
typedef struct {
  int64_t n;               /* global node count                     */
  const int64_t *rowptr;   /* [n+1], rowptr[0] == 0, non-decreasing */
  const int32_t *col;      /* [rowptr[n]], values in [0, n)         */
} pgcn_csr;

/* Which partition owns each node (Algorithm 1's input: partition id i, count n). */
typedef struct {
  int32_t nparts;          /* partition count, >= 1                 */
  int32_t self;            /* the partition to build, in [0, nparts) */
  const int32_t *owner;    /* [n] host, values in [0, nparts)        */
} pgcn_boundary_map;

typedef struct pgcn_partition pgcn_partition;

/* Tuning overrides (environment variables; none is needed for correct use):
 *   PGCN_AGG_CHUNKS    column chunks of the aggregation plans, 1..64 (read by
 *                      pgcn_partition_setup; default: about 8,000 gathered rows
 *                      per chunk, 32,000 for rows of at most 64 floats, while
 *                      rows keep >= 32 non-zeros per chunk);
 *   PGCN_AGG_CHUNKS_T  the same for the plans of P_i^T alone (takes precedence);
 *   PGCN_AGG_CHUNKS_NARROW  the same for the plans of rows of at most 64 floats
 *                      (takes precedence over both);
 *   PGCN_AGG_SLICED    0 / 1: never / always aggregate rows wider than 64 floats with the
 *                      kernel of L2-resident row slices, over a plan of its own (read by
 *                      pgcn_partition_setup; default: on matrices of at least 2^20
 *                      non-zeros, for widths, strides, alignments and source sizes
 *                      where that is faster, chunks of about 11,000 rows, none across
 *                      the inner and boundary rows; PGCN_AGG_CHUNKS and
 *                      PGCN_AGG_CHUNKS_T give plain plans alone unless this is 1).
 *                      Sources of 4 GiB and more always take the plain plan;
 *   PGCN_SEGMENT       length at which long rows are split into segments,
 *                      16..1048576 (read by pgcn_partition_setup; default 512; at
 *                      least twice that in sliced plans);
 *   PGCN_AGG_SLICE_F4  float4 columns per lane slice of the plain aggregation: 16, 32
 *                      or 64 (read per call; default 64);
 *   PGCN_TN_BM=128     keeps the fp32 weight-gradient GEMM in 128-row tiles
 *                      (read once; default: 256-row tiles for f_in >= 384);
 *   PGCN_GEMM_F32=native  fp32 update GEMMs on the fp32 matrix cores instead of
 *                      by bf16 parts (read per call; see pgcn_dtype);
 *   PGCN_HUB=0         no dense block on the matrix cores (read by
 *                      pgcn_partition_setup; default: a block of the rows with
 *                      the most non-zeros x the most referenced columns where it
 *                      saves >= 5% of the gathers, reported by pgcn_info);
 *   PGCN_HUB_ROWS, PGCN_HUB_COLS  both > 0: force the block to that many rows
 *                      and columns (clamped to the matrix).
 * Chunks, segments and the dense block set the order in which a row's terms are
 * added (results stay deterministic for a given setting, row width, stride and
 * alignment); the slice width and PGCN_TN_BM change only speed; PGCN_GEMM_F32
 * changes the order of the GEMMs' fp32 sums within the same rounding bound. */

/* Largest layer width (f_in, f_out) the layer entry points accept: the
 * aggregation covers a row in at most 32 launches of up to 512 float4
 * columns.  Wider layers are rejected with PGCN_EINVAL before any launch. */
#define PGCN_MAX_WIDTH 63740

/* Sizes of a built partition. */
typedef struct {
  int64_t n_inner;         /* |V_i|                                           */
  int64_t n_bd;            /* |B_i|                                           */
  int64_t nnz;             /* non-zeros of P_i (with one self loop per inner row
                              unless built with PGCN_SETUP_NO_SELF_LOOP)      */
  int64_t n_send;          /* sum_j |S_{i,j}|                                 */
  int64_t max_row_len;     /* longest row of P_i                              */
  int64_t max_row_len_t;   /* longest row of P_i^T                            */
  int32_t nparts;
  int32_t self;
  int32_t host_only;       /* 1 if built with PGCN_SETUP_HOST_ONLY            */
  int32_t spmm_segment;    /* runs longer than this are split (fixed order); at
                              least twice this in sliced plans                */
  int64_t spmm_items;      /* work items of the forward aggregation (here and
                              below: of the sliced plan where there is one)   */
  int64_t spmm_split_slots;/* partial-sum slots of split rows (forward)       */
  int64_t spmmt_items;     /* work items of the transposed aggregation        */
  int64_t spmmt_split_slots;
  int32_t spmm_chunks;     /* column chunks (cache blocking) of P_i           */
  int32_t spmmt_chunks;    /* column chunks of P_i^T                          */
  int32_t symmetric;       /* 1 if built with PGCN_SETUP_SYMMETRIC            */
  int32_t self_loop;       /* 0 if built with PGCN_SETUP_NO_SELF_LOOP         */
  int32_t spmm_chunks_narrow;  /* column chunks of P_i when the aggregated rows
                                  have at most 64 floats                      */
  int32_t spmmt_chunks_narrow; /* the same for P_i^T                          */
  int32_t spmm_hub_rows;   /* rows x columns of the dense block of P_i taken  */
  int32_t spmm_hub_cols;   /* by the matrix cores (0: none)                   */
  int64_t spmm_hub_nnz;    /* its non-zeros                                   */
  int32_t spmmt_hub_rows;  /* the same for P_i^T                              */
  int32_t spmmt_hub_cols;
  int64_t spmmt_hub_nnz;
} pgcn_info;

/* Caller-allocated host buffers for pgcn_partition_export, sized from pgcn_info.
 * Local numbering: inner local id = rank of the global id among owner == self;
 * boundary local id = n_inner + rank by (owner, global id).  Rows of P_i and
 * P_i^T list columns in ascending local id.  The send list holds S_{i,j} for
 * ascending j, each in ascending global id. */
typedef struct {
  int64_t *inner_gid;      /* [n_inner]                       */
  int64_t *bd_gid;         /* [n_bd]                          */
  int64_t *recv_ptr;       /* [nparts+1] boundary rows of owner j: [recv_ptr[j], recv_ptr[j+1]) */
  int64_t *rowptr;         /* [n_inner+1]                     */
  int32_t *col;            /* [nnz]                           */
  int64_t *rowptr_t;       /* [n_inner+n_bd+1]                */
  int32_t *col_t;          /* [nnz]                           */
  int64_t *send_ptr;       /* [nparts+1]                      */
  int32_t *send_idx;       /* [n_send] inner local ids        */
  int64_t *inv_ptr;        /* [n_inner+1]                     */
  int32_t *inv_k;          /* [n_send] positions into send_idx, ascending per row */
  int64_t *deg;            /* [n_inner+n_bd] whole-graph degree + 1 (distinct
                              neighbours, no self loop, plus one) */
} pgcn_arrays;

/*
 * Partition set-up (Algorithm 1, set-up block; Section 3.1).
 * Builds V_i, B_i, the CSR of P_i (entries 1/d_v, d_v = row length = degree
 * + 1), its transpose, the send sets S_{i,j} = B_j ∩ V_i, the inverse send
 * map and the fixed-order work plan of the aggregation kernels; uploads them
 * to the current device.  Host-synchronous.  `flags` is a mask of
 * pgcn_setup_flags.  On success *out receives a handle freed by
 * pgcn_partition_destroy.  Errors: PGCN_EINVAL (bad graph or map),
 * PGCN_ENOMEM, PGCN_EHIP, PGCN_EUNSUPPORTED (current device not gfx950).
 */
int pgcn_partition_setup(const pgcn_csr *csr, const pgcn_boundary_map *bmap, uint32_t flags,
                         pgcn_partition **out);
int pgcn_partition_info(const pgcn_partition *part, pgcn_info *out);
/* Copies every index array into caller buffers (host).  Any member may be NULL to skip it. */
int pgcn_partition_export(const pgcn_partition *part, const pgcn_arrays *host_out);
void pgcn_partition_destroy(pgcn_partition *part);

/* Bytes of workspace that pgcn_layer_fwd / pgcn_layer_bwd / pgcn_loss_fwd_bwd need
 * for these widths (the maximum over the three), aggregate-first layers. */
size_t pgcn_workspace_size(const pgcn_partition *part, int32_t f_in, int32_t f_out, int32_t gemm_dtype);
/* The same for a GCN or GraphSAGE layer evaluated in `order`
 * (pgcn_layer_order); returns 0 for a bad order.  PGCN_ORDER_AGG gives
 * pgcn_workspace_size. */
size_t pgcn_layer_workspace_size(const pgcn_partition *part, int32_t f_in, int32_t f_out, int32_t gemm_dtype,
                                 int32_t order);

/*
 * One layer forward (Algorithm 1's forward update; Section 3.2 forward
 * equation; Appendix A.1 layer function):
 *     A = P_i [H_in ; H_bd]        fresh inner rows, stale boundary rows
 *     Z = A W ;  H_out = relu(Z) if relu else Z
 * H_bd holds the boundary rows to use (the received stale buffer, or its
 * smoothing state); NULL means all-zero boundary rows (iteration 1).
 * With gemm_dtype == PGCN_BF16, A is rounded once to bf16 (round to nearest
 * even) into A_bf16, W is rounded to bf16 and the product accumulates in
 * fp32; A (fp32) may then be NULL, or A_bf16 may be NULL when A is given
 * (A is then rounded while staged: the same values).  With PGCN_F32, A is
 * required and A_bf16 ignored.
 * order == PGCN_ORDER_TRANSFORM evaluates the same layer as
 *     Y = [H_in ; H_bd] W            (n_inner + n_bd rows, in the workspace)
 *     H_out = relu(P_i Y) if relu else P_i Y
 * (bf16 path: H and W rounded to bf16, fp32 accumulation; the aggregation
 * stays fp32).  A and A_bf16 are then unused and may be NULL; the backward
 * takes the layer input instead.  Workspace: pgcn_layer_workspace_size with
 * the same order.
 * a_given == 1 (aggregate first only) skips the aggregation: A is an input
 * holding P_i [H_in ; H_bd], e.g. a layer-1 aggregate kept across iterations
 * (the input features are constant); H_in / H_bd are then not read.
 * With PGCN_MXFP4, A is required, A_bf16 ignored, H_out, W and the workspace
 * are 16-byte aligned, and the sent rows are copied after the product.
 */
typedef struct {
  int32_t f_in, f_out;         /* 1 .. PGCN_MAX_WIDTH                            */
  int32_t gemm_dtype;          /* pgcn_dtype                                    */
  int32_t relu;                /* 1: H_out = relu(Z); 0: H_out = Z (last layer)  */
  int64_t ld_in;               /* stride of H_in, H_bd, A, A_bf16 (elements)     */
  int64_t ld_out;              /* stride of H_out                                */
  const float *H_in;           /* [n_inner, ld_in]                               */
  const float *H_bd;           /* [n_bd, ld_in] or NULL                          */
  const float *W;              /* [f_in, f_out]                                  */
  float *A;                    /* [n_inner, ld_in] out                           */
  uint16_t *A_bf16;            /* [n_inner, ld_in] out (bf16 bits)               */
  float *H_out;                /* [n_inner, ld_out] out                          */
  void *workspace;
  size_t workspace_bytes;
  int32_t order;               /* pgcn_layer_order (0: aggregate first)           */
  int32_t a_given;             /* 1: A (fp32) already holds P_i [H_in ; H_bd]; only
                                  the update runs (aggregate first; on the bf16
                                  path A is rounded while staged, A_bf16 unused) */
  float *send_out;             /* [n_send, ld_out] or NULL: also writes the rows of
                                  H_out that this partition sends (Algorithm 1's
                                  forward send of the next layer's input), row k =
                                  H_out[send_idx[k]], columns [0, f_out); the kernel
                                  that writes H_out writes them (no second pass over
                                  H_out). 16-byte aligned. */
} pgcn_fwd_args;
int pgcn_layer_fwd(const pgcn_partition *part, const pgcn_fwd_args *args, hipStream_t stream);

/*
 * For callers that cannot allocate device memory (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same
 * layer forward as pgcn_layer_fwd (same kernels, same results bit for bit),
 * with its workspace taken from a fixed array inside this library instead of
 * args->workspace.  Nothing is allocated by the call.
 *
 * args->workspace must be NULL and args->workspace_bytes 0 (else
 * PGCN_EINVAL); every other argument is as for pgcn_layer_fwd, and the
 * caller still owns and passes every input and output.  A layer whose
 * workspace (pgcn_layer_workspace_size's forward share) exceeds
 * PGCN_NOALLOC_SCRATCH_BYTES is rejected with PGCN_EWORKSPACE before any
 * launch.  The array holds PGCN_NOALLOC_SCRATCH_BYTES on every GPU the
 * library runs on, until the process ends; its address on a device is
 * resolved when a partition is set up there.
 *
 * All calls on one GPU share that GPU's array and it keeps the last call's
 * contents (nothing in it needs to start at zero): calls that overlap on one
 * GPU (two streams, two threads, two graphs replayed concurrently) race and
 * must be serialised by the caller.
 */
#define PGCN_NOALLOC_SCRATCH_BYTES (32u << 20)
int pgcn_layer_fwd_noalloc(const pgcn_partition *part, const pgcn_fwd_args *args, hipStream_t stream);

/*
 * One layer backward (Algorithm 1's weight- and feature-gradient lines;
 * Appendix A.1 gradients):
 *     M      = J_out ∘ 1[H_out > 0] if relu else J_out
 *     dW     = A^T M
 *     J_full = P_i^T (M W^T)      rows [0, n_inner) -> J_in,
 *                                 rows [n_inner, n_inner+n_bd) -> J_bd_out
 * J_in and J_bd_out are both NULL for the first layer (no feature gradient).
 * Stale gradients from peers are added afterwards with pgcn_pack_boundary
 * (PGCN_ACCUM_GRAD), as Algorithm 1 does after waiting for them.
 * dW accumulates split-K partials in a fixed order (deterministic).
 * order == PGCN_ORDER_TRANSFORM (the layer's forward used that order):
 *     T      = P_i^T M               [n_inner + n_bd, f_out], in the workspace
 *     dW     = [H_in ; H_bd]^T T
 *     J_full = T W^T                 rows split into J_in / J_bd_out as above
 * H_in / H_bd are the input rows the forward used (stride ld_in; H_bd NULL
 * means zero boundary rows); A and A_bf16 are unused.  bf16 path: H, T and W
 * rounded to bf16 (nearest even) for the products, fp32 accumulation.
 * Aggregate first on the bf16 path, A_bf16 may be NULL when A (fp32) is
 * given: A is then rounded to bf16 while staged (the same values).
 */
typedef struct {
  int32_t f_in, f_out;
  int32_t gemm_dtype;
  int32_t relu;
  int64_t ld_in, ld_out;
  const float *J_out;          /* [n_inner, ld_out]                              */
  const float *H_out;          /* [n_inner, ld_out] mask source (when relu)      */
  const float *A;              /* [n_inner, ld_in] (PGCN_F32)                    */
  const uint16_t *A_bf16;      /* [n_inner, ld_in] (PGCN_BF16)                   */
  const float *W;              /* [f_in, f_out]                                  */
  float *dW;                   /* [f_in, f_out] out                              */
  float *J_in;                 /* [n_inner, ld_in] out or NULL                   */
  float *J_bd_out;             /* [n_bd, ld_in] out or NULL                      */
  void *workspace;
  size_t workspace_bytes;
  int32_t order;               /* pgcn_layer_order (0: aggregate first)           */
  const float *H_in;           /* [n_inner, ld_in] layer input (PGCN_ORDER_TRANSFORM) */
  const float *H_bd;           /* [n_bd, ld_in] or NULL       (PGCN_ORDER_TRANSFORM) */
} pgcn_bwd_args;
int pgcn_layer_bwd(const pgcn_partition *part, const pgcn_bwd_args *args, hipStream_t stream);

/*
 * Moving-average smoothing of stale features or gradients (Section 3.4):
 *     state[r, c] = gamma * state[r, c] + (1 - gamma) * incoming[r, c]
 * for r < rows, c < cols; both matrices share stride ld (ld % 4 == 0).
 */
int pgcn_smooth_ema(float *state, const float *incoming, int64_t rows, int32_t cols, int64_t ld,
                     float gamma, hipStream_t stream);

/*
 * Boundary packing (Algorithm 1's send of H_{S_{i,j}} and the accumulation of
 * received gradients C_j into rows S_{i,j}, ascending j):
 *   PGCN_PACK_FEAT : dst[k, :] = src[send_idx[k], :],   src [n_inner, ld], dst [n_send, ld]
 *   PGCN_ACCUM_GRAD: dst[u, :] += src[k, :] for each k with send_idx[k] == u, in
 *                    ascending k;                      src [n_send, ld], dst [n_inner, ld]
 */
int pgcn_pack_boundary(const pgcn_partition *part, int32_t kind, const float *src, float *dst,
                       int32_t cols, int64_t ld, hipStream_t stream);

/*
 * Smoothing of the received gradients (Section 3.4) fused with their
 * accumulation (Algorithm 1's loop over peers j): for every send row k,
 *     state[k, :] = gamma * state[k, :] + (1 - gamma) * incoming[k, :]
 * and dst[u, :] += state[k, :] for each k with send_idx[k] == u, in ascending
 * k.  The same values as pgcn_smooth_ema(state, incoming, n_send, ...)
 * followed by pgcn_pack_boundary(PGCN_ACCUM_GRAD, state, dst, ...), in one
 * pass.  incoming and state: [n_send, ld]; dst: [n_inner, ld]; ld % 4 == 0,
 * 16-byte aligned; state must not alias incoming or dst.
 */
int pgcn_accum_smoothed(const pgcn_partition *part, const float *incoming, float *state, float gamma, float *dst,
                        int32_t cols, int64_t ld, hipStream_t stream);

/*
 * Loss and its gradient w.r.t. the logits (Algorithm 1's J^(L)):
 *   PGCN_SOFTMAX_CE : loss = scale * sum_r -log softmax(Z_r)[labels[r]]
 *                     J_r  = scale * (softmax(Z_r) - onehot(labels[r]))
 *   PGCN_SIGMOID_BCE: loss = scale * sum_{r,c} BCE(sigmoid(Z_rc), targets_rc)
 *                     J_rc = scale * (sigmoid(Z_rc) - targets_rc)
 * Z and J: [rows, ld]; labels: [rows] int32 in [0, classes); targets: [rows, ld_t].
 * loss_out: one device float, written (not accumulated), reduced in a fixed order.
 */
int pgcn_loss_fwd_bwd(int32_t kind, const float *Z, int64_t rows, int32_t classes, int64_t ld,
                      const int32_t *labels, const float *targets, int64_t ld_t, float scale,
                      float *J, float *loss_out, void *workspace, size_t workspace_bytes,
                      hipStream_t stream);

/* Algorithm 1's update after the AllReduce (a sum): W -= eta * (G + G_peer).
 * G_peer may be NULL (one partition: the AllReduce is the identity). */
int pgcn_sgd_update(float *W, const float *G, const float *G_peer, int64_t count, float eta,
                    hipStream_t stream);

/*
 * Adam update after the AllReduce (the optimiser of the paper's experiments,
 * its setup table; Kingma and Ba, ICLR 2015, Algorithm 1), element-wise for
 * i < count, with g = G + G_peer (G_peer may be NULL):
 *     m = beta1 m + (1 - beta1) g ;  v = beta2 v + (1 - beta2) g^2
 *     W -= lr * (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps)
 * t >= 1 is the step count; m and v (caller-owned, zero before the first
 * step) are updated in place.  The coefficients (beta, 1 - beta, the bias
 * corrections) are computed on the host in double precision and rounded
 * once to fp32; the element-wise update runs in fp32.
 */
int pgcn_adam_update(float *W, const float *G, const float *G_peer, float *m, float *v, int64_t count, double lr,
                     double beta1, double beta2, double eps, int32_t t, hipStream_t stream);

/*
 * Dropout of a layer input, applied after the boundary receive with one mask
 * for the forward and the backward (the paper's implementation notes; rates
 * in its setup table).  For r < rows, c < cols, with global row R = row0 + r
 * (the partition's local numbering: inner rows, then boundary rows at
 * row0 = n_inner) and element index q = R * cols + c:
 *     u = word (q mod 4) of Philox4x32-10(counter = (lo32(q / 4), hi32(q / 4),
 *         layer, iteration), key = (seed, part))
 *     out[r, c] = u < floor(p * 2^32) ? 0 : in[r, c] * (1 / (1 - p))
 * Philox4x32-10 is the counter-based generator of Salmon, Moraes, Dror and
 * Shaw (SC 2011).  The same call on a gradient (same arguments) applies the
 * forward's mask in the backward.  in and out share stride ld (ld % 4 == 0,
 * 16-byte aligned) and may alias.  out_bf16 (optional, stride ld_bf16,
 * ld_bf16 % 8 == 0) receives out rounded to bf16 (nearest even).  0 <= p < 1.
 */
int pgcn_dropout(float *out, const float *in, int64_t rows, int32_t cols, int64_t ld, int64_t row0, double p,
                 uint32_t seed, uint32_t part, uint32_t layer, uint32_t iteration, uint16_t *out_bf16,
                 int64_t ld_bf16, hipStream_t stream);

/*
 * GraphSAGE layer forward (Section 2: the update function takes
 * CONCAT(z_v, h_v); the model of the paper's experiments), on a partition
 * built with PGCN_SETUP_NO_SELF_LOOP:
 *     z = P_i [X_in ; X_bd]          (mean over N(v); stale boundary rows)
 *     Z = [z, X_in] W ;  H_out = relu(Z) if relu else Z
 * X_in / X_bd are the layer input after dropout (pgcn_dropout); X_bd NULL
 * means all-zero boundary rows.  W is [2 f_in, f_out]: rows [0, f_in) act
 * on z, rows [f_in, 2 f_in) on X_in.  The product is evaluated as z W_top
 * followed by an accumulation of X_in W_bot (two passes over H_out).
 * PGCN_F32: z -> A (required).  PGCN_BF16: z rounded once to bf16 -> A_bf16,
 * and X_in_bf16 (the bf16 copy of X_in, e.g. from pgcn_dropout) is the
 * self operand; W is rounded to bf16; fp32 accumulation.
 * Workspace: pgcn_workspace_size(part, f_in, f_out, gemm_dtype).
 * order == PGCN_ORDER_TRANSFORM evaluates z W_top as P_i (X W_top):
 *     Y = [X_in ; X_bd] W_top        (n_inner + n_bd rows, in the workspace)
 *     H_out = act(P_i Y + X_in W_bot)
 * (bf16 path: X and W rounded to bf16 for the products); A and A_bf16 are
 * unused.  Workspace: pgcn_layer_workspace_size with that order.
 */
typedef struct {
  int32_t f_in, f_out;
  int32_t gemm_dtype;
  int32_t relu;
  int64_t ld_in, ld_out;       /* strides of X_in, X_bd, A, A_bf16, X_in_bf16 / of H_out */
  const float *X_in;           /* [n_inner, ld_in]                               */
  const uint16_t *X_in_bf16;   /* [n_inner, ld_in] (PGCN_BF16)                   */
  const float *X_bd;           /* [n_bd, ld_in] or NULL                          */
  const float *W;              /* [2 f_in, f_out]                                */
  float *A;                    /* [n_inner, ld_in] out: z (PGCN_F32)             */
  uint16_t *A_bf16;            /* [n_inner, ld_in] out: z in bf16 (PGCN_BF16)    */
  float *H_out;                /* [n_inner, ld_out] out                          */
  void *workspace;
  size_t workspace_bytes;
  int32_t order;               /* pgcn_layer_order (0: aggregate first)           */
  float *send_out;             /* [n_send, ld_out] or NULL: the sent rows of H_out,
                                  as in pgcn_fwd_args                            */
} pgcn_sage_fwd_args;
int pgcn_sage_layer_fwd(const pgcn_partition *part, const pgcn_sage_fwd_args *args, hipStream_t stream);

/*
 * GraphSAGE layer backward (gradients of the forward above):
 *     M        = J_out ∘ 1[H_out > 0] if relu else J_out
 *     dW       = [z, X_in]^T M          (rows [0, f_in): z^T M; rows [f_in, 2 f_in): X_in^T M)
 *     [dz, ds] = M W^T
 *     J_full   = P_i^T dz, plus ds on the inner rows:
 *                rows [0, n_inner) -> J_in, rows [n_inner, n_inner + n_bd) -> J_bd_out
 * J_full is the gradient of the dropped input; apply the dropout mask to it
 * with pgcn_dropout (same arguments as in the forward) before it is sent or
 * accumulated.  J_in and J_bd_out are both NULL for the first layer.
 * order == PGCN_ORDER_TRANSFORM (the forward used that order):
 *     T = P_i^T M                    [n_inner + n_bd, f_out], in the workspace
 *     dW rows [0, f_in) = [X_in ; X_bd]^T T,  rows [f_in, 2 f_in) = X_in^T M
 *     J_full = T W_top^T, plus M W_bot^T on the inner rows
 * X_bd is the (dropped) boundary input the forward used (NULL: zero rows); A
 * and A_bf16 are unused.  bf16 path: X, T, M and W rounded to bf16 for the
 * products.
 */
typedef struct {
  int32_t f_in, f_out;
  int32_t gemm_dtype;
  int32_t relu;
  int64_t ld_in, ld_out;
  const float *J_out;          /* [n_inner, ld_out]                              */
  const float *H_out;          /* [n_inner, ld_out] mask source (when relu)      */
  const float *A;              /* [n_inner, ld_in] z (PGCN_F32)                  */
  const uint16_t *A_bf16;      /* [n_inner, ld_in] z (PGCN_BF16)                 */
  const float *X_in;           /* [n_inner, ld_in] (PGCN_F32)                    */
  const uint16_t *X_in_bf16;   /* [n_inner, ld_in] (PGCN_BF16)                   */
  const float *W;              /* [2 f_in, f_out]                                */
  float *dW;                   /* [2 f_in, f_out] out                            */
  float *J_in;                 /* [n_inner, ld_in] out or NULL                   */
  float *J_bd_out;             /* [n_bd, ld_in] out or NULL                      */
  void *workspace;
  size_t workspace_bytes;
  int32_t order;               /* pgcn_layer_order (0: aggregate first)           */
  const float *X_bd;           /* [n_bd, ld_in] or NULL        (PGCN_ORDER_TRANSFORM) */
} pgcn_sage_bwd_args;
int pgcn_sage_layer_bwd(const pgcn_partition *part, const pgcn_sage_bwd_args *args, hipStream_t stream);

/* Activation applied after a group norm: u, max(u, 0), u / (1 + e^-u), u (1 + erf(u / sqrt 2)) / 2. */
enum pgcn_act { PGCN_ACT_NONE = 0, PGCN_ACT_RELU = 1, PGCN_ACT_SILU = 2, PGCN_ACT_GELU = 3 };

/*
 * The operators below (top logits, distillation loss, group norm) take matrices in
 * `dtype`: PGCN_F32 (fp32, ld % 4 == 0) or PGCN_BF16 (bf16 bits, ld % 8 == 0), 16-byte
 * aligned.  They compute in fp32 (loss sums in fp64) and round a bf16 result once, to
 * nearest even.  Columns past the matrix's width are neither used nor written, whatever
 * they hold.  Outputs overlap no other buffer of the call (else PGCN_EINVAL).  A
 * workspace is 16-byte aligned, of the size that the call's _workspace_size function
 * gives (0 bytes: it may be NULL), may hold anything before the call and is the call's
 * own until its work has ended.  A stream of another device than the current one is
 * refused with PGCN_EINVAL, and so are more than 2^31 - 1 rows.  The _workspace_size
 * functions return 0 for sizes that the call rejects.
 */

/* Largest number of listed classes, of classes, and of channels that they take. */
#define PGCN_MAX_TOP 256
#define PGCN_MAX_CLASSES 262144
#define PGCN_MAX_CHANNELS 8192

/*
 * The `top` largest logits of every row: what a trained partition model keeps of its
 * answers to teach another one (pgcn_distill_loss_fwd_bwd).
 *     top_values[r, k], top_ids[r, k]: the k-th largest logit of row r and its class; of
 *         equal logits (-0 equals +0) the lower class comes first;
 *     tail_lse[r] = log sum of e^{Z[r, c] / temperature} over the classes not listed
 * A logit of -inf marks a class that is no answer: it is never listed and adds nothing to
 * the tail.  Where a row has fewer than `top` others, the slots left hold -inf and -1; a
 * tail of nothing is -inf.  A NaN is never listed either and makes the row's tail NaN; an unlisted
 * +inf makes it +inf or NaN.
 */
typedef struct {
  int32_t dtype;               /* pgcn_dtype of Z                                */
  int32_t classes;             /* 1 .. PGCN_MAX_CLASSES                          */
  int32_t top;                 /* 1 .. min(classes, PGCN_MAX_TOP)                */
  float temperature;           /* 1e-4 .. 1e4                                    */
  int64_t rows;
  int64_t ld;                  /* stride of Z (elements)                         */
  int64_t ld_top;              /* stride of top_values and top_ids, >= top       */
  const void *Z;               /* [rows, ld]                                     */
  float *top_values;           /* [rows, ld_top] out                             */
  int32_t *top_ids;            /* [rows, ld_top] out                             */
  float *tail_lse;             /* [rows] out or NULL                             */
  void *workspace;
  size_t workspace_bytes;
} pgcn_top_logits_args;
size_t pgcn_top_logits_workspace_size(int32_t dtype, int64_t rows, int32_t classes, int32_t top);
int pgcn_top_logits(const pgcn_top_logits_args *args, hipStream_t stream);

/*
 * Loss of a student's logits Z against a teacher's top logits, with its gradient.  With
 * T = temperature, row by row:
 *     p_k  = e^{top_values[k] / T - L},  rho = e^{tail_lse - L},  L so that sum_k p_k + rho = 1
 *     q    = softmax(Z / T),  s = sum of q over the classes not listed
 *     loss = soft_scale * (sum_k p_k log(p_k / q_{top_ids[k]}) + rho log(rho / s))
 *          + hard_scale * -log softmax(Z)[label]                  (summed over the rows)
 *     J    = d loss / d Z
 * tail_lse NULL: rho = 0, the listed classes share the whole of p.  A T^2 that keeps the
 * gradient's size over temperatures belongs into soft_scale.
 *   - A slot with id -1 (any negative one) or value -inf lists no probability; the latter's
 *     class still counts as listed.  A class listed twice counts with its lowest slot.  A
 *     row that lists none adds no soft term.
 *   - labels NULL, or a label -1: no hard term (a node without a label).
 *   - p log(p / q) is 0 where p is 0, also where q is 0 (a logit of -inf masks its class);
 *     it is +inf where p > 0 and q = 0.
 *   - A scale of 0 takes its term out, whatever it would have been.
 *   - An id or label >= classes (a label < -1 too) makes the loss NaN; the id is otherwise
 *     ignored.  A row without any finite logit that has a soft or hard term makes it NaN.
 *   - A NaN among the logits of a row that has a term makes the loss NaN, and J at each of the
 *     row's classes whose logit is not -inf; in a row without a term J may be NaN at the NaN
 *     itself, and is 0 elsewhere.  A NaN among a row's listed values makes its J NaN (a masked
 *     class's may be 0), and the loss.
 * J: [rows, ld], the dtype and stride of Z.  loss_out: one device float, written (not
 * accumulated), reduced in a fixed order.
 */
typedef struct {
  int32_t dtype;               /* pgcn_dtype of Z and J                          */
  int32_t classes;             /* 1 .. PGCN_MAX_CLASSES                          */
  int32_t top;                 /* 1 .. min(classes, PGCN_MAX_TOP)                */
  float temperature;           /* 1e-4 .. 1e4                                    */
  int64_t rows;
  int64_t ld;                  /* stride of Z and J (elements)                   */
  int64_t ld_top;              /* stride of top_values and top_ids, >= top       */
  float soft_scale, hard_scale;
  const void *Z;               /* [rows, ld]                                     */
  const float *top_values;     /* [rows, ld_top]                                 */
  const int32_t *top_ids;      /* [rows, ld_top]                                 */
  const float *tail_lse;       /* [rows] at the same temperature, or NULL        */
  const int32_t *labels;       /* [rows] or NULL                                 */
  void *J;                     /* [rows, ld] out                                 */
  float *loss_out;             /* [1] out                                        */
  void *workspace;
  size_t workspace_bytes;
} pgcn_distill_args;
size_t pgcn_distill_workspace_size(int32_t dtype, int64_t rows, int32_t classes, int32_t top);
int pgcn_distill_loss_fwd_bwd(const pgcn_distill_args *args, hipStream_t stream);

/*
 * Group normalisation of features-last rows with an activation, for use between a layer's
 * product (relu = 0) and the next layer.  The rows [i sample_rows, (i + 1) sample_rows) are
 * sample i: 1 row normalises every node by itself (groups = 1: layer norm), the
 * partition's n_inner rows all its nodes together.  Per sample and group of channels /
 * groups neighbouring channels:
 *     mean, rstd = 1 / sqrt(variance + eps)    over the sample's rows and the group's channels
 *     u = (X - mean) rstd gamma + beta ;  Y = act(u)
 * gamma or beta NULL: 1 and 0.  mean and rstd ([samples, groups]) are kept for the backward;
 * either may be NULL where none follows.
 */
typedef struct {
  int32_t dtype;               /* pgcn_dtype of X and Y                          */
  int32_t act;                 /* pgcn_act                                       */
  int32_t channels;            /* 1 .. PGCN_MAX_CHANNELS                         */
  int32_t groups;              /* divides channels                               */
  int64_t samples, sample_rows;
  int64_t ld_x, ld_y;
  float eps;                   /* > 0                                            */
  const void *X;               /* [samples * sample_rows, ld_x]                  */
  const float *gamma, *beta;   /* [channels] or NULL                             */
  void *Y;                     /* [samples * sample_rows, ld_y] out              */
  float *mean, *rstd;          /* [samples, groups] out or NULL                  */
  void *workspace;
  size_t workspace_bytes;
} pgcn_group_norm_fwd_args;
int pgcn_group_norm_fwd(const pgcn_group_norm_fwd_args *args, hipStream_t stream);

/*
 * Its gradients, from the forward's input, mean and rstd, and the gradient J_out of Y:
 *     du = J_out act'(u) ;  dbeta = sum du ;  dgamma = sum du xhat       over all rows
 *     J_in = rstd (gamma du - mean(gamma du) - xhat mean(gamma du xhat))
 * with xhat = (X - mean) rstd and the means over the sample's group.  ReLU's slope is
 * 1[u > 0], with u formed as in the forward.  J_in, dgamma and dbeta may each be NULL.
 * The sums over rows are reduced in a fixed order.
 */
typedef struct {
  int32_t dtype;               /* pgcn_dtype of X, J_out and J_in                */
  int32_t act;
  int32_t channels;
  int32_t groups;
  int64_t samples, sample_rows;
  int64_t ld_x, ld_j_out, ld_j_in;
  const void *X;               /* [samples * sample_rows, ld_x]                  */
  const void *J_out;           /* [samples * sample_rows, ld_j_out]              */
  const float *gamma, *beta;   /* as in the forward                              */
  const float *mean, *rstd;    /* [samples, groups]                              */
  void *J_in;                  /* [samples * sample_rows, ld_j_in] out or NULL   */
  float *dgamma, *dbeta;       /* [channels] out or NULL                         */
  void *workspace;
  size_t workspace_bytes;
} pgcn_group_norm_bwd_args;
int pgcn_group_norm_bwd(const pgcn_group_norm_bwd_args *args, hipStream_t stream);
/* Bytes that pgcn_group_norm_fwd and pgcn_group_norm_bwd need (the larger of both). */
size_t pgcn_group_norm_workspace_size(int32_t dtype, int32_t channels, int32_t groups, int64_t samples,
                                      int64_t sample_rows);

/*
 * Rows in 8 and 4 bits.  A row is held in blocks of PGCN_MX_BLOCK neighbouring elements (the last one
 * filled up with zeros), each with a power of two as scale:
 *     Q  [rows, ld_q] bytes: PGCN_MX_INT8 a signed byte q for q / 64 (32 bytes a block); PGCN_MX_FP4 a sign
 *        (bit 3) and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0 .. 2), the even element of a pair in the low
 *        half of its byte (16 bytes a block)
 *     S  [rows, ld_s] bytes: s for the scale 2^(s - 127); 255 makes the block's elements NaN
 * which are the element and scale types of the OCP microscaling formats MXINT8 and MXFP4.  Q is 16-byte
 * aligned with ld_q a multiple of 16, S 4-byte aligned with ld_s a multiple of 4; bytes past a row's
 * blocks are neither used nor written.  Every finite value is exact in bf16.
 *
 * The calls below take up to PGCN_MAX_MX_COLS elements a row.  Their other matrices, outputs, workspaces and
 * streams are as for the operators above (top logits, distillation loss, group norm).
 */
enum pgcn_mx_format { PGCN_MX_INT8 = 0, PGCN_MX_FP4 = 1 };
#define PGCN_MX_BLOCK 32
#define PGCN_MAX_MX_COLS 16777216

/*
 * Rows quantised as they are written.  Per block, s is the smallest for which the block's largest
 * magnitude rounds to at most 127 / 64 (INT8) or 6 (FP4), at most 254 and 252 (what is larger then
 * takes the format's largest value); every element is rounded once, to nearest, ties to even: it is off
 * by at most half a step.  A NaN or an infinity makes its block NaN (s = 255, elements 0).  An FP4
 * element that rounds to 0 keeps its sign.
 *   transpose 0: row k of Q is row index[k] of X, or row k where index is NULL (rows <= src_rows).  A
 *       negative index gives a row of zeros, one >= src_rows a row of NaN.  With a partition's send list
 *       as index this packs the rows that it sends.
 *   transpose 1: Q holds the transpose of X, [cols rows of `rows` elements each] (rows == src_rows, index
 *       NULL): weights [f_in, f_out] laid out for a product over f_in.
 */
typedef struct {
  int32_t format;              /* pgcn_mx_format                                 */
  int32_t dtype;               /* pgcn_dtype of X                                */
  int32_t transpose;           /* 0 or 1                                         */
  int32_t cols;                /* of X: 1 .. PGCN_MAX_MX_COLS                    */
  int64_t rows;                /* transpose: up to PGCN_MAX_MX_COLS              */
  int64_t src_rows;            /* rows of X                                      */
  int64_t ld_x, ld_q, ld_s;
  const void *X;               /* [src_rows, ld_x]                               */
  const int32_t *index;        /* [rows] or NULL                                 */
  uint8_t *Q;                  /* [rows, ld_q] out; transpose: [cols, ld_q]      */
  uint8_t *S;                  /* [rows, ld_s] out; transpose: [cols, ld_s]      */
} pgcn_mx_quantize_args;
int pgcn_mx_quantize(const pgcn_mx_quantize_args *args, hipStream_t stream);

/*
 * Rows read back: out = v, the values that Q and S stand for, or with 0 < gamma <= 1 the moving average of
 * Section 3.4 over them, out = gamma out + (1 - gamma) v (fp32 only; a NaN in out stays one).
 */
typedef struct {
  int32_t format;              /* pgcn_mx_format                                 */
  int32_t dtype;               /* pgcn_dtype of out                              */
  int32_t cols;                /* 1 .. PGCN_MAX_MX_COLS                          */
  float gamma;                 /* 0 .. 1; 0: out is not read                     */
  int64_t rows;
  int64_t ld_q, ld_s, ld_out;
  const uint8_t *Q;            /* [rows, ld_q]                                   */
  const uint8_t *S;            /* [rows, ld_s]                                   */
  void *out;                   /* [rows, ld_out] out (in and out where gamma > 0) */
} pgcn_mx_dequantize_args;
int pgcn_mx_dequantize(const pgcn_mx_dequantize_args *args, hipStream_t stream);

/*
 * Weight gradient of a layer from its input or aggregate held in 8 bits (PGCN_MX_INT8, values v):
 *     dW = v^T (J o 1[H > 0])             [f_in, f_out], a sum over the rows in a fixed order
 * H NULL: no mask.  PGCN_F32: J in three bf16 parts that add up to it (v is exact in one), three exact
 * products each, fp32 sums: fp32 accuracy.  PGCN_BF16: J o mask rounded once to bf16, fp32 sums.  No rows: dW = 0.
 * A masked place of J adds nothing, whatever it holds.  A non-finite value among the others gives non-finite
 * or NaN results.  Values and parts below 2^-126 may be taken for 0.
 */
typedef struct {
  int32_t dtype;               /* pgcn_dtype: the arithmetic, as for the update GEMMs */
  int32_t f_in, f_out;         /* 1 .. PGCN_MAX_WIDTH                            */
  int64_t rows;
  int64_t ld_q, ld_s, ld_j, ld_h;
  const uint8_t *Q;            /* [rows, ld_q] PGCN_MX_INT8                      */
  const uint8_t *S;            /* [rows, ld_s]                                   */
  const float *J;              /* [rows, ld_j], ld_j % 4 == 0                    */
  const float *H;              /* [rows, ld_h], ld_h % 4 == 0, or NULL           */
  float *dW;                   /* [f_in, f_out] out, compact                     */
  void *workspace;
  size_t workspace_bytes;
} pgcn_mx_wgrad_args;
size_t pgcn_mx_wgrad_workspace_size(int32_t dtype, int64_t rows, int32_t f_in, int32_t f_out);
int pgcn_mx_wgrad(const pgcn_mx_wgrad_args *args, hipStream_t stream);

/*
 * A layer's backward whose kept operands are held in 8 bits: pgcn_layer_bwd and pgcn_sage_layer_bwd, aggregate
 * first, with dW from pgcn_mx_wgrad's product over A (for GraphSAGE: z, and X_in where it is given too).  The args'
 * A, A_bf16 (and X_in, X_in_bf16) are then not read; everything else, the workspace among it, is as there.
 */
typedef struct {
  const uint8_t *Q, *S;        /* [n_inner, ld_q], [n_inner, ld_s] PGCN_MX_INT8 of f_in elements */
  int64_t ld_q, ld_s;
} pgcn_mx_rows;
int pgcn_layer_bwd_mx(const pgcn_partition *part, const pgcn_bwd_args *args, const pgcn_mx_rows *A, hipStream_t stream);
int pgcn_sage_layer_bwd_mx(const pgcn_partition *part, const pgcn_sage_bwd_args *args, const pgcn_mx_rows *A,
                           const pgcn_mx_rows *X_in, hipStream_t stream);

/*
 * Product of two matrices of FP4 rows (PGCN_MX_FP4, values a and b) on the scaled matrix instructions:
 *     C[i, j] = sum over t of a[i, t] b[j, t],  relu: where negative 0           [m, n]
 * in fp32, sums in a fixed order: PGCN_MXFP4's product.  The elements that fill up a row's last block count: zeros, as
 * pgcn_mx_quantize writes them.  Terms or sums below 2^-126 may be taken for 0.  No rows of A: nothing to do.
 */
typedef struct {
  int32_t dtype;               /* pgcn_dtype of C                                */
  int32_t relu;                /* 0 or 1                                         */
  int64_t m;                   /* rows of A and C                                */
  int32_t n, k;                /* rows of B; elements a row: 1 .. PGCN_MAX_MX_COLS */
  int64_t ld_a, ld_a_scales, ld_b, ld_b_scales, ld_c;
  const uint8_t *A, *A_scales; /* [m, ld_a], [m, ld_a_scales] PGCN_MX_FP4        */
  const uint8_t *B, *B_scales; /* [n, ld_b], [n, ld_b_scales] PGCN_MX_FP4        */
  void *C;                     /* [m, ld_c] out                                  */
  void *workspace;
  size_t workspace_bytes;
} pgcn_mx_matmul_args;
size_t pgcn_mx_matmul_workspace_size(int32_t dtype, int64_t m, int32_t n, int32_t k);
int pgcn_mx_matmul(const pgcn_mx_matmul_args *args, hipStream_t stream);

/* Refill of a stale buffer (Algorithm 1's send/receive threads; the paper runs
 * them on a second stream): an asynchronous copy of `bytes` bytes into device
 * memory `dst`, enqueued on `stream`.  flags = 0: device-to-device on the
 * compute units; copies of at least 4 MiB between 16-byte-aligned device
 * buffers by the library's copy kernel with
 * non-temporal loads and stores (the copied rows are read in the next
 * iteration, so they bypass the caches the current one uses), others by
 * the runtime's copy; PGCN_REFILL_DMA:
 * device-to-device by the DMA engines, using no compute units (as a transfer
 * arriving from a peer GPU would); PGCN_REFILL_FROM_HOST: `src` is pinned
 * (page-locked) host memory, copied by DMA over the host link (the paper's
 * CPU-staged exchange); other host memory is rejected with PGCN_EINVAL. */
enum pgcn_refill_flags { PGCN_REFILL_DMA = 1, PGCN_REFILL_FROM_HOST = 2 };
int pgcn_refill_async(void *dst, const void *src, size_t bytes, uint32_t flags, hipStream_t stream);

/*
 * Kernel tracing (measurement support).  While enabled, every kernel launch
 * (and every refill copy) of the library is bracketed by a HIP event pair
 * recorded on the launch stream, except that the chunk launches of one
 * aggregation column range (PGCN_TK_AGG_FWD / _BWD), which run back to back,
 * share one pair: each event record costs the stream several microseconds.
 * pgcn_trace_collect waits for the recorded pairs and returns each record's
 * kind (pgcn_trace_kind), duration in ms and the number of launches it spans
 * (`launches`, may be NULL; 1 except for the shared aggregation records,
 * which may span 0 launches when every chunk is empty), then clears the
 * record.  pgcn_trace_enable creates `capacity` event pairs
 * up front (timing-only events without the system-scope cache flush a
 * default event record performs, so tracing does not disturb the caches of
 * the kernels it brackets) and resets the kind filter to "all kinds";
 * launches beyond the capacity are not recorded.  pgcn_trace_filter limits
 * recording to the kinds whose bit (1u << kind) is set in `kind_mask`.  Not
 * for use under graph capture.
 */
enum pgcn_trace_kind {
  PGCN_TK_AGG_FWD = 0, PGCN_TK_AGG_BWD = 1, PGCN_TK_AGG_FIXUP = 2, PGCN_TK_GEMM_FWD = 3,
  PGCN_TK_GEMM_DGRAD = 4, PGCN_TK_GEMM_WGRAD = 5, PGCN_TK_WGRAD_REDUCE = 6, PGCN_TK_EMA = 7,
  PGCN_TK_PACK = 8, PGCN_TK_ACCUM = 9, PGCN_TK_LOSS = 10, PGCN_TK_SGD = 11, PGCN_TK_REFILL = 12,
  PGCN_TK_GEMM_PACK = 13, PGCN_TK_DROPOUT = 14, PGCN_TK_ADAM = 15, PGCN_TK_MASK_SCALE = 16,
  PGCN_TK_ACCUM_EMA = 17, PGCN_TK_TOP_LOGITS = 18, PGCN_TK_DISTILL = 19, PGCN_TK_GROUP_NORM = 20,
  PGCN_TK_GROUP_NORM_BWD = 21, PGCN_TK_MX_QUANTIZE = 22, PGCN_TK_MX_DEQUANTIZE = 23,
  PGCN_TK_MX_WGRAD = 24, PGCN_TK_MX_MATMUL = 25
};
int pgcn_trace_enable(int32_t capacity);
int pgcn_trace_filter(uint32_t kind_mask);
int pgcn_trace_collect(int32_t *kinds, float *ms, int32_t *launches, int32_t max_records, int32_t *count);
int pgcn_trace_disable(void);

const char *pgcn_last_error(void);
int pgcn_version(void);

#ifdef __cplusplus
}
#endif
#endif /* PGCN_H */
