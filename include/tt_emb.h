/*
 * tt_emb.h -- C ABI of the Tensor-Train (TT) embedding-bag hot path for MI355X (gfx950).
 *
 * The operator is an nn.EmbeddingBag-style lookup (flat index list + CSR bag
 * offsets, sum pooling) whose trainable parameters are three TT cores (paper,
 * Section II-B; Section III-A..F for the optimised lookup / backward).
 *
 * Conventions shared by every call
 * --------------------------------
 * - "DEVICE" pointers are HIP device memory of the current device; "HOST"
 *   pointers are ordinary host memory.  The library allocates no device memory:
 *   every buffer, including the workspace a plan lives in, is owned by the caller
 *   and merely borrowed until the work enqueued by the call has finished on
 *   `stream`.  The only process-wide state is a once-per-process set-up of kernel
 *   launch attributes (thread-safe); calls may be issued from several host threads.
 * - All work is enqueued on `stream` (a hipStream_t passed as void*, NULL = the
 *   default stream).  No call synchronises or copies device->host, except
 *   tt_plan_status.
 * - Core k (k = 0,1,2) is a flat fp32 array indexed G_k[r[k]][n[k]][d[k]][r[k+1]],
 *   row-major, with r[0] = r[3] = 1 (Section II-B: boundary ranks are 1).
 *   A table has num_rows <= n[0]*n[1]*n[2] rows; rows >= num_rows are padding
 *   and are never valid.  Row i uses slices (i1,i2,i3) with
 *   i3 = i mod n[2], i2 = (i div n[2]) mod n[1], i1 = i div (n[1]*n[2])
 *   (Section III-B, TT-index equation; i1 is the most significant digit), and
 *   its D = d[0]*d[1]*d[2] columns are ordered j = (j1*d[1] + j2)*d[2] + j3.
 * - Bags are CSR: offsets has num_bags+1 entries, offsets[0] = 0,
 *   offsets[num_bags] = nnz, non-decreasing.  An empty bag gives a zero row.
 *   Indices and offsets are int64 (the PyTorch default); everything else fp32.
 * - Every call returns a tt_status and never throws.  Host-visible arguments
 *   (NULL pointers, shapes, sizes) are validated synchronously.  Errors only
 *   the device can see (an index < 0 or >= num_rows, offsets that are not
 *   monotone) set a status word inside the plan; the offending lookup then
 *   contributes nothing, and tt_plan_status reports it.  Without a plan
 *   (naive arms) an out-of-range lookup is skipped silently.
 * - With a plan every result is bitwise reproducible from run to run (sorted
 *   segmented reductions, no floating-point atomics).  The plan == NULL
 *   backward accumulates with floating-point atomics and is not.
 * - Limits (TT_ERR_SHAPE otherwise): n[0]*n[1]*n[2] < 2^31 - 1, nnz < 2^31 - 1,
 *   r[1], r[2] <= 128, d[0]*d[1]*r[2] <= 4096, d[1]*r[2] <= 4096, D <= 1024.
 */
#ifndef TT_EMB_H_
#define TT_EMB_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  TT_OK = 0,
  TT_ERR_INVALID_ARG = -1, /* NULL pointer, negative size                                */
  TT_ERR_SHAPE = -2,       /* table shape violates the conventions or limits above       */
  TT_ERR_WORKSPACE = -3,   /* workspace too small or misaligned (needs 256-byte align)   */
  TT_ERR_INDEX_RANGE = -4, /* reported by tt_plan_status: bad index or bad offsets seen  */
  TT_ERR_HIP = -5,         /* a HIP runtime call or kernel launch failed                 */
  TT_ERR_UNAVAILABLE = -6  /* the entry point is switched off in this build              */
} tt_status;

/* One TT table.  HOST struct, caller-owned, read during the call only. */
typedef struct {
  int64_t num_rows; /* N, number of valid rows                                         */
  int32_t n[3];     /* row factors, n[0]*n[1]*n[2] >= N                                */
  int32_t d[3];     /* column factors, D = d[0]*d[1]*d[2]                              */
  int32_t r[4];     /* TT ranks, r[0] = r[3] = 1                                       */
  float *core[3];   /* DEVICE, core k is [r[k]][n[k]][d[k]][r[k+1]] row-major          */
} tt_table;

/*
 * The reorder plan: a HOST struct of DEVICE pointers into the caller's
 * workspace, filled by tt_index_reorder.  It is the deterministic counterpart
 * of the paper's reuse-buffer bookkeeping (Section III-C, pointer-preparation
 * algorithm) and of the "distinct embeddings" bookkeeping of the gradient
 * aggregation (Section III-E): lookups stably sorted by row, the distinct rows,
 * and the distinct (i1,i2) prefixes (prefix = row div n[2], the reuse-buffer
 * key), each in increasing order.  U_r = number of distinct valid rows, U_p =
 * number of distinct prefixes; both live on the device (counts[0], counts[1]).
 * All index arrays are int32.  Entries beyond the stated valid length are
 * unspecified.  The same plan serves forward, backward and update of the batch
 * it was built from, for this table shape only.
 */
typedef struct {
  int64_t nnz, num_bags;  /* the batch the plan was built for                            */
  int64_t max_rows;       /* capacity for distinct rows     = min(nnz, num_rows)          */
  int64_t max_prefixes;   /* capacity for distinct prefixes = min(nnz, n[0]*n[1])         */
  int32_t n[3], d[3], r[4];
  /* -- lookup order ------------------------------------------------------------------ */
  int32_t *sorted_row;    /* [nnz] row of the s-th lookup in (row, position) order; the
                             valid lookups come first, invalid ones hold n0*n1*n2         */
  int32_t *perm;          /* [nnz] original position of the s-th sorted lookup            */
  int32_t *bag_of_sorted; /* [nnz] bag that holds the s-th sorted lookup                  */
  int32_t *slot_of_sorted;/* [nnz] distinct-row slot of the s-th sorted lookup, -1 invalid*/
  int32_t *lookup2row;    /* [nnz] distinct-row slot of original position l, -1 invalid   */
  /* -- distinct rows and prefixes ------------------------------------------------------ */
  int32_t *uniq_row;      /* [U_r] distinct rows, strictly increasing                     */
  int32_t *row_seg;       /* [U_r+1] sorted-lookup range of each distinct row             */
  int32_t *row2pref;      /* [U_r] prefix slot of each distinct row                       */
  int32_t *uniq_pref;     /* [U_p] distinct prefixes i1*n[1]+i2, strictly increasing      */
  int32_t *pref_seg;      /* [U_p+1] distinct-row range of each prefix                    */
  /* -- groupings used by the core-gradient reductions ---------------------------------- */
  int32_t *rows_by_i3;    /* [U_r] distinct-row slots stably sorted by i3                 */
  int32_t *i3_of_sorted;  /* [U_r] the i3 key of rows_by_i3[.] (non-decreasing)           */
  int32_t *i3_seg;        /* [n[2]+1] range in rows_by_i3 of each i3                      */
  int32_t *prefs_by_i2;   /* [U_p] prefix slots stably sorted by i2                       */
  int32_t *i2_seg;        /* [n[1]+1] range in prefs_by_i2 of each i2                     */
  int32_t *i1_seg;        /* [n[0]+1] prefix-slot range of each i1                        */
  int32_t *pref_meta;     /* [max_prefixes][4] per prefix in i2 order: i1, first distinct-row
                             slot, distinct rows, prefix slot (one 16-byte load per prefix for
                             the matrix-core kernels)                                        */
  int32_t *counts;        /* [16] counts[0]=U_r, [1]=U_p, [2]=valid lookups, [3]=nnz,
                             [4]=status bits (1: index out of range, 2: bad offsets)      */
  /* -- float scratch used by forward / backward (contents are transient) --------------- */
  float *rowbuf;          /* [max_rows][D] reconstructed distinct rows                    */
  float *gagg;            /* [max_rows][D] output gradients merged per distinct row       */
  float *hbuf;            /* [max_prefixes][d0*d1*r2] per-prefix right partial gradients;
                             NULL when the table is served by the matrix-core kernels, which
                             keep them on chip                                               */
  float *t3buf;           /* [max_rows][r2*d2] per-row contributions to core 2            */
  float *t1buf;           /* [max_prefixes][d0*r1] per-prefix contributions to core 0     */
  float *partial;         /* segmented-reduction partials                                 */
  float *dg2part;         /* [split][core-1 shape] partial core-1 gradients when the backward
                             workgroups of a table with few core-1 slices are split        */
  void *sort_tmp;         /* radix-sort ping-pong buffers, histograms, scan temporaries   */
  void *prof;             /* HOST, optional tt_prof* attached by the caller (NULL after
                             tt_index_reorder): brackets one kernel with HIP events       */
  void *workspace;        /* the caller's workspace this plan points into                 */
  size_t workspace_bytes;
} tt_plan;

/* Bytes of DEVICE workspace tt_index_reorder needs for this table shape and batch size
 * (0 on invalid arguments).  The workspace must be 256-byte aligned.  The size depends on which
 * kernels serve the table (shape, and whether table->core[1] and core[2] are 16-byte aligned): pass
 * the table with the cores it will be used with.  A backward call whose cores are less aligned than
 * those the workspace was sized for returns TT_ERR_WORKSPACE. */
size_t tt_workspace_bytes(const tt_table *table, int64_t nnz, int64_t num_bags);

/*
 * Index reordering (Section III-G: each batch's lookups are put in increasing
 * index order so that equal TT prefixes become adjacent and reusable; Section
 * III-C: detect which prefix products must be computed; Section III-E: find the
 * distinct rows whose gradients are merged).
 *   indices  DEVICE int64[nnz]        row index of each lookup
 *   offsets  DEVICE int64[num_bags+1] CSR bag offsets
 *   remap    DEVICE int64[num_rows] or NULL: the index bijection f_index of
 *            Section III-G applied before the lookup (row = remap[index]);
 *            NULL = identity.  It changes which row is read.
 *   workspace DEVICE, workspace_bytes >= tt_workspace_bytes(...), 256-byte aligned
 *   plan_out HOST, filled on return (its arrays become valid when the enqueued
 *            work has run).
 * Ties between equal rows keep their original order, so the plan is unique.
 */
tt_status tt_index_reorder(const tt_table *table, const int64_t *indices, const int64_t *offsets,
                           int64_t nnz, int64_t num_bags, const int64_t *remap, void *workspace,
                           size_t workspace_bytes, tt_plan *plan_out, void *stream);

/*
 * Forward (Section III-B): out[b][:] = sum over the lookups l of bag b of the
 * reconstructed row W[index[l]][:], where W[i] = G1[i1] x G2[i2] x G3[i3].
 *   plan != NULL: each distinct prefix product G1[i1] x G2[i2] and each distinct
 *                 row is computed once (batch-level reuse, Section III-C), then
 *                 bags are summed; `indices` may be NULL (the plan holds them).
 *   plan == NULL: naive arm, every lookup runs the full chain (no reuse).
 *   out  DEVICE float[num_bags][D], overwritten.
 * The remap given to tt_index_reorder is baked into the plan; the naive arm
 * reads `indices` as they are.
 * Accuracy and bits: sums are fp32 and reproducible, the same batch gives the same bits.  The last
 * bits of a row may differ between batches: for d = (4, 8, 4) and ranks (32, 32) / (64, 64) the planned
 * arm forms prefix products on the fp32 matrix instruction up to 16384 / 8192 lookups in the call, and above
 * on bf16 ones, of operands split into three parts (no less exact, infinities and NaN as in fp32).
 * So one row in two batches on either side of that limit, or in a table alone and in a fused one, agrees
 * to fp32 rounding.  tt_emb_bag_forward_sample follows the same limit.
 */
tt_status tt_emb_bag_forward(const tt_table *table, const tt_plan *plan, const int64_t *indices,
                             const int64_t *offsets, int64_t nnz, int64_t num_bags, float *out,
                             void *stream);

/*
 * Backward (Section III-D backward equation; Section III-E in-advance gradient
 * aggregation): gradients of L w.r.t. the three cores given grad_out[b][:] =
 * dL/d out[b][:].  Gradients of repeated rows add up.
 *   plan != NULL: output gradients are first merged per distinct row, then
 *                 contracted once per distinct row / prefix, and slice gradients
 *                 are combined by sorted segmented reductions.
 *   plan == NULL: naive arm, one contraction per lookup, atomic accumulation.
 *   grad_out DEVICE float[num_bags][D]
 *   dcore    HOST array of 3 DEVICE pointers, core-shaped, fully overwritten
 *            (slices no lookup touches are exactly 0).
 */
tt_status tt_emb_bag_backward(const tt_table *table, const tt_plan *plan, const int64_t *indices,
                              const int64_t *offsets, int64_t nnz, int64_t num_bags,
                              const float *grad_out, float *const dcore[3], void *stream);

/*
 * Gradient-descent update of the cores (training algorithm, update step):
 * G_k <- G_k - lr * dG_k for k = 0,1,2, in place.
 *   plan != NULL: only the slices the batch touched are visited (the others have
 *                 zero gradient, so the result is identical);
 *   plan == NULL: dense sweep over the three cores.
 */
tt_status tt_core_sgd_update(const tt_table *table, const tt_plan *plan,
                             const float *const dcore[3], float lr, void *stream);

/*
 * Backward with the core update fused in (Section III-F, fused TT-core update): the same
 * gradients as tt_emb_bag_backward with a plan, but every gradient slice is applied as
 * G_k <- G_k - lr * dG_k at the point where its reduction completes (the workgroup that holds the
 * finished core-1 strip in registers, the final step of the segmented sums for cores 0 and 2), so
 * no core-shaped gradient is written to or re-read from memory and the separate update launch
 * disappears.  The cores end up bitwise equal to tt_emb_bag_backward followed by
 * tt_core_sgd_update on the same plan; all contractions use the pre-update cores.
 *   plan     required (the naive arm accumulates with atomics and has no completion point);
 *   table->core[k] are updated IN PLACE; no gradient is returned.
 */
tt_status tt_emb_bag_backward_sgd(const tt_table *table, const tt_plan *plan, const int64_t *indices,
                                  const int64_t *offsets, int64_t nnz, int64_t num_bags,
                                  const float *grad_out, float lr, void *stream);

/*
 * Forward by sample-level reuse (Section III-B, reuse equation) on top of the reuse buffer of
 * Section III-C: first the product G1[i1] x G2[i2] of every distinct prefix of the batch is written
 * to `reuse_buffer` (the paper's Reuse Buffer, [prefix slot][(j1,j2)][r2] fp32); then each bag
 * groups its lookups by prefix, sums the core-2 slices G3[:, i3, :] of a group and multiplies the
 * group's buffered product by that sum ONCE -- one second-stage multiplication per (bag, prefix)
 * group instead of one per lookup -- adding the results into the bag's output row.  Same result
 * as tt_emb_bag_forward up to the order of the fp32 additions; bitwise reproducible.
 * It pays when bags are long and their lookups share prefixes; with few lookups per bag the
 * batch-level route of tt_emb_bag_forward (each distinct row once, then a gather) moves less data.
 *   plan          required (built by tt_index_reorder for this batch)
 *   reuse_buffer  DEVICE, 256-byte aligned, at least tt_reuse_buffer_bytes(table, nnz) bytes,
 *                 borrowed until the enqueued work has finished; contents are transient.
 *   out           DEVICE float[num_bags][D], overwritten.
 * tt_reuse_buffer_bytes returns 0 on invalid arguments.
 */
size_t tt_reuse_buffer_bytes(const tt_table *table, int64_t nnz);
tt_status tt_emb_bag_forward_sample(const tt_table *table, const tt_plan *plan, const int64_t *offsets,
                                    int64_t nnz, int64_t num_bags, void *reuse_buffer,
                                    size_t reuse_buffer_bytes, float *out, void *stream);

/*
 * Reduced-precision cores (deployment discussion of the paper: devices with half-precision
 * arithmetic): the three cores are STORED as bf16, all accumulation stays fp32.
 * tt_cores_to_bf16 rounds table->core[0..2] (round to nearest, ties to even) into `bf16_cores`, a
 * DEVICE buffer of tt_bf16_cores_bytes(table) bytes, 256-byte aligned, in a layout private to the
 * library (core 1 is regrouped for the matrix-core kernel).  tt_emb_bag_forward_bf16 is the
 * planned forward of tt_emb_bag_forward reading those copies: the prefix products run on the bf16
 * matrix-core instruction (products of bf16 values are exact in fp32, sums are fp32), the products
 * stay fp32 and the second stage is the fp32 kernel with core-2 values widened exactly.  The result
 * therefore equals the fp32 forward of the ROUNDED cores to fp32 rounding (tolerance 1e-5 as for
 * tt_emb_bag_forward), and differs from the forward of the unrounded cores by at most
 * ((1 + 2^-9)^3 - 1) * sum over the TT paths of |G1 G2 G3|, about 0.6 % of that sum.
 * Only tables the matrix-core kernels serve (d = (4, 8, 4), ranks (32, 32) or (64, 64)):
 * TT_ERR_SHAPE otherwise (0 from the size query).  table->core[] are not read by the forward.
 */
size_t tt_bf16_cores_bytes(const tt_table *table);
tt_status tt_cores_to_bf16(const tt_table *table, void *bf16_cores, size_t bf16_cores_bytes, void *stream);
tt_status tt_emb_bag_forward_bf16(const tt_table *table, const void *bf16_cores, const tt_plan *plan,
                                  const int64_t *offsets, int64_t nnz, int64_t num_bags, float *out,
                                  void *stream);

/*
 * The same bag sums without a plan, in one launch and without scratch: every lookup multiplies its own
 * chain, so repeated rows and prefixes are computed again.  Same shapes, same alignment of bf16_cores and
 * same tolerance as tt_emb_bag_forward_bf16; invalid indices are skipped and malformed offsets clamped, and
 * there is no plan that would report them.  tt_forward_bf16_direct_pays says (1 / 0, from the
 * sizes alone) whether this is the faster way for a batch whose plan serves nothing else; 0 on invalid
 * arguments.  The two ways add in different orders: a program that asks tt_forward_bf16_direct_pays, as
 * the Python module's forward_bf16 does, gets a bag's last bits by the sizes of its batch.
 */
int tt_forward_bf16_direct_pays(const tt_table *table, int64_t nnz, int64_t num_bags);
tt_status tt_emb_bag_forward_bf16_direct(const tt_table *table, const void *bf16_cores, const int64_t *indices,
                                         const int64_t *offsets, int64_t nnz, int64_t num_bags, float *out,
                                         void *stream);

/*
 * Forward for callers that cannot allocate device memory or hand over a workspace: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  One call = index reorder +
 * planned forward (the result is bitwise that of tt_index_reorder followed by tt_emb_bag_forward
 * with the plan; short batches get it without a plan), with the plan's workspace in a static device array of TT_STATIC_SCRATCH_BYTES
 * that the library's code object holds on every GPU it runs on until the process ends.  The call
 * allocates and frees nothing.
 *   indices, offsets, out  DEVICE, as in tt_emb_bag_forward; no remap.
 * Returns TT_ERR_WORKSPACE when the batch needs more than TT_STATIC_SCRATCH_BYTES (at D = 128
 * about 50 000 lookups).  All calls on one GPU share that GPU's array: calls that overlap on one
 * GPU (different streams, or host threads without ordering) race; calls on one stream are safe.
 * Nothing in the array has to be cleared between calls (the reorder initialises what it reads).
 * The first call on a device looks the array's address up (hipGetSymbolAddress); make that call
 * outside a stream capture.  Index errors are skipped silently (there is no plan to query).
 */
#define TT_STATIC_SCRATCH_BYTES ((size_t)32 << 20)
tt_status tt_emb_bag_forward_static(const tt_table *table, const int64_t *indices, const int64_t *offsets,
                                    int64_t nnz, int64_t num_bags, float *out, void *stream);

/*
 * Batched calls: the same four operations for several tables with ONE launch per kernel, so that
 * small tables share the chip with large ones and the host enqueues dozens, not thousands, of
 * launches per step.  All tables of a call must share d[] and r[] (n[] may differ) and must all
 * have a plan or all lack one.  Each item names one table's arguments exactly as in the
 * single-table calls; fields a call does not use are ignored.
 *   items  HOST array of num_tables items (1..256); for reorder, items[t].plan is filled.
 *   desc   DEVICE scratch of at least tt_batch_desc_bytes(num_tables) bytes, 16-byte aligned,
 *          into which the call writes the kernels' per-table descriptors (small launches on
 *          `stream` that carry them as arguments, so the write is ordered like any kernel).  It
 *          is borrowed until the enqueued work has finished: consecutive calls on ONE stream may
 *          share a buffer, calls that may overlap on different streams need different buffers.
 * Results are bitwise identical to the single-table calls.
 * STATUS: switched off.  Every batched call currently returns TT_ERR_UNAVAILABLE without
 * touching the device: the first GPU run of the batched path ended in a memory fault whose cause
 * has not been found yet, so the path stays disabled until it is.  The single-table calls are
 * unaffected (they share the kernels but pass one descriptor by value).
 */
typedef struct {
  const tt_table *table;   /* HOST                                                         */
  tt_plan *plan;           /* HOST; out for reorder, in otherwise (NULL = naive arm)       */
  const int64_t *indices;  /* DEVICE int64[nnz]                                            */
  const int64_t *offsets;  /* DEVICE int64[num_bags+1]                                     */
  int64_t nnz, num_bags;
  const int64_t *remap;    /* DEVICE or NULL (reorder)                                     */
  void *workspace;         /* DEVICE (reorder)                                             */
  size_t workspace_bytes;
  float *out;              /* DEVICE float[num_bags][D] (forward)                          */
  const float *grad_out;   /* DEVICE float[num_bags][D] (backward)                         */
  float *dcore[3];         /* DEVICE core-shaped (backward: written; update: read)         */
} tt_batch_item;

size_t tt_batch_desc_bytes(int num_tables);
tt_status tt_index_reorder_batched(int num_tables, tt_batch_item *items, void *desc,
                                   size_t desc_bytes, void *stream);
tt_status tt_emb_bag_forward_batched(int num_tables, tt_batch_item *items, void *desc,
                                     size_t desc_bytes, void *stream);
tt_status tt_emb_bag_backward_batched(int num_tables, tt_batch_item *items, void *desc,
                                      size_t desc_bytes, void *stream);
tt_status tt_core_sgd_update_batched(int num_tables, tt_batch_item *items, float lr, void *desc,
                                     size_t desc_bytes, void *stream);

/*
 * Fused tables.  TT tables with the same column factors d[] and ranks r[] can be stored as ONE TT
 * table whose core k is the members' cores k laid side by side along the row-factor axis:
 * [r_k][sum over members of n_k][d_k][r_k+1], member t owning the range [o_k(t), o_k(t) + n_k(t)) of
 * that axis (o_k = sum of n_k over the members before t).  Row i = (i1, i2, i3) of member t
 * (index split of Section III-B) is row ((o_1 + i1) * N2 + o_2 + i2) * N3 + o_3 + i3 of the fused
 * table (N_k = sum of n_k): the same three slices, hence the same product (TT-matrix equation,
 * Section II-B), the same bag sums and the same core gradients, found at the members' ranges of the
 * fused cores.  Fused rows that mix slices of different members exist but are never looked up.
 * One reorder, one forward and one backward over the fused table then replace the members' calls:
 * fewer, larger launches (the batched prefix products of Section III-C now batch over tables too).
 *
 * tt_fuse_shape fills fused->num_rows and fused->n[] (d[], r[] and core[] are the caller's):
 * TT_ERR_SHAPE if a row factor sum or the row count does not fit (N1*N2*N3 must stay below 2^31).
 *
 * tt_fuse_lookups maps one batch of every member into the fused table, member after member:
 *   indices, offsets  HOST arrays [num_tables] of DEVICE pointers: member t's int64[nnz[t]] and
 *                     CSR int64[num_bags[t] + 1], as tt_index_reorder takes them
 *   remaps            HOST array of DEVICE pointers or NULL; a non-NULL entry is member t's row
 *                     bijection f_index (int64[num_rows of t]), applied before the split
 *   nnz, num_bags     HOST int64[num_tables]
 *   fused_indices     DEVICE int64[sum nnz]: member t's lookups at [sum of nnz before t, ...);
 *                     an index outside [0, num_rows of t) becomes -1, which tt_index_reorder
 *                     reports and skips like any invalid index
 *   fused_offsets     DEVICE int64[sum num_bags + 1]: member t's bags at [sum of num_bags before
 *                     t, ...), so that rows of `out` / `grad_out` of the fused calls are the
 *                     members' rows, member after member.  An offset outside [0, nnz[t]], a first
 *                     offset other than 0 or a last one other than nnz[t] is written as -1, which
 *                     tt_index_reorder reports as an invalid CSR array.
 * One launch on `stream`; nothing is read on the host.  At most TT_FUSE_MAX_TABLES members.
 *
 * tt_fuse_lookups_starts is the same for members whose offsets hold the bag STARTS only
 * (int64[num_bags[t]], torch.nn.EmbeddingBag's default): member t's last bag ends at nnz[t].
 *
 * tt_fuse_lookups_ranges is one or the other (`starts` != 0: the offsets are starts) and also writes
 * bag_ranges, DEVICE int64[num_tables + 1]: the first row of every member in the fused `out`, and the
 * end -- the `offsets` with which tt_dense gives every member's rows a weight of their own.
 */
#define TT_FUSE_MAX_TABLES 32
typedef struct {
  int32_t num_tables;
  int32_t n[TT_FUSE_MAX_TABLES][3];     /* row factors of member t                             */
  int64_t num_rows[TT_FUSE_MAX_TABLES]; /* rows of member t (<= n[t][0]*n[t][1]*n[t][2])       */
} tt_fuse_members;

tt_status tt_fuse_shape(const tt_fuse_members *members, tt_table *fused);
tt_status tt_fuse_lookups(const tt_fuse_members *members, const int64_t *const *indices,
                          const int64_t *const *offsets, const int64_t *const *remaps,
                          const int64_t *nnz, const int64_t *num_bags, int64_t *fused_indices,
                          int64_t *fused_offsets, void *stream);
tt_status tt_fuse_lookups_starts(const tt_fuse_members *members, const int64_t *const *indices,
                                 const int64_t *const *starts, const int64_t *const *remaps,
                                 const int64_t *nnz, const int64_t *num_bags, int64_t *fused_indices,
                                 int64_t *fused_offsets, void *stream);
tt_status tt_fuse_lookups_ranges(const tt_fuse_members *members, const int64_t *const *indices,
                                 const int64_t *const *offsets, int starts, const int64_t *const *remaps,
                                 const int64_t *nnz, const int64_t *num_bags, int64_t *fused_indices,
                                 int64_t *fused_offsets, int64_t *bag_ranges, void *stream);

/*
 * Index-graph edges of one batch (Section III-G, index-graph generation algorithm): the weighted
 * co-occurrence graph the offline index bijection is built from.  Offline preprocessing, not part
 * of a training step.
 *   node of a lookup = max(rank[index], hot_thresh) - hot_thresh, with rank[] the frequency rank
 *   of every row (0 = most frequent); node 0 (all hot rows) is dropped.  Every bag contributes one
 *   pair (u < v) per two of its distinct nodes; a bag with more than max_group (<= 64) distinct
 *   nodes keeps its max_group smallest ones, and only the first 256 lookups of a bag are looked at.
 *   Equal pairs are merged; weight = number of bags that hold both ends.
 *   indices, offsets  DEVICE, as in tt_index_reorder (invalid indices are skipped)
 *   rank              DEVICE int32[num_rows]
 *   workspace         DEVICE, 256-byte aligned, tt_index_graph_workspace_bytes(num_bags, max_pairs)
 *   edge_u/v/w        DEVICE int32[max_pairs] each: the edges, sorted by (u, v), weights in edge_w
 *   counts            DEVICE int32[4]: [0] pairs before merging, [1] edges, [2] 1 if the batch has
 *                     more than max_pairs pairs (then no edge is produced)
 * The result is unique (integer work, stable sorts).
 */
size_t tt_index_graph_workspace_bytes(int64_t num_bags, int64_t max_pairs);
tt_status tt_index_graph_edges(const int64_t *indices, const int64_t *offsets, int64_t nnz, int64_t num_bags,
                               const int32_t *rank, int64_t num_rows, int64_t hot_thresh, int32_t max_group,
                               void *workspace, size_t workspace_bytes, int64_t max_pairs, int32_t *edge_u,
                               int32_t *edge_v, int32_t *edge_w, int32_t *counts, void *stream);

/*
 * Dense side.  What a model does with pooled rows right behind the bags, and how cores and dense weights
 * are updated by their orthogonalised gradients.  These calls take fp32, bf16 or fp16 data; sums are fp32
 * on the matrix cores and reproducible: the same call gives the same bits (no atomics; the order of a sum
 * follows types, sizes and alignment).  fp32 operands are multiplied as three bf16 parts each, six products of
 * them, no less exact than the fp32 instruction, which takes over where infinities, NaN or numbers or products near the
 * ends of the range would cost precision.  The calls allocate nothing and follow the conventions above.
 */
typedef enum { TT_F32 = 0, TT_BF16 = 1, TT_F16 = 2 } tt_dtype;
typedef enum {
  TT_ACT_NONE = 0,
  TT_ACT_RELU = 1,   /* z <= 0 ? 0 : z, slope 0 at 0; a z of fp32 tensors that rounding could take to
                        the other side of 0 is formed in 64 bits                                */
  TT_ACT_GELU = 2,   /* z Phi(z), with the normal distribution's Phi                            */
  TT_ACT_SILU = 3,   /* z / (1 + exp(-z))                                                       */
  TT_ACT_SIGMOID = 4 /* 1 / (1 + exp(-z))                                                       */
} tt_activation;

/*
 * The product of rows with a weight, its epilogue and its gradients:
 *   z = x W^T + bias,  out = act(z) + residual       x [rows][in_dim], W [out_dim][in_dim]
 *   groups == 0: one W and one bias [out_dim] for all rows.
 *   groups >= 1: W [groups][out_dim][in_dim], bias [groups][out_dim]; group g's are used for the rows
 *     [offsets[g], offsets[g+1]) -- the tables of a fused table (their bags follow each other in `out` of
 *     the bag calls), or the experts of a router.  Groups may be empty.  Offsets are read on the device
 *     only and need no order: each is clamped to [0, rows] and counts at least as much as those
 *     before it.  Rows before offsets[0] and behind offsets[groups] belong to no group: in `out`, `pre` and
 *     `dx` they are left as they were (zero_rest: cleared in `out` and `dx`), and no gradient gets anything from them.
 * HOST struct, read during the call only.
 */
#define TT_DENSE_MAX_DIM (1 << 20)
#define TT_DENSE_MAX_GROUPS 32768
typedef struct {
  int32_t dtype;       /* tt_dtype of every tensor of the call                                   */
  int32_t activation;  /* tt_activation                                                          */
  int64_t rows;        /* rows of x, fewer than 2^31 - 2^16 - 1                                  */
  int32_t in_dim, out_dim; /* 1 .. TT_DENSE_MAX_DIM                                              */
  int32_t groups;      /* 0, or 1 .. TT_DENSE_MAX_GROUPS                                         */
  int32_t zero_rest;   /* rows of no group: 0 left as they were, 1 cleared                       */
  const int64_t *offsets; /* DEVICE int64[groups + 1]; NULL if groups == 0                       */
  int64_t ld_x;        /* elements between rows of x; 0: in_dim                                  */
  int64_t ld_out;      /* ... of out; 0: out_dim                                                 */
  int64_t ld_residual; /* ... of residual; 0: out_dim                                            */
  int64_t ld_grad;     /* ... of grad_out; 0: out_dim                                            */
  int64_t ld_dx;       /* ... of dx; 0: in_dim                                                   */
} tt_dense;

/*
 * Forward.  bias and residual may be NULL.  pre (nullable) receives z, [rows][out_dim] packed, rounded to
 * the dtype (in fp16 a z that would round to zero keeps its sign as the smallest number): what
 * tt_dense_backward needs if there is an activation.  out may be the residual's own memory with the same
 * row step; otherwise outputs overlap nothing (TT_ERR_INVALID_ARG where one starts where another tensor does).  Tensors need the alignment of an element only.
 *   workspace  DEVICE, 256-byte aligned, tt_dense_workspace_bytes(op, 0) bytes (NULL if that is 0), borrowed
 *              until the work has finished: calls that may overlap need one each.
 * Backward, from grad_out = dL/d out:
 *   dz = grad_out act'(z), dx = dz W, dW = dz^T x (per group, zeros for an empty one), dbias = sums of dz;
 *   any of dx, dw, dbias may be NULL.  dL/d residual is grad_out itself.  dz is rounded to the dtype
 *   before the products and dbias's sums.  x is needed for dw, w for dx, pre if there is an activation.
 *   workspace  tt_dense_workspace_bytes(op, 1) bytes, as above.
 * tt_dense_workspace_bytes returns 0 on invalid arguments too.
 */
size_t tt_dense_workspace_bytes(const tt_dense *op, int backward);
tt_status tt_dense_forward(const tt_dense *op, const void *x, const void *w, const void *bias, const void *residual,
                           void *out, void *pre, void *workspace, size_t workspace_bytes, void *stream);
tt_status tt_dense_backward(const tt_dense *op, const void *x, const void *w, const void *pre, const void *grad_out,
                            void *dx, void *dw, void *dbias, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Orthogonalised updates (Newton-Schulz products, as the Muon optimiser takes them): for each matrix G of
 * a batch
 *   X = G / (|G| + eps) with the Frobenius norm;  for each step, with its coefficients (a, b, c):
 *   X <- a X + (b A + c A^2) X,  A = X X^T           (a tall X from the other side: the same polynomial)
 * which takes every singular value s to a s + b s^3 + c s^5, step after step.  fp32 arithmetic whatever the
 * dtype (norms in 64 bits), the result rounded once; for 16-bit dtypes the factors of the products have 16
 * bits of significand, for fp32 24.  A zero matrix gives zeros (NaN if eps is 0); one with an infinity or
 * a NaN gives NaN in all its entries and does not touch the others of the batch.
 *   coefficients HOST float[steps][3], finite; steps 1 .. TT_ORTHO_MAX_STEPS; eps >= 0
 *   g, out       DEVICE; out may be g itself (with the same steps).
 *   workspace    DEVICE, 256-byte aligned, tt_orthogonalize_workspace_bytes(m) (0 on invalid arguments)
 */
#define TT_ORTHO_MAX_STEPS 32
#define TT_ORTHO_MAX_SIDE (1 << 20)
typedef struct {
  int32_t dtype;              /* tt_dtype of g and out                                           */
  int64_t batch, rows, cols;  /* sides 1 .. TT_ORTHO_MAX_SIDE, batch * rows * cols <= 2^36;
                                 batch <= 65535 above 64 x 512                                  */
  int64_t batch_step, row_step;         /* elements between matrices / rows of g; 0: packed       */
  int64_t out_batch_step, out_row_step; /* ... of out                                            */
} tt_matrices;
size_t tt_orthogonalize_workspace_bytes(const tt_matrices *m);
tt_status tt_orthogonalize(const tt_matrices *m, const void *g, void *out, int steps, const float *coefficients,
                           float eps, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The core update that goes with it, beside tt_core_sgd_update: with momentum, slice by slice,
 *   m <- mu m + dG,  u = nesterov ? dG + mu m : m,
 *   G <- G - lr sqrt(max(1, rows / cols)) ortho(u)   for each slice G of each core,
 * the slices being the matrices that multiply in a row of the table: G1[i1] d1 x R1, G2[i2] R1 x (d2 R2),
 * G3[i3] R2 x d3.  A slice whose u is zero stays as it is (eps > 0; else it
 * becomes NaN).  table->core[] and momentum[] are updated in place.
 *   dcore, momentum  HOST arrays of 3 DEVICE pointers, core-shaped
 *   workspace        DEVICE, 256-byte aligned, tt_core_ortho_workspace_bytes(table) (0 on invalid arguments)
 */
size_t tt_core_ortho_workspace_bytes(const tt_table *table);
tt_status tt_core_ortho_update(const tt_table *table, const float *const dcore[3], float *const momentum[3], float lr,
                               float mu, int nesterov, int steps, const float *coefficients, float eps,
                               void *workspace, size_t workspace_bytes, void *stream);

/*
 * The top of a model.  Layer norm, a router that deals rows to experts, and the softmax loss over a
 * catalogue.  fp32, bf16 or fp16 data with fp32 arithmetic (64 bits where said), rounded once; reproducible, no
 * floating-point atomics; nothing is allocated.  Tensors need the alignment of an element only; outputs
 * overlap nothing (TT_ERR_INVALID_ARG where one starts where another tensor of the call does).
 *
 * Layer norm of each row of x [rows][dim], mean and variance (of dim, not dim - 1) over the row:
 *   y = (x - mean) rstd weight + bias,  rstd = 1 / sqrt(variance + eps)
 * weight and bias [dim] may be NULL (one and zero).  Backward, with h = grad weight and x^ = (x - mean) rstd:
 *   dx = rstd (h - mean(h) - x^ mean(h x^)),  dweight = sum over rows of grad x^,  dbias = sum of grad
 * A row of equal values gives the bias if eps > 0 (without eps it has no answer: NaN or the bias); infinities and
 * NaN stay in their row of out and dx.  Any finite x will do: a row whose sum or squares leave the range of fp32 is taken
 * times a power of two.  What has to be a float is rstd (below 2^-126, of deviations beyond 2^126, it has fewer bits in the gradients).
 *   stats      DEVICE float[rows][2]: mean and rstd, written by the forward (may be NULL), read by the backward
 *   workspace  DEVICE, 256-byte aligned, tt_layer_norm_workspace_bytes(op) bytes; only for dweight and dbias
 */
#define TT_NORM_MAX_DIM (1 << 20)
typedef struct {
  int32_t dtype;  /* tt_dtype of every tensor but stats                                         */
  int32_t dim;    /* 1 .. TT_NORM_MAX_DIM                                                       */
  int64_t rows;   /* fewer than 2^31 - 1                                                        */
  int64_t ld_x;   /* elements between rows of x; 0: dim                                         */
  int64_t ld_out; /* ... of out; 0: dim                                                         */
  int64_t ld_grad; /* ... of grad_out; 0: dim                                                   */
  int64_t ld_dx;  /* ... of dx; 0: dim                                                          */
  float eps;      /* >= 0                                                                       */
} tt_norm;
size_t tt_layer_norm_workspace_bytes(const tt_norm *op);
tt_status tt_layer_norm_forward(const tt_norm *op, const void *x, const void *weight, const void *bias, void *out, float *stats, void *stream);
tt_status tt_layer_norm_backward(const tt_norm *op, const void *x, const void *weight, const float *stats, const void *grad_out,
                                 void *dx, void *dweight, void *dbias, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Routing.  For each row of logits z [rows][experts]:
 *   s = softmax(z), or sigmoid of each z;  c = s + bias[e] (bias chooses only, it is not in the weights)
 *   groups > 1: the experts are `groups` equal runs; the top_groups with the largest sum of their two best c
 *     (one, where a group has one) stay
 *   the `choices` experts with the largest c, largest first; equal ones by number, lowest first
 *   weights[j] = scale s, divided by the sum of the row's chosen s if renormalize (0 if that sum is 0)
 * Scores and comparisons are in 64 bits: which experts a row gets does not hang on rounding.  An expert whose
 * logit or c is -infinity is masked: never chosen, and no group's strength.  Where fewer than `choices` are left the numbers
 * are -1 and the weights 0 (a row of -infinity, as padding has, goes nowhere).  A NaN counts as the
 * largest (so it shows in the weights); a logit of +infinity makes a softmax row NaN.
 * Backward: from grad_weights the gradient of the logits through the weights (s only; numbers are fixed), in 64 bits as well.  Renormalised weights
 * hang on the chosen logits alone, and the others' gradient is zero.
 *   experts DEVICE int64[rows][choices]; weights, grad_weights float[rows][choices]; bias float[experts], nullable
 */
#define TT_ROUTE_MAX_EXPERTS 1024
#define TT_ROUTE_MAX_CHOICES 64
#define TT_ROUTE_MAX_GROUPS 64
typedef enum { TT_SCORES_SOFTMAX = 0, TT_SCORES_SIGMOID = 1 } tt_scores;
typedef struct {
  int32_t dtype;       /* tt_dtype of logits and dlogits                                         */
  int32_t scores;      /* tt_scores                                                              */
  int64_t rows;        /* rows * choices fewer than 2^31 - 2^16 - 1                              */
  int32_t experts;     /* 1 .. TT_ROUTE_MAX_EXPERTS                                              */
  int32_t choices;     /* 1 .. min(TT_ROUTE_MAX_CHOICES, experts of top_groups groups)           */
  int32_t groups;      /* 1 .. TT_ROUTE_MAX_GROUPS, a divisor of experts                         */
  int32_t top_groups;  /* 1 .. groups                                                            */
  int32_t renormalize; /* 0 or 1                                                                 */
  float scale;         /* finite                                                                 */
  int64_t ld_logits;   /* elements between rows of logits; 0: experts                            */
  int64_t ld_dlogits;  /* ... of dlogits; 0: experts                                             */
} tt_route;
tt_status tt_route_forward(const tt_route *op, const void *logits, const float *bias, int64_t *experts, float *weights, void *stream);
tt_status tt_route_backward(const tt_route *op, const void *logits, const int64_t *experts, const float *grad_weights, void *dlogits,
                            void *stream);

/*
 * The experts' order of n choices (the numbers above, row after row): the choices of one expert stand next to
 * each other, in the order in which they come.  Numbers outside [0, num_experts) go nowhere.
 *   offsets DEVICE int64[num_experts + 1]: each expert's first place, and the end (what tt_dense takes)
 *   slots   DEVICE int32[n]: each choice's place, -1 for none
 *   sources DEVICE int32[n]: each place's choice, -1 for places behind the end
 *   workspace DEVICE, 256-byte aligned, tt_expert_order_workspace_bytes(n, num_experts) (0: none needed, or invalid)
 */
size_t tt_expert_order_workspace_bytes(int64_t n, int32_t num_experts);
tt_status tt_expert_order(const int64_t *experts, int64_t n, int32_t num_experts, int64_t *offsets, int32_t *slots, int32_t *sources,
                          void *workspace, size_t workspace_bytes, void *stream);
/* tt_route_forward and the order of what it gives, in one call (workspace: of tt_expert_order for rows * choices). */
tt_status tt_route_order(const tt_route *op, const void *logits, const float *bias, int64_t *experts, float *weights, int64_t *offsets,
                         int32_t *slots, int32_t *sources, void *workspace, size_t workspace_bytes, void *stream);

/*
 * Rows to their experts and back.  slots [rows][choices] and sources [rows * choices] as above; places outside
 * [0, rows * choices) count as none, and a place is one choice's at most (of two, which one it gets is open).
 *   tt_expert_rows:     out[slots[r][j]] = x[r];  places without a source: left as they were, zeros with zero_rest
 *   tt_expert_combine:  out[r] = residual[r] + sum over j of weights[r][j] y[slots[r][j]]   (weights NULL: ones; what a
 *                       choice without a place would weigh is left out).  Also the gradient of tt_expert_rows.
 *   tt_expert_combine_backward:  dy[slots[r][j]] = weights[r][j] grad[r], zeros in places without a source;
 *                       dweights[r][j] = <grad[r], y[slots[r][j]]>, 0 without a place.  dy or dweights may be NULL.
 *                       The residual's gradient is grad itself.
 * out may be the residual's own memory with the same row step.
 */
typedef struct {
  int32_t dtype;       /* tt_dtype of the rows; weights are float                                */
  int32_t dim;         /* columns, 1 .. TT_NORM_MAX_DIM                                          */
  int64_t rows;        /* of x, and of combine's out and grad; rows * choices as in tt_route     */
  int32_t choices;     /* 1 .. TT_ROUTE_MAX_CHOICES                                              */
  int32_t zero_rest;
  int64_t ld_rows;     /* elements between rows of x, of combine's out and of grad; 0: dim       */
  int64_t ld_residual; /* ... of residual; 0: dim                                                */
  int64_t ld_places;   /* ... of tt_expert_rows' out and of y; 0: dim                            */
  int64_t ld_dy;       /* ... of dy; 0: dim                                                      */
} tt_deal;
tt_status tt_expert_rows(const tt_deal *op, const void *x, const int32_t *slots, const int32_t *sources, void *out, void *stream);
tt_status tt_expert_combine(const tt_deal *op, const void *y, const int32_t *slots, const float *weights, const void *residual, void *out,
                            void *stream);
tt_status tt_expert_combine_backward(const tt_deal *op, const void *y, const int32_t *slots, const int32_t *sources, const float *weights,
                                     const void *grad, void *dy, float *dweights, void *stream);

/*
 * Softmax cross entropy of rows against a catalogue of classes, without keeping the logits:
 *   z = x W^T + bias,  loss[r] = log(sum over classes of exp(z[r])) - z[r][label[r]]     x [rows][dim], W [classes][dim]
 * Rows whose label is ignore_index count for nothing: their loss and gradients are zero, whatever x holds
 * there.  A label that is neither that nor in [0, classes) gives a loss of NaN, and gradients with it.  A class whose bias is -infinity
 * is left out; a row with a logit of NaN or +infinity, or without a class, has the loss NaN.
 *   loss: TT_REDUCE_NONE float[rows]; TT_REDUCE_SUM, TT_REDUCE_MEAN float[1], the mean over the rows that count (0 if
 *     there are none)
 * Backward, from grad_loss (float[rows], or float[1]): with G = (softmax(z) - onehot(label)) times the row's share of it
 *   dx = G W,  dW = G^T x,  dbias = sums of G's columns;  any of dx, dw, dbias may be NULL.
 * G is formed again, a piece of the classes at a time (of rows of up to 128 elements it is never stored), and in 16 bits rounded to the
 * dtype before the products: without the share that all rows have of a sum or a mean, which is multiplied in at the end, and in fp16 by
 * powers of two that keep it in the range.  fp32 products are of three bf16 parts, as in tt_dense; those of rows of up to 128 elements do
 * without the fp32 instruction where parts cannot do (numbers below 2^-100 have fewer bits, numbers that bf16 cannot hold give NaN).  Losses
 * and lse are float whatever the dtype: lse is rounded by up to 2^-24 of itself, and G's probabilities are off by that, relative to their size.
 *   labels DEVICE int64[rows];  stats DEVICE float[rows][2]: the log of the sum and the loss of each row, 0 in rows that do not
 *   count; written by the forward (not NULL), read by the backward (which forms the label's softmax - 1 from the loss; the
 *   loss is of the other classes' share beside the label, so the relative precision of both lasts however sure a row is, and no loss is below zero)
 *   workspace DEVICE, 256-byte aligned, tt_cross_entropy_workspace_bytes(op, backward) (0 on invalid arguments).  For rows of up
 *   to 128 elements it grows with the classes: W's rows over again, padded to 64 or 128 elements of 2 bytes (fp32: 6), forward and backward
 *   (500001 x 128 in fp32 384 MB; 16-bit rows of just these lengths are read where they are).  For longer ones: a piece of G, 128 MB or 256 classes of
 *   all rows, x and its gradient's sums.
 */
typedef enum { TT_REDUCE_NONE = 0, TT_REDUCE_SUM = 1, TT_REDUCE_MEAN = 2 } tt_reduce;
#define TT_LOSS_MAX_CLASSES (1 << 30)
typedef struct {
  int32_t dtype;        /* tt_dtype of x, w, bias and their gradients                            */
  int32_t reduce;       /* tt_reduce                                                             */
  int64_t rows;         /* fewer than 2^31 - 2^16 - 1                                            */
  int32_t dim;          /* 1 .. TT_DENSE_MAX_DIM                                                 */
  int32_t classes;      /* 1 .. TT_LOSS_MAX_CLASSES                                              */
  int64_t ignore_index;
  int64_t ld_x;         /* elements between rows of x; 0: dim                                    */
  int64_t ld_dx;        /* ... of dx; 0: dim                                                     */
} tt_loss;
size_t tt_cross_entropy_workspace_bytes(const tt_loss *op, int backward);
tt_status tt_cross_entropy_forward(const tt_loss *op, const void *x, const void *w, const void *bias, const int64_t *labels, float *loss, float *stats,
                                   void *workspace, size_t workspace_bytes, void *stream);
tt_status tt_cross_entropy_backward(const tt_loss *op, const void *x, const void *w, const void *bias, const int64_t *labels, const float *stats,
                                    const float *grad_loss, void *dx, void *dw, void *dbias, void *workspace, size_t workspace_bytes,
                                    void *stream);

/*
 * Waits for `stream`, copies the plan's device-side counters to the host and
 * reports deferred errors.  counts_out (HOST, nullable) receives
 * {U_r, U_p, valid lookups, status bits}.  Returns TT_ERR_INDEX_RANGE if any
 * index was out of range or the offsets were not a valid CSR array.
 */
tt_status tt_plan_status(const tt_plan *plan, void *stream, int64_t counts_out[4]);

const char *tt_strerror(tt_status status);

/*
 * Kernel timing helper for benchmarks (not needed by the operator itself, and the one place
 * where the library owns anything: a host object holding HIP events).  A tt_prof selects one
 * kernel of the planned path; while it is attached to a plan (plan->prof), every launch of that
 * kernel made with the plan is bracketed by two HIP events recorded on the launch stream.
 * tt_prof_collect waits for the recorded events, returns the summed duration and the number of
 * launches since the last collect, and rearms the object.  At most `capacity` launches are
 * recorded between two collects; later ones run untimed.
 */
typedef enum {
  TT_KERNEL_FWD_CONTRACT = 0, /* prefix products + distinct rows (forward)                   */
  TT_KERNEL_BAG_SUM = 1,      /* per-bag sum of distinct rows                                */
  TT_KERNEL_GRAD_MERGE = 2,   /* stage 1 of merging grad_out per distinct row                */
  TT_KERNEL_BWD_CONTRACT = 3, /* backward contraction kernel (without the sum of split parts)  */
  TT_KERNEL_SORT_SCATTER = 4, /* one radix-sort scatter pass of the main lookup sort         */
  TT_KERNEL_SGD = 5,          /* core update                                                 */
  TT_KERNEL_P12_FILL = 6,     /* reuse buffer of the sample-level forward                    */
  TT_KERNEL_BAG_CHAINS = 7,   /* per-bag chains of the sample-level forward                  */
  TT_KERNEL_COUNT = 8
} tt_kernel;

typedef struct tt_prof tt_prof;
tt_prof *tt_prof_create(int kernel, int capacity); /* NULL on failure                        */
void tt_prof_destroy(tt_prof *prof);
/* HOST out-params; returns TT_ERR_HIP if an event query fails */
tt_status tt_prof_collect(tt_prof *prof, double *total_ms, int64_t *launches);
const char *tt_kernel_name(int kernel);

#ifdef __cplusplus
}
#endif
#endif /* TT_EMB_H_ */
