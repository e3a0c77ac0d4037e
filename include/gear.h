/*
 * libgear - the Gear Training sparse-part step on one MI355X (gfx950).
 *
 * "Gear Training: A new way to implement high-performance model-parallel
 * training" splits a model into a Sparse Part (user id, URL, ...) trained every
 * step by a Fastgear Worker and a Dense Part (image CNN) owned by a Slowgear
 * Worker.  The Dense Part is neither run forward nor backward in a training
 * step: its outputs, the Dense Feature Vectors (DFVs), are fetched from a cache
 * by image id (Section 1, second point; Section 3, steps 1-3), and the
 * gradients with respect to the DFVs are collected per image until M have
 * arrived and are then averaged (Section 1, third point; Section 3, step 6).
 *
 * This library is that per-step work.  All pointers named "device" are device
 * memory owned by the caller; the library allocates no device memory and keeps
 * no state between calls except one helper stream and five events per device,
 * created at the first gear_step that uses them (default priority; part of a long step
 * runs on the helper stream, forked from and joined back into the caller's stream).
 * Calls enqueue their kernels on the given hipStream_t (passed as void*) and return
 * without synchronising.  Results are valid once the caller has synchronised that
 * stream.  The stream must belong to the current device.  The entry points may
 * be called from several host threads; steps issued on one device are enqueued
 * one after the other (a per-device lock is held while a step enqueues), and what
 * they do to counts and grad_accum happens in the order they were issued, also from
 * different streams: steps with tables of their own may share such a store.  (Steps
 * with one_stream set, gear_step_static and steps being captured into a graph take no
 * part in that order: they run in their stream's, or their graph's.)  Each
 * step needs a workspace of its own while it is in flight.  If a call returns
 * GEAR_ERR_HIP part-way through its enqueue, whatever it had put on the helper
 * stream is still joined back into the caller's stream before it returns.
 *
 * Errors.  Everything the host can check (NULL pointers, dimensions, M < 1,
 * sizes over the configured maxima, a workspace that is too small) is reported
 * through the return value and nothing is enqueued.  What only the device can
 * see (an id outside its table, offsets that are not a CSR index, a ready list
 * longer than ready_cap) is written to the device word `status`, and the step
 * then leaves every table, accumulator and counter as it was.  A step writes that
 * word and never reads it (it keeps its own in the workspace): other calls may
 * report into the same word while a step runs without disturbing the step.
 */
#ifndef GEAR_H
#define GEAR_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define GEAR_MAX_LAYERS 8

typedef enum gear_status {
  GEAR_OK = 0,
  GEAR_ERR_INVALID = 1,  /* host-checked: NULL, bad dims, M < 1, lr not finite, B or nnz over max */
  GEAR_ERR_RANGE = 2,    /* device-checked: id out of range, offsets not a CSR index            */
  GEAR_ERR_CAPACITY = 3, /* workspace too small (host) or ready list over ready_cap (device)    */
  GEAR_ERR_HIP = 4       /* a HIP call failed                                                    */
} gear_status;

typedef enum gear_dtype { GEAR_F32 = 0, GEAR_BF16 = 1 } gear_dtype;

/* Shape of the Sparse Part and of the tables.  Plain data, read by every call.
 * The Sparse Part is x = [user row | URL row | mean of the view's DFVs] of width
 * F = 2*emb_dim + dfv_dim, followed by n_layers affine layers of output widths
 * layer_out[0..n_layers-1] with ReLU between them; the last width must be 1 (the
 * logit).  Requirements: 2 <= n_layers <= GEAR_MAX_LAYERS, emb_dim % 8 == 0,
 * dfv_dim % 8 == 0, hidden widths % 8 == 0, last hidden width <= 1024, table sizes below 2^31. */
typedef struct gear_config {
  int64_t n_users, n_urls, n_images;
  int32_t emb_dim, dfv_dim;
  int32_t n_layers;
  int32_t layer_out[GEAR_MAX_LAYERS];
  int32_t emb_dtype;     /* gear_dtype of user_emb / url_emb rows                              */
  int32_t dfv_dtype;     /* gear_dtype of dfv_cache rows                                       */
  int32_t mlp_dtype;     /* operand type of the MLP contractions; accumulation is always fp32  */
  int32_t max_batch;     /* largest B a step may carry                                         */
  int32_t max_nnz;       /* largest number of (view, image) occurrences a step may carry       */
  uint64_t seed;         /* seed of gear_init_tables                                           */
  float emb_init_std;    /* standard deviation of the initial embedding rows                   */
} gear_config;

/* Trainable state of the Sparse Part (device).  mlp_params packs, layer after layer,
 * W_l [layer_out[l] x in_l] row-major then b_l [layer_out[l]], all fp32 (master copy). */
typedef struct gear_tables {
  void *user_emb;        /* [n_users x emb_dim], emb_dtype, row-major */
  void *url_emb;         /* [n_urls  x emb_dim], emb_dtype, row-major */
  float *mlp_params;     /* gear_mlp_param_count(cfg) floats          */
} gear_tables;

/* One batch of page views (Section 1, Table 1: user id, URL, several image ids).
 * All arrays are device memory.  View b owns img_id[img_off[b] .. img_off[b+1]);
 * img_off[0] = 0, img_off[B] = nnz.  A view may have no image (its pooled DFV is 0
 * and it produces no DFV gradient).  The same image may occur several times, also
 * inside one view; every occurrence counts. */
typedef struct gear_batch {
  int32_t B, nnz;
  const int32_t *user_id; /* [B]   in [0, n_users)        */
  const int32_t *url_id;  /* [B]   URL hash bucket in [0, n_urls) */
  const int32_t *img_off; /* [B+1]                         */
  const int32_t *img_id;  /* [nnz] in [0, n_images)        */
  const float *label;     /* [B]   click label in {0, 1}   */
} gear_batch;

/* Outputs of one step (device memory, caller-owned). */
typedef struct gear_step_out {
  float *loss;            /* [1] mean sigmoid cross-entropy of the batch                         */
  int32_t *n_ready;       /* [1] number of emitted averages (0 when status is not 0)             */
  int32_t *ready_ids;     /* [ready_cap] image ids, ascending; an image that completed several
                             groups of M in this step appears once per group, oldest first       */
  float *ready_grads;     /* [ready_cap x dfv_dim] fp32, row r = average for ready_ids[r]        */
  int32_t ready_cap;      /* rows available; max_nnz is always enough                            */
  int32_t *status;        /* [1] 0, GEAR_ERR_RANGE or GEAR_ERR_CAPACITY                          */
  /* Optional exports of the image grouping (NULL = skip).  Sizes: [max_nnz], [max_nnz+1],
   * [max_nnz], [1].  unique = distinct image ids ascending; segment s of the stable
   * permutation perm is perm[segoff[s] .. segoff[s+1]), flat CSR positions ascending. */
  int32_t *dbg_img_unique, *dbg_img_segoff, *dbg_img_perm, *dbg_n_img_unique;
  /* Optional timing (NULL = off): a gear_profile from gear_profile_create.  Every kernel launch of
   * the step is then bracketed by HIP events on the stream it is launched on (the caller's or the
   * helper stream); read them with gear_profile_span after synchronising the caller's stream. */
  void *profile;
  /* Nonzero: every kernel of the step is launched on the caller's stream, one after another, and
   * the helper stream is not used.  Same results; for timing each kernel alone, or for callers
   * that want no second stream and no event.  (With zero a step too short to gain from the helper
   * stream does without it as well, and keeps its place in the order of the device's steps.) */
  int32_t one_stream;
} gear_step_out;

/* Bytes of scratch device memory gear_step needs for this configuration (0 on a bad config). */
size_t gear_workspace_bytes(const gear_config *cfg);

/* Number of floats in gear_tables.mlp_params, and the float offset of W_l (which = 0) or
 * b_l (which = 1) inside it; -1 on a bad argument. */
int64_t gear_mlp_param_count(const gear_config *cfg);
int64_t gear_mlp_param_offset(const gear_config *cfg, int32_t layer, int32_t which);

/* Byte offset and size, inside the workspace, of an intermediate of the last gear_step, for
 * inspection by tests: "x" [max_batch x F] mlp_dtype, "logits" [max_batch] f32, and dLoss/dx in two
 * pieces: "dx_emb" [max_batch x 2*emb_dim] f32 (user and URL slots) and "dx_dfv" [max_batch x dfv_dim]
 * in mlp_dtype (the DFV slot), and "h0", "h1", ... [max_batch x layer_out[l]] mlp_dtype, the stored
 * activations of the hidden layers (zero where the unit is off).
 * Returns GEAR_ERR_INVALID for an unknown name. */
gear_status gear_workspace_region(const gear_config *cfg, const char *name, size_t *offset, size_t *bytes);

/* Fill dst [n_rows x dim] (device, `dtype`) with zero-mean noise of standard deviation `std`:
 * element (r, c) is a fixed function of (seed, stream_id, r*dim + c) - Philox4x32-10 with counter
 * (idx_lo, idx_hi, stream_id, 0) and key (seed_lo, seed_hi); the eight 16-bit halves of its output
 * are summed, centred, and scaled by one fp32 multiply.  (Section 4.1 fixes only a standard
 * deviation for the initial values.) */
gear_status gear_fill_normal(void *dst, int32_t dtype, int64_t n_rows, int32_t dim, uint64_t seed,
                             uint32_t stream_id, float std, void *stream);

/* Initial state: user_emb (stream 1) and url_emb (stream 2) ~ N(0, emb_init_std^2); W_l (stream
 * 16+l) ~ N(0, 2/in_l), b_l = 0; grad_accum [n_images x dfv_dim] f32 and counts [n_images] i32
 * zeroed (no gradient has arrived yet: Section 1, third point). */
gear_status gear_init_tables(const gear_config *cfg, gear_tables *tables, float *grad_accum,
                             int32_t *counts, void *stream);

/* One Fastgear training step (Section 3, steps 4 and 5) plus the Slowgear gradient bookkeeping
 * (Section 1, third point; Section 3, step 6; Eq. 1, left factor):
 *   x_b   = [user_emb[user_b] | url_emb[url_b] | mean_j dfv_cache[img_j]]
 *   loss  = mean_b BCE(sigmoid(MLP(x_b)), label_b)
 *   MLP parameters and the touched embedding rows take one SGD step with rate lr, gradients
 *     of a row summed over its views in batch order;
 *   every occurrence j of image i in view b contributes g_j = dLoss/dx_b[DFV slot] / n_b;
 *   the gradients of image i, in flat CSR order and continuing from earlier steps, are cut into
 *     groups of M: a completed group is emitted as (i, mean of the group) and forgotten, an
 *     unfinished one stays summed in grad_accum[i];  counts[i] += occurrences of i.
 * dfv_cache [n_images x dfv_dim] (dfv_dtype) is read only.  grad_accum [n_images x dfv_dim] f32 and
 * counts [n_images] i32 must be the arrays given to gear_init_tables and M must not change over
 * their life.  workspace: gear_workspace_bytes(cfg) bytes, 256-byte aligned; the tables,
 * mlp_params, dfv_cache, grad_accum and ready_grads 16-byte aligned.  Results do not depend on the
 * order in which the device schedules its work. */
gear_status gear_step(const gear_config *cfg, const gear_batch *batch, gear_tables *tables,
                      const void *dfv_cache, float *grad_accum, int32_t *counts, int32_t M, float lr,
                      void *workspace, size_t workspace_bytes, gear_step_out *out, void *stream);

/* gear_step for callers that cannot allocate device memory or must not see an allocation happen:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  The workspace
 * is a static device array inside the library (64 MiB = 67 108 864 bytes per GPU, held until the
 * process ends) instead of a caller's buffer, and every kernel is launched on the caller's stream
 * (no helper stream, no event).  The call allocates nothing.  Configurations whose
 * gear_workspace_bytes(cfg) exceeds 67 108 864 are rejected with GEAR_ERR_CAPACITY and nothing is
 * enqueued (of the workloads this library is measured on that admits batches of about 8 000 views
 * with 256-wide DFVs; the largest needs 760 MiB and has to bring its own workspace to gear_step).
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two streams,
 * two host threads) race on it and must be ordered by the caller; nothing in it has to survive
 * between calls and nothing in it has to be cleared beforehand.  Inputs, outputs, alignment, errors
 * and results (bit for bit) as for gear_step with one_stream set. */
gear_status gear_step_static(const gear_config *cfg, const gear_batch *batch, gear_tables *tables,
                             const void *dfv_cache, float *grad_accum, int32_t *counts, int32_t M, float lr,
                             gear_step_out *out, void *stream);

/* Adam for the Sparse Part (Section 4.1 trains with the Adam optimiser at rate 1e-4; its other
 * constants are not given).  Kingma & Ba, Algorithm 1, at step t = 1, 2, ...:
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g^2;
 *   w -= lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps).
 * MLP parameters: every element every step; mlp_m, mlp_v are laid out like mlp_params.  Embedding
 * rows: only the rows a step touches move, moments included (their decay is applied per touch, not
 * per elapsed step), with the global t in the bias corrections; user_m/v and url_m/v are fp32 tables
 * [n x emb_dim] whatever emb_dtype is.  All moment arrays are device memory, caller-owned, 16-byte
 * aligned, zero before the first step. */
typedef struct {
  float beta1, beta2, eps;
  int32_t t;                  /* this step's number, from 1 */
  float *user_m, *user_v;     /* [n_users x emb_dim] */
  float *url_m, *url_v;       /* [n_urls x emb_dim] */
  float *mlp_m, *mlp_v;       /* [gear_mlp_param_count] */
} gear_adam;

/* gear_step with Adam instead of plain SGD for every parameter of the Sparse Part; adam = NULL is
 * gear_step.  Everything else as for gear_step. */
gear_status gear_step_adam(const gear_config *cfg, const gear_batch *batch, gear_tables *tables,
                           const void *dfv_cache, float *grad_accum, int32_t *counts, int32_t M, float lr,
                           const gear_adam *adam, void *workspace, size_t workspace_bytes,
                           gear_step_out *out, void *stream);

/* Overwrite cached DFVs (Section 1, second point: cached inference results are replaced after the
 * inference expired time).  Row image_ids[r] of dfv_cache becomes new_dfv[r] (device, dfv_dtype,
 * [n x dfv_dim]); image_ids = NULL means rows 0..n-1.  Ids must be distinct.  Gradient accumulators
 * and counters are a different table and are not touched.  status (device word, may be NULL) is
 * set to GEAR_ERR_RANGE if an id is outside [0, n_images); such rows are skipped. */
gear_status gear_refresh_dfv(const gear_config *cfg, void *dfv_cache, const int32_t *image_ids,
                             const void *new_dfv, int64_t n, int32_t *status, void *stream);

/* Which cached inference results a batch asks for have expired (Section 1, second point and
 * Section 3: a cache entry is recomputed once it is older than the inference expired time;
 * Section 4.1, Table 2: that time trades freshness for speed).  dfv_stamp [n_images] i32 (device,
 * caller-owned) holds the time each row was last written, in the caller's unit (steps, seconds).
 * expired_ids (device, room for n entries) receives, ascending, the distinct ids among
 * image_ids [n] (device, a batch's flat image list) with now - dfv_stamp[id] >= expiry, and
 * n_expired (device word) their number.  The caller recomputes those rows and hands them to
 * gear_refresh_dfv and gear_stamp_dfv.  expiry >= 0.  status (device word, not NULL) becomes
 * GEAR_ERR_RANGE if an id is outside [0, n_images); then n_expired is 0.  workspace as for
 * gear_step, with max_nnz >= n. */
gear_status gear_expired_ids(const gear_config *cfg, const int32_t *image_ids, int32_t n,
                             const int32_t *dfv_stamp, int32_t now, int32_t expiry, void *workspace,
                             size_t workspace_bytes, int32_t *expired_ids, int32_t *n_expired,
                             int32_t *status, void *stream);

/* dfv_stamp[image_ids[r]] = now for r < n; image_ids = NULL means rows 0..n-1.  status (device
 * word, may be NULL) becomes GEAR_ERR_RANGE if an id is outside [0, n_images); such ids are skipped. */
gear_status gear_stamp_dfv(const gear_config *cfg, int32_t *dfv_stamp, const int32_t *image_ids, int64_t n,
                           int32_t now, int32_t *status, void *stream);

/* gear_refresh_dfv and gear_stamp_dfv for a list whose length is only known on the device (the
 * output of gear_expired_ids, say): rows r < *n_rows are used, where n_rows is a device word read
 * when the kernels run, 0 <= *n_rows <= max_rows (a larger value is cut to max_rows); image_ids and
 * new_dfv hold max_rows entries.  The host need not read the count and can keep enqueuing.
 * Otherwise as the calls above (image_ids must be given). */
gear_status gear_refresh_dfv_n(const gear_config *cfg, void *dfv_cache, const int32_t *image_ids,
                               const void *new_dfv, const int32_t *n_rows, int64_t max_rows, int32_t *status,
                               void *stream);
gear_status gear_stamp_dfv_n(const gear_config *cfg, int32_t *dfv_stamp, const int32_t *image_ids,
                             const int32_t *n_rows, int64_t max_rows, int32_t now, int32_t *status, void *stream);

/* A stand-in Dense Part, so that the loop of the method can be closed on one device: a linear map
 * DFV[i] = Wd raw[i] from fixed per-image features raw [n_images x raw_dim] (f32, device) with
 * weights Wd [dfv_dim x raw_dim] (f32, device).  Not the paper's CNN: the smallest model that has
 * an inference pass feeding the cache (Section 3, steps 1-2) and a backward pass consuming the
 * averaged gradients (Section 3, step 6; Eq. 1, right factor).  raw_dim and dfv_dim are multiples
 * of 8; max_rows bounds n and n_ready of the calls below. */
typedef struct {
  int64_t n_images;
  int32_t raw_dim, dfv_dim;
  gear_dtype dfv_dtype; /* type of the rows gear_dense_infer writes (the cache's) */
  int32_t max_rows;
} gear_dense_config;

size_t gear_dense_workspace_bytes(const gear_dense_config *cfg);

/* out_rows [n x dfv_dim] (device, dfv_dtype) = Wd raw[image_ids[r]]; image_ids = NULL means images
 * 0..n-1.  The rows are what gear_refresh_dfv takes.  workspace: gear_dense_workspace_bytes(cfg)
 * bytes, 256-byte aligned.  status (device word, not NULL): GEAR_ERR_RANGE if an id is outside
 * [0, n_images) (that row is then computed from image 0). */
gear_status gear_dense_infer(const gear_dense_config *cfg, const float *raw, const float *wd,
                             const int32_t *image_ids, int32_t n, void *out_rows, void *workspace,
                             size_t workspace_bytes, int32_t *status, void *stream);

/* Back-propagation of a step's ready list through the stand-in (Eq. 1, right factor):
 * Wd -= lr * sum_e ready_grads[e] (outer) raw[ready_ids[e]], e < n_ready (a host count: the caller
 * reads n_ready back first), summed in a fixed shape that depends on n_ready only.  status (device
 * word, not NULL): GEAR_ERR_RANGE if an id is outside [0, n_images); Wd is then unchanged. */
gear_status gear_dense_backward(const gear_dense_config *cfg, const float *raw, float *wd,
                                const int32_t *ready_ids, const float *ready_grads, int32_t n_ready,
                                float lr, void *workspace, size_t workspace_bytes, int32_t *status,
                                void *stream);

/* The same with the number of emissions read from the device word n_ready when the kernels run
 * (a step's gear_step_out.n_ready; at most max_rows, which ready_ids and ready_grads must hold): the
 * host need not read it back.  The sum is split into a fixed number of ranges over *n_ready. */
gear_status gear_dense_backward_n(const gear_dense_config *cfg, const float *raw, float *wd,
                                  const int32_t *ready_ids, const float *ready_grads, const int32_t *n_ready,
                                  float lr, void *workspace, size_t workspace_bytes, int32_t *status,
                                  void *stream);

/* Sort-by-key grouping used for the embedding updates and the per-image accumulation, exposed
 * for tests: keys [n] in [0, key_range) -> distinct keys ascending (unique [n]), segment offsets
 * (segoff [n+1]), stable permutation (perm [n]) and the number of distinct keys (n_unique [1]).
 * All device memory; workspace as for gear_step with max_batch, max_nnz >= n. */
gear_status gear_group_ids(const gear_config *cfg, const int32_t *keys, int32_t n, int64_t key_range,
                           void *workspace, size_t workspace_bytes, int32_t *unique, int32_t *segoff,
                           int32_t *perm, int32_t *n_unique, void *stream);

/* The MLP's matrix products (Section 3, step 4: forward and back-propagation on the Sparse Part),
 * exposed for tests.  All device memory, 16-byte aligned; accumulation is fp32.
 *   form 0 (forward / dgrad): out[M x N] = A[M x K] * B[N x K]^T, operands of `dtype`, K and N
 *     multiples of 8; epilogue 0: out(dtype) = max(acc + bias[n], 0); 1: out(dtype) = aux[m,n] > 0
 *     ? acc : 0 with aux [M x N] of `dtype`; 2: out(f32) = acc.
 *   form 1 (wgrad): out[M x N] (f32) = A[K x M]^T * B[K x N], M and N multiples of 8, contracted in
 *     `splits` (1..64) ranges of K whose partial results (partial: [splits x M x N] f32) are added in
 *     ascending order.
 * status: device word, must be 0 on entry (a non-zero word makes the kernels return at once). */
gear_status gear_gemm(int32_t dtype, int32_t form, const void *A, const void *B, int32_t M, int32_t N, int32_t K,
                      int32_t epilogue, const float *bias, const void *aux, void *out, int32_t splits,
                      float *partial, int32_t *status, void *stream);

/* ---- Operators of a Dense Part made of experts ------------------------------------------------------------------
 * What a Dense Part larger than the stand-in is made of: a root-mean-square norm of its features, products with
 * weights of its own for every kind of image (rows grouped by expert), the same products in 8-bit floating point for
 * the inference that refreshes the cache (Section 3, steps 1-2), the gradients of all of them for its back-propagation
 * (Section 3, step 6), and the clipping of those by their global norm.
 *
 * As elsewhere: device memory of the caller's, no allocation, nothing kept between calls, kernels enqueued on `stream`,
 * results independent of how the device schedules its work.  Widths (dim, K, N) are multiples of 8; the distance
 * between rows (ld_*, in elements) is a multiple of 8 and at least the width, below 2^20; matrices start on 16 bytes.
 * At most 2^30 rows.  A call on no rows does nothing but what it says it does then.  Sums are fp32 (norms of lists of gradients
 * and norms in 8 bits: fp64).
 *
 * 8 bits.  A row of `dim` values in 8 bits is gear_rows8_ld(dim) bytes of e4m3 (4 exponent, 3 fraction bits, largest
 * 448, no infinity), whole blocks of 128 with zeros behind the row's end, and gear_scales8_ld(dim) scale bytes, one for
 * each block, a multiple of four of them.  Scale byte b stands for 2^(b - 127).  It is the smallest power of two with
 * max |v| <= 448 2^(b - 127) over the block's finite values v (not below 2^-127; 1 for a block of zeros), so scaling
 * loses nothing and what is rounded (to nearest, ties to even) is only the value's fraction.  Infinities and NaN
 * become NaN and do not count for the scale.  The matrix instruction takes the scales as they are.  It adds eight
 * neighbouring products at once and keeps of each what is at least 2^-13 of the largest one's power of two; everything
 * beyond these eight is added in fp32.  Of random rows that is 1.5e-5 of the result (576 to 4096 columns; the rounding of the
 * operands to 8 bits: 4e-2), so results in fp32 are no more exact than that. */
#define GEAR_E4M3 2            /* beside gear_dtype, where a call says that it takes it: 8 bits with scales */
#define GEAR_MAX_NORM_DIM 65536
#define GEAR_MAX_EXPERTS 1024

int64_t gear_rows8_ld(int32_t dim);
int64_t gear_scales8_ld(int32_t dim);

/* y = h / sqrt(mean(h^2) + eps) * gain with h = x + residual (residual may be NULL: h = x), a row at a time.
 * Outputs, each NULL where it is not wanted, one at least: sum = h (of `dtype`, may be x or residual itself), y (of
 * `dtype`), and q8 with scale, y in 8 bits.  With both y and q8, y holds what the 8 bits stand for (as far as `dtype`
 * holds it), so that gradients can be taken of what the 8-bit product saw.  y may be x or residual itself unless sum is the same.
 * gain [dim] fp32, 16-byte aligned; eps >= 0; dim at most GEAR_MAX_NORM_DIM.  The norm is that of h before it is rounded to `dtype`.
 * Squares and their sum are fp32 (without q8) and have to lie in its range: rows of a root mean square up to 7e16 (at any dim), and from
 * 1e-18 where eps is smaller than their squares. */
typedef struct {
  int64_t rows;
  int32_t dim, dtype;    /* gear_dtype of x, residual, sum and y */
  float eps;
  const void *x, *residual;
  const float *gain;
  void *sum, *y;
  int64_t ld_x, ld_residual, ld_sum, ld_y;
  uint8_t *q8, *scale;   /* [rows x gear_rows8_ld], [rows x gear_scales8_ld]; 16-byte and 4-byte aligned */
} gear_norm_args;
gear_status gear_rmsnorm(const gear_norm_args *a, void *stream);

/* Backward pass at h (the forward pass's sum, or x): with s = (mean(h^2) + eps)^-1/2 and a = dy * gain
 *   dx = s a - h s^3 mean(a h) + dsum        (dsum, what flows into h itself; may be NULL; s^3 is not formed: h may be as large or small
 *                                             as the norm in fp32 takes it)
 *   dgain = sum over rows of dy h s          ([dim] fp32, 16-byte aligned; may be NULL)
 * dx is the gradient of both x and residual; it may be dy or dsum itself.  workspace (256-byte aligned) as
 * gear_norm_backward_workspace_bytes says; not needed where dgain is NULL.  No rows: dgain is zero. */
typedef struct {
  int64_t rows;
  int32_t dim, dtype;    /* gear_dtype of h, dy, dsum and dx */
  float eps;
  const void *h, *dy, *dsum;
  const float *gain;
  void *dx;
  float *dgain;
  int64_t ld_h, ld_dy, ld_dsum, ld_dx;
} gear_norm_backward_args;
size_t gear_norm_backward_workspace_bytes(int64_t rows, int32_t dim);
gear_status gear_rmsnorm_backward(const gear_norm_backward_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* x [rows x dim] (dtype, ld_x; dim at most GEAR_MAX_NORM_DIM) in 8 bits: q8 and scale as above. */
gear_status gear_rows8(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t dim, uint8_t *q8, uint8_t *scale,
                       void *stream);

/* Weights laid out for the products.  w [experts x N x K] (src_dtype GEAR_F32 or GEAR_BF16, contiguous) is converted to
 * operand_dtype (GEAR_F32, GEAR_BF16 or GEAR_E4M3) and stored in the order in which the matrix instruction takes it: in
 * `packed` for products that contract over K (Y = X W^T), in `packed_transposed` for those that contract over N (dX = dY W);
 * either may be NULL.  GEAR_E4M3 (packed only): one scale byte for each 128 x 128 weights, in scale
 * [experts x ceil(N / 128) x gear_scales8_ld(K)] (gear_weight_scales_bytes, 4-byte aligned), else NULL.  Both take
 * gear_packed_weights_bytes bytes, 16-byte aligned.  (0 bytes on a bad argument.) */
size_t gear_packed_weights_bytes(int32_t operand_dtype, int32_t experts, int32_t N, int32_t K, int32_t transposed);
size_t gear_weight_scales_bytes(int32_t experts, int32_t N, int32_t K);
gear_status gear_pack_weights(const void *w, int32_t src_dtype, int32_t operand_dtype, int32_t experts, int32_t N, int32_t K,
                              void *packed, void *packed_transposed, uint8_t *scale, void *stream);

/* out[r] = x[r] W_e^T for the rows r in [off[e], off[e+1]) of every expert e: W_e [N x K] as packed above (from weights
 * [N x K], or transposed from [K x N]).  off [experts + 1] is device memory, 0 = off[0] <= off[1] <= ... <=
 * off[experts] <= rows; the host need not know it.  Rows from off[experts] on belong to nobody and are not written.
 * off = NULL: one expert takes all rows.  rows is at most 2^30.
 * x [rows x K] of `dtype` (GEAR_E4M3: ld_x in bytes, at least gear_rows8_ld(K) and a multiple of 16; x_scale
 * [rows x gear_scales8_ld(K)], 4-byte aligned).  out [rows x N] of out_dtype: fp32, or bf16 where dtype is not GEAR_F32.
 * status (device word, may be NULL where off is): GEAR_ERR_RANGE if off is not as said, and out is then left as it was;
 * otherwise 0, or what it was before where keep_status is not 0: many calls, on any streams, may then share a word that holds an error
 * until the caller clears it. */
typedef struct {
  int32_t dtype, out_dtype;
  int64_t rows;
  int32_t K, N, experts;
  const void *x;
  const uint8_t *x_scale;
  const void *packed;
  const uint8_t *w_scale;
  const int32_t *off;
  void *out;
  int64_t ld_x, ld_out;
  int32_t *status;
  int32_t keep_status;
} gear_expert_args;
gear_status gear_expert_product(const gear_expert_args *a, void *stream);

/* dw_e [N x K] = dy_e^T x_e over the rows of every expert, dw [experts x N x K] fp32 contiguous, 16-byte aligned (zeros
 * for an expert without rows).  dy [rows x N] and x [rows x K] of `dtype` (GEAR_F32 or GEAR_BF16); off, status and
 * keep_status as above, a bad off leaves dw as it was.  workspace (256-byte aligned) as gear_expert_wgrad_workspace_bytes says. */
typedef struct {
  int32_t dtype;
  int64_t rows;
  int32_t K, N, experts;
  const void *dy, *x;
  const int32_t *off;
  float *dw;
  int64_t ld_dy, ld_x;
  int32_t *status;
  int32_t keep_status;
} gear_expert_wgrad_args;
size_t gear_expert_wgrad_workspace_bytes(int32_t dtype, int64_t rows, int32_t experts, int32_t N, int32_t K);
gear_status gear_expert_wgrad(const gear_expert_wgrad_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* A list of gradients, for their global norm and for clipping.  The caller describes its tensors on the host (contiguous,
 * n >= 0 elements, aligned to an element; dst may be src or another tensor, and may be NULL where only the norm is wanted.
 * No dst may share memory with its src in part, with another entry's dst or with another entry's src: who scales an element first
 * would be chance.  gear_grad_list_pack does not look for that, the caller knows its tensors), gear_grad_list_pack writes the
 * list's device form into host memory
 * (gear_grad_list_bytes(count) bytes) and the caller copies that to the device (16-byte aligned) and keeps it as long as
 * the tensors live where they are.  chunks (out): pieces of work in the list, handed to the calls below. */
typedef struct {
  const void *src;
  void *dst;
  int64_t n;
  int32_t dtype;         /* GEAR_F32 or GEAR_BF16, of both */
} gear_grad_tensor;
size_t gear_grad_list_bytes(int32_t count);
gear_status gear_grad_list_pack(const gear_grad_tensor *tensors, int32_t count, void *host_list, int64_t *chunks);
/* norm (device, fp32 [1]) = sqrt(sum of all squares); squares and their sum in fp64, so nothing overflows or vanishes on
 * the way.  workspace: gear_grad_workspace_bytes(chunks) bytes, 256-byte aligned. */
size_t gear_grad_workspace_bytes(int64_t chunks);
gear_status gear_grad_norm(const void *list, int32_t count, int64_t chunks, void *workspace, size_t workspace_bytes,
                           float *norm, void *stream);
/* The same, and dst = c src for every tensor with c = min(1, max_norm / (norm + 1e-6)), max_norm > 0, from the norm in fp64:
 * gradients that are finite are scaled by it also where fp32 can only report an infinite norm.  An infinity among the gradients makes
 * c 0, a NaN makes c NaN. */
gear_status gear_clip_grads(const void *list, int32_t count, int64_t chunks, float max_norm, void *workspace,
                            size_t workspace_bytes, float *norm, void *stream);

/* ---- Rows that choose their experts ------------------------------------------------------------------------------
 * A Dense Part whose rows go to experts by learned scores: the choice and its gradient, the rows' way to their experts and
 * back and its gradients (Section 3, step 6), for the products above.  The rules of that section hold (widths, distances between rows,
 * alignment); only logits may have any width, distance and alignment of their elements.
 *
 * Scores of a row are the softmax or the sigmoid of its logits.  An expert is eligible where its logit is not -inf and its bias
 * neither -inf nor NaN; a row with a NaN logit (softmax: or +inf) has no eligible expert and NaN for all its weights.  Experts are ordered
 * by score + bias in fp64, without a bias by logit, ties by the lowest number.  Experts may come in groups of equal size, one
 * group's behind the other's: a group's value is the largest score + bias in it, or the sum of the two largest (of as many as
 * are eligible), and only experts of the groups_kept groups of the largest values (ties by the lowest number) can be chosen.  The k first are chosen; a slot for which
 * no eligible expert is left holds expert -1 and weighs 0.  The weight of an expert is its score, without the bias, divided by
 * the sum of the chosen ones' if `renormalise`, times scale.
 *
 * Pairs (row, slot) that have an expert are lined up by expert, then row, then slot: place is where, off [experts + 1] where every
 * expert's begin, as gear_expert_product takes it; place is -1 for a slot without an expert. */
#define GEAR_SCORE_SOFTMAX 0
#define GEAR_SCORE_SIGMOID 1
#define GEAR_MAX_CHOSEN 32
#define GEAR_MAX_GROUPS 64

/* rows * k is at most 2^30.  n (device word, may be NULL): rows from *n on are padding, whatever they hold, and have no expert.  off and place may
 * both be NULL where only the choice is wanted; the workspace (256-byte aligned, gear_route_workspace_bytes) is not needed then.
 * scale > 0.  No rows: off is all zeros. */
typedef struct {
  int64_t rows;
  int32_t experts, k, dtype;              /* gear_dtype of the logits */
  int32_t score, groups, groups_kept, group_best;   /* group_best: 1 the largest, 2 the sum of two; groups = 1: no groups */
  int32_t renormalise;
  float scale;
  const void *logits;                     /* [rows x experts] */
  int64_t ld_logits;
  const float *bias;                      /* [experts], may be NULL */
  const int32_t *n;
  int32_t *expert;                        /* [rows x k], best first */
  float *weight;                          /* [rows x k] */
  int32_t *off, *place;                   /* [experts + 1], [rows x k] */
} gear_route_args;
size_t gear_route_workspace_bytes(int64_t rows, int32_t experts, int32_t k, int32_t groups);
gear_status gear_route(const gear_route_args *a, void *workspace, size_t workspace_bytes, void *stream);

/* Gradient of the weights with respect to the logits, the choice held fixed: dlogits [rows x experts] of the logits' type, every
 * element written.  expert and weight are what gear_route left; experts of a row are distinct.  dweight is not read as a number where a slot has no
 * expert; rows without any expert have zeros, rows whose weights hold a NaN have NaN.  dlogits may not be logits. */
typedef struct {
  int64_t rows;
  int32_t experts, k, dtype;
  int32_t score, renormalise;
  float scale;
  const void *logits;
  int64_t ld_logits;
  const int32_t *expert;
  const float *weight, *dweight;          /* [rows x k] */
  void *dlogits;
  int64_t ld_dlogits;
} gear_route_backward_args;
gear_status gear_route_backward(const gear_route_backward_args *a, void *stream);

/* Rows to their experts: xs[place[r, j]] = x[r], a copy for every slot that has a place.  xs [rows * k x dim] of x's type shares no memory with x or place.  Rows of xs that
 * are nobody's place (from off[experts] on) are left as they were.  Places outside [0, rows * k) are taken for none, here and below;
 * places other than gear_route's have to be distinct.  rows * k is at most 2^30. */
gear_status gear_expert_gather(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t dim, const int32_t *place, int32_t k,
                               void *xs, int64_t ld_xs, void *stream);

/* Back again: out[r] = residual[r] + sum over j of weight[r, j] y[place[r, j]], added up in fp32 in the order of the slots.  residual may
 * be NULL (nothing), weight may be NULL (1 each: the gradient of gear_expert_gather, y being that of xs and residual what flows
 * into x itself).  A slot without a place counts as a row of zeros: a NaN weight makes the row NaN, other weights nothing.
 * out may be residual itself, but shares no memory with y, place or weight.  y may be fp32 where residual and out are bf16: products that come in fp32 (the out_dtype of
 * gear_expert_product and gear_product_i8) are then rounded once, as a part of the sum, and not each by itself before it. */
typedef struct {
  int64_t rows;
  int32_t dim, k, dtype;                  /* gear_dtype of residual and out, and of y unless y_f32 */
  int32_t y_f32;                          /* y is fp32, whatever dtype is */
  const void *y, *residual;
  const int32_t *place;
  const float *weight;
  void *out;
  int64_t ld_y, ld_residual, ld_out;
} gear_expert_combine_args;
gear_status gear_expert_combine(const gear_expert_combine_args *a, void *stream);

/* Its gradients: dy[place[r, j]] = weight[r, j] dout[r] (rows that are nobody's place are left as they were; dy may be y itself, or NULL,
 * and shares no memory with dout, place, weight or dweight), dweight[r, j] = dout[r] . y[place[r, j]] in fp32, 0 for a slot without a place (may be NULL).
 * The residual's gradient is dout. */
typedef struct {
  int64_t rows;
  int32_t dim, k, dtype;                  /* gear_dtype of dout, y and dy, also where the sum took y in fp32 */
  const void *dout, *y;
  const int32_t *place;
  const float *weight;
  void *dy;
  float *dweight;
  int64_t ld_dout, ld_y, ld_dy;
} gear_expert_combine_backward_args;
gear_status gear_expert_combine_backward(const gear_expert_combine_backward_args *a, void *stream);

/* ---- Products in 8-bit integers ---------------------------------------------------------------------------------------
 * A row of `dim` values v as integers q with one scale: scale = max|v| / 127 (fp32), q the integer nearest to 127 v / max|v|, ties to
 * even, so q scale stands for v.  A row of zeros has scale 0; a row that holds an infinity or a NaN has integers 0 and scale
 * NaN, and so has everything made from it.  The same for weights, a scale for every output's [K] weights.  Sums are exact (32-bit integers: K is
 * at most 65536), so a product is off by its operands' rounding to 8 bits and three roundings of fp32.  Rows take gear_rows8_ld(dim) bytes, zeros behind
 * their end. */

/* x [rows x dim] in 8-bit integers.  place NULL (k then 1): row r of q and scale is x[r].  Otherwise x[r] goes to row place[r, j] for every
 * slot that has a place, as gear_expert_gather does it; q and scale have rows * k rows then.  They share no memory with x, place or each other. */
gear_status gear_rows_i8(const void *x, int32_t dtype, int64_t ld_x, int64_t rows, int32_t dim, const int32_t *place, int32_t k, int8_t *q,
                         float *scale, void *stream);

/* Weights for gear_product_i8: w [experts x N x K] contiguous, GEAR_F32 or GEAR_BF16, made into integers with a scale for every output (scale
 * [experts x N] is written), or GEAR_I8, integers already (scale is the caller's and not touched; -128 is allowed).  packed: gear_packed_i8_bytes,
 * 16-byte aligned (0 bytes on a bad argument); scale 16-byte aligned. */
#define GEAR_I8 3                         /* beside gear_dtype, for these weights alone */
size_t gear_packed_i8_bytes(int32_t experts, int32_t N, int32_t K);
gear_status gear_pack_weights_i8(const void *w, int32_t src_dtype, int32_t experts, int32_t N, int32_t K, int8_t *packed, float *scale, void *stream);

/* out[r, n] = x_scale[r] w_scale[e, n] sum over k of x[r, k] w_e[n, k] for the rows of every expert: off, status, keep_status and out as for
 * gear_expert_product; x rows of ld_x bytes, at least gear_rows8_ld(K) and a multiple of 16.  out shares no memory with what is read. */
typedef struct {
  int32_t out_dtype;
  int64_t rows;
  int32_t K, N, experts;
  const int8_t *x;
  const float *x_scale;                   /* [rows] */
  const int8_t *packed;
  const float *w_scale;                   /* [experts x N], 16-byte aligned */
  const int32_t *off;
  void *out;
  int64_t ld_x, ld_out;
  int32_t *status;
  int32_t keep_status;
} gear_i8_args;
gear_status gear_product_i8(const gear_i8_args *a, void *stream);

/* Per-kernel timing of a step, for benchmarks.  gear_profile_create allocates a fixed pool of HIP
 * events on the current device (host memory; NULL on failure), gear_profile_destroy releases it.
 * After a gear_step that was given the profile and after the stream has been synchronised,
 * gear_profile_count returns the number of timed launches and gear_profile_span the name of
 * launch i (a static string) and its duration in milliseconds. */
typedef struct gear_profile gear_profile;
gear_profile *gear_profile_create(void);
void gear_profile_destroy(gear_profile *p);
int32_t gear_profile_count(const gear_profile *p);
gear_status gear_profile_span(const gear_profile *p, int32_t i, const char **name, float *ms);

/* Test hooks for the error paths of a step (no device needs to fail for them to be walked).
 * gear_debug_fail_launch(n): on the calling thread, the n-th launch of a step counted from now (n >= 1, as
 * a profile counts them) is not enqueued and the step returns GEAR_ERR_HIP there, leaving caller state
 * half-updated as any failed launch would; 0 switches it off.  gear_debug_helper_idle(): 1 if the current device's helper
 * stream has nothing left to run (or was never created), 0 if it is still busy, -1 on a HIP error. */
void gear_debug_fail_launch(int32_t nth);
int32_t gear_debug_helper_idle(void);

const char *gear_status_string(gear_status s);

#ifdef __cplusplus
}
#endif
#endif /* GEAR_H */
