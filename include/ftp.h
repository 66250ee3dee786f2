/*
 * ftp.h — C ABI of the MI355X stage-training library.
 *
 * One pipeline stage's training step of FTPipeHD: a worker builds the sub-model
 * given by its partition points (paper, section "Initialization"), forwards and
 * backwards batches under the one-forward-one-backward rule with weight
 * stashing (section "Async Pipeline Training"), updates its weights with SGD,
 * momentum and weight decay (section "Experiment Setup"), and the central node
 * profiles per-layer execution time and output size (section "Initialization",
 * model profiling phase) and solves the partition dynamic programme (section
 * "Dynamic Model Partition").
 *
 * Conventions
 *   - Every function returns 0 (FTP_OK) or a negative ftp_status; on error the
 *     outputs are untouched and ftp_last_error() holds a thread-local message.
 *     No C++ exception and no abort crosses this boundary.
 *   - "dev" pointers are device (HBM) addresses, "host" pointers are host
 *     addresses.  `stream` is a hipStream_t passed as void* (NULL = default
 *     stream).  Compute calls are asynchronous on that stream; import / export /
 *     profile / solve are synchronous.
 *   - The compute calls of one stage share its workspace: issue them in program
 *     order on one stream (or on streams the caller has ordered with events).
 *     A large stage runs its weight gradients on a stream of its own inside
 *     ftp_stage_backward; that work is ordered before anything enqueued on the
 *     caller's stream after the call.  Different stages are independent.
 *   - Activations are NHWC (channels fastest): [batch, H, W, C]; a 1-D window of
 *     T steps is H = 1, W = T.  Their element type is the model's ftp_dtype
 *     (float, or bfloat16 with fp32 accumulation, statistics, gradients of
 *     weights, momentum and master weights).
 *   - The caller owns x / y / dy / dx / labels / loss buffers.  The stage owns
 *     everything that lives between calls (weights, momentum, gradients, BN
 *     running statistics, per-slot stash, workspace) and frees it in
 *     ftp_stage_destroy.
 *   - A partition unit ("layer" in the paper) is the smallest piece a stage
 *     boundary may fall between; a residual connection is never cut.
 */
#ifndef FTP_H
#define FTP_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  FTP_OK = 0,
  FTP_ERR_ARG = -1,         /* NULL pointer, bad range, bad size              */
  FTP_ERR_SHAPE = -2,       /* unit list does not chain / count mismatch      */
  FTP_ERR_UNSUPPORTED = -3, /* valid request the kernels do not cover         */
  FTP_ERR_SLOT = -4,        /* slot busy on forward / empty on backward       */
  FTP_ERR_VALUE = -5,       /* NaN, infinite or non-positive cost / capacity  */
  FTP_ERR_HIP = -6,         /* HIP runtime failure (message has the detail)   */
  FTP_ERR_NOMEM = -7
} ftp_status;

typedef enum { FTP_F32 = 0, FTP_BF16 = 1 } ftp_dtype;

typedef enum {
  FTP_UNIT_CONV = 0,   /* conv (kh x kw, stride, zero pad) + BatchNorm + act     */
  FTP_UNIT_INVRES = 1, /* inverted residual: [1x1 expand+BN+ReLU6 if expand>1]
                          -> depthwise 3x3 (stride)+BN+ReLU6 -> 1x1 project+BN;
                          adds its input when stride == 1 and cin == cout        */
  FTP_UNIT_GAP = 2,    /* mean over H and W                                      */
  FTP_UNIT_FC = 3,     /* y = x W^T + b                                          */
  FTP_UNIT_LOSS = 4    /* softmax cross-entropy, mean over the batch             */
} ftp_unit_kind;

/* Units take the first three; the token operators below take all (GELU in its tanh form). */
typedef enum { FTP_ACT_NONE = 0, FTP_ACT_RELU = 1, FTP_ACT_RELU6 = 2, FTP_ACT_SILU = 3, FTP_ACT_GELU = 4 } ftp_act;

typedef struct {
  int32_t kind;          /* ftp_unit_kind                                        */
  int32_t cin, cout;     /* channels in / out (LOSS: cin = cout = classes)       */
  int32_t kh, kw;        /* CONV only                                            */
  int32_t stride;        /* CONV, INVRES                                         */
  int32_t pad_h, pad_w;  /* CONV only                                            */
  int32_t expand;        /* INVRES only: expansion factor t                      */
  int32_t act;           /* CONV only: ftp_act after the BatchNorm               */
} ftp_unit_desc;

/* SGD with momonentum and weight decay: g += wd*w; v = momentum*v + g; w -= lr*v. */
typedef struct { float lr, momentum, weight_decay; } ftp_sgd;

typedef struct ftp_model ftp_model; /* immutable unit list of the whole network  */
typedef struct ftp_stage ftp_stage; /* units [a,b) at one batch size, on one GPU */

const char* ftp_last_error(void);

/* ---- model description ---------------------------------------------------- */

/* The network every worker partitions (section "Initialization": the central node sends the model and the initial
 * partition points; a worker builds its sub-model from layer start_i to layer end_i).  Copies `units` (host, L
 * entries).  in_h/in_w/in_c: shape of the network input.  Channel counts that feed a BatchNorm must be multiples
 * of 8. */
int ftp_model_create(const ftp_unit_desc* units, int L, int in_h, int in_w, int in_c,
                     ftp_dtype act_dtype, ftp_model** out);
void ftp_model_destroy(ftp_model*);
int ftp_model_num_units(const ftp_model*);
/* Shape (H, W, C) of the tensor entering unit `u` (u == L: leaving the last). */
int ftp_model_unit_in_shape(const ftp_model*, int u, int* h, int* w, int* c);
/* Number of fp32 parameters of unit u.  Layout of a unit's parameter vector:
 *   CONV   : w[cout][kh][kw][cin], gamma[cout], beta[cout]
 *   INVRES : (expand > 1: w1[ce][cin], gamma1[ce], beta1[ce],)
 *            wd[ce][3][3], gamma2[ce], beta2[ce], w3[cout][ce], gamma3[cout], beta3[cout]
 *            with ce = cin * expand
 *   FC     : w[cout][cin], b[cout]
 *   GAP, LOSS : none */
int ftp_model_unit_param_count(const ftp_model*, int u, size_t* n);
/* Number of BatchNorm channels of unit u, summed over its BatchNorms in order. */
int ftp_model_unit_bn_channels(const ftp_model*, int u, size_t* n);

/* ---- stage ------------------------------------------------------------------ */

/* The sub-model of one worker (section "Initialization": layers start_i .. end_i of the partition points; section
 * "Async Pipeline Training": stage i of n keeps n-i batches in flight, hence the slots).
 * Builds units [a,b) for `batch` samples with `n_slots` in-flight batches on the
 * current HIP device; allocates all device memory it will ever need.  Weights
 * start at zero (import them), momentum and gradients at zero, BN running mean
 * 0 / variance 1. */
int ftp_stage_create(const ftp_model*, int a, int b, int batch, int n_slots, ftp_stage** out);
/* The same with options.  FTP_STAGE_RECOMPUTE: a slot keeps only the stage input of its batch (and, after
 * ftp_stage_snapshot_weights, its weight version); the intermediates of the batch forwarded last live in one
 * stash that all slots share, and the backward of any other slot first runs the forward again from the kept
 * input with that slot's weights (paper, section "Synchronous Pipeline Parallelism Training": intermediates
 * are thrown away and re-computed when the gradient arrives).  The second forward leaves the BatchNorm running
 * statistics alone, and the kernels being deterministic, a run gives bit for bit the weights of a stage
 * that keeps everything.  Memory: one stash + n_slots inputs instead of n_slots stashes.  With this option
 * ftp_stage_loss(slot) must follow ftp_stage_forward(slot) before any other forward (the logits are not kept),
 * and ftp_stage_export_conv_output sees only the slot forwarded or recomputed last.
 * Unknown flag bits: FTP_ERR_ARG. */
enum { FTP_STAGE_RECOMPUTE = 1 };
int ftp_stage_create_ex(const ftp_model*, int a, int b, int batch, int n_slots, unsigned flags, ftp_stage** out);
void ftp_stage_destroy(ftp_stage*);
/* Device memory, in bytes, that the stage allocated at creation (host pointer out). */
int ftp_stage_device_bytes(const ftp_stage*, size_t* bytes);

/* Weights travel between workers and the central node as per-layer vectors (sections "Weight Replication" and
 * "Fault Tolerance Mechanism": a worker fetches the layers it lacks; here the host side of that exchange).
 * Host <-> device copies of one unit's parameter vector (layout above), its
 * accumulated gradient, its momentum buffer, and its BN running statistics
 * (running_mean then running_var of each BatchNorm in order; 2 * bn_channels). */
int ftp_stage_import_weights(ftp_stage*, int unit, const float* host_w, size_t n);
int ftp_stage_export_weights(const ftp_stage*, int unit, float* host_w, size_t n);
int ftp_stage_export_grads(const ftp_stage*, int unit, float* host_g, size_t n);
int ftp_stage_export_momentum(const ftp_stage*, int unit, float* host_v, size_t n);
int ftp_stage_export_bn_stats(const ftp_stage*, int unit, float* host_s, size_t n);

/* Inspection of a busy slot (between its forward and its backward): the raw
 * output z of convolution number `conv` of `unit` (0-based within the unit, in
 * execution order) converted to float, n = batch*Hout*Wout*Cout values in NHWC
 * order; and that convolution's BatchNorm batch statistics as 4*Cout floats:
 * mean, 1/sqrt(var+eps), scale = gamma/sqrt(var+eps), shift = beta - mean*scale.
 * The value the next layer consumes is act(scale*z + shift).  Synchronous. */
int ftp_stage_export_conv_output(const ftp_stage*, int slot, int unit, int conv, float* host_z, size_t n);
int ftp_stage_export_bn_batch_stats(const ftp_stage*, int slot, int unit, int conv, float* host_s, size_t n);

/* Section "Async Pipeline Training": a worker forwards a batch through its sub-model with its newest weights and
 * passes the result on.  Forward of one batch through units [a,b) with the current weights.
 * x_dev: [batch, H, W, C] of unit a's input, read only, copied into the slot
 * (the stashed stage input).  y_dev: output of the last unit, or NULL; when the
 * stage ends with the LOSS unit, y receives the logits [batch, classes].
 * The slot must be free; it is busy until its backward. */
int ftp_stage_forward(ftp_stage*, int slot, const void* x_dev, void* y_dev, void* stream);

/* Section "Async Pipeline Training": the last stage computes the loss of a batch and starts its backward pass.
 * Stages that end with the LOSS unit: mean cross-entropy of the slot's logits
 * against labels_dev (int32 [batch], 0 <= label < classes) into loss_dev (one
 * float); also seeds the slot's backward so dy_dev may be NULL there. */
int ftp_stage_loss(ftp_stage*, int slot, const int32_t* labels_dev, float* loss_dev, void* stream);

/* The loss of ftp_stage_loss for callers that cannot allocate device memory and have no stage object at hand: code
 * under HIP graph capture, tight serving or evaluation loops, harnesses that forbid hipMalloc.  Same kernels, same
 * results bit for bit; the per-row losses that ftp_stage_loss keeps in memory the stage allocated live in a
 * file-scope device array of FTP_STATIC_LOSS_MAX_BATCH floats (256 KiB per GPU, held until the process ends), next to
 * the counters by which the last block to arrive takes their mean.
 * logits_dev [batch, classes] and dlogits_dev (same shape, receives (softmax - onehot) / batch) are of `dtype`;
 * labels_dev int32 [batch], 0 <= label < classes (a label outside gives a NaN loss); loss_dev one float.  The caller
 * owns all four buffers.  batch > FTP_STATIC_LOSS_MAX_BATCH: FTP_ERR_ARG, nothing is launched.  Calls no hipMalloc,
 * hipFree or other allocating routine (the first call on a device looks up that device's address of the array);
 * nothing in the array has to be cleared between calls.  All calls on one GPU share the array: calls that may run
 * concurrently there (different streams without an ordering) race on it.  Asynchronous on `stream`. */
#define FTP_STATIC_LOSS_MAX_BATCH 65536
int ftp_softmax_ce_static(const void* logits_dev, const int32_t* labels_dev, int batch, int classes, ftp_dtype dtype,
                          void* dlogits_dev, float* loss_dev, void* stream);

/* Section "Async Pipeline Training" (weight stashing: the backward of a batch uses the weight version its forward
 * used).  Copies the current weights into the slot (weight stashing): the slot's
 * backward then differentiates with respect to that version.  Call it between
 * the slot's forward and the next update.  Without it, backward uses the
 * weights current at that time. */
int ftp_stage_snapshot_weights(ftp_stage*, int slot, void* stream);

/* Weight aggregation (section "Async Pipeline Training": stage i of n has n-i weight
 * versions in use at once and merges them at an interval that is a multiple of
 * n-i).  The live weights become the arithmetic mean, element by element in fp32
 * (summed in the order given, then divided by n), of the versions stashed by
 * ftp_stage_snapshot_weights() in slots[0..n); the bfloat16 working copy is
 * re-derived; momentum, gradients and the snapshots themselves are not touched.
 * `slots` is a host array, 1 <= n <= 8, every listed slot must hold a snapshot
 * (FTP_ERR_SLOT otherwise), a slot may not be listed twice.  Asynchronous on
 * `stream`.  When to call it is the caller's schedule: the paper's example merges
 * the versions of the n-i batches in flight right after the forward that follows
 * every (n-i)-th backward. */
int ftp_stage_aggregate_weights(ftp_stage*, const int* slots, int n, void* stream);

/* Section "Async Pipeline Training": the backward pass of a batch through the sub-model, with the stashed weight
 * version.  Backward of the slot's batch.  dy_dev: gradient of the stage output (same
 * shape and type as y), or NULL after ftp_stage_loss.  dx_dev: receives the
 * gradient of the stage input, or NULL (e.g. a == 0).  Weight gradients are
 * ACCUMULATED into the stage's gradient buffers.  Frees the slot. */
int ftp_stage_backward(ftp_stage*, int slot, const void* dy_dev, void* dx_dev, void* stream);

/* Section "Experiment Setup" (SGD, momentum 0.9, weight decay 4e-5): g += wd*w; v = momentum*v + g; w -= lr*v.
 * One step on all parameters of the stage from the accumulated gradients, which are then zeroed. */
int ftp_stage_update(ftp_stage*, const ftp_sgd* opt, void* stream);

/* ---- profiling and partition ------------------------------------------------ */

/* Model profiling (section "Initialization", model profiling phase: the central node measures the running time
 * of the forward and backward pass of each layer, averaged over ten executions, and the size of each layer's
 * output).  Runs forward and backward of every unit of the whole model on synthetic data `reps` times (the paper
 * uses 10) after 2 discarded warm-up runs, and returns per unit the mean forward+backward time in nanoseconds
 * rounded to an integer value (t_ns, host, [L]) and the output size in bytes (out_bytes, host, [L]).  The
 * per-unit times are measured unit after unit on one stream and then scaled by one common factor so that their
 * sum is the mean forward+backward time of a whole batch under the execution plan training uses (`reps` more
 * runs): ftp_estimate_capacity of this same device on the whole model is then 1.  Synchronous. */
int ftp_profile_layers(const ftp_model*, int batch, int reps, double* t_ns, int64_t* out_bytes,
                       void* stream);

/* Section "Dynamic Model Partition": the dynamic programme A(j, n) over contiguous splits that minimises the slowest
 * stage (base case: the prefix on device 0; recurrence: the last cut, with the optional transfer term and the
 * last-stage time), every layer's time on worker k being its profiled time times the capacity C_k.
 * layer_costs[L] > 0: execution time of each unit
 * on the profiling device; device_capacities[N] > 0: TIME MULTIPLIERS (the
 * paper's computing capacity C_k = worker time / central-node time, so larger =
 * slower; stage k on device k costs C_k * sum of its costs).  Optional
 * out_bytes[L] and bandwidth[N-1] (both non-NULL) add the transfer term
 * 2 * out_bytes[l-1] / bandwidth[k-1] for the cut in front of stage k.
 * bounds[N+1] receives bounds[0] = 0 < ... < bounds[N] = L, stage k = units
 * [bounds[k], bounds[k+1]); *bottleneck (may be NULL) the minimised slowest
 * time.  Every stage is non-empty (N <= L).  Ties: smallest last cut.
 * All host pointers; float64 arithmetic, bit-reproducible. */
int ftp_solve_partition(const double* layer_costs, int L, const double* device_capacities, int N,
                        const double* out_bytes, const double* bandwidth, int32_t* bounds,
                        double* bottleneck);

/* Section "Dynamic Model Partition", capacity equation: a worker's measured stage time divided by the
 * profiling device's time for the same units [start, end] (inclusive). */
int ftp_estimate_capacity(double stage_time, const double* layer_costs, int L, int start, int end,
                          double* capacity);

/* Re-partition schedule (section "Dynamic Model Partition"): *due = 1 when a re-partition follows the
 * batches_done-th trained batch: the first after 10 batches, then every 100 (10, 110, 210, ...). */
int ftp_repartition_due(int64_t batches_done, int* due);

/* Capacities for the next re-partition (capacity equations of the same section).  mean_times[n]: the mean
 * execution time each worker reported for its current stage [bounds_cur[i], bounds_cur[i+1]) in the unit of
 * layer_costs[L]; a value that is not finite and positive means "no report".  capacities[0] = 1.0 (the central
 * node, whose report is not used); capacities[i] = mean_times[i] / sum of layer_costs over worker i's stage; if
 * any worker i >= 1 has no report every capacity is 1.0 (the re-partition then uses the central node's times
 * alone).  All host pointers. */
int ftp_repartition_capacities(const double* mean_times, const double* layer_costs, int L, const int32_t* bounds_cur,
                               int n, double* capacities);

/* Online execution profiling (section "Dynamic Model Partition", execution
 * profiling phase: every worker records the execution time of every batch and
 * reports the average, which becomes the numerator of its capacity).
 * ftp_stage_timing(stage, 1) starts recording, per forwarded batch, the time of
 * its forward plus its backward on the streams they were enqueued on (HIP
 * events; up to 256 batches between reads, later ones are not recorded);
 * ftp_stage_timing(stage, 0) stops and discards.  Switch only while no batch is
 * in flight.  ftp_stage_timing_read waits for the recorded batches, returns their
 * number and the mean forward+backward time in nanoseconds (0 if none), and
 * starts a new window; batches in flight at that moment are left out.  Feed the
 * mean to ftp_estimate_capacity together with the profiled costs of the stage's
 * units.  Off by default: a step then records no events at all. */
int ftp_stage_timing(ftp_stage*, int enable);
int ftp_stage_timing_read(ftp_stage*, double* mean_ns, int* n_batches);

/* Weight redistribution after a re-partition or a single worker failure (the
 * paper's Algorithm "Weight Redistribution", sections "Dynamic Model Partition"
 * and "Fault Tolerance Mechanism"), for the worker that holds stage i_cur of
 * bounds_cur[n_cur+1] and will hold stage i_new of bounds_new[n_new+1] (half-open
 * unit bounds as returned by ftp_solve_partition, same total).  i_fail: index in
 * the CURRENT numbering of the failed worker, or -1 for a plain re-partition.
 * source[j], j = 0 .. bounds_new[i_new+1]-bounds_new[i_new]-1, receives for unit
 * bounds_new[i_new]+j either -1 (the worker holds it already) or the index, in
 * the NEW numbering, of the worker to fetch it from: the current holder, moved
 * up by one if it sat behind the failed worker; the failed worker's chain
 * successor (which now carries the failed index) for a unit of the failed stage;
 * worker 0 (the central node) if the failed stage was the last one.  Host
 * pointers only; no device work. */
int ftp_redistribution_plan(const int32_t* bounds_new, int n_new, const int32_t* bounds_cur, int n_cur, int i_fail,
                            int i_cur, int i_new, int32_t* source);

/* Worker list after failures (section "Fault Tolerance Mechanism": with one failed worker every index greater
 * than its index decreases by one and the smaller ones stay; with several, each failed worker is replaced by the
 * alive workers that follow it, one by one).  worker_ids[n]: the current list (device ids in training order,
 * entry 0 the central node); failed[n_failed]: indices into it, each in 1..n-1 (the central node runs the fault
 * handler and cannot be listed), no index twice.  new_ids (room for n entries) receives the alive entries in
 * their old order and *n_new their number; new_index (n entries, may be NULL) receives for every old index its
 * new index, or -1 for a failed worker.  The index a failed worker had is thereby carried by the alive worker
 * that followed it, which is what ftp_redistribution_plan's `source` refers to.  Host pointers only. */
int ftp_renumber_workers(const int32_t* worker_ids, int n, const int32_t* failed, int n_failed, int32_t* new_ids,
                         int32_t* new_index, int* n_new);

/* Device-side half of the redistribution: copies weights, momentum and BatchNorm
 * running statistics of units [unit_lo, unit_hi) from `src` to `dst` (both
 * stages must contain the range and be built from the same model and type),
 * device to device on `stream`, and refreshes dst's bfloat16 working copy of
 * them.  Pending gradients are not copied. */
int ftp_stage_copy_units(ftp_stage* dst, const ftp_stage* src, int unit_lo, int unit_hi, void* stream);

/* ---- token operators --------------------------------------------------------------- */

/* What a stage of a token model is made of, on buffers the caller owns: the table lookup of the first stage, linear
 * layers, gated feed-forward blocks, and the 8-bit form in which a stage can hold the activations of its batches in
 * flight (section "Async Pipeline Training": stage i of n keeps n-i of them).  A call takes a record of sizes, pointers
 * and options (zero it first: a NULL pointer or 0 is "not wanted"); the caller keeps it for as long as its buffers live.
 *   - Matrices are row-major; ld... is the distance between rows in elements (bytes for 8-bit forms), at least the
 *     row's length, at most 2^20.  Pointers are aligned to their elements; sizes, strides and offsets are otherwise
 *     free, but an operand whose rows do not start on 4 bytes, or are not a multiple of 16 bytes long, is first copied into ws.
 *   - `rows` counts tokens, 0 .. 2^30; with 0 a forward does nothing and a backward writes zero gradients
 *     (accumulate: leaves them).
 *   - `dtype` is the type of activations, their gradients and the weights.  Sums, activations and scales are fp32;
 *     what is stored between two products (hidden, its gradients) is rounded to dtype once, as their operands.
 *   - Weight gradients are [out][in] one row behind the other, fp32 or of dtype (grad_dtype), overwritten, or with
 *     `accumulate` (fp32 only) added to.
 *   - ws: device memory of at least the bytes the ..._workspace function names for the same record and direction (it
 *     goes by sizes, strides and the pointers' alignment), on 16 bytes; contents are free between calls; calls that may
 *     overlap need one each.  Nothing is allocated, everything is enqueued on `stream`, calls can be captured into a
 *     graph.  Results do not depend on what else runs: the same inputs give the same bits.
 *   - Outputs may not overlap inputs, except that y may be the residual's buffer. */

/* out[t] = scale * table[ids[t]]; an id that is none of 0 .. vocab-1 gives a row of NaN.
 * Gradient: dtable[v] = scale * (sum of dy[t] over the tokens t with ids[t] = v), fp32, all vocab rows written, or with
 * `accumulate` added to the rows that came up.  Tokens whose id is pad_id (-1: none) or not the table's add nothing.
 * Sorted by id, each id's tokens added in their order. */
typedef struct {
  int64_t rows;
  int32_t vocab, width;
  int32_t dtype;          /* ftp_dtype of table, out, dy                            */
  int32_t ids64;          /* ids are int64 (otherwise int32)                        */
  int32_t accumulate;
  float scale;            /* finite                                                 */
  int64_t pad_id;
  const void* ids;
  const void* table; int64_t ldt;
  void* out; int64_t ldo;
  const void* dy; int64_t lddy;
  float* dtable; int64_t lddt;
  void* ws; size_t ws_bytes;
} ftp_embed_args;
int ftp_embed_forward(const ftp_embed_args*, void* stream);
int ftp_embed_backward_workspace(const ftp_embed_args*, size_t* bytes);
int ftp_embed_backward(const ftp_embed_args*, void* stream);

/* Forward: y = act(z) + residual, z = x w^T + bias; x [rows][n_in], w [n_out][n_in], bias fp32 [n_out] or NULL, residual
 * or NULL; z is written where it is wanted (the backward of an activation needs it).
 * Backward: dz = dy * act'(z); dx = dz w, dw = dz^T x, dbias = sum of dz over the rows; each where wanted.  Derivatives of
 * ReLU and ReLU6 are 1 strictly inside.  (dy is also the residual's gradient.)
 * x_scales: x is held in 8 bits (ftp_act8_pack), its scales ldxs apart. */
typedef struct {
  int64_t rows;
  int32_t n_in, n_out;
  int32_t dtype, act;
  int32_t grad_dtype, accumulate;
  const void* x; int64_t ldx;
  const uint8_t* x_scales; int64_t ldxs;
  const void* w; int64_t ldw;
  const float* bias;
  const void* residual; int64_t ldr;
  void* y; int64_t ldy;
  void* z; int64_t ldz;
  const void* dy; int64_t lddy;
  void* dx; int64_t lddx;
  void* dw;
  void* dbias;
  void* ws; size_t ws_bytes;
} ftp_linear_args;
int ftp_linear_workspace(const ftp_linear_args*, int backward, size_t* bytes);
int ftp_linear_forward(const ftp_linear_args*, void* stream);
int ftp_linear_backward(const ftp_linear_args*, void* stream);

/* Gated feed-forward block: gate = x w_gate^T, up = x w_up^T, hidden = act(gate) * up, y = hidden w_down^T + residual;
 * w_gate, w_up [hidden][width], w_down [width][hidden].  The hidden rows are the workspace's.
 * save: FTP_SAVE_FULL keeps gate and up in dtype, [rows][hidden]; FTP_SAVE_ACT8 in 8 bits with gate_scales, up_scales
 * [rows][ceil(hidden / 32)], formed from the fp32 sums: 33/64 of the bytes a bfloat16 stash takes.
 * Backward, from what was kept: dhidden = dy w_down; dgate = dhidden * up * act'(gate); dup = dhidden * act(gate);
 * dx = dgate w_gate + dup w_up (+ dy with dx_residual: the block's residual was x); dw_gate = dgate^T x, dw_up = dup^T x,
 * dw_down = dy^T hidden, the three together or none.  x_scales as above. */
typedef enum { FTP_SAVE_NONE = 0, FTP_SAVE_FULL = 1, FTP_SAVE_ACT8 = 2 } ftp_save;
typedef struct {
  int64_t rows;
  int32_t width, hidden;
  int32_t dtype, act;
  int32_t save;           /* ftp_save                                               */
  int32_t grad_dtype, accumulate, dx_residual;
  const void* x; int64_t ldx;
  const uint8_t* x_scales; int64_t ldxs;
  const void* w_gate; int64_t ldwg;
  const void* w_up; int64_t ldwu;
  const void* w_down; int64_t ldwd;
  const void* residual; int64_t ldr;
  void* y; int64_t ldy;
  void *gate, *up;
  uint8_t *gate_scales, *up_scales;
  const void* dy; int64_t lddy;
  void* dx; int64_t lddx;
  void *dw_gate, *dw_up, *dw_down;
  void* ws; size_t ws_bytes;
} ftp_ffn_args;
int ftp_ffn_workspace(const ftp_ffn_args*, int backward, size_t* bytes);
int ftp_ffn_forward(const ftp_ffn_args*, void* stream);
int ftp_ffn_backward(const ftp_ffn_args*, void* stream);

/* Activations in 8 bits: groups of 32 columns share a scale 2^(s-127), the smallest (s >= 0) with which the group's
 * largest finite magnitude is at most 448; q holds value / scale as e4m3 (4 exponent bits, 3 mantissa bits, no infinity),
 * to nearest even.  Infinities and NaN become NaN.  q [rows][ldq], scales [rows][lds], lds >= ceil(cols / 32).
 * pack: x -> q, scales.  unpack: q, scales -> y. */
typedef struct {
  int64_t rows;
  int32_t cols, dtype;
  const void* x; int64_t ldx;
  uint8_t* q; int64_t ldq;
  uint8_t* scales; int64_t lds;
  void* y; int64_t ldy;
} ftp_act8_args;
int ftp_act8_pack(const ftp_act8_args*, void* stream);
int ftp_act8_unpack(const ftp_act8_args*, void* stream);

/* What stands between the products: dropout, the join of a block's output with the stream and the norms around it, a gated linear
 * recurrence along the sequences, log probabilities of tokens.  Rows, types, strides, workspaces and results as above; no stride
 * has to be aligned and nothing is copied.  Where a result may lie in an operand's buffer it has that operand's row distance.  `seed`, `seed_dev`, `site`, `row0`, `p` name a mask wherever there is one. */

/* A mask of dropout is never stored: it is made again wherever it is needed, by the counter-based generator Philox4x32-10 (Salmon,
 * Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3; 2011).  Columns 8 j .. 8 j + 7 of a row have the counter (j, site,
 * low and high word of row0 + row) under the key seed + *seed_dev (modulo 2^64, low word first; seed_dev NULL: seed); column
 * 8 j + i has 16 bits of word i / 2, the low ones where i is even.  Values whose bits are below q = round(65536 p) become 0 (also infinities
 * and NaN), others are multiplied by 65536 / (65536 - q).  So a mask goes by seed, site and row number alone: a call on some of the rows, a
 * backward and a recomputation have the same one, and a captured call gets a new one with what is written at seed_dev.
 * p: 0 <= p, q < 65536 (0: nothing is dropped).
 * Forward: y = dropped x + residual.  Backward: dx = dropped dy.  y may be the buffer of x or of the residual, dx that of dy. */
typedef struct {
  int64_t rows;
  int32_t cols, dtype;
  float p;
  uint32_t site;
  uint64_t seed;
  const uint64_t* seed_dev;
  int64_t row0;           /* number of the first row, >= 0                          */
  const void* x; int64_t ldx;
  const void* residual; int64_t ldr;
  void* y; int64_t ldy;
  const void* dy; int64_t lddy;
  void* dx; int64_t lddx;
} ftp_dropout_args;
int ftp_dropout_forward(const ftp_dropout_args*, void* stream);
int ftp_dropout_backward(const ftp_dropout_args*, void* stream);

/* Between two blocks of a model: with the stream x, the block's output b and norm(v) = (v - mean) / sqrt(var + eps) of a row
 * (FTP_NORM_LAYER) or v / sqrt(mean of squares + eps) (FTP_NORM_RMS),
 *   c = norm(b) * post_w + post_bias (with `post`; otherwise b),   y = x + scale * gate * dropped c,   n = norm(y) * pre_w + pre_bias.
 * Means and means of squares are fp32: a row whose squares add up to more than its range has the norm 0.
 * x NULL: 0; b NULL: y = x (and n is x normed: the call in front of the first block).  Weights fp32 [width], NULL: 1; biases NULL: 0.
 * gate [ceil(rows / gate_rows)][width] of gate_dtype (fp32 or dtype): row t takes row t / gate_rows; NULL: 1.
 * y and n each where wanted; n is of y before it is rounded.  y may be the buffer of x or of b.
 * Backward, from x, b, gate and the weights (statistics and y are computed again): of dy, which arrives at y, and dn, which arrives at n
 * (one of the two may be NULL), dx, db, dgate (of gate_dtype) and the weights' gradients (fp32 [width]), each where wanted; those of pre_w
 * and pre_bias need dn.  `accumulate`: the weights' gradients are added to what is there; `gate_accumulate`: dgate is (fp32 only).
 * dx may be the buffer of dy. */
typedef enum { FTP_NORM_RMS = 0, FTP_NORM_LAYER = 1 } ftp_norm;
typedef struct {
  int64_t rows;
  int32_t width, dtype;
  int32_t norm;           /* ftp_norm                                               */
  int32_t post;
  float eps;              /* > 0, finite                                            */
  float scale;            /* finite                                                 */
  float p;                /* the mask of c, as above                                */
  uint32_t site;
  uint64_t seed;
  const uint64_t* seed_dev;
  int64_t row0;
  const void* x; int64_t ldx;
  const void* b; int64_t ldb;
  const float *post_w, *post_bias;
  const void* gate; int64_t ldg;
  int64_t gate_rows;      /* >= 1 with a gate                                       */
  int32_t gate_dtype, gate_accumulate;
  void* y; int64_t ldy;
  const float *pre_w, *pre_bias;
  void* n; int64_t ldn;
  const void* dy; int64_t lddy;
  const void* dn; int64_t lddn;
  void* dx; int64_t lddx;
  void* db; int64_t lddb;
  void* dgate; int64_t lddg;
  float *dpost_w, *dpost_bias, *dpre_w, *dpre_bias;
  int32_t accumulate;
  void* ws; size_t ws_bytes;
} ftp_join_args;
int ftp_join_forward(const ftp_join_args*, void* stream);
/* The backward's: for each column sum that is asked for a row of fp32 from each block, 8 MiB in all or less up to 8192 columns, and 1 KiB a column past them (1 GiB at 2^20); up to
 * twice that where a gate's groups do not divide the rows evenly.  The forward has none. */
int ftp_join_workspace(const ftp_join_args*, size_t* bytes);
int ftp_join_backward(const ftp_join_args*, void* stream);

/* Gated linear recurrence, column by column along each sequence:
 *   a = sigmoid(f),   h[t] = a[t] h[t-1] + c(a[t]) x[t],   y[t] = h[t] act(g[t])   (g NULL: y = h)
 * with c = 1 (FTP_SCAN_ADD), 1 - a (FTP_SCAN_MIX) or sqrt(1 - a^2) (FTP_SCAN_UNIT).  Sequence s has the rows starts[s] ..
 * starts[s+1] - 1 (int32 [seqs + 1] in device memory, not falling, within 0 .. rows; where they are neither, results are undefined but
 * nothing outside the buffers is touched), or with starts NULL the rows s * length .. of rows = seqs * length.  A sequence may
 * be empty; rows of no sequence stay as they were in every result.  An infinity or NaN stays in its sequence: results of the others are what they
 * are without it.
 * h0: states in front of the sequences, fp32 [seqs], NULL: 0; h_end: those behind them, where wanted, may be h0's buffer (a step of one
 * token for each of seqs requests is length = 1).  States inside a call are fp32.
 * Backward, from f, x, g, h0 (states are computed again): of dy (and dh_end, fp32, NULL: 0) df, dx, dg (with g) and dh0, each where
 * wanted; dh0 may be dh_end's buffer. */
typedef enum { FTP_SCAN_ADD = 0, FTP_SCAN_MIX = 1, FTP_SCAN_UNIT = 2 } ftp_scan_form;
typedef struct {
  int64_t rows, length;
  int32_t width, seqs;
  int32_t dtype, form, act;       /* form: ftp_scan_form                            */
  const int32_t* starts;
  const void* f; int64_t ldf;
  const void* x; int64_t ldx;
  const void* g; int64_t ldg;
  const float* h0; int64_t ldh0;
  void* y; int64_t ldy;
  float* h_end; int64_t ldhe;
  const void* dy; int64_t lddy;
  const float* dh_end; int64_t lddhe;
  void* df; int64_t lddf;
  void* dx; int64_t lddx;
  void* dg; int64_t lddg;
  float* dh0; int64_t lddh0;
  void* ws; size_t ws_bytes;
} ftp_scan_args;
int ftp_scan_workspace(const ftp_scan_args*, int backward, size_t* bytes);
int ftp_scan_forward(const ftp_scan_args*, void* stream);
int ftp_scan_backward(const ftp_scan_args*, void* stream);

/* What a model answers: with z = scale * logits and lse = log(sum of e^z) of a row, logp = z[id] - lse, entropy = -sum of p log p
 * (p = e^(z - lse)), and the `top` tokens of the largest logits with their log probabilities; each where wanted, fp32 (top_ids int32),
 * top_ids and top_logp [rows][top] together.  Equal logits: the lower token first.
 *   - A logit of -inf is a token that cannot come: p = 0, never among the top; places without a token hold -1 and -inf.
 *   - A row with nothing but -inf: lse and logp -inf, entropy 0, gradient 0.  With NaN or +inf in a row: lse, logp, entropy,
 *     top_logp and the row's gradient are NaN; top_ids are the largest that are numbers.
 *   - id = pad_id: logp 0, and dlogp adds nothing; an id that is none of 0 .. vocab-1: logp NaN, and dlogp adds nothing.
 *   - stats [rows][2]: what the backward needs, the row's largest logit and lse - scale * that (lse alone would not tell a row of the type's
 *     lowest value from one token).
 * Backward, from logits, stats and (with dentropy) entropy: dlogits = scale * (dlogp ([v = id] - p) - dentropy p (log p + entropy)) of
 * dlogp and dentropy, fp32 [rows], one of which may be NULL.  dlogits may be the logits' buffer. */
typedef struct {
  int64_t rows;
  int32_t vocab, dtype;
  int32_t ids64;          /* ids are int64 (otherwise int32)                        */
  int32_t top;            /* 0 .. 64                                                */
  float scale;            /* > 0, finite                                            */
  int64_t pad_id;
  const void* logits; int64_t ldl;
  const void* ids;
  float *logp, *entropy, *lse, *stats;
  int32_t* top_ids; float* top_logp;
  const float *dlogp, *dentropy;
  void* dlogits; int64_t lddl;
  void* ws; size_t ws_bytes;
} ftp_logp_args;
int ftp_logp_workspace(const ftp_logp_args*, size_t* bytes);           /* the forward's       */
int ftp_logp_forward(const ftp_logp_args*, void* stream);
int ftp_logp_backward(const ftp_logp_args*, void* stream);             /* without a workspace */

/* ---- diagnostics ---------------------------------------------------------------- */

/* Per-kernel timing for benchmarks (not part of the paper's method).  Between
 * begin and end every kernel launch of this library is bracketed by HIP events
 * on its own stream; end synchronises the device and returns one row per kernel
 * family: launches, summed duration, summed algorithmic bytes (every operand of
 * a launch counted once) and floating-point operations.  max_launches bounds the
 * event pool; exceeding it makes end return FTP_ERR_ARG with partial rows.  A
 * negative max_launches (pool size = its magnitude) splits the rows further by
 * problem shape: the name then reads "family d0 d1 d2" (GEMMs: M K N).  Where a family has a kernel on several tiles, rows
 * "__route <kernel> <tile> family d0 d1 d2" count its launches (no time of their own).
 * One more row, named "__event_pair_overhead" (launches = 1), gives in total_ms what a pair of events adds
 * to the launch it brackets, measured at begin on empty kernels: take it off every launch's time to get kernel
 * durations comparable with a profiler's.
 * Process-wide, not thread-safe, and the event records slow small steps down. */
typedef struct {
  char name[48];
  int64_t launches;
  double total_ms, alg_bytes, flops;
} ftp_ktrace_row;
int ftp_ktrace_begin(int max_launches);
int ftp_ktrace_end(ftp_ktrace_row* rows, int max_rows, int* n_rows);

/* Test hook for the error path of the compute calls: marks, for the calling thread, a launch plan as failed, exactly
 * as a kernel launcher does when a shape falls outside what its kernel was written for.  The next compute call of
 * this thread (forward, loss, backward, update, aggregate, copy_units) then returns FTP_ERR_UNSUPPORTED with the
 * reason in ftp_last_error() and clears the mark; other threads are not affected. */
int ftp_diag_fail_next_launch_plan(void);

/* Copies `bytes` (a multiple of 16) from src_dev to dst_dev with a plain kernel: a launch of
 * exactly known HBM traffic (bytes read + bytes written) against which hardware traffic counters
 * (rocprofv3 FETCH_SIZE / WRITE_SIZE) are scaled.  Asynchronous on `stream`. */
int ftp_calibration_copy(void* dst_dev, const void* src_dev, size_t bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FTP_H */
