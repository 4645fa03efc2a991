/*
 * omni.h -- C ABI of the OmniLearn data-parallel hot path on one GPU.
 *
 * The library implements, for K workers whose gradients sit in K device buffers:
 *   - the proportional batch-size controller (paper Eq. 6a/6b, dead-band Eq. 7, batch bounds,
 *     global-batch rule Eq. 8; procedures getBsz of Algorithm 1 and evalBsz of Algorithm 2),
 *   - the batch-size-weighted aggregation of the K gradients fused with the parameter update
 *     (Eq. 4b, Eq. 4c; Algorithm 1 "AllReduce(lambda_k g)" and "theta - eta gbar"),
 *   - the asynchronous per-arrival update with the batch-scaled learning rate
 *     (Eq. 5b; Algorithm 2 "eta_k = eta b / B", "theta - eta_k g").
 *
 * Conventions
 *   - Every function returns 0 (OMNI_OK) or a negative omni_status.  Nothing throws, aborts or
 *     traps.  Arguments are validated before any state changes or any kernel is enqueued: a
 *     failed call leaves the context and all buffers as they were.
 *   - "device pointer" = memory of the CUDA device that is current when the call is made;
 *     "host pointer" = ordinary host memory.  Parameter-sized buffers are owned by the caller
 *     and must stay alive until the stream has executed the call.
 *   - Kernels are enqueued on the caller's stream (a cudaStream_t passed as void*, NULL = the
 *     default stream) and the call returns without synchronising, unless stated otherwise.
 *   - A context is not thread-safe.  It owns a small device workspace (per-block partial sums
 *     and the gradient-norm cell, a few tens of KB) that is allocated by the first call that
 *     launches a kernel and freed by omni_destroy; calls on different streams that share a
 *     context and overlap on the GPU race on it.  The synchronous step leaves one partial sum of
 *     the squared gradient norm per thread block there; they are added up, in a fixed order, by
 *     a one-warp kernel that omni_get_stats and omni_aggregate_bsp_host enqueue, so a step that
 *     nobody asks the norm of pays nothing for it.
 *   - OMNI_MAX_K = 32 workers.
 */
#ifndef OMNI_H_
#define OMNI_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OMNI_MAX_K 32
#define OMNI_TAU_BINS 33 /* staleness 0..31 and one overflow bin */

typedef enum {
    OMNI_OK = 0,
    OMNI_ERR_NULL = -1,            /* a required pointer is NULL */
    OMNI_ERR_BAD_K = -2,           /* K outside 1..OMNI_MAX_K */
    OMNI_ERR_BAD_WORKER = -3,      /* worker index outside 0..K-1 */
    OMNI_ERR_BAD_BATCH = -4,       /* some b_k < 1, or sum b_k != B in synchronous mode */
    OMNI_ERR_INFEASIBLE = -5,      /* K*b_min > B or K*b_max < B in synchronous mode */
    OMNI_ERR_BAD_MEASUREMENT = -6, /* throughput/time not finite or <= 0 */
    OMNI_ERR_ALIGN = -7,           /* a device pointer is not 16-byte aligned */
    OMNI_ERR_BAD_TAU = -8,         /* negative staleness */
    OMNI_ERR_CUDA = -9,            /* a CUDA call failed; see omni_last_cuda_error */
    OMNI_ERR_TIMEOUT = -10,        /* a bounded device-side wait ran out */
    OMNI_ERR_BAD_CONFIG = -11,     /* invalid omni_config field or call argument */
    OMNI_ERR_TOO_LARGE = -12,      /* size beyond a stated maximum */
    OMNI_ERR_NO_MEMORY = -13       /* a host allocation failed */
} omni_status;

typedef enum { OMNI_BSP = 0, OMNI_ASP = 1 } omni_mode;
typedef enum { OMNI_F32 = 0, OMNI_BF16 = 1 } omni_dtype;

/* omni_config.flags */
#define OMNI_UNSCALED_MEAN 1u   /* lambda_k = 1/K: the unweighted arm of the paper's "weighted aggregation" table */
#define OMNI_ASP_NO_LR_SCALE 2u /* eta_k = eta: the "w/o LR scaling" arm of the paper's ASP table */
#define OMNI_INPUT_IS_TIME 4u   /* measurements are compute times t_k instead of throughputs T_k */
/* Global-batch rule, second reading.  Eq. 8 subtracts the same Delta B / K from every worker
 * (the default); the sentence after it (Sec. III-B, "Control Stability") speaks of reducing the
 * adjusted batches "proportionately".  With this flag the synchronous re-batch renormalises the
 * real-valued getBsz results c_k of all workers, c_k <- c_k * B / sum_i c_i, before the rounding
 * step, and the unit steps of the default rule only close what rounding and the bounds leave.
 * From equal batches without dead-band and bounds this gives B * T_k / sum(T) in one step
 * (Eq. 4a with the throughputs as capacities).  Ignored in asynchronous mode. */
#define OMNI_CONSERVE_MULTIPLICATIVE 32u
/* Kernel family.  By default the device calls stage their inputs through shared memory with
 * bulk (TMA) copies and an mbarrier ring; register-staged 128/256-bit-load kernels exist for
 * every call as well (and serve omni_aggregate_bsp_noalloc).  The ring
 * kernels also alternate the direction in which successive calls walk the parameters and keep
 * theta and v in L2 with evict-last priority, so that a call finds the part its predecessor
 * touched last still in cache, and are launched with programmatic stream serialization (they
 * wait for the previous launch themselves, after their set-up).  The two flags force
 * one family; results are the same bit for bit.  A bounded wait of the ring that runs out
 * surfaces as OMNI_ERR_TIMEOUT from omni_get_stats.
 * Contract for the caller's own kernels on the same stream: the ring kernels (and the one-warp
 * kernels of the device-resident controller) signal "dependents may launch" (griddepcontrol.launch_dependents) as soon as
 * their set-up is done, long before their last store.  A kernel enqueued after a library call
 * in the ordinary way is not affected: the stream still runs it after the library's kernel has
 * finished.  A kernel that the caller launches WITH the programmatic-stream-serialization
 * attribute, however, may start while the library's kernel is still writing: it must execute
 * griddepcontrol.wait (cudaGridDependencySynchronize) before it touches theta, v, the bf16
 * copy, the batches or any other buffer of the call.  Contexts created with OMNI_NO_BULK_COPY
 * launch only ordinary kernels and never signal early. */
#define OMNI_BULK_COPY 8u
#define OMNI_NO_BULK_COPY 16u
/* omni_create refuses flag bits it does not know and both kernel-family flags together (BAD_CONFIG). */

/* The "Input:" line of Algorithm 1 / Algorithm 2 (K, B, Delta b_k, b_min, b_max) plus the EWMA weight. */
typedef struct {
    int32_t K;            /* workers, 1..OMNI_MAX_K */
    int32_t global_batch; /* B; initial b_k = B / K (first B mod K workers take one more) */
    int32_t b_min, b_max; /* batch-size bounds, 1 <= b_min <= b_max */
    double deadband;      /* Delta b_k of Eq. 7 as a fraction, >= 0 */
    double ewma_alpha;    /* weight of the newest compute-time sample, (0, 1]; 1 = no smoothing */
    int32_t mode;         /* OMNI_BSP: Eq. 8 keeps sum b_k = B.  OMNI_ASP: no such rule. */
    uint32_t flags;
} omni_config;

/* One bucket = contiguous storage holding one or more whole tensors.  A flat model is one bucket. */
typedef struct {
    void *param;              /* device, float[n], 16-byte aligned, read and written: master parameters theta */
    void *momentum;           /* device, float[n], 16-byte aligned, read and written: v.  May be NULL iff momentum == 0 */
    void *param_lp;           /* device, bfloat16[n], 16-byte aligned, written: rounded copy of the new theta; or NULL */
    const void *const *grads; /* HOST array of K device pointers (float[n] or bfloat16[n], 16-byte aligned, read only) */
    uint64_t n;               /* elements; 0 is allowed (the bucket is skipped) */
} omni_bucket;

typedef struct {
    double grad_sqnorm;  /* sum_j gbar_j^2 of the aggregated gradient of the last omni_aggregate_bsp call */
    double weight_sum;   /* sum_k lambda_k (as rounded to float) of that call */
    uint64_t steps;      /* synchronous steps enqueued */
    uint64_t arrivals;   /* asynchronous arrivals enqueued */
    uint64_t tau_hist[OMNI_TAU_BINS]; /* arrivals by staleness 0..31, last bin: 32 and more */
    int32_t tau_max;
    uint64_t tau_sum;    /* sum of the staleness of all arrivals (mean = tau_sum / arrivals) */
} omni_stats;

typedef struct omni_ctx omni_ctx;

const char *omni_strerror(int status);

/* Create a controller context with b_k = B / K (Algorithm 1, first line of Train).  Needs no GPU.
 * Errors: NULL, BAD_K, BAD_CONFIG, INFEASIBLE, NO_MEMORY. */
int omni_create(const omni_config *cfg, omni_ctx **out);
void omni_destroy(omni_ctx *ctx);

/* Current batch sizes, b[K] host array (BSP: the controller's b_k; ASP: the server's wrkB map). */
int omni_get_batches(const omni_ctx *ctx, int32_t *b);
/* Overwrite them.  BAD_BATCH if some b_k < 1 or, in BSP mode, sum != B. */
int omni_set_batches(omni_ctx *ctx, const int32_t *b);

/* Controller state for checkpoints (the paper notes that a batch re-adjustment goes through a
 * checkpoint of the job, Sec. III-B): the batches, the smoothed compute times and which workers
 * have one yet, as one flat record.  omni_ctl_export: *size (host, in/out) holds the capacity of
 * `record` (host) and receives the record's size; record == NULL only queries the size.
 * omni_ctl_import restores a record into a context created with the same K and global batch;
 * batch sizes and times are validated and a failed import changes nothing.  Parameter buffers,
 * momentum and the device copy of the controller are the caller's to save.
 * Errors: NULL, TOO_LARGE (capacity below the record's size), BAD_CONFIG (not a record, or made
 * for another K or global batch), BAD_BATCH, BAD_MEASUREMENT. */
int omni_ctl_export(const omni_ctx *ctx, void *record, uint64_t *size);
int omni_ctl_import(omni_ctx *ctx, const void *record, uint64_t size);

/* Synchronous re-batch: getAvgComputeTime + getBsz for every worker (Algorithm 1) + Eq. 8.
 * measured[K] (host): throughput T_k in samples per time unit seen with the current b_k, or the
 * compute time t_k if OMNI_INPUT_IS_TIME.  Steps, all in IEEE double, sums in ascending k:
 *   t_k = b_k / T_k;  s_k = EWMA(t_k);  tbar = (sum s_k) / K;                      (Eq. 6a)
 *   b*_k = b_k - (b_k / s_k) (s_k - tbar);                                          (Eq. 6b)
 *   if |(b*_k - b_k) / b*_k| >= deadband: b*_k clamped to [b_min, b_max], else b_k;  (Eq. 7)
 *   round half up to an integer; BSP: shift all workers not pinned at a bound, one unit at a
 *   time, until sum = B; leftover units go to the largest batches, lowest index first.  (Eq. 8)
 * new_b[K] (host, out) receives the batches; changed[K] (host, out, may be NULL) 0/1 flags.
 * Errors: NULL, BAD_MEASUREMENT, INFEASIBLE. */
int omni_rebatch(omni_ctx *ctx, const double *measured, int32_t *new_b, int32_t *changed);

/* Asynchronous re-batch: evalBsz of Algorithm 2.  Worker `worker` reports the batch it ran and
 * its measurement; both are stored.  Until every worker has reported once, *new_b_k = b_used.
 * Afterwards getBsz is re-evaluated for all K stored entries against their mean time (no Eq. 8)
 * and *new_b_k is the caller's entry.  Errors: NULL, BAD_WORKER, BAD_BATCH, BAD_MEASUREMENT. */
int omni_asp_report(omni_ctx *ctx, int32_t worker, int32_t b_used, double measured, int32_t *new_b_k);

/* Static variable batching, Eq. 4a: b_k = c_k / sum(c) * B from worker capacities c_k (host,
 * K positive values, e.g. core counts), rounded to integers within the bounds with sum = B in
 * BSP mode.  Stores and returns the batches.  Errors: NULL, BAD_MEASUREMENT, INFEASIBLE. */
int omni_rebatch_static(omni_ctx *ctx, const double *capacity, int32_t *new_b);

/* One synchronous step over all buckets: Eq. 4b/4c fused with the optimiser update.  Per element j:
 *   lambda_k = float(b_k / sum_i b_i)          (1/K with OMNI_UNSCALED_MEAN)
 *   gbar = fma(lambda_{K-1}, g_{K-1,j}, ... fma(lambda_0, g_{0,j}, 0))   ascending k, single precision
 *   d = weight_decay ? fma(weight_decay, theta_j, gbar) : gbar
 *   v_j = momentum ? fma(momentum, v_j, d) : d          (stored when the momentum buffer is given)
 *   theta_j = fma(-lr, v_j, theta_j);  param_lp_j = bfloat16(theta_j) round-to-nearest-even
 * and the squared norm of gbar over all buckets is left in the context (omni_get_stats).
 * buckets: host array of n_buckets descriptors; b: host int32[K], the batches these gradients
 * were computed with (each >= 1; in BSP mode sum must equal B).  grad_dtype selects float or
 * bfloat16 gradients (bfloat16 is widened exactly).  Enqueues on `stream`, does not synchronise.
 * Errors: NULL, BAD_BATCH, ALIGN, BAD_CONFIG (n_buckets < 0, bad dtype, momentum != 0 with a
 * NULL momentum buffer), CUDA. */
int omni_aggregate_bsp(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                       const int32_t *b, float lr, float momentum, float weight_decay, void *stream);

/* One iteration of Algorithm 1's training loop in a single call: the aggregate + update of
 * omni_aggregate_bsp with the controller's CURRENT batches (the ones the workers computed these
 * gradients with: lambda_k = b_k / B), followed by omni_rebatch from `measured` (host, K values
 * observed during this iteration), whose result applies to the next iteration's gradients.
 * next_b[K] (host, out) receives the new batches, changed[K] (host, out, may be NULL) the 0/1 flags.
 * Same arithmetic and the same kernels as the two calls made one after the other; it exists so
 * that a step costs one trip through the binding instead of two, which matters for models small
 * enough to be bound by the host's launch rate.  All arguments, the measurements included, are
 * validated before the kernel is enqueued or the controller changes.
 * Errors: those of omni_aggregate_bsp and omni_rebatch. */
int omni_step_bsp(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                  const double *measured, float lr, float momentum, float weight_decay, int32_t *next_b,
                  int32_t *changed, void *stream);

/* One asynchronous arrival: worker `worker`'s gradient (buckets[i].grads[worker]), computed on
 * b_used samples, is applied to the server parameters with eta_k = float(lr * b_used / B)
 * (Eq. 5b; eta_k = lr with OMNI_ASP_NO_LR_SCALE):
 *   d = weight_decay ? fma(weight_decay, theta_j, g_j) : g_j;  v_j = momentum ? fma(momentum, v_j, d) : d;
 *   theta_j = fma(-eta_k, v_j, theta_j)
 * tau = server updates since this worker last read the parameters; the paper defines no
 * staleness-dependent factor, so tau is only tallied (omni_stats.tau_hist, tau_max).
 * Errors: NULL, BAD_WORKER, BAD_BATCH (b_used < 1), BAD_TAU, ALIGN, BAD_CONFIG, CUDA. */
int omni_apply_asp(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                   int32_t worker, int32_t b_used, int32_t tau, float lr, float momentum, float weight_decay,
                   void *stream);

/* A batch of m queued asynchronous arrivals applied in one pass over the parameters, in the order
 * given: exactly the result of m successive omni_apply_asp calls (the element goes through the
 * m updates of Eq. 5b one after the other, theta and v staying in registers), but theta and v
 * are read and written once, so the traffic is 4m+8 (+8 with momentum) bytes per parameter
 * instead of 12m (20m).  workers[m], b_used[m], tau[m]: host arrays; a worker may appear more
 * than once (its buffer is then applied again).  1 <= m <= OMNI_MAX_ASP_BATCH.
 * Errors: as omni_apply_asp, plus TOO_LARGE for m out of range. */
#define OMNI_MAX_ASP_BATCH 16
int omni_apply_asp_batch(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype, int32_t m,
                         const int32_t *workers, const int32_t *b_used, const int32_t *tau, float lr, float momentum,
                         float weight_decay, void *stream);

/* Algorithm 2 taken literally (pull / local update / push with overwrite), for callers that want
 * the paper's parameter-server semantics instead of "apply to the current copy".
 * omni_asp_pull: pullFromPS -- snapshots[i] (HOST array of n_buckets device pointers, float[n]
 * each, 16-byte aligned, caller-owned, one set per worker) <- buckets[i].param, by device copies
 * enqueued on `stream`.
 * omni_asp_push_overwrite: the worker's local step and pushToPS in one launch --
 *   theta_j <- fma(-eta_k, d, s_j),  d = weight_decay ? fma(weight_decay, s_j, g_j) : g_j,
 * with s the snapshot that worker pulled, g = buckets[i].grads[worker], eta_k as in omni_apply_asp.
 * The server copy is OVERWRITTEN: whatever other workers pushed since this worker's pull is lost
 * (the paper's "overridden" updates), so here the staleness tau changes the result, although it
 * still enters no formula; it is tallied as in omni_apply_asp.  Plain SGD as in Algorithm 2 (no
 * momentum buffer is read or written).  With tau = 0 the result equals omni_apply_asp's.
 * omni_asp_push_pull: the push above followed at once by the same worker's next pull, as in the
 * worker loop of Algorithm 2 (pushToPS at the end of one iteration, pullFromPS at the start of the
 * next), in the same launch: the server copy AND the worker's snapshot receive the new
 * parameters (snapshots are read and written).  Same result as omni_asp_push_overwrite followed
 * by omni_asp_pull of that worker, at 16 instead of 20 bytes per parameter.
 * Errors: NULL, BAD_WORKER, BAD_BATCH, BAD_TAU, ALIGN, BAD_CONFIG, CUDA. */
int omni_asp_pull(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, void *const *snapshots, void *stream);
int omni_asp_push_overwrite(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                            int32_t worker, int32_t b_used, int32_t tau, const void *const *snapshots, float lr,
                            float weight_decay, void *stream);
int omni_asp_push_pull(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                       int32_t worker, int32_t b_used, int32_t tau, void *const *snapshots, float lr,
                       float weight_decay, void *stream);

/* Device-resident controller: the synchronous re-batch (getBsz of Algorithm 1 for every worker,
 * Eq. 6a/6b, dead-band Eq. 7, bounds, Eq. 8) as a one-warp kernel on a device copy of the
 * controller state, so that a whole step -- re-batch from measurements that are already on the
 * GPU, then aggregate + update with the new weights -- is enqueued (or captured in a CUDA graph)
 * without a host round trip.  Arithmetic and results are those of omni_rebatch, bit for bit:
 * single correctly rounded double operations in the same order, then integers.
 *
 * omni_ctl_to_device: copies the host controller state (b_k, smoothed times) and the weights
 *   lambda_k = float(b_k / sum b) to the device copy, allocating it on a context's first call
 *   (make that call outside stream capture).  Enqueued on `stream`.
 * omni_rebatch_device: measured_dev = DEVICE double[K] (throughputs, or times with
 *   OMNI_INPUT_IS_TIME), 8-byte aligned; new_b_dev = DEVICE int32[K] out, or NULL.  Updates the
 *   device copy's batches, smoothed times and weights.  A measurement that is not finite or not
 *   positive leaves the device copy untouched and records OMNI_ERR_BAD_MEASUREMENT, which the
 *   next omni_ctl_from_device returns (once).  The host controller is not touched: host calls
 *   (omni_rebatch, omni_get_batches, ...) keep seeing the state of the last
 *   omni_ctl_from_device.
 * omni_asp_report_device: evalBsz of Algorithm 2 (omni_asp_report) on the device copy: worker and
 *   b_used are host values, measured_dev = DEVICE double[1] (8-byte aligned), new_b_k_dev = DEVICE
 *   int32[1] out or NULL.  Stores the worker's batch and smoothed time in the device copy and,
 *   once every worker has an entry, re-evaluates all K entries (no Eq. 8); a bad measurement is
 *   recorded as for omni_rebatch_device.  Same integers as omni_asp_report, bit for bit.
 * omni_aggregate_bsp_device_batches: omni_aggregate_bsp with the weights the device copy holds
 *   (no `b` argument; nothing is checked against B on the host).  Always the bulk-copy ring kernel.
 * omni_ctl_from_device: synchronises `stream`, copies the device copy back into the host
 *   controller and omni_stats.weight_sum; returns a recorded device re-batch failure, if any.
 * omni_ctl_to_device and omni_ctl_from_device copy between pageable host memory and the device and
 * are not meant to be captured; omni_rebatch_device and omni_aggregate_bsp_device_batches are
 * plain kernel launches.
 * Errors: NULL, BAD_CONFIG (no device copy yet; or as omni_aggregate_bsp), ALIGN, CUDA;
 * omni_asp_report_device also BAD_WORKER, BAD_BATCH. */
int omni_ctl_to_device(omni_ctx *ctx, void *stream);
int omni_ctl_from_device(omni_ctx *ctx, void *stream);
int omni_rebatch_device(omni_ctx *ctx, const double *measured_dev, int32_t *new_b_dev, void *stream);
int omni_asp_report_device(omni_ctx *ctx, int32_t worker, int32_t b_used, const double *measured_dev,
                           int32_t *new_b_k_dev, void *stream);
int omni_aggregate_bsp_device_batches(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                                      float lr, float momentum, float weight_decay, void *stream);

/* Parameter-range sharding for one rank per GPU (no counterpart in the paper, whose workers
 * all-reduce whole gradients; this is the reduce-scatter form of the same sum).  Every element of
 * the step is independent of every other, so the AllReduce of Algorithm 1 followed by the update
 * can run as: rank r owns the elements [begin, begin + count) of each bucket, reads that range of
 * all K workers' gradients (its own locally, the others through peer-mapped pointers placed in
 * omni_bucket.grads), runs omni_aggregate_bsp on the sub-range, and the ranks then exchange the
 * updated ranges (all-gather) and add their squared norms.  This call only computes the range:
 * n elements are cut into units of OMNI_SHARD_UNIT elements (so that every range starts on a
 * 256-byte boundary of a float buffer and a 128-byte boundary of a bfloat16 buffer) and the
 * units are dealt out contiguously, rank counts differing by at most one unit; the ranges of
 * ranks 0..world-1 tile [0, n) in order.  count may be 0 when n is small.
 * Errors: NULL, BAD_CONFIG (world < 1, rank outside 0..world-1). */
#define OMNI_SHARD_UNIT 64
int omni_shard_range(uint64_t n, int32_t world, int32_t rank, uint64_t *begin, uint64_t *count);

/* Same step as omni_aggregate_bsp for gradients that arrive in HOST memory (pinned memory gives
 * asynchronous copies).  host_grads: host array of n_buckets*K host pointers, entry [i*K + k] =
 * worker k's gradient for bucket i.  buckets[i].grads must point at K device staging buffers of
 * n elements each, owned by the caller; the call copies every host gradient into its staging
 * buffer on `stream`, runs the fused step, copies the squared gradient norm back, synchronises
 * the stream and stores it in *grad_sqnorm (host, may be NULL).
 * Errors: as omni_aggregate_bsp.  Unlike the other calls, a CUDA failure part-way (a copy or the
 * launch refused by the runtime) can leave the staging buffers holding some of the new
 * gradients; theta and v are only ever changed by the fused step itself. */
int omni_aggregate_bsp_host(omni_ctx *ctx, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                            const void *const *host_grads, const int32_t *b, float lr, float momentum,
                            float weight_decay, void *stream, double *grad_sqnorm);

/* The same fused step as omni_aggregate_bsp for callers that are not allowed to allocate device
 * memory when they run a step.  (The paper has no counterpart: this is a deployment variant of
 * the call above, not part of the method.)
 *
 * Who needs it: code that runs inside another framework's allocator callback or under its
 * allocator lock, processes whose device memory has all been handed to a pool at start-up, and
 * latency-critical loops that ban calls which may synchronise the device, as cudaMalloc and
 * cudaFree may.  omni_aggregate_bsp allocates a small workspace on a context's first launch;
 * this function calls no cudaMalloc, cudaFree or other allocating routine (see "Warm-up" below
 * for what the CUDA runtime does on its own the first time a kernel is used).  Its kernel's
 * scratch (one partial sum of the squared norm per CTA, about 19 KB) is a fixed
 * array inside the library's device image: every GPU that loads the library holds it until the
 * process exits.
 *
 * It takes no context: K, the batches and the flags (OMNI_UNSCALED_MEAN) come as arguments and
 * lambda_k = b_k / sum b.  Arithmetic, layouts and alignment rules are those of
 * omni_aggregate_bsp.  grad_sqnorm_dev (DEVICE pointer, 8-byte aligned, may be NULL) receives
 * the squared norm of the aggregate from a one-warp kernel enqueued after the step (it adds the
 * partial sums in a fixed order; with NULL it is not launched).  Enqueues on `stream`, does not
 * synchronise.
 *
 * Limits: at most OMNI_NOALLOC_MAX_BUCKETS non-empty buckets and OMNI_NOALLOC_MAX_ELEMENTS
 * elements in total; more returns OMNI_ERR_TOO_LARGE and does nothing.
 * Sharing: all calls on one device use the same array, which keeps the previous call's
 * contents; no cell has to start at zero (each launch overwrites every cell it later reads).  Calls
 * whose kernels overlap on the GPU (issued on different streams without ordering) race on it
 * and give wrong norms: keep them on one stream or order them with events.
 * First call: the first call on each device looks up the array's device address
 * (cudaGetSymbolAddress) with that device current; make that call before any stream capture.
 * It is not thread-safe against another first call on the same device.
 * Warm-up: "never allocates" is what this function does itself.  The CUDA runtime loads a
 * kernel's code, and whatever device memory that code needs, the first time the kernel is
 * launched, and the first call for a combination of (device, gradient type, K, all buffers
 * 32-byte aligned or not) also asks the runtime once for that kernel's occupancy.  A caller
 * whose restriction covers the runtime's own lazy loading should therefore make one call per
 * combination it will use (tiny buffers will do) before it enters the restricted region; every
 * later call is one kernel launch and, with grad_sqnorm_dev, a second one-warp launch, both
 * asynchronous.
 * flags: OMNI_UNSCALED_MEAN or 0; any other bit returns OMNI_ERR_BAD_CONFIG.
 * Errors: BAD_K, NULL, BAD_CONFIG, BAD_BATCH (some b_k < 1), ALIGN, TOO_LARGE, CUDA. */
#define OMNI_NOALLOC_MAX_BUCKETS 8
#define OMNI_NOALLOC_MAX_ELEMENTS (1ull << 31)
int omni_aggregate_bsp_noalloc(int32_t K, const omni_bucket *buckets, int32_t n_buckets, int32_t grad_dtype,
                               const int32_t *b, uint32_t flags, float lr, float momentum, float weight_decay,
                               double *grad_sqnorm_dev, void *stream);

/* Synchronises `stream` and fills *out (host).  The squared norm of the last synchronous step is
 * summed here, by a one-warp kernel enqueued on `stream`: pass the stream that step was enqueued
 * on, or one that has been ordered after it. */
int omni_get_stats(omni_ctx *ctx, omni_stats *out, void *stream);

/* Failure-path self-test (no counterpart in the paper).  Every device-side wait of the library is
 * bounded; when one runs out the kernel records it and the next omni_get_stats returns
 * OMNI_ERR_TIMEOUT once, then clears the record.  This call enqueues a one-warp kernel that waits,
 * with a short limit, on a barrier nothing completes, so that the path can be observed without
 * any kernel misbehaving: afterwards omni_get_stats must return OMNI_ERR_TIMEOUT, the context
 * stays usable, and the following omni_get_stats returns OMNI_OK.  Errors: NULL, CUDA. */
int omni_selftest_wait_expiry(omni_ctx *ctx, void *stream);

/* The cudaError_t of the last failed CUDA call made through this context (0 if none). */
int omni_last_cuda_error(const omni_ctx *ctx);

/* Persistent-grid size and block size the synchronous kernel for this K and dtype is launched
 * with on the current device for a launch of ordinary length (32-byte aligned buffers assumed;
 * block = 224 means the bulk-copy ring: 6 consumer warps + 1 producer warp; very short launches
 * may use a ring of 288 threads), and the number of kernels enqueued so far. */
int omni_query_launch(omni_ctx *ctx, int32_t K, int32_t grad_dtype, int32_t *grid, int32_t *block);
uint64_t omni_kernel_launches(const omni_ctx *ctx);

/* ==================================================================================================
 * Operators of a language model's training pass: what a worker computes its gradients with.  The
 * embedding at the bottom (its dense gradient is a slice of a gradient bucket), head norms with rotation and attention in the
 * blocks, the distillation or the policy loss on top; and AdamW on the workers' weighted gradients.  They take the context of the step for their launches,
 * their errors and the status word of bounded waits; scratch memory is the caller's (a query
 * function gives its size), so calls on different streams are independent as long as their
 * buffers are.  Kernels are enqueued on `stream`; nothing synchronises.  Sums, norms and softmax
 * statistics are float; a result is rounded once where it is stored.  No result depends on the
 * order of atomics: the same call gives the same bits.
 * Strides are in elements; the last dimension is contiguous.  "dtype" is an omni_dtype.  Pointers belong to the
 * current device.  The calls can be captured in a graph once the context has been used: its first call on a device allocates.
 * ================================================================================================== */
typedef enum { OMNI_I32 = 0, OMNI_I64 = 1 } omni_index;   /* type of token and vocabulary indices */

/* Embedding lookup: out_i = scale * table_{tokens[i]}, i = 0..n-1, computed in float and rounded to
 * out_dtype.  A token outside 0..vocab-1 gives a row of zeros.  tokens: device, n contiguous
 * indices; table: device, vocab rows of dim elements, table_stride apart; out: device, n rows.
 * Any dim and any stride >= dim; pointers need the alignment of their elements (rows on 16-byte
 * boundaries with dim a multiple of 8 run with wide accesses).
 * Errors: NULL, BAD_CONFIG (dtype, dim or vocab < 1, stride < dim), ALIGN, TOO_LARGE (n >= 2^31), CUDA. */
int omni_embed_forward(omni_ctx *ctx, const void *tokens, int32_t index_type, uint64_t n, const void *table,
                       int32_t table_dtype, uint64_t table_stride, int32_t vocab, int32_t dim, float scale, void *out,
                       int32_t out_dtype, uint64_t out_stride, void *stream);

/* Gradient of the lookup, dense, as a gradient bucket wants it:
 *   grad_v = (accumulate ? grad_v : 0) + scale * sum over i with tokens[i] = v of grad_out_i
 * for every v = 0..vocab-1.  The tokens are sorted on the device (stable, so that a row's terms are
 * added in ascending i within blocks of 32 sorted tokens, and the blocks in order).  Without accumulate all rows are set to
 * zero first, and the sums are stored over that; with it rows that no token names are not touched.  `padding` is a token without gradient (-1: none); tokens outside 0..vocab-1 have none
 * either.  grad_out: device, n rows of dim; grad: device, vocab rows of dim, not overlapping.
 * workspace: device, 16-byte aligned, at least omni_embed_workspace() bytes; its contents are free
 * again when the stream has executed the call.
 * Errors: as omni_embed_forward; TOO_LARGE also for a workspace below the size asked for. */
int omni_embed_workspace(uint64_t n, int32_t vocab, int32_t dim, uint64_t *bytes);
int omni_embed_backward(omni_ctx *ctx, const void *tokens, int32_t index_type, uint64_t n, const void *grad_out,
                        int32_t grad_out_dtype, uint64_t grad_out_stride, int32_t vocab, int32_t dim, float scale,
                        int64_t padding, void *grad, int32_t grad_dtype, uint64_t grad_stride, int32_t accumulate,
                        void *workspace, uint64_t workspace_bytes, void *stream);

/* Attention over [batch, length, head, dim] bfloat16 tensors, softmax in float:
 *   S = scale * Q K^T;  a query i of a sequence sees the keys j < kv length, with `causal` only those
 *   j <= i + (kv length - q length): the two sequences are aligned at their ends.
 *   lse_i = log sum_j exp(S_ij) over the keys seen;  O_i = sum_j exp(S_ij - lse_i) V_j
 * A query that sees no key has O = 0 and lse = -inf, and takes part in no gradient.  heads may be a
 * multiple of kv_heads: query head h uses key head h / (heads / kv_heads), whose gradients are summed.
 * q_lengths, kv_lengths: device int32[batch] or NULL, the lengths of a padded batch (clamped to
 * 0..q_len, 0..kv_len); what stands behind them in the inputs (NaN included) is not used, outputs there are 0 (lse: -inf).
 * dim: a multiple of 8 up to OMNI_ATTN_MAX_DIM; scale > 0. */
typedef struct {
    int32_t batch, q_len, kv_len, heads, kv_heads, dim;
    int32_t causal;
    float scale;
    const int32_t *q_lengths, *kv_lengths;
} omni_attn;
/* One operand: element (b, i, h, c) at data[b * batch + i * row + h * head + c].  data 16-byte aligned,
 * strides multiples of 8 elements (those of an extent of one do not matter). */
typedef struct {
    void *data;
    uint64_t batch, row, head;
} omni_attn_view;
#define OMNI_ATTN_MAX_DIM 128
/* omni_attn_forward writes out and lse (device float [batch, heads, q_len], contiguous).
 * omni_attn_backward recomputes the probabilities from lse:
 *   P = exp(S - lse), D_i = sum_c dO_ic O_ic, dS = P (dO V^T - D)
 *   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO
 * with P and dS rounded to bfloat16 for the products and every sum in float, in a fixed order.
 * workspace: device, 16-byte aligned, omni_attn_forward_workspace() bytes for the forward call (0 unless there are few
 * query rows for the GPU, whose walk along the keys is then split; NULL will do for 0) and omni_attn_workspace() for the
 * backward call.  Inputs, outputs and workspace do not overlap.
 * Errors: NULL, BAD_CONFIG (negative sizes, heads not a multiple of kv_heads, dim, scale, a stride below dim), ALIGN,
 * TOO_LARGE (dim, batch or heads > 65535, lengths > 2^30, a workspace below the size asked for), CUDA;
 * a bounded wait of the kernels that runs out surfaces as TIMEOUT from omni_get_stats. */
int omni_attn_forward(omni_ctx *ctx, const omni_attn *a, const omni_attn_view *q, const omni_attn_view *k,
                      const omni_attn_view *v, const omni_attn_view *out, float *lse, void *workspace, uint64_t workspace_bytes,
                      void *stream);
int omni_attn_forward_workspace(const omni_attn *a, uint64_t *bytes);
int omni_attn_workspace(const omni_attn *a, uint64_t *bytes);
int omni_attn_backward(omni_ctx *ctx, const omni_attn *a, const omni_attn_view *q, const omni_attn_view *k,
                       const omni_attn_view *v, const omni_attn_view *out, const float *lse, const omni_attn_view *dout,
                       const omni_attn_view *dq, const omni_attn_view *dk, const omni_attn_view *dv, void *workspace,
                       uint64_t workspace_bytes, void *stream);

/* Distillation from a teacher's top logits.  Per row, with temperature T, the student's logits z over
 * the vocabulary and the teacher's logits t_j at the indices i_j, j = 0..top-1:
 *   p = softmax(t / T) over the row's entries;  lse = log sum_v exp(z_v / T)
 *   loss = T^2 * sum_j p_j * (log p_j - z_{i_j} / T + lse)               (KL divergence, times T^2)
 *   grad_v = grad_loss * T * (exp(z_v / T - lse) - sum over j with i_j = v of p_j)
 * An entry whose index is outside 0..vocab-1 (-1 by convention) is not there, one whose logit is -inf
 * has p = 0; a row without any p > 0 has no target: its loss is 0 and its gradient row is zeros (lse
 * is still written).  A student logit of -inf has probability 0 (and an infinite loss if the teacher
 * gives it p > 0; in a row of -inf throughout every token has).  Logits far from zero are taken by their distances:
 * a row masked throughout by the type's lowest value is uniform (its lse is that value / T, -inf below float's range).
 * top = 1 with T = 1 is the ordinary cross-entropy of the index.
 * top_logits: device float; top_index: device, both rows of `top` elements, top_stride apart. */
typedef struct {
    const void *logits;     /* device, rows x vocab of dtype */
    uint64_t rows, row_stride;
    int32_t vocab, dtype;
    const float *top_logits;
    const void *top_index;  /* of index_type */
    uint64_t top_stride;
    int32_t top, index_type;
    float temperature;      /* > 0 */
} omni_distill;
#define OMNI_DISTILL_MAX_TOP 256
/* omni_distill_forward: loss[rows] and lse[rows] (device float).
 * omni_distill_backward: grad (rows x vocab of the logits' dtype, grad_stride apart) from the kept lse, as the float it is,
 * and grad_loss[rows] (device float; 0 for rows that do not count).  grad may be the logits' own
 * storage (same pointer and stride): each value is read before it is overwritten.
 * omni_distill_step: both in one pass over the logits (one read, one write), for a caller that knows
 * grad_loss beforehand, as with a mean over rows.
 * A gradient whose rows lie to 16-byte boundaries as the logits' do (the same storage, or the same stride and alignment) is
 * written in groups of eight; any other layout element by element, at a fifth to a half of the rate.
 * Errors: NULL, BAD_CONFIG (dtype, vocab or top < 1, temperature not finite or <= 0, a stride below the
 * row), ALIGN, TOO_LARGE (top > OMNI_DISTILL_MAX_TOP, rows >= 2^31), CUDA. */
int omni_distill_forward(omni_ctx *ctx, const omni_distill *d, float *loss, float *lse, void *stream);
int omni_distill_backward(omni_ctx *ctx, const omni_distill *d, const float *lse, const float *grad_loss, void *grad,
                          uint64_t grad_stride, void *stream);
int omni_distill_step(omni_ctx *ctx, const omni_distill *d, const float *grad_loss, float *loss, float *lse, void *grad,
                      uint64_t grad_stride, void *stream);

/* Norms of the query and key heads with the rotation by positions, in one pass.  Per head vector x of dim elements:
 *   n_c = w_c x_c (mean_c x_c^2 + eps)^(-1/2), with the side's weights; without weights (both NULL) n = x
 *   a pair (a, b) of n turns by the angle position * frequency:  y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin
 * Pair i = 0..pairs-1 is elements (i, i + pairs), or (2 i, 2 i + 1) with `interleaved`; the elements from 2 * pairs on are not
 * turned.  Its position is that of axis[i] (time, height, width of an image or video, say), its frequency frequency[i] in radians
 * per position.  Angles are taken in turns, in 64 bits modulo whole turns (off by 2^-60 turns per position and turn of frequency, so far
 * positions keep their phase), everything else in float with one rounding where a result is stored.
 * Backward, dn being the results' gradients turned back and g = w dn:
 *   dx = r (g - x r^2 mean_c(g_c x_c)),  r = (mean_c x_c^2 + eps)^(-1/2);  dw_c = sum over rows and heads of dn_c x_c r
 * A row of zeros is zeros (with eps = 0 not a number).
 * lengths: device int32[batch] or NULL: rows from there on are not read (NaN included), their results are 0 and they are in no sum. */
typedef struct {
    int32_t batch, length, heads, kv_heads;
    int32_t dim;                  /* even, up to OMNI_ROTARY_MAX_DIM */
    int32_t pairs;                /* 1..dim / 2 */
    int32_t axes;                 /* 1..OMNI_ROTARY_MAX_AXES */
    int32_t interleaved;
    int32_t dtype, weight_dtype;  /* of q, k and the results; of the weights */
    int32_t position_type;        /* omni_index */
    float eps;                    /* >= 0 */
    const double *frequency;      /* HOST, pairs values */
    const int32_t *axis;          /* HOST, pairs values in 0..axes-1; or NULL: all 0 */
    const void *positions;        /* device: that of axis a, sequence b, row i at a * position_axis + b * position_batch + i * position_row */
    uint64_t position_axis, position_batch, position_row;
    const void *q_weight, *k_weight;   /* device, dim values each, or both NULL */
    const int32_t *lengths;
} omni_rotary;
#define OMNI_ROTARY_MAX_DIM 256
#define OMNI_ROTARY_MAX_AXES 4
/* Operands are omni_attn_views of dtype (element (b, i, h, c) at data[b * batch + i * row + h * head + c]), aligned as their elements;
 * on 16-byte boundaries throughout, with dim a multiple of 16, they run with wide accesses, otherwise with those of 8, 4 or 2 bytes.  A result may be its operand's own storage (same pointer and strides).
 * omni_rotary_backward: dq_out, dk_out are the gradients of the forward call's results, dq and dk those of q and k.  With weights it
 * writes their gradients, dim values each of weight_grad_dtype (zeros if there are no rows), and needs a workspace (device,
 * 16-byte aligned, omni_rotary_workspace() bytes); without weights q, k, the weight gradients and the workspace are not looked at.
 * Sums over rows are added in an order that the sizes alone decide.
 * Errors: NULL, BAD_CONFIG (sizes, dim odd, pairs, axes, dtype, eps, a frequency that is not finite, a result's stride below dim, results
 * that write an element twice or share one with each other), ALIGN, TOO_LARGE (dim, batch * length >= 2^31, heads > 65535, strides >= 2^40, a workspace below the size asked for), CUDA. */
int omni_rotary_forward(omni_ctx *ctx, const omni_rotary *r, const omni_attn_view *q, const omni_attn_view *k,
                        const omni_attn_view *q_out, const omni_attn_view *k_out, void *stream);
int omni_rotary_workspace(const omni_rotary *r, uint64_t *bytes);
int omni_rotary_backward(omni_ctx *ctx, const omni_rotary *r, const omni_attn_view *q, const omni_attn_view *k,
                         const omni_attn_view *dq_out, const omni_attn_view *dk_out, const omni_attn_view *dq, const omni_attn_view *dk,
                         void *dq_weight, void *dk_weight, int32_t weight_grad_dtype, void *workspace, uint64_t workspace_bytes,
                         void *stream);

/* Clipped policy loss on sampled tokens, with a divergence from a reference policy.  Per row, with logits z over the vocabulary, the
 * token t, its log-probability `old` when it was sampled and `reference` under the reference, the advantage A:
 *   lse = log sum_v exp(z_v / T);  logp = z_t / T - lse;  ratio = exp(logp - old)
 *   surrogate = min(ratio A, clamp(ratio, 1 - clip_low, 1 + clip_high) A);  gap = reference - logp
 *   loss = -surrogate + kl (exp(gap) - gap - 1)
 *   grad_v = grad_loss c / T ([v = t] - exp(z_v / T - lse)),
 *            c = -(ratio A where ratio A is the smaller or equal, else 0) + kl (1 - exp(gap))
 * A token outside 0..vocab-1 (-1 by convention) is none: the row's loss, logp and gradient are 0, and nothing of it but the logits is
 * looked at (lse is still written).  A row whose grad_loss c is 0 has a gradient of zeros, and an advantage of 0 has no surrogate, whatever the ratio.
 * A logit of -inf has probability 0; logits far from zero are taken by their distances, as in omni_distill. */
typedef struct {
    const void *logits;           /* device, rows x vocab of dtype */
    uint64_t rows, row_stride;
    int32_t vocab, dtype;
    const void *tokens;           /* device, rows values of index_type */
    const float *old, *advantage; /* device, rows values each */
    const float *reference;       /* device, rows values; not looked at if kl is 0 */
    int32_t index_type;
    float clip_low, clip_high;    /* >= 0 */
    float kl;                     /* >= 0 */
    float temperature;            /* > 0 */
} omni_policy;
/* omni_policy_logprob: logp[rows] and lse[rows] (device float) alone; old, advantage, reference, clip and kl are not looked at.
 * omni_policy_forward: loss, logp, lse.  omni_policy_backward: grad (rows x vocab of the logits' dtype, grad_stride apart) from the
 * kept lse and grad_loss[rows]; a row whose |lse| or token's |z_t / T| is 128 or more, or whose ratio is within that float's rounding of a border, is
 * walked once more for its own sum: its gradient is the step's, on the side of the border that forward found.
 * omni_policy_step: both in one pass over the logits, for a caller that knows grad_loss beforehand.
 * logp and lse are the same bits from the three calls that return them: the ratio to an `old` that one of them gave is exactly 1.
 * grad may be the logits' own storage (same pointer and stride).  A gradient whose rows lie to 16-byte boundaries as the logits' do
 * is written in groups of eight, any other element by element.
 * Errors: NULL, BAD_CONFIG (dtype, vocab < 1, temperature, clip or kl negative or not finite, a stride below the row), ALIGN,
 * TOO_LARGE (rows >= 2^31), CUDA. */
int omni_policy_logprob(omni_ctx *ctx, const omni_policy *d, float *logp, float *lse, void *stream);
int omni_policy_forward(omni_ctx *ctx, const omni_policy *d, float *loss, float *logp, float *lse, void *stream);
int omni_policy_backward(omni_ctx *ctx, const omni_policy *d, const float *lse, const float *grad_loss, void *grad, uint64_t grad_stride,
                         void *stream);
int omni_policy_step(omni_ctx *ctx, const omni_policy *d, const float *grad_loss, float *loss, float *logp, float *lse, void *grad,
                     uint64_t grad_stride, void *stream);

/* AdamW over many tensors in one launch, on the batch-weighted gradients of K workers (the aggregation of omni_aggregate_bsp with
 * another update).  Per element of a tensor, in float, every operation rounded once, with lambda_k = float(b_k / sum b):
 *   g = fma(lambda_{K-1}, g_{K-1}, ... fma(lambda_0, g_0, 0));  m = fma(beta1, m, c1 g);  v = fma(c2 g, g, beta2 v)
 *   theta = fma(-rate, m / fma(sqrt(v), spread, eps), keep theta);  param_lp = bfloat16(theta)
 * c = float(1 - beta), rate = float(lr / (1 - beta1^t)), spread = float((1 - beta2^t)^(-1/2)), keep = float(1 - lr weight_decay), t = 1,
 * 2, ... the step's number.  m and v are exact.  With an eps between 2^-41 (1 - beta2)^(-1/2) and 2^100 the quotient, its root
 * included, is off by up to 2^-20.5 of itself, with any other theta is exact too.  An eps of 0 is allowed: the quotient of a v of 0 is not finite then.
 * bits = 8: m and v are kept as codes of the float's bits 20 to 30 (exponent and three bits of the fraction), counted from the largest
 * of their block of OMNI_ADAMW_BLOCK consecutive elements.  With top the block's largest, a code c > 0 is the float of bits (c + top - 127) << 20
 * for m, bit 7 of the byte its sign, and (c + top - 255) << 20 for v; c = 0 is 0.  theta is computed from m and v before they are
 * rounded: 16 random bits are added to bits 4 to 19 and what is below bit 20 is dropped; then m below code 1 is 0, v below it is code 1
 * unless it is 0.  The random bits are x = (x ^ x >> 15) of x = (y ^ y >> 16) * 0x7FEB352D, y = i * 0x9E3779B1 + t * 0x85EBCA77 +
 * tensor * 0xC2B2AE3D modulo 2^32 for element i of a tensor (numbered from 0 in the list): the low half for m, the high half for v.
 * So the same state, gradients and step give the same bits.  A gradient that is not finite spoils its element as in float, and the
 * codes of its block. */
#define OMNI_ADAMW_BLOCK 256
typedef struct {
    float *param;                 /* device, n values, read and written */
    void *param_lp;               /* device, bfloat16[n], written; or NULL */
    const void *const *grads;     /* HOST array of K device pointers, n values of grad_dtype each */
    void *m, *v;                  /* device, float[n], or uint8[n] for 8 bits, read and written; zeros at first */
    void *tops;                   /* device, 8 bits: int16[2] (m, v) for each block, 4-byte aligned, zeros at first; else not looked at */
    uint64_t n;                   /* 0 is allowed */
    double weight_decay;
} omni_adamw_tensor;
/* omni_adamw_plan writes a record of the tensors to host memory (8-byte aligned, omni_adamw_plan_bytes() bytes).  The caller copies
 * it to the device (16-byte aligned) and keeps both while it steps; pointers in it stay as they are.  Pointers need the alignment of
 * their elements; with all of a tensor's on 16-byte boundaries (8 for codes) it runs with wide accesses.
 * omni_adamw_step: one step; b: host int32[K], the batches of the gradients.  The step's number is `step`, or, if clock_dev is not
 * NULL, the int64 that clock_dev (device, 8-byte aligned) holds when the kernel runs, for a step that is captured in a graph; lr is the host's.
 * omni_adamw_moments: what the codes stand for, into m[i], v[i] (HOST arrays of device float pointers, one for each tensor); 8 bits only.
 * Errors: NULL, BAD_K, BAD_CONFIG (dtype, bits, what is written overlaps other tensors, not a record, lr or weight_decay not finite, beta outside [0, 1), eps, step < 1), BAD_BATCH,
 * ALIGN, TOO_LARGE (a tensor of 2^42 elements, 2^31 pieces of 1024 in all, a record that is too small), NO_MEMORY, CUDA. */
int omni_adamw_plan_bytes(const omni_adamw_tensor *tensors, int32_t count, int32_t K, int32_t grad_dtype, int32_t bits, uint64_t *bytes);
int omni_adamw_plan(const omni_adamw_tensor *tensors, int32_t count, int32_t K, int32_t grad_dtype, int32_t bits, void *record, uint64_t bytes);
int omni_adamw_step(omni_ctx *ctx, const void *record, const void *record_dev, const int32_t *b, double lr, double beta1, double beta2,
                    float eps, int64_t step, const int64_t *clock_dev, void *stream);
int omni_adamw_moments(omni_ctx *ctx, const void *record, const void *record_dev, float *const *m, float *const *v, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* OMNI_H_ */
