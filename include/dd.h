/*
 * dd.h -- batched what-if simulation of trace-derived task dependency graphs
 * on AMD Instinct MI355X (gfx950).
 *
 * The library answers "what if" questions the way Daydream does (Zhu,
 * Phanishayee, Pekhimenko, arXiv 2006.03318): a kernel-granularity task
 * graph recorded from one training iteration is transformed (tasks scaled,
 * removed, dependencies switched) and then simulated to predict the new
 * iteration time.  Here thousands of transformed variants of one graph are
 * simulated in one batch on the GPU.
 *
 * Semantics (the simulation of Sec. 4.1, Algorithm 1, "Daydream's Simulation
 * Algorithm"; task fields of Sec. 4.2.1; dependency types of Sec. 4.2.2):
 *   every task u has an execution thread (a CPU thread, a GPU stream or a
 *   communication channel), a duration d_u and a gap g_u (CPU time between
 *   the end of u and the next task on its thread), all int64 nanoseconds.
 *   Parents of u are its dependency in-edges plus the previous task on its
 *   thread.  With release R_p = start_p + d_p + g_p,
 *       start_u  = max(0, max over parents p of R_p)
 *       finish_u = start_u + d_u
 *       makespan = max over tasks not removed of finish_u   (0 if none)
 *   which is what Algorithm 1 computes: every child's start is raised to the
 *   parent's start + duration + gap, and tasks on one thread run in their
 *   recorded order (that order does not change between executions,
 *   Sec. 4.2.2).
 *
 * Transformations per variant (Sec. 4.4, graph-transformation primitives):
 *   shrink/scale: task of class c in variant v gets duration
 *                 floor(d * p / q) with (p, q) = scale[c][v];
 *   Remove:       a removed task gets duration 0 and gap 0, which is the
 *                 same as unlinking it and connecting each predecessor to
 *                 each successor; its start = finish = the time all its
 *                 inputs are available; it is left out of the makespan;
 *   re-route:     each dependency edge has a class k < 64; edges of class k
 *                 exist in variant v only if bit k of edge_on[v] is set
 *                 (tasks moved to another thread or re-ordered on a
 *                 channel are expressed by such edges).
 *   Gaps are never scaled.
 *
 * Conventions for every call:
 *   - All functions return dd_status; DD_OK (0) on success.  On failure
 *     dd_last_error() gives a message (per host thread) and no output
 *     handle is created.
 *   - Input arrays may be host or device pointers (each one independently);
 *     they are copied during the call and remain owned by the caller.
 *   - Output arrays of dd_simulate_batch are device pointers owned by the
 *     caller; the library never frees them.
 *   - Handles are owned by the library until the matching *_free.  A handle
 *     keeps device memory, released on the stream it was created on, which
 *     must stay valid until the handle is freed.  A handle may be used on
 *     any stream: the library records an event after each use on a stream
 *     other than the handle's own, and *_free makes the handle's stream wait
 *     for those events before its memory can be handed out again.  Released
 *     device memory stays in a cache of the library, kept per device and
 *     stream, and is handed out again to later calls on that same stream
 *     (stream order makes the reuse safe); it returns to the device when an
 *     allocation would otherwise fail, on dd_release_cache(), or at process
 *     exit.
 *   - `stream` is a hipStream_t (NULL = default stream).  Work is
 *     stream-ordered.  Input validation is synchronous: load, levelize and
 *     apply_transforms wait for their own device checks before returning.
 *     dd_simulate_batch is asynchronous; a device fault surfaces as DD_EHIP
 *     from the same or a later call.
 *   - Limits: 0 <= n < 2^31, n_threads >= 1, edges < 2^31, edge classes < 64,
 *     task classes < 65536, durations and gaps in [0, 2^62).
 */
#ifndef DD_H
#define DD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DD_OK = 0,
    DD_EINVAL = 1,     /* bad argument: NULL, out-of-range index or size, negative time */
    DD_ECYCLE = 2,     /* dependencies plus thread order contain a cycle */
    DD_ECHAIN = 3,     /* thread order is not one simple chain per thread */
    DD_ERANGE = 4,     /* scaled times could overflow int64 */
    DD_ENOMEM = 5,     /* device allocation failed */
    DD_EHIP = 6,       /* HIP runtime error */
    DD_EMISMATCH = 7,  /* handles from different graphs, or a variant uses an
                          edge class the schedule was not built for */
    DD_ELIMIT = 8      /* a fixed capacity of a device path was exceeded */
} dd_status;

typedef struct dd_graph dd_graph;
typedef struct dd_sched dd_sched;
typedef struct dd_variants dd_variants;

/* A duration scale p/q: p >= 0, q >= 1. */
typedef struct { int32_t p, q; } dd_ratio;

#define DD_LEVELS 0   /* steps = Kahn topological levels (longest hop path) */
#define DD_PHASES 1   /* steps = phases (longest path counting only edges
                         between different threads); one step holds one
                         contiguous run of each thread's tasks */

/*
 * dd_graph_load -- the task graph G(V, E) of Sec. 4.2 (tasks, Sec. 4.2.1;
 * dependencies, Sec. 4.2.2).
 *   n            number of tasks.
 *   n_threads    number of execution threads; thread ids are 0..n_threads-1.
 *   in_ptr       int64 [n+1], CSR offsets of dependency in-edges per task;
 *                in_ptr[0] == 0, non-decreasing.
 *   in_src       int32 [in_ptr[n]], source task of each in-edge.
 *   edge_cls     uint8 [in_ptr[n]], class (< 64) of each edge; NULL = 0.
 *   thread_prev  int32 [n], previous task on the same thread, -1 for the
 *                first; each thread must form one chain.
 *   thread_id    int32 [n], execution thread of each task.
 *   dur_ns       int64 [n], durations.   gap_ns  int64 [n], gaps.
 *   node_cls     uint16 [n], transform class of each task; NULL = 0.
 * Validates everything (DD_EINVAL, DD_ECHAIN, DD_ECYCLE for a self loop or
 * a dependency that goes backwards along one thread, DD_ERANGE), ranks the
 * thread chains, drops dependencies between tasks of the same thread (the
 * thread order already implies them) and builds the cross-thread edge lists
 * in both directions.  *out receives the handle.
 */
dd_status dd_graph_load(int32_t n, int32_t n_threads,
                        const int64_t *in_ptr, const int32_t *in_src, const uint8_t *edge_cls,
                        const int32_t *thread_prev, const int32_t *thread_id,
                        const int64_t *dur_ns, const int64_t *gap_ns, const uint16_t *node_cls,
                        void *stream, dd_graph **out);

/*
 * dd_graph_load_ex -- dd_graph_load with flags.
 *   DD_LOAD_SHARED_THREADS  a thread may hold several chains: tasks with
 *       thread_prev == -1 other than the first, and chains that share a
 *       thread, have no recorded order among themselves (for example the
 *       push and pull slices a what-if recipe inserts on a communication
 *       channel, Sec. 5.1 P3).  Their order is decided while simulating, by
 *       the schedule() rule of Sec. 4.4 ("Schedule"), so such a graph is
 *       simulated only by dd_simulate_policy; dd_levelize and
 *       dd_runtime_breakdown return DD_EINVAL for it.  Each task still has at
 *       most one thread successor (DD_ECHAIN otherwise), and dependencies
 *       between tasks of one thread are kept (no thread order implies them).
 * flags == 0 is dd_graph_load.  Unknown flag bits: DD_EINVAL.
 */
#define DD_LOAD_SHARED_THREADS 1u
dd_status dd_graph_load_ex(int32_t n, int32_t n_threads,
                           const int64_t *in_ptr, const int32_t *in_src, const uint8_t *edge_cls,
                           const int32_t *thread_prev, const int32_t *thread_id,
                           const int64_t *dur_ns, const int64_t *gap_ns, const uint16_t *node_cls,
                           uint32_t flags, void *stream, dd_graph **out);

/*
 * dd_levelize -- topological schedule of the graph restricted to the edge
 * classes in `active_edge_classes` (bit k = class k; thread order is always
 * present), computed on the GPU with Kahn's algorithm (the reference counts
 * and frontier of Algorithm 1, processed a whole frontier at a time).
 *   mode == DD_LEVELS: step of a task = its Kahn level.
 *   mode == DD_PHASES: step = its phase; every step consists of one
 *                      contiguous run of tasks per thread at most, and all
 *                      cross-thread inputs of a step come from earlier steps.
 * *n_steps_out (may be NULL) receives the number of steps.  DD_ECYCLE if
 * the active dependencies plus thread order contain a cycle.
 */
dd_status dd_levelize(const dd_graph *g, uint64_t active_edge_classes, int32_t mode,
                      void *stream, dd_sched **out, int64_t *n_steps_out);

/*
 * dd_apply_transforms -- per-variant transform tables (Sec. 4.4 primitives).
 *   n_variants   V >= 1.
 *   n_cls        rows of `scale`; must exceed every node_cls of the graph.
 *   scale        dd_ratio [n_cls][V]; NULL = all 1/1.
 *   remove_bits  uint32 [n][ceil(V/32)]; bit v%32 of word v/32 of row u set =
 *                task u removed in variant v; NULL = none removed.
 *   edge_on      uint64 [V]; bit k = edges of class k present; NULL = all.
 * DD_EINVAL for p < 0 or q < 1, DD_ERANGE if a scaled time could overflow.
 */
dd_status dd_apply_transforms(const dd_graph *g, int32_t n_variants, int32_t n_cls,
                              const dd_ratio *scale, const uint32_t *remove_bits,
                              const uint64_t *edge_on, void *stream, dd_variants **out);

/*
 * dd_simulate_batch -- simulate every variant (the hot path).
 *   d_finish    device int64 [n][V] (task-major, variant-minor), required
 *               unless n == 0: finish time of each task in each variant.
 *   d_start     device int64 [n][V] or NULL: start times.
 *   d_makespan  device int64 [V], required: iteration time of each variant.
 * All three handles must come from the same graph; every edge class some
 * variant switches on must be in the schedule's active classes
 * (DD_EMISMATCH otherwise).
 */
dd_status dd_simulate_batch(const dd_graph *g, const dd_sched *sched, const dd_variants *var,
                            int64_t *d_finish, int64_t *d_start, int64_t *d_makespan,
                            void *stream);

/*
 * dd_simulate_batch_vs -- dd_simulate_batch with an explicit launch shape.
 *   variants_per_wg  variants that each workgroup owns for the whole
 *                    schedule: 0 = chosen by the library (as
 *                    dd_simulate_batch), or 1, 2, 4, 8, 16 (1 runs the kernel
 *                    made for one variant per workgroup where its arithmetic
 *                    holds the times, see below);
 *                    -1, -2, -4, -8 = the few-variant path with that many
 *                    variants per workgroup: one launch per step, each step
 *                    cut into chunks of 256 positions taken by separate
 *                    workgroups (DD_EINVAL when the schedule has more than
 *                    512 steps); any other value returns DD_EINVAL.
 *   dd_simulate_batch itself takes the few-variant path when the variants
 *   are fewer than 1,024, the schedule has at most 512 steps, and its steps
 *   hold more than about 4.4 rounds of 512 positions on average (where that
 *   path measured faster).  Otherwise up to 768 variants (2,048 when steps
 *   hold at most 32 positions on average) run one per workgroup, in a kernel
 *   that holds times as integers in doubles (scaled times below 2.0e15 ns in
 *   sum, durations and gaps below 2^32, each duration times p below 2^50, at
 *   most 2,048 task classes) and needs V * (256 KiB + n / 8 bytes) of scratch
 *   at most, which stays in the library's cache (dd_release_cache); the strip
 *   kernel serves every other call, and those for which that scratch cannot
 *   be had.
 * The results do not depend on the shape (Algorithm 1 per variant, Sec. 4.1);
 * only the number of workgroups and the kernel instance do.  For tuning, and
 * for checking the compiled instances (the strip kernel with one variant per
 * workgroup is reached by dd_simulate_batch_noalloc with up to 256 variants).
 */
dd_status dd_simulate_batch_vs(const dd_graph *g, const dd_sched *sched, const dd_variants *var,
                               int64_t *d_finish, int64_t *d_start, int64_t *d_makespan,
                               int32_t variants_per_wg, void *stream);

/*
 * dd_set_lookback_polls -- how long a chunk of the few-variant path waits
 * for an earlier chunk (Sec. 4.1: the releases of one thread's run carried
 * across chunks).  A chunk reads the aggregate that each earlier chunk of its
 * run publishes; after `polls` unanswered reads it folds that chunk itself
 * from the inputs, which come from earlier launches, so no chunk ever depends
 * on another workgroup being resident.  The results do not depend on the
 * value.  polls < 0 restores the default (4,096); 0 makes every chunk fold
 * its predecessors itself (for tests of that fallback).  Applies to calls
 * made after it, process-wide.
 */
void dd_set_lookback_polls(int32_t polls);

/*
 * dd_simulate_batch_noalloc -- dd_simulate_batch for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc).  Same arguments, results and errors as
 * dd_simulate_batch; it always runs the one-workgroup-per-strip kernel with
 * the library's strip width (never the few-variant path, whose look-back
 * slots it would have to allocate), calls no hipMalloc, hipFree or other
 * allocating routine and records no events.
 *   Its working memory (round table, scan sums, per-position removal bits)
 *   lives in one array of 64 MiB per GPU inside the library, held until the
 *   process ends.  A batch needs about n*V/8 + 16*n_steps + 4*n/64 bytes of
 *   it (n*V up to about 5 * 10^8 task-variant pairs); a larger one returns
 *   DD_EINVAL with the size in dd_last_error() and launches nothing.
 *   Every call on one GPU uses that GPU's array: calls that overlap on one
 *   GPU (on different streams, or from several host threads) race and give
 *   wrong results.  The array keeps the last call's contents; nothing in it
 *   needs to start at zero.
 *   Handles used here on a stream other than their own are not tracked (no
 *   event is recorded): free them only after that stream's work is done.
 */
dd_status dd_simulate_batch_noalloc(const dd_graph *g, const dd_sched *sched, const dd_variants *var,
                                    int64_t *d_finish, int64_t *d_start, int64_t *d_makespan,
                                    void *stream);

/*
 * dd_runtime_breakdown -- where each variant's iteration time goes when the
 * CPU and the GPU overlap: the breakdown the paper uses to explain the AMP
 * speedups (Sec. 6.2, Fig. 6), computed by its own rules from a finished
 * dd_simulate_batch of the same graph and variants:
 *   total    = makespan;
 *   CPU-only = total - all GPU kernel runtime (the sum of the scaled
 *              durations of the kernels kept in the variant);
 *   GPU-only = the time the CPU is blocked on the GPU: for every call that
 *              waits for GPU work (synchronization, device-to-host copy), its
 *              start minus the moment its thread reached it (the release
 *              start + duration + gap of the previous task on the thread, 0
 *              for the first task);
 *   CPU+GPU parallel = total - CPU-only - GPU-only.
 *   role        uint8 [n], host or device: 1 = GPU kernel, 2 = CPU call that
 *               waits for GPU work, any other value = neither.  On the
 *               device it is read by the work that the call queues.
 *   d_finish    device int64 [n][V], d_makespan device int64 [V]: the outputs
 *               of dd_simulate_batch for (g, var), complete on `stream`.
 *   d_out       device int64 [V][4]: total, CPU-only, GPU-only, CPU+GPU
 *               parallel of each variant.
 * Asynchronous like dd_simulate_batch.  DD_EMISMATCH if var comes from
 * another graph.
 */
dd_status dd_runtime_breakdown(const dd_graph *g, const dd_variants *var, const uint8_t *role,
                               const int64_t *d_finish, const int64_t *d_makespan,
                               int64_t *d_out, void *stream);

/*
 * dd_simulate_policy -- simulate every variant with an overridden schedule()
 * (Sec. 4.4, "Schedule"): Algorithm 1 task by task, where schedule() picks
 * the next task from the frontier Q of ready tasks, kept in trace order
 * (ascending task id).  With time(x) = max(P[x's thread], x's start):
 *   DD_POLICY_EARLIEST  the first task of least time (the default rule);
 *   DD_POLICY_PRIORITY  P3's rule (the appendix's P3 model, its Schedule
 *                       function): scanning Q in order, a task of least time
 *                       is chosen, and a later task of equal time replaces
 *                       the choice when both are push/pull tasks (pp != 0)
 *                       and its priority is strictly higher.
 * On graphs whose threads are single chains every rule gives the result of
 * dd_simulate_batch.  Transformations as above (removed tasks run with zero
 * duration and gap); every variant's own edge classes apply, so one call
 * covers all variants of `var` without a schedule handle.
 *   pp, prio    uint8 [n] and int32 [n], host or device, read by
 *               DD_POLICY_PRIORITY (may be NULL for DD_POLICY_EARLIEST).
 *   d_finish    device int64 [n][V] (task-major, variant-minor), required
 *               unless n == 0.   d_start: the same or NULL.
 *   d_makespan  device int64 [V], required.
 * Limits: n < 2^22, n_threads <= 4096, in_ptr[n] + n < 2^31, and at most
 * 1024 tasks ready at once in any variant (DD_ELIMIT beyond, outputs
 * undefined).
 * Synchronous: returns when the simulation is done, with DD_ECYCLE if some
 * variant's active dependencies and thread chains contain a cycle.  Working
 * memory: at most 12 * n * V bytes of device memory for the call (with at
 * most 64 threads, 512 classes, durations and gaps below 2^32 and every edge
 * class on, 40 bytes per task, 4 per dependency and at most 6.3 KiB per
 * variant, with the 12 * n * V bytes only if more than 256 tasks are ready, or
 * wait for a part of their parents, at once, or times lie 2^31 ns apart).
 */
#define DD_POLICY_EARLIEST 0
#define DD_POLICY_PRIORITY 1
dd_status dd_simulate_policy(const dd_graph *g, const dd_variants *var, int32_t policy,
                             const uint8_t *pp, const int32_t *prio,
                             int64_t *d_finish, int64_t *d_start, int64_t *d_makespan,
                             void *stream);

/* ---------------------------------------------------------------------------
 * The operators that three of the what-if models predict, to run them and
 * hold the prediction against the measurement (the paper's own check, Sec. 6):
 * a fused weight update (What_If_Fused_Adam), low-precision weights with f32
 * masters (What_If_AMP), and the element-wise kernels around a block's
 * normalization fused into one (What_If_Restructuring_Batchnorm).
 *
 *   - All tensors are device memory of the caller, on the current device, and
 *     are aligned to their elements; nothing is copied.
 *   - Every call but dd_tensors_load is asynchronous on `stream`, and its
 *     results are the same bits on every run.
 *   - Values are computed in 32 bits or more and rounded once, to nearest
 *     even, where they are stored.
 */
#define DD_F32 0
#define DD_BF16 1
#define DD_F16 2
#define DD_E4M3 3     /* 8 bits, largest value 448, no infinities (OCP) */
#define DD_I8 4

typedef struct dd_tensors dd_tensors;

/*
 * One tensor of a model: n elements in a row.  grad is required when n > 0.
 * For dd_adam_step, param (the weights the model reads), m and v are required
 * for all tensors of a list or for none, and master for a param of 16 bits
 * (NULL for one of 32).
 */
typedef struct {
    void *grad;           /* grad_type [n] */
    void *param;          /* param_type [n] */
    float *master;        /* [n] f32 weights that a 16-bit param is the rounding of */
    float *m, *v;         /* [n] moments */
    int64_t n;
    int32_t grad_type, param_type;   /* DD_F32, DD_BF16 or DD_F16 */
    int32_t no_decay;     /* 1: weight decay does not apply to this tensor */
    int32_t reserved;     /* 0 */
} dd_tensor;

/*
 * dd_tensors_load -- a list of tensors that is worked on in one launch.
 *   t   host array of `count` tensors (copied).
 * The tensors stay where they are for the life of the handle.  The handle
 * keeps 64 bytes of device memory for every 8,192 elements of a tensor (or
 * fewer), and working memory of 8 KiB for dd_grad_norm and dd_adam_step: their
 * calls on several streams are put in order by the library (so those two are
 * captured into a graph on the stream the list was loaded on, DD_EINVAL on
 * another, and the replays are ordered with other calls on the list by the
 * caller).  A list outlives the graphs that work on it.  Waits for `stream`.
 */
dd_status dd_tensors_load(int32_t count, const dd_tensor *t, void *stream, dd_tensors **out);
void dd_tensors_free(dd_tensors *t);

/*
 * dd_grad_norm -- the norm of all gradients of a list taken as one vector.
 *   d_inv_scale  device float [1] or NULL: 1 / loss scale, u below (NULL: 1).
 *   d_stats      device float [3], written:
 *                [0] norm    u * sqrt(sum of grad^2), summed in 64 bits;
 *                [1] factor  u * min(1, max_norm / norm), what to multiply
 *                            the gradients with; u if max_norm <= 0; 0 if [2];
 *                [2] skip    1 if some gradient is infinite or not a number
 *                            (or the norm is, in 64 bits), else 0.
 */
dd_status dd_grad_norm(const dd_tensors *t, float max_norm, const float *d_inv_scale, float *d_stats,
                       void *stream);

/*
 * dd_grad_clip -- gradients times d_stats[1], rounded to dst's types, into the
 * gradients of dst (which may be src): unscaled and clipped, or zeros where
 * the factor is 0.  Both lists have the same number of tensors and sizes
 * (DD_EMISMATCH); their types and everything but the gradients may differ.
 * Unless dst is src, the memory of the two must not overlap.
 */
dd_status dd_grad_clip(const dd_tensors *src, const dd_tensors *dst, const float *d_stats, void *stream);

/*
 * dd_adam_step -- one step of Adam on every tensor of a list, in place.
 *   d_step       device int64 [1]: steps taken before; one more after the call.
 *   d_stats      as dd_grad_norm wrote it, or NULL: the gradients are
 *                multiplied with [1] as they are read, and nothing changes
 *                (d_step neither) if [2] is not 0.
 *   decoupled    1: weight decay shrinks the weight by lr * weight_decay;
 *                0: it is added to the gradient.
 * With t = d_step + 1, g = grad * factor (+ weight_decay * w if not decoupled):
 *   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *   w = (1 - lr weight_decay) w (if decoupled)
 *   w = w - lr / (1 - beta1^t) * m / (sqrt(v / (1 - beta2^t)) + eps)
 * where w is master if there is one (param becomes its rounding), else param.
 * DD_EINVAL unless lr >= 0, 0 <= beta < 1, eps >= 0 and weight_decay >= 0, all
 * finite, or when the list has no params.
 */
dd_status dd_adam_step(const dd_tensors *t, int64_t *d_step, const float *d_stats, double lr, double beta1,
                       double beta2, double eps, double weight_decay, int32_t decoupled, void *stream);

/*
 * dd_rms_norm -- for every row, with s = x + residual (x alone if residual is
 * NULL), in 32 bits:
 *   rstd = 1 / sqrt(mean of s^2 over the row + eps),   y = s * rstd * weight
 *   out  = y in `type`, or in 8 bits (out_type DD_E4M3 or DD_I8): for the row,
 *          or each group of columns (the last may be shorter),
 *          scale = max(largest |y|, 2^-100) / 448 (/ 127 for DD_I8) and
 *          out = y / scale.  A NaN in a group makes its scale a NaN.
 *   h    = s in `type` (optional).
 * A row is `cols` consecutive elements; rows start `*_stride` elements apart
 * (of an input any stride, 0 included: the same row for all; of an output at
 * least cols).  out (of 16 or 32 bits) and h may each be x or residual
 * themselves, element for element; outputs must not overlap otherwise.
 */
typedef struct {
    int64_t rows, cols;
    int64_t x_stride, residual_stride, h_stride, out_stride;
    const void *x, *residual;    /* type; residual may be NULL */
    const void *weight;          /* weight_type [cols]; NULL: ones */
    void *h, *out;               /* h: type, may be NULL; out: out_type */
    float *scales;               /* [rows][groups] for an output of 8 bits, else NULL */
    float *rstd;                 /* [rows] or NULL */
    int32_t type;                /* DD_F32, DD_BF16 or DD_F16 */
    int32_t weight_type;         /* DD_F32, or type */
    int32_t out_type;            /* type, DD_E4M3 or DD_I8 */
    int32_t group;               /* columns per scale: 0 (a row), 32, 64 or 128 */
    float eps;
    int32_t reserved;            /* 0 */
} dd_rms_norm_args;
dd_status dd_rms_norm(const dd_rms_norm_args *a, void *stream);

/*
 * dd_rms_norm_grad -- from the gradient dy of y: with xh = h * rstd,
 *   dx = (weight dy - xh mean over the row of (weight dy xh)) * rstd + dh
 *   dw = sum over rows of dy xh, rounded to weight_type
 * h and rstd as dd_rms_norm gave them (h is x without a residual), dh the
 * gradient that reaches h on its other ways (NULL: none).  dx is the gradient
 * of x and of residual alike.  An output of 8 bits counts as y.
 * dx may be dy, dh or h themselves (the same stride); otherwise outputs must
 * not overlap inputs.
 *   work   device memory of dd_rms_norm_grad_work(rows, cols) bytes, aligned to
 *          16, which the call overwrites, or NULL: the library takes it from its
 *          cache for the time of the call.  A call with dw that is captured into
 *          a graph needs it (DD_EINVAL): the replays write there too.
 */
typedef struct {
    int64_t rows, cols;
    int64_t dy_stride, h_stride, dh_stride, dx_stride;
    const void *dy, *h, *dh;     /* type; dh may be NULL */
    const void *weight;          /* weight_type [cols]; NULL: ones */
    const float *rstd;           /* [rows] */
    void *dx;                    /* type */
    void *dw;                    /* weight_type [cols], or NULL */
    void *work;
    int32_t type, weight_type;   /* as above */
} dd_rms_norm_grad_args;
dd_status dd_rms_norm_grad(const dd_rms_norm_grad_args *a, void *stream);
size_t dd_rms_norm_grad_work(int64_t rows, int64_t cols);

/* ---------------------------------------------------------------------------
 * The rest of a training iteration between its norms and its weight update:
 * the products of a block with what is fused into them, dropout, and the
 * embedding.  Tensors, streams and rounding as above, and:
 *
 *   - Strides count elements and are those of rows; the elements of a row are
 *     consecutive.  An input's rows may start at any stride (0: the same row
 *     for all), an output's at least a row apart.
 *   - Outputs must not overlap inputs or each other but where it is said.
 *   - work   device memory of the size that the function of that name gives,
 *            aligned to 16, which the call overwrites, or NULL: the library
 *            takes it from its cache for the time of the call.  A call that
 *            needs some and is captured into a graph has to bring it
 *            (DD_EINVAL): the replays write there too.  That size goes by the sizes
 *            alone; where there is a function that ends in _need, it gives what a call
 *            with these strides and addresses uses (work itself is not looked at; 0 if the
 *            call would be refused), which for aligned operands is less.
 */
#define DD_ACT_NONE 0
#define DD_ACT_RELU 1
#define DD_ACT_GELU 2        /* z Phi(z) */
#define DD_ACT_GELU_TANH 3   /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
#define DD_ACT_SILU 4        /* z / (1 + exp(-z)) */
/* At infinities the derivatives are their limits, 0 or 1: a z of 16 bits is infinite where the
 * sum lies beyond its range.  DD_ACT_GELU of -infinity (of a sum in 32 bits) is 0 too, DD_ACT_GELU_TANH
 * and DD_ACT_SILU of it are NaN. */

/*
 * dd_linear -- for rows x [rows][k] and a weight w of k by n, summed in 32 bits:
 *   z = x w + bias,   y = act(z) + residual
 * y and z (what the gradient needs of an activation) are each rounded from
 * these sums.  y may be residual, element for element.
 */
typedef struct {
    int64_t rows, k, n;
    int64_t x_stride, w_stride, residual_stride, y_stride, z_stride;
    const void *x, *w;           /* type; w: [k][n], or [n][k] if turned */
    const void *bias;            /* bias_type [n], or NULL */
    const void *residual;        /* type [rows][n], or NULL */
    void *y, *z;                 /* type [rows][n]; z may be NULL */
    void *work;                  /* dd_linear_work(rows, k, n) bytes, or NULL */
    int32_t type;                /* DD_BF16 or DD_F16 */
    int32_t bias_type;           /* DD_F32, or type */
    int32_t act;                 /* DD_ACT_... */
    int32_t turned;              /* 0 or 1 */
} dd_linear_args;
dd_status dd_linear(const dd_linear_args *a, void *stream);
size_t dd_linear_work(int64_t rows, int64_t k, int64_t n);
size_t dd_linear_need(const dd_linear_args *a);

/*
 * dd_linear_grad -- from the gradient dy [rows][n] of x w + bias (with an
 * activation: what dd_act_grad makes of y's), each optional (NULL: not wanted):
 *   dx = (dy w^T) * act'(in_z)   [rows][k]; in_z: x is act(in_z), and dx the
 *                                gradient of in_z (NULL: that of x)
 *   dw = x^T dy                  laid out as w is (turned or not)
 *   db = sum over rows of dy     in bias_type
 * dw and db of no rows are zeros.  dx may be in_z or x, element for element.
 * Sums over many rows are cut into parts whose sums are joined in order: the same
 * bits on every call that has these sizes, strides and alignments and wants the same.  (Copies
 * of operands are shared where dx and dw are both wanted, and may change how sums are cut.)
 *   work holds these parts and copies of operands whose rows 16 bytes do not divide
 * (in dd_linear too).
 */
typedef struct {
    int64_t rows, k, n;
    int64_t dy_stride, x_stride, w_stride, in_z_stride, dx_stride, dw_stride;
    const void *dy;              /* type [rows][n] */
    const void *x;               /* type [rows][k]; needed for dw */
    const void *w;               /* type, as in dd_linear; needed for dx */
    const void *in_z;            /* type [rows][k], or NULL */
    void *dx, *dw, *db;
    void *work;                  /* dd_linear_grad_work(rows, k, n) bytes, or NULL */
    int32_t type, bias_type, in_act, turned;
} dd_linear_grad_args;
dd_status dd_linear_grad(const dd_linear_grad_args *a, void *stream);
size_t dd_linear_grad_work(int64_t rows, int64_t k, int64_t n);
size_t dd_linear_grad_need(const dd_linear_grad_args *a);

/*
 * dd_act_grad -- dz = dy * act'(z), element by element.  dz may be dy or z.
 */
typedef struct {
    int64_t rows, cols;
    int64_t dy_stride, z_stride, dz_stride;
    const void *dy, *z;
    void *dz;
    int32_t type;                /* DD_F32, DD_BF16 or DD_F16 */
    int32_t act;
} dd_act_grad_args;
dd_status dd_act_grad(const dd_act_grad_args *a, void *stream);

/*
 * dd_dropout -- out = residual + (x / (1 - q) where kept, else 0), with q = p to
 * the nearest 65,536th (halves to even) and the quotient as x times 65536 / (65536
 * - 65536 q), rounded to 32 bits.  The gradient of x is the same call on out's
 * gradient without a residual; no mask is stored.
 *   Element i (row * cols + column) is kept if its number of 16 bits is at least
 * 65536 q: the (i mod 8)-th half, low halves first, of the four words that
 * Philox 4x32-10 (Salmon et al., SC 2011) gives for the counter (low and high
 * word of i / 8, low and high word of c) and the key d_state[0], low word first,
 * where c = d_state[1] + call.  It depends on nothing else: not on strides, types or where
 * the call runs.
 *   d_state   device uint64 [2]: key and counter; read as the work runs, so that
 *             replays of a captured call go on where the caller has moved it to.
 *   d_used    device uint64 [2] or NULL, written: key and c, which with call = 0
 *             give the gradient this mask.  Apart from d_state.
 * out may be x or residual, element for element.  What is dropped counts for
 * nothing, also if it is infinite or not a number.  0 <= p <= 1.
 */
typedef struct {
    int64_t rows, cols;
    int64_t x_stride, residual_stride, out_stride;
    const void *x, *residual;    /* type; residual may be NULL */
    void *out;                   /* type */
    const uint64_t *d_state;
    uint64_t *d_used;
    uint64_t call;
    double p;
    int32_t type;                /* DD_F32, DD_BF16 or DD_F16 */
    int32_t reserved;            /* 0 */
} dd_dropout_args;
dd_status dd_dropout(const dd_dropout_args *a, void *stream);

/*
 * dd_embed -- out[t] = scale * table[ids[t]], for `tokens` rows of cols.  An id
 * that the table does not have (negative, or vocab and more) gives a row of NaNs.
 */
typedef struct {
    int64_t tokens, vocab, cols;
    int64_t table_stride, out_stride;
    const void *ids;             /* int64 or int32 [tokens] */
    const void *table;           /* type [vocab][cols] */
    void *out;                   /* type [tokens][cols] */
    float scale;
    int32_t type;                /* DD_F32, DD_BF16 or DD_F16 */
    int32_t id_bytes;            /* 8 or 4 */
    int32_t reserved;            /* 0 */
} dd_embed_args;
dd_status dd_embed(const dd_embed_args *a, void *stream);

/*
 * dd_embed_grad -- dtable[v] = scale * sum of dy[t] over the tokens with ids[t] =
 * v, for every row of the table (zeros where there is none), each sum taken in 32 bits
 * in the tokens' order, in parts of fixed lengths: the same bits on every call.  Tokens
 * with the id `pad`, and ids that the table does not have, count for nothing.  Fewer
 * than 2^28 tokens (dd_embed too) and 2^29 rows.
 */
typedef struct {
    int64_t tokens, vocab, cols;
    int64_t dy_stride, dtable_stride;
    const void *ids;             /* int64 or int32 [tokens] */
    const void *dy;              /* type [tokens][cols] */
    void *dtable;                /* type [vocab][cols] */
    void *work;                  /* dd_embed_grad_work(tokens, vocab, cols) bytes, or NULL */
    int64_t pad;                 /* -1: none */
    float scale;
    int32_t type, id_bytes;
    int32_t reserved;            /* 0 */
} dd_embed_grad_args;
dd_status dd_embed_grad(const dd_embed_grad_args *a, void *stream);
size_t dd_embed_grad_work(int64_t tokens, int64_t vocab, int64_t cols);

/*
 * dd_release_cache -- wait for all work on the current device, then return
 * every block of the library's device-memory cache for that device to the
 * device (hipFree), and the pinned host buffers (68 KiB each) that ended host
 * threads left.  Memory held by live handles is not touched.  For callers that
 * share the GPU with another allocator (e.g. torch) and need the space.
 */
dd_status dd_release_cache(void);

/* Step (level or phase) of every task: int32 [n], host or device pointer. */
dd_status dd_sched_task_steps(const dd_sched *sched, int32_t *steps_out, void *stream);

/*
 * dd_simulate_plan -- the launch shape dd_simulate_batch takes for these
 * handles, in the terms of dd_simulate_batch_vs: *variants_per_wg = 1, 2, 4,
 * 8 or 16 (one workgroup per strip of that many variants for the whole
 * schedule, one launch; 1 for either kernel that owns one variant) or -1, -2,
 * -4, -8 (the few-variant path, one launch per step).  DD_EINVAL on a NULL
 * argument.
 */
dd_status dd_simulate_plan(const dd_sched *sched, const dd_variants *var,
                           int32_t *variants_per_wg);

/* Schedule shape: steps, thread runs (segments), widest step, gather entries. */
dd_status dd_sched_info(const dd_sched *sched, int64_t *n_steps, int64_t *n_segments,
                        int64_t *max_step_width, int64_t *n_gathers);

void dd_graph_free(dd_graph *g);
void dd_sched_free(dd_sched *s);
void dd_variants_free(dd_variants *v);

const char *dd_status_str(dd_status s);
const char *dd_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* DD_H */
