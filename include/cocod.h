/*
 * libcocod -- one round of CoCoD-SGD (computation and communication decoupled
 * SGD) for W simulated workers resident in one GPU's memory.
 *
 * The round is the body of the while loop of Algorithm 1 of the paper:
 *   Step I   store every worker's model x_t^i and form the weighted mean of the
 *            stored models, x^_t = sum_i p_i x_t^i           (cocod_average_begin)
 *   Step II  k local stochastic-gradient steps on the live model, concurrently
 *            with Step I                                     (cocod_local_steps)
 *   line 6   x_{t+k}^i = x^_t + (x_{t+k}^i - x_t^i)         (cocod_average_end_apply)
 *   line 7   t = t + k                                       (the step counter)
 * The paper's all-reduce between workers is, on one GPU, a reduction over the
 * worker axis on a second stream that overlaps the local steps.
 *
 * Conventions
 *   - plain C ABI; every function returns a cocod_status (0 = ok, < 0 = error)
 *     unless stated otherwise; no exception crosses the boundary.
 *   - "device" pointers are HIP device memory, "host" pointers ordinary memory.
 *   - every call only ENQUEUES work on the caller's streams; nothing waits for
 *     the GPU except cocod_sync, cocod_step_timing_read and cocod_destroy
 *     (cocod_create copies its small tables synchronously).
 *   - the caller owns all large device buffers and both streams; they must
 *     outlive the context.  The context owns its small tables (chunk table, weight and
 *     noise-scale vectors), two events, the MLP work space, the scratch and the pinned
 *     result words of the diagnostics, and the recorded graphs with their step-counter word.
 *   - argument errors are detected before any GPU call is made.
 *   - a context is not thread safe; use it from one host thread at a time.
 */
#ifndef COCOD_H
#define COCOD_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct cocod_ctx cocod_ctx;

typedef enum cocod_status {
    COCOD_OK = 0,
    COCOD_ERR_INVALID = -1,      /* bad argument (null, misaligned, out of range, inconsistent) */
    COCOD_ERR_STATE = -2,        /* call not legal in the current state of the round */
    COCOD_ERR_HIP = -3,          /* a HIP runtime call failed; see cocod_last_error */
    COCOD_ERR_NOMEM = -4,        /* host or device allocation failed */
    COCOD_ERR_UNSUPPORTED = -5   /* valid request this build does not implement */
} cocod_status;

/* Where the stochastic gradient G of Step II comes from. */
typedef enum cocod_grad_kind {
    /* G_j = h_ij (x_j - c_ij) + sigma z(seed, i, t, j): separable quadratic with seeded noise
       standing in for the mini-batch gradient of Step II. */
    COCOD_GRAD_QUADRATIC = 0,
    /* G = gradient of the mean softmax cross-entropy of a two-layer ReLU perceptron on a fresh
       seeded mini-batch per (worker, step): a real mini-batch gradient, dense contractions. */
    COCOD_GRAD_MLP = 1,
    /* G is computed by the caller (a real model's backward pass) and handed to cocod_external_step;
       h, c and the MLP fields are unused. */
    COCOD_GRAD_EXTERNAL = 2
} cocod_grad_kind;

/* How Step I is scheduled relative to Step II (the arithmetic is the same in all of them). */
typedef enum cocod_schedule {
    COCOD_SCHED_OVERLAP = 0,   /* mean on avg_stream, concurrent with the local steps (the paper's scheme); with line
                                  6 inside them, concurrent with all launches but the last, which waits for it: where
                                  that is the only one (see cocod_local_steps_end_apply) nothing runs beside the
                                  mean, and COCOD_SCHED_HEAD or a replayed round spares the hand-overs between streams */
    COCOD_SCHED_SERIAL = 1,    /* mean on compute_stream after the local steps, then line 6 (sequential, as
                                  the paper's Local-SGD timeline) */
    COCOD_SCHED_FUSED = 2,     /* mean and line 6 in one kernel after the local steps */
    COCOD_SCHED_HEAD = 3       /* mean formed inside the first local step of the round, which reads every
                                  stored model anyway: Step I costs one 4/W-byte store per parameter and no
                                  pass of its own; where the round's steps are one launch of
                                  cocod_local_steps_end_apply (k = 1; untimed up to k = 16) the mean,
                                  the steps and line 6 are ONE kernel (built-in quadratic gradient, W <= 131
                                  workers, d < 2^30; whenever the round's first step is not such a step, or one
                                  of several in a launch whose blocks, one for all workers, would leave much of
                                  the chip idle, the mean is formed on compute_stream just before line 6 needs it) */
} cocod_schedule;

enum {
    COCOD_FLAG_DRY_RUN = 1u    /* validate, plan and track state but make no GPU call at all (host tests) */
};

/*
 * Memory layout.  Every per-worker array is worker-major: element e of worker i
 * lives at base[i * stride + e], 0 <= e < padded_d.  A flat model (n_tensors <= 1)
 * has padded_d = d rounded up to 4.  A parameter list of n_tensors tensors is
 * packed in list order, each tensor starting on a 4 KiB boundary (offset multiple
 * of 1024 elements) and the end of the list rounded up to 4; see
 * cocod_plan_layout.  The elements in the gaps are pads: the local step and line 6
 * never touch them, the mean kernels may carry them along, and they never
 * influence real elements (their contents are unspecified).  Any stride that is a
 * multiple of 4 is legal.  For full memory bandwidth choose a multiple of 32
 * elements (every worker's row then starts on a 128-byte line): the plain and line-6
 * steps follow the lines of each row by themselves, the kernels that work on the
 * same columns of all workers (mean, mean + line 6, mean-forming steps) cannot.
 */
typedef struct cocod_config {
    uint32_t struct_size;          /* sizeof(cocod_config); checked */
    uint32_t W;                    /* number of workers N of Algorithm 1, >= 1 */
    uint64_t d;                    /* parameters per worker (sum of tensor sizes), >= 1, < 2^34; and
                                      W * ceil(d / 1024) <= 2^31 - 1 (blocks of one launch; tensors of a
                                      list each round up on their own); the padded extent (every tensor
                                      of a list starts on a 1024-element boundary) must not exceed 2^34 - 1024 */
    uint32_t n_tensors;            /* 0 or 1: one flat vector; else length of tensor_numel */
    uint32_t grad;                 /* cocod_grad_kind */
    const uint64_t *tensor_numel;  /* host, [n_tensors], each >= 1, sum == d; copied */
    uint64_t bucket_bytes;         /* averaging granularity: tensors are grouped, in order, into buckets of
                                      at most this many bytes (a larger tensor gets its own); 0 = one bucket */
    float lr;                      /* gamma */
    float momentum;                /* mu of the experiments' optimizer; 0 = the update of Algorithm 1 */
    float weight_decay;            /* lambda, added to the gradient as lambda x */
    float noise_sigma;             /* sigma of the gradient noise (quadratic kind) */
    uint64_t seed;                 /* key of the counter-based generator */
    const float *weights;          /* host, [W], p_i = M_i / sum M_l, must sum to 1 within 1e-4; NULL = 1/W */
    const float *noise_sigma_w;    /* host, [W], copied; NULL = noise_sigma for every worker.  Heterogeneous
                                      workers (quadratic kind): worker i's mini-batch of M_i samples has
                                      gradient variance sigma^2 / M_i (bounded-variance assumption), so the
                                      caller passes sigma / sqrt(M_i); each finite and >= 0 */
    float *xA;                     /* device [W][stride]: holds the models at create time (the live buffer) */
    float *xB;                     /* device [W][stride]: second model buffer; need not be initialised */
    float *v;                      /* device [W][stride]: momentum buffer, caller-initialised (0 for a fresh
                                      run); may be NULL when momentum == 0 */
    float *mean;                   /* device [stride]: receives x^_t */
    const float *h;                /* device [W][stride]: curvatures (quadratic kind) */
    const float *c;                /* device [W][stride]: centres (quadratic kind) */
    uint64_t stride;               /* elements between consecutive workers; >= padded_d, multiple of 4 */
    void *compute_stream;          /* hipStream_t for Step II and line 6 (NULL = the null stream) */
    void *avg_stream;              /* hipStream_t for Step I; equal to compute_stream = no overlap.
                                      The share of the device that the averaging may occupy (the fraction a% of
                                      the paper's time-speedup analysis) is a property of THIS stream and
                                      therefore the caller's: create it with a compute-unit mask if the
                                      platform allows.  The library offers no field for it: it never creates
                                      streams, and on the machines this was built on the runtime refused
                                      masked streams, so the setting could not be tested. */
    uint32_t mlp_in, mlp_hidden, mlp_out, mlp_batch;   /* MLP kind: layer widths and mini-batch size.  Supported
                                      shapes (else COCOD_ERR_UNSUPPORTED): mlp_in and mlp_batch multiples of 128,
                                      mlp_batch <= 1024, mlp_hidden a multiple of 64, 1 <= mlp_out <= 16,
                                      mlp_hidden * (mlp_out rounded up to odd) <= 32768 */
    uint32_t flags;                /* COCOD_FLAG_* */
} cocod_config;

/*
 * Plan the packed layout of a parameter list (pure host arithmetic, no GPU).
 *   d, n_tensors, tensor_numel, bucket_bytes: as in cocod_config.
 *   padded_d      out: elements per worker including alignment pads.
 *   tensor_offset out, may be NULL: [n_tensors] element offset of each tensor inside a worker.
 *   n_buckets     out, may be NULL.
 *   bucket_begin  out, may be NULL: [n_tensors + 1] capacity; bucket b covers elements
 *                 [bucket_begin[b], bucket_begin[b+1]) of a worker; n_buckets + 1 entries written.
 * Follows the packed-buffer practice of the communication library the paper used
 * (tensor fusion); Algorithm 1 itself treats the model as one vector.
 */
int cocod_plan_layout(uint64_t d, uint32_t n_tensors, const uint64_t *tensor_numel,
                      uint64_t bucket_bytes, uint64_t *padded_d, uint64_t *tensor_offset,
                      uint32_t *n_buckets, uint64_t *bucket_begin);

/*
 * Initialisation of Algorithm 1: validates cfg, plans the layout, builds the
 * device chunk table and creates the events.  xA must already hold x_0^i for
 * every worker (the paper starts all workers from the same point; the library
 * does not require it).  On success *out receives the context (state IDLE,
 * step counter t = 0, live buffer xA).  On failure *out is NULL and
 * cocod_last_error(NULL) describes the reason.
 */
int cocod_create(const cocod_config *cfg, cocod_ctx **out);

/* Waits for both streams, frees what the context owns.  NULL is accepted. */
int cocod_destroy(cocod_ctx *ctx);

/*
 * Step II: enqueue k >= 0 local steps on compute_stream.  Each step computes the
 * stochastic gradient G_t^i at the live model and applies
 *     g = G + lambda x ;  v = mu v + g ;  x = x - gamma v          (mu = 0: x = x - gamma g)
 * and advances the step counter t by one.  Legal in both states; outside a round
 * it is plain local SGD.  The first step after cocod_average_begin reads the
 * stored model and writes the other model buffer, so storing x_t^i costs no copy.
 * The built-in quadratic gradient of a coordinate depends on that coordinate alone, so its k steps are
 * taken up to 16 to a launch, in registers, with the bits of one launch per step (also inside
 * cocod_local_steps_end_apply and cocod_graph_round); while step timing is armed every step of an
 * eager call is a launch of its own (replayed rounds are never timed).  The other gradients need the
 * whole model between two steps.
 */
int cocod_local_steps(cocod_ctx *ctx, int k);

/*
 * Step I: marks the live models as the stored models x_t^i and (OVERLAP schedule)
 * enqueues the weighted mean on avg_stream, ordered after all work already on
 * compute_stream.  IDLE -> AVERAGING; COCOD_ERR_STATE if already averaging.
 */
int cocod_average_begin(cocod_ctx *ctx);

/*
 * Join and line 6: compute_stream waits for the mean and then applies
 * x^i = x^_t + (x^i - x_t^i) to every worker (with zero local steps since begin this
 * leaves every worker at x^_t).  AVERAGING -> IDLE; COCOD_ERR_STATE if not averaging.
 */
int cocod_average_end_apply(cocod_ctx *ctx);

/*
 * Step I and line 6 in ONE pass over the models, with nothing overlapped: the weighted mean of the
 * stored models is formed and x^i = x^_t + (x^i - x_t^i) applied by the same kernel (read x_t^i, read
 * x^i, write x^i: 12 + 4/W bytes per parameter; the mean is still written to `mean`).  This is the
 * sequential timeline that the paper's time-speedup analysis sets against the decoupled one
 * (communication AFTER the k local steps instead of beside them); it exists to measure what the
 * overlap buys.  Whatever schedule is set:
 *   - while a round is open (after cocod_average_begin and any local steps) it closes the round;
 *     if the overlapped schedule has already started the mean on avg_stream, compute_stream first
 *     waits for it (same values, so the result does not change);
 *   - while IDLE it is the blocking average of Local SGD: every worker is set to the weighted mean
 *     of the live models (a round with zero local steps).
 * Same bits as cocod_average_end_apply under any schedule.  Always ends IDLE.
 */
int cocod_average_apply_fused(cocod_ctx *ctx);

/*
 * Step II and line 6 together: k local steps of which the LAST one applies line 6 to the model it
 * has just computed, before storing it (x = x^_t + ((x - gamma v) - x_t^i) in the step kernel's
 * registers), and closes the round.  Same arithmetic, in the same order, as
 * cocod_local_steps(k) followed by cocod_average_end_apply, but the separate pass of line 6 over
 * the models (read x, read x_t, write x) disappears: 8 bytes per parameter less per round, 12 where
 * the round's steps are one launch, which reads the stored models anyway (k = 1, and untimed up to
 * k = 16 with the built-in quadratic gradient).  The join moves in front of the last launch, so the
 * mean overlaps the launches before it only: none of them where the only launch is the last.
 * k = 0 is cocod_average_end_apply.
 * AVERAGING -> IDLE; COCOD_ERR_STATE if no round is open.
 */
int cocod_local_steps_end_apply(cocod_ctx *ctx, int k);

/*
 * Step II with the caller's stochastic gradient: one local step x = x - gamma v,
 * v = mu v + (g + lambda x), with g [W][stride] in device memory in the same packed layout as the
 * models (pads ignored), ordered after the work already on compute_stream; the caller makes sure g
 * is complete on that stream and stays untouched until the step has run.  Advances t by one.  Legal
 * for every gradient kind.  close_round != 0 also applies line 6 inside this step and closes the
 * open round (as cocod_local_steps_end_apply does); COCOD_ERR_STATE if no round is open then.
 * Reads x, v, g and writes x, v: 20 bytes per parameter.
 */
int cocod_external_step(cocod_ctx *ctx, const float *g, int close_round);

/*
 * The same step of Step II with g stored as 16-bit brain floats (the upper 16 bits of an fp32, as
 * mixed-precision training produces): g is [W][stride] 16-bit elements, element (i, j) at
 * g[i * stride + j], device memory, 8-byte aligned.  Each value is widened exactly to fp32 and the
 * step then proceeds as cocod_external_step does.  18 bytes per parameter.  Same state rules and
 * error behaviour.
 */
int cocod_external_step_bf16(cocod_ctx *ctx, const uint16_t *g, int close_round);

/*
 * One whole pass of the while-loop body of Algorithm 1 (Step I and Step II side by side, then line
 * 6 and line 7) replayed from a HIP graph: the same kernels, in the same order and, where the models
 * are large enough for it to pay, on the same two branches, as cocod_average_begin +
 * cocod_local_steps(k) + cocod_average_end_apply (fused_tail == 0)
 * or cocod_average_begin + cocod_local_steps_end_apply(k) (fused_tail != 0), with bit-identical
 * results, but submitted with ONE call instead of one per kernel and event: for small models, where
 * the launches and not the memory traffic bound a round.  The first call for a given (k, fused_tail,
 * schedule, live buffer) records and instantiates the graph (this allocates, and is the only slow
 * call); later calls only launch it on compute_stream.  The averaging branch runs inside the graph,
 * not on avg_stream.  Kernels in the graph read the step counter t from a device word the library
 * owns, so a replay continues the noise stream exactly where eager calls would.  Graph rounds and
 * the eager calls may be mixed freely between rounds.  cocod_set_lr drops the recorded graphs (it
 * then waits for compute_stream).  Launches inside a graph are not seen by cocod_step_timing.
 * Only legal while IDLE (COCOD_ERR_STATE otherwise); k >= 0; needs a built-in gradient when k > 0.
 * compute_stream must be a stream of the caller's own: the null stream cannot be captured, and a
 * context created on it gets COCOD_ERR_INVALID here, before any GPU call.
 */
int cocod_graph_round(cocod_ctx *ctx, int k, int fused_tail);

/* Choose how Step I is scheduled; only legal while IDLE.  Default COCOD_SCHED_OVERLAP. */
int cocod_set_schedule(cocod_ctx *ctx, int schedule);

/* Learning-rate schedules live in the caller: set gamma between steps. */
int cocod_set_lr(cocod_ctx *ctx, float lr);

/* The global step counter t (line 7).  It keys the noise / mini-batch streams, so a run that is
   saved (models, momentum, t) and restored continues bit-identically.  t < 2^32. */
int cocod_get_step(const cocod_ctx *ctx, uint64_t *step);
int cocod_set_step(cocod_ctx *ctx, uint64_t step);

/* Which of xA / xB currently holds the models (device pointer, [W][stride]). */
int cocod_live_model(const cocod_ctx *ctx, float **x_live);

/* 1 while a round is open (between begin and end_apply), else 0; < 0 on error. */
int cocod_is_averaging(const cocod_ctx *ctx);

/* Number of chunks of the step kernel's chunk table and number of buckets (for inspection). */
int cocod_get_plan(const cocod_ctx *ctx, uint64_t *padded_d, uint32_t *n_chunks, uint32_t *n_buckets);

/*
 * Measurement aid.  cocod_step_timing(ctx, n) with n > 0 makes each of the next n local steps a launch
 * of its own that carries the runtime's own start/stop timestamps (events on compute_stream, owned by the
 * context); n = 0 switches it off.  cocod_step_timing_read waits for compute_stream, returns the
 * summed kernel durations and the number of launches measured since the last read, and rearms.
 * It times steps, not the launches that an untimed call makes of them: with the built-in quadratic
 * gradient, whose steps share launches, an armed round moves more bytes than an unarmed one and
 * takes longer.  The duration of an unarmed call is the caller's to take, with events of its own on
 * compute_stream.
 * A local step of the MLP kind is several kernels: its duration runs from the start of the first
 * to the end of the last.
 * Index 0 of both arrays: plain local steps; index 1: steps that carry line 6
 * (cocod_local_steps_end_apply's last step, one that also forms the mean included); index 2: first steps
 * of a round that also form the mean (COCOD_SCHED_HEAD).
 */
int cocod_step_timing(cocod_ctx *ctx, int max_launches);
int cocod_step_timing_read(cocod_ctx *ctx, double total_ms[3], uint32_t launches[3]);

/*
 * Diagnostic: the weighted consensus distance sum_i p_i || x^ - x^i ||^2 of the live models, with
 * x^ = sum_i p_i x^i (the quantity that Lemma 2 of the paper bounds), over the real parameters
 * (alignment pads excluded).  Runs a reduction on compute_stream after the work already queued
 * there, WAITS for it and writes the scalar to *result (host).  The first call allocates a small
 * scratch buffer owned by the context.
 */
int cocod_consensus_distance(cocod_ctx *ctx, double *result);

/*
 * cocod_consensus_distance for callers that cannot allocate device memory: code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation.  Same kernels and same bits, but
 *   - the block partials live in a static device array of the library (2 MiB per GPU, held until the
 *     process ends) instead of a buffer allocated on first use;
 *   - the scalar goes to *result_device, DEVICE memory of the caller (one double, 8-byte aligned);
 *   - the call only enqueues on compute_stream and returns: no wait, no copy, no allocation of any
 *     kind (cocod_create has looked up the array's device address once for its GPU).
 * Limit: at most 2^18 chunks of 1024 parameters per worker (tensors of a list round up each on their
 * own), i.e. d up to 268 M for a flat model; beyond that COCOD_ERR_UNSUPPORTED.  All contexts on one
 * GPU share the array: calls that overlap in time on one GPU (two streams, two threads) race on it and
 * must be ordered by the caller; calls on one stream are ordered by the stream.  Nothing in the array
 * has to be cleared between calls.
 */
int cocod_consensus_distance_noalloc(cocod_ctx *ctx, double *result_device);

/*
 * Diagnostic (quadratic kind only): the objective of the paper's problem definition,
 * f(x) = sum_i p_i f_i(x) with f_i(x) = 1/2 sum_j h_ij (x_j - c_ij)^2, evaluated at the averaged
 * model x^ = sum_i p_i x^i of the live models, and || grad f(x^) ||^2, the quantity whose running
 * mean Theorem 1 bounds.  Real parameters only.  Same scheduling, waiting and scratch behaviour as
 * cocod_consensus_distance; both results are host doubles.  COCOD_ERR_INVALID for other kinds.
 */
int cocod_quadratic_objective(cocod_ctx *ctx, double *f_at_mean, double *grad_norm_sq_at_mean);

/* Block the host until both streams have drained. */
int cocod_sync(cocod_ctx *ctx);

/*
 * Draw the synthetic objective on the device (quadratic kind): fills the buffers
 * behind cfg.h and cfg.c on compute_stream with h_ij = 0.5 + 1.5 U and c_ij ~ N(0,1)
 * from the counter-based generator (streams 1 and 2 of the seed), pads set to 0.
 * For models too large to generate on the host.
 */
int cocod_fill_quadratic(cocod_ctx *ctx);

/*
 * Inspection of the MLP kind's work space after a local step (device pointers owned by the
 * context, valid until cocod_destroy; any output pointer may be NULL):
 *   X [W][batch][mlp_in] last mini-batch, H [W][batch][mlp_hidden] relu output,
 *   dA [W][batch][mlp_hidden] gradient at the hidden pre-activation,
 *   dZ [W][batch][*dz_pitch] gradient at the logits (first mlp_out entries of each row),
 *   y [W][batch] labels.
 * X and y are those of the most recent local step: the context keeps two mini-batch buffers (a step
 * draws the next step's batch into the other one beside its backward product), so the two pointers
 * change from step to step - ask again after each.
 */
int cocod_mlp_workspace(const cocod_ctx *ctx, float **X, float **H, float **dA, float **dZ, int32_t **y,
                        uint32_t *dz_pitch);

/*
 * Generator check: n standard normals of stream `tag` for (worker, step) at flat
 * indices j0 .. j0+n-1, written to device memory `out` on `stream`, produced by the
 * same device routine as the local step's noise (fast = 1) or by the accurate routine
 * used for the objective data (fast = 0).  No context needed.
 */
int cocod_debug_normals(void *stream, uint64_t seed, uint32_t tag, uint32_t worker, uint32_t step,
                        uint64_t j0, uint64_t n, int fast, float *out);

/*
 * Measurement aid: plain streaming copy of n fp32 elements (n multiple of 4, both pointers device,
 * 16-byte aligned, not overlapping) on `stream`.  A kernel of exactly known traffic (4n bytes read,
 * 4n written) against which hardware memory counters are calibrated.  No context needed.
 */
int cocod_debug_copy(void *stream, const float *src, float *dst, uint64_t n);

/*
 * ---- Operators for the caller's own models (COCOD_GRAD_EXTERNAL) -----------------------------------
 *
 * A caller whose gradient comes from a model of its own needs the products, the loss and the stored
 * activations of that model for all W workers at a time.  A group is a worker (or an expert): group g
 * owns the rows offsets[g] .. offsets[g + 1] - 1 of every row-wise array and its own matrix.  Batches may
 * be of any sizes, empty ones included; offsets lie in device memory, so a replayed graph or a router
 * may change them without the host knowing.  Rows in front of offsets[0] and from offsets[groups] on are
 * neither read nor written.  Offsets ought to ascend; entries outside 0 .. rows are taken as the nearer
 * end, and with offsets that do not ascend no access leaves the arrays but the results are undefined.
 *
 * The calls need no context.  Each only enqueues on `stream` (a hipStream_t of any device, NULL = the
 * null stream of the current device), allocates nothing, keeps nothing and may be captured into a graph.
 * The caller's workspace belongs to a call until the stream has passed it: two calls or two graphs that
 * may run at the same time need two.  Descriptions are read during the call.  Arrays are row-major
 * with a pitch ("ld", elements from row to row) of their own; any alignment to whole elements and any
 * pitch work.  16-bit operands that start on 16 bytes, with pitches, group strides and a summed axis that
 * are multiples of 8, are the fast ones; of such a row the whole 16-byte piece that holds its last
 * element is read.  Row-wise arrays may be NULL where rows is 0.  COCOD_ERR_UNSUPPORTED: the result has more tiles than one
 * launch holds (2^32 threads: 2^23 tiles of 128 x 128 or larger, 2^24 of 64 x 64 or of 32 x 64 where groups have few rows, a tile begun per
 * group counted); nothing is then begun.  Outputs must not overlap other arguments: arrays
 * count from their first to their last element, so that one which lies in the gaps of another is refused, too.  Sums are kept in fp32 (fp32 operands are multiplied
 * at fp32 accuracy) and rounded once.
 */
typedef enum cocod_dtype {
    COCOD_F32 = 0,
    COCOD_BF16 = 1,              /* the upper 16 bits of an fp32 */
    COCOD_F16 = 2                /* IEEE half */
} cocod_dtype;

enum {
    COCOD_GROUPED_RELU_OUT = 1u,    /* forward: y = max(x w, 0) */
    COCOD_GROUPED_RELU_IN = 2u      /* x is the output of a relu: the input's gradient is taken through it */
};
enum { COCOD_GROUPED_FORWARD = 0, COCOD_GROUPED_INPUT_GRAD = 1, COCOD_GROUPED_WEIGHT_GRAD = 2 };

/*
 * One linear layer of all groups, y_g = x_g w_g.  A call reads the fields it names; the others are
 * ignored.  w may lie inside the workers' models ([W][stride], w_stride = stride) and dw inside the gradient that
 * cocod_external_step or cocod_external_step_bf16 takes.  The backward calls do not read COCOD_GROUPED_RELU_OUT: the gradient comes
 * through a layer's relu where it is formed, by COCOD_GROUPED_RELU_IN of the layer that follows or by COCOD_CROSS_ENTROPY_RELU_IN of the loss.
 */
typedef struct cocod_grouped {
    uint32_t struct_size;           /* sizeof(cocod_grouped); checked */
    uint32_t dtype;                 /* cocod_dtype of x, w, y, dy, dx */
    uint32_t groups;                /* 1 .. 65535 */
    uint32_t flags;                 /* COCOD_GROUPED_RELU_* */
    uint64_t rows;                  /* rows of x, y, dy, dx in memory, < 2^31; 0 is legal */
    uint32_t inner, outer;          /* columns of x, columns of y; 1 .. 2^30 */
    const int64_t *offsets;         /* device, [groups + 1], 8-byte aligned */
    const void *x;   uint64_t ldx;          /* [rows][inner] */
    const uint8_t *x_codes;  uint64_t ld_codes;    /* where x is NULL: x as cocod_checkpoint_store left it, [rows][inner] */
    const uint8_t *x_scales; uint64_t ld_scales;   /*   and its scales, [rows][ceil(inner / 32)] */
    const void *w;   uint64_t ldw, w_stride;       /* [groups][inner][outer]; w_stride 0: one matrix for all groups */
    void *y;         uint64_t ldy;          /* [rows][outer] */
    const void *dy;  uint64_t lddy;         /* [rows][outer] gradient at x w, in front of the relu that y may have gone through */
    void *dx;        uint64_t lddx;         /* [rows][inner] gradient at x */
    void *dw;        uint64_t lddw, dw_stride;     /* [groups][inner][outer] gradient at w, a matrix of its own for every group */
    uint32_t dw_dtype;              /* dtype, or COCOD_F32 */
    uint32_t reserved;
    void *workspace;                /* device, 16-byte aligned; NULL: long sums of small results are not split over the chip */
    uint64_t workspace_bytes;
} cocod_grouped;

/* Bytes of workspace with which the call of this direction splits its sums (0: it would not); reads the sizes and checks the address of offsets, no other. */
int cocod_grouped_workspace(const cocod_grouped *g, int direction, uint64_t *bytes);
/* y_g = x_g w_g, through a relu with COCOD_GROUPED_RELU_OUT (a NaN stays one). */
int cocod_grouped_forward(void *stream, const cocod_grouped *g);
/* dx_g = dy_g w_g^T; with COCOD_GROUPED_RELU_IN zero where x (x NULL: its codes) is not above zero. */
int cocod_grouped_input_grad(void *stream, const cocod_grouped *g);
/* dw_g = x_g^T dy_g (x NULL: the product takes the codes and scales as they are); zero for a group without rows. */
int cocod_grouped_weight_grad(void *stream, const cocod_grouped *g);

enum {
    COCOD_CROSS_ENTROPY_SUM = 1u,       /* a group's loss is the sum of its rows' losses, not their mean */
    COCOD_CROSS_ENTROPY_RELU_IN = 4u    /* h is the output of a relu: dh is taken through it (zero where h is not above zero) */
};

/*
 * Softmax cross-entropy of logits h_g e_g^T over a vocabulary, without the logits in memory, and the gradients of
 * grad_scale * (loss of the group).  A row whose target is not in 0 .. vocab - 1 has none: its loss and its
 * row of dh are zero, it does not count in the mean, and nothing of its h is used.  A group without
 * targets has loss 0 and gradient 0.  16-bit types: the slopes at the logits are rounded to the type before the products (bf16: by up to
 * 2^-8 + 2^-11 of themselves, fp16: 2^-11, not below steps of 2^-38), so an entry of dh or de is off by up to that part of the sum of its
 * products' magnitudes, beside its own rounding; near a minimum, where they cancel, that may be much of the entry.  COCOD_F32 keeps the slopes in fp32.
 */
typedef struct cocod_cross_entropy_call {
    uint32_t struct_size;           /* sizeof(cocod_cross_entropy_call); checked */
    uint32_t dtype;                 /* cocod_dtype of h, e, dh, de */
    uint32_t groups;                /* 1 .. 65535 */
    uint32_t flags;                 /* COCOD_CROSS_ENTROPY_* */
    uint64_t rows;                  /* < 2^26; 0 is legal */
    uint32_t dim, vocab;            /* 1 .. 2^30 */
    const int64_t *offsets;         /* device, [groups + 1], 8-byte aligned */
    const void *h;   uint64_t ldh;              /* [rows][dim] hidden states */
    const void *e;   uint64_t lde, e_stride;    /* [groups][vocab][dim]; e_stride 0: one table for all groups */
    const int32_t *targets;         /* device, [rows] */
    float *loss;                    /* device, [rows] */
    float *group_loss;              /* device, [groups]; may be NULL */
    void *dh;        uint64_t lddh;             /* [rows][dim]; NULL: not wanted */
    void *de;        uint64_t ldde, de_stride;  /* [groups][vocab][dim], a table of its own for every group; NULL: not wanted */
    float grad_scale;               /* finite */
    uint32_t piece;                 /* vocabulary entries whose slopes are in memory at a time, rounded down to a multiple of 256 (at least
                                       256); 0: as many as make 2^28 values */
    void *workspace;                /* device, 256-byte aligned */
    uint64_t workspace_bytes;
} cocod_cross_entropy_call;

/* Bytes of workspace that the call needs; reads the sizes, piece, and whether dh and de are NULL. */
int cocod_cross_entropy_workspace(const cocod_cross_entropy_call *c, uint64_t *bytes);
int cocod_cross_entropy(void *stream, const cocod_cross_entropy_call *c);

enum {
    COCOD_TOKEN_SCORES_RELU_IN = 1u         /* h is the output of a relu: dh is taken through it (zero where h is not above zero) */
};
enum { COCOD_TOKEN_SCORES_FORWARD = 0, COCOD_TOKEN_SCORES_GRAD = 1 };

/*
 * Log probabilities of given tokens, entropies and the most probable alternatives, with logits z = scale * h_g e_g^T over a vocabulary that are not kept:
 *   logp[r] = log softmax(z_r)[targets[r]],  entropy[r] = - sum over v of p_rv log p_rv  (an entry with p = 0 counts as 0),
 *   top_ids[r][j], top_logp[r][j]: the entry with the j-th largest logit (of equal ones the lowest index first) and its log probability; -1 and minus
 *   infinity behind the last entry of a vocabulary with fewer.
 * targets NULL: every row takes part, without logp.  Otherwise a row whose target is not in 0 .. vocab - 1 takes no part: its logp and entropy
 * are 0, its alternatives -1 and minus infinity, its row of dh is 0, and nothing of its h is used.  Entries whose logits differ by less than the roundings of their
 * sums may change places, and the log probability of an alternative may differ from logp of the same entry by as much.  A NaN logit counts as minus
 * infinity among the alternatives, and makes the log probabilities and the entropy of its row NaN.
 *
 * The gradient is that of sum over r of d_logp[r] logp[r] + d_entropy[r] entropy[r]; the call reads norms as the forward call of the same h, e, scale and targets left
 * them (and offsets, h, e, targets, scale).  A row where both slopes are 0 takes no part.  16-bit types: the slopes at the logits are rounded to the type before the products
 * (bf16: by up to 2^-8 of themselves, fp16: 2^-11, not below 2^-38 of the group's largest |d_logp| + 32 |d_entropy|), so an entry of dh is off by up to that part of the sum
 * of its products' magnitudes, beside its own rounding.  For de a row of h is taken times a number of its own and rounded as well (fp16: not below 2^-39 of the largest finite
 * |h| in the group's rows that take part), so an entry of de is off by up to twice that part.  COCOD_F32 keeps both in fp32.  A group without rows that take part has gradient 0.
 */
typedef struct cocod_token_scores_call {
    uint32_t struct_size;           /* sizeof(cocod_token_scores_call); checked */
    uint32_t dtype;                 /* cocod_dtype of h, e, dh, de */
    uint32_t groups;                /* 1 .. 65535 */
    uint32_t flags;                 /* COCOD_TOKEN_SCORES_* */
    uint64_t rows;                  /* < 2^26; 0 is legal */
    uint32_t dim, vocab;            /* 1 .. 2^30 */
    const int64_t *offsets;         /* device, [groups + 1], 8-byte aligned */
    const void *h;   uint64_t ldh;              /* [rows][dim] hidden states */
    const void *e;   uint64_t lde, e_stride;    /* [groups][vocab][dim]; e_stride 0: one table for all groups */
    const int32_t *targets;         /* device, [rows]; may be NULL */
    float scale;                    /* of the logits (1 / temperature), finite, > 0 */
    uint32_t top;                   /* alternatives of a row, 0 .. 32 */
    float *logp, *entropy;          /* device, [rows]; NULL: not wanted */
    int32_t *top_ids;               /* device, [rows][top] */
    float *top_logp;                /* device, [rows][top] */
    uint64_t ld_top;                /* of both */
    float *norms;                   /* device, [rows][4], 16-byte aligned: written forward (NULL: not wanted), read by the gradient */
    const float *d_logp, *d_entropy;            /* device, [rows]; NULL: 0 */
    void *dh;        uint64_t lddh;             /* [rows][dim]; NULL: not wanted */
    void *de;        uint64_t ldde, de_stride;  /* [groups][vocab][dim], a table of its own for every group; NULL: not wanted */
    uint32_t piece;                 /* gradient: vocabulary entries whose slopes are in memory at a time, as in cocod_cross_entropy_call */
    uint32_t reserved;
    void *workspace;                /* device, 256-byte aligned */
    uint64_t workspace_bytes;
} cocod_token_scores_call;

/* Bytes of workspace that the call of this direction needs; reads dtype, groups and sizes, top, piece, and whether dh and de are NULL.  Forward: for every row one of dim elements,
   16 bytes for every 128 entries of the vocabulary (64 where rows are few), with alternatives vocab + 8 top bytes more, and a little.  Gradient: for every row one of dim
   elements (16-bit types with de: two) and one of `piece` elements, with several pieces and dh one of dim floats; partial sums; and a little. */
int cocod_token_scores_workspace(const cocod_token_scores_call *c, int direction, uint64_t *bytes);
int cocod_token_scores(void *stream, const cocod_token_scores_call *c);
int cocod_token_scores_grad(void *stream, const cocod_token_scores_call *c);

/*
 * Activations in 8 bits from the forward to the backward pass.  32 consecutive values of a row (the last ones of a
 * row may be fewer) share a scale 2^e, stored as e + 127: the smallest power of two, not below 2^-117 (COCOD_F16: 2^-15), for
 * which their largest finite magnitude is at most 448 * 2^e.  A value is stored as the e4m3 code (1 + 4 + 3
 * bits, bias 7, no infinities) nearest to value / 2^e, ties to the even code; what is not zero becomes no
 * zero but at least the smallest code; magnitudes above 1.875 * 2^127 (COCOD_F16: 1.875 * 2^15) are stored as that;
 * infinities and NaN become NaN and do not count for the scale.  Every stored value is a value of the
 * type it came from, so load is exact.  The codes of a row are followed by nothing: pitches may be any.
 */
int cocod_checkpoint_store(void *stream, int dtype, uint64_t rows, uint64_t cols, const void *x, uint64_t ldx,
                           uint8_t *codes, uint64_t ld_codes, uint8_t *scales, uint64_t ld_scales);
int cocod_checkpoint_load(void *stream, int dtype, uint64_t rows, uint64_t cols, const uint8_t *codes, uint64_t ld_codes,
                          const uint8_t *scales, uint64_t ld_scales, void *x, uint64_t ldx);

/*
 * Tokens (rows of x) to the rows of the groups that own them, the ragged batches of the calls above, and back.  Every token has `choices`
 * choices of a group; pair (t, j) is token t's j-th.  cocod_route_sort gives every pair a row: pairs in the order of group, token and choice.
 * A pair whose choice is not in 0 .. groups - 1 has no row, nor has one that finds `capacity` pairs of its group in front of it: place is
 * -1, the pair takes no part, nothing of its weight is used and its dweights is 0.  A token may choose a group more than once.  The other
 * calls read place (entries outside 0 .. tokens * choices - 1 count as -1) and so also serve a caller who sorts by other means; rows that
 * no pair has are neither read nor written.  Two pairs with one row: no access leaves the arrays, but the results are undefined.
 * Sums are kept in fp32, over the choices in their order, and rounded once.
 */
typedef struct cocod_route {
    uint32_t struct_size;           /* sizeof(cocod_route); checked */
    uint32_t dtype;                 /* cocod_dtype of x, xs, ys, y, dy, dys, dxs, dx (to cocod_route_sort any of them is the same) */
    uint32_t groups;                /* 1 .. 65535 */
    uint32_t choices;               /* 1 .. 64 */
    uint64_t tokens;                /* tokens * choices < 2^31; 0 is legal */
    uint64_t capacity;              /* rows that a group takes at most; 0: as many as come (the calls but cocod_route_sort do not read it) */
    uint32_t width;                 /* columns of the rows, 1 .. 2^30 (cocod_route_sort does not read it) */
    uint32_t flags;                 /* 0 */
    const int32_t *experts; uint64_t ld_experts;   /* [tokens][choices] groups chosen */
    int32_t *place;  uint64_t ld_place;     /* [tokens][choices] written by cocod_route_sort, read by the others */
    int64_t *offsets;               /* [groups + 1], 8-byte aligned, written by cocod_route_sort */
    const float *weights; uint64_t ld_weights;     /* [tokens][choices]; NULL: 1 */
    const void *x;   uint64_t ldx;          /* [tokens][width] */
    void *xs;        uint64_t ldxs;         /* [tokens * choices][width], as the other row-wise arrays of the groups: ys, dys, dxs */
    const void *ys;  uint64_t ldys;
    void *y;         uint64_t ldy;          /* [tokens][width] */
    const void *dy;  uint64_t lddy;         /* [tokens][width] gradient at y */
    void *dys;       uint64_t lddys;        /* gradient at ys; NULL: not wanted */
    float *dweights; uint64_t ld_dweights;  /* [tokens][choices] gradient at weights; NULL: not wanted, ys is not read */
    const void *dxs; uint64_t lddxs;        /* gradient at xs */
    void *dx;        uint64_t lddx;         /* [tokens][width] gradient at x */
    void *workspace;                /* cocod_route_sort: device, 16-byte aligned; may be NULL where none is needed */
    uint64_t workspace_bytes;
} cocod_route;

/* Bytes of workspace that cocod_route_sort needs (0 for small batches); reads tokens, choices and groups. */
int cocod_route_workspace(const cocod_route *r, uint64_t *bytes);
/* place and offsets from experts. */
int cocod_route_sort(void *stream, const cocod_route *r);
/* xs[place[t][j]] = x[t] */
int cocod_route_dispatch(void *stream, const cocod_route *r);
/* dx[t] = sum over j of dxs[place[t][j]] */
int cocod_route_dispatch_grad(void *stream, const cocod_route *r);
/* y[t] = sum over j of weights[t][j] * ys[place[t][j]] */
int cocod_route_combine(void *stream, const cocod_route *r);
/* dys[place[t][j]] = weights[t][j] * dy[t],  dweights[t][j] = <dy[t], ys[place[t][j]]> */
int cocod_route_combine_grad(void *stream, const cocod_route *r);

enum {
    COCOD_ADAMW_STATE_F32 = 0,      /* m and v as fp32 */
    COCOD_ADAMW_STATE_8BIT = 1      /* m and the square root of v as 8-bit codes with a scale for every 32 */
};

/* What changes from step to step. */
typedef struct cocod_adamw_now {
    float lr, grad_scale;
    float bias1, bias2;             /* 1 - beta1^step, 1 - beta2^step */
    uint32_t seed;
    uint32_t skip;                  /* not 0: the step leaves everything as it is (gradients that overflowed) */
    uint32_t reserved[2];
} cocod_adamw_now;

/*
 * A tensor of worker 0; worker i's arrays lie i * stride elements behind (scales: i * stride / 32).  8-bit states: 32 consecutive elements
 * of the tensor share a scale, its last ones may be fewer; m_scales and v_scales hold ceil(n / 32).  All zero codes and scales are zero states.
 */
typedef struct cocod_adamw_tensor {
    uint64_t n;                     /* elements, up to 2^40; 0: nothing is done */
    void *p;                        /* parameters, in place */
    const void *g;                  /* gradient */
    void *m, *v;                    /* states, in place: float, or uint8_t codes */
    uint8_t *m_scales, *v_scales;
    void *copy;                     /* NULL, or the new parameters once more, rounded to copy_dtype (dtype COCOD_F32 only) */
    float weight_decay;
    float lr_scale;                 /* the tensor's learning rate is lr * lr_scale */
} cocod_adamw_tensor;

/*
 * One AdamW step of all workers:  g' = grad_scale g,  m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2,
 * p = p (1 - lr weight_decay) - lr (m / bias1) / (sqrt(v / bias2) + eps).  p, m and v go through fp32; p (and copy) are rounded to nearest.
 * It stands in the place of cocod_external_step for callers whose local step is AdamW: on the live model of an idle context, with
 * cocod_average_apply_fused after k of them.
 *
 * 8-bit states are kept as cocod_checkpoint_store keeps activations (cocod_checkpoint_load with one row of n columns, fp32, reads m, and the root of v; the
 * smallest scale is 2^-117 for m, 2^-51 for the root), but rounded up or down by chance, so that the stored m and the square of
 * the stored root are the new m and v in the mean: by 16 random bits each that depend on (seed, number of the tensor, worker,
 * element) alone.  The caller gives every step another seed.  A root that is not zero is not stored as zero.  The new p comes from
 * m and v before they are rounded.  A state that is not finite is stored as NaN and does not count for the scale.
 * Arrays may begin at any element.  The arrays of a call must not overlap each other; within a tensor and a worker that is checked.
 * A launch takes up to 55 (8-bit states with copies) .. 64 tensors with up to 16 pairs of weight_decay and lr_scale; the next one begins behind them, and
 * behind a tensor without elements between others.
 */
typedef struct cocod_adamw_call {
    uint32_t struct_size;           /* sizeof(cocod_adamw_call); checked */
    uint32_t dtype, grad_dtype, copy_dtype;       /* cocod_dtype of p, g, copy */
    uint32_t state;                 /* COCOD_ADAMW_STATE_* */
    uint32_t flags;                 /* 0 */
    uint32_t workers;               /* 1 .. 65535 */
    uint32_t seed;
    uint64_t stride;                /* elements from worker to worker, of all arrays; a multiple of 32 for 8-bit states; not read with one worker */
    const cocod_adamw_tensor *tensors;            /* HOST memory, read during the call (a captured call keeps what it says) */
    uint64_t count;                 /* of tensors, up to 2^20 */
    float lr, beta1, beta2, eps;    /* betas in 0 .. 1, 1 excluded; eps 0 or at least 2^-126 */
    float grad_scale;               /* gradients are multiplied by it */
    uint32_t reserved;
    uint64_t step;                  /* the number of this step, from 1 */
    const cocod_adamw_now *now;     /* device, 4-byte aligned; not NULL: read by the kernels in place of lr, grad_scale, step and seed, for steps
                                       that are replayed from a graph or decided on the device */
} cocod_adamw_call;

/* Fills *now (host memory) from lr, grad_scale, betas, step and seed of the call. */
int cocod_adamw_now_of(const cocod_adamw_call *c, cocod_adamw_now *now);
int cocod_adamw(void *stream, const cocod_adamw_call *c);

/*
 * For tests: how the products of a call would run.  Makes no GPU call and reads no memory that the description points to.  Of the loss: the logits'
 * statistics, the slopes, the gradients of the hidden states and of the table (splits 0: no such product).  Of the token scores: the logits' statistics
 * alone, or the slopes and the two gradients, by direction.
 */
typedef struct cocod_product_plan {
    uint32_t tile;                  /* of the result: 0 256x256, 1 128x128, 2 32x64, 3 128x128 with four slices in flight, 4 192x128, 5 64x64 */
    uint32_t splits;                /* of the sums */
    uint32_t operands;              /* 0: both go to LDS directly, 1: through registers, 2: the first one is codes, 3: both directly, the second past the caches */
} cocod_product_plan;
int cocod_debug_grouped_plan(const cocod_grouped *g, int direction, cocod_product_plan *out);
int cocod_debug_cross_entropy_plan(const cocod_cross_entropy_call *c, cocod_product_plan out[4], uint32_t *pieces);
int cocod_debug_token_scores_plan(const cocod_token_scores_call *c, int direction, cocod_product_plan out[3], uint32_t *pieces);

/* Last error text of ctx, or of the last failed cocod_create / context-free call when ctx is NULL.
   Never NULL; owned by the library; valid until the next call on the same context / thread. */
const char *cocod_last_error(const cocod_ctx *ctx);

/* Library version, major * 1000 + minor. */
int cocod_version(void);

#ifdef __cplusplus
}
#endif
#endif /* COCOD_H */
