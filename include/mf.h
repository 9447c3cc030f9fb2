/*
 * mf.h -- C ABI of the GB300 MeanField joint-configuration scorer.
 *
 * The library scores joint co-location configurations of N models that share
 * one GPU, following arXiv 2609.02109:
 *   - the joint space Lambda = prod_i Lambda_i of per-model option sets (Sec. II, Eq. 1),
 *     enumerated as a mixed-radix index, last model fastest;
 *   - the aggregate GPU state of a candidate (summed SM share, VRAM and bandwidth
 *     demand of the chosen options, plus N) (Eq. 2, in the coupled reading where the
 *     aggregate is formed from the candidate's own demands);
 *   - one MeanField predictor per model, (thr_i, lat_i) = g_i(local_i, aggregate)
 *     (Sec. III-B, Eq. 6): an MLP Linear-ReLU-[Linear-ReLU]-Linear with an optional
 *     sigmoid on the two outputs;
 *   - the hard constraints sum_i VRAM_i <= R and lat_i <= SLA_i (Eq. 4), infeasible
 *     candidates scoring -inf (Sec. II);
 *   - the objective J = sum_i w_i thr_i (the throughput-weighted term of Eq. 3), or,
 *     with MF_OBJ_SOFT_LAT, J = sum_i w_i thr_i - lambda sum_i max(0, lat_i - SLA_i)
 *     with only the VRAM constraint hard;
 *   - exhaustive argmax / top-k / feasible count over Lambda (Sec. II, Sec. IV-C), and
 *     the GA scheduler's per-generation fitness batch and operators (Sec. IV-C).
 *
 * Conventions for every call:
 *   - Functions return an mf_status and never abort or throw.  mf_last_error()
 *     returns a human-readable detail string for the calling thread's last failure.
 *   - "d_" pointers are device pointers owned by the caller; they must stay valid
 *     until the work on `stream` completes.  `stream` is a cudaStream_t (NULL =
 *     the legacy default stream).  Host pointers are caller-owned too.
 *   - A context is thread-compatible: calls on one context must not run
 *     concurrently from several host threads.  Different contexts are independent.
 *   - Indices are uint64; digits/genes are int32 with 0 <= o_i < K_i.
 *   - The total order of results is (J descending, index ascending).  Infeasible
 *     candidates have J = -INFINITY and never enter a top-k.  Unfilled top-k slots
 *     are (UINT64_MAX, -INFINITY).  No feasible candidate is not an error.
 *   - A candidate whose J is NaN counts as infeasible.
 */
#ifndef MF_H
#define MF_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  MF_OK = 0,
  MF_EINVAL = 1,        /* invalid argument (see each call) */
  MF_ENOMEM = 2,        /* device or host allocation failed */
  MF_ECUDA = 3,         /* a CUDA runtime call failed; see mf_last_error() */
  MF_EUNSUPPORTED = 4,  /* valid but unsupported shape/precision combination */
  MF_ETIMEOUT = 5,      /* a bounded device-side wait gave up */
  MF_EDEVICE = 6        /* the device reported an invalid input (e.g. an index >= |Lambda|) */
} mf_status;

/* MF_FP32: fp32 results (scores within 1e-5 of the fp64 definition).  For the
 * d_L 8, 12 -> 64 -> 64 -> 2 predictor shape (up to 8 models) the scoring runs on the
 * tensor cores with every operand split into two tf32 parts (hi.hi + hi.lo + lo.hi,
 * about 22 bits per product, fp32 accumulation); other shapes run on the CUDA cores.
 * MF_FP32_SIMT: the same results on the CUDA cores for every shape.
 * MF_BF16: bf16 tensor-core scoring, search results re-scored in fp32. */
typedef enum { MF_FP32 = 0, MF_BF16 = 1, MF_FP32_SIMT = 2 } mf_precision;
/* MF_OBJ_UTILITY (Eq. 3 utility with floors) is set with mf_set_utility only. */
typedef enum { MF_OBJ_WEIGHTED_THR = 0, MF_OBJ_SOFT_LAT = 1, MF_OBJ_UTILITY = 2 } mf_objective;
typedef enum { MF_ACT_IDENTITY = 0, MF_ACT_SIGMOID = 1 } mf_out_act;

#define MF_MAX_MODELS 16
#define MF_MAX_OPTIONS 255
#define MF_MAX_D_LOCAL 28
#define MF_MAX_HIDDEN 256
#define MF_MAX_TOPK 1024

typedef struct mf_ctx mf_ctx;

/* Problem description (Sec. II and Sec. III-B).  All arrays are host memory and
 * are deep-copied by mf_create; the caller may free them afterwards. */
typedef struct {
  int32_t n_models;            /* N, 1..MF_MAX_MODELS */
  const int32_t *n_options;    /* [N] K_i = |Lambda_i|, each 1..MF_MAX_OPTIONS */
  int32_t d_local;             /* d_L, 1..MF_MAX_D_LOCAL; predictor input d_in = d_L + 4 */
  int32_t hidden1;             /* first hidden width, 1..MF_MAX_HIDDEN */
  int32_t hidden2;             /* second hidden width, 0 (one hidden layer) or 1..MF_MAX_HIDDEN */
  const float *local_feats;    /* [sum K_i][d_L] row-major, model-major option rows */
  const float *demand;         /* [sum K_i][3]: SM share, VRAM GB, bandwidth GB/s */
  const float *weights;        /* per model, PyTorch Linear layout (weight[out][in]):
                                  W1[h1][d_in], b1[h1], (W2[h2][h1], b2[h2]), W3[2][h], b3[2];
                                  output 0 = throughput, output 1 = latency */
  const float *agg_scale;      /* [4] multipliers of (sum SM, sum VRAM, sum BW, N) before the
                                  predictor; NULL = (1/(0.6N), 1/(20N), 1/(1500N), 1/8) */
  const float *sla;            /* [N] latency ceilings SLA_i */
  const float *obj_w;          /* [N] objective weights w_i */
  float vram_cap;              /* R, GB; feasibility needs sum VRAM <= R */
  float soft_penalty;          /* lambda of MF_OBJ_SOFT_LAT (ignored otherwise) */
  int32_t out_act;             /* mf_out_act */
  int32_t objective;           /* mf_objective */
  int32_t precision;           /* mf_precision of the scoring kernels */
  int32_t device;              /* CUDA device ordinal, or -1 for the current device */
} mf_problem;

/* Result of an exhaustive search.  topk_idx/topk_score are caller-owned host
 * arrays of k entries (either may be NULL). */
typedef struct {
  uint64_t best_idx;           /* UINT64_MAX if no feasible candidate */
  float best_score;            /* -INFINITY if no feasible candidate */
  uint64_t feasible_count;
  int32_t k;
  uint64_t *topk_idx;
  float *topk_score;
} mf_result;

/* GA parameters (Sec. IV-C): population, generations, tournament size, per-gene
 * mutation probability, elitism (0 or 1).  Crossover is uniform. */
typedef struct {
  int32_t pop;                 /* 2..65536 */
  int32_t gens;                /* >= 1 fitness evaluations */
  int32_t tournament;          /* 1..256 */
  double mutation_p;           /* [0, 1] */
  int32_t elitism;             /* 0 or 1 */
} mf_ga_params;

/* Instrumentation of the last calls on a context (host-side bookkeeping plus
 * stamps of the device's nanosecond timer; no extra synchronisation). */
typedef struct {
  uint64_t h2d_bytes_create;   /* bytes mf_create copied host -> device */
  uint64_t d2h_bytes_last;     /* bytes the last synchronous call copied device -> host */
  int32_t kernel_launches_last;/* library kernels launched by the last search / GA run */
  int32_t score_launches_last; /* of which scoring launches (one per chunk) */
  float score_ms_last;         /* device time from the first to the end of the last scoring
                                  launch of the last search */
  float total_ms_last;         /* device time of the whole last search (scoring, merge,
                                  re-scoring, result copy) */
  int32_t scoring_path;        /* the context's scoring kernels: 0 fp32 on the CUDA cores,
                                  1 bf16 tensor cores, 2 fp32 tensor cores (3-term split) */
} mf_stats;

/* Name of a status code (static string). */
const char *mf_status_string(mf_status s);

/* Detail of the calling thread's last failing call ("" if none). */
const char *mf_last_error(void);

/* Validate `p` (Sec. II problem statement), copy it to the device and prepare
 * the kernels.  MF_EINVAL: N, K_i, d_L or widths out of range, NULL arrays, or
 * prod K_i overflowing uint64.  MF_EUNSUPPORTED: MF_BF16 with a shape the
 * tensor-core kernel does not cover.  On success *out owns device memory until
 * mf_destroy. */
mf_status mf_create(const mf_problem *p, mf_ctx **out);

/* Release the context and its device memory (synchronises the device first).
 * NULL is accepted. */
mf_status mf_destroy(mf_ctx *ctx);

/* |Lambda| = prod_i K_i (Eq. 1). */
mf_status mf_space_size(const mf_ctx *ctx, uint64_t *out);

/* Replace SLA_i and w_i (a new scheduling scenario); NULL keeps the old array.
 * Takes effect for calls issued afterwards. */
mf_status mf_set_objective(mf_ctx *ctx, const float *sla, const float *obj_w);

/* Score n candidates given by index (Eqs. 1-6 and the constraints of Eq. 4).
 *   d_idx      [n] uint64 indices into Lambda
 *   d_score    [n] J (or -INFINITY when infeasible)
 *   d_feasible [n] 1 feasible / 0 not (may be NULL)
 *   d_pred     [n][N][2] (thr_i, lat_i) per model (may be NULL)
 * Asynchronous on `stream`.  An index >= |Lambda| scores -INFINITY, infeasible,
 * and raises the context's device status, read by mf_check_device_status. */
mf_status mf_score_batch(mf_ctx *ctx, const uint64_t *d_idx, uint64_t n, float *d_score,
                         uint8_t *d_feasible, float *d_pred, void *stream);

/* Exhaustive surrogate search over [lo, hi) of Lambda (the argmax of Sec. II,
 * extended to top-k and the feasible count), processed in launches of `chunk`
 * candidates (0 = the library's default) while the running top-k and count are
 * carried across launches.  k in 1..MF_MAX_TOPK.  Synchronous: returns after
 * `out` is filled.  The BF16 precision keeps a shortlist of max(8k, 256)
 * candidates by tensor-core score and re-scores it in fp32, so reported scores
 * and the top-k order are the fp32 ones; its feasible count is taken at bf16
 * precision. */
mf_status mf_search_range(mf_ctx *ctx, uint64_t lo, uint64_t hi, int32_t k, uint64_t chunk,
                          mf_result *out, void *stream);

/* mf_search_range over the whole space [0, |Lambda|). */
mf_status mf_search_exhaustive(mf_ctx *ctx, int32_t k, uint64_t chunk, mf_result *out,
                               void *stream);

/* GA fitness batch (Sec. IV-C): d_pop [P][N] int32 genes -> d_fitness [P] (J or
 * -INFINITY).  Asynchronous.  A gene outside [0, K_i) gives -INFINITY and raises
 * the device status. */
mf_status mf_ga_generation(mf_ctx *ctx, const int32_t *d_pop, int32_t P, float *d_fitness,
                           void *stream);

/* Initial population: gene i of slot c is uniform on [0, K_i) from the
 * counter-based generator (seed, generation 0, c, purpose 0, i).  Asynchronous. */
mf_status mf_ga_init(mf_ctx *ctx, const mf_ga_params *g, uint64_t seed, int32_t *d_pop,
                     void *stream);

/* One GA generation (Sec. IV-C operators): from population `gen` and its
 * fitness to population gen + 1.  Slot 0 keeps the fittest individual (lowest
 * slot among equals) when elitism is on; every other slot draws two parents by
 * tournament (draws with replacement, best fitness, lowest slot among equals),
 * takes each gene from either parent with probability 1/2, and redraws a gene
 * uniformly with probability mutation_p.  All draws are SplitMix64 outputs at
 * counter (gen + 1) << 32 | slot << 12 | purpose << 8 | j of the stream `seed`.
 * Asynchronous.  d_next must not alias d_pop. */
mf_status mf_ga_step(mf_ctx *ctx, const mf_ga_params *g, uint64_t seed, int32_t gen,
                     const int32_t *d_pop, const float *d_fitness, int32_t *d_next,
                     void *stream);

/* A complete GA decision: init, then g->gens fitness batches with a generation
 * step between consecutive ones; returns the fittest individual of the last
 * population (lowest slot among equals) in best_genome[N] (host) and its
 * fitness.  Synchronous.  The operators and random draws are those of
 * mf_ga_init / mf_ga_step.  For fp32 predictors with d_L = 8, h1 = h2 = 64,
 * N <= 8 and pop <= 8 x the SM count, the whole decision runs as one
 * cooperative kernel (mf_stats.kernel_launches_last = 1); otherwise as one CUDA
 * graph of init, fitness and step kernels.  MF_ETIMEOUT if the cooperative
 * kernel's grid barrier gave up waiting (the result is then not valid). */
mf_status mf_ga_run(mf_ctx *ctx, const mf_ga_params *g, uint64_t seed, int32_t *best_genome,
                    float *best_fitness, void *stream);

/* ---------------------------------------------------------------------------
 * Fixed-context mode (Sec. III-B): the observed GPU state s_t is held fixed during
 * the search, so predictor i sees its own option and the observed state only, and
 * the utility of Eq. 3 separates into one term per model:
 *   J = sum_i [omega_i f_i Q_i - alpha eta_i c_i - beta max(0, tau_i + delta - f_i)^2]
 * with f_i = (fhat_i - f_min) / (f_max - f_min) the per-variant min-max normalised
 * predicted throughput (fhat_i: the predictor's throughput output) and eta_i = 1 when
 * option i's variant differs from the variant in use.  Constraints (Eq. 4): the
 * summed VRAM of the chosen options <= vram_cap and f_i >= tau_i for every model;
 * otherwise J = -inf.
 * ------------------------------------------------------------------------- */
typedef struct {
  const float *obs;            /* [4] observed state in the aggregate's raw units
                                  (Sigma SM share, Sigma VRAM GB, Sigma BW GB/s, N);
                                  fed to the predictors scaled by agg_scale */
  const int32_t *variant;      /* [sum K_i] variant of each option (>= 0), model-major */
  const float *quality;        /* [sum K_i] Q of the option's variant */
  const float *f_min;          /* [sum K_i] throughput extrema of the option's variant, */
  const float *f_max;          /*           f_max > f_min */
  const float *omega;          /* [N] priority weights */
  const float *tau;            /* [N] floors on the normalised throughput */
  const float *reload_cost;    /* [N] c_i^rel */
  const int32_t *prev_variant; /* [N] variant in use, -1 for none (eta_i = 0) */
  float alpha, beta, delta;    /* paper: 1/60, 5.0, 0.05 */
} mf_fc_params;

/* Evaluate the sum K_i local predictions under p->obs with the fp32 predictor and
 * build the per-option table (fhat, f, floor flag, utility term) on the device; the
 * context keeps it for mf_fc_search until the next call.  Host arrays, copied.
 * Synchronous on `stream`.  MF_EINVAL: NULL arrays, f_max <= f_min, variant < 0,
 * prev_variant < -1, non-finite constants. */
mf_status mf_fc_set(mf_ctx *ctx, const mf_fc_params *p, void *stream);

/* Copy the table of the last mf_fc_set into caller-owned device arrays of sum K_i
 * entries (model-major; any may be NULL): fhat, f, u (the option's term of J), ok
 * (1: f >= tau_i).  Asynchronous on `stream`.  MF_EINVAL before mf_fc_set. */
mf_status mf_fc_table(mf_ctx *ctx, float *d_fhat, float *d_f, float *d_u, uint8_t *d_ok, void *stream);

/* Fixed-context exhaustive search over [lo, hi): J(lambda) = sum of the options'
 * terms (fp32, model order), the same result contract as mf_search_range (top-k by
 * J desc then index asc, feasible count, empty slots (UINT64_MAX, -inf)).  An
 * ALU-bound table-lookup scan.  MF_EINVAL before mf_fc_set. */
mf_status mf_fc_search(mf_ctx *ctx, uint64_t lo, uint64_t hi, int32_t k, uint64_t chunk, mf_result *out,
                       void *stream);

/* The paper's GA (Sec. IV-C) on the fixed-context landscape of the last mf_fc_set:
 * tournament selection, uniform crossover applied with probability crossover_p (else
 * a copy of the first parent), per-gene mutation, elitism, and repair of an
 * infeasible individual (J = -inf) by a feasible one drawn by rejection from the
 * uniform distribution over Lambda (at most floor(256 / N) attempts; the initial
 * uniform population is repaired the same way).  Fitness is the table sum of
 * mf_fc_search (fp32).  Random draws: the counter-based generator of mf_ga_step
 * plus purposes 6 (crossover coin) and 7 (repair, j = attempt * N + gene).
 * Result (host): the fittest individual of the last population, lowest slot among
 * equals; best_genome has N entries.  Synchronous.  One CTA: pop <= 1024.
 * MF_EINVAL: NULL arguments, called before mf_fc_set, a parameter out of its range. */
typedef struct {
  int32_t pop;                 /* 2..1024 */
  int32_t gens;                /* >= 1 fitness evaluations */
  int32_t tournament;          /* 1..256 */
  double crossover_p;          /* [0, 1]; paper 0.7 */
  double mutation_p;           /* [0, 1]; paper 0.1 */
  int32_t elitism;             /* 0 or 1 */
  int32_t repair;              /* 0 or 1 */
} mf_fc_ga_params;

mf_status mf_fc_ga_run(mf_ctx *ctx, const mf_fc_ga_params *g, uint64_t seed, int32_t *best_genome,
                       float *best_fitness, void *stream);

/* Lambda without its VRAM-infeasible configurations (Eq. 4 applied when Lambda is
 * built): writes the ascending indices of [lo, hi) whose summed VRAM <= vram_cap to
 * d_out (device, capacity cap; indices beyond cap are counted, not written) and
 * their number to *count (host).  Synchronous. */
mf_status mf_vram_feasible(mf_ctx *ctx, uint64_t lo, uint64_t hi, uint64_t *d_out, uint64_t cap,
                           uint64_t *count, void *stream);

/* Score with the Eq. 3 utility on the coupled aggregate: predictor i sees the
 * candidate's own summed demands (as every other call of this library) and its
 * throughput output fhat_i enters J = sum_i [omega_i f_i Q_i - alpha eta_i c_i -
 * beta max(0, tau_i + delta - f_i)^2], f_i = (fhat_i - f_min) / (f_max - f_min) of
 * the option's variant; a candidate is feasible iff its summed VRAM <= vram_cap and
 * f_i >= tau_i for every model (the latency outputs and SLA ceilings are not used).
 * Applies to mf_score_batch, mf_search_range / mf_search_exhaustive (fp32 and bf16),
 * mf_ga_generation and mf_ga_run until mf_set_utility(ctx, NULL) restores the
 * problem's own objective.  p->obs is not used.  MF_EINVAL as mf_fc_set. */
mf_status mf_set_utility(mf_ctx *ctx, const mf_fc_params *p);

/* Read the context's instrumentation (see mf_stats). */
mf_status mf_get_stats(const mf_ctx *ctx, mf_stats *out);

/* Exhaustive search without any device allocation.
 *
 * The paper has no counterpart to this call; it exists for callers that cannot
 * call cudaMalloc -- for example a serving process whose memory pool has already
 * claimed the device's memory, or a per-decision control loop that must not pay
 * cudaMalloc's implicit device synchronisation.  It runs the exact fp32 search of
 * mf_search_exhaustive on the problem `p` (host arrays, as for mf_create;
 * precision must be MF_FP32) and fills `out` (host memory) the same way, without
 * creating a context.  All device memory it uses -- a copy of the problem's
 * tables and weights, the per-CTA running top-k lists, the merge buffers, the
 * feasible counter and the status word -- lives in one fixed array of
 * MF_NOALLOC_SCRATCH_BYTES that the library declares in device memory; every GPU
 * that loads the library holds that array until the process exits.  The call
 * allocates nothing (no cudaMalloc, cudaFree or other allocating routine).
 *
 * Limits (MF_EINVAL with a message beyond them): k <= MF_NOALLOC_MAX_TOPK, packed
 * predictor weights <= MF_NOALLOC_MAX_WEIGHT_BYTES, and the whole layout within
 * MF_NOALLOC_SCRATCH_BYTES.  At most MF_NOALLOC_MAX_CTAS CTAs are launched.
 *
 * The first call on a device looks up the array's device address (once per
 * device, with that device current), and that lookup is what makes the runtime
 * load the library's module and reserve the array on the device: a caller whose
 * memory pool will claim the device's memory makes the first call before the pool
 * does, and before any stream capture.  A cudaDeviceReset releases the array but
 * not the cached address, so after resetting a device do not call this entry point
 * on it again.  A call that fails after it has queued work waits for that work
 * before returning.  Every call on a device shares the one array and overwrites it
 * (what must start at zero is cleared at the start of each call), so calls
 * that overlap on the GPU -- from several host threads or streams -- race and
 * must be serialised by the caller.  Synchronous: returns after `out` is filled. */
#define MF_NOALLOC_SCRATCH_BYTES (4u << 20)
#define MF_NOALLOC_MAX_TOPK 64
#define MF_NOALLOC_MAX_CTAS 256
#define MF_NOALLOC_MAX_WEIGHT_BYTES (1u << 20)
mf_status mf_search_exhaustive_noalloc(const mf_problem *p, int32_t k, uint64_t chunk,
                                       mf_result *out, void *stream);

/* Synchronise `stream`, then return MF_EDEVICE if any asynchronous call since the
 * last check saw an invalid index or gene (and clear that flag), else MF_OK. */
mf_status mf_check_device_status(mf_ctx *ctx, void *stream);

/* For tests of the failure path of the bounded device waits; the paper has no
 * counterpart.  With polls > 0, every later launch on `ctx` of a kernel that waits
 * on the device (the tensor-core scorer behind mf_search_* / mf_score_batch in
 * MF_BF16, and the single-kernel GA of mf_ga_run) first waits on a flag that
 * nothing sets, giving up after `polls` polls (about a millisecond each in the
 * scorer, a few nanoseconds in the GA kernel).  The kernel then flags the context's
 * device status and runs to its end without waiting again, except for its own
 * MMAs and weight copies in flight, which it always drains before it frees its
 * tensor memory; the call returns MF_ETIMEOUT and its results are undefined.  The
 * context stays usable: polls = 0 restores normal operation.  MF_EINVAL: ctx NULL. */
mf_status mf_debug_wait_test(mf_ctx *ctx, uint32_t polls);

/* ---------------------------------------------------------------------------
 * Operators that train the predictors and their monitor state
 *
 * The paper trains its predictors offline and reads the observed state s_t off a
 * runtime monitor (Sec. III-A, III-B, Eq. 2); neither has a kernel there.  These calls
 * need no context.  They run on the current device, are asynchronous on `stream`,
 * allocate nothing and keep nothing: `d_work` is the caller's scratch of at least the
 * bytes that the *_sizes / *_workspace call gives for the same arguments (16-byte
 * aligned; its contents need not be set and mean nothing afterwards; calls that may
 * overlap need one each).  `d_status` (device, may be NULL) is or-ed with 2 if a
 * bounded device-side wait gave up; the outputs of that call are then undefined.  (With 1
 * where an embedding saw an invalid id.)
 * mf_operators_status gives a word of the library's own for it.
 * Equal calls give equal bits.  Inputs may be broadcast views (strides of 0);
 * outputs may not overlap themselves, each other or an input.
 * MF_EINVAL: NULL argument or required pointer, unknown type, size or stride out of
 * range, output that overlaps itself, pointer not aligned to its type, workspace too
 * small.  A size of zero is not an error.
 * ------------------------------------------------------------------------- */
typedef enum { MF_TYPE_F32 = 0, MF_TYPE_BF16 = 1, MF_TYPE_F16 = 2 } mf_type;

/* A [batch][time][dim] tensor: strides in elements, the last axis contiguous. */
typedef struct {
  void *d_ptr;
  int64_t stride_batch, stride_time;
} mf_seq;

/* Gated linear recurrence over sequences: per batch row b and channel c,
 *   f_t = 1 / (1 + exp(-z_t)),   h_t = f_t h_{t-1} + (1 - f_t) x_t,
 * a running mean of x whose memory the gate sets.  A mark says what step t is:
 *   MF_MARK_MISSING  no sample: h_t = h_{t-1}; x_t and z_t are not used (they may be NaN)
 *   MF_MARK_SAMPLE   as above (any value but 0 and 2 is read as this)
 *   MF_MARK_FIRST    the first sample of another trace: h_t = (1 - f_t) x_t, whatever
 *                    h_{t-1} was
 * The state is held in fp32; 1 - f_t is computed without cancellation; h is rounded
 * once to the tensors' type. */
typedef enum { MF_MARK_MISSING = 0, MF_MARK_SAMPLE = 1, MF_MARK_FIRST = 2 } mf_mark;

typedef struct {
  int32_t type;                 /* mf_type of x, z and h */
  int64_t batch, time, dim;     /* each >= 0; batch, time, dim < 2^31 */
  mf_seq x, z;                  /* inputs */
  const uint8_t *d_marks;       /* [batch][time] with the strides below; NULL: all MF_MARK_SAMPLE */
  int64_t marks_stride_batch, marks_stride_time;
  const float *d_h0;            /* [batch][dim] state before step 0; NULL: zeros */
  mf_seq h;                     /* output */
  float *d_last;                /* [batch][dim] state after the last step (h0 where time is 0); may be NULL */
  float *d_saved;               /* for mf_recurrence_backward: mf_recurrence_sizes' floats; NULL: not kept */
  uint32_t *d_status;
} mf_recurrence_args;

/* Gradients of the above: from dh (the gradient of h) and dlast (of last; NULL: zeros)
 *   l_t = dh_t + (what step t + 1 passes back: f_{t+1} l_{t+1}; l_{t+1} where t + 1 is
 *         missing; 0 where it is a first sample; dlast behind the last step)
 *   dx_t = (1 - f_t) l_t,  dz_t = l_t (h_{t-1} - x_t) f_t (1 - f_t),  dh0 = what step 0 passes back,
 * with h_{t-1} read as 0 at a first sample and dx_t = dz_t = 0 at a missing one. */
typedef struct {
  int32_t type;                 /* mf_type of x, z, dh, dx and dz */
  int64_t batch, time, dim;
  mf_seq x, z;                  /* inputs, as for the forward call */
  const uint8_t *d_marks;
  int64_t marks_stride_batch, marks_stride_time;
  const float *d_saved;         /* written by the forward call on the same inputs */
  mf_seq dh;
  const float *d_dlast;         /* [batch][dim] or NULL */
  mf_seq dx, dz;                /* outputs */
  float *d_dh0;                 /* [batch][dim]; may be NULL */
  uint32_t *d_status;
} mf_recurrence_grad_args;

/* Floats of `d_saved` and the scratch bytes of the two calls for these sizes, on the
 * current device. */
mf_status mf_recurrence_sizes(int32_t type, int64_t batch, int64_t time, int64_t dim, uint64_t *saved_floats,
                              uint64_t *forward_bytes, uint64_t *backward_bytes);
mf_status mf_recurrence_forward(const mf_recurrence_args *p, void *d_work, uint64_t work_bytes, void *stream);
mf_status mf_recurrence_backward(const mf_recurrence_grad_args *p, void *d_work, uint64_t work_bytes, void *stream);

/* Orthogonalises each matrix G of a batch by Newton-Schulz products, as an optimiser does
 * with a layer's update before it applies it:
 *   X = G / (|G|_F + eps);  `steps` times:  A = X X^T,  X <- a X + (b A + c A A) X
 * (A = X^T X, on the other side, where a matrix has more rows than columns; that is the
 * same polynomial).  With the default coefficients (3.4445, -4.7750, 2.0315) five steps
 * bring every singular value that is not far below |G|_F near 1.
 * Products run on the tensor cores with fp32 accumulation.  fp32 and fp16 results: every
 * operand is split into two fp16 parts (about 22 bits).  bf16 results: so in all steps but
 * the last two, whose operands are rounded to fp16 (later steps no longer amplify a
 * rounding error; its share of the result's error is below that of rounding to bf16).
 * Operands are scaled matrix by matrix, so |G| far below eps (down to 1e-34 of it) costs no bits.
 * A matrix of zeros gives zeros; one that holds a NaN or an infinity gives NaN throughout.
 * steps = 0 gives G / (|G|_F + eps). */
#define MF_ORTH_MAX_STEPS 32
typedef struct {
  int32_t type;                 /* mf_type of g and out */
  int64_t batch, rows, cols;    /* each >= 0; rows, cols <= 2^20; batch < 2^31 */
  const void *d_g;              /* rows contiguous; strides in elements */
  int64_t g_stride_batch, g_stride_row;
  void *d_out;
  int64_t out_stride_batch, out_stride_row;
  int32_t steps;                /* 0..MF_ORTH_MAX_STEPS */
  float a, b, c;                /* finite; the polynomial a s + b s^3 + c s^5 must keep
                                   [0, 1] within [-4, 4] at every step (MF_EINVAL) */
  float eps;                    /* finite, >= 0 */
  uint32_t *d_status;
} mf_orthogonalize_args;
mf_status mf_orthogonalize_workspace(const mf_orthogonalize_args *p, uint64_t *bytes);
mf_status mf_orthogonalize(const mf_orthogonalize_args *p, void *d_work, uint64_t work_bytes, void *stream);

/* Linear attention over sequences whose state decays: per batch row and head, with f = exp(log_decay)
 * of the head,
 *   S_t = f S_{t-1} + k_t v_t^T,   o_t = scale q_t S_t      (S: dim_k x dim_v, held in fp32).
 * A mark says what step t is, as for the recurrence:
 *   MF_MARK_MISSING  no sample: S_t = S_{t-1}; k_t and v_t are not used (they may be NaN); o_t is what
 *                    q_t finds in the state
 *   MF_MARK_SAMPLE   as above (any value but 0 and 2 is read as this)
 *   MF_MARK_FIRST    the first sample of another trace: S_t = k_t v_t^T, whatever S_{t-1} was
 * Steps pass one by one, or, where heads of 16-bit types are wide, in chunks whose rows attend each other
 * and the state before the chunk.  An infinite or NaN value makes what depends on it NaN or
 * infinite, and nothing else.  o is rounded once to the tensors' type.
 * Before that, a result is off relative to the sizes of its own terms, whatever stands beside them in a row or a
 * sequence: as in fp32 arithmetic (the states always; 1.5e-7 to 7e-7 of them for traces of 1000 to 86400 steps, where the
 * sum of products by chunks is off by 1.5e-7 to 3e-7), and for bf16 in chunks by up to 2^-16 of a term more: there the state before
 * the chunk and the weighted products of q and k pass as 16 bits (bf16 rounds o to 8).  The gradients are sums
 * of the same kind. */
#define MF_ATTEND_MAX_DIM 128

/* A [batch][time][heads][dim] tensor: strides in elements, the last axis contiguous. */
typedef struct {
  void *d_ptr;
  int64_t stride_batch, stride_time, stride_head;
} mf_heads;

typedef struct {
  int32_t type;                        /* mf_type of q, k, v and o */
  int64_t batch, time, heads, dim_k, dim_v;  /* each >= 0; dim_k, dim_v <= MF_ATTEND_MAX_DIM, the others < 2^31 */
  mf_heads q, k, v;                    /* inputs */
  const float *d_log_decay;            /* [heads]; any value: -infinity forgets at each sample, 0 never */
  const float *d_state;                /* [batch][heads][dim_k][dim_v] state before step 0; NULL: zeros */
  const uint8_t *d_marks;              /* [batch][time] with the strides below; NULL: all MF_MARK_SAMPLE */
  int64_t marks_stride_batch, marks_stride_time;
  float scale;
  mf_heads o;                          /* output */
  float *d_last;                       /* [batch][heads][dim_k][dim_v] state after the last step; may be NULL, and
                                          may be d_state itself (updated in place) */
  float *d_saved;                      /* for mf_linear_attention_backward; NULL: not kept */
  uint32_t *d_status;
} mf_linear_attention_args;

/* Gradients of the above from those of o and of the last state (NULL: zeros):
 *   G_t = scale q_t do_t^T + (what step t + 1 passes back: f G_{t+1}; G_{t+1} where t + 1 is missing; 0
 *         where it is a first sample; dlast behind the last step)
 *   dq_t = scale S_t do_t,  dk_t = G_t v_t,  dv_t = G_t^T k_t,  dstate = what step 0 passes back,
 * with dk_t = dv_t = 0 at a missing sample.  The decays are constants. */
typedef struct {
  int32_t type;                        /* mf_type of q, k, v, dout, dq, dk and dv */
  int64_t batch, time, heads, dim_k, dim_v;
  mf_heads q, k, v;                    /* inputs, as for the forward call */
  const float *d_log_decay;
  const float *d_saved;                /* written by the forward call on the same inputs */
  const uint8_t *d_marks;
  int64_t marks_stride_batch, marks_stride_time;
  float scale;
  mf_heads dout;                       /* the gradient of o */
  const float *d_dlast;                /* [batch][heads][dim_k][dim_v] or NULL */
  mf_heads dq, dk, dv;                 /* outputs */
  float *d_dstate;                     /* [batch][heads][dim_k][dim_v]; may be NULL */
  uint32_t *d_status;
} mf_linear_attention_grad_args;

/* Floats of `d_saved` and the scratch bytes of the two calls for these sizes, on the current device. */
mf_status mf_linear_attention_sizes(int32_t type, int64_t batch, int64_t time, int64_t heads, int64_t dim_k, int64_t dim_v,
                                    uint64_t *saved_floats, uint64_t *forward_bytes, uint64_t *backward_bytes);
mf_status mf_linear_attention_forward(const mf_linear_attention_args *p, void *d_work, uint64_t work_bytes, void *stream);
mf_status mf_linear_attention_backward(const mf_linear_attention_grad_args *p, void *d_work, uint64_t work_bytes,
                                       void *stream);

/* Embedding lookup: out[i] = scale * table[ids[i]], a row of zeros where ids[i] is MF_NO_TOKEN (the
 * padding of a batch).  An id that is neither that nor a row of the table gives a row of zeros too, and
 * or-s d_status with 1. */
#define MF_NO_TOKEN (-1)
typedef struct {
  int32_t type;                        /* mf_type of table and out */
  int32_t id_bits;                     /* 32 or 64: ids are int32_t or int64_t */
  int64_t rows, dim, tokens;           /* each >= 0 and < 2^31 */
  const void *d_table;                 /* [rows][dim]: rows contiguous, stride in elements */
  int64_t table_stride;
  const void *d_ids;                   /* [tokens] */
  void *d_out;                         /* [tokens][dim] */
  int64_t out_stride;
  float scale;
  uint32_t *d_status;
} mf_embedding_args;

/* The gradient of the table: dtable[r] = scale * the sum of dout[i] over the tokens i with ids[i] = r, in fp32
 * and in the tokens' order by parts, rounded once; zeros where no token names the row.  (Not added to what
 * dtable holds.) */
typedef struct {
  int32_t type;                        /* mf_type of dout and dtable */
  int32_t id_bits;
  int64_t rows, dim, tokens;
  const void *d_dout;                  /* [tokens][dim] */
  int64_t dout_stride;
  const void *d_ids;
  void *d_dtable;                      /* [rows][dim] */
  int64_t dtable_stride;
  float scale;
  uint32_t *d_status;
} mf_embedding_grad_args;
mf_status mf_embedding_forward(const mf_embedding_args *p, void *stream);
mf_status mf_embedding_workspace(const mf_embedding_grad_args *p, uint64_t *bytes);
mf_status mf_embedding_backward(const mf_embedding_grad_args *p, void *d_work, uint64_t work_bytes, void *stream);

/* The norm of all values of `count` tensors, and the tensors scaled so that it is at most max_norm:
 *   norm = sqrt(sum of squares),  out = in * min(1, max_norm / (norm + eps)).
 * A norm that is no finite float32 (a NaN, an infinity) scales nothing: out = in, and the norm says so.
 * in and out of a tensor may be the same memory (nothing is written then where nothing is scaled); else no
 * out may overlap an in or another out (MF_EINVAL).  The norm is a sum of fp32 sums, off by about 1e-7 of it.  The arrays of the arguments are read before the call
 * returns.  Equal bits for equal calls: tensors of the same sizes at addresses that are alike modulo 16. */
typedef struct {
  int64_t count;                       /* tensors: >= 0 and < 2^31 */
  const void *const *d_in;             /* [count] */
  void *const *d_out;                  /* [count] */
  const int64_t *sizes;                /* [count] values; each, and all together, < 2^40 */
  const int32_t *types;                /* [count] mf_type */
  float max_norm, eps;                 /* not negative; eps finite */
  float *d_norm;                       /* one value; may be NULL */
} mf_clip_args;
mf_status mf_clip_workspace(const mf_clip_args *p, uint64_t *bytes);
mf_status mf_clip_gradients(const mf_clip_args *p, void *d_work, uint64_t work_bytes, void *stream);

/* The current device's status word for calls that share one as their d_status: a variable
 * of the library, zero when the library is loaded, which callers read and clear.  May be
 * called while a stream is captured. */
mf_status mf_operators_status(uint32_t **d_word);

/* For tests of the failure path of the operators' bounded waits; the paper has no
 * counterpart.  With polls > 0, the waits of every later mf_recurrence_*,
 * mf_orthogonalize or mf_linear_attention_* call of the calling host thread expect what
 * nothing sends, and give up after `polls` polls (at most 4096; a millisecond each at
 * most).  The kernels then flag the call's d_status, run to their end without waiting
 * again, except for their own copies and products in flight, and the outputs are
 * undefined; a call whose kernels have nothing to wait for is as ever.
 * polls = 0 restores normal operation. */
mf_status mf_debug_operators_wait_test(uint32_t polls);

#ifdef __cplusplus
}
#endif
#endif /* MF_H */
