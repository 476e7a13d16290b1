/*
 * bkmoo.h -- C ABI of the Bucket-Level MOO resolve library for GB300 (sm_103a).
 *
 * The method ("Multilingual Fine-Tuning via Localized Gradient Conflict
 * Resolution", arXiv 2606.05613, Section 3.2 and Algorithm 1) splits the
 * parameters into disjoint buckets and, for every bucket, resolves the K
 * per-language gradients restricted to that bucket into one update
 * direction with a multi-objective rule (MGDA, CAGrad or PCGrad).  The global
 * update is the concatenation of the bucket directions (Section 3.2).
 *
 * Every rule needs the gradients only through the bucket's K x K Gram matrix
 * G[i][j] = <g_i, g_j> (Eq. 3, Eq. 4, Eq. 5 are functions of inner products),
 * and every rule's result is a linear combination d_b = sum_k beta_k g_k.  So
 * one resolve is three device passes: Gram, per-bucket solve for beta, and
 * combination.
 *
 * Notation: K = number of languages (the paper's T), B = number of buckets
 * (the paper's K), N = elements per language gradient.
 *
 * Conventions common to every entry point:
 *  - Every buffer is owned by the caller.  No entry point allocates device
 *    memory; scratch lives in a caller-supplied workspace.
 *  - Device work is asynchronous on the caller's `stream` (a cudaStream_t
 *    passed as void*; NULL = the legacy default stream).  Argument errors are
 *    returned synchronously; conditions found on the device are written to
 *    per-bucket status words and to the workspace status word
 *    (bkmoo_workspace_status).
 *  - Gradients are K separate device buffers, each the flat per-language
 *    gradient in the layout the plan describes, N elements, fp32 or bf16,
 *    16-byte aligned.
 *  - Offsets are int64 element offsets: offsets[0] = 0, strictly
 *    increasing, offsets[B] = N.  Bucket b is [offsets[b], offsets[b+1]).
 *  - 1 <= K <= 16.
 */
#ifndef BKMOO_H
#define BKMOO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Return codes and per-bucket status values. */
typedef enum {
  BKMOO_OK = 0,
  BKMOO_ERR_INVALID = 1,          /* bad argument; nothing was launched    */
  BKMOO_ERR_CUDA = 2,             /* a CUDA call failed                    */
  BKMOO_ERR_NONFINITE = 3,        /* per bucket: Gram not finite, beta=1/K */
  BKMOO_ERR_WORKSPACE = 4,        /* workspace not initialised for this
                                     plan, or too small                    */
  BKMOO_ERR_TIMEOUT = 5,          /* a bounded device wait gave up         */
  BKMOO_ERR_BUFFER_TOO_SMALL = 6, /* an output array is too short          */
  BKMOO_ERR_NOT_CONVERGED = 7     /* per bucket: the solver hit its
                                     iteration cap without meeting the
                                     stopping test; beta is the last
                                     iterate                               */
} bkmoo_status;

/* The multi-objective rule applied to every bucket (Algorithm 1). */
typedef enum {
  BKMOO_MGDA = 0,   /* Eq. 3 / Eq. 6: min-norm point of the convex hull     */
  BKMOO_PCGRAD = 1, /* Eq. 5 / Eq. 8: sequential projection of conflicts   */
  BKMOO_CAGRAD = 2, /* Eq. 4 / Eq. 7: conflict-averse direction            */
  BKMOO_MEAN = 3    /* the averaged gradient of plain fine-tuning          */
} bkmoo_rule;

typedef enum {
  BKMOO_F32 = 0,
  BKMOO_BF16 = 1,
  BKMOO_E4M3 = 2 /* moments of bkmoo_adamw only                             */
} bkmoo_dtype;

/* bkmoo_params.flags */
#define BKMOO_FLAG_CLOSED_FORM_K2 0x1u /* K = 2 MGDA by its closed form      */
#define BKMOO_FLAG_POLISH 0x2u         /* exact active-set completion after
                                          the Frank-Wolfe phase (MGDA and
                                          CAGrad)                            */
#define BKMOO_FLAG_FUSED 0x4u          /* one launch in which the combination
                                          follows the Gram bucket by bucket
                                          while the gradients are still on
                                          the chip, for K <= 8; above, ignored
                                          (three launches), and where a solve
                                          may be long: MGDA (but for the K = 2
                                          closed form) and CAGrad with max_iter
                                          above 1024 or, for K >= 3, without
                                          BKMOO_FLAG_POLISH.  The results are
                                          those of the three launches, bit for
                                          bit.  Without this flag the faster
                                          of the two is taken.              */
#define BKMOO_FLAG_THREE_PASS 0x8u     /* always the three-launch path (Gram,
                                          solve, combination)               */
#define BKMOO_FLAG_TEST_WITHHOLD 0x100u /* testing failure detection, with
                                          BKMOO_FLAG_FUSED only, where the one
                                          launch runs: it never publishes its
                                          first bucket's coefficients, so its
                                          bounded waits (about 2 s) run out and
                                          the call ends with BKMOO_ERR_TIMEOUT in the
                                          workspace status word; the output
                                          is then undefined                 */
#define BKMOO_FLAG_TEST_WITHHOLD_EXCHANGE 0x200u /* testing failure detection,
                                          with BKMOO_FLAG_FUSED only, where the
                                          one launch runs: its first CTA never
                                          publishes its first chunk's partial
                                          Gram, so the bounded wait for it
                                          (about 2 s) runs out, every other
                                          wait ends at once, and the call ends
                                          with
                                          BKMOO_ERR_TIMEOUT in the workspace
                                          status word; the output is then
                                          undefined                         */

typedef struct {
  int32_t max_iter; /* Frank-Wolfe iterations per bucket (MGDA, CAGrad)     */
  double tol;       /* relative duality-gap stop of the Frank-Wolfe phase   */
  double cagrad_c;  /* CAGrad c in [0, 1) (Eq. 4); the paper uses 0.5       */
  uint64_t seed;    /* PCGrad "random order" (Algorithm 1) is a function of */
  uint64_t step;    /*   (seed, step, bucket, task), see bkmoo_resolve      */
  uint32_t flags;   /* BKMOO_FLAG_*                                         */
  void* events;     /* tracing: NULL, or an array of 4 cudaEvent_t that
                       bkmoo_resolve records on `stream` before the Gram pass,
                       after it, after the solve and after the combination
                       (one launch: the last three are recorded together
                       after it).  Owned by the caller.                    */
} bkmoo_params;

/* Fill *p with the defaults: max_iter 256, tol 1e-12, cagrad_c 0.5, seed 0,
 * step 0, flags CLOSED_FORM_K2 | POLISH, events NULL. */
void bkmoo_default_params(bkmoo_params* p);

/*
 * bkmoo_plan -- bucket partition (Section 3.2, Figure 4 caption: fixed-size
 * buckets filled during the backward pass starting from the last
 * parameters).  Host only, pure.
 *
 * param_sizes[n_params]: element counts of the model's tensors in
 * registration order.  The flat gradient the other calls read lists them in
 * REVERSE registration order, each tensor in its own flat order.  A bucket
 * holds at most cap = floor(bucket_bytes / elem_bytes) elements: a tensor
 * that does not fit in the open bucket closes it; a tensor larger than cap is
 * cut into cap-sized pieces; the rest joins the open bucket.  Empty tensors
 * are skipped.
 *
 * Two-call use: with out_offsets == NULL only *n_buckets is set.  Otherwise
 * out_offsets[0 .. *n_buckets] is written; out_cap is its length (>= B + 1,
 * else BKMOO_ERR_BUFFER_TOO_SMALL).  BKMOO_ERR_INVALID on a NULL pointer,
 * negative size, elem_bytes <= 0 or cap < 1.
 */
int bkmoo_plan(const int64_t* param_sizes, int32_t n_params, int32_t elem_bytes,
               int64_t bucket_bytes, int64_t* out_offsets, int64_t out_cap,
               int64_t* n_buckets);

/*
 * bkmoo_workspace_size -- bytes of device workspace that bkmoo_gram and
 * bkmoo_resolve need for K languages of `in_dtype` over the buckets given by
 * offsets[0 .. n_buckets] (host array).  Writes *bytes.  The workspace holds
 * the device copy of the bucket table, per-block Gram partials (fp64), the
 * per-bucket coefficients and a status word.
 */
int bkmoo_workspace_size(int32_t K, int32_t in_dtype, const int64_t* offsets,
                         int64_t n_buckets, size_t* bytes);

/*
 * bkmoo_workspace_init -- write the bucket table for (K, in_dtype, offsets)
 * into the workspace `ws` (device, ws_bytes >= bkmoo_workspace_size, 256-byte
 * aligned).  Call once per plan and workspace, before the first bkmoo_gram or
 * bkmoo_resolve with them.  Copies from host memory and synchronises
 * `stream`.  Later calls must pass the same offsets: a different plan is
 * detected on the device and reported as BKMOO_ERR_WORKSPACE.
 */
int bkmoo_workspace_init(int32_t K, int32_t in_dtype, const int64_t* offsets,
                         int64_t n_buckets, void* ws, size_t ws_bytes,
                         void* stream);

/*
 * bkmoo_gram -- per-bucket Gram matrices, the inner products every rule is
 * built on (Eq. 2, the QP of Eq. 3 / Eq. 6 and the tests of Eq. 8 depend on
 * the gradients only through them).
 *
 * grads: host array of K device pointers.  out_gram: device, fp64,
 * [n_buckets][K][K], row-major, both triangles written.  Results are
 * deterministic: each element is summed in fp32 within a thread over at most
 * 128 elements, then reduced in a fixed order (warp tree in fp32, CTA and
 * cross-CTA in fp64); no atomics.
 */
int bkmoo_gram(const void* const* grads, int32_t K, int32_t in_dtype,
               const int64_t* offsets, int64_t n_buckets, double* out_gram,
               void* ws, size_t ws_bytes, void* stream);

/*
 * bkmoo_conflicts -- the gradient-conflict statistics of Figure 1, per
 * bucket, from Gram matrices (bkmoo_gram's out_gram): the pairwise cosines
 * cos_ij = G_ij / sqrt(G_ii G_jj) -- a pair conflicts when its cosine is
 * negative (Eq. 2, Definition A.4) -- their mean, population standard
 * deviation and minimum over the K(K-1)/2 pairs, and a flag for "at least
 * one pair conflicts" (the event whose per-layer frequency over training
 * steps Figure 1 plots).  A pair with a zero-norm gradient has cosine 0.
 *
 * gram: device fp64 [n_buckets][K][K].  Outputs (device, each may be NULL):
 * out_cos fp32 [n_buckets][K][K] (diagonal 1, or 0 for a zero gradient),
 * out_stats fp32 [n_buckets][3] = (mean, std, min), out_conflict int32
 * [n_buckets] in {0, 1}.  2 <= K <= 16, else BKMOO_ERR_INVALID.
 */
int bkmoo_conflicts(const double* gram, int32_t K, int64_t n_buckets, float* out_cos,
                    float* out_stats, int32_t* out_conflict, void* stream);

/*
 * bkmoo_gram_noalloc -- bkmoo_gram without a workspace argument; it allocates
 * no memory at all.  The paper has no counterpart: this is a service for
 * callers that hold their input and output buffers but cannot get more
 * device memory, for instance a hook inside a training framework whose
 * device memory all belongs to the framework's caching allocator, or a C
 * caller in a process where another component owns device allocation.
 *
 * Same arguments, results (bit for bit) and determinism as bkmoo_gram.  The
 * scratch (bucket table and per-chunk partial sums) lives in a
 * static device array of BKMOO_NOALLOC_SCRATCH_BYTES that every GPU which
 * loads this library keeps until the process exits; the bucket table reaches
 * it through kernel parameters, so no copy or allocating call is made.
 * Limits: at most BKMOO_NOALLOC_MAX_BUCKETS buckets and a problem whose
 * bucket table and partial sums fit the array -- about 13 billion
 * elements per language for K = 4 and 1 billion for K = 16 with bf16
 * gradients (half as many with fp32); larger problems return
 * BKMOO_ERR_WORKSPACE.
 *
 * Each call made outside stream capture looks up the array's device address
 * in the current context (cudaGetSymbolAddress, with the device current);
 * a call made while its stream is being captured reuses the last address
 * seen on that device, so make the first call on each device before any
 * stream capture.  Every call shares the one array and rewrites
 * the parts it reads, so results never depend on an earlier call; but calls
 * whose work overlaps on the GPU (other streams or host threads on the same
 * device) race on it and must be serialised by the caller.
 */
#define BKMOO_NOALLOC_SCRATCH_BYTES (32u << 20)
#define BKMOO_NOALLOC_MAX_BUCKETS 4096
int bkmoo_gram_noalloc(const void* const* grads, int32_t K, int32_t in_dtype,
                       const int64_t* offsets, int64_t n_buckets, double* out_gram,
                       void* stream);

/*
 * bkmoo_resolve -- the resolve of Algorithm 1 for every bucket: Gram ->
 * rule -> d_b = sum_k beta_k g_k, written into the flat direction out_dir
 * (the concatenation of Section 3.2).
 *
 * grads / K / in_dtype / offsets / n_buckets as in bkmoo_gram.
 * rule: bkmoo_rule.  p: parameters (NULL = defaults).
 *  - MGDA: Frank-Wolfe on the simplex QP from the best pair (exact line
 *    search, at most p->max_iter steps, stop at duality gap <= p->tol
 *    relative to max_k G_kk), then, with BKMOO_FLAG_POLISH, an exact
 *    active-set (Wolfe minimum-norm-point) completion.  K = 2 with
 *    BKMOO_FLAG_CLOSED_FORM_K2 uses
 *    gamma = clamp(<g2 - g1, g2> / ||g1 - g2||^2, 0, 1).  beta = alpha.
 *  - CAGrad: the dual min_{w in simplex} <g0, g_w> + c ||g0|| ||g_w||
 *    (g0 the mean) by Frank-Wolfe with exact line search, then the same
 *    active-set completion; beta = 1/K + c ||g0|| w / ||g_w||.  No rescaling.
 *  - PCGrad: for each task t, other tasks j in t's order, project the
 *    running d_t off the ORIGINAL g_j when <d_t, g_j> < 0; d = sum_t d_t.
 *    The order of task t in bucket b is a Fisher-Yates shuffle of the
 *    ascending list [0..K-1] without t, slot i = m-1 .. 1 (m = K-1) swapped
 *    with slot r mod (i+1), r the draws mix64(k3 + (n+1) * 0x9E3779B97F4A7C15)
 *    for n = 0, 1, ..., where k1 = mix64(seed + (step+1) * G),
 *    k2 = mix64(k1 + (b+1) * G), k3 = mix64(k2 + (t+1) * G),
 *    G = 0x9E3779B97F4A7C15 and mix64 is the SplitMix64 output function.
 *  - MEAN: beta = 1/K.
 * out_dir: device, N elements of out_dtype (fp32 or bf16, round to nearest
 *   even).  It may be exactly one of the grads buffers when the dtypes match
 *   (in-place); any other overlap with a gradient is BKMOO_ERR_INVALID.
 * out_weights: device fp32 [n_buckets][K] = beta, or NULL.
 * out_status: device int32 [n_buckets] = BKMOO_OK, BKMOO_ERR_NONFINITE (the
 *   Gram had a NaN/Inf; beta = 1/K), BKMOO_ERR_NOT_CONVERGED or
 *   BKMOO_ERR_WORKSPACE; or NULL.
 * ws / ws_bytes: the workspace after bkmoo_workspace_init with the same
 *   K, in_dtype and offsets.
 * Path: three launches (Gram, solve, combination) or one launch that does the
 *   same bucket by bucket (see BKMOO_FLAG_FUSED), whichever is faster for the
 *   plan and rule (bkmoo_resolve_launches tells); the results are the same bit
 *   for bit and deterministic.  The one launch is cooperative: it starts once
 *   every SM is free and holds them all until it ends, so work on other streams
 *   runs before or after it, not beside it; on a device or context that cannot
 *   hold it the three launches run.  Its CTAs wait for one another, at most 2 s
 *   at a time: a wait that runs out ends the call with BKMOO_ERR_TIMEOUT in the
 *   workspace status word and out_dir partly written (in place: that gradient).
 *   With BKMOO_FLAG_THREE_PASS neither holds: the launches share the GPU, and
 *   no CTA waits for another.
 * Returns BKMOO_OK once the work is queued on `stream`.
 */
int bkmoo_resolve(const void* const* grads, int32_t K, int32_t in_dtype,
                  const int64_t* offsets, int64_t n_buckets, int32_t rule,
                  const bkmoo_params* p, void* out_dir, int32_t out_dtype,
                  float* out_weights, int32_t* out_status, void* ws,
                  size_t ws_bytes, void* stream);

/*
 * bkmoo_resolve_buckets -- bkmoo_resolve for the buckets b_lo .. b_hi-1 of
 * the plan only.  Algorithm 1 resolves bucket k as soon as the backward pass
 * has filled it (its interception "when bucket k is full", Figure 4), while
 * the rest of the backward pass still runs: this entry point lets a caller
 * resolve each bucket as it completes, on any stream.
 *
 * Arguments as in bkmoo_resolve (the whole plan's offsets and workspace),
 * plus 0 <= b_lo <= b_hi <= n_buckets (else BKMOO_ERR_INVALID; b_lo == b_hi
 * queues nothing).  Only those buckets' Gram, rule and combination run: the
 * elements of out_dir, the rows of out_weights / out_status and the
 * workspace partials of other buckets are not touched, so calls for disjoint
 * bucket ranges may run concurrently on different streams.  Results are
 * bit-identical to those of bkmoo_resolve for the same buckets.  Ranges of
 * more than two buckets take one launch where bkmoo_resolve would for a plan of
 * these buckets; one or two always three launches, which share the SMs with
 * whatever runs beside them.  The workspace status word is not cleared (other calls may be in flight); device-side
 * errors are recorded into it.  BKMOO_FLAG_FUSED and p->events are ignored.
 */
int bkmoo_resolve_buckets(const void* const* grads, int32_t K, int32_t in_dtype,
                          const int64_t* offsets, int64_t n_buckets, int64_t b_lo, int64_t b_hi,
                          int32_t rule, const bkmoo_params* p, void* out_dir, int32_t out_dtype,
                          float* out_weights, int32_t* out_status, void* ws, size_t ws_bytes,
                          void* stream);

/*
 * bkmoo_host_staging_size -- device staging bytes bkmoo_resolve_host needs
 * so that every window holds at least max(window_elems, the largest bucket)
 * elements per language.  Host only, pure.  Writes *bytes.
 */
int bkmoo_host_staging_size(int32_t K, int32_t in_dtype, int32_t out_dtype,
                            const int64_t* offsets, int64_t n_buckets, int64_t window_elems,
                            size_t* bytes);

/*
 * bkmoo_resolve_host -- bkmoo_resolve for gradients held in HOST memory, the
 * direction written back to host memory.  It follows the per-bucket loop of
 * Algorithm 1 -- bring a bucket's K gradients to the device, resolve it,
 * send its direction on and free the bucket's device copy -- so that device
 * memory holds only a bounded window of buckets, not the K full gradients.
 *
 * Buckets go through three device staging slots in windows of whole buckets:
 * while window w is resolved (Gram -> rule -> combination on `stream`, the
 * same kernels and the same per-chunk arithmetic as bkmoo_resolve's
 * three-launch path, so beta and the direction are bit-identical to it),
 * the next windows are copied
 * in and earlier windows' directions copied out on two internal copy
 * streams, created and destroyed by the call.  Work already queued on `stream` comes first;
 * `stream` completes only after the last byte reaches host_out.
 *
 * host_grads: host array of K host pointers (16-byte aligned), N elements
 *   each.  Page-locked memory (cudaHostAlloc / cudaHostRegister) lets the
 *   copies overlap; pageable memory gives the same results more slowly.
 * host_out: host, N elements of out_dtype; may be exactly one of host_grads
 *   (same dtype); any other overlap is BKMOO_ERR_INVALID.
 * out_weights, out_status, ws, ws_bytes, rule, p: as in bkmoo_resolve (device
 *   buffers; ws initialised for this plan).  p->events and
 *   BKMOO_FLAG_FUSED are ignored.
 * staging: device, 256-byte aligned, staging_bytes long.  It holds three
 *   slots of K input regions and one output region of
 *   round_up(cap e + 16, 256) bytes each (e the region's element size); cap,
 *   the window length in elements per language, is the largest that fits.
 *   A bucket longer than cap is BKMOO_ERR_WORKSPACE (bkmoo_host_staging_size
 *   gives the size for a chosen cap).  Larger staging means fewer, longer
 *   windows.  Calls that share a staging buffer or a workspace must not
 *   overlap on the GPU.
 * Returns BKMOO_OK once everything is queued.
 */
int bkmoo_resolve_host(const void* const* host_grads, int32_t K, int32_t in_dtype,
                       const int64_t* offsets, int64_t n_buckets, int32_t rule,
                       const bkmoo_params* p, void* host_out, int32_t out_dtype,
                       float* out_weights, int32_t* out_status, void* ws, size_t ws_bytes,
                       void* staging, size_t staging_bytes, void* stream);

/*
 * bkmoo_workspace_status -- synchronise `stream` and read the workspace
 * status word: BKMOO_OK, or the first device-side error recorded since the
 * last bkmoo_gram / bkmoo_resolve started (BKMOO_ERR_WORKSPACE,
 * BKMOO_ERR_TIMEOUT).  Writes *status.
 */
int bkmoo_workspace_status(const void* ws, void* stream, int32_t* status);

/*
 * bkmoo_resolve_launches -- the kernels that bkmoo_resolve launches for this
 * plan, rule and *p (NULL: the defaults): *launches = 1 for the one launch (see
 * BKMOO_FLAG_FUSED), 3 for Gram, solve and combination, 4 when a bucket has
 * more than 1024 chunks and its partials are pre-reduced, 0 for no bucket.  (A
 * device or context that cannot hold the one launch takes three where this
 * says 1.)  Host only; BKMOO_ERR_INVALID on bad arguments.
 * bkmoo_resolve_buckets decides by the same rule over its range, except that
 * ranges of one or two buckets always take the three launches;
 * bkmoo_resolve_host takes the three launches per window.
 */
int bkmoo_resolve_launches(int32_t K, int32_t in_dtype, int32_t rule, const int64_t* offsets,
                           int64_t n_buckets, const bkmoo_params* p, int32_t* launches);

/*
 * bkmoo_resolve_path -- a classification of plans from two earlier one-launch
 * kernels, kept with its answers for programs that record it.  It decides
 * nothing and does not tell the path (bkmoo_resolve_launches does).
 * BKMOO_FLAG_THREE_PASS gives 0; BKMOO_FLAG_FUSED gives 1 for K <= 4 (2 with
 * BKMOO_FLAG_TEST_WITHHOLD), 2 for K = 5..8, 0 above.  Without either flag: 1
 * when K <= 2 and the plan has at most 8 buckets and 4 Mi elements per
 * language, or when 2 <= K <= 4, the largest bucket holds at least 2 MiB per
 * language and its K gradients together at most 12 MiB (and at least 6 MiB for
 * bf16; for CAGrad fp32 only and at least 8 MiB), and at least 90 % of the
 * elements lie in buckets of at least half the largest; 0 otherwise.  Host
 * only; BKMOO_ERR_INVALID on bad arguments.
 */
int bkmoo_resolve_path(int32_t K, int32_t in_dtype, int32_t rule, const int64_t* offsets,
                       int64_t n_buckets, uint32_t flags, int32_t* path);

/*
 * The gated projections of a feed-forward block, with weight gradients kept
 * apart by language.  The resolve needs one gradient per language.  K backward
 * passes give them one by one; where the K languages' rows are in one batch, a
 * linear layer's weight gradients come apart in one pass instead, because each
 * is a sum over rows: dW_k = sum over language k's rows t of dy_t x_t^T.
 *
 * Common to the calls below: matrices are bf16, row-major, rows of `ld*`
 * elements (>= the width, a multiple of 8) from a 16-byte aligned address;
 * widths and row counts are arbitrary.  Sums are fp32, each result is rounded
 * once.  Outputs must not overlap inputs or one another (columns of one wider
 * matrix may hold different ones).  The kernels wait for nothing but their own
 * copies and products; a wait that takes more than 2 s all the same gives up
 * (BKMOO_ERR_TIMEOUT from bkmoo_op_status, the output then undefined).  The
 * first call on each device comes before any stream capture.
 */
typedef enum {
  BKMOO_SILU = 0,     /* a / (1 + e^-a)                                       */
  BKMOO_GELU = 1,     /* a Phi(a), Phi the normal distribution                */
  BKMOO_GELU_TANH = 2 /* a (1 + tanh(sqrt(2/pi) (a + 0.044715 a^3))) / 2      */
} bkmoo_act;

/*
 * bkmoo_gate_forward -- a = x Wg^T, b = x Wu^T, h = act(a) b, in one kernel.
 *
 * x: [T][D]; w_gate, w_up: [F][D], both with rows of ldw.  h, a, b: [T][F]; h
 * from the unrounded a and b.  a and b (the backward pass's inputs) may both be
 * NULL; h may be NULL if they are not.  T = 0 queues nothing.
 */
int bkmoo_gate_forward(const void* x, int64_t ldx, const void* w_gate, const void* w_up,
                       int64_t ldw, int64_t T, int64_t D, int64_t F, int32_t act, void* h,
                       int64_t ldh, void* a, void* b, int64_t ld_ab, void* stream);

/* Bytes of device workspace bkmoo_gate_backward needs (da and db).  Host only. */
int bkmoo_gate_backward_workspace_size(int64_t T, int64_t F, size_t* bytes);

/*
 * bkmoo_gate_backward -- from dh, the gradient of h, with a and b as the
 * forward call gave them: da = dh b act'(a), db = dh act(a), and
 *   dx = da Wg + db Wu,
 *   dWg_k = sum_t da_t x_t^T, dWu_k = sum_t db_t x_t^T over language k's rows.
 *
 * rows: host, K + 1 row bounds, 0 = rows[0] <= ... <= rows[K] = T; language k
 * has the rows from rows[k] to rows[k + 1], none if they are equal (its
 * gradients are then 0).  dx: [T][D], or NULL.  dw_gate, dw_up: host arrays of K
 * device pointers, each to a contiguous [F][D] of dw_dtype at any element's
 * address (a place in a flat per-language gradient, say); or both NULL.
 * accumulate: 0 writes them, 1 adds to what they hold (in fp32, rounded once).
 * da and db, the operands of bf16 products, are rounded to bf16 between; fp32
 * gradients are the unrounded fp32 sums of those.  ws: device, 256-byte
 * aligned, ws_bytes >= bkmoo_gate_backward_workspace_size, not shared by calls
 * that overlap; the call leaves da there, and db from half of the workspace size
 * on, as [T][F] with rows of F rounded up to 8.
 */
int bkmoo_gate_backward(const void* dh, int64_t ld_dh, const void* a, const void* b, int64_t ld_ab,
                        const void* x, int64_t ldx, const void* w_gate, const void* w_up,
                        int64_t ldw, int64_t T, int64_t D, int64_t F, int32_t act, int32_t K,
                        const int64_t* rows, void* dx, int64_t ld_dx, void* const* dw_gate,
                        void* const* dw_up, int32_t dw_dtype, int32_t accumulate, void* ws,
                        size_t ws_bytes, void* stream);

/*
 * bkmoo_language_wgrad -- dW_k = sum over language k's rows t of dy_t x_t^T for
 * a linear layer y = x W^T: dy [T][M], x [T][N], dW_k [M][N].  rows, dw,
 * dw_dtype and accumulate as in bkmoo_gate_backward.
 */
int bkmoo_language_wgrad(const void* dy, int64_t ld_dy, const void* x, int64_t ldx, int64_t T,
                         int64_t M, int64_t N, int32_t K, const int64_t* rows, void* const* dw,
                         int32_t dw_dtype, int32_t accumulate, void* stream);

/*
 * The operators of a language model around its layers, for the same batches: the
 * embedding at its front, the norms of queries and keys, and the log probabilities at its
 * end.  Common to the calls below: `ids`, `positions` and `targets` are device arrays
 * [T] of int32 (id_bytes 4) or int64 (8).  rows, dw pointers, dw_dtype and accumulate
 * are those of bkmoo_gate_backward.  Sums are fp32 in an order fixed by the sizes, the
 * bounds and, but for the embedding, the device's number of SMs: the same call on the same
 * kind of device gives the same bits.  Results are rounded once.  T = 0 queues nothing
 * (gradients that are not added to are set to 0).
 *
 * bkmoo_embedding_forward -- y_t = scale W[id_t].  table: [V][D] of dtype (fp32 or bf16)
 * with rows of ld_table elements, y: [T][D] of the same with rows of ldy, both at any
 * element's address (16-byte vectors where all rows start on 16 bytes).  An id outside
 * 0 .. V - 1 is padding: its y is 0.  V < 2^28, D <= 2^23; scale is finite as fp32; y does
 * not overlap the table.
 */
int bkmoo_embedding_forward(const void* table, int64_t ld_table, int32_t dtype, int64_t V,
                            int64_t D, const void* ids, int32_t id_bytes, int64_t T, double scale,
                            void* y, int64_t ldy, void* stream);

/* Bytes of device workspace bkmoo_embedding_backward needs.  Host only. */
int bkmoo_embedding_backward_workspace_size(int64_t T, int64_t D, size_t* bytes);

/*
 * bkmoo_embedding_backward -- dW_k[v] = scale sum of dy_t over language k's rows t with
 * id_t = v, in the order of t.  dy: [T][D] of dtype, rows of ld_dy, at any element's
 * address; padding has no gradient, and its rows are not read.  dw: host array of K device
 * pointers, each to a contiguous [V][D] of dw_dtype at any element's address, none of which
 * overlap.  accumulate:
 * 0 writes every row, 1 adds to the rows that have a token and leaves the others alone.
 * ws: device, 256-byte aligned, ws_bytes >= the size above, not shared by calls that
 * overlap.
 */
int bkmoo_embedding_backward(const void* dy, int64_t ld_dy, int32_t dtype, const void* ids,
                             int32_t id_bytes, int64_t T, int64_t V, int64_t D, double scale,
                             int32_t K, const int64_t* rows, void* const* dw, int32_t dw_dtype,
                             int32_t accumulate, void* ws, size_t ws_bytes, void* stream);

/*
 * bkmoo_qk_norm_forward -- every head x of the queries and keys normed, weighed and
 * rotated by its token's position: y = w x / sqrt(mean(x^2) + eps), then pair i of the
 * first `rot` elements, (a, b), becomes (a cos - b sin, b cos + a sin) of the angle
 * position inv_freq[i]; pairs are (i, i + rot / 2), or with `interleaved` (2i, 2i + 1).
 *
 * q: bf16, head h of token t at q + t ldq + h head_dim; k, q_out and k_out likewise (columns
 * of one wider matrix may hold several).  16-byte aligned, row strides multiples of 8.
 * head_dim: a multiple of 16 up to 256; rot: a multiple of 16 up to head_dim, 0 for none.
 * q_out may be q, with the same stride, and k_out k; otherwise nothing overlaps.  w_q, w_k:
 * [head_dim] of w_dtype (fp32 or bf16).  inv_freq: host, rot / 2 radians a position (read
 * before the call returns); positions may be negative.  An angle is off by at most 2^-26 of
 * a turn and, for every position, by 2^-64 of a turn and 2^-52 of its own inv_freq / 2 pi (inv_freq
 * = 1: 2^-34 at position 2^20, 2^-14 at 2^40).  Squares are summed in fp32, so elements beyond 1.8e19
 * leave nothing of their head.
 */
int bkmoo_qk_norm_forward(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* w_q,
                          const void* w_k, int32_t w_dtype, int64_t T, int64_t q_heads,
                          int64_t k_heads, int64_t head_dim, const void* positions,
                          int32_t id_bytes, const double* inv_freq, int64_t rot,
                          int32_t interleaved, double eps, void* q_out, int64_t ldq_out,
                          void* k_out, int64_t ldk_out, void* stream);

/* Bytes of device workspace bkmoo_qk_norm_backward needs for weight gradients.  Host only. */
int bkmoo_qk_norm_backward_workspace_size(int64_t head_dim, size_t* bytes);

/*
 * bkmoo_qk_norm_backward -- from dq_out and dk_out, the gradients of the forward call's
 * results, and its inputs: dq and dk (dq may be dq_out, with the same stride, and dk dk_out),
 * and every language's own gradients of the two weights, dw_q[k] and dw_k[k]: contiguous
 * [head_dim] of dw_dtype at any element's address, none of which overlap; both arrays NULL:
 * not wanted (then ws is not used).  ws: device, 256-byte aligned, ws_bytes >= the size above, not shared by calls
 * that overlap.
 */
int bkmoo_qk_norm_backward(const void* dq_out, int64_t ld_dq_out, const void* dk_out,
                           int64_t ld_dk_out, const void* q, int64_t ldq, const void* k, int64_t ldk,
                           const void* w_q, const void* w_k, int32_t w_dtype, int64_t T,
                           int64_t q_heads, int64_t k_heads, int64_t head_dim, const void* positions,
                           int32_t id_bytes, const double* inv_freq, int64_t rot,
                           int32_t interleaved, double eps, int32_t K, const int64_t* rows, void* dq,
                           int64_t ld_dq, void* dk, int64_t ld_dk, void* const* dw_q,
                           void* const* dw_k, int32_t dw_dtype, int32_t accumulate, void* ws,
                           size_t ws_bytes, void* stream);

/*
 * bkmoo_token_logp_forward -- for each row z of logits, with m = max z and
 * L = log sum e^(z - m): logp = z[target] - m - L; stats (m, L), what the backward call
 * needs; entropy -sum p log p; and the n_top most likely tokens with their log
 * probabilities, the likeliest first, the lower index first among equal logits.
 *
 * logits: [T][V] of dtype (fp32 or bf16), rows of ld, at any element's address.  A target
 * outside 0 .. V - 1 is padding: its logp is 0.  stats: [T][2], 8-byte aligned, or NULL;
 * entropy: [T] or NULL; n_top: 0 to min(32, V), top_ids and top_logp [T][n_top], unused
 * where 0.  Minus infinity is a token that is ruled out; a row of nothing else has logp
 * and top_logp minus infinity (padding 0) and entropy 0; so has a log probability below
 * fp32's range minus infinity.  A NaN, or plus infinity, makes
 * its row's results NaN (NaN ranks below minus infinity in top_ids, which are distinct
 * and in range all the same).  V <= 2^30.
 */
int bkmoo_token_logp_forward(const void* logits, int64_t ld, int32_t dtype, int64_t T, int64_t V,
                             const void* targets, int32_t id_bytes, float* logp, float* stats,
                             float* entropy, int32_t n_top, int64_t* top_ids, float* top_logp,
                             void* stream);

/*
 * bkmoo_token_logp_backward -- d_logits from d_logp [T] and d_entropy [T] (or NULL), the
 * gradients of logp and entropy, with the forward call's stats and, for d_entropy, entropy:
 *   d_logits_v = d_logp ([v = target] - p_v) - d_entropy p_v (log p_v + entropy).
 * The d_logp of padding counts as 0.  A row whose d_logp and d_entropy are 0 gets zeros and
 * is not read, nor is a row of nothing but minus infinity.  d_logits: [T][V] of dtype, rows
 * of ld_d; it may be logits, with the same stride.
 */
int bkmoo_token_logp_backward(const void* logits, int64_t ld, int32_t dtype, int64_t T, int64_t V,
                              const void* targets, int32_t id_bytes, const float* stats,
                              const float* entropy, const float* d_logp, const float* d_entropy,
                              void* d_logits, int64_t ld_d, void* stream);

/*
 * bkmoo_op_status -- synchronise `stream` and read the current device's status
 * word of the gate and weight-gradient calls: BKMOO_OK, or BKMOO_ERR_TIMEOUT if
 * one of them gave up since it was last read.  Clears it.  Writes *status.
 */
int bkmoo_op_status(void* stream, int32_t* status);

/*
 * bkmoo_op_status_copy -- queue a copy of that word into *status (device memory, or
 * pinned host memory for a copy that returns at once), neither waiting nor
 * clearing it.
 */
int bkmoo_op_status_copy(void* stream, int32_t* status);

/*
 * bkmoo_selftest_give_up -- queue a kernel that gives up, so that the word says so (a
 * self-test of that and of what follows).  what 0: a single wait of the kind those
 * kernels make, for an arrival that nothing makes, 1 ms long; 1 and 2: the forward
 * pass's kernel of one CTA and of a pair, whose operands are never copied (2 s).
 */
int bkmoo_selftest_give_up(int32_t what, void* stream);

/*
 * bkmoo_grad_norm -- the 2-norm of a flat gradient (the direction), n elements
 * of fp32 or bf16, 16-byte aligned.  out_norm: device fp32, one value.  Squares
 * are summed in fp32 over at most 64 elements, then in fp64, in an order fixed
 * by n: deterministic; the sum and its root are rounded to fp32.  Infinite where a
 * square or the sum leaves fp32, NaN with a NaN, and where bkmoo_op_status would
 * report a call ahead of it that gave up, until that is read: the gradient may be one
 * of its undefined outputs.  ws: device, 256-byte aligned, BKMOO_NORM_WS_BYTES, not
 * shared by calls that overlap.
 */
#define BKMOO_NORM_WS_BYTES 16384
int bkmoo_grad_norm(const void* grad, int32_t dtype, int64_t n, float* out_norm, void* ws,
                    size_t ws_bytes, void* stream);

typedef struct {
  double lr;       /* finite                                                  */
  double beta1;    /* in [0, 1)                                               */
  double beta2;    /* in [0, 1)                                               */
  double eps;      /* >= 0                                                    */
  double max_norm; /* > 0: g is multiplied by min(1, max_norm / (norm + 1e-6)),
                      norm being *grad_norm; 0: not clipped                   */
  int64_t step;    /* 1, 2, ...: bias corrections and the key of the rounding */
  uint64_t seed;   /* of the rounding to 8 bits                               */
} bkmoo_adamw_params;

/* Fill *p with lr 1e-3, beta1 0.9, beta2 0.999, eps 1e-8, max_norm 0, step 1,
 * seed 0. */
void bkmoo_adamw_default_params(bkmoo_adamw_params* p);

/*
 * bkmoo_adamw -- one AdamW step of every tensor with the direction as gradient,
 * the optimizer step of Algorithm 1:
 *   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2,
 *   p = (1 - lr weight_decay) p
 *       - lr (m / (1 - beta1^step)) / (sqrt(v / (1 - beta2^step)) + eps).
 *
 * params[n_params]: host array of device pointers, tensors of sizes[i] elements
 *   of param_dtype (fp32 or bf16), in the order in which the flat buffers hold
 *   them (a bkmoo_plan layout: last registered first); any element-aligned
 *   address, empty ones allowed.  weight_decay: host, one per tensor, or NULL.
 * grad: the flat gradient, N = sum of sizes, fp32 or bf16.
 * master: NULL, or flat fp32 [N], with bf16 params only: the weights that the
 *   step reads and writes; the tensors then receive them rounded to nearest.
 *   Without it bf16 weights are widened, stepped and rounded to nearest.
 * state_dtype BKMOO_F32: m, v flat fp32 [N]; m_scale, v_scale unused.
 * state_dtype BKMOO_E4M3: m, v flat bytes [N], one fp32 scale for every 256 flat
 *   elements in m_scale, v_scale [(N + 255) / 256]: m = m_scale e4m3(byte), and
 *   v's bytes hold its ROOT, sqrt(v) = v_scale e4m3(byte), which spans half as
 *   many powers of two.  A scale is the largest magnitude of its elements / 448
 *   (0 below 2^-100).  Values are rounded up with the chance that their rest
 *   gives, else down: by nearest, a beta2 of 0.999 moves no value of 4 bits'
 *   precision.  A root that is not 0 never becomes 0.  The chance of flat element
 *   i is u / 65536 with u the low (m) or high (v) 16 bits of the low (i even) or
 *   high (i odd) half of mix64(mix64(seed + (step + 1) G) + (i / 2 + 1) G), with
 *   mix64 and G of bkmoo_resolve.  All zeros is the state before the first step.
 * grad, m, v, master: 16-byte aligned; none may overlap another or a tensor.
 * grad_norm: device, as bkmoo_grad_norm gives it, needed where max_norm > 0.
 *   Where it is given and not finite, nothing is changed: the step is skipped.
 *   So it is, without one, where bkmoo_op_status would report a call ahead of it
 *   that gave up, until that is read (with one, the norm of such a gradient is NaN).
 *   Without it a NaN or infinity in g reaches the state (an infinity in 8 bits
 *   its whole block).
 * Moments are computed in fp32.  In 8 bits the root of a v below 2^-126 (gradients
 * below about 1e-19) comes out up to 100 times too small, which an eps of 1e-15 or
 * more hides from the weights.  Up to 1024 tensors take one launch.
 */
int bkmoo_adamw(void* const* params, const int64_t* sizes, const float* weight_decay,
                int32_t n_params, int32_t param_dtype, const void* grad, int32_t grad_dtype,
                float* master, void* m, void* v, float* m_scale, float* v_scale,
                int32_t state_dtype, const bkmoo_adamw_params* p, const float* grad_norm,
                void* stream);

/* Static English text for a bkmoo_status value. */
const char* bkmoo_status_string(int32_t status);

/* Library version, major * 10000 + minor * 100 + patch. */
int32_t bkmoo_version(void);

/*
 * bkmoo_selftest_fp64 -- runs, element by element on the device, the fp64
 * division and square root that the fast per-bucket solvers use for the
 * CAGrad and PCGrad coefficients (Eq. 4 / Eq. 7, Eq. 5 / Eq. 8): an fp32
 * seed refined by one Newton-Raphson step with a residual correction
 * (q = a r, q + (a - b q) r with r = 1/b rounded to fp32; s + (x - s^2) / (2 s)
 * with s = sqrt(x) rounded to fp32), relative error at most about 2^-46;
 * arguments outside [1e-30, 1e30] take the correctly rounded operation.
 * A test entry point, so that its accuracy can be checked against the
 * correctly rounded fp64 operations.
 * op 0: out[i] = a[i] / b[i]; op 1: out[i] = sqrt(a[i]) (0 for a[i] <= 0;
 * b unused, may be NULL).  a, b, out: device fp64 [n].  Asynchronous on
 * `stream`.  Returns BKMOO_ERR_INVALID for another op, n < 0 or a NULL
 * array, BKMOO_ERR_CUDA if the launch fails.
 */
int bkmoo_selftest_fp64(int32_t op, const double* a, const double* b, double* out, int64_t n,
                        void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BKMOO_H */
