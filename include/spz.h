/*
 * spz.h -- C ABI of the large-batch actor-critic update on one MI355X (gfx950).
 *
 * The library implements the network-update process of Spreeze (Section 3.2:
 * one updater drawing large uniform batches from a shared replay pool and
 * training the actor and the double-Q critics with target networks; Section
 * 3.2.2: actor and critic updated independently, here as two concurrent HIP
 * streams on one GPU). SAC is the paper's worked example; TD3 is the
 * alternative algorithm of Section 4.2.4, Fig. 8. One update step:
 *   1. Philox-sampled replay indices and a row gather from the HBM ring buffer;
 *   2. critic stream: target action (actor + tanh-Gaussian head, or TD3 target
 *      actor + smoothing), target critics, TD target, online critics, critic
 *      loss, critic backward;
 *   3. actor stream: actor forward on s, critics at their step-start parameters
 *      on (s, a~), actor loss, backward to the actor, temperature gradient;
 *   4. one fused Adam + Polyak pass over all parameters.
 *
 * Conventions
 *   - Every call returns SPZ_OK (0) or a negative SPZ_E* code; no C++ exception
 *     crosses the ABI. spz_create returns NULL on failure. The message of the
 *     last failure on the calling thread is spz_last_error(NULL); per-context
 *     messages are spz_last_error(ctx).
 *   - Pointers are HOST pointers unless stated. The caller keeps ownership of
 *     every array it passes; the library copies what it needs before returning.
 *   - A context is not thread-safe; distinct contexts are independent.
 *   - Flat parameter layout of one network (spz_read_params / spz_write_params):
 *     layer by layer, W as [out, in] row-major float32, then b [out].
 *     Actor (SAC): obs -> hidden... -> 2*act (mean | log-std); actor (TD3):
 *     obs -> hidden... -> act; critic: (obs | act) -> hidden... -> 1.
 */
#ifndef SPZ_H
#define SPZ_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct spz_ctx spz_ctx;

/* Return codes. */
#define SPZ_OK 0
#define SPZ_EINVAL (-1) /* bad argument (dimension, pointer, hyper-parameter, selector) */
#define SPZ_ENOMEM (-2) /* device or host allocation failed                             */
#define SPZ_EEMPTY (-3) /* spz_update on an empty replay buffer                          */
#define SPZ_ESIZE (-4)  /* caller's array length does not match the requested object     */
#define SPZ_EHIP (-5)   /* a HIP runtime call failed (message has the HIP error string)  */
#define SPZ_EIO (-6)    /* checkpoint file not writable / readable, or not this learner's */

/* Algorithms and GEMM operand precisions. */
#define SPZ_ALGO_SAC 0
#define SPZ_ALGO_TD3 1
#define SPZ_PREC_FP32 0 /* float32 operands, float32 accumulate                        */
#define SPZ_PREC_BF16 1 /* bfloat16 operands (RNE), float32 accumulate, fp32 master    */

/* Selectors for spz_param_count / spz_read_params / spz_write_params. */
#define SPZ_ACTOR 0
#define SPZ_CRITIC1 1
#define SPZ_CRITIC2 2
#define SPZ_TCRITIC1 3
#define SPZ_TCRITIC2 4
#define SPZ_TACTOR 5 /* TD3 only */
#define SPZ_LOG_ALPHA 6
#define SPZ_M_ACTOR 7 /* Adam first moments */
#define SPZ_M_CRITIC1 8
#define SPZ_M_CRITIC2 9
#define SPZ_M_LOG_ALPHA 10
#define SPZ_V_ACTOR 11 /* Adam second moments */
#define SPZ_V_CRITIC1 12
#define SPZ_V_CRITIC2 13
#define SPZ_V_LOG_ALPHA 14
#define SPZ_G_ACTOR 15 /* gradients of the last completed step (read only) */
#define SPZ_G_CRITIC1 16
#define SPZ_G_CRITIC2 17
#define SPZ_G_LOG_ALPHA 18
#define SPZ_N_SELECTORS 19

/* Selectors for spz_debug_read (per-row values of the last step, float32 unless
 * noted; the actor-side values are those of the last step that updated the actor). */
#define SPZ_DBG_INDICES 0   /* int32 [batch]: replay rows sampled by the last step     */
#define SPZ_DBG_TD_TARGET 1 /* [batch]: TD target y                                   */
#define SPZ_DBG_Q 2         /* [2, batch]: online critics q1, q2 on (s, a)            */
#define SPZ_DBG_QPI 3       /* [2, batch]: critics 1, 2 on (s, a~) (TD3: critic 1 twice) */
#define SPZ_DBG_LOGPI 4     /* [batch]: log pi of the actor sample (SAC only)         */
#define SPZ_DBG_DACTION 5   /* [batch, act_dim]: gradient of the actor loss with respect
                               to the actor's action a~ (Section 3.2.2's twin minimum
                               for SAC, critic 1 for TD3)                              */
#define SPZ_DBG_BATCH 6     /* [batch, 2*obs_dim + act_dim + 2]: the transitions the last
                               step gathered from the replay pool (Section 3.3.2), one
                               row (s | a | s' | r | d) per batch row, as the update's
                               kernels read them (bf16 contexts: the stored bfloat16
                               values, widened to float32 exactly)                      */

/* Loss record of one step: 8 floats. */
#define SPZ_REC_LQ 0        /* mean (q1-y)^2 + mean (q2-y)^2                      */
#define SPZ_REC_LPI 1       /* actor loss (0 on TD3 steps without an actor update) */
#define SPZ_REC_LALPHA 2    /* -log(alpha) * mean(log pi + target entropy)         */
#define SPZ_REC_ALPHA 3     /* alpha used by the step                              */
#define SPZ_REC_LOGPI 4     /* mean log pi of the actor sample                     */
#define SPZ_REC_Q1 5        /* mean q1(s, a)                                       */
#define SPZ_REC_NONFINITE 6 /* 1 if any of the values above is not finite          */
#define SPZ_REC_ACTOR 7     /* 1 if the actor was updated in this step             */
#define SPZ_REC_WIDTH 8

/* Hyper-parameters. Fill with spz_hparams_default, then override. */
typedef struct spz_hparams {
  int32_t algo;      /* SPZ_ALGO_SAC | SPZ_ALGO_TD3                                */
  int32_t gemm_prec; /* SPZ_PREC_FP32 | SPZ_PREC_BF16                              */
  int64_t capacity;  /* replay ring rows (> 0)                                     */
  float gamma;       /* discount                                                   */
  float tau;         /* Polyak rate: tbar <- (1-tau) tbar + tau theta, in [0, 1]    */
  float lr_actor, lr_critic, lr_alpha;
  float beta1, beta2, eps; /* Adam                                                 */
  float alpha_init;        /* SAC temperature at step 0 (> 0)                      */
  int32_t learn_alpha;     /* SAC: 1 learns log(alpha) against target_entropy      */
  float target_entropy;
  float log_std_min, log_std_max; /* SAC log-std clamp                             */
  float policy_noise, noise_clip; /* TD3 target policy smoothing                   */
  int32_t policy_delay;           /* TD3: actor and targets every policy_delay steps */
  int32_t device;                 /* HIP device ordinal                            */
  int32_t n_streams;              /* 2: actor and critic on concurrent streams; 1: one stream
                                     (networks narrow enough for row tiles run both in one
                                     launch either way)                               */
  int32_t ordering;               /* SPZ_ORDER_SNAPSHOT | SPZ_ORDER_SEQUENTIAL (below)     */
  int32_t actor_row_split;        /* SAC: 1 takes the actor loss's gradient through each
                                     critic only on the rows where that critic attains
                                     min(Q1, Q2) (the other rows carry zero gradient
                                     there, Section 3.2.2's twin-critic minimum), with
                                     the same results as 0, which takes both critics
                                     over every row. Used where the ReLU masks are kept
                                     as bits (bf16 with 128-multiple hidden widths) and the
                                     layers run one by one.                           */
  int32_t graphs;                 /* 1: spz_update replays each step from a captured HIP
                                     graph (one per step kind: SAC has one, TD3 one with
                                     and one without the delayed actor update) instead of
                                     launching its kernels one by one; bit-identical
                                     results. A graph is captured the first time a step
                                     kind runs (that step itself runs eagerly) and again
                                     after the batch size, the replay fill level or the
                                     seed changed. Ignored while kernel timing is on.  */
} spz_hparams;

/* Update ordering within a step.
 * SPZ_ORDER_SNAPSHOT: every loss of step t reads the parameters of the start of
 *   step t and all Adam / Polyak writes follow both gradients: the actor and the
 *   critics are updated independently (Section 3.2.2); the two halves may run on
 *   concurrent streams.
 * SPZ_ORDER_SEQUENTIAL: the critics take their Adam step (and Polyak) first and
 *   the actor loss of the same step is taken through the updated critics, as in
 *   the published SAC and TD3 algorithms; the temperature uses the step-start
 *   actor sample and alpha. Runs on one stream whatever n_streams says. */
#define SPZ_ORDER_SNAPSHOT 0
#define SPZ_ORDER_SEQUENTIAL 1

/* Defaults: SAC, fp32, capacity 1e6, gamma 0.99, tau 0.005, lr 3e-4, Adam
 * (0.9, 0.999, 1e-8), alpha_init 1, learned alpha, target_entropy 0, log-std
 * clamp [-20, 2], TD3 noise 0.2 clipped to 0.5, delay 2, device 0, 2 streams,
 * snapshot ordering, actor row split on, no graphs. */
void spz_hparams_default(spz_hparams* hp);

/* Create a learner: the single network-update process of Section 3.2 (its actor
 * and double-Q critics with target critics, Section 3.2.2; TD3 adds a target
 * actor), on one GPU. obs_dim, act_dim >= 1; hidden[0..n_hidden) >= 1 with
 * 1 <= n_hidden <= 6; batch >= 1. Parameters are initialised on the host from
 * `seed` with the fan-in uniform rule U(-1/sqrt(fan_in), 1/sqrt(fan_in)) drawn
 * from Philox4x32-10 (counter = (i>>2, 0, 0, net*16 + layer*2 + {W:0,b:1}),
 * word i&3); targets start as exact copies; log(alpha) = ln(alpha_init).
 * `hidden` and `hp` are copied. NULL on failure (see spz_last_error(NULL)). */
spz_ctx* spz_create(int32_t obs_dim, int32_t act_dim, const int32_t* hidden, int32_t n_hidden,
                    int32_t batch, const spz_hparams* hp, uint64_t seed);

/* Release every device and host resource of ctx (NULL is ignored). Waits for
 * the context's outstanding work first. */
void spz_destroy(spz_ctx* ctx);

/* Append n transitions to the replay ring (Section 3.3.2's shared experience
 * pool). Host float32 arrays, row-major: obs [n, obs_dim], act [n, act_dim],
 * rew [n], done [n] (0 or 1), next_obs [n, obs_dim]. Row i goes to slot
 * (ptr + i) mod capacity; size = min(size + n, capacity). bf16 contexts store
 * obs, act and next_obs rounded to bfloat16 (RNE). Synchronous: the arrays may
 * be freed when the call returns. Errors: SPZ_EINVAL (n < 0, or a NULL array
 * with n > 0), SPZ_EHIP. */
int spz_buffer_push(spz_ctx* ctx, const float* obs, const float* act, const float* rew,
                    const float* done, const float* next_obs, int64_t n);

/* Asynchronous form of spz_buffer_push (Section 3.3.2: experience reaches the
 * update process without taking its time). The rows are copied into library-owned
 * pinned staging before the call returns (the caller may reuse its arrays), moved
 * to the device on the library's own ingestion stream, and written into the ring
 * on the stream of the last spz_update (or an internal stream before the first):
 * they are seen by exactly the steps enqueued after this call, and the fill level
 * and write pointer (spz_buffer_size) advance at once. The same sequence of calls
 * therefore gives the same results as with spz_buffer_push. Blocks only when all
 * four staging slots (65536 rows each) still wait for their rows to be committed.
 * Errors: SPZ_EINVAL (n < 0, or NULL with n > 0), SPZ_ENOMEM, SPZ_EHIP. */
int spz_buffer_push_async(spz_ctx* ctx, const float* obs, const float* act, const float* rew,
                          const float* done, const float* next_obs, int64_t n);

/* Rows currently held by the ring (0 .. capacity). */
int64_t spz_buffer_size(const spz_ctx* ctx);

/* Enqueue n_steps update steps on `hip_stream` (a hipStream_t; NULL = the null
 * stream) and return without waiting. One step is one large-batch update of the
 * actor and the critics from a uniform sample of the replay pool (Section 3.2.1,
 * with the two halves updated independently as in Section 3.2.2 and Fig. 3's SAC
 * computation graph). Step t (1-based, counted across calls)
 * samples idx[b] = mulhi32(Philox(seed; b>>2, t, 1, 0)[b&3], size) with
 * replacement, draws its normal deviates from purposes 2 (target) and 3
 * (policy), and ends with the Adam/Polyak pass. Non-finite values do not make
 * the call fail; they set SPZ_REC_NONFINITE in the step's loss record.
 * Errors: SPZ_EEMPTY (no rows), SPZ_EINVAL (n_steps < 0), SPZ_EHIP. */
int spz_update(spz_ctx* ctx, int32_t n_steps, void* hip_stream);

/* Wait for all work the context enqueued. */
int spz_synchronize(spz_ctx* ctx);

/* Actions for the experience-sampling processes (Section 3.1.1: the policy
 * network acts on the observations collected from N samplers; Section 3.1.2: the
 * test and visualisation processes use the policy without randomisation).
 * obs: host float32 [n, obs_dim]; act: host float32 [n, act_dim] (caller-owned).
 * SAC: stochastic = 0 gives the mean action tanh(mu); stochastic = 1 a policy
 * sample tanh(mu + exp(clip(log_std)) eps) with eps from Philox purpose 4 at
 * counter `counter` (step word), element index row * act_dim + j, so a call is
 * reproducible from (seed, counter). TD3: tanh of the actor output (stochastic must
 * be 0; samplers add their own exploration noise). Uses the current online actor
 * with the context's GEMM precision; rows are processed in chunks of at most the
 * created batch. Waits for the context's outstanding work; synchronous.
 * Errors: SPZ_EINVAL, SPZ_EHIP. */
int spz_act(spz_ctx* ctx, const float* obs, int64_t n, int32_t stochastic, uint32_t counter, float* act);

/* spz_act without allocation, for callers that cannot allocate device memory: code
 * under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.
 * obs: DEVICE float32 [n, obs_dim]; act: DEVICE float32 [n, act_dim]; both owned by
 * the caller. Same actions as spz_act (same kernels, bit for bit), enqueued on
 * `hip_stream` (a hipStream_t; NULL = the null stream) without waiting: the actor
 * weights used are the ones current when the kernels run in that stream's order.
 * Intermediate values (observation operand, hidden activations, head output) live
 * in a 64 MiB device array of the library, one per GPU, held until the process ends
 * and shared by every call on that GPU: calls that overlap on one GPU (other streams,
 * other threads, other contexts) race, so order them on one stream or synchronize
 * between them. The call writes every scratch byte it reads, so the previous call's
 * contents do not matter. (Calls that take row tiles keep these values on chip and do not
 * touch the array; which do may change.) n is limited by that array: at most the largest multiple
 * of 256 rows with e * (pad32(obs_dim) + 2 * max_l pad32(hidden[l])) + 4 * pad32(out)
 * bytes per row (e = 2 for bf16 GEMM operands, 4 for fp32; out = 2*act_dim for SAC,
 * act_dim for TD3), plus alignment, within 64 MiB; larger n gives SPZ_EINVAL with
 * the limit in the message. Calls no hipMalloc / hipFree.
 * Errors: SPZ_EINVAL, SPZ_EHIP. */
int spz_act_noalloc(spz_ctx* ctx, const float* obs, int64_t n, int32_t stochastic, uint32_t counter, float* act,
                    void* hip_stream);

/* Checkpoints (the paper publishes weights through files, Section 3.3.1). A file
 * holds the whole learner state: online and target parameters, Adam moments,
 * log(alpha), the step counter, the Philox seed, the loss records and, with
 * SPZ_CKPT_RING, the replay ring with its write pointer and fill level. Loading it
 * into a context with the same dimensions, algorithm and GEMM precision (and ring
 * capacity, if the ring is in the file) continues bit-exactly where the saved one
 * stood. Hyper-parameters (rates, tau, ...) and the batch size are the loading
 * context's own. Both calls wait for the context's outstanding work.
 * Errors: SPZ_EINVAL (NULL), SPZ_EIO (file or mismatch), SPZ_EHIP, SPZ_ENOMEM. */
#define SPZ_CKPT_RING 1
int spz_save(spz_ctx* ctx, const char* path, int32_t flags);
int spz_load(spz_ctx* ctx, const char* path);

/* Batch size of subsequent updates (the paper's adaptive batch size, Sections
 * 3.2.1 and 3.4). 1 <= batch <= the batch given to spz_create, which sizes every
 * batch buffer. Waits for the context's outstanding work. A row's replay index
 * and noise depend only on (seed, step, row), so a context set to `batch`
 * computes what a context created with `batch` computes. Errors: SPZ_EINVAL. */
int spz_set_batch(spz_ctx* ctx, int32_t batch);

/* Current batch size (SPZ_EINVAL for NULL). */
int32_t spz_batch(const spz_ctx* ctx);

/* Adaptive batch size (Section 3.4: geometric enumeration, stopping where the
 * update frame rate saturates). Probes batch sizes b_min, 2 b_min, 4 b_min, ...
 * (the last one capped at the created batch): at each, one untimed update step,
 * then probe_steps timed steps on hip_stream (events); frame rate = batch x steps
 * / seconds. Stops after the first probe that is below (1 + tolerance) x the best
 * rate so far, or at the created batch, then sets the batch to the smallest probed
 * size within (1 - tolerance) of the best rate and returns it in *chosen. The
 * probes are real update steps: they advance the step counter and the networks.
 * batches / frames_per_s (host, max_probes entries, may be NULL when max_probes
 * is 0) receive the probes in order; *n_probes (may be NULL) their number.
 * Synchronous. Errors: SPZ_EINVAL (b_min outside [1, created batch],
 * probe_steps < 1, tolerance outside [0, 1)), SPZ_EEMPTY, SPZ_EHIP. */
int spz_autotune_batch(spz_ctx* ctx, int32_t b_min, int32_t probe_steps, float tolerance, void* hip_stream,
                       int32_t* chosen, int32_t* batches, float* frames_per_s, int32_t max_probes,
                       int32_t* n_probes);

/* Number of update steps enqueued so far (the step counter t of the last step). */
int64_t spz_step(const spz_ctx* ctx);

/* Set the step counter (checkpoint resume, teacher forcing). Waits first. */
int spz_set_step(spz_ctx* ctx, int64_t step);

/* Float count of the object `which` in the flat layout of the published weights
 * (Section 3.3.1; negative code on error). */
int64_t spz_param_count(const spz_ctx* ctx, int32_t which);

/* Copy object `which` to the host array out[0..n_floats): the network weights the
 * update process publishes to the other processes and to checkpoints (Section
 * 3.3.1), plus the optimizer state and gradients. Waits for the context's work first. SPZ_ESIZE if n_floats != spz_param_count(ctx, which);
 * SPZ_EINVAL for a selector the algorithm does not have. */
int spz_read_params(spz_ctx* ctx, int32_t which, float* out, int64_t n_floats);

/* Overwrite object `which` from the host array in[0..n_floats): weights read back
 * from a published copy (Section 3.3.1: checkpoints; also teacher forcing). Gradient selectors are read only (SPZ_EINVAL). */
int spz_write_params(spz_ctx* ctx, int32_t which, const float* in, int64_t n_floats);

/* Copy the loss records of steps first_step .. first_step+n-1 (1-based) into
 * out[n * SPZ_REC_WIDTH]: the critic, actor and temperature losses of each update
 * step of Section 3.2 (the training curves the test process of Section 3.1.2 is
 * there to show), with the non-finite and actor-updated flags. The library keeps the last 65536 records; older or
 * not yet enqueued steps give SPZ_EINVAL. Waits first. */
int spz_read_losses(spz_ctx* ctx, float* out, int64_t first_step, int32_t n);

/* Debug copies of internal state of the last step (see SPZ_DBG_*). `bytes`
 * must equal the object's size (SPZ_ESIZE otherwise). Waits first. */
int spz_debug_read(spz_ctx* ctx, int32_t what, void* out, int64_t bytes);

/* Kernel timing (measurement). While enabled, every kernel launch of
 * spz_update is bracketed by a pair of HIP events recorded on the stream the
 * kernel runs on; spz_profile_read aggregates them per kernel shape. Enabling
 * pre-creates events for `reserve_launches` launches (more are created on
 * demand); disabling drops the records. Waits for the context's work first. */
int spz_profile_enable(spz_ctx* ctx, int32_t on, int64_t reserve_launches);

/* Restrict kernel timing to the launches of one kernel family and shape (as
 * reported by spz_profile_read: name, M, N, K), e.g. so that a timed run carries
 * the events of only the kernel it measures; name NULL times every launch again
 * (the default). Applies to launches enqueued after the call; existing records are
 * kept. `name` is copied. Errors: SPZ_EINVAL (NULL ctx). */
int spz_profile_only(spz_ctx* ctx, const char* name, int32_t M, int32_t N, int32_t K);

/* Time launches only in the update steps whose step number t (1-based, global) is a
 * multiple of `stride` (1, the default: every step), so that a long timed run carries
 * few events; launches outside update steps are timed as before. Applies to steps
 * enqueued after the call. Errors: SPZ_EINVAL (NULL ctx, stride < 1). */
int spz_profile_stride(spz_ctx* ctx, int32_t stride);

/* One aggregated kernel shape. flops / bytes are the algorithmic work of one
 * launch (2*M*N*K for matrix products; bytes the kernel must move for the
 * memory-bound kernels, 0 when not meaningful). */
typedef struct spz_kernel_stat {
  char name[32];   /* kernel family, e.g. "gemm_fwd", "gather", "adam_polyak" */
  int32_t M, N, K; /* launch shape (0 where not applicable)                   */
  int32_t bf16;    /* operand precision of a matrix product                   */
  int64_t launches;
  double total_ms; /* sum of event-measured durations                         */
  double flops;    /* per launch                                              */
  double bytes;    /* per launch                                              */
} spz_kernel_stat;

/* Copy up to max aggregated records (sorted by total time, largest first)
 * into out and their count into *n_out; waits for the context's work first. */
int spz_profile_read(spz_ctx* ctx, spz_kernel_stat* out, int32_t max, int32_t* n_out);

/* ---------------------------------------------------------------------------------------
 * Operators of a recurrent residual block. The policy of a task that one observation does
 * not describe acts on a history: sequences of transitions in training (beside Section
 * 3.2's update process), one step a call for N samplers (as in Section 3.1.1). They are for
 * a learner that the caller builds: a context's networks are feed-forward, its ring holds
 * single transitions, and none of its calls uses them. One block of such a network is
 *     u = norm(x);  f, v, z = products of u;  h = scan(f, v);
 *     x' = x + scale * dropout(gate(z) * norm(h));  u' = norm(x')  (the next block's)
 * Conventions of all of them
 *   - No context. Pointers are DEVICE pointers of the current HIP device, owned by the
 *     caller; work is enqueued on `hip_stream` (a hipStream_t of that device; NULL = the
 *     null stream) without waiting. Nothing is allocated, copied to the host or kept, so
 *     calls may be captured into a HIP graph and may run on any streams and threads at
 *     once, each with its own workspace. The workspace's contents before and after a call
 *     do not matter; it is 16-byte aligned and at least as large as the *_workspace call
 *     of the same arguments says (0: may be NULL).
 *   - `prec` is the type of the named arrays (SPZ_PREC_FP32, SPZ_PREC_BF16). Statistics,
 *     states and sums are float32 and every output is rounded once. Parameter vectors,
 *     their gradients and states are float32.
 *   - Strides are in elements; the last dimension is contiguous. Rows may be any distance
 *     apart (inputs: 0 repeats a row); an output's rows must not overlap each other, nor
 *     any other array of the call unless said otherwise. Any alignment of the element
 *     type is taken; 16-byte aligned rows are faster.
 *   - Every extent may be 0 and is below 2^31, and their product within what a device may
 *     hold (2^38 states, 2^40 to 2^44 elements); a call without elements checks its
 *     arguments and writes what remains (zero sums, the state).
 *   - Results depend on the arguments alone: sums are taken in a fixed order.
 *   - Errors: SPZ_EINVAL (NULL where an array is needed, an extent, stride, selector or
 *     rate out of range, a pointer not aligned to its type), SPZ_ESIZE (workspace too
 *     small), SPZ_EHIP (launch).
 */

/* Gated linear recurrence over `steps` of each of `batch` sequences, `width` channels:
 *     a_t = 1 / (1 + exp(-f_t)),   h_t = a_t k_t h_{t-1} + (1 - a_t) v_t,   y_t = h_t
 * with h_{-1} = h0 and k_t = 0 where reset[t] != 0 (step t starts an episode: nothing of
 * the state before it, finite or not, passes), else 1. Sequence b has lengths[b] steps
 * (clamped to [0, steps]): behind them nothing is read, y is 0 and the state stays, so
 * hT = h of the last step (h0 of an empty sequence). The state is float32 throughout.
 * steps = 1 is the samplers' form; hT may be h0 (the state is updated in place).
 *
 * Backward, from dy and dhT (the gradient to hT): with c = dhT behind the last step,
 *     g_t = dy_t + c,  dv_t = g_t (1 - a_t),  df_t = g_t a_t (1 - a_t) (k_t h_{t-1} - v_t),
 *     c = k_t a_t g_t;   dh0 = c in front of the first step
 * df, dv are 0 behind a sequence's length. It needs `saved` of the forward call with the same
 * f, v, h0, reset and lengths: the states it recomputes h from. */
typedef struct spz_scan_args {
  int64_t batch, steps, width;
  const void *f, *v;                       /* [batch, steps, width]                              */
  int64_t f_batch, f_step, v_batch, v_step;
  const uint8_t* reset;                    /* [batch, steps] or NULL (no episode starts)         */
  int64_t reset_batch, reset_step;
  const int32_t* lengths;                  /* [batch] or NULL (all of them `steps`)              */
  const float* h0;                         /* [batch, width] contiguous, or NULL (zeros)         */
  void* y;                                 /* forward: [batch, steps, width]                     */
  int64_t y_batch, y_step;
  float* hT;                               /* forward: [batch, width] contiguous, or NULL        */
  float* saved;                            /* spz_scan_saved floats: written by the forward call
                                              (NULL: not wanted), read by the backward one       */
  const void* dy;                          /* backward: [batch, steps, width] or NULL (zeros)    */
  int64_t dy_batch, dy_step;
  const float* dhT;                        /* backward: [batch, width] contiguous, or NULL       */
  void *df, *dv;                           /* backward: [batch, steps, width]                    */
  int64_t df_batch, df_step, dv_batch, dv_step;
  float* dh0;                              /* backward: [batch, width] contiguous, or NULL       */
  int32_t prec;                            /* of f, v, y, dy, df, dv                             */
} spz_scan_args;

/* Floats of `saved` (negative code on error). Only batch, steps, width and prec are read. */
int64_t spz_scan_saved(const spz_scan_args* args);
/* Bytes of the workspace (negative code on error). Only batch, steps, width and prec are read. */
int64_t spz_scan_workspace(const spz_scan_args* args, int32_t backward);
int spz_scan_forward(const spz_scan_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream);
int spz_scan_backward(const spz_scan_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* Norms before and after a block, its gate, dropout and residual scale, row by row:
 *     n  = post(h) * w_post + b_post;   o = dropout(gate(z) * n)
 *     x' = x + scale * o;               u = pre(x') * w_pre + b_pre
 * post, pre: none (identity, without w and b), RMS: t / sqrt(mean(t^2) + eps), or layer:
 * (t - mean(t)) / sqrt(mean((t - mean(t))^2) + eps). gate: 1 (z unused), sigmoid(z) or
 * z sigmoid(z). dropout: spz_dropout's, of element row * width + column (drop_p = 0: none).
 * h NULL: no block in front, x' = x, and x_out is not written (may be NULL): the first
 * block's pre norm. Vectors of `width` floats; NULL stands for ones (w_post, w_pre, scale)
 * or zeros (b_post, b_pre). u is taken from x' before x' is rounded. Rows r with
 * valid[r] == 0 are not read: their outputs are zero and they give no gradient.
 *
 * Backward, from dx_out and du (NULL: zeros): dx, dh, dz (rounded to prec) and the sums
 * over the rows dw_post, db_post, dscale, dw_pre, db_pre (float32, written; NULL: not
 * wanted; zeros for the vectors of a norm that is none). dx, dh, dz may be NULL too. */
#define SPZ_NORM_NONE 0
#define SPZ_NORM_RMS 1
#define SPZ_NORM_LAYER 2
#define SPZ_GATE_NONE 0
#define SPZ_GATE_SIGMOID 1
#define SPZ_GATE_SILU 2
typedef struct spz_block_norm_args {
  int64_t rows, width;
  const void *x, *h, *z;                   /* [rows, width]                                      */
  int64_t x_row, h_row, z_row;
  const float *w_post, *b_post, *scale, *w_pre, *b_pre;
  const uint8_t* valid;                    /* [rows] or NULL (all of them)                       */
  void *x_out, *u;                         /* forward: [rows, width]; u NULL where pre is none   */
  int64_t x_out_row, u_row;
  const void *dx_out, *du;                 /* backward: [rows, width]                            */
  int64_t dx_out_row, du_row;
  void *dx, *dh, *dz;                      /* backward: [rows, width]                            */
  int64_t dx_row, dh_row, dz_row;
  float *dw_post, *db_post, *dscale, *dw_pre, *db_pre;
  uint64_t seed;                           /* dropout's, as in spz_dropout                       */
  uint32_t step, tensor;
  float drop_p, eps;                       /* eps: a normal number > 0                             */
  int32_t post, pre, gate;
  int32_t prec;                            /* of x, h, z, x_out, u and their gradients           */
} spz_block_norm_args;

/* Bytes of the backward call's workspace (negative code on error). */
int64_t spz_block_norm_workspace(const spz_block_norm_args* args);
int spz_block_norm_forward(const spz_block_norm_args* args, void* hip_stream);
int spz_block_norm_backward(const spz_block_norm_args* args, void* workspace, int64_t workspace_bytes,
                            void* hip_stream);

/* Dropout whose mask is never stored: y = x * 65536 / (65536 - d) on kept elements, else 0,
 * d = p rounded to 65536ths. Element i = row * width + column is kept when 16-bit word i & 7
 * of Philox4x32-10 (key seed; counter (i >> 3 low 32 bits, step, 5 + 256 (i >> 35), tensor);
 * low half of each 32-bit word first) is at least d. The same call on the gradient is the
 * backward pass. p in [0, 1]. y may be x (with the same row stride). */
int spz_dropout(int32_t prec, int64_t rows, int64_t width, const void* x, int64_t x_row, void* y, int64_t y_row,
                float p, uint64_t seed, uint32_t step, uint32_t tensor, void* hip_stream);

/* 8-bit integers with a scale for each row: scale[r] = max_c |x[r, c]| * (1 / 127), the
 * factor and the product rounded to float32, and q[r, c] = x[r, c] / scale[r] (float32)
 * rounded to the nearest integer, ties to even, within +-127; 0 and 0 for a row of zeros. A row with an
 * infinity or NaN gets a NaN scale and zeros. */
int spz_quant_rows(int32_t prec, int64_t rows, int64_t width, const void* x, int64_t x_row, int8_t* q, int64_t q_row,
                   float* scale, void* hip_stream);

/* Weights q [outer, inner] in the order in which the product reads them, made once per set of
 * weights: spz_quant_image_bytes (negative code on error) bytes, 16-byte aligned. */
int64_t spz_quant_image_bytes(int64_t outer, int64_t inner);
int spz_quant_pack(int64_t outer, int64_t inner, const int8_t* q, int64_t q_row, void* image, void* hip_stream);

/* y[m, n] = s[m] w_scale[n] sum_k q[m, k] w[n, k] + bias[n], with q and s of spz_quant_rows
 * of x (taken within the call) and the sum exact in 32-bit integers (inner <= 131072).
 * x [rows, inner] and y [rows, outer] in `prec`; bias NULL: zeros. For the samplers' few rows
 * (Section 3.1.1) as for whole batches. */
int64_t spz_quant_linear_workspace(int32_t prec, int64_t rows, int64_t outer, int64_t inner);
int spz_quant_linear(int32_t prec, int64_t rows, int64_t outer, int64_t inner, const void* x, int64_t x_row,
                     const void* image, const float* w_scale, const float* bias, void* y, int64_t y_row,
                     void* workspace, int64_t workspace_bytes, void* hip_stream);

/* ---------------------------------------------------------------------------------------
 * Operators of a block whose memory is a matrix, and an optimizer for a learner's own
 * tensors, under the conventions above: norms and rotation of queries and keys, linear
 * attention that forgets at a rate of its own in each head, AdamW over many tensors.
 */

/* Norms of each head of queries and keys, and their rotation by position, in one pass:
 *     n = norm(x) * w + b over the `dim` columns of a head (norm as in spz_block_norm, or none,
 *         where w and b still apply);
 *     pair i < pairs of n is turned by the angle t = positions[row] * freqs[i]:
 *         (a, b) -> (a cos t - b sin t, a sin t + b cos t), and the columns behind stay.
 * layout SPZ_PAIRS_HALVES: pair i is columns i and pairs + i; SPZ_PAIRS_NEIGHBOURS: 2 i and
 * 2 i + 1. 2 pairs <= dim <= 1024. Angles are taken in 64 bits, so positions may be far
 * (off by 2^-52 of the angle, 1e-6 at 2^31 and a frequency of 1). heads_k may be 0 (no
 * keys: any heads' norms). Rows r with valid[r] == 0 are not read: their outputs are zero
 * and they give no gradient. q_out may be q and k_out may be k (with the same strides), as
 * dq may be q or dq_out and dk k or dk_out. Beyond that an output shares no element with another
 * output or an operand (refused where addresses and strides show it).
 *
 * Backward, from dq_out and dk_out (NULL: zeros): dq, dk (NULL: not wanted) and the sums over
 * rows and heads dw_q, db_q, dw_k, db_k (float32 [dim], written; NULL: not wanted). */
#define SPZ_PAIRS_HALVES 0
#define SPZ_PAIRS_NEIGHBOURS 1
typedef struct spz_head_norm_args {
  int64_t rows, heads_q, heads_k, dim, pairs;
  const void *q, *k;                       /* [rows, heads, dim]                                 */
  int64_t q_row, q_head, k_row, k_head;
  const float *w_q, *b_q, *w_k, *b_k;      /* [dim]; NULL: ones and zeros                        */
  const int32_t* positions;                /* [rows]; needed where pairs > 0                     */
  const double* freqs;                     /* [pairs], radians a position                        */
  const uint8_t* valid;                    /* [rows] or NULL (all of them)                       */
  void *q_out, *k_out;                     /* forward: [rows, heads, dim]                        */
  int64_t q_out_row, q_out_head, k_out_row, k_out_head;
  const void *dq_out, *dk_out;             /* backward: [rows, heads, dim]                       */
  int64_t dq_out_row, dq_out_head, dk_out_row, dk_out_head;
  void *dq, *dk;                           /* backward: [rows, heads, dim]                       */
  int64_t dq_row, dq_head, dk_row, dk_head;
  float *dw_q, *db_q, *dw_k, *db_k;        /* backward: [dim]                                    */
  float eps;                               /* a normal number > 0                                */
  int32_t norm, layout;
  int32_t prec;                            /* of q, k, their outputs and gradients               */
} spz_head_norm_args;

/* Bytes of the backward call's workspace (negative code on error). */
int64_t spz_head_norm_workspace(const spz_head_norm_args* args);
int spz_head_norm_forward(const spz_head_norm_args* args, void* hip_stream);
int spz_head_norm_backward(const spz_head_norm_args* args, void* workspace, int64_t workspace_bytes, void* hip_stream);

/* Linear attention over `steps` of each of `batch` sequences, in each of `heads` heads (at most 65536) with a
 * state of key_width x value_width (both at most 256):
 *     S_t = d k_t S_{t-1} + key_t^T value_t,   y_t = scale query_t S_t,   d = exp(-rate[head])
 * with S_{-1} = state and k_t = 0 where reset[t] != 0 (step t starts an episode: nothing of the
 * state before it, finite or not, passes), else 1. An infinite rate is d = 0. Sequence b has
 * lengths[b] steps (clamped to [0, steps]): behind them nothing is read, y is 0 and the state
 * stays, so last = S of the last step (`state` of an empty sequence). The states are float32
 * throughout, in the products too. steps = 1 is the samplers' form; last may be state (updated in place).
 * Queries, keys or values may be shared by heads (stride 0). y may be v (with the same strides).
 * Beyond that an output shares no element with another output or an operand, dstate none with dlast
 * or state (refused where addresses and strides show it).
 *
 * Sequences are worked on in chunks of up to 64 steps: products of queries and keys, and of queries and the
 * state in front, are taken in float32 before the decay and the values meet them. Where such a product (of
 * finite numbers) or exp(-64 rate) passes float32's range, results may be infinite or NaN though S itself
 * is finite, and below the range they are 0; with rates >= 0 and operands and |scale| below 1e6 none passes it.
 *
 * Backward, from dy and dlast (the gradient to last): with C = dlast behind the last step,
 *     G_t = C + scale query_t^T dy_t,  dquery_t = scale dy_t S_t^T,
 *     dkey_t = value_t G_t^T,  dvalue_t = key_t G_t,  C = d k_t G_t;   dstate = C in front of the first step
 * dq, dk, dv are 0 behind a sequence's length; those of shared heads are one for each head. It
 * takes the forward call's `state`; the rates get no gradient. */
typedef struct spz_linear_attention_args {
  int64_t batch, steps, heads, key_width, value_width;
  const void *q, *k, *v;                   /* [batch, steps, heads, key_width or value_width]    */
  int64_t q_batch, q_step, q_head, k_batch, k_step, k_head, v_batch, v_step, v_head;
  const float* rate;                       /* [heads] or NULL (zeros: nothing is forgotten)      */
  const uint8_t* reset;                    /* [batch, steps] or NULL (no episode starts)         */
  int64_t reset_batch, reset_step;
  const int32_t* lengths;                  /* [batch] or NULL (all of them `steps`)              */
  const float* state;                      /* [batch, heads, key_width, value_width] contiguous, or NULL (zeros) */
  void* y;                                 /* forward: [batch, steps, heads, value_width]        */
  int64_t y_batch, y_step, y_head;
  float* last;                             /* forward: as state, or NULL                         */
  const void* dy;                          /* backward: as y, or NULL (zeros)                    */
  int64_t dy_batch, dy_step, dy_head;
  const float* dlast;                      /* backward: as state, or NULL (zeros)                */
  void *dq, *dk, *dv;                      /* backward: as q, k, v                               */
  int64_t dq_batch, dq_step, dq_head, dk_batch, dk_step, dk_head, dv_batch, dv_step, dv_head;
  float* dstate;                           /* backward: as state, or NULL                        */
  float scale;                             /* finite                                             */
  int32_t prec;                            /* of q, k, v, y and their gradients                  */
} spz_linear_attention_args;

/* Bytes of the workspace (negative code on error). Only the extents and prec are read. */
int64_t spz_linear_attention_workspace(const spz_linear_attention_args* args, int32_t backward);
int spz_linear_attention_forward(const spz_linear_attention_args* args, void* workspace, int64_t workspace_bytes,
                                 void* hip_stream);
int spz_linear_attention_backward(const spz_linear_attention_args* args, void* workspace, int64_t workspace_bytes,
                                  void* hip_stream);

/* An AdamW step over `count` tensors at once, each element by itself:
 *     g = grad_scale grad,   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
 *     p = p - lr (m / (1 - beta1^t) / (sqrt(v / (1 - beta2^t)) + eps) + weight_decay p)
 * in float32, the moments with a rounding after each operation in this order (c = 1 - beta in 64
 * bits, then float32: m = beta1 m + c1 g, v = beta2 v + (c2 g) g); p is rounded once to its type,
 * and so is the bfloat16 copy for products to read. m and v are two arrays of `moments` elements
 * for all tensors: tensor i has elements at .. at + n - 1 of both, `at` a multiple of
 * SPZ_ADAMW_BLOCK; what lies between is left as it is. Two tensors may share no element, and
 * a gradient none with another tensor's p or copy.
 *
 * bits 32: m and v are float32. bits 8: m holds codes of m and v codes of sqrt(v) in the 8-bit
 * floating point type e4m3 (1 sign, 4 exponent, 3 mantissa bits, largest 448), m_scale and v_scale
 * a float32 for each SPZ_ADAMW_BLOCK of them: m = code m_scale, v = (code v_scale)^2. A step
 * writes scale = max * (1 / 448) over the block's elements of the tensor (the factor and the
 * product rounded to float32) and rounds x = |m| / scale and sqrt(v) / scale (at most 448) up or
 * down to a value of the type with the probability of its distance: x below 2^-6 has 2^-6 added
 * and taken off again; to its float32 bits 16 w + 8 is added and the low 20 bits are cleared. w is
 * a 16-bit word of Philox4x32-10 (key seed; element e: counter (e >> 2 low 32 bits, low 32 bits of
 * t, 6 + 256 (e >> 34), 0); words 2 (e & 3) for m and the one behind it for v, low half of each 32-bit word
 * first). So small steps count on average, which rounding to nearest would lose. A positive
 * sqrt(v) is at least 2^-9. A scale of 0 gives zeros, a maximum that is not finite a NaN scale and
 * zeros. The step itself uses m and v before they are rounded. */
#define SPZ_ADAMW_BLOCK 256
typedef struct spz_adamw_tensor {
  void* p;                                 /* [n], p_prec: updated in place                      */
  const void* g;                           /* [n], g_prec                                        */
  uint16_t* copy;                          /* bfloat16 [n], written, or NULL                     */
  int64_t n, at;
  double weight_decay;
} spz_adamw_tensor;
typedef struct spz_adamw_args {
  int64_t count, moments;
  const spz_adamw_tensor* tensors;         /* HOST [count], read within the call                 */
  void *m, *v;                             /* [moments]: float32, or 8-bit codes                 */
  float *m_scale, *v_scale;                /* bits 8: [moments / SPZ_ADAMW_BLOCK]                */
  const float* grad_scale;                 /* device [1], or NULL (1)                            */
  const int64_t* step_at;                  /* device [1]: t >= 1, read when the kernel runs, or NULL */
  const float* lr_at;                      /* device [1], as step_at, or NULL                    */
  int64_t step;                            /* t >= 1 where step_at is NULL                       */
  double lr, beta1, beta2, eps;            /* lr where lr_at is NULL; betas in [0, 1), eps >= 0  */
  uint64_t seed;
  int32_t bits, p_prec, g_prec, reserved;  /* reserved: 0                                        */
} spz_adamw_args;
int spz_adamw(const spz_adamw_args* args, void* hip_stream);

/* Message of the last failure: of ctx, or of the calling thread when ctx is
 * NULL. Never NULL; empty when there was none. Valid until the next call. */
const char* spz_last_error(const spz_ctx* ctx);

#ifdef __cplusplus
}
#endif

#endif /* SPZ_H */
