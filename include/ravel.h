/*
 * ravel.h -- C ABI of the MI355X rolling-denoise-step library (libravel.so).
 *
 * One call of ravel_step performs one control step of rolling flow denoising
 * for B independent environments:
 *   - one pass of the flow-matching action expert over every env's H-slot
 *     action buffer, each slot at its own flow time, conditioned on the
 *     env's latest VLM context (layer-wise prefix K/V caches) and its age,
 *     and on Fast-Observation-Pathway tokens (paper Sec. 3.1 Eq. 3, Sec. 3.2
 *     Eq. 4, App. A.1);
 *   - a per-slot Euler update, release of the now-clean first slot as the
 *     env's action, and a fresh N(0, I) action appended in its place by
 *     advancing a ring index (the rule stated right after Eq. 3).
 *
 * Time convention: logical slot i = 0..H-1 holds the action executed i+1
 * steps from now at flow time tau_i = (i+1)/H (1 = noise, 0 = clean), and a
 * step applies a_i <- a_i - (1/H) v_i.  This is the paper's Eq. 3 mirrored
 * (tau_paper = 1 - tau, v_paper = -v, K = H).
 *
 * Threading: ravel_set_context / ravel_context_acquire (the VLM worker, paper
 * Sec. 3.2 and Sec. 4.3's separate workers) may run on another host thread
 * concurrently with ravel_step (the control loop).  Two ravel_step calls on
 * one buffer must not overlap, and consecutive steps must be ordered (same
 * stream, or the caller orders them).
 *
 * Errors: every entry point returns a ravel_status and never throws; the
 * message of the calling thread's last failure is in ravel_last_error().
 * Shape and argument errors are returned synchronously.  Asynchronous device
 * faults surface as RAVEL_E_HIP on a later call that synchronises.  A failed
 * launch of the persistent layers' kernel (a grid barrier or split meeting
 * that timed out) is not left silent: that step and every step enqueued after
 * it release NaN actions and leave the ring and t unchanged, and the next
 * ravel_step / ravel_step_state / ravel_full_denoise / ravel_train_loss call
 * that finds the release kernel's pinned host flag raised (read without
 * synchronising), or the next ravel_buffer_sync / ravel_debug_state, waits for
 * the device, re-arms the kernel's counters and returns RAVEL_E_HIP; the call
 * after that runs normally from the unchanged state.
 *
 * Streams are hipStream_t values passed as void* (NULL = the default stream).
 */
#ifndef RAVEL_H
#define RAVEL_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  RAVEL_OK = 0,
  RAVEL_E_INVALID = -1, /* bad argument (null pointer, out-of-range value)   */
  RAVEL_E_NOMEM = -2,   /* device or host allocation failed                   */
  RAVEL_E_HIP = -3,     /* a HIP runtime call or kernel failed                */
  RAVEL_E_SHAPE = -4,   /* tensor shape or config inconsistent                */
  RAVEL_E_STATE = -5    /* call not valid in the current state (no context,
                           t_obs going backwards, missing weight, ...)        */
} ravel_status;

enum { RAVEL_F32 = 0, RAVEL_BF16 = 1 };

/* Velocity model.  TRANSFORMER is the action expert.  The two analytic fields
 * need no weights beyond one tensor and exist to pin the rolling scheduler:
 *   ANALYTIC_OT:     v_i = (x_i - a*) / tau_i      weight "analytic.target" [D_a]
 *   ANALYTIC_LINEAR: v_i = lambda * x_i            weight "analytic.lambda" [1]   */
enum { RAVEL_TRANSFORMER = 0, RAVEL_ANALYTIC_OT = 1, RAVEL_ANALYTIC_LINEAR = 2 };

typedef struct {
  int32_t layers;      /* L transformer blocks                                  */
  int32_t width;       /* w residual width (even, multiple of 8)                */
  int32_t n_q_heads;   /* query heads                                           */
  int32_t n_kv_heads;  /* KV heads (divides n_q_heads), grouped-query attention */
  int32_t head_dim;    /* hd (multiple of 32, <= 256)                           */
  int32_t mlp_dim;     /* F gated-GeLU hidden size (multiple of 16)             */
  int32_t horizon;     /* H buffer slots (the paper's K), 1..128                 */
  int32_t action_dim;  /* D_a per slot (the paper's h low-level actions folded)  */
  int32_t prefix_len;  /* P prefix tokens of the VLM context per layer (>= 0)    */
  int32_t n_fop;       /* FOP tokens per env (0 disables adapters)              */
  int32_t fop_obs_dim; /* observation size of the FOP stand-in encoder          */
  int32_t fop_stride;  /* adapter in layers l with l % stride == stride - 1     */
  int32_t dtype;       /* RAVEL_F32 or RAVEL_BF16 (bf16 weights/activations,
                          fp32 accumulation, fp32 residual stream and ring)     */
  int32_t model_kind;  /* RAVEL_TRANSFORMER / RAVEL_ANALYTIC_OT / _LINEAR        */
  float delta_bias;    /* delta_0 added to the offset p/H (Sec. 4.4, App. B.1)   */
  float rms_eps;       /* RMSNorm epsilon (1e-6)                                 */
  int32_t offset_mode; /* how the offset delta enters the expert (App. A.1):
                          RAVEL_OFFSET_MLP    an MLP of delta added to the flow-time
                                              embedding (the pi0.5 expert);
                          RAVEL_OFFSET_CONCAT delta concatenated to every slot's noisy
                                              action at the action encoder (the X-VLA
                                              expert): in.w is [w, D_a + 1], its last
                                              column multiplies delta, and the
                                              conditioning is silu(c_tau(i)) alone;
                          RAVEL_OFFSET_ADAPTER delta concatenated with the action and
                                              flow-time embeddings before an
                                              action-time MLP, whose tokens then pass
                                              a gated residual adapter conditioned on
                                              delta's sinusoidal embedding (the
                                              DynamicVLA expert, App. A.1):
                                              e_i = in.w a_i + in.b,
                                              g_i = at.w2 silu(at.w1 [e_i; emb(tau_i);
                                              delta] + at.b1) + at.b2,
                                              h_i = g_i + tanh(ta.alpha) ta.w2
                                              silu(ta.w1 [g_i; emb(delta)] + ta.b1),
                                              emb the flow-time sinusoid; the
                                              conditioning is silu(c_tau(i)) alone;
                                              w a multiple of 32                     */
  float rope_base;     /* 0: no positional encoding of the buffer tokens (the
                          paper's expert); > 0: rotary embedding of their
                          self-attention queries and keys, rotate-half pairs
                          (d, d + hd/2) turned by (P + i) base^(-2d/hd) for
                          logical slot i, the prefix keys used as given        */
} ravel_config;

enum { RAVEL_OFFSET_MLP = 0, RAVEL_OFFSET_CONCAT = 1, RAVEL_OFFSET_ADAPTER = 2 };

/* A named host or device tensor, row-major, [out, in] for linear layers.
 * dtype RAVEL_F32 or RAVEL_BF16 (raw bf16 bits).  Names and shapes:
 *   in.w [w,D_a] ([w,D_a+1] with RAVEL_OFFSET_CONCAT)  in.b [w]
 *   time.w1 [w,w] time.b1 [w] time.w2 [w,w] time.b2 [w]
 *   delta.w1 [w,1] delta.b1 [w] delta.w2 [w,w] delta.b2 [w]  (RAVEL_OFFSET_MLP only)
 *   at.w1 [w,2w+1] at.b1 [w] at.w2 [w,w] at.b2 [w]
 *   ta.w1 [w/4,2w] ta.b1 [w/4] ta.w2 [w,w/4] ta.alpha [1]     (RAVEL_OFFSET_ADAPTER only)
 *   layers.<l>.mod.w [6w,w] .mod.b [6w] .qkv.w [(nq+2nkv)hd,w] .o.w [w,nq hd]
 *   layers.<l>.gate.w [F,w] .up.w [F,w] .down.w [w,F]
 *   adapter layers: layers.<l>.fop.gamma [w] .fop.q.w [nq hd,w]
 *                   .fop.kv.w [2 nkv hd,w] .fop.o.w [w,nq hd] .fop.alpha [1]
 *   final.mod.w [3w,w] final.mod.b [3w] (third chunk unused)  out.w [D_a,w] out.b [D_a]
 *   FOP encoder (optional): fop.w1 [w,d_obs] fop.b1 [w] fop.w2 [n_fop w,w] fop.b2 [n_fop w]
 * The modulation rows of layers.<l>.mod are the chunks (s1,b1,g1,s2,b2,g2) of
 * w rows each: attention-norm scale/shift/gate, MLP-norm scale/shift/gate.  */
typedef struct {
  const char* name;
  int32_t dtype;
  int32_t rank;
  int64_t dims[4];
  const void* data;
} ravel_tensor;

typedef struct ravel_model ravel_model;
typedef struct ravel_buffer ravel_buffer;

/* Build a model on the current HIP device.  Copies every tensor (the caller
 * keeps ownership), converts to the model dtype (bf16 round-to-nearest-even)
 * and lays weights out for the kernels; precomputes each slot's flow-time
 * conditioning c_tau(i), fixed because tau_i is fixed (Sec. 3.1 after Eq. 1).
 * Synchronous.  Errors: E_SHAPE (config or tensor shape), E_STATE (missing
 * weight), E_NOMEM, E_HIP. */
ravel_status ravel_create(const ravel_config* cfg, const ravel_tensor* weights, int32_t n_weights,
                          ravel_model** out);
void ravel_destroy(ravel_model* model);

/* Bytes of device memory held by the model's weights (for roofline accounting). */
int64_t ravel_model_weight_bytes(const ravel_model* model);

/* Create the rolling state of `batch` environments.  Every slot starts as
 * pure N(0, I) noise: initial action r = 0..H-1 of env e sits in physical
 * slot r mod H and is Philox noise for (seed, e, r) (App. A.1: no additional
 * initialisation).  Noise is Philox4x32-10 (Salmon et al., SC'11) keyed by
 * (seed lo, seed hi) with counter (j/4, env, r lo, r hi) and Box-Muller in
 * float64 rounded to float32.  Synchronous.
 * Environment variables read here (each "1" to apply), for tests and comparisons:
 *   RAVEL_NO_PERSISTENT   the per-kernel path even where the persistent kernel is the default;
 *   RAVEL_NO_FUSED_XATTN  a separate attention phase for the FOP adapters in the
 *                         persistent kernel (default for one env with 256-dim heads
 *                         and <= 16 FOP tokens: computed inside the output projection);
 *   RAVEL_NO_SIDE_MOD     the modulation of every layer in one launch before the
 *                         persistent kernel (default: layer 0's only, the others
 *                         computed by blocks the kernel's phases leave idle);
 *   RAVEL_NO_FUSED_PROLOGUE  the persistent step's offset conditioning, input
 *                         projection, layer-0 modulation and FOP keys/values in
 *                         separate launches (default: two launches, same results);
 *   RAVEL_NO_WHOLE_K      split-K items instead of whole-K items for the persistent
 *                         kernel's phases with K <= 1024;
 *   RAVEL_NO_WHOLE_K_GEMM (read once per process) few-row GEMMs with K <= 1024 split
 *                         K across blocks instead of one block per 32 columns;
 *   RAVEL_SYNC_CONTEXT    RAVEL_OPT_SYNC_CONTEXT on;  RAVEL_NO_GRAPH  RAVEL_OPT_USE_GRAPH off;
 *   RAVEL_COOPERATIVE     not supported: set to a nonzero value, buffer creation
 *                         fails with RAVEL_E_INVALID (the persistent kernel is
 *                         launched ordinarily; its waits are bounded). */
ravel_status ravel_buffer_create(ravel_model* model, int32_t batch, uint64_t seed, ravel_buffer** out);
void ravel_buffer_destroy(ravel_buffer* buf);

/* Options (ravel_buffer_set_option):
 *   RAVEL_OPT_SYNC_CONTEXT  1: a published context is applied at the very next
 *                           step, which waits on the GPU (not the host) for its
 *                           data; 0 (default): applied at the first step whose
 *                           host-side event query finds the data ready.
 *   RAVEL_OPT_USE_GRAPH     1 (default): replay a captured hipGraph per step (the
 *                           whole step after the host's publish check, on either
 *                           execution path; one graph per pointer set); 0: launch
 *                           the step's kernels eagerly.
 *   RAVEL_OPT_DEBUG         1: synchronise and check for NaN/Inf after each kernel.
 *   RAVEL_OPT_PERSISTENT    1 (available for a bf16 model whose B*H rows fit one 64-row
 *                           tile, of width up to 2048 with the MLP offset form and 4096
 *                           otherwise; the default up to 3 layers of width 512): run the
 *                           transformer layers as a single persistent kernel (one
 *                           block per CU, grid barriers between phases) between the
 *                           few kernels around it; 0: one kernel per operation.
 *                           E_STATE if the buffer does not qualify.
 *   RAVEL_OPT_FAIL_LAYERS   test hook, 1: mark the persistent layers' kernel as failed
 *                           (synchronises, then sets its error word as a grid barrier
 *                           that timed out would; every later launch then returns at
 *                           once and the error handling described at the top of this
 *                           file takes over).  E_STATE on a buffer without the
 *                           persistent kernel. */
enum { RAVEL_OPT_SYNC_CONTEXT = 1, RAVEL_OPT_USE_GRAPH = 2, RAVEL_OPT_DEBUG = 3, RAVEL_OPT_PERSISTENT = 4,
       RAVEL_OPT_FAIL_LAYERS = 5 };
ravel_status ravel_buffer_set_option(ravel_buffer* buf, int32_t option, int64_t value);

/* Context plane (paper Sec. 3.2: the latest available context is reused
 * across steps until a newer one is ready; refreshing never blocks a step).
 *
 * Each env owns two device context slots; steps read the active one.
 * ravel_context_acquire returns device pointers to the env's inactive slot,
 * K and V each [L, P, n_kv, hd] in the model dtype, after making `producer`
 * wait (on the GPU) until no enqueued step still reads that slot.  The
 * producer writes the new context there (e.g. its own kernels), then calls
 * ravel_set_context with k = v = NULL.  Acquiring cancels a publish of this
 * env that has not yet been applied.
 *
 * ravel_set_context publishes a context for env (0..B-1) computed from the
 * observation of control step t_obs.  With non-NULL k and v (host or device,
 * [L, P, n_kv, hd] model dtype) it first copies them into the inactive slot
 * on `producer` (acquire + copy); the sources must stay valid until that copy
 * has run.  env = -1 publishes one context per env at once: k and v are then
 * [B, L, P, n_kv, hd] (env e's block at offset e * L*P*n_kv*hd) and must not be
 * NULL; t_obs is checked for every env before anything is copied (E_STATE for
 * all if one env's would decrease).  The swap happens at a later ravel_step: the slot index flips in
 * device memory and the step's offset becomes p = t - t_obs.  t_obs must not
 * decrease per env (E_STATE).  Never blocks on the GPU. */
ravel_status ravel_context_acquire(ravel_buffer* buf, int32_t env, void** k_slot, void** v_slot,
                                   void* producer_stream);
ravel_status ravel_set_context(ravel_buffer* buf, int32_t env, const void* k, const void* v,
                               int64_t t_obs, void* producer_stream);

/* One rolling denoise step for all envs, enqueued on `stream` (asynchronous).
 *   fop_tokens: device [B, n_fop, w] in the model dtype (NULL only when the
 *               model has no adapters);
 *   action_out: device float [B, D_a], the action released by this step.
 * The step number t lives in device memory (starts at 0, +1 per step).
 * Errors: E_STATE if some env has no context yet (transformer model). */
ravel_status ravel_step(ravel_buffer* buf, const void* fop_tokens, float* action_out, void* stream);

/* FOP stand-in encoder z = reshape(W_f2 gelu_tanh(W_f1 obs + b_f1) + b_f2)
 * (paper Eq. 4 with a 2-layer MLP in place of the image encoder).
 *   obs: device float [B, d_obs]; fop_tokens: device [B, n_fop, w] model dtype. */
ravel_status ravel_fop_encode(ravel_buffer* buf, const float* obs, void* fop_tokens, void* stream);

/* ravel_fop_encode for callers that cannot allocate device memory -- code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc: the
 * same encoder (same kernels, same results as ravel_fop_encode on a buffer of
 * `batch` envs) without a buffer, its staging rows, split-K partials and tickets
 * kept in a fixed device array of 16 MiB that the library holds on every GPU it
 * runs on until the process ends (set up by ravel_create on the device current
 * then).  Calls no allocating routine; enqueued on `stream` (its tickets are
 * cleared with a kernel, not a memset).
 *   obs: device float [batch, d_obs]; fop_tokens: device [batch, n_fop, w] model dtype.
 * Every call on one GPU shares that GPU's array (the last call's contents stay):
 * calls that overlap on one GPU (different streams or threads without ordering)
 * race and must be serialised by the caller.  Errors: E_INVALID (null pointer, or
 * a batch whose workspace exceeds the fixed array -- the message gives both sizes),
 * E_SHAPE (batch < 1), E_STATE (no FOP encoder weights, or no model created on
 * the current device). */
ravel_status ravel_fop_encode_noalloc(const ravel_model* model, int32_t batch, const float* obs, void* fop_tokens,
                                      void* stream);

/* Wait until every enqueued step and context copy of this buffer finished. */
ravel_status ravel_buffer_sync(ravel_buffer* buf);

/* Synchronises, then copies the state out (any pointer may be NULL):
 *   X_host float [B, H, D_a] ring in PHYSICAL slot order (slot (t+i) mod H is
 *   logical slot i); t = step counter; t_obs_host int64 [B]. */
ravel_status ravel_debug_state(ravel_buffer* buf, float* X_host, int64_t* t, int64_t* t_obs_host);

/* Facts about a buffer's execution (for tests and tooling):
 *   RAVEL_Q_GRAPHS      step graphs captured so far (one per (fop, state, action)
 *                       pointer set and execution path while RAVEL_OPT_USE_GRAPH is on;
 *                       a set's first step is launched directly, its second captures);
 *   RAVEL_Q_PERSISTENT  1 if the transformer layers run as the persistent kernel;
 *   RAVEL_Q_PHASES      phases of that kernel's list (0 on the per-kernel path);
 *   RAVEL_Q_STEPS       steps enqueued (the host's copy of t).
 * Errors: E_INVALID (null pointer, unknown key). */
enum { RAVEL_Q_GRAPHS = 1, RAVEL_Q_PERSISTENT = 2, RAVEL_Q_PHASES = 3, RAVEL_Q_STEPS = 4 };
ravel_status ravel_buffer_query(ravel_buffer* buf, int32_t key, int64_t* value);

/* Publish log: entries (env, t_apply, t_obs) as int64 triples, oldest first.
 * On input *n is the capacity in entries; on output the number written. */
ravel_status ravel_publish_log(ravel_buffer* buf, int64_t* entries, int32_t* n);

/* Bit-exact checkpoint of the rolling state (ring, t, seed, per-env t_obs and
 * active context).  Call with host_blob = NULL to get the size in *n.
 * Synchronises.  Load requires a buffer of the same model and batch. */
ravel_status ravel_buffer_save(ravel_buffer* buf, void* host_blob, size_t* n);
ravel_status ravel_buffer_load(ravel_buffer* buf, const void* host_blob, size_t n);

/* Relative actions (App. B.1, pi0.5 on RoboTwin 2.0; App. B.3, DynamicVLA): a model that
 * predicts actions relative to the robot state keeps its buffer across a moving state by
 * holding the clean targets absolute, converting them relative to the latest state before
 * each expert pass and back afterwards, with the paired noise in model coordinates.  On the
 * buffer of noisy actions this is a shift of every slot i by (1 - tau_i) * (s_prev - s) on
 * the relative dimensions before the pass (s_prev: the state of the env's previous step; no
 * shift at its first step), and the released action is slot 0 plus s on those dimensions.
 * ravel_set_relative_dims marks the relative dimensions: mask [D_a] host int32, nonzero =
 * relative (NULL or all zero: absolute actions, the default); only before the first step
 * (RAVEL_E_STATE after).  With relative dimensions set, every step is ravel_step_state:
 * ravel_step with state [B, D_a] fp32 device, the latest robot state in the actions'
 * normalised units (ravel_step is then RAVEL_E_STATE, as is ravel_step_state without
 * relative dimensions).  The analytic OT field's target is then absolute. */
ravel_status ravel_set_relative_dims(ravel_buffer* buf, const int32_t* mask);
ravel_status ravel_step_state(ravel_buffer* buf, const void* fop_tokens, const float* state, float* action_out,
                              void* stream);

/* Full-horizon synchronous denoising: the baseline rolling inference is compared with
 * (Sec. 4.1 synchronous evaluation and App. B.1: the same budget of expert passes spent on
 * full-horizon denoising steps, and the first-action latency table of Sec. 4.1).  A fresh
 * chunk of H slots per env starts as the given noise at flow time 1; every slot shares one
 * flow time, and `steps` Euler steps of size 1/steps -- step k evaluates the expert with
 * every slot at tau = (steps - k)/steps and applies chunk -= v / steps -- bring it to 0.
 * Each step is one expert pass over the chunk with the buffer's contexts at age 0 (offset
 * delta = delta_bias) and the given FOP tokens (as in ravel_step; NULL only for a model
 * without adapters).  Context publications are applied first exactly as ravel_step applies
 * them (and logged at the current step index).  Analytic models use their velocity field
 * at the shared tau.
 *   noise: [B, H, D_a] fp32, device; chunk_out: [B, H, D_a] fp32, device (may be noise
 *   itself); chunk_out holds the denoised chunk when the stream reaches the end of the call.
 *   steps: 1 .. 1024.
 * Does not touch the rolling ring or the step counter t; it shares the buffer's
 * activations with ravel_step, so it must not overlap a step (or
 * another call of this) on the same buffer.  The first call with a given step count builds
 * that count's flow-time conditioning table on the device and synchronises; later calls
 * enqueue on `stream` and return.  Errors: RAVEL_E_INVALID (null pointers, missing FOP
 * tokens), RAVEL_E_SHAPE (steps), RAVEL_E_STATE (an env without a context). */
ravel_status ravel_full_denoise(ravel_buffer* buf, int32_t steps, const void* fop_tokens, const float* noise,
                                float* chunk_out, void* stream);

/* Streaming-aligned training objective, forward and loss (Sec. 3.3, Eq. 5 and 6): for
 * every sample e of the batch, the training buffer at the rolling flow-time profile,
 * slot i = tau_i * noise + (1 - tau_i) * target with tau_i = (i+1)/H (this build's time
 * direction: the paper's (1 - tau_k) eps + tau_k a_hat), one expert pass with the buffer's
 * context of sample e as the observation-time context and offset delta = ages[e] / H
 * (no lead bias delta_0), and loss[e] = (1/H) sum_i ||v_i - (noise_i - target_i)||^2 (the
 * paper's ||v - (a_hat - eps)||^2 with velocities of the opposite sign).
 *   target, noise: [B, H, D_a] fp32, device (slot i = the action i+1 steps after t_a);
 *   ages: [B] int64, device, context age p = t_a - t_o per sample;
 *   fop_tokens: as ravel_step; loss_out: [B] fp32, device;
 *   v_out: optional [B, H, D_a] fp32, device: the predicted velocities (NULL: none; may be
 *   target or noise itself).
 * Context publications are applied first as ravel_step applies them.  Does not touch the
 * ring or t; shares the buffer's activations with ravel_step (no overlap on one buffer).
 * No backward pass.  Errors: RAVEL_E_INVALID (null pointers, missing FOP tokens),
 * RAVEL_E_STATE (a sample without a context). */
ravel_status ravel_train_loss(ravel_buffer* buf, const float* target, const float* noise, const int64_t* ages,
                              const void* fop_tokens, float* loss_out, float* v_out, void* stream);

/* Per-kernel timing of one eagerly launched step (HIP events around every
 * launch on `stream`; synchronises).  Each record: kernel class name,
 * algorithmic bytes and flops of that launch, and its duration.  With the
 * persistent path on, further records "persistent/<phase class>" split the
 * "persistent_layers" record by phase class (time between the kernel's grid
 * barriers as seen by its first block, summed over layers), followed by one
 * record "phase/<index>/<phase class>" per phase in launch order; neither kind
 * is an additional launch.  Launches whose row count is decided on the device
 * (the modulation GEMMs run on the rows of distinct offset conditionings,
 * class "gemm_rows") carry bytes = flops = 0.  Contexts in 8 bits count the
 * tokens that they hold: "cache_attn", "cache_join" (the join of its key ranges)
 * and, while tracking, "cache_weight".  On input *n is the
 * capacity; on output the number of records. */
typedef struct {
  char name[48];
  double bytes;
  double flops;
  float ms;
} ravel_kernel_record;
ravel_status ravel_profile_step(ravel_buffer* buf, const void* fop_tokens, float* action_out,
                                void* stream, ravel_kernel_record* records, int32_t* n);

/* -------------------------------------------------------------------------
 * Key/value cache in 8 bits.
 *
 * A cache holds, for each of n_seq sequences, the keys and values of up to `capacity` tokens as
 * e4m3 codes (8-bit floating point, largest value 448) with one 32-bit scale per (sequence, KV
 * head, block of `block` tokens), for keys and values apart; token t's key is code * scale of
 * block t / block.  Scales are powers of two from 2^-100 on, the smallest by which the block's
 * largest magnitude stays within 448 when the block is written: division and products by them
 * are exact, so a stored value is off by at most half an e4m3 step (2^-4 of it, 2^-10 of the
 * scale below the format's normal numbers).  All memory is the caller's device memory on the current
 * device; the struct may be copied and is read during the call only.  k and v must be 16-byte
 * aligned.  The calls are enqueued on `stream` and allocate nothing; they may be captured into a
 * graph, and read lengths, indices and positions from device memory when they run.  Calls that
 * write one sequence must be ordered with every other call on it.  Codes, scales and weights behind
 * a sequence's length are no part of any result and need not be initialised (unless an append skips
 * them: tokens between the length and its pos become the sequence's as they are).
 *
 *   seq  [batch] device int32: the sequence of each batch row; NULL: row b is sequence b.  A row
 *        whose index is outside 0..n_seq-1 (say -1, for padding) takes no part in the call.
 * ------------------------------------------------------------------------- */
typedef struct {
  int32_t n_seq;
  int32_t n_kv_heads;
  int32_t head_dim; /* 32, 64, 128 or 256                                      */
  int32_t capacity; /* tokens of a sequence, 1 .. 2^24                         */
  int32_t block;    /* tokens of a scale: 16, 32, 64 or 128                    */
  int32_t reserved; /* 0 */
  void* k;          /* [n_seq, n_kv_heads, capacity, head_dim] e4m3            */
  void* v;
  float* k_scale;   /* [n_seq, n_kv_heads, ceil(capacity / block)]             */
  float* v_scale;
  int32_t* len;     /* [n_seq] tokens held (values outside 0..capacity count
                       as the nearer bound)                                    */
  float* weight;    /* [n_seq, n_kv_heads, capacity] accumulated attention
                       weights, or NULL                                        */
} ravel_cache;

/* Store the keys and values of up to n new tokens per batch row from position pos[b] on (NULL: from
 * the sequence's length on); the length becomes pos[b] + the tokens stored, so a smaller pos takes
 * earlier tokens back.  count[b] (NULL: n) of the row's n tokens are stored, clamped to 0..n, and
 * no more than fit; a row with pos outside 0..capacity is left alone.
 *   k, v: device, dtype RAVEL_F32 or RAVEL_BF16, element (b, t, h, d) at b * batch_stride +
 *   t * token_stride + h * head_stride + d (in elements; 16-byte aligned rows: strides multiples
 *   of 8, or 4 in 32 bits).
 * A block that also holds older tokens keeps its scale, or, where the new tokens need a larger one,
 * has its older codes rounded to that.  Infinities become the largest code, NaN stays NaN; neither
 * counts for the scale.  Magnitudes from 1.9375 * 2^127 on round to 2^128, which is infinite in 32 bits.  Accumulated weights of the stored tokens start at 0.  seq, pos and count
 * must not lie in the cache's len (but pos == len is taken as NULL).  A sequence that an earlier row names
 * already is not written again.
 * Errors: E_INVALID (null pointer, alignment, dtype, block), E_SHAPE (sizes, strides). */
ravel_status ravel_cache_append(const ravel_cache* cache, int32_t batch, const int32_t* seq, const int32_t* pos,
                                const int32_t* count, int32_t n, int32_t dtype, const void* k, const void* v,
                                int64_t batch_stride, int64_t token_stride, int64_t head_stride, void* stream);

/* Attention of `rows` query rows per batch row and head over [cached tokens ; own tokens]: the
 * sequence's len tokens, then the n_self tokens whose keys and values come with the call in the
 * queries' dtype (every row sees all of both; query head j uses KV head j / (n_q_heads /
 * n_kv_heads)).  out = softmax(scale q k) v; scores, softmax and sums in 32 bits, in a bf16 call the
 * probabilities are rounded to bf16 for the second product (with many rows of up to 128 dims those of
 * 32 keys a second time, where the next 32 raise the row's maximum far) and out at the end; in a 32-bit
 * call products are as good as 32 bits.  Values of magnitudes up to 2^90 leave the sums finite.  A row
 * that sees nothing (len 0 and no own tokens, or no sequence) is 0.  With track, every cached token's
 * softmax weights, summed over the rows and the query heads of its KV head, are added to the cache's
 * accumulated weight (batch rows that name one sequence are added in row order).  out shares no element
 * with the inputs; scale is in 0..2^100.
 * Strides in elements, (b, row or token, head); 16-byte aligned vectors (multiples of 8 elements, or
 * 4 in 32 bits).  workspace: ravel_cache_attention_workspace() bytes, 256-byte aligned, of this call
 * alone until it has run (NULL when that is 0). */
typedef struct {
  int32_t dtype; /* RAVEL_F32 or RAVEL_BF16: q, self_k, self_v, out */
  int32_t batch;
  int32_t n_q_heads;
  int32_t rows;   /* query rows per batch row, >= 1            */
  int32_t n_self; /* own tokens per batch row, >= 0            */
  int32_t track;  /* nonzero: add to the accumulated weights   */
  float scale;    /* of the scores, e.g. 1 / sqrt(head_dim)    */
  int32_t reserved;
  const int32_t* seq;
  const void* q;
  const void* self_k;
  const void* self_v;
  void* out;
  int64_t q_stride[3];
  int64_t self_stride[3]; /* of self_k and of self_v */
  int64_t out_stride[3];
  void* workspace;
  int64_t workspace_bytes;
} ravel_cache_query;

/* Bytes of workspace for such a call (only the sizes of both structs are read), in *bytes. */
ravel_status ravel_cache_attention_workspace(const ravel_cache* cache, const ravel_cache_query* query, int64_t* bytes);
/* Errors: E_INVALID (null pointer, alignment, dtype, workspace too small, track without weights),
 * E_SHAPE (sizes, strides, head counts). */
ravel_status ravel_cache_attention(const ravel_cache* cache, const ravel_cache_query* query, void* stream);

/* Evict: of each (batch row, KV head) the `keep` tokens with the largest accumulated weights stay (of
 * equal ones those of lower index; NaN counts as the lowest; the sequence's first `first` tokens stay
 * in any case), each head its own; a sequence of at most keep tokens loses none.  Kept tokens of index
 * below keep stay at their places, the others fill the holes in ascending order (attention does not
 * depend on the order of the tokens); codes, scales and weights go along, and the length becomes
 * min(len, keep).  A block's scale becomes the largest of its tokens' scales, codes of smaller ones
 * are rounded to it.
 *   into NULL: in place.  Otherwise the kept tokens go to sequence into_seq[b] (NULL: b) of that
 *   cache, which shares no memory with the first, has the same heads, head_dim and block, and a
 *   capacity of at least min(keep, capacity); the first cache is left as it is.
 *   kept: [batch, n_kv_heads, keep] device int32: the index each place's token had, -1 for places
 *   beyond the tokens kept (all of them for a row without a sequence).
 * workspace: ravel_cache_evict_workspace() bytes, 256-byte aligned, of this call alone until it has
 * run.  A destination that an earlier row names already is not written again.
 * kept and the workspace lie in neither cache, seq and into_seq not in the cache that is written
 * (its len, say), kept or the workspace.
 * Errors: E_INVALID (null pointer, no weights, workspace too small, shared memory), E_SHAPE (sizes,
 * first > keep). */
ravel_status ravel_cache_evict_workspace(const ravel_cache* cache, int32_t batch, int32_t keep, int64_t* bytes);
ravel_status ravel_cache_evict(const ravel_cache* cache, int32_t batch, const int32_t* seq, int32_t keep, int32_t first,
                               const ravel_cache* into, const int32_t* into_seq, int32_t* kept, void* workspace,
                               int64_t workspace_bytes, void* stream);

/* A buffer that holds its contexts in such a cache (otherwise as ravel_buffer_create makes it): its steps
 * read half the bytes of a bf16 model's contexts (a quarter in 32 bits), and scales, accumulated weights
 * and an eviction's indices included they take 51 % of their memory with heads of 256 dims and 56 % of 32
 * (25 and 28 % in 32 bits).
 * ravel_set_context stores the given keys and values, in the model dtype, through ravel_cache_append's
 * kernel, which reads them where they lie if that is 16-byte aligned memory of the buffer's device.
 * Others are copied first, into staging rows of one context in the model dtype that the first such call
 * allocates and the buffer keeps (as much as another half of one env's contexts, which a single env's
 * buffer then takes in full; E_NOMEM).  k and v must not be NULL: there is no zero-copy publication, and
 * ravel_context_acquire is E_STATE.
 * Every expert pass attends through ravel_cache_attention's kernels; one kernel per operation
 * (RAVEL_OPT_PERSISTENT is E_STATE).  Sequence (slot * batch + env) * layers + layer of the cache holds
 * one layer's prefix, slot 0 or 1.  Saved states go with buffers of the same block only.
 * Errors: as ravel_buffer_create; E_SHAPE for analytic models, models without prefix tokens or with a
 * head_dim that the cache does not take; E_INVALID (block). */
ravel_status ravel_buffer_create_quantized(ravel_model* model, int32_t batch, uint64_t seed, int32_t block,
                                           ravel_buffer** out);

/* on != 0: every later expert pass over this buffer's contexts adds the softmax weights that its self-
 * attention gives the prefix tokens to their accumulated weights (a token's start at 0 when its context
 * is stored); 0 (the default): not.  E_STATE on a buffer without a quantized context. */
ravel_status ravel_context_track(ravel_buffer* buf, int32_t on);

/* ravel_cache_evict, in place, on every layer of env's active context (env = -1: of every env's),
 * enqueued on `stream` in the order of the steps: later passes attend over the `keep` tokens of each
 * layer and KV head with the largest accumulated weights.  The next context published starts whole.
 * Must be ordered with the buffer's steps as these are among themselves.  Errors: E_STATE (no quantized
 * contexts, an env without an applied context), E_INVALID (env), E_SHAPE (keep < 1, first outside 0..keep). */
ravel_status ravel_context_evict(ravel_buffer* buf, int32_t env, int32_t keep, int32_t first, void* stream);

/* env's active context as a cache of `layers` sequences in the buffer's own memory, for reading and for
 * the ravel_cache_* calls; it stays the active one until a step applies a newer context.  E_STATE (no
 * quantized contexts, no applied context), E_INVALID (null pointer, env). */
ravel_status ravel_context_cache(ravel_buffer* buf, int32_t env, ravel_cache* cache);

/* -------------------------------------------------------------------------
 * A layer's operators, with their gradients: gated residual and norm, cross attention, gated MLP.
 *
 * What an expert layer computes between its linear layers, as calls of their own, for programs that
 * train on the loss above or run adapters of their own.  All memory is the caller's device memory on
 * the current device; the structs are read during the call only.  The calls are enqueued on `stream`,
 * allocate nothing and may be captured into a graph.  Elements of a tensor's innermost dimension are
 * adjacent; other strides are in elements.  Tensors of RAVEL_BF16 and RAVEL_F32 are 16-byte aligned
 * with strides of whole 16 bytes; vectors of 32-bit numbers that modulate rows likewise.  Inputs and
 * outputs share no memory unless a call says so.  A workspace is ...workspace() bytes, 256-byte
 * aligned, of this call alone until it has run (NULL when that is 0); the sizes come from the
 * struct's sizes and from which of its pointers are NULL.  No result depends on the order in which
 * blocks run: sums over rows are formed in one order, with no atomics.
 *
 * 1. Gated residual and norm.  For rows r of `width` elements:
 *
 *      F = f, or f / rms(f) * (1 + post) with post           rms(z) = sqrt(mean z^2 + eps)
 *      t = x + alpha * gate * F                              (x without f)
 *      y = t / rms(t) * (1 + scale) + shift
 *
 * x and t (x_out) have stream_dtype, f and y dtype; post, alpha, gate, scale and shift are 32-bit,
 * each NULL where it is not there.  gate, scale and shift are vectors of `width` with stride 0, or
 * hold `mods` rows, of which row r uses (r / group) % mods: rows of their own (group 1, mods =
 * rows), one for each environment (group = its rows), one for each slot (group 1, mods = slots).
 * The norm is that of t as x_out holds it.  Sums are in 32 bits: the squares of a row have to be
 * finite there.
 * ------------------------------------------------------------------------- */
typedef struct {
  int32_t stream_dtype; /* of x, x_out and their gradients                    */
  int32_t dtype;        /* of f, y and their gradients; RAVEL_BF16 with a
                           RAVEL_BF16 stream                                  */
  int32_t rows;         /* 0 .. 2^23 - 1                                      */
  int32_t width;        /* multiple of 8, <= 8192                             */
  int32_t mods;         /* rows of gate, scale and shift, >= 1                */
  int32_t group;        /* neighbouring rows that share one, >= 1             */
  float eps;            /* > 0                                                */
  int32_t reserved;     /* 0 */
  const void* x;        /* [rows, width]                                      */
  const void* f;        /* [rows, width], the block's output, or NULL         */
  const float* post;    /* [width], or NULL: f is taken as it is              */
  const float* alpha;   /* one number, or NULL: 1                             */
  const float* gate;    /* or NULL: 1                                         */
  const float* scale;   /* or NULL: 0                                         */
  const float* shift;   /* or NULL: 0                                         */
  void* x_out;          /* [rows, width]; NULL without f; may be x            */
  void* y;              /* [rows, width], or NULL: only the residual          */
  int64_t x_stride, f_stride, x_out_stride, y_stride, gate_stride, scale_stride, shift_stride;
} ravel_norm;

/* Errors: E_INVALID (null pointer, alignment, dtype, eps), E_SHAPE (sizes, strides). */
ravel_status ravel_norm_residual(const ravel_norm* norm, void* stream);

/* Its gradients: dy and d_out are those of y and x_out (either may be NULL: zero), every output may be
 * NULL.  Of the struct above, x_out is read (x without f), f, post, alpha, gate and scale; x (with f),
 * y and shift are not.  A vector's gradient is summed over all rows, a modulation row's over the rows
 * that use it (0 if none does).  dx may be d_out. */
typedef struct {
  const void* dy;    /* [rows, width], dtype               */
  const void* d_out; /* [rows, width], stream_dtype        */
  void* dx;          /* [rows, width], stream_dtype        */
  void* df;          /* [rows, width], dtype; needs f      */
  float* dpost;      /* [width]; needs post                */
  float* dalpha;     /* one number; needs alpha            */
  float* dgate;      /* as gate; needs gate                */
  float* dscale;     /* as scale; needs scale              */
  float* dshift;     /* [mods, width], or [width] with stride 0 */
  int64_t dy_stride, d_out_stride, dx_stride, df_stride;
  int64_t dgate_stride, dscale_stride, dshift_stride; /* 0 where the vector's is (dshift: where it is summed over all rows) */
  void* workspace;
  int64_t workspace_bytes;
} ravel_norm_grad;
ravel_status ravel_norm_residual_grad_workspace(const ravel_norm* norm, const ravel_norm_grad* grad, int64_t* bytes);
/* Errors: as above; E_INVALID also for a workspace too small or a gradient of what is not there. */
ravel_status ravel_norm_residual_grad(const ravel_norm* norm, const ravel_norm_grad* grad, void* stream);

/* 2. Cross attention: `rows` query rows per batch row over `keys` states of another length.
 *
 *      out = softmax(scale q k^T) v      over the first k_len[b] keys, for the first q_len[b] rows
 *
 * Query head j uses KV head j / (n_q_heads / n_kv_heads); every row sees all of its batch row's keys.
 * Keys behind k_len and rows behind q_len take no part, whatever they hold: out is 0 for such rows and
 * for all rows of a batch row without keys.  lse, if given, is the logarithm of each row's sum of
 * exp(scale q k), -infinity for rows that are 0.  Scores, softmax and sums are in 32 bits; in bf16
 * calls probabilities (and in the gradients the scores') are rounded to bf16 before they are
 * multiplied, outputs at the end, and the gradients take out as it was rounded (but not for up to 32
 * keys): results are 2.3e-3 off 64 bits where rounding them alone makes 1.7e-3, gradients of rows that
 * one key dominates up to 5.9e-3.  Calls in RAVEL_F32 round nothing in between (4e-7 and 7e-6).  scale
 * is 0 or in 2^-100..2^100. */
typedef struct {
  int32_t dtype; /* RAVEL_F32 or RAVEL_BF16: q, k, v, out and their gradients */
  int32_t batch;
  int32_t n_q_heads;  /* at most 256                            */
  int32_t n_kv_heads; /* divides n_q_heads                      */
  int32_t head_dim;   /* 32, 64, 128 or 256                     */
  int32_t rows;       /* 0 .. 2^20; batch * n_kv_heads * tiles of rows
                         (times query heads of a KV head) or, for dk and
                         dv, of keys: below 2^24 (tiles of at least 64;
                         of 16 up to 32 rows or 64 keys)        */
  int32_t keys;       /* 0 .. 2^24                              */
  float scale;        /* of the scores, e.g. 1 / sqrt(head_dim) */
  const int32_t* q_len; /* [batch] or NULL: rows; outside 0..rows: the nearer bound */
  const int32_t* k_len; /* [batch] or NULL: keys; likewise                          */
  const void* q;
  const void* k;
  const void* v;
  void* out;
  float* lse;           /* [batch, n_q_heads, rows], or NULL (the gradients need it) */
  int64_t q_stride[3];  /* (batch row, row or key, head); the latter two at most 2^22 bytes */
  int64_t k_stride[3];
  int64_t v_stride[3];
  int64_t out_stride[3];
  void* workspace;      /* of ravel_cross_attention */
  int64_t workspace_bytes;
} ravel_cross;

ravel_status ravel_cross_attention_workspace(const ravel_cross* cross, int64_t* bytes);
/* Errors: E_INVALID (null pointer, alignment, dtype, scale, workspace too small), E_SHAPE (sizes,
 * strides, head counts). */
ravel_status ravel_cross_attention(const ravel_cross* cross, void* stream);

/* Its gradients from dout, with out and lse as the call above left them.  dk and dv sum over the query
 * heads of their KV head; gradients of keys behind k_len and of rows behind q_len are 0.  dq may be
 * NULL, and so may dk and dv together.  dout behind q_len is not read. */
typedef struct {
  const void* dout;
  void* dq;
  void* dk;
  void* dv;
  int64_t dout_stride[3];
  int64_t dq_stride[3];
  int64_t dk_stride[3];
  int64_t dv_stride[3];
  void* workspace;
  int64_t workspace_bytes;
} ravel_cross_grad;
ravel_status ravel_cross_attention_grad_workspace(const ravel_cross* cross, const ravel_cross_grad* grad, int64_t* bytes);
ravel_status ravel_cross_attention_grad(const ravel_cross* cross, const ravel_cross_grad* grad, void* stream);

/* 3. Gated MLP, up to its hidden values: h = act(x Wg^T) * (x Wu^T), products and activation in 32 bits.
 * gate and up, if given, receive x Wg^T and x Wu^T, for the gradients: in dtype, or with RAVEL_GATE_F32 in
 * 32 bits.  A bf16 call's gradients are 2.3e-3 off 64 bits with gate and up in 32 bits, 3.1e-3 in bf16, where
 * rounding the results alone makes 1.7e-3. */
enum { RAVEL_GELU_TANH = 0, RAVEL_SILU = 1, RAVEL_GATE_F32 = 256 };
typedef struct {
  int32_t dtype;    /* RAVEL_F32 or RAVEL_BF16, of all tensors      */
  int32_t act;      /* RAVEL_GELU_TANH or RAVEL_SILU; | RAVEL_GATE_F32:
                       gate and up are RAVEL_F32 whatever dtype     */
  int32_t rows;     /* 0 .. 2^28                                    */
  int32_t width;    /* of x: multiple of 8, <= 2^18                 */
  int32_t hidden;   /* of h: multiple of 8, <= 2^18                 */
  int32_t reserved; /* 0 */
  const void* x;    /* [rows, width]                                */
  const void* wg;   /* [hidden, width]                              */
  const void* wu;   /* [hidden, width]                              */
  void* h;          /* [rows, hidden]                               */
  void* gate;       /* [rows, hidden], or NULL; with up             */
  void* up;         /* [rows, hidden], or NULL; with gate           */
  int64_t x_stride, w_stride, h_stride, gate_stride; /* of a row; w_stride of wg and wu, gate_stride of gate and up;
                                                       at most 2^22 bytes */
  void* workspace;  /* of ravel_gated_mlp, which needs none so far */
  int64_t workspace_bytes;
} ravel_mlp;

ravel_status ravel_gated_mlp_workspace(const ravel_mlp* mlp, int64_t* bytes);
/* Errors: E_INVALID (null pointer, alignment, dtype, workspace too small), E_SHAPE (sizes, strides). */
ravel_status ravel_gated_mlp(const ravel_mlp* mlp, void* stream);

/* Its gradients from dh, with gate and up as the call above left them; h is not read.  dx may be NULL,
 * and so may dwg and dwu together.  act says what gate and up are, as above.  Their gradients, dh * up *
 * act'(gate) and dh * act(gate), are rounded to dtype before they are multiplied. */
typedef struct {
  int32_t weight_dtype; /* of dwg and dwu: dtype or RAVEL_F32 */
  int32_t reserved;     /* 0 */
  const void* dh;       /* [rows, hidden], dtype  */
  void* dx;             /* [rows, width], dtype   */
  void* dwg;            /* [hidden, width]        */
  void* dwu;            /* [hidden, width]        */
  int64_t dh_stride, dx_stride, dw_stride; /* of a row; dw_stride of dwg and dwu */
  void* workspace;
  int64_t workspace_bytes;
} ravel_mlp_grad;
ravel_status ravel_gated_mlp_grad_workspace(const ravel_mlp* mlp, const ravel_mlp_grad* grad, int64_t* bytes);
ravel_status ravel_gated_mlp_grad(const ravel_mlp* mlp, const ravel_mlp_grad* grad, void* stream);

/* Message of the calling thread's last non-OK status ("" if none). */
const char* ravel_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* RAVEL_H */
