/*
 * reflex.h -- C ABI of the MI355X (gfx950) Reflex denoise hot path.
 *
 * The library computes the per-denoising-step forward of a flow-matching
 * action expert over a three-region KV cache, following the paper "Reflex:
 * Real-Time Vision-Language-Action Control through Streaming Inference":
 *
 *   - a pinned static prefix (language tokens), written once (Section 3.1);
 *   - a sliding FIFO window of the last W observation frames, held in a
 *     pre-allocated ring and overwritten in O(1) per frame (Section 3.1,
 *     Section 3.4 "Ring Buffer Architecture", Appendix B.1-B.2);
 *   - a dynamic suffix (one state token + H action tokens) recomputed at every
 *     Euler step; attention over [static; window; dynamic] is Eq. 1 and equals
 *     full-batch attention (Appendix A, Proposition A.1).
 *
 * Every layer uses AdaRMSNorm with fp32 statistics (Eq. 2, Section 3.2),
 * packed QKV and gate|up projections (Section 3.4 "Operator Fusion"), and the
 * chunk is integrated with explicit Euler from noise at tau = 1 to actions at
 * tau = 0.
 *
 * Memory ownership: the caller allocates and owns every device buffer
 * (weights, cache, workspace, inputs, outputs).  The library never allocates
 * or frees device memory; it owns only the host-side context.  All device
 * work is enqueued on the stream given to reflex_cache_init and is
 * asynchronous unless stated otherwise.  A context is bound to one stream and
 * is not thread-safe.
 *
 * Status codes: 0 on success, a negative REFLEX_E* value on failure;
 * reflex_strerror() describes a code (and the last HIP error for
 * REFLEX_EHIP).  On failure no context state changes.
 */
#ifndef REFLEX_H
#define REFLEX_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define REFLEX_OK 0
#define REFLEX_EINVAL (-1)   /* null pointer, bad shape or unsupported size */
#define REFLEX_EDTYPE (-2)   /* weight dtype differs from the config's dtype */
#define REFLEX_EHIP (-3)     /* a HIP call or kernel launch failed */
#define REFLEX_ESTATE (-4)   /* context not initialised or already destroyed */
#define REFLEX_ENONFINITE (-5) /* reflex_check_status: a denoise produced a non-finite action */
#define REFLEX_ESCRATCH (-6) /* reflex_denoise_chunk_static: the chunk needs more scratch than
                                the library's static device array holds */

#define REFLEX_DTYPE_F32 0
#define REFLEX_DTYPE_BF16 1

#define REFLEX_MOD_FULL 0        /* y = n(x)(1+scale)+shift; h += gate * f(y) */
#define REFLEX_MOD_SCALE_ONLY 1  /* shift = 0, gate = 1: Eq. 2 exactly */

#define REFLEX_MAX_STEPS 64

/* Precision of the residual stream and of the RMS statistics of every
 * AdaRMSNorm.  REFLEX_NORM_FP32 is the method (fp32 statistics, Section 3.2).
 * The other two reproduce the baselines of the stability stress test
 * (Section 4.6): a bf16 residual stream with the statistics accumulated in
 * bf16 (every product and partial sum rounded to bf16), and a bf16 residual
 * stream with fp32 statistics ("FP32 norm-only"). */
#define REFLEX_NORM_FP32 0
#define REFLEX_NORM_BF16 1
#define REFLEX_NORM_BF16_FP32_STATS 2

/* Attention kernel of the bf16 path.  All compute the same masked softmax
 * over [static; ring window; dynamic] (Eq. 1) and agree to rounding.
 * REFLEX_ATTN_AUTO picks by the launch geometry: one wave pair per 32 query
 * rows when the launch would reach one key tile per split (a few envs and a
 * short context; heads of 128 also two), two four-wave teams per 128 query
 * rows with up to 64 key splits (a few envs, more keys, head_dim 128 or 256),
 * otherwise 16-row waves sharing each key tile over 128 query rows,
 * software-pipelined (a tile's scores and softmax run under the previous
 * tile's P.V MFMAs).  REFLEX_ATTN_ROWS16 forces the 16-row kernel
 * without that pipelining (the same results bit for bit); the other values
 * force one kernel (tests, tuning).  The fp32 path has one kernel and
 * ignores the field. */
#define REFLEX_ATTN_AUTO 0
#define REFLEX_ATTN_ROWS16 1
#define REFLEX_ATTN_PAIR 2
#define REFLEX_ATTN_ROWS16_PIPE 3

/*
 * Shape of the action expert and of the cache.
 *
 * Model: n_layers transformer layers of width `width`; a gated-GELU MLP of
 * width mlp_dim; n_q_heads query heads sharing n_kv_heads K/V heads of size
 * head_dim; one state token (state_dim) and action_horizon action tokens
 * (action_dim each) form the dynamic region (T = 1 + action_horizon rows).
 * The conditioning MLP of each AdaRMSNorm site maps c = [sinusoidal(tau) (width
 * values); state] through cond_hidden SiLU units to 3*width outputs
 * (scale, shift, gate).  Sites: 2*l (attention norm of layer l), 2*l+1 (MLP norm
 * of layer l), 2*n_layers (final norm before the action head).
 *
 * Cache: static_len prefix tokens; window_frames ring slots of frame_tokens
 * tokens, plus one spare slot when spare_slot = 1 (the pipelined ring of the
 * reflex_pipeline_* calls: frame f then goes to slot f mod (window_frames + 1),
 * and a chunk still sees exactly window_frames frames).
 * frame_dim > 0: frames arrive as [frame_tokens, frame_dim]
 * embeddings and K/V come from the per-layer frame projection w_kv;
 * frame_dim == 0: frames arrive as pre-RoPE per-layer K/V.  batch independent
 * environments advance in lockstep and share the weights.
 *
 * Numerics: dtype is the storage/compute type of weights, cache and GEMM
 * operands (accumulation, statistics, residual stream and actions are fp32).
 * RoPE: rotate-half, base rope_theta; positions are absolute: static
 * 0..static_len-1, frame f token j at static_len + f*frame_tokens + j, dynamic
 * token i at static_len + frames_written*frame_tokens + i.  The token embeddings
 * are multiplied by embed_scale.
 *
 * Supported by this build: n_kv_heads == 1; head_dim in {64, 128, 256};
 * width, mlp_dim, cond_hidden multiples of 64; state_dim, action_dim, frame_dim
 * multiples of 8; dynamic rows T <= 128 per env.
 */
typedef struct reflex_config {
  int32_t n_layers;
  int32_t width;
  int32_t mlp_dim;
  int32_t n_q_heads;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t state_dim;
  int32_t action_dim;
  int32_t action_horizon;
  int32_t cond_hidden;
  int32_t static_len;
  int32_t frame_tokens;
  int32_t window_frames;
  int32_t frame_dim;
  int32_t batch;
  int32_t dtype;       /* REFLEX_DTYPE_* */
  int32_t mod_mode;    /* REFLEX_MOD_* */
  int32_t max_steps;   /* largest num_steps a denoise call may use (<= 64) */
  float rms_eps;
  float embed_scale;
  double rope_theta;
  double temb_min_period;
  double temb_max_period;
  int32_t spare_slot;      /* 0 or 1, see "Cache" above */
  int32_t norm_precision;  /* REFLEX_NORM_*: REFLEX_NORM_FP32 for the method */
  int32_t attn_kernel;     /* REFLEX_ATTN_*: REFLEX_ATTN_AUTO unless forcing one */
} reflex_config;

/*
 * Device pointers to the weights, row-major, rows are output features
 * (y = x W^T), element type `dtype`.  The library reads them in place; they
 * must stay valid and unchanged for the life of the context.
 *
 *   w_qkv  [n_layers][(Hq + 2) * head_dim][width]  rows: q heads, k, v
 *   w_o    [n_layers][width][Hq * head_dim]
 *   w_gu   [n_layers][2 * mlp_dim][width]           rows: gate, then up
 *   w_down [n_layers][width][mlp_dim]
 *   w_state[width][state_dim]
 *   w_ain  [width][action_dim]
 *   w_aout [action_dim][width]
 *   w_mod1 [2*n_layers+1][cond_hidden][width + state_dim]
 *   w_mod2 [2*n_layers+1][3 * width][cond_hidden]  rows: scale, shift, gate
 *   w_kv   [n_layers][2 * head_dim][frame_dim]     rows: k, then v; NULL when
 *                                                   frame_dim == 0
 *
 * dtype: the element type the caller's framework reports for the output
 * projection w_o (the dtype probe of Section 3.2 "Robust Dtype Inference").
 */
typedef struct reflex_weights {
  const void* w_qkv;
  const void* w_o;
  const void* w_gu;
  const void* w_down;
  const void* w_state;
  const void* w_ain;
  const void* w_aout;
  const void* w_mod1;
  const void* w_mod2;
  const void* w_kv;
  int32_t dtype;
} reflex_weights;

/* Host-side bookkeeping of one FIFO write (Section 3.1; Appendix B.1). */
typedef struct reflex_ring_step {
  int64_t frame_index; /* f: index of the frame being written (0-based)      */
  int32_t slot;        /* ring slot f mod W                                   */
  int32_t n_valid;     /* frames visible after the write: min(f + 1, W)       */
  int64_t pos0;        /* absolute position of the frame's first token        */
  int64_t dyn_pos0;    /* absolute position of dynamic token 0 afterwards     */
  int32_t evicted;     /* tokens evicted by the write: frame_tokens if f >= W */
  int32_t reserved;
} reflex_ring_step;

typedef struct reflex_ctx reflex_ctx;

/*
 * Bytes the caller must allocate for the cache and the workspace.  Pure host
 * function (no device calls).  Both buffers need 256-byte alignment.
 *
 * Cache layout (element type `dtype`), R = static_len + (window_frames + spare_slot)*frame_tokens:
 *   K at offset 0:           [batch][n_layers][R][head_dim]   RoPE applied
 *   V at offset K bytes:     [batch][n_layers][head_dim][R]   stored transposed
 * Rows [0, static_len) hold the static prefix; ring slot s holds rows
 * [static_len + s*frame_tokens, static_len + (s+1)*frame_tokens).
 * The first 32 bytes of the workspace hold the device tick state as four
 * int64 values {frames_written, n_valid, dyn_pos0, hole_row} (read-only for
 * callers): the frames, window length and dynamic position the next chunk
 * uses, and the logical cached row from which the physical rows skip the
 * spare slot (a value past the window means no skip).  Bytes 32..35 hold the
 * status word that reflex_check_status reads.  The rest of the workspace is
 * private scratch of the library.
 * The caller allocates both buffers once, before the control loop: no
 * allocation happens per frame or per chunk (the pre-allocated ring and
 * buffers of Section 3.4 and Appendix B.2).
 * Returns REFLEX_EINVAL for an unsupported config.
 */
int reflex_query_sizes(const reflex_config* cfg, size_t* cache_bytes, size_t* workspace_bytes);

/*
 * Validate the config, check the weights' dtype against cfg->dtype (dtype
 * probe, Section 3.2), bind the caller's buffers and write the pinned static
 * prefix: K rows get RoPE at positions 0..static_len-1, V rows are copied.
 *
 * static_k, static_v: device, [batch][n_layers][static_len][head_dim], pre-RoPE,
 * element type dtype; read during this call's stream work only.
 * cache_mem / workspace_mem: device buffers of the sizes reflex_query_sizes
 * returned.  stream: a hipStream_t (NULL = the null stream).
 * On success *out receives a new context with frames_written = 0.
 * Errors: REFLEX_EINVAL, REFLEX_EDTYPE, REFLEX_EHIP; *out untouched on error.
 */
int reflex_cache_init(const reflex_config* cfg, const reflex_weights* w, void* cache_mem,
                      void* workspace_mem, const void* static_k, const void* static_v,
                      void* stream, reflex_ctx** out);

/*
 * Write one new frame for all envs (FIFO, incremental prefill of the newest
 * frame only, Section 3.1): slot f mod W is overwritten; K gets RoPE at
 * positions static_len + f*frame_tokens + j.
 *
 * frame: device, element type dtype;
 *   frame_dim > 0:  [batch][frame_tokens][frame_dim] embeddings;
 *   frame_dim == 0: [batch][n_layers][2][frame_tokens][head_dim] pre-RoPE K, V.
 * frame_index_out / evicted_tokens_out (nullable host pointers) receive f and
 * the evicted token count (the eviction count of add_new_prefix, Appendix B.1).
 * The host metadata is returned synchronously; the device work is async.
 * Errors: REFLEX_EINVAL, REFLEX_ESTATE, REFLEX_EHIP; on error f is not advanced.
 */
int reflex_cache_write_frame(reflex_ctx* ctx, const void* frame, int64_t* frame_index_out,
                             int32_t* evicted_tokens_out);

/*
 * Denoise one action chunk per env over the current cache (static prefix +
 * the n_valid written frames + the dynamic region), num_steps Euler steps.
 *
 * state:  device fp32 [batch][state_dim]
 * noise:  device fp32 [batch][action_horizon][action_dim], x at tau_0
 * actions_out: device fp32 [batch][action_horizon][action_dim], x at tau_K;
 *         may alias noise.
 * tau_schedule: fp32 array of num_steps + 1 values, tau_0 = 1 > ... >
 *         tau_K = 0, or NULL for tau_k = 1 - k/num_steps (the uniform Euler
 *         grid from noise at tau = 1, Section 3.2).  Host memory, or device
 *         memory: a device array is copied to the host on the context's
 *         stream and that copy is waited for, so the call then blocks until
 *         the stream's earlier work is done.
 * The cache is only read (timestep invariance, Section 3.1).  An empty ring
 * is allowed.  Launches are captured once into a HIP graph per distinct
 * (pointers, num_steps, schedule) and replayed.
 * Timing: a wait for this chunk queued on another stream while the chunk
 * runs (an event wait in another hardware queue) lengthens the gaps between
 * its kernels: a batch-1 pi0 chunk took 9.78 ms against 8.73 ms without one.
 * Queue work that depends on the result on this context's stream, or order
 * other streams after it once it has completed.
 * Errors: REFLEX_EINVAL (null pointer, num_steps outside [1, max_steps]),
 * REFLEX_ESTATE, REFLEX_EHIP.
 */
int reflex_denoise_chunk(reflex_ctx* ctx, const float* state, const float* noise, int32_t num_steps,
                         const float* tau_schedule, float* actions_out);

/* Cache strategies of the comparison in Section 4 (Baselines) and the
 * partitioned-attention ablation table of Section 4.6. */
#define REFLEX_MODE_REFLEX 0   /* the method: cached regions read, dynamic K/V fresh at every step */
#define REFLEX_MODE_STANDARD 1 /* full history recomputation: before every Euler step the static
                                  prefix and every window frame are encoded into the cache again */
#define REFLEX_MODE_NAIVE 2    /* a K/V cache that ignores the timestep: the dynamic K/V computed at
                                  the first Euler step are reused at every later step */
#define REFLEX_MODE_UNFUSED 3  /* the method without operator fusion (the fusion ablation of Section
                                  4.6): conditioning MLPs at every step, RoPE, gated GELU, residual add,
                                  norm, action head and Euler update as separate launches */

/* Sources the Standard strategy re-encodes at every step. */
typedef struct reflex_sources {
  const void* static_k;       /* device, as given to reflex_cache_init (may be NULL if static_len == 0) */
  const void* static_v;
  const void* const* frames;  /* host array of n_frames device pointers, each laid out as the frame
                                 argument of reflex_cache_write_frame, oldest first: frames[i] is frame
                                 number frames_written - n_frames + i */
  int32_t n_frames;           /* must equal n_valid = min(frames_written, window_frames) */
  int32_t reserved;
} reflex_sources;

/*
 * reflex_denoise_chunk under a chosen cache strategy, for the comparisons of
 * Section 4: the full-recomputation "Standard" baseline and the "Naive Cache"
 * negative control.  Arguments as reflex_denoise_chunk, plus:
 *   mode: REFLEX_MODE_REFLEX (identical to reflex_denoise_chunk),
 *         REFLEX_MODE_STANDARD, REFLEX_MODE_NAIVE or REFLEX_MODE_UNFUSED;
 *   src:  required for REFLEX_MODE_STANDARD, ignored otherwise (may be NULL).
 *         The frame and static buffers are read by the device work of this
 *         call and must stay unchanged until it completes.
 * Standard re-writes every window frame into its own slot at its own absolute
 * positions and the static prefix at positions 0..static_len-1 before each
 * step, with the same kernels as reflex_cache_write_frame; the cache bytes
 * therefore end up unchanged and the actions equal those of the method.  The
 * graph of a Standard call is also keyed by frames_written and the source
 * pointers.  Naive keeps one set of dynamic K/V per layer in the workspace.
 * Errors: REFLEX_EINVAL (unknown mode, missing or inconsistent sources, and as
 * reflex_denoise_chunk), REFLEX_ESTATE, REFLEX_EHIP.
 */
int reflex_denoise_chunk_baseline(reflex_ctx* ctx, int32_t mode, const reflex_sources* src,
                                  const float* state, const float* noise, int32_t num_steps,
                                  const float* tau_schedule, float* actions_out);

/*
 * Asynchronous pipeline (Section 3.3): a producer writes frames on a stream of
 * its own while the context's stream denoises chunks over frames whose write
 * has completed, so the two overlap on the GPU.  Both calls need a context
 * created with cfg.spare_slot = 1: the ring then has window_frames + 1 slots
 * and the frame being written never lands in a slot that an in-flight chunk
 * reads.  Ordering between the two streams is done on the device with events;
 * neither call blocks the host.
 *
 * reflex_pipeline_write_frame: reflex_cache_write_frame with the device work
 * enqueued on writer_stream (a hipStream_t; may be the context's stream).  On
 * the device it first waits for the previous frame write and for every chunk,
 * enqueued earlier, whose window contains the frame in the target slot.  It
 * does not change the frames a chunk sees: each chunk picks its window.
 * The frame buffer must stay unchanged until the write has completed.
 *
 * reflex_pipeline_denoise_chunk: reflex_denoise_chunk on the context's stream
 * over the window of the first n_frames frames (frames max(0, n_frames - W) ..
 * n_frames - 1, dynamic tokens at positions static_len + n_frames*frame_tokens
 * + i).  With F frames written so far, n_frames must lie in [max(0, F - 1), F];
 * the context's stream waits on the device for the write of frame
 * n_frames - 1.  n_frames = -1 takes F if the newest write has completed when
 * the call is made, else F - 1 (the consumer querying the latest cache state;
 * the host never waits).  *n_frames_out (nullable) receives the value used.
 * reflex_denoise_chunk on such a context is this call with n_frames = F.
 *
 * Errors: REFLEX_EINVAL (cfg.spare_slot == 0, n_frames outside the range, and
 * as the calls they extend), REFLEX_ESTATE, REFLEX_EHIP.  The Standard
 * strategy of reflex_denoise_chunk_baseline is not available on a context
 * with a spare slot (it would re-encode frames on the context's stream while
 * the writer stream uses the same scratch); the Naive strategy is.
 */
int reflex_pipeline_write_frame(reflex_ctx* ctx, const void* frame, void* writer_stream,
                                int64_t* frame_index_out, int32_t* evicted_tokens_out);
int reflex_pipeline_denoise_chunk(reflex_ctx* ctx, const float* state, const float* noise,
                                  int32_t num_steps, const float* tau_schedule, float* actions_out,
                                  int64_t n_frames, int64_t* n_frames_out);

/*
 * reflex_denoise_chunk for callers that cannot allocate (code under HIP graph
 * capture, tight serving loops, harnesses that forbid allocation): the same
 * chunk, with the same kernels and the same results, but the chunk's
 * transient buffers (modulation, residual stream, activations, attention and
 * split-K partials) live in one static device array of the library
 * (64 MiB, allocated with the library's code on each device it runs on and
 * held until the process ends) instead of the context's workspace, and the
 * launches are enqueued directly on the context's stream (no graph is
 * instantiated).  No hipMalloc, hipFree or allocating library routine is
 * called.  Arguments, the tau schedule and the window as for
 * reflex_denoise_chunk; only the method's strategy is offered.
 * Every call on a device shares that device's array: calls that overlap on
 * one device (two contexts on two streams, or a call while another's work is
 * still in flight on another stream) race and give wrong results; calls in
 * stream order, on any contexts, are safe.  The array keeps the last call's
 * contents; the call clears what its kernels need zeroed.
 * Errors: REFLEX_ESCRATCH when the chunk needs more than 64 MiB (16 MiB at
 * batch 1 at the pi0 shapes with max_steps 10, so up to batch 4 fits; the
 * transient bytes grow with batch and max_steps), and as reflex_denoise_chunk.
 */
int reflex_denoise_chunk_static(reflex_ctx* ctx, const float* state, const float* noise, int32_t num_steps,
                                const float* tau_schedule, float* actions_out);

/*
 * Status of the chunks denoised on this context since the last check: waits
 * for the context's stream, reads and clears the device status word, and
 * returns REFLEX_ENONFINITE when any action written by the method's final
 * kernel was NaN or infinite (the NaN/Inf events that the BF16 stability
 * comparison of Section 4.6 counts), else 0.  Denoise calls stay
 * asynchronous; the check is the one synchronizing call.
 * Errors: REFLEX_ESTATE, REFLEX_EHIP.
 */
int reflex_check_status(reflex_ctx* ctx);

/* Release the host context and its captured graphs; never frees caller
 * memory (the caller-owned cache and workspace of Section 3.4's
 * pre-allocated buffers outlive it).  NULL is a no-op.  Returns 0. */
int reflex_destroy(reflex_ctx* ctx);

/* Text for a status code (for REFLEX_EHIP, the last HIP error string). */
const char* reflex_strerror(int status);

/*
 * Bookkeeping of writing frame number frames_written into a ring of
 * window_frames slots (pure host function, Section 3.1 FIFO; Appendix B.2).
 * Errors: REFLEX_EINVAL for a null out, a negative frames_written or
 * non-positive sizes.
 */
int reflex_ring_plan(int64_t frames_written, int32_t window_frames, int32_t frame_tokens,
                     int32_t static_len, reflex_ring_step* out);

/* Frames written so far into the context (host mirror).  Returns a negative
 * status for a NULL context. */
int64_t reflex_frames_written(const reflex_ctx* ctx);

/*
 * Per-kernel-class device timing (diagnostics).  While enabled, every
 * reflex_denoise_chunk and reflex_cache_write_frame runs its launches eagerly
 * (no graph) with hipEvents around each launch and synchronizes the context's
 * stream before returning; reflex_profile_read then returns the summed
 * milliseconds and launch counts per class of the last such call (the class
 * names are "embed_norm", "gemm_qkv", "attention", "attn_merge", "gemm_o",
 * "resid_norm", "gemm_gate_up", "gemm_down", "final_euler", "modulation",
 * "rope_table", "frame_proj", "ring_write").
 * n_classes in/out: capacity of the arrays in, number written out.
 */
int reflex_profile_enable(reflex_ctx* ctx, int enable);
int reflex_profile_read(reflex_ctx* ctx, const char** names, double* ms, int32_t* launches,
                        int32_t* n_classes);

/*
 * Device time of some kernel classes inside the chunk's graph (diagnostics;
 * the launch-level timing of Appendix D's measurement).  One
 * reflex_denoise_chunk call (same arguments and rules; it computes and writes
 * actions_out) is captured into a HIP graph in which every launch of a class
 * whose bit is set in class_mask (bit i: class i in reflex_profile_read's
 * order) is bracketed by one-thread kernels that write the GPU's wall clock:
 * two back to back before it, one after.  Per launch the time is (t2 - t1) -
 * (t1 - t0), the bracket minus the cost of a launch boundary measured at the
 * same point of the graph, so every kernel runs in the chunk's own order and
 * cache state.  The graph is replayed once untimed and then reps times, the
 * stamps read back after each.  Out: the summed milliseconds of the selected
 * classes per chunk (mean over the replays) and their launches per chunk (0
 * and 0 when they launch nothing).  Allocates and frees a stamp buffer;
 * synchronizes the stream.  Errors: REFLEX_ESTATE, REFLEX_EINVAL (null
 * pointers, num_steps out of range, reps < 1, no known class selected),
 * REFLEX_EHIP.
 */
int reflex_profile_graph(reflex_ctx* ctx, const float* state, const float* noise, int32_t num_steps,
                         const float* tau_schedule, float* actions_out, uint32_t class_mask, int32_t reps,
                         double* ms_per_replay, int32_t* launches);

/*
 * ---------------------------------------------------------------------------
 * Backbone operators: rotary positions, the paged cache and its attention
 * ---------------------------------------------------------------------------
 *
 * The cache above takes pre-RoPE K/V of its prefix and frames from a
 * vision-language backbone.  These calls are what such a backbone runs to
 * produce them: rotary positions over several axes, a paged K/V cache that may
 * hold 8-bit values, and the attention of a chunk of new tokens over it.  They
 * need no reflex_ctx.
 *
 * Memory and streams: every buffer belongs to the caller; nothing is allocated
 * and no call waits for the device.  Work is enqueued on `stream` (a
 * hipStream_t, NULL = the null stream) of the current device, on which every
 * buffer has to lie; it may be captured into a HIP graph, which then reads the
 * device arrays (lengths, page table, positions) anew at every replay.  The
 * host structs are read during the call only.  The calls keep no state, so
 * several threads may make them at once.
 *
 * Element types: `dtype` (REFLEX_DTYPE_*) is the type of queries, keys, values
 * and results outside the cache.  Arithmetic is fp32 or wider and results are
 * rounded once; only the attention rounds before that, its probabilities.
 */

/* Packed rows of heads: element (row r, head h, d) at data[r*row_stride +
 * h*head_stride + d], strides in elements.  data is 16-byte aligned and the
 * strides are multiples of 16 bytes.  Rows of an output must not overlap. */
typedef struct reflex_rows {
  void* data;
  int64_t row_stride;
  int64_t head_stride;
} reflex_rows;

/* How the frequencies of a rotary plan fall: with REFLEX_LADDER_SHARED pair i
 * of head_dim/2 turns by theta^(-i / (head_dim/2)) per position whichever axis
 * it follows; with REFLEX_LADDER_PER_AXIS the j-th of an axis's m pairs turns
 * by theta^(-j / m). */
#define REFLEX_LADDER_SHARED 0
#define REFLEX_LADDER_PER_AXIS 1

#define REFLEX_MAX_AXES 4
#define REFLEX_MAX_PAIRS 128

/* A rotary plan (host memory, filled by reflex_rotary_init, read-only after). */
typedef struct reflex_rotary {
  int32_t head_dim;
  int32_t n_axes;
  uint8_t axis[REFLEX_MAX_PAIRS];   /* the axis that pair i follows */
  double turns[REFLEX_MAX_PAIRS];   /* full turns of pair i per position */
} reflex_rotary;

/*
 * Fill a rotary plan (pure host function).  Pair i is dimensions i and
 * i + head_dim/2 of a head (rotate-half, as in the action expert).  The first
 * sections[0] pairs follow axis 0, the next sections[1] axis 1, and so on (for
 * image tokens: time, height, width); their sum is head_dim/2.  One axis with
 * the shared ladder is the rotary embedding of the action expert.
 * head_dim: a multiple of 16 from 16 to 256.  Errors: REFLEX_EINVAL.
 */
int reflex_rotary_init(reflex_rotary* plan, int32_t head_dim, int32_t n_axes, const int32_t* sections, double theta,
                       int32_t ladder);

/*
 * Rotate n_rows rows of n_heads heads by their positions: y[i] = x[i] cos(a) -
 * x[i + half] sin(a), y[i + half] = x[i + half] cos(a) + x[i] sin(a) with a the
 * pair's angle at the row's position on the pair's axis.  inverse != 0 turns
 * the other way: the gradient of the rotation, and what gives a rotated key
 * its pre-RoPE values back.
 * positions: device int64, row r's position on axis a at [a*pos_stride + r].
 * Angles are reduced in 64 bits; |position| < 2^40.
 * y may be x (the same data and strides); otherwise they must not overlap.
 * n_rows: at most 2^27, in this call and in those below; 0 does nothing.
 * Errors: REFLEX_EINVAL, REFLEX_EHIP.
 */
int reflex_rotary_apply(const reflex_rotary* plan, const int64_t* positions, int64_t pos_stride, const reflex_rows* x,
                        const reflex_rows* y, int64_t n_rows, int32_t n_heads, int32_t dtype, int32_t inverse,
                        void* stream);

/* Element types of the pages.  F32 and BF16 pages hold the inputs' own type.
 * FP8 (e4m3) and INT8 pages hold, per token and K/V head, head_dim codes and
 * one fp32 scale; a value is code * scale.
 *   INT8: scale = max|x| * (1/127) (fp32 product with the fp32 nearest 1/127; at
 *         least 2^-126), code = x / scale to nearest.
 *   FP8:  scale = the smallest power of two (at least 2^-126) with max|x| <=
 *         448 * scale, code = x / scale to nearest.
 * Ties go to the even code.  What lies next to a border is decided exactly: K
 * is rotated and divided in 64 bits.  A row with an infinity or a NaN gets the
 * scale NaN: all of it reads as NaN.  Pages that a caller fills may hold any
 * codes, and scales that are finite or NaN. */
#define REFLEX_STORE_F32 0
#define REFLEX_STORE_BF16 1
#define REFLEX_STORE_FP8 2
#define REFLEX_STORE_INT8 3

/*
 * A paged cache: n_pages pages of page_size tokens.
 *   k, v              [n_pages][n_kv_heads][page_size][head_dim], 16-byte aligned
 *   k_scale, v_scale  [n_pages][n_kv_heads][page_size] fp32 (8-bit stores; else NULL)
 * page_size: a power of two from 1 to 1024; head_dim: 64, 128 or 256;
 * n_pages * n_kv_heads * page_size < 2^31.
 */
typedef struct reflex_paged_cache {
  void* k;
  void* v;
  float* k_scale;
  float* v_scale;
  int32_t n_pages;
  int32_t page_size;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t store;      /* REFLEX_STORE_* */
  int32_t reserved;
} reflex_paged_cache;

/*
 * Which tokens a call is about (device int32 arrays).  Sequence b has
 * lengths[b] tokens, the last n_b = cu_rows[b+1] - cu_rows[b] of which are the
 * call's rows cu_rows[b] .. cu_rows[b+1] - 1, oldest first.  Token p of the
 * sequence lies in slot p % page_size of page page_table[b][p / page_size].
 * Rows outside [cu_rows[0], cu_rows[n_seqs]) belong to no sequence: they have
 * no part in the call, and what an output holds there stays.
 * A table entry outside [0, n_pages), and every token beyond max_pages pages
 * or before the sequence's start, is absent: nothing is written for it, it
 * reads as zeros and no query sees it.  Sequences may share pages that a call
 * only reads.  No two rows of one write may be for the same slot unless their
 * values (and positions) are equal: what the slot holds then is undefined, and
 * may be codes, a scale, K and V of different rows.
 * cu_rows is non-decreasing from a value >= 0; what exceeds the call's n_rows
 * is cut off there.
 * max_length: the length that the longest sequence is expected to reach (0:
 * max_pages * page_size).  It only sizes the launch: longer ones stay correct.
 */
typedef struct reflex_paged_batch {
  const int32_t* cu_rows;     /* [n_seqs + 1] */
  const int32_t* lengths;     /* [n_seqs] */
  const int32_t* page_table;  /* [n_seqs][max_pages] */
  int32_t n_seqs;
  int32_t max_pages;
  int32_t max_length;
  int32_t reserved;
} reflex_paged_batch;

/*
 * Write K and V of the batch's rows ([n_rows][n_kv_heads][head_dim], dtype)
 * into their pages.  With a rotary plan (may be NULL) the keys are rotated
 * first, by `positions` as in reflex_rotary_apply, or, with positions NULL, by
 * the token's index in its sequence on every axis.
 * Errors: REFLEX_EINVAL; REFLEX_EDTYPE where an F32 or BF16 store differs from
 * dtype; REFLEX_EHIP.
 */
int reflex_paged_write(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* k,
                       const reflex_rows* v, int64_t n_rows, int32_t dtype, const reflex_rotary* rotary,
                       const int64_t* positions, int64_t pos_stride, void* stream);

/*
 * Read K and V of the batch's rows back: code * scale, rounded to dtype.  A
 * batch whose n_b is lengths[b] reads whole sequences.  Keys come as they were
 * written; reflex_rotary_apply with inverse gives their pre-RoPE values, which
 * is what reflex_cache_init and reflex_cache_write_frame take.
 * Errors: as reflex_paged_write.
 */
int reflex_paged_read(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* k,
                      const reflex_rows* v, int64_t n_rows, int32_t dtype, void* stream);

/*
 * Attention of the batch's rows over the pages of their sequences, which hold
 * the rows' own K/V already:
 *   out[r][h] = sum_j softmax_j(scale * q[r][h] . k[j][g]) v[j][g],
 * g = h / (n_q_heads / n_kv_heads), over the keys j that row r sees.  With p
 * the row's token index in its sequence (rows are the last n_b tokens) and L
 * the sequence's length, these are the present tokens j < L, with causal != 0
 * only j <= p, and with window > 0 only j > p - window.  A row that sees none
 * gets zeros, and so does one all of whose scores are below -2e38.
 * scale * log2(e) is finite in fp32.
 * Keys that a row does not see have no part in its result, whatever they hold
 * (NaN and infinities included).  Probabilities enter the second product
 * rounded to dtype or finer (in bf16 to 8 bits, with few rows to 16), all sums
 * are fp32; equal calls give equal bits.  The sums are divided last: values up
 * to V over L keys need 2^8 L V to be finite in fp32.
 * q, out: [n_rows][n_q_heads][head_dim], not overlapping.  n_q_heads: a
 * multiple of n_kv_heads; n_rows * n_q_heads <= 2^23.
 * workspace: at least the bytes that reflex_paged_attention_workspace gives
 * (which may be 0), 256-byte aligned; private to the call until its work is
 * done.
 * Errors: as reflex_paged_write.
 */
int reflex_paged_attention_workspace(const reflex_paged_cache* cache, const reflex_paged_batch* batch, int64_t n_rows,
                                     int32_t n_q_heads, int32_t dtype, size_t* bytes);
int reflex_paged_attention(const reflex_paged_cache* cache, const reflex_paged_batch* batch, const reflex_rows* q,
                           const reflex_rows* out, int64_t n_rows, int32_t n_q_heads, int32_t dtype, float scale,
                           int32_t causal, int32_t window, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* REFLEX_H */
