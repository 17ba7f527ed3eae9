/*
 * libwam — MI355X (gfx950) hot path of training-free World Action Model
 * inference with adaptive intermediate states.
 *
 * The library runs the iterative flow-denoising step of a DiT-style joint
 * video-latent + action-token transformer, and the three state-adaptation
 * operators that let a replan continue from retained state instead of
 * re-denoising from noise:
 *
 *   Trajectory Remapping  (Sec. 3.1, Eq. direction and Eq. transport, with the
 *                          unit-RMS normalisation of Eq. app-transport-rms),
 *   Observation Rebinding (Sec. 3.2, Eq. bind-discrepancy and the kappa rule),
 *   Residual Rescaling    (Sec. 3.3, Eq. crr-reference, crr-alpha, crr-gate,
 *                          residual-injection and refresh on failure),
 *
 * coordinated as in Sec. 3.4 (joint runtime).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 *  - Ownership: the caller allocates every device buffer (packed weights,
 *    workspace, trajectories, conditions, noise, outputs) and keeps it alive
 *    while the handle uses it.  The library never allocates device memory; the
 *    retained-state cache lives inside the caller's workspace.  Host pointers
 *    are only read during the call.
 *  - Streams: all device work is enqueued on the hipStream_t given to
 *    wam_init.  Calls that need a host-side decision (Residual Rescaling gate,
 *    Observation Rebinding score) synchronise that stream before returning;
 *    the others are asynchronous.
 *  - Randomness: the library draws no random numbers.  Noise is an input.
 *  - Layouts (all row-major, all device float32 unless stated):
 *      trajectory  x [B][traj], traj = Nv*Cv + Na*A, per sample
 *                  [video tokens (Nv x Cv) | action tokens (Na x A)];
 *      condition   cond [B][No][Co] (observation-conditioning tokens);
 *      hidden      h [B][T][D] with T = Nv + Na + No rows ordered
 *                  [video | action | observation].
 *  - Errors: every int-returning call returns WAM_OK (0) or a negative status
 *    and, given a handle, stores a message for wam_last_error.  Nothing throws
 *    across the ABI.  A failing call leaves retained state unchanged unless
 *    documented otherwise.
 *  - Threading: a handle is used by one host thread at a time.
 */
#ifndef WAM_H
#define WAM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ---------------------------------------------------- */
#define WAM_OK 0
#define WAM_E_ARG (-1)         /* invalid scalar argument or null pointer     */
#define WAM_E_SHAPE (-2)       /* model dimensions not supported / mismatched */
#define WAM_E_STATE (-3)       /* call not valid in the handle's state        */
#define WAM_E_HIP (-4)         /* HIP runtime error                           */
#define WAM_E_WORKSPACE (-5)   /* weight or workspace buffer too small        */
#define WAM_E_UNSUPPORTED (-6) /* valid request the library does not implement */

/* ---- numeric modes --------------------------------------------------- */
#define WAM_FP32 0 /* all activations and contractions in float32            */
#define WAM_BF16 1 /* projection / attention operands bf16, fp32 accumulate;
                      residual stream, trajectory, layer state, norms and all
                      reductions stay float32 (or float64 for gate sums)      */
#define WAM_FP8 2  /* as WAM_BF16, but the four projections of a layer multiply
                      e4m3 blocks: weights 128 x 128, packed by wam_init,
                      activations 1 x 128, each with a float32 scale (as
                      wam_quantize_fp8 makes them), by the 8-bit matrix
                      instruction (wam_matmul_fp8 with a bf16 result) also where
                      they add to the float32 residual; modulation, attention and
                      everything else stay as they are.  As an element type: e4m3 */

/* ---- Residual Rescaling modes ------------------------------------------ */
#define WAM_RR_OFF 0        /* plain full forward, no layer state kept        */
#define WAM_RR_AUTO 1       /* gate of Eq. crr-gate decides reuse or refresh  */
#define WAM_RR_FORCE_SKIP 2 /* reuse whenever a layer state exists            */
#define WAM_RR_FORCE_FULL 3 /* always compute the middle and refresh          */
/* wam_rr_profile.branches */
#define WAM_RR_JOINT 0  /* video (+ observation) and action rows: two checks */
#define WAM_RR_SINGLE 1 /* all rows: one check                                */

/* ---- wam_adapt_state operations ---------------------------------------- */
#define WAM_ADAPT_REMAP 1       /* args: const wam_remap_args*               */
#define WAM_ADAPT_RESET_LAYER 2 /* args: NULL; drop retained (p_a, R_a)      */
#define WAM_ADAPT_RESET_ALL 3   /* args: NULL; drop layer and replan state   */
#define WAM_ADAPT_SET_REPLAN 4  /* args: const wam_replan_state_args*        */
#define WAM_ADAPT_REBIND 5      /* args: const wam_rebind_args*              */

/* ---- replan paths (Sec. 3.4) ------------------------------------------- */
#define WAM_PATH_FIRST 0  /* first replan: K steps from fresh noise           */
#define WAM_PATH_ACCEPT 1 /* prefix under the predicted condition, rebound    */
#define WAM_PATH_REJECT 2 /* prefix failed the check: restart under c         */
#define WAM_PATH_FORCED 3 /* kappa reached kappa_max: refresh, no prefix      */
#define WAM_PATH_DIRECT 4 /* rebinding disabled: K-b0 steps under c           */

/* ---- wam_set_option ------------------------------------------------------ */
#define WAM_OPT_DEVICE_DECISION 1 /* 1: the Residual Rescaling decision stays on the
                                     device; the gate writes a flag that predicates
                                     the inject / middle / refresh launches, and step
                                     reports are read back once per call (default 0:
                                     the host reads the gate and launches one path) */
#define WAM_OPT_GRAPHS 2          /* 1: wam_replan replays one captured graph per
                                     (stage, RR variant); needs the device decision
                                     and a non-default stream; graphs are re-captured
                                     when the schedule or the RR profile changes */
#define WAM_OPT_ATTENTION 3       /* bf16 attention kernel (WAM_ATTN_*); every form
                                     gives the same result up to rounding */
#define WAM_ATTN_AUTO 0           /* default: a bounded form where the layer allows
                                     it (tile shape chosen by sequence length and
                                     grid size), else the running max */
#define WAM_ATTN_RUNNING_MAX 1    /* online softmax with a running maximum          */
#define WAM_ATTN_BOUNDED 2        /* QK-norm bounds every score by mref <= 60 (log2
                                     units, from the gains): mref is the fixed
                                     softmax reference, no running max; software-
                                     pipelined loop (QK of the next key tile
                                     issued before PV of this one)                 */
#define WAM_ATTN_PINGPONG 3       /* bounded, 8 waves in two groups that alternate
                                     MFMA and exp2 phases on each SIMD            */
#define WAM_ATTN_PLAIN 4          /* bounded, plain loop (one score buffer, more
                                     waves per SIMD); on grids too small to fill
                                     the chip, two wave groups split the keys and
                                     add their partial sums                      */
/* A bounded form asked for on a layer whose gains allow no bound (mref > 60)
   runs the running-max kernel. */

/* pairs of rotary positions in a head (wam_rope) */
#define WAM_ROPE_HALVES 0 /* elements i and i + P      */
#define WAM_ROPE_PAIRS 1  /* elements 2 i and 2 i + 1  */
#define WAM_MAX_HEAD 256
#define WAM_MAX_ROWS 16777215 /* of wam_rope and wam_norm_residual: B * T */

#define WAM_MAX_BATCH 16
#define WAM_MAX_COMPONENTS 8
#define WAM_MAX_STEPS 64

/* Kernel classes for wam_profile_* (per-launch timing from dispatch timestamps). */
#define WAM_KC_GEMM_QKV 0
#define WAM_KC_GEMM_PROJ 1
#define WAM_KC_GEMM_FC1 2
#define WAM_KC_GEMM_FC2 3
#define WAM_KC_ATTENTION 4
#define WAM_KC_RR_GATE 5
#define WAM_KC_RR_INJECT 6
#define WAM_KC_RR_REFRESH 7
#define WAM_KC_COUNT 8

typedef struct wam_handle *wam_t;

/* Model configuration.  D % 64 == 0 (D <= 2048), D % H == 0, head size D/H in
 * {32, 64}, Cv <= 16, A <= 16, Co <= 64; bf16 and fp8 modes additionally need
 * D/H == 64 and F % 128 == 0 (any head count, odd ones included).  Nv >= 0, Na >= 0, Nv + Na >= 1:
 * a model of an independently executed pair has only video (Na = 0) or only
 * action (Nv = 0) tokens; Cv and A stay >= 1 (their weights exist). */
typedef struct {
  int32_t B;       /* batch (samples denoised together), 1..WAM_MAX_BATCH */
  int32_t L;       /* DiT layers                                            */
  int32_t D;       /* hidden size                                           */
  int32_t H;       /* attention heads                                       */
  int32_t F;       /* MLP hidden size                                       */
  int32_t Nv, Cv;  /* video-latent tokens, channels per token               */
  int32_t Na, A;   /* action tokens (chunk length), action dimension        */
  int32_t No, Co;  /* observation tokens, channels per token                */
  int32_t dtype;   /* WAM_FP32 | WAM_BF16 | WAM_FP8                         */
  int32_t qk_norm; /* 1: RMS-normalise q and k per head (with gains)        */
  float ln_eps;    /* epsilon of LayerNorm and QK RMSNorm                   */
} wam_config;

/* Residual Rescaling profile (Sec. 3.3; thresholds as in Table app-guards).
 * Layer boundaries 0 < q < s < e < L partition the DiT into head [0,q),
 * probe [q,s), middle [s,e) and tail [e,L). */
typedef struct {
  int32_t q, s, e;
  int32_t mode; /* WAM_RR_* */
  float alpha_min, alpha_max, eps;
  float gamma_cos, gamma_fit;
  /* WAM_RR_JOINT: the jointly executed video (+ observation) and action
   * branches each get an alpha, and the middle is skipped only when both
   * pass (Sec. 3.3, joint execution).  WAM_RR_SINGLE: the model's whole token
   * set is one branch, as for each model of an independently executed video /
   * action pair (Sec. 3.3, independent execution; the branch-1 statistics of
   * wam_step_info are then NaN). */
  int32_t branches;
} wam_rr_profile;

/* Per-denoising-step report.  alpha/cos/fit are per sample and per branch
 * (branch 0 = video and observation rows, 1 = action rows; with
 * WAM_RR_SINGLE branch 0 = all rows and branch 1 = NaN); valid when
 * rr_attempted. */
typedef struct {
  int32_t rr_active;    /* RR mode was not OFF                              */
  int32_t rr_attempted; /* a retained state existed and the gate was run    */
  int32_t rr_accepted;  /* the middle layers were skipped                   */
  int32_t layers_evaluated;
  int32_t layers_skipped;
  int32_t reserved;
  double alpha[WAM_MAX_BATCH][2];
  double cos[WAM_MAX_BATCH][2];
  double fit[WAM_MAX_BATCH][2];
} wam_step_info;

/* Trajectory Remapping arguments (Eq. direction, Eq. transport). */
typedef struct {
  const float *x_bar; /* device [B][traj]: final output of the previous replan  */
  const float *x_r;   /* device [B][traj]: latent retained at stage r           */
  float sigma_r;      /* noise level of stage r, must be > 0                    */
  float sigma_b0;     /* noise level of the entry stage b0                      */
  int32_t shift_action; /* target action slot j takes source slot j+shift (>=0) */
  int32_t shift_video;  /* same for video tokens (>=0)                          */
  const float *noise; /* device [B][traj] N(0,1); unmapped slots get sigma_b0*noise */
  float *x_out;       /* device [B][traj]: remapped initialisation              */
} wam_remap_args;

/* Observation Rebinding's rebinding step (Sec. 3.2): the retained denoising
 * state (the working latent an anticipatory prefix produced under the
 * predicted condition c_hat, the latent captured at stage r, and the Residual
 * Rescaling layer state, which persists across the rebinding point, Sec. 3.3)
 * continues under the real condition c.  The library copies cond into its own
 * condition buffer (stream-ordered; the caller's buffer may be reused once the
 * stream passes this point) and from then on a NULL cond in wam_velocity,
 * wam_denoise_step, wam_continue and wam_hidden means that bound condition.
 * Nothing else of the retained state changes; the rebinding counter kappa
 * and the decision S < tau and kappa < kappa_max belong to wam_replan, which
 * performs the same step on its accept path (and leaves its real condition
 * bound after every replan).  cond: device [B][No][Co], may be NULL only when
 * No == 0.  WAM_E_ARG for a NULL cond otherwise. */
typedef struct {
  const float *cond;
} wam_rebind_args;

/* Adopt an externally held replan state (teacher forcing / resume). */
typedef struct {
  const float *x_bar; /* device [B][traj] */
  const float *x_r;   /* device [B][traj] */
  int32_t kappa;
} wam_replan_state_args;

/* One closed-loop replan (Sec. 3.4). */
typedef struct {
  const float *cond_real; /* device [B][No][Co]: real condition c_{t+1}          */
  const float *cond_pred; /* device [B][No][Co]: predicted condition (OR prefix) */
  /* consistency components compared before encoding (Eq. bind-discrepancy) */
  int32_t n_components;
  const float *u_hat[WAM_MAX_COMPONENTS]; /* device, n[m] floats each         */
  const float *u[WAM_MAX_COMPONENTS];
  int64_t n[WAM_MAX_COMPONENTS];
  double delta[WAM_MAX_COMPONENTS];
  double weight[WAM_MAX_COMPONENTS];
  const float *noise_first; /* device [B][traj] N(0,1): first replan's x at sigma_0 */
  const float *noise_remap; /* device [B][traj] N(0,1): unmapped slots / fresh init */
  float *x_out;             /* device [B][traj]: receives the new x_bar             */
  wam_rr_profile rr;
  int32_t b0, r;             /* entry stage and retained stage, b0 <= r < K    */
  int32_t shift_action, shift_video;
  int32_t k1;                /* anticipatory prefix steps, 0 < k1 < K-b0       */
  double tau;                /* accept iff S < tau and kappa < kappa_max       */
  int32_t kappa_max;
  int32_t tr_enabled, or_enabled;
  int32_t rr_first, rr_prefix, rr_refresh; /* RR allowed on each path       */
} wam_replan_args;

typedef struct {
  int32_t path;  /* WAM_PATH_* */
  int32_t kappa; /* after this replan */
  int32_t steps; /* denoising steps executed (prefix + continuation/restart) */
  int32_t n_start, n_bind; /* 0/1 for this replan (Eq. app-rebinding-rates) */
  int32_t rr_attempts, rr_reuses, layers_skipped, layers_dense;
  int32_t reserved;
  double S; /* consistency score, or -1 when no prefix was checked */
  int8_t decision[WAM_MAX_STEPS]; /* per step: -1 no attempt, 0 refresh, 1 reuse */
} wam_replan_info;

/* ---- sizes --------------------------------------------------------------- */
/* Number of float32 values of the canonical host weight buffer, which holds,
 * each row-major with Linear weights stored [in][out] (y = x W + b):
 *   t_w1[256][D] t_b1[D] t_w2[D][D] t_b2[D]
 *   in_wv[Cv][D] in_bv[D] in_wa[A][D] in_ba[D] in_wo[Co][D] in_bo[D]
 *   for each layer l: mod_w[D][6D] mod_b[6D] qkv_w[D][3D] qkv_b[3D]
 *                     q_g[dh] k_g[dh] proj_w[D][D] proj_b[D]
 *                     fc1_w[D][F] fc1_b[F] fc2_w[F][D] fc2_b[D]
 *   f_mod_w[D][2D] f_mod_b[2D] out_wv[D][Cv] out_bv[Cv] out_wa[D][A] out_ba[A]
 * Returns 0 for an invalid configuration. */
size_t wam_host_weight_count(const wam_config *cfg);
/* Device bytes of the packed weights (with the constant position-embedding
 * table) and of the workspace (0 if invalid). */
size_t wam_weight_bytes(const wam_config *cfg);
size_t wam_workspace_bytes(const wam_config *cfg);
/* Trajectory elements per sample, Nv*Cv + Na*A. */
int64_t wam_traj_elems(const wam_config *cfg);

/* ---- lifetime ------------------------------------------------------------ */
/* Validates cfg, converts and packs the host weights (bf16 mode: projection
 * and modulation matrices rounded to bf16, nearest-even) into dev_weights,
 * carves the workspace, and returns a handle.  Synchronous. */
int wam_init(const wam_config *cfg, const float *host_weights, size_t n_host_weights,
             void *dev_weights, size_t weight_bytes, void *dev_workspace,
             size_t workspace_bytes, void *hip_stream, wam_t *out);
void wam_destroy(wam_t h);
int wam_sync(wam_t h);
const char *wam_last_error(wam_t h);
const char *wam_status_string(int status);
/* Execution options (WAM_OPT_*); results are identical either way up to the
 * order of independent work.  Returns WAM_E_STATE for an invalid combination
 * and WAM_E_UNSUPPORTED for graphs on the default (null) stream. */
int wam_set_option(wam_t h, int option, int value);

/* Rotary positions of the model's rows: from the next step on every layer turns
 * q and k (after their norm) by wam_rope's rule, row t of every sample by pos[t].
 * The additive sinusoidal table of the embedding is left out unless keep_table is
 * set.  pos is read by every step (also by replayed graphs) and stays the
 * caller's; freq is copied.  2 P <= head size.  args NULL: back to the table
 * alone.  Drops the retained layer state and captured graphs; WAM_E_STATE while a
 * replan is open. */
typedef struct {
  const float *pos;     /* device [T][3] (time, height, width)              */
  int32_t sections[3];  /* pairs of each axis                               */
  int32_t layout;       /* WAM_ROPE_*                                       */
  const double *freq;   /* host [P]: radians per unit of position           */
  int32_t keep_table;
} wam_rotary_args;
int wam_set_rotary(wam_t h, const wam_rotary_args *args);
/* Post-norms: from the next step on the output of a layer's attention and MLP
 * blocks (their last projection with its bias) is divided by its root mean square
 * (ln_eps) and multiplied by its gains before gate and residual:
 *   h <- h + gate * gain * y / sqrt(mean(y^2) + ln_eps).
 * gains: device [L][2][D] (attention, MLP), read by every step, caller-owned;
 * NULL: none.  State as for wam_set_rotary. */
int wam_set_post_norm(wam_t h, const float *gains);

/* Noise levels sigma_0 = 1 > ... > sigma_K = 0 of the flow schedule
 * (host float[K+1]); K <= WAM_MAX_STEPS.  Required before any step. */
int wam_set_schedule(wam_t h, const float *sigmas, int K);

/* ---- denoising ------------------------------------------------------------ */
/* Denoiser prediction v(x, sigma_k, cond) into v_out [B][traj]; runs the
 * embedding, the L DiT layers (with Residual Rescaling per rr, which may be
 * NULL = off), the final layer and the output heads.  Updates the retained
 * layer state as Sec. 3.3 prescribes. */
int wam_velocity(wam_t h, int k, const float *x, const float *cond, float *v_out,
                 const wam_rr_profile *rr, wam_step_info *info);
/* One Euler step of the flow ODE: x <- x + (sigma_{k+1} - sigma_k) v. */
int wam_denoise_step(wam_t h, int k, float *x, const float *cond,
                     const wam_rr_profile *rr, wam_step_info *info);
/* Steps k_from .. k_to-1 in place on x.  If k_from <= capture_stage <= k_to
 * the latent at that stage is copied to x_capture (device [B][traj]).
 * infos may be NULL or hold k_to - k_from entries. */
int wam_continue(wam_t h, int k_from, int k_to, float *x, const float *cond,
                 const wam_rr_profile *rr, int capture_stage, float *x_capture,
                 wam_step_info *infos);
/* Hidden state after the first n_layers layers (no RR) at stage k into
 * h_out [B][T][D]; for layer-level parity checks. */
int wam_hidden(wam_t h, int k, const float *x, const float *cond, int n_layers, float *h_out);

/* ---- state adaptation ------------------------------------------------------ */
int wam_adapt_state(wam_t h, int op, const void *args);
/* Observation Rebinding score (Eq. bind-discrepancy) over device arrays,
 * accumulated in float64: S = sqrt(sum w e^2 / sum w),
 * e_m = sqrt(mean(((u_hat_m - u_m)/delta_m)^2)).  u_hat[m], u[m]: device
 * float[n[m]], caller-owned; n_components in 1..WAM_MAX_COMPONENTS, n >= 1,
 * delta > 0, weight >= 0 with a positive sum (else WAM_E_ARG).  The squared
 * differences are summed on the device in runs (float64, fixed order) and the
 * run sums on the host.  Only this device form exists: the components are the
 * condition tensors, which already live on the device.  Uses the handle's
 * stream and its pinned host buffer; synchronises. */
int wam_consistency_score(wam_t h, int n_components, const float *const *u_hat,
                          const float *const *u, const int64_t *n, const double *delta,
                          const double *weight, double *S_out);
/* Condition tokens of the action model of an independently executed video /
 * action pair (Sec. 3.3; the action model reads the observation and the video
 * model's latent): cond [B][No][Co] = the n_obs observation tokens obs
 * [B][n_obs][c_obs] followed by the n_ctx tokens of ctx (sample b, token j,
 * channel c at ctx[b * ctx_stride + j * c_ctx + c], e.g. the video part of
 * the video model's trajectory), each zero-padded to Co channels.  Needs
 * n_obs + n_ctx == No and c_obs, c_ctx <= Co.  Device pointers, caller-owned;
 * enqueued on the handle's stream (no synchronisation). */
int wam_pack_condition(wam_t h, const float *obs, int n_obs, int c_obs, const float *ctx, int n_ctx,
                       int c_ctx, int64_t ctx_stride, float *cond);
/* One replan of the joint runtime.  The first call (or after RESET_ALL) runs
 * the native K steps from noise_first; later calls apply Trajectory
 * Remapping, the anticipatory prefix under cond_pred, the consistency check
 * and rebinding or restart, with Residual Rescaling inside each step.  The
 * retained replan state (x_bar, x^r, kappa) lives in the workspace. */
int wam_replan(wam_t h, const wam_replan_args *args, wam_replan_info *info);
/* The same replan in two halves, so that the anticipatory prefix overlaps
 * action execution (Sec. 3.2).  wam_replan_begin applies Trajectory Remapping
 * and enqueues the prefix under cond_pred; with WAM_OPT_DEVICE_DECISION it
 * returns without waiting for the GPU.  wam_replan_end, called once the real
 * observation is available, computes the consistency score, rebinds or
 * restarts under cond_real, and fills info.  Both take the same args (the
 * buffers must stay valid until wam_replan_end returns); wam_replan_end
 * without a begin runs the whole replan.  A second begin before end is
 * WAM_E_STATE. */
int wam_replan_begin(wam_t h, const wam_replan_args *args);
/* While a replan is open (after wam_replan_begin, before wam_replan_end) the
 * other calls that touch the handle's state (wam_velocity, wam_denoise_step,
 * wam_continue, wam_hidden, wam_adapt_state except RESET_ALL,
 * wam_consistency_score, wam_get_replan_state, wam_set_schedule,
 * wam_set_option) return WAM_E_STATE; RESET_ALL abandons the open replan. */
int wam_replan_end(wam_t h, const wam_replan_args *args, wam_replan_info *info);
/* Copies of the retained replan state (device [B][traj] each; may be NULL). */
int wam_get_replan_state(wam_t h, float *x_bar, float *x_r, int32_t *kappa);

/* Trajectory Remapping that allocates nothing, for callers that cannot
 * allocate device memory (code under HIP graph capture, tight serving loops,
 * harnesses that forbid allocation): the same computation and kernels as
 * wam_adapt_state(WAM_ADAPT_REMAP), without a handle.  From cfg only B, Nv,
 * Cv, Na and A are read (1 <= B <= WAM_MAX_BATCH, Nv, Na >= 0, Nv + Na >= 1,
 * Cv, A >= 1, B * traj < 2^31); args as for WAM_ADAPT_REMAP (device buffers,
 * caller-owned).  Enqueued on hip_stream (NULL: the default stream) with no
 * synchronisation.  The reduction scratch (at most WAM_MAX_BATCH x 2 x 1025
 * float64, 256.3 KiB) is a static array of the library on each GPU, held until
 * the process ends; every call on one GPU shares it, so calls that overlap on
 * one GPU (different streams or threads) race.  The call makes no device
 * allocation and no hipMalloc / hipFree.  Errors: WAM_E_SHAPE for sizes
 * beyond those limits, WAM_E_ARG for invalid arguments, WAM_E_HIP for a
 * runtime error; wam_noalloc_last_error() returns this thread's message of
 * the last failing call without a handle. */
int wam_remap_noalloc(const wam_config *cfg, const wam_remap_args *args, void *hip_stream);
const char *wam_noalloc_last_error(void);

/* ---- layer operators ---------------------------------------------------------- */
/* Operators of a transformer layer on caller-owned device buffers, without a
 * handle: rotary positions over several axes, the norms around a block with
 * its gate and residual, 8-bit and 4-bit blocks and their products, a cache of
 * keys and values and attention over it.  Each is enqueued on
 * hip_stream (NULL: the default stream) of the current device, allocates
 * nothing, shares no scratch between calls (calls may overlap), does not
 * synchronise and may be captured into a graph.  Struct and host pointers are
 * read during the call only.  Strides count elements, up to 2^40;
 * the last dimension is contiguous.  An input stride may be 0 (the same values
 * for every index); the elements of an output must be distinct.  An input and
 * an output must not overlap, except where a call says that they may be the
 * same buffer.  A call with an empty dimension does nothing.  Errors: WAM_E_ARG
 * for an invalid argument, WAM_E_SHAPE for a size beyond the limits stated,
 * WAM_E_HIP for a runtime error; wam_noalloc_last_error() returns this thread's
 * message.  Element types: WAM_FP32, WAM_BF16 and, where said, WAM_FP8 (e4m3:
 * 4 exponent and 3 mantissa bits, largest value 448, no infinity). */

/* Rotary positions.  Row t of sample b has one position per axis, pos[t][a]
 * (time, height, width; fractions allowed), and pair i of a head, which belongs
 * to axis 0 for i < sections[0], to axis 1 for the next sections[1], to axis 2
 * for the rest, turns by the angle pos[t][axis(i)] * freq[i]:
 *   (x1, x2) -> (x1 cos - x2 sin, x1 sin + x2 cos)
 * with P = sections[0] + sections[1] + sections[2] pairs, 2 P <= dh, of
 *   WAM_ROPE_HALVES  elements i and i + P,
 *   WAM_ROPE_PAIRS   elements 2 i and 2 i + 1;
 * elements from 2 P on pass unchanged.  Angles are formed in float64.  With
 * q_gain / k_gain (float32 [dh]) each head vector x is first divided by its
 * root mean square and multiplied by the gain: x gain / sqrt(mean(x^2) + eps);
 * NULL leaves it out.  Results are rounded once.  q_out may be q and k_out may be k
 * (with the same strides).  Hk = 0 leaves k out (Hq = 0: q).  dh <= 256,
 * B * T <= WAM_MAX_ROWS, Hq + Hk <= WAM_MAX_ROWS. */
typedef struct {
  int32_t B, T, Hq, Hk, dh;
  int32_t dtype;              /* of q, k and the results: WAM_FP32 | WAM_BF16  */
  int32_t layout;             /* WAM_ROPE_*                                    */
  int32_t sections[3];        /* pairs of each axis, >= 0                      */
  const void *q, *k;          /* device [B][T][H][dh] by the strides below     */
  void *q_out, *k_out;
  int64_t q_stride[3], k_stride[3];         /* of sample, row, head            */
  int64_t q_out_stride[3], k_out_stride[3];
  const float *pos;           /* device [T][3] per sample, contiguous          */
  int64_t pos_stride;         /* floats between samples; 0: the same for all   */
  const double *freq;         /* host [P]: radians per unit of position        */
  const float *q_gain, *k_gain; /* device [dh] or NULL                         */
  float eps;                  /* >= 0; used with a gain                        */
} wam_rope_args;
int wam_rope(const wam_rope_args *args, void *hip_stream);
/* Frequencies of the usual ladder into freq (host [P]): pair j of an axis of n
 * pairs gets theta^(-j / n); with shared != 0 one ladder runs over all P pairs,
 * pair i gets theta^(-i / P).  theta > 0. */
int wam_rope_frequencies(const int32_t *sections, double theta, int32_t shared, double *freq);

/* Norms around a block.  h is the residual stream, y the block's output:
 *   h_out = res_scale * h + gate * post(y)
 *   u     = pre(h_out before its rounding) * (1 + scale) + shift
 * post and pre are WAM_NORM_NONE (x), WAM_NORM_RMS (x / sqrt(mean(x^2) + eps))
 * or WAM_NORM_LAYER ((x - mean) / sqrt(mean((x - mean)^2) + eps)), times
 * post_gain / pre_gain (NULL: 1).  gate, scale and shift are float32 vectors of
 * D values per row, by strides of sample and row (0: shared); NULL: gate 1,
 * scale 0, shift 0.  y NULL: h_out = res_scale * h.  u NULL: no second part;
 * h_out NULL: not stored (u must be asked for).  Sums are float32.  u of type
 * WAM_FP8 is stored as blocks of 128 columns of a row, as wam_quantize_fp8
 * does, with its float32 scales in u_scale [B][T][ceil(D / 128)].  h_out may
 * be h and u may be y (with the same type and strides).  1 <= D <= 8192,
 * B * T <= WAM_MAX_ROWS. */
#define WAM_NORM_NONE 0
#define WAM_NORM_RMS 1
#define WAM_NORM_LAYER 2
#define WAM_MAX_NORM_D 8192
typedef struct {
  int32_t B, T, D;
  int32_t h_dtype, y_dtype, u_dtype; /* h and h_out, y: WAM_FP32 | WAM_BF16; u: any */
  int32_t post, pre;                 /* WAM_NORM_*                                   */
  const void *h, *y;                 /* device [B][T][D]                             */
  void *h_out, *u;
  float *u_scale;
  int64_t h_stride[2], y_stride[2], h_out_stride[2], u_stride[2], u_scale_stride[2]; /* of sample, row */
  const float *gate, *scale, *shift;
  int64_t gate_stride[2], scale_stride[2], shift_stride[2];
  const float *post_gain, *pre_gain; /* device [D] or NULL                           */
  float res_scale, eps;
} wam_norm_args;
int wam_norm_residual(const wam_norm_args *args, void *hip_stream);

/* 8-bit blocks: x [M][K] is cut into blocks of block_rows (1 or 128) rows and
 * 128 columns (the last ones smaller); a block's scale is max|x| / 448 in
 * float32, at least 2^-126 (1 where the block is zero), and q the float32 quotient
 * x / scale rounded to e4m3, to nearest, ties to even.  A block with a NaN or an
 * infinity has that as its scale, and stands for NaN.  scale: [ceil(M / block_rows)][ceil(K / 128)].
 * Bytes of a row of q past K are left as they are.  At most 2^29 - 32 blocks of
 * one row or 2^24 - 1 of 128 rows. */
typedef struct {
  int32_t M, K;
  int32_t dtype;       /* of x: WAM_FP32 | WAM_BF16 */
  int32_t block_rows;  /* 1 (activations) or 128 (weights) */
  const void *x;
  int64_t x_stride;    /* of a row */
  void *q;
  int64_t q_stride;
  float *scale;
  int64_t scale_stride;
} wam_quantize_args;
int wam_quantize_fp8(const wam_quantize_args *args, void *hip_stream);

/* Product of e4m3 matrices with a float32 scale per block of 128:
 *   out[m][n] = act(sum_j a_scale[m][j] w_scale[n / 128][j]
 *                   sum_{k in block j} a[m][k] w[n][k] + bias[n])
 * a [M][K] with scales per row (blocks of 1 x 128), w [N][K] with scales per
 * block of 128 x 128, as wam_quantize_fp8 makes them.  Block products and their
 * scaled sum are float32.  The two scales of a block are multiplied first, in float32:
 * where that is below 2^-126 the block's share of the result has a subnormal's digits,
 * and where it passes the range the result is an infinity or NaN.  With a bf16 or e4m3
 * result the products of 8 consecutive k are cut below 2^-13 of the power of two of
 * the largest of them (the 8-bit matrix instruction), with a float32 result they are
 * not.  a and w must start on 16 bytes and their row strides be multiples of 16; the
 * bytes of a row past K, up to the next multiple of 16, are read but may hold
 * anything (behind the last row too: they lie in the same 16 bytes as its last
 * value).  WAM_E_SHAPE where the tiles pass a grid (from 2^24 of 32 x 32 on).  act:
 * WAM_ACT_NONE or WAM_ACT_GELU (tanh form).  out: WAM_FP32, WAM_BF16, or WAM_FP8:
 * blocks of 1 x 128 of the result before any rounding, with their scales in out_scale
 * [M][ceil(N / 128)], as wam_quantize_fp8 makes them, for the next product (rows
 * of a and w then at most 2^23 bytes apart, else WAM_E_UNSUPPORTED). */
#define WAM_ACT_NONE 0
#define WAM_ACT_GELU 1
typedef struct {
  int32_t M, N, K;
  int32_t out_dtype, act;
  const void *a;
  int64_t a_stride;
  const float *a_scale;
  int64_t a_scale_stride;
  const void *w;
  int64_t w_stride;
  const float *w_scale;
  int64_t w_scale_stride;
  const float *bias;   /* device [N] or NULL */
  void *out;
  int64_t out_stride;
  float *out_scale;    /* out of WAM_FP8 */
  int64_t out_scale_stride;
} wam_matmul_args;
int wam_matmul_fp8(const wam_matmul_args *args, void *hip_stream);

/* 4-bit blocks.  A block is 32 neighbouring values of a row: their codes, two to a
 * byte (the first value in the low half; 1 sign, 2 exponent and 1 mantissa bit: 0, 0.5,
 * 1, 1.5, 2, 3, 4, 6 and their negatives), and one byte s that stands for 2^(s - 127),
 * or for NaN where it is 255.
 *
 * wam_quantize_fp4: x [M][K] into q [M][ceil(K / 2)] and scale [M][ceil(K / 32)]
 * (the last block of a row smaller).  With the largest magnitude of a block in
 * [2^e, 2^(e + 1)) its byte is e - 2 + 127, at least 0, and a code the nearest value to
 * x / 2^(e - 2), ties to the even code, magnitudes above 6 to 6.  A block of zeros has
 * the byte 0; one with a NaN or an infinity has 255, codes zero, and stands for NaN.
 * With an odd K the last byte's high half is zero.  No other byte is written.
 *
 * wam_dequantize_fp4: the values of q, scale as x [M][K], float32 or bf16 (which holds
 * each of them but those past its range; K columns of q, odd ones too).
 *
 * Both: at most 2^29 - 32 blocks, strides of rows in elements and bytes. */
#define WAM_FP4_BLOCK 32
typedef struct {
  int32_t M, K;
  int32_t dtype;       /* of x: WAM_FP32 | WAM_BF16 */
  const void *x;
  int64_t x_stride;
  uint8_t *q;
  int64_t q_stride;
  uint8_t *scale;
  int64_t scale_stride;
} wam_quantize_fp4_args;
int wam_quantize_fp4(const wam_quantize_fp4_args *args, void *hip_stream);
typedef struct {
  int32_t M, K;
  int32_t dtype;       /* of x: WAM_FP32 | WAM_BF16 */
  const uint8_t *q;
  int64_t q_stride;
  const uint8_t *scale;
  int64_t scale_stride;
  void *x;
  int64_t x_stride;
} wam_dequantize_fp4_args;
int wam_dequantize_fp4(const wam_dequantize_fp4_args *args, void *hip_stream);

/* Product of matrices in 4-bit blocks:
 *   out[m][n] = act(sum_j 2^(a_scale[m][j] + w_scale[n][j] - 254)
 *                   sum_{k in block j} a[m][k] w[n][k] + bias[n])
 * a [M][K] and w [N][K] with K even, as wam_quantize_fp4 makes them (an odd K: one more
 * column, which is zero).  Sums are float32: each step of the scaled matrix instruction
 * (128 of K) is off by at most 2^-22 of the sum of its products' magnitudes and of what
 * it adds to; where those pass the float32 range the result may be infinite or NaN.
 * Data must start on 16 bytes with row strides a multiple of 16, scales on
 * 4 bytes with row strides a multiple of 4; the bytes of a row past its end, up to the
 * next multiple of 16 (4), are read but may hold anything (behind the last row too).
 * act: WAM_ACT_NONE or WAM_ACT_GELU (tanh form).  out: WAM_FP32, WAM_BF16, or WAM_FP4:
 * blocks of the result before any rounding in out [M][ceil(N / 2)] and out_scale
 * [M][ceil(N / 32)], for the next product.  WAM_E_SHAPE where the tiles pass a grid. */
#define WAM_FP4 3
typedef struct {
  int32_t M, N, K;
  int32_t out_dtype, act;
  const uint8_t *a;
  int64_t a_stride;
  const uint8_t *a_scale;
  int64_t a_scale_stride;
  const uint8_t *w;
  int64_t w_stride;
  const uint8_t *w_scale;
  int64_t w_scale_stride;
  const float *bias;   /* device [N] or NULL */
  void *out;
  int64_t out_stride;  /* in elements; bytes of WAM_FP4 */
  uint8_t *out_scale;  /* out of WAM_FP4 */
  int64_t out_scale_stride;
} wam_matmul_fp4_args;
int wam_matmul_fp4(const wam_matmul_fp4_args *args, void *hip_stream);

/* A cache of keys and values in 4-bit blocks: a pool of pages of `page` tokens (a power
 * of two, 16 to 4096) with H heads of dh values (32, 64, 96 or 128), i.e. dh / 2 bytes of
 * codes and dh / 32 scales a head, all contiguous; strides in bytes of page, token and
 * head, those of codes (and their base) multiples of 4, those of tokens at most 2^26.  A sequence has a row of
 * table: its token t lies at place t % page of page table[b][t / page].  An entry
 * outside 0 .. pages - 1 stands for no page, and tokens past the table for none. */
typedef struct {
  int32_t pages, page, H, dh;
  uint8_t *k, *k_scale, *v, *v_scale;
  int64_t k_stride[3], k_scale_stride[3], v_stride[3], v_scale_stride[3]; /* of page, token, head */
} wam_cache;
typedef struct {
  const int32_t *entry; /* device [B][width] */
  int64_t stride;       /* of a sequence, in entries */
  int32_t width;
} wam_page_table;

/* Appends T rows of B sequences: row t of sequence b becomes token start[b] + t.  v goes
 * into blocks as it is; k first gets the RMS norm with k_gain (NULL: none) and the
 * rotary positions of wam_rope (sections, layout, pos, freq; no pairs: none), both in
 * float64, and is rounded to float32 once.  rows[b] (NULL: T) is how many rows of b
 * count; those past it, tokens below 0 and tokens without a page are dropped.  Nothing
 * but the tokens' own bytes is written.  The tokens of a call must lie at
 * different places of the pool.  B * T <= WAM_MAX_ROWS. */
typedef struct {
  int32_t B, T, dtype;             /* of k and v: WAM_FP32 | WAM_BF16 */
  int32_t layout, sections[3];
  wam_cache cache;
  wam_page_table table;
  const void *k, *v;               /* device [B][T][H][dh] */
  int64_t k_stride[3], v_stride[3]; /* of sample, row, head */
  const int32_t *start, *rows;     /* device [B]; rows may be NULL */
  const float *pos;                /* device [T][3] per sample, contiguous; NULL without pairs */
  int64_t pos_stride;              /* floats between samples; 0: the same for all */
  const double *freq;              /* host [P]: radians per unit of position */
  const float *k_gain;             /* device [dh] or NULL */
  double eps;                      /* >= 0; used with a gain */
} wam_cache_append_args;
int wam_cache_append(const wam_cache_append_args *args, void *hip_stream);

/* Attention of T rows of B sequences over the cache:
 *   out[b][t][h] = sum_j softmax_j(scale q[b][t][h] . k_j) v_j
 * over the tokens j < seen(b, t) of key head h / (Hq / cache.H), without those that
 * have no page.  seen is lengths[b], or, causal, lengths[b] - rows[b] + t + 1 (the last
 * rows[b] tokens are the rows' own), between 0 and the table's end.  A row that sees no
 * token, or only ones whose scores are -infinity in float32 (in units of log2), or past
 * rows[b] (NULL: T), is 0.  What lies in tokens that a row does not see,
 * NaN included, does not enter; a value of v past the bf16 range counts as NaN, one of k as
 * an infinity (where 2^8 times the sum of the probabilities' products with |v|, the largest
 * probability being 1, passes the float32 range, a result may be NaN).  lse
 * (NULL: not stored) is the natural logarithm of the sum of the exponentials, -inf for
 * such a row; two results over different tokens join with it.  Scores and sums are
 * float32; with bf16 q a probability is rounded to bf16 once, with float32 q neither q nor
 * the probabilities lose a bit that float32 holds (but q's below 2^-133).  Hq is a multiple
 * of cache.H, scale > 0.
 * How rows and tokens are shared among blocks goes by the width of the table, as the lengths
 * are on the device: one much wider than the sequences costs time (a row over 864 tokens
 * 9.4 us, 13.6 with a table for 101760).
 * Where a sequence's tokens are shared among blocks, their parts meet in workspace:
 * wam_cache_attention_workspace bytes (0: none) on 16 bytes, any content, which the
 * call owns until its work is done.  B * T <= WAM_MAX_ROWS, B * T * Hq <= 2^31 - 2^16. */
typedef struct {
  int32_t B, T, Hq, dtype;         /* of q and out: WAM_FP32 | WAM_BF16 */
  int32_t causal;
  wam_cache cache;
  wam_page_table table;
  const void *q;                   /* device [B][T][Hq][dh] */
  int64_t q_stride[3];             /* of sample, row, head */
  void *out;
  int64_t out_stride[3];
  float *lse;                      /* device [B][T][Hq] or NULL */
  int64_t lse_stride[3];
  const int32_t *lengths, *rows;   /* device [B]; rows may be NULL */
  double scale;
  void *workspace;
  size_t workspace_bytes;
} wam_cache_attention_args;
size_t wam_cache_attention_workspace(const wam_cache_attention_args *args);
int wam_cache_attention(const wam_cache_attention_args *args, void *hip_stream);

/* ---- measurement ------------------------------------------------------------ */
/* Time every launch of kernel class kc (WAM_KC_*), up to max_launches
 * launches: a HIP event pair per launch, stamped by the dispatches themselves
 * (begin of the class's first kernel, end of its last; hipExtLaunchKernel), so
 * no event packets sit between the timed kernels.  Launches inside a graph
 * capture are not timed.  enable = 0 stops. */
int wam_profile_enable(wam_t h, int kc, int enable, int max_launches);
/* Sum of launch durations (ms), launch count and algorithmic work (FLOP for
 * contractions, bytes for streaming kernels) of the recorded launches.
 * Synchronises. */
int wam_profile_read(wam_t h, int kc, double *total_ms, int64_t *launches, double *work);

/* Achievable-peak probes (no handle; synchronous on hip_stream, which may be
 * NULL for the default stream).  They measure what the chip reaches in
 * practice, beside the vendor peaks that the roofline fractions use.
 *
 * wam_probe_mfma_bf16: n_blocks blocks of 256 threads each run iters rounds
 * of independent bf16 MFMA chains on register operands (shape 0:
 * v_mfma_f32_16x16x32_bf16, the instruction of the GEMM and attention
 * kernels; shape 1: v_mfma_f32_32x32x16_bf16), 131072 FLOP per wave per
 * round, after one untimed warm-up launch.  sink: device float[n_blocks *
 * 256], caller-owned, receives one value per thread.  Outputs the rate in
 * TFLOP/s and the timed launch in ms.  Size iters so that a launch lasts
 * tens of ms or more: the shader clock ramps up from idle over that time,
 * and launches of a few ms read up to ~20% low.
 *
 * wam_probe_copy: copies bytes (a multiple of 16, both pointers 16-byte
 * aligned, device, caller-owned, not overlapping) from src to dst reps times
 * after one warm-up; outputs the rate counting the bytes read plus written
 * (GB/s, 1e9) and the time per copy in ms.
 *
 * Both return WAM_E_ARG for invalid arguments and WAM_E_HIP for a runtime
 * error (no handle, so no message). */
int wam_probe_mfma_bf16(void *hip_stream, int shape, int n_blocks, int iters, float *sink, double *tflops,
                        double *ms);
int wam_probe_copy(void *hip_stream, const void *src, void *dst, size_t bytes, int reps, double *gbs,
                   double *ms);

#ifdef __cplusplus
}
#endif
#endif /* WAM_H */
