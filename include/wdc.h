/*
 * wdc.h -- C ABI of libwdc.so: the WorldDynCache cached denoising rollout on
 * one NVIDIA GB300 (sm_103a).
 *
 * The method (arxiv 2608.01845, "WorldDynCache: Risk-Controlled Latent Dynamics
 * Approximation for Diffusion World Models") replaces some exact transitions
 *     z_{t-1} = Psi_t(z_t, F_theta(z_t, t, c))                       (Eq. 1)
 * of a diffusion world model's rollout by a surrogate
 *     z_hat_{t-1} = G_t(z_t, H_t)                                   (Eq. 1-5)
 * whenever a calibrated, accumulated transition risk allows it (Eq. 6-10).
 *
 * Conventions for every entry point:
 *  - Errors are reported by return code only; nothing aborts or throws across
 *    the ABI.  Argument errors are detected before any launch.  After an error
 *    wdc_last_error(ctx) holds a one-line description.
 *  - Pointers named "device" must point to memory of the context's device;
 *    latents are fp32, contiguous [C, F, H, W] (flat N = C*F*H*W elements) and
 *    16-byte aligned.  The caller owns every pointer it passes; the context
 *    owns its weights, bank latents, workspace and controller state.
 *  - Work is enqueued on the given stream (a cudaStream_t; NULL = the legacy
 *    default stream).  Calls that must return a decision to the host
 *    (wdc_surrogate_step, wdc_rollout) synchronise that stream.
 *  - Step index convention: step k = 0..T-1 maps z_k to z_{k+1}; the paper's
 *    t counts down (t = T - k).  Noise levels sigma_k = 1 - k/T (optionally
 *    time-shifted), model timestep 1000*sigma_k, phase q_k = sigma_k.
 *  - A context is not thread-safe; use one per host thread.
 */
#ifndef WDC_H
#define WDC_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum wdc_status {
    WDC_OK = 0,
    WDC_ERR_INVALID_ARG = 1,   /* bad pointer, size, alignment or config        */
    WDC_ERR_CUDA = 2,          /* a CUDA runtime/driver call failed              */
    WDC_ERR_UNSUPPORTED = 3,   /* valid request this library does not implement    */
    WDC_ERR_TIMEOUT = 4,       /* a bounded device-side wait gave up             */
    WDC_ERR_NONFINITE = 5,     /* reserved: non-finite data where it is an error */
    WDC_ERR_STATE = 6,         /* call out of order for the context's state      */
    WDC_ERR_OOM = 7            /* device allocation failed                       */
} wdc_status;

enum { WDC_F32 = 0, WDC_BF16 = 1 };

#define WDC_MAX_BANK 8          /* largest supported bank capacity K           */
#define WDC_MAX_BATCH 16        /* most latents one batched forward may hold   */
#define WDC_SUMMARY_DIM 256     /* the fixed summary s(.) (section "Kernelized Nonlinear Observation") */
#define WDC_SKETCH 120          /* buckets of each latent block of s(.)        */

typedef struct wdc_ctx wdc_ctx;
typedef void* wdc_stream;       /* a cudaStream_t */

/* The denoiser F_theta: an adaLN DiT over video-latent tokens.  The paper
 * takes F_theta from the backbone (Introduction, Eq. 1); layer layout:
 *   x = [Linear(cond tokens); Linear(patchify(z)) + sinusoidal position]
 *   per block: x += g1*(Wo Attn(LN(x)(1+s1)+b1) + bo);
 *              x += g2*(W2 GELU_tanh(W1(LN(x)(1+s2)+b2) + b1') + b2')
 *   v = unpatchify(Wf(LN(x_video)(1+sf)+bf) + bf')
 * layers == 0 creates a context without a denoiser (controller and fused step
 * kernels only); then the latent shape [in_ch, frames, height, width] is
 * arbitrary. */
typedef struct wdc_dit_config {
    int layers, hidden, heads, head_dim, mlp, temb_dim, freq_dim;
    int in_ch, frames, height, width, patch;
    int cond_tokens, cond_dim;
    int dual_stream;            /* 1: separate block weights for condition tokens */
    int dtype;                  /* WDC_F32 (fp32 parity mode) or WDC_BF16          */
    int max_batch;              /* latents one batched forward may hold, counting
                                   both halves of a guided pair (0 or 1: single;
                                   at most WDC_MAX_BATCH); activation buffers
                                   are sized for it */
} wdc_dit_config;

/* Flow-matching Euler schedule: sigma_k = 1 - k/T, shifted by
 * s*sigma/(1+(s-1)*sigma) when shift != 1. */
typedef struct wdc_schedule {
    int T;
    double shift;
} wdc_schedule;

/* Constants of Eq. 3-10.  The paper defers their values to supplementary
 * material; wdc_default_cache_params() fills the readings this library uses. */
typedef struct wdc_cache_params {
    int bank_capacity;          /* FIFO capacity K of the bank, 1..WDC_MAX_BANK  */
    int min_support;            /* |N_t| needed for adequate support             */
    double sim_min, q_gap_max;  /* compatibility (Eq. 3 text)                    */
    double gamma_q, tau_in;     /* retrieval score and temperature (Eq. 3)       */
    double tau_obs;             /* observation temperature tau (Eq. 5)           */
    double alpha_min, alpha_max;/* clip of the scheduler scaling (Eq. 4)         */
    double eps, eps_nu;         /* Eq. 4/7/8 epsilon; RMS-normalisation epsilon  */
    uint32_t sketch_seed;       /* seed of the summary's sign hash               */
    double w_z, w_age, w_phase, w_cam, w_depth;   /* proxy weights (Eq. 6)       */
    double eta_init, eta_min, eta_max, beta_d;    /* calibration (Eq. 8)         */
    double a_cam, a_depth, a_phase;               /* impact weight (Eq. 9)       */
    double lambda_, tau_risk;                     /* decay and threshold (Eq. 9-10) */
    int max_age;                /* pre-decision anchor age limit (Eq. 10 text)   */
    int n_init_exact, n_final_exact;              /* mandatory-exact phases      */
    int flags;                  /* WDC_ABL_* ablation bits, WDC_OBS_RESIDUAL     */
    int period;                 /* WDC_ABL_PERIODIC: exact step every `period`   */
    double ridge;               /* WDC_ABL_LINEAR_OBS: relative ridge            */
} wdc_cache_params;

/* Ablation variants (section "Ablation Study", Tables 3 and 4), bits of
 * wdc_cache_params.flags.  The paper names them and defers their definitions
 * to supplementary material; these are this library's readings.  Any
 * combination is accepted (WDC_ABL_SECANT makes WDC_ABL_LINEAR_OBS and
 * WDC_ABL_NO_SUPPORT moot: the secant uses no retrieval or observation).
 *   PERIODIC      Eq. 10's risk test replaced by a fixed period: Surrogate iff
 *                 Available_t and age_t + 1 < period (Available_t kept).
 *   SECANT        native latent secant candidate z_hat = z_t + alpha_t
 *                 (z_a - z_a,in): the latest exact displacement scaled by
 *                 Eq. 4's alpha; its support term holds whenever the bank is
 *                 non-empty.  The context keeps that displacement (one more
 *                 latent-sized buffer, written by the exact-step pass).
 *   INSTANT_RISK  instantaneous risk: lambda = 0 in Eq. 9 (R_cand = Delta_t).
 *   NO_IMPACT     w/o impact weighting: w_t = 1 in Eq. 9.
 *   NO_CALIB      w/o counterfactual calibration: eta_d stays eta_init (d_cf
 *                 is still measured and reported).
 *   NO_SUPPORT    w/o support constraint: retrieval over the whole bank (no
 *                 compatibility filter); the support term always holds.
 *   LINEAR_OBS    linear observation: Eq. 5's softmax weights replaced by the
 *                 ridge least-squares coefficients beta of s(phi_hat) on the
 *                 records' output summaries, (G + rho I) beta = S_out s_hat,
 *                 G_ij = s_out_i . s_out_j, rho = ridge * trace(G) / n_bank;
 *                 z_hat = sum_i beta_i z_out_i.
 *   NO_COND       condition descriptors left out of the lift (Eq. 2): the
 *                 camera / depth entries of every summary are zero; the
 *                 controller (Eq. 6, 9) still uses them. */
#define WDC_ABL_PERIODIC     0x01
#define WDC_ABL_SECANT       0x02
#define WDC_ABL_INSTANT_RISK 0x04
#define WDC_ABL_NO_IMPACT    0x08
#define WDC_ABL_NO_CALIB     0x10
#define WDC_ABL_NO_SUPPORT   0x20
#define WDC_ABL_LINEAR_OBS   0x40
#define WDC_ABL_NO_COND      0x80
#define WDC_ABL_ALL          0xFF

/* Reading flag (also in wdc_cache_params.flags), not an ablation:
 *   OBS_RESIDUAL  residual reading of Eq. 5's observation: the kernel weights
 *                 blend the records' exact latent displacements instead of
 *                 their outputs, z_hat = z_t + sum_i kappa_i (z_out_i - z_in_i).
 *                 Eq. 5 as printed (the default) is a convex combination of
 *                 stored exact outputs and so cannot move the latent past the
 *                 bank; this reading can.  The context keeps one displacement
 *                 buffer per bank slot (written by the exact-step pass); like
 *                 the secant's, they are not part of wdc_state_host and
 *                 wdc_state_set clears them. */
#define WDC_OBS_RESIDUAL     0x100

/* Model condition c of one step.  tokens: [cond_tokens, cond_dim] fp32, device
 * or host memory (NULL only when layers == 0).  cam/depth: the camera/motion
 * and depth/geometry descriptors of the lift (Eq. 2); zero when missing. */
typedef struct wdc_cond {
    const float* tokens;
    double cam[4];
    double depth[4];
} wdc_cond;

/* Per-step record filled by the step calls (host memory). */
typedef struct wdc_step_info {
    int k;
    int decision;               /* 1 Surrogate, 0 Exact (Eq. 10)                 */
    int finite, supported, n_compat, n_bank, age;
    double q, alpha, p, d_hat, w, delta, R_cand, R, eta, d_cf, d_z, r;
    double kappa[WDC_MAX_BANK], pi[WDC_MAX_BANK];
} wdc_step_info;

/* One bank record's small fields (section "Local Lifted Evolution"): the
 * summaries of the lifted input and output and their increment, the phases,
 * the relative RMS increment r of the transition and its descriptors. */
typedef struct wdc_record_host {
    double s_in[WDC_SUMMARY_DIM], s_out[WDC_SUMMARY_DIM], s_dphi[WDC_SUMMARY_DIM];
    double q_in, q_out, r;
    double cam[4], depth[4];
} wdc_record_host;

/* Host view of the controller and memory state.  In wdc_state_set the
 * "derived" fields are ignored and recomputed on the device from the latents. */
typedef struct wdc_state_host {
    int n_bank;                 /* records rec[0..n_bank-1], oldest first        */
    int age;                    /* surrogate steps since the latest exact step   */
    double R, eta;              /* stored risk and calibration gain              */
    double q_a_in, q_a_out;     /* latest exact interval                         */
    double cam_a[4], depth_a[4];/* descriptors of the latest exact step          */
    wdc_record_host rec[WDC_MAX_BANK];
    /* derived (read back only) */
    double cur_sketch[WDC_SKETCH], cur_sumsq, cur_sumsq_anchor;
    double anchor_sketch[WDC_SKETCH], anchor_sumsq;
    double s_phi[WDC_SUMMARY_DIM];
    int cand_supported, cand_finite;
    double cand_p;
} wdc_state_host;

/* Parameter tensors of the denoiser (wdc_set_tensor).  Shapes, [out, in] for
 * Linear weights; D hidden, E temb_dim, M mlp, P = in_ch*patch*patch, Fd freq_dim. */
enum wdc_tensor_id {
    WDC_T_PATCH_W = 0,  /* [D, P]    */  WDC_T_PATCH_B = 1,  /* [D]   */
    WDC_T_COND_W = 2,   /* [D, Dc]   */  WDC_T_COND_B = 3,   /* [D]   */
    WDC_T_T1_W = 4,     /* [E, Fd]   */  WDC_T_T1_B = 5,     /* [E]   */
    WDC_T_T2_W = 6,     /* [E, E]    */  WDC_T_T2_B = 7,     /* [E]   */
    WDC_T_FMOD_W = 8,   /* [2D, E]   */  WDC_T_FMOD_B = 9,   /* [2D]  */
    WDC_T_FINAL_W = 10, /* [P, D]    */  WDC_T_FINAL_B = 11, /* [P]   */
    /* per (layer, stream) */
    WDC_T_MOD_W = 12,   /* [6D, E]   */  WDC_T_MOD_B = 13,   /* [6D]  */
    WDC_T_QKV_W = 14,   /* [3D, D]   */  WDC_T_QKV_B = 15,   /* [3D]  */
    WDC_T_O_W = 16,     /* [D, D]    */  WDC_T_O_B = 17,     /* [D]   */
    WDC_T_FC1_W = 18,   /* [M, D]    */  WDC_T_FC1_B = 19,   /* [M]   */
    WDC_T_FC2_W = 20,   /* [D, M]    */  WDC_T_FC2_B = 21,   /* [D]   */
    WDC_T_COUNT = 22
};

/* ------------------------------------------------------------------ lifetime */
const char* wdc_status_string(wdc_status s);
/* Fills the parameter readings used by default (see wdc_cache_params). */
wdc_status wdc_default_cache_params(wdc_cache_params* out);
/* Creates a context on CUDA device `device`: validates the configs, allocates
 * the weights (when layers > 0), the K bank latents, two candidate buffers,
 * the velocity buffer, the DiT workspace and the device controller state.
 * WDC_ERR_OOM if device memory is short. */
wdc_status wdc_create(const wdc_dit_config* cfg, const wdc_schedule* sched,
                      const wdc_cache_params* params, int device, wdc_ctx** out);
void wdc_destroy(wdc_ctx* ctx);
/* Replaces the constants of Eq. 3-10 (validated as in wdc_create).  The bank
 * capacity must stay the same (WDC_ERR_INVALID_ARG otherwise); the state is
 * kept, so call it between rollouts. */
wdc_status wdc_set_cache_params(wdc_ctx* ctx, const wdc_cache_params* params);
const char* wdc_last_error(const wdc_ctx* ctx);
size_t wdc_latent_numel(const wdc_ctx* ctx);
/* Number of kernels this context has launched so far (all streams). */
unsigned long long wdc_launch_count(const wdc_ctx* ctx);
/* Which kernels ran a bf16 context's GEMMs so far (a diagnostic: the kernel is
 * chosen from the shape).  counts[kernel * WDC_GEMM_FORMS + form] += 1 for a
 * launch of one problem, += 1 << 32 for a grouped one (a dual-stream block's
 * video and condition rows).  WDC_ERR_INVALID_ARG on a null pointer. */
enum wdc_gemm_kernel {
    WDC_GEMM_PAIR256 = 0, WDC_GEMM_PAIR192 = 1, WDC_GEMM_PAIR128 = 2,   /* CTA pairs, 256-row tiles this wide */
    WDC_GEMM_ONE128 = 3, WDC_GEMM_ONE64 = 4,                            /* one CTA, 128-row tiles this wide   */
    WDC_GEMM_SPLIT2 = 5, WDC_GEMM_SPLIT4 = 6, WDC_GEMM_SPLIT8 = 7,      /* K over this many CTAs              */
    WDC_GEMM_KERNELS = 8
};
enum wdc_gemm_form {
    WDC_GEMM_STORE = 0, WDC_GEMM_GELU = 1, WDC_GEMM_RESID = 2, WDC_GEMM_QKV = 3, WDC_GEMM_UNPATCH = 4,
    WDC_GEMM_RESID_GELU = 5, WDC_GEMM_RESID_REPEAT = 6, WDC_GEMM_FORMS = 7
};
wdc_status wdc_gemm_launches(const wdc_ctx* ctx, unsigned long long* counts);
/* Synchronises the device and returns (then clears) the bits the kernels have
 * set in the context's error word: 1 = a bounded device-side wait timed out,
 * 2 = a chunk operator met a page number, length, start or position out of range,
 * 4 = the two CTAs of a tensor-core pair saw different tensor-memory bases,
 * 8 = a bf16 model's QKV projection produced a value of V beyond fp16's range
 * (|v| > 65504), which was saturated to +-65504 when V^T was stored for the
 * attention (NaN is kept).  Also makes the counters of split 4-bit products zero
 * again, which products that ran at the same time against the rule may have left otherwise. */
wdc_status wdc_device_errors(wdc_ctx* ctx, unsigned* bits);
/* Self-test of the bounded device-side waits (the paper has no counterpart):
 * one CTA waits on an mbarrier that nothing completes, through the same
 * bounded wait the tensor-core kernels use, with a limit of `limit_ns`
 * (1 us .. 1 s).  When the limit passes the wait gives up, sets bit 1 in the
 * context's error word and raises the CTA's abort flag, which releases the
 * CTA's other waiting thread and a waiting warp; another warp waits out a limit
 * of its own; the kernel then returns normally.  Lets a test
 * check the timeout path and that the context stays usable afterwards,
 * without faulting or hanging the GPU.  Asynchronous on `stream`. */
wdc_status wdc_selftest_wait_timeout(wdc_ctx* ctx, unsigned long long limit_ns, wdc_stream stream);
/* Self-test of what wdc_device_errors puts right: leaves the counters of the split 4-bit products
 * (see wdc_op_gemm_fp4) as products that ran at the same time may, so that the next of them would
 * join sums too early.  Lets a test check that wdc_device_errors clears them.  Synchronises the device. */
wdc_status wdc_selftest_fp4_counters(wdc_ctx* ctx);

/* ------------------------------------------------------------------ weights */
/* Copies one parameter tensor (host fp32, `count` elements, shape as listed in
 * wdc_tensor_id) into the model, converting to the model dtype (bf16:
 * round-to-nearest-even).  layer/stream are ignored for global tensors.
 * Synchronous: the tensor is on the device on return, for calls on any stream;
 * calls that still run on a non-blocking stream are not waited for. */
wdc_status wdc_set_tensor(wdc_ctx* ctx, int tensor_id, int layer, int stream,
                          const float* host, size_t count);
/* Reads one parameter tensor back into `host` (fp32, `count` elements, the
 * wdc_set_tensor layout); bf16 values are widened exactly.  Synchronous.  Lets
 * a checker evaluate the model the device actually holds (e.g. after
 * wdc_init_weights).  WDC_ERR_INVALID_ARG on a size mismatch or bad id. */
wdc_status wdc_get_tensor(wdc_ctx* ctx, int tensor_id, int layer, int stream,
                          float* host, size_t count);
/* Initialises every matrix N(0, std^2) and every bias to 0 on the device from
 * a counter-based Philox4x32-10 stream (Salmon et al., SC'11) keyed by seed. */
wdc_status wdc_init_weights(wdc_ctx* ctx, unsigned long long seed, float std);

/* ------------------------------------------------------------------ F_theta */
/* v = F_theta(z_t, t, c) (Eq. 1): z_t device fp32 latent, t the model timestep,
 * cond_tokens device fp32 [cond_tokens, cond_dim], v device fp32 latent-shaped
 * output.  Asynchronous. */
wdc_status wdc_dit_forward(wdc_ctx* ctx, const float* z_t, float t, const float* cond_tokens,
                           float* v, wdc_stream stream);
/* Batched F_theta (the paper runs one trajectory at a time and is silent on
 * batching and on classifier-free guidance; both are serving extensions that
 * do not change what one sample computes).  B latents z_t[b] (device fp32,
 * 16-byte aligned) at the same model timestep t, each with its own condition
 * tokens cond_tokens[b] (device fp32 [cond_tokens, cond_dim]; the array may
 * be NULL when the model has no condition tokens).  One forward holds all of
 * them: every GEMM and row-wise kernel runs once over all samples' tokens,
 * the attention once over all samples' heads (each sample attends to its own
 * tokens only).  Writes v[b] (device fp32, 16-byte aligned, latent-shaped).
 *   cfg == 0: v[b] = F(z_t[b], t, c_b); needs B <= max_batch.
 *   cfg == 1: guided velocity v[b] = F(z, t, 0) + guidance (F(z, t, c_b) -
 *             F(z, t, 0)), where 0 is the all-zero token set (the null
 *             condition); the 2B forwards share one batch, so 2B <= max_batch.
 * A sample's velocity is bitwise the same as that of wdc_dit_forward on it
 * alone.  Host arrays z_t, cond_tokens and v hold B pointers each.  Errors:
 * WDC_ERR_INVALID_ARG for B < 1, B (2B) > max_batch or a null / unaligned
 * pointer.  Asynchronous. */
wdc_status wdc_dit_forward_batch(wdc_ctx* ctx, int B, const float* const* z_t, float t,
                                 const float* const* cond_tokens, int cfg, float guidance,
                                 float* const* v, wdc_stream stream);
/* One DiT block in place on the token sequence x (device, model dtype,
 * [cond_tokens + video_tokens, hidden]) with modulation mod6 (device fp32,
 * [streams][6][hidden] = shift1, scale1, gate1, shift2, scale2, gate2). */
wdc_status wdc_dit_block_forward(wdc_ctx* ctx, int layer, void* x, const float* mod6,
                                 wdc_stream stream);
/* Timestep conditioning: writes [layers][streams][6][hidden] block modulations
 * followed by the final layer's [2][hidden] into mod_out (device fp32). */
wdc_status wdc_dit_modulation(wdc_ctx* ctx, float t, float* mod_out, wdc_stream stream);

/* The schedule's T + 1 noise levels sigma_0..sigma_T (fp64, as the context
 * computes them: sigma_k = 1 - k/T, time-shifted when shift != 1) into the
 * host array out[T + 1].  Step k runs the denoiser at model timestep
 * (float)(1000 sigma_k) and its phase is q_k = sigma_k (section
 * "Condition-Aware Lifted State": the normalised timestep stands in for the
 * scheduler phase). */
wdc_status wdc_schedule_sigmas(const wdc_ctx* ctx, double* out);

/* ------------------------------------------------------------------ diagnostics
 * Device reductions for the synthetic diagnostics of section "Motivation and
 * Observations" (Fig. 2) and section "Transition Risk Controller" (Fig. 3a):
 * for latents a, b and c (device fp32, N elements each, 16-byte aligned; c may
 * be NULL, read as zero) writes to the host array out[5]
 *   out[0] = sum (a - c)^2,  out[1] = sum (b - c)^2,  out[2] = sum (a - c)(b - c),
 *   out[3] = sum (a - b)^2,  out[4] = sum b^2
 * (fp32 arithmetic, deterministic fixed-order reductions), from which the
 * downstream impact ||a - b|| / ||b|| and the direction error between the
 * increments a - c and b - c follow.  Synchronises the stream. */
wdc_status wdc_latent_pair_stats(wdc_ctx* ctx, const float* a, const float* b, const float* c, double* out,
                                 wdc_stream stream);
/* Pearson and Spearman (average ranks) correlations of two host samples x, y
 * of n >= 2 values (Fig. 3a: predicted versus counterfactual defect); NaN
 * when a sample is constant.  Host code, no context or device needed. */
wdc_status wdc_correlations(const double* x, const double* y, int n, double* pearson, double* spearman);

/* ------------------------------------------------------------------ Psi_t */
/* z_next = Psi_k(z_t, v) = z_t + (sigma_{k+1} - sigma_k) v (Eq. 1, flow-matching
 * Euler), elementwise fp32 (one fused multiply-add).  z_next may equal z_t. */
wdc_status wdc_scheduler_step(wdc_ctx* ctx, int k, const float* z_t, const float* v,
                              float* z_next, wdc_stream stream);

/* ------------------------------------------------------------------ cache state */
/* Starts a rollout from z_T (device): empties the bank, R = 0,
 * eta = eta_init, age = 0, anchor z_a := a copy of z_T, and computes the
 * current latent's statistics. */
wdc_status wdc_state_reset(wdc_ctx* ctx, const float* z_T, wdc_stream stream);
/* Reads the controller/memory state back (synchronises the stream). */
wdc_status wdc_state_get(wdc_ctx* ctx, wdc_state_host* out, wdc_stream stream);
/* Installs a state: the small fields from `in`, bank latents copied from
 * z_out[0..in->n_bank-1] (device), the anchor = the newest record's latent
 * (or a copy of z_cur when the bank is empty), and recomputes the derived
 * statistics from z_cur (device) and the anchor.  For tests and resume.  The
 * exact-step displacements kept for WDC_ABL_SECANT / WDC_OBS_RESIDUAL are not
 * part of this state: they are cleared to zero (those candidates equal z_t
 * until exact steps refill them). */
wdc_status wdc_state_set(wdc_ctx* ctx, const wdc_state_host* in, const float* const* z_out,
                         const float* z_cur, wdc_stream stream);

/* ------------------------------------------------------------------ steps */
/* Surrogate candidate and decision of step k (Eq. 2-6, 9, 10) in one fused,
 * HBM-bound pass: lifts the current state (its statistics are held by the
 * context), retrieves and evolves in summary space, and when supported writes
 * z_hat = sum_i kappa_i z_out_i (Eq. 5) to `z_hat` (device, N floats) while
 * reducing the statistics the next step needs; then decides.  On Surrogate the
 * state advances (R <- R_cand, age += 1) and z_hat becomes the current latent
 * (keep the buffer alive until the next step).  On Exact the caller runs
 * F_theta and wdc_risk_update.  Synchronises the stream; `info` (host) gets
 * the step record. */
wdc_status wdc_surrogate_step(wdc_ctx* ctx, int k, const wdc_cond* c, float* z_hat,
                              wdc_step_info* info, wdc_stream stream);
/* Exact branch of step k (Eq. 1, 7, 8; section "Reliability Decision"): one
 * fused pass writes z_exact = Psi_k(z_t, v) straight into the bank's FIFO slot,
 * reduces the counterfactual defect against z_cf (the candidate of the same
 * step, or NULL), calibrates eta_d when that candidate was supported and
 * finite, decays R <- lambda R and inserts the record lifted with the
 * pre-insertion anchor and history.  *z_next receives the device address of
 * z_exact (owned by the context, valid until that slot is recycled).
 * `info` may be NULL; when given, the stream is synchronised and it is
 * completed with d_cf, R, eta and r. */
wdc_status wdc_risk_update(wdc_ctx* ctx, int k, const wdc_cond* c, const float* z_t,
                           const float* v, const float* z_cf, const float** z_next,
                           wdc_step_info* info, wdc_stream stream);

/* ------------------------------------------------------------------ rollouts */
/* The cached rollout (section "Inference and Complexity"): T steps from z_T,
 * each a wdc_surrogate_step and, on Exact, wdc_dit_forward + wdc_risk_update.
 * z_T and z_out may be device or host pointers (host ones are staged through
 * the context's buffers).  conds: n_cond == 1 (used for every step) or T
 * entries; their tokens may be device or host memory (host tokens are copied
 * into a staging buffer the context keeps, grown on the first call that needs
 * more; the call allocates device memory then).  decisions (host int[T]) and trace (host wdc_step_info[T]) may be
 * NULL.  Synchronises the stream once per step. */
wdc_status wdc_rollout(wdc_ctx* ctx, const float* z_T, const wdc_cond* conds, int n_cond,
                       float* z_out, int* decisions, wdc_step_info* trace, wdc_stream stream);
/* The cached rollout of wdc_rollout with device-side control flow (the
 * paper has no counterpart; it changes where the per-step bookkeeping runs,
 * not what is computed): one CUDA graph with a WHILE node over the T steps,
 * a SWITCH node on the bank size selecting the fused skip pass, and IF nodes
 * on the decision, which the skip pass's last CTA sets on the device; so there
 * is no host synchronisation between steps.  Same decisions and latents as
 * wdc_rollout with one condition `cond` for every step.  z_T / z_out and the
 * condition tokens may be host or device memory.  The graph is built on the
 * first call (and again when the pass mode flags WDC_ABL_SECANT /
 * WDC_OBS_RESIDUAL change); the event profiler must be off.  Afterwards the
 * context's step-API state is that of the rollout's end. */
wdc_status wdc_rollout_graph(wdc_ctx* ctx, const float* z_T, const wdc_cond* cond, float* z_out,
                             int* decisions, wdc_step_info* trace, wdc_stream stream);
/* B independent cached rollouts advanced in lockstep (the paper's method per
 * sample; batching itself has no counterpart in the paper).  ctxs[b] holds
 * sample b's cache state and controller parameters; ctxs[0] also owns the
 * denoiser that every sample's exact steps run through (its max_batch must
 * cover the largest exact batch: B, or 2B with cfg), the others may be
 * created with layers == 0.  All contexts must be distinct, on one device,
 * with the same latent size and schedule.  At step k every sample's skip pass
 * runs and decides (one stream synchronisation for all), then the samples
 * that decided Exact share one batched forward (wdc_dit_forward_batch, with
 * cfg / guidance as there) and each runs its anchor pass.  z_T[b] and z_out[b]
 * may be device or host pointers; conds holds B * n_cond entries (sample-major,
 * n_cond 1 or T) whose tokens must be device pointers when the model has
 * condition tokens.  decisions (host int[B*T]) and trace (host
 * wdc_step_info[B*T]), sample-major, may be NULL.  Each sample's decisions,
 * trace and final latent equal those of wdc_rollout on that sample alone
 * (with cfg, of the guided velocity).  Argument errors are reported on
 * ctxs[0]; an error inside one sample's step pass on that sample's context. */
wdc_status wdc_rollout_batch(wdc_ctx* const* ctxs, int B, const float* const* z_T,
                             const wdc_cond* conds, int n_cond, int cfg, float guidance,
                             float* const* z_out, int* decisions, wdc_step_info* trace,
                             wdc_stream stream);
/* The uncached rollout: wdc_dit_forward + wdc_scheduler_step at every step. */
wdc_status wdc_native_rollout(wdc_ctx* ctx, const float* z_T, const wdc_cond* conds, int n_cond,
                              float* z_out, wdc_stream stream);

/* ------------------------------------------------------------------ profiling
 * Per-kernel-class timing for roofline reporting: when enabled, every launch
 * of the library is bracketed by two CUDA events recorded on its launch
 * stream.  wdc_profile_read synchronises the device and returns, per class,
 * the summed event time (ms) and the number of timed launches since the last
 * enable or read (which clears them).  Every launch of the library is on the
 * caller's stream (a dual-stream model's condition rows share their GEMM
 * launches with the video rows), so the per-class times do not overlap.
 * Disabled by default; costs two cudaEventRecord calls per launch when on.
 * Not a method step (no counterpart in the paper). */
enum wdc_kernel_class {
    WDC_K_GEMM = 0,    /* tcgen05 / SIMT GEMMs of the denoiser            */
    WDC_K_ATTN = 1,    /* attention                                      */
    WDC_K_NORM = 2,    /* LayerNorm + modulation                         */
    WDC_K_SKIP = 3,    /* fused skip pass (wdc_surrogate_step)           */
    WDC_K_ANCHOR = 4,  /* fused anchor pass (wdc_risk_update)            */
    WDC_K_OTHER = 5,   /* timestep MLP, patchify, Psi, statistics, init  */
    WDC_K_COUNT = 6
};
wdc_status wdc_profile_enable(wdc_ctx* ctx, int on);
wdc_status wdc_profile_read(wdc_ctx* ctx, double* ms, unsigned long long* launches);

/* ------------------------------------------------------------------ operators
 * The denoiser's hot kernels, exposed for parity tests and roofline timing.   */
/* C = epilogue(A W^T): A [M, K], W [N, K] (model dtype, device, row-major);
 * bias [N] fp32 or NULL; gelu != 0 applies GELU_tanh; when res != NULL
 * C = res + gate * (.) with gate [N] fp32 (NULL = 1) and res/C [M, N] in the
 * model dtype (res may equal C).  A bf16 model runs every GEMM on the tcgen05
 * kernel, which needs N % 32 == 0 and K % 8 == 0: other shapes return
 * WDC_ERR_UNSUPPORTED (the fp32 parity mode takes any shape). */
wdc_status wdc_op_gemm(wdc_ctx* ctx, const void* A, const void* W, const float* bias, void* C,
                       int M, int N, int K, int gelu, const void* res, const float* gate,
                       wdc_stream stream);
/* O = softmax(Q K^T / sqrt(d)) V per head, non-causal: q, k [heads, L, d],
 * vt [heads, d, ldv] (V transposed, row stride ldv), o [L, heads*d]; device
 * memory, 16-byte aligned.  q, k and o are in the model dtype; vt is fp32
 * for an fp32 model (ldv = L) and fp16 for a bf16 model (the QKV projection
 * stores V that way so that the PV product takes the probabilities in fp16),
 * with ldv = L rounded up to a multiple of 8 so that every V^T row starts on
 * a 16-byte boundary; the padding columns are never read.  Any L >= 1; d 64
 * or 128.  A bf16 model may split the last (head, query block) units of the
 * launch over the key range and merge them with a second kernel through a
 * workspace the context owns, so two attention calls of one context must
 * not run concurrently on different streams. */
wdc_status wdc_op_attention(wdc_ctx* ctx, const void* q, const void* k, const void* vt, void* o,
                            int heads, int L, int d, wdc_stream stream);

/* ------------------------------------------------------------------ chunk operators
 * A model rolled out chunk by chunk: the projections of a chunk's tokens in
 * 8-bit floating point, the norms and rotations of its heads, and its attention
 * over a paged cache of the tokens before it (the paper's models attend densely
 * over one clip; these stand beside wdc_op_gemm and wdc_op_attention).  All are
 * asynchronous on `stream`, need a context with a denoiser (layers > 0: it gives
 * the model dtype), check their arguments before any launch (pointers 16-byte
 * aligned unless said) and may be captured into a graph.  A call with no rows
 * (M, T, max_new or the number of sequences 0) returns WDC_OK and launches nothing.  What
 * only the device knows (page numbers, lengths, starts, positions) cannot be
 * refused: a value out of range sets bit 2 (wdc_device_errors), in a sequence
 * without new tokens too (a page number where a token or key of the call lies in the
 * page), and nothing is read or written outside the arrays given here. */

/* q = e4m3(x / s) with a scale for each block of 128 columns of one row
 * (block_rows 1) or of 128 rows (block_rows 128): s = max |x| / 448 over the
 * block, so the block's largest magnitude becomes 448, and a row of M or K that
 * 128 does not divide ends in a narrower block.  x [M, K] in the model dtype,
 * row stride ldx >= K elements; q [M, K] e4m3, contiguous; scale fp32
 * [ceil(K/128)][M] (block_rows 1: one block column's scales side by side, as
 * wdc_op_gemm_fp8 reads them) or [ceil(M/128)][ceil(K/128)] (block_rows 128,
 * for weights).  Division and rounding (to nearest even) are IEEE's; a block of
 * zeros has scale 0; an infinity makes its block's scale infinite (finite
 * values there become 0, infinities NaN), a NaN makes scale and block NaN.
 * K % 16 == 0, K <= 2^31 - 512 and ldx % 8 == 0 (WDC_ERR_UNSUPPORTED otherwise). */
wdc_status wdc_op_quantize_fp8(wdc_ctx* ctx, const void* x, long long ldx, void* q, float* scale, int M, int K,
                               int block_rows, wdc_stream stream);

/* C = epilogue(A W^T) of e4m3 matrices with block scales: A [M, K] with
 * a_scale [ceil(K/128)][M], W [N, K] with w_scale [ceil(N/128)][ceil(K/128)]
 * (wdc_op_quantize_fp8's layouts), any fp32 scales:
 *   sum over blocks b of a_scale[b][m] w_scale[n/128][b] sum_{k in b} A[m,k] W[n,k].
 * A block's 128 products are summed by the tensor core, the scaled block sums
 * in fp32 (the two scales are multiplied first, in fp32 too: their product is to
 * be 0 or a normal number).  bias, gelu, res, gate and C as in wdc_op_gemm (C and res
 * [M, N] in the model dtype, res may equal C); GELU's exponential and quotient
 * are approximations, for either dtype: the result is within 2^-18 of its value for arguments above -5/2 and
 * within 2^-15 below, and may be 0 where it is below 2^-54 in size.  N % 8 == 0 and K % 16 == 0, both at most
 * 2^31 - 512 (WDC_ERR_UNSUPPORTED otherwise). */
wdc_status wdc_op_gemm_fp8(wdc_ctx* ctx, const void* A, const float* a_scale, const void* W, const float* w_scale,
                           const float* bias, void* C, int M, int N, int K, int gelu, const void* res,
                           const float* gate, wdc_stream stream);

/* A paged cache of keys and values: sequence b's token p lies in row p % page
 * of page table[b][p / page].  bf16 models only. */
typedef struct wdc_paged_cache {
    void* k;                    /* device bf16 [pages][kv_heads][page][head_dim]  */
    void* v;                    /* device fp16, the same shape (fp16: see wdc_op_attention) */
    const int* table;           /* device [sequences][table_width] page numbers (4-byte aligned) */
    const int* length;          /* device [sequences]: tokens of each sequence, those of the
                                   present chunk included (4-byte aligned) */
    int pages, page;            /* pages of the pool; tokens a page: 16, 32, 64, 128 or 256 */
    int kv_heads, head_dim;     /* head_dim 64 or 128 */
    int sequences, table_width;
} wdc_paged_cache;

/* What is done to the heads of a chunk's QKV rows: each query and key head is
 * normalised to y = x / sqrt(mean(x^2) + eps) * weight and its first rot_dim
 * elements are turned by the angles of the token's position p: of each pair
 * (a, b), a' = a cos - b sin and b' = b cos + a sin.  Statistics, weights and
 * angles in fp32, one rounding to the model dtype.  (The squares too: a head with
 * elements above about 10^18 comes out zero; without eps, one below 10^-19 is
 * imprecise, and below 10^-23 infinite or NaN.) */
typedef struct wdc_head_norm {
    const float* q_weight;      /* device [head_dim], or NULL (= 1)               */
    const float* k_weight;
    float eps;                  /* >= 0                                           */
    const float* rot;           /* device [rot_positions][rot_dim / 2][cos, sin], or NULL: no rotation */
    int rot_positions, rot_dim; /* rot_dim a multiple of 16, at most head_dim (not looked at
                                   without rot)                                   */
    int interleaved;            /* 1: pairs (2 i, 2 i + 1); 0: pairs (i, i + rot_dim / 2) */
    const int* positions;       /* device [T] (4-byte aligned), or NULL: the token's place in its
                                   sequence.  A position outside the table sets bit 2, and the
                                   nearest one of the table is used */
} wdc_head_norm;

/* Norm and rotation of T rows qkv [T][(heads + 2 kv_heads) * d] (model dtype,
 * row stride ld elements, ld % 8 == 0: query heads, key heads, value heads) into
 * the layout of wdc_op_attention's operands (which has as many key heads as query
 * heads: fewer of them are the caller's to repeat): q [heads, T, d], k [kv_heads,
 * T, d] and, unless vt is NULL, V^T [kv_heads, d, ldv] (fp16 for a bf16 model, beyond whose range
 * values are saturated and set bit 8; ldv as there, its padding columns are left
 * as they are).  d 64 or 128. */
wdc_status wdc_op_qk_norm_rope(wdc_ctx* ctx, const void* qkv, long long ld, int T, int heads, int kv_heads, int d,
                               const wdc_head_norm* norm, void* q, void* k, void* vt, wdc_stream stream);
/* The same for a chunk of new tokens of the cache's sequences: rows
 * q_start[b] .. q_start[b + 1] - 1 are the last tokens of sequence b (q_start
 * device [sequences + 1], non-decreasing, 4-byte aligned).  Writes q [T, heads, d]
 * and appends keys and values to their pages (values fp16, saturated as above).
 * What rows from q_start[sequences] on hold does not matter, and their q is left
 * as it is.
 * The pages that a chunk is appended to belong to one sequence each. */
wdc_status wdc_op_qk_norm_rope_append(wdc_ctx* ctx, const void* qkv, long long ld, int T, int heads,
                                      const wdc_head_norm* norm, const wdc_paged_cache* cache, const int* q_start,
                                      void* q, wdc_stream stream);

/* Attention of a chunk of new tokens over the cache, which already holds their
 * own keys and values: o = softmax(q K^T / sqrt(d)) V for rows q_start[b] ..
 * q_start[b + 1] - 1 of q and o ([T, heads, d] and [T, heads * d], bf16; heads a
 * multiple of kv_heads, at most 128 of them to a key head), the last tokens of
 * sequence b.  max_new: no sequence has more new tokens (rows beyond set bit 2
 * and are left as they are).  The token at place p of a sequence of length L sees
 *   frame == 0: all L tokens;   frame == 1: tokens 0 .. p;
 *   frame >= 2: its frame and those before it, tokens 0 .. min(L, (p / frame + 1) frame) - 1.
 * A row that sees nothing is zero.  Scores, row sums and O are fp32; a
 * probability is held in fp16, as is its exponent relative to its row's base (a
 * maximum of the row's, up to 2^8 below it): those above 2^-8 of the base are off by
 * less than 2^-8 of themselves, relatively, smaller ones by less than twice that
 * down to 2^-14, and below 2^-25 they are 0.  Scores are to stay below 2^27 in
 * size.  Whatever a page holds behind its sequence's last token is not used,
 * infinities and NaN included; a non-finite value V of a token within the
 * sequence may reach every row of the chunk.  Rows from
 * q_start[sequences] on are left as they are.  A sequence's keys may be split over
 * several CTAs and merged, through the workspace wdc_op_attention uses: two
 * attention calls of one context, and graphs that hold some, must not run
 * concurrently.  How they are split follows from the lengths of all sequences of
 * the call (the results of equal calls are equal bit for bit). */
wdc_status wdc_op_attention_paged(wdc_ctx* ctx, const void* q, const wdc_paged_cache* cache, const int* q_start,
                                  int T, int heads, int max_new, int frame, void* o, wdc_stream stream);

/* ------------------------------------------------------------------ a block in four bits
 * What a chunk's block does between its attention and its projections, in few
 * bits: the residual's sum with its norm and modulation, rows and weights in 4-bit
 * floating point, their products, a gated MLP's among them, and the rotation of a
 * video's heads by frame, row and column.  As the chunk operators: asynchronous on
 * `stream`, checked before any launch, capturable, and nothing is launched where there
 * are no rows.  A product may split the sums of some of its tiles and join them through a
 * workspace of its own that the context owns: such calls of one context wait for one another on the
 * device where their streams differ, but a graph that holds calls of wdc_op_gemm_fp4 or
 * wdc_op_gated_fp4 must not run concurrently with another such graph or such a call of its context
 * (the sums would be mixed, those of later calls too until wdc_device_errors is called).
 * (The results of equal calls are equal bit for bit.) */

/* Positions of several axes (frame, row and column of a video's token, say): the
 * turned pairs of a head are in sections, the first pairs[0] of them turned by the
 * first axis, the next pairs[1] by the second, and so on, pair j of a section by
 * table[a][coordinate][j] = (cos, sin) with the token's coordinate on that axis.
 * All pairs together are a multiple of 8, at most head_dim / 2; which elements make
 * pair i of a head is said by wdc_head_norm's `interleaved`, with rot_dim twice all
 * pairs.  An axis may have no pairs: its table, rows and coordinates are not looked
 * at.  A coordinate outside its table sets bit 2, and the nearest one is used. */
typedef struct wdc_rot_axes {
    int axes;                   /* 1 .. 4                                         */
    const float* table[4];      /* device [rows][pairs][cos, sin] of each axis (8-byte aligned) */
    int rows[4], pairs[4];
    const int* coords;          /* device [T][axes] (4-byte aligned)              */
} wdc_rot_axes;

/* wdc_op_qk_norm_rope and wdc_op_qk_norm_rope_append with positions of several axes;
 * the norm's rot is NULL (its rot_positions, rot_dim and positions are not looked at).
 * Where a token is appended still follows from its place in its sequence. */
wdc_status wdc_op_qk_norm_rope_axes(wdc_ctx* ctx, const void* qkv, long long ld, int T, int heads, int kv_heads, int d,
                                    const wdc_head_norm* norm, const wdc_rot_axes* axes, void* q, void* k, void* vt,
                                    wdc_stream stream);
wdc_status wdc_op_qk_norm_rope_append_axes(wdc_ctx* ctx, const void* qkv, long long ld, int T, int heads,
                                           const wdc_head_norm* norm, const wdc_rot_axes* axes,
                                           const wdc_paged_cache* cache, const int* q_start, void* q, wdc_stream stream);

/* A matrix [rows, K] of e2m1 numbers (0, 1/2, 1, 3/2, 2, 3, 4, 6 and their negatives)
 * with an e4m3 scale for 16 columns and an fp32 scale for each row: element (r, k) stands
 * for code * (scale * row_scale).  K is a multiple of 64. */
typedef struct wdc_fp4 {
    void* codes;                /* device [rows][K / 2]: the even column's code in the low four bits */
    void* scale;                /* device e4m3 [ceil(rows / 128)][K / 64][512]: row r's scale of columns
                                   16 j .. 16 j + 15 is byte (r % 32) * 16 + (r / 32 % 4) * 4 + j % 4 of
                                   piece [r / 128][j / 4], without a sign; what rows behind the last hold
                                   is not used */
    float* row_scale;           /* device [rows]                                  */
} wdc_fp4;

/* Rows to e2m1, x [M, K] in the model dtype (row stride ldx >= K elements, ldx % 8 == 0),
 * all in IEEE fp32, roundings to nearest even:
 *   row_scale = max |x| * (1 / 2688) over the row, 0 where that maximum is below 2^-100;
 *   scale     = e4m3(max |x| / (6 row_scale)) over 16 columns, at most 448;
 *   code      = e2m1(x * (1 / (scale * row_scale))), at most 6 in size; 0 where the scale is.
 * A row that holds an infinity or NaN has a NaN row_scale and zeros for the rest: it reads
 * back, and comes out of a product, as NaN.  Scales of the rows behind M of the last 128
 * are written as zeros. */
wdc_status wdc_op_quantize_fp4(wdc_ctx* ctx, const void* x, long long ldx, const wdc_fp4* q, int M, int K,
                               wdc_stream stream);
/* And back: x[m, k] = code * (scale * row_scale) in fp32, rounded to the model dtype. */
wdc_status wdc_op_dequantize_fp4(wdc_ctx* ctx, const wdc_fp4* q, void* x, long long ldx, int M, int K,
                                 wdc_stream stream);

/* C = epilogue(A W^T) of e2m1 matrices A [M, K] and W [N, K]:
 *   sum_k (code scale)_A (code scale)_W, in fp32, times A's row_scale[m], times W's row_scale[n];
 * bias, gelu, res, gate and C as in wdc_op_gemm (C and res [M, N] in the model dtype, res may
 * equal C); GELU's accuracy as in wdc_op_gemm_fp8.  N % 8 == 0 (WDC_ERR_UNSUPPORTED otherwise). */
wdc_status wdc_op_gemm_fp4(wdc_ctx* ctx, const wdc_fp4* A, const wdc_fp4* W, const float* bias, void* C, int M, int N,
                           int K, int gelu, const void* res, const float* gate, wdc_stream stream);
/* A gated MLP's first half in one kernel: C [M, N] = f(A W_gate^T + gate_bias) * (A W_up^T +
 * up_bias) with f(x) = x / (1 + exp(-x)), or GELU_tanh with gelu != 0; W_gate and W_up [N, K],
 * the biases [N] fp32 or NULL.  The products as above; f is within 2^-18
 * of its value for arguments above -5/2 and within 2^-17 below (GELU: 2^-15), and may be 0 where it is below
 * 2^-54 in size. */
wdc_status wdc_op_gated_fp4(wdc_ctx* ctx, const wdc_fp4* A, const wdc_fp4* W_gate, const wdc_fp4* W_up,
                            const float* gate_bias, const float* up_bias, void* C, int M, int N, int K, int gelu,
                            wdc_stream stream);

/* How the two take a shape (a diagnostic: the kernel is chosen from the shape): plan[0] rows of A a tile, 16 to
 * 128, or 256 of the kernel of CTA pairs; plan[1] CTAs that share a tile's K (0: the pairs); plan[2] of the pairs'
 * tiles those that are split over K, plan[3] the parts of each (0: none).  WDC_ERR_INVALID_ARG unless it is
 * one that they take, with rows. */
wdc_status wdc_fp4_plan(wdc_ctx* ctx, int M, int N, int K, int gated, int* plan);

/* The residual's sum, its norm and its modulation, rows [M, D] in the model dtype:
 *   r = x + gate * delta                      (x alone without delta; gate NULL = 1)
 *   y = r / sqrt(mean(r^2) + eps)             (center: (r - mean r) / sqrt(var r + eps))
 *   out = y * (weight + weight_offset) + shift   (weight NULL: y + shift; shift NULL = 0)
 * in fp32 from x and delta to the one rounding of each output: the norm is that of the sum
 * before it is rounded into `total`.  One of out, q8 and q4 takes the result: in the model
 * dtype, in e4m3 as wdc_op_quantize_fp8 (block_rows 1) lays A out, or in e2m1 as
 * wdc_op_quantize_fp4 does, both from the fp32 values.  total and out may be x or delta
 * (the same rows, so the same row stride), but not the same place; q8, q4 and their scales have places of
 * their own (WDC_ERR_INVALID_ARG where an address shows otherwise).  D % 16 == 0 (q4: 64), at most 16384; row strides multiples of 8.  (The
 * squares are fp32 too: a row with values above about 10^18 comes out as shift; without
 * eps, one of zeros, or centred one of equal values, is NaN.) */
typedef struct wdc_add_norm {
    const void* x;              /* device [M, D], row stride ldx elements         */
    const void* delta;          /* device [M, D], row stride ldd, or NULL         */
    void* total;                /* device [M, D], row stride ldt: receives r; or NULL */
    void* out;                  /* device [M, D], row stride ldo; or NULL         */
    long long ldx, ldd, ldt, ldo;
    void* q8;                   /* device e4m3 [M, D], contiguous; or NULL        */
    float* scale;               /* with q8: device fp32 [ceil(D / 128)][M]        */
    const wdc_fp4* q4;          /* host pointer to an e2m1 matrix [M, D]; or NULL */
    const float *gate, *weight, *shift;   /* device [sets][D] fp32, or NULL        */
    float weight_offset;        /* 1 for a modulation by 1 + scale                */
    float eps;                  /* >= 0                                           */
    int rows_per_set;           /* row m goes by vectors m / rows_per_set; 0: one set for all */
    int center;                 /* 0: root-mean-square norm; 1: layer norm        */
} wdc_add_norm;
wdc_status wdc_op_add_norm(wdc_ctx* ctx, const wdc_add_norm* norm, int M, int D, wdc_stream stream);

/* ------------------------------------------------------------------ allocation-free variant
 * wdc_observe_noalloc: the streaming half of the skip pass -- the kernelised
 * observation z_hat = sum_i kappa_i z_out_i over K latents together with the
 * statistics the next lift needs -- for callers that cannot call cudaMalloc
 * (code running under another framework's memory manager or inside a
 * pre-sized arena, processes that must not allocate device memory after set-up).
 * The paper has no counterpart: it is a deployment variant of the same kernel.
 *
 * It allocates nothing and needs no wdc_ctx.  Its scratch (per-CTA partial sums
 * and a completion counter, 256 CTAs x 248 floats + 256 bytes = 254 KB) is a
 * file-scope __device__ array that every GPU loading libwdc.so holds until the
 * process exits.  The first call on a device, with that device current, looks
 * up the array's device address (cudaGetSymbolAddress) and caches it; make that
 * first call before any stream capture.  The cached address belongs to the
 * device's primary context as it was at that first call: after a
 * cudaDeviceReset (or anything else that destroys and re-creates the primary
 * context) restart the process before calling this entry point again.  Each
 * call clears the counter on `stream` before its kernel.  All calls on a
 * device share the scratch, so
 * calls that overlap on the GPU (different streams, no ordering) race; order
 * them on one stream.
 *
 *   z_out      host array of K device pointers (fp32 latents, n elements,
 *              16-byte aligned), 1 <= K <= WDC_MAX_BANK
 *   kappa      host array of K weights (used in fp32, as the skip pass does)
 *   z_a        device fp32 latent (the anchor) for sum (z_hat - z_a)^2
 *   z_hat      device fp32 output, n elements (must not alias the inputs)
 *   stats      device output, 123 doubles: [0..119] raw signed bucket sums
 *              sum_{bucket(i)=b} sign(i) z_hat_i (the summary sketch before its
 *              sqrt(120/n) scale), [120] sum z_hat^2, [121] sum (z_hat - z_a)^2,
 *              [122] count of non-finite z_hat elements
 *   n          elements, 1 <= n < 2^31 (the sign hash indexes 32 bits)
 *   sketch_seed  seed of the sign hash (wdc_cache_params.sketch_seed)
 * Returns WDC_ERR_INVALID_ARG for sizes or pointers outside these limits,
 * WDC_ERR_CUDA if the symbol lookup or the launch fails.  Asynchronous. */
wdc_status wdc_observe_noalloc(const float* const* z_out, int K, const double* kappa, const float* z_a,
                               float* z_hat, double* stats, size_t n, uint32_t sketch_seed, wdc_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* WDC_H */
