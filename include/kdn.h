/*
 * kdn.h -- C ABI of the GB300 (sm_103a) Kalman Delta Network token-mixer
 * library (libkdn.so).
 *
 * Operations (all from "Kalman Delta Networks"):
 *   kdn_diag_fwd / kdn_iso_fwd
 *       Chunked prefill / training forward of the Diagonal KDN (Prop. 3) and
 *       the Isotropic KDN (Prop. 5; App. E): the Moebius uncertainty scan
 *       (eq. kla-box-mobius, eq. iso-kla-box-mobius), the Kalman gain emitted
 *       from the pre-write predictive variance (eq. kla-box-gain,
 *       eq. iso-kla-box-gain, App. F.1 eq. chunk-gain-emission) and the
 *       asymmetric delta-rule memory scan in compact-WY form (App. F.2,
 *       eq. chunk-memory-wy and eq. chunk-memory-output-state).
 *   kdn_diag_bwd / kdn_iso_bwd
 *       Gradients of the forward.  The paper gives no backward; these are
 *       the exact adjoints of the forward recurrence.
 *   kdn_diag_decode_step / kdn_iso_decode_step
 *       One token of the recurrence (the boxed update of Prop. 3 / Prop. 5)
 *       applied in place to a batch of states.
 *
 * Per token t and head h the layer computes, with alpha_t = exp(g_t):
 *   Diagonal:  phat = alpha^2 p + omega;  kappa = phat k / (r + sum phat k^2)
 *              u = mu k^2 / r;            p' = phat / (1 + u phat)
 *   Isotropic: a = mean_i alpha_i^2 (alpha^2 for scalar decay);
 *              bhat = a b + omega;  beta = bhat / (r + bhat |k|^2); kappa = beta k
 *              u = mu |k|^2 / (d_k r); b' = bhat / (1 + u bhat)
 *   Memory:    S' = (I - kappa k^T) diag(alpha) S + kappa v^T;  o = scale * S'^T q
 *
 * Conventions
 *   Ownership  The caller owns every buffer, device and host.  Entry points
 *              allocate no memory (scratch lives in the caller's workspace),
 *              keep no global state between calls and are reentrant.
 *   Pointers   Device pointers unless stated otherwise, 16-byte aligned.
 *   Streams    `stream` is a cudaStream_t passed as void* (NULL = the legacy
 *              default stream).  Every call is asynchronous on that stream.
 *   Errors     Argument errors are detected before anything is launched and
 *              leave all outputs untouched.  A failed launch returns
 *              KDN_ERR_CUDA.
 *   Inputs     q, k, v, g, omega, r are post-activation values: g = log(alpha)
 *              <= 0 (alpha = sigmoid(.) in the paper), omega > 0, r > 0.  The
 *              library does not normalise q or k and applies no gate
 *              activation.
 *   Layouts    (row-major, last index fastest)
 *              q, k            [B, T, H, dk]        v, o, dO      [B, T, H, dv]
 *              r               [B, T, H]
 *              diag: g, omega  [B, T, H, dk]
 *              iso:  omega     [B, T, H];  g [B, T, H, dk] (decay_per_channel=1)
 *                                           or [B, T, H]     (decay_per_channel=0)
 *              S0, ST, dST, dS0 (float32)   [B, H, dk, dv]
 *              p0, pT, dpT, dp0 (float32)   diag [B, H, dk];  iso [B, H]
 *              Gradients have the layout of the input they belong to.
 *   Dtypes     q, k, v, g, omega, r and dO have desc->dtype (float32 or
 *              bfloat16); o and the input gradients have desc->out_dtype.
 *              State is always float32.  Accumulation is float32; the
 *              bf16 d = 128 forward runs its intra-chunk products on the
 *              tensor cores with tf32 and fp16 operands (Sec. 4.2 products,
 *              float32 accumulators).
 *   Sizes      dk, dv in {32, 64, 128}; T >= 0 (any length; a ragged last
 *              chunk is padded with identity tokens); B, H >= 0.  At most
 *              T = 2^21 tokens, B*H = 65535*1024 sequences and B*T*H =
 *              2^31 - 1 token-heads per call; larger problems return
 *              KDN_ERR_UNSUPPORTED (split them over calls).
 */
#ifndef KDN_H
#define KDN_H

#include <stddef.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  KDN_OK = 0,
  KDN_ERR_INVALID_ARG = 1, /* null / misaligned pointer, bad size or field */
  KDN_ERR_UNSUPPORTED = 2, /* valid but not built (e.g. dk = 96) */
  KDN_ERR_WORKSPACE = 3,   /* workspace missing or smaller than required */
  KDN_ERR_CUDA = 4,        /* a CUDA launch or runtime call failed */
  KDN_ERR_TIMEOUT = 5,     /* a bounded device-side wait gave up */
  KDN_ERR_RANGE = 6        /* device status only: a 64-token chunk's cumulative log-decay
                              G_C left a fused kernel's range in some channel (results of
                              that call are invalid).  The single-pass bf16 d = 128
                              diagonal forward (kdn_diag_fwd) takes any decay.  The calls
                              that write or read the backward context (the *_fwd_save /
                              *_bwd_saved pairs, the fused backwards), the isotropic fused
                              forward and the sequence-parallel forward take
                              exp(G_C) >= 1e-36, G_C >= -82.8.  desc->chunk = 32 halves
                              the exposure. */
} kdn_status_t;

/* KDN_F8E4M3 is an output type of kdn_add_rmsnorm_fwd only. */
typedef enum { KDN_F32 = 0, KDN_BF16 = 1, KDN_F8E4M3 = 2 } kdn_dtype_t;

typedef struct {
  int B, T, H;           /* batch, tokens, heads */
  int dk, dv;            /* key and value head dimensions */
  int chunk;             /* memory-chunk length C_m of App. F.2: 0 (= 64), 32 or 64;
                            a tuning choice, results agree to rounding */
  int dtype;             /* kdn_dtype_t of q, k, v, g, omega, r and dO (the
                            stored dtype of o and the gradients is out_dtype) */
  float mu;              /* information scale of eq. diag-cov-update; <= 0 -> dk */
  float scale;           /* query scale tau of App. F.2; NaN -> 1/sqrt(dk) */
  int decay_per_channel; /* isotropic only: 1 -> g is [B,T,H,dk], 0 -> [B,T,H].
                            Ignored by the diagonal variant (always per channel). */
  int out_dtype;         /* kdn_dtype_t of o and of dq, dk, dv, dg, domega, dr.
                            0 (KDN_F32, the zero-initialised default) keeps the
                            float32 accumulators; KDN_BF16 rounds them once on
                            store. */
  int gates;             /* kdn_gates_t: what g, omega and r hold (below) */
  float r_min;           /* observation-noise floor of KDN_GATES_LOGITS (>= 0) */
} kdn_desc_t;

/* The gate inputs.  KDN_GATES_POST (0, the zero-initialised default): g = log
   alpha <= 0, omega > 0 and r > 0 as the recurrence uses them.  KDN_GATES_LOGITS:
   g, omega and r are the pre-activation values x, y, z of the layer's
   parameterisation (eq. kla-box-parameterization; r_min of Sec. 5):
   alpha = sigmoid(x), omega = softplus(y), r = r_min + softplus(z), applied
   in float32 inside the kernels.  The backward then returns the gradients with
   respect to x, y and z (in dg, domega, dr). */
typedef enum { KDN_GATES_POST = 0, KDN_GATES_LOGITS = 1 } kdn_gates_t;

/* Library version as major*10000 + minor*100 + patch. */
int kdn_version(void);

/* Human-readable name of a status code (static string, never NULL). */
const char *kdn_status_string(kdn_status_t status);

/* Workspace (device scratch) bytes that kdn_*_fwd / kdn_*_bwd need for this
   descriptor; variant 0 = diagonal, 1 = isotropic.  Returns 0 for an invalid
   descriptor.  The workspace must be 256-byte aligned; its contents need no
   initialisation and are clobbered by every call.
   For bf16 inputs with d_k = d_v = 128 and few long sequences (B*H*P <= 152
   for some P >= 4 that divides the T/64 chunks into segments of >= 8 chunks,
   T a multiple of 64) the forward runs sequence-parallel: it cuts each
   sequence into P segments, joined exactly (uncertainty by a scan of per-chunk
   Moebius summaries, memory by the linearity of the chunk recurrence in
   (S_in, v)), and kdn_fwd_workspace_bytes includes its segment buffers
   (160 KB per (batch, head, segment), 2 KB per (batch, head, chunk), and
   2 bytes per element of o, 6 when out_dtype is KDN_BF16).
   A smaller workspace that still holds the single-pass layout (256 bytes)
   runs the single pass. */
size_t kdn_fwd_workspace_bytes(const kdn_desc_t *desc, int variant);
size_t kdn_bwd_workspace_bytes(const kdn_desc_t *desc, int variant);

/* Forward over T tokens (Prop. 3, App. F).
   S0 NULL -> zero initial memory; p0 NULL -> unit initial uncertainty
   (z_0 = [p_0, 1] of eq. chunk-gain-carry with p_0 = 1).
   ST / pT NULL -> final state not written.  o is always written. */
kdn_status_t kdn_diag_fwd(const kdn_desc_t *desc, const void *q, const void *k,
                          const void *v, const void *g, const void *omega,
                          const void *r, const float *S0, const float *p0,
                          void *o, float *ST, float *pT, void *workspace,
                          size_t workspace_bytes, void *stream);

/* Forward of the Isotropic KDN (Prop. 5, App. E); p0 / pT are b_0 / b_T [B,H]. */
kdn_status_t kdn_iso_fwd(const kdn_desc_t *desc, const void *q, const void *k,
                         const void *v, const void *g, const void *omega,
                         const void *r, const float *S0, const float *p0,
                         void *o, float *ST, float *pT, void *workspace,
                         size_t workspace_bytes, void *stream);

/* Backward: gradients of <dO, o> + <dST, ST> + <dpT, pT> with respect to every
   forward input.  It recomputes the forward from the inputs (no saved
   context).  dST / dpT NULL -> zero cotangent.  dS0 / dp0 / dmu NULL -> not
   written; all other gradient pointers are required.  dmu [B,H] float32: the
   gradient with respect to the information scale mu of each sequence (mu
   enters only through u of eq. diag-cov-update / Prop. 5); a mu shared by all
   sequences has the sum.  The gradient of a learned initial uncertainty
   c_{0,h} (p_0 = c_{0,h} in every channel) is the per-head sum of dp0. */
kdn_status_t kdn_diag_bwd(const kdn_desc_t *desc, const void *q, const void *k,
                          const void *v, const void *g, const void *omega,
                          const void *r, const float *S0, const float *p0,
                          const void *dO, const float *dST, const float *dpT,
                          void *dq, void *dk, void *dv, void *dg, void *domega,
                          void *dr, float *dS0, float *dp0, float *dmu, void *workspace,
                          size_t workspace_bytes, void *stream);

kdn_status_t kdn_iso_bwd(const kdn_desc_t *desc, const void *q, const void *k,
                         const void *v, const void *g, const void *omega,
                         const void *r, const float *S0, const float *p0,
                         const void *dO, const float *dST, const float *dpT,
                         void *dq, void *dk, void *dv, void *dg, void *domega,
                         void *dr, float *dS0, float *dp0, float *dmu, void *workspace,
                         size_t workspace_bytes, void *stream);

/* Training pair.  kdn_diag_fwd_save is kdn_diag_fwd that also keeps, in
   `saved`, the context the chunked backward needs (App. F): for every 64-token
   chunk the memory S entering it, its R = U - W S_in, -W, A_qk,
   A = (I + T)^-1 and (Diagonal KDN) Y = V - Kbar S_in as fp16 tiles (96 KB),
   the pre-write variance phat and the cumulative decay gamma of every
   (token, channel) in float32 (64 KB), per-token scalars (2 KB), and the
   float32 uncertainty p entering it.  kdn_diag_bwd_saved is kdn_diag_bwd that starts from that
   context instead of recomputing the forward (same gradients, one kernel).
   kdn_iso_fwd_save / kdn_iso_bwd_saved are the same for the Isotropic KDN.
   Served for bfloat16 activations, dk = dv = 128 and the default chunk; for
   every other descriptor kdn_saved_bytes() returns 0 and the calls return
   KDN_ERR_UNSUPPORTED (use kdn_*_fwd / kdn_*_bwd).
   saved: caller-owned device buffer of kdn_saved_bytes(desc, variant) bytes, 256-byte
   aligned (a smaller or misaligned one -> KDN_ERR_WORKSPACE).  It is written
   by kdn_diag_fwd_save and read by kdn_diag_bwd_saved, which must see the same
   descriptor and the same q, k, v, g, omega, r (and the forward's S0, p0).
   workspace: kdn_fwd_workspace_bytes(desc, variant) bytes for both calls.  The
   other arguments are those of kdn_*_fwd / kdn_*_bwd. */
size_t kdn_saved_bytes(const kdn_desc_t *desc, int variant);

kdn_status_t kdn_diag_fwd_save(const kdn_desc_t *desc, const void *q,
                               const void *k, const void *v, const void *g,
                               const void *omega, const void *r,
                               const float *S0, const float *p0, void *o,
                               float *ST, float *pT, void *saved,
                               size_t saved_bytes, void *workspace,
                               size_t workspace_bytes, void *stream);

kdn_status_t kdn_diag_bwd_saved(const kdn_desc_t *desc, const void *q,
                                const void *k, const void *v, const void *g,
                                const void *omega, const void *r,
                                const void *saved, size_t saved_bytes,
                                const void *dO, const float *dST,
                                const float *dpT, void *dq, void *dk, void *dv,
                                void *dg, void *domega, void *dr, float *dS0,
                                float *dp0, float *dmu, void *workspace,
                                size_t workspace_bytes, void *stream);

kdn_status_t kdn_iso_fwd_save(const kdn_desc_t *desc, const void *q,
                              const void *k, const void *v, const void *g,
                              const void *omega, const void *r,
                              const float *S0, const float *p0, void *o,
                              float *ST, float *pT, void *saved,
                              size_t saved_bytes, void *workspace,
                              size_t workspace_bytes, void *stream);

kdn_status_t kdn_iso_bwd_saved(const kdn_desc_t *desc, const void *q,
                               const void *k, const void *v, const void *g,
                               const void *omega, const void *r,
                               const void *saved, size_t saved_bytes,
                               const void *dO, const float *dST,
                               const float *dpT, void *dq, void *dk, void *dv,
                               void *dg, void *domega, void *dr, float *dS0,
                               float *dp0, float *dmu, void *workspace,
                               size_t workspace_bytes, void *stream);

/* Effective write strength of every token, beta_eff,t = k_t^T kappa_t (the
   coefficient of the residual identity of eq. appendix-effective-write:
   v_t - S_t^T k_t = (1 - beta_eff,t)(v_t - Shat_t^T k_t); 0 <= beta_eff < 1),
   read from the per-token gain scalars a kdn_*_fwd_save call stored in `saved`
   (same descriptor and variant).  Diagonal: 1 - r_t / s_t with
   s_t = r_t + sum_i phat_i k_i^2; Isotropic: beta_t |k_t|^2.
   r: the r input that call was given (logits when desc->gates says so).
   beta_eff: float32 [B,T,H].  One small kernel, asynchronous on `stream`.
   Returns KDN_ERR_UNSUPPORTED for descriptors kdn_*_fwd_save does not serve,
   KDN_ERR_INVALID_ARG for a null or misaligned pointer, KDN_ERR_WORKSPACE when
   saved_bytes < kdn_saved_bytes(desc, variant). */
kdn_status_t kdn_diag_beta_eff(const kdn_desc_t *desc, const void *saved,
                               size_t saved_bytes, const void *r, float *beta_eff,
                               void *stream);
kdn_status_t kdn_iso_beta_eff(const kdn_desc_t *desc, const void *saved,
                              size_t saved_bytes, const void *r, float *beta_eff,
                              void *stream);

/* One decode token for all B*H heads (the update of Prop. 3), in place:
   S [B,H,dk,dv] and p [B,H,dk] are read and overwritten; o [B,H,dv] is
   written.  Per-step inputs drop the T axis: q, k [B,H,dk], v [B,H,dv],
   g, omega [B,H,dk], r [B,H].  desc->T is ignored.  Needs no workspace. */
kdn_status_t kdn_diag_decode_step(const kdn_desc_t *desc, const void *q,
                                  const void *k, const void *v, const void *g,
                                  const void *omega, const void *r, float *S,
                                  float *p, void *o, void *stream);

/* Isotropic decode step (Prop. 5): p is b [B,H]; omega [B,H];
   g [B,H,dk] or [B,H] per desc->decay_per_channel. */
kdn_status_t kdn_iso_decode_step(const kdn_desc_t *desc, const void *q,
                                 const void *k, const void *v, const void *g,
                                 const void *omega, const void *r, float *S,
                                 float *p, void *o, void *stream);

/* Size of the library-owned scratch array used by kdn_diag_fwd_noalloc. */
#define KDN_NOALLOC_SCRATCH_BYTES ((size_t)32 << 20)

/* Diagonal-KDN forward that allocates nothing and takes no workspace.  The
   paper has no counterpart: this exists for callers that are handed only
   input and output buffers and may not call cudaMalloc (e.g. a latency-
   critical thread where cudaMalloc can stall on a device synchronisation, or
   a framework that forbids allocation outside its own allocator).  Arguments
   and results are those of kdn_diag_fwd without the workspace pair.
   Scratch is a fixed array of KDN_NOALLOC_SCRATCH_BYTES in the library's
   device memory, held by a GPU from the first use of the library on it (CUDA
   loads the module lazily) until the process exits; a problem whose
   single-pass workspace (kdn_fwd_workspace_bytes without the segment buffers
   of the sequence-parallel forward) exceeds it is rejected with
   KDN_ERR_WORKSPACE before anything runs.  The sequence-parallel forward is
   used when its larger workspace fits the array, else the single pass.  The
   first call on a device looks up the array's device address
   (cudaGetSymbolAddress, with that device current) and caches it with the
   device's CUDA context; a later call under another context (after a device
   reset) looks it up again.  Make the first call before any stream capture.
   All calls on a device share the array, so calls that overlap on the GPU
   race and must be serialised by the caller. */
kdn_status_t kdn_diag_fwd_noalloc(const kdn_desc_t *desc, const void *q,
                                  const void *k, const void *v, const void *g,
                                  const void *omega, const void *r,
                                  const float *S0, const float *p0, void *o,
                                  float *ST, float *pT, void *stream);

/* Device status word of the most recent kdn_diag_fwd_noalloc call on the
   current device (kept in the library's scratch array, which the caller cannot
   address): synchronises `stream`, then returns and clears it, as
   kdn_get_device_status does for a workspace (KDN_OK, KDN_ERR_RANGE or
   KDN_ERR_TIMEOUT).  The paper has no counterpart.  Allocates nothing; the
   first call on a device performs the same address look-up as
   kdn_diag_fwd_noalloc. */
kdn_status_t kdn_noalloc_device_status(void *stream);

/* Number of CUDA kernels one call of an entry point launches for this
   descriptor when T > 0 (op 0 = kdn_*_fwd, 1 = kdn_*_bwd, 2 = kdn_*_decode_step,
   3 = kdn_*_fwd_save, 4 = kdn_*_bwd_saved, 5 = kdn_*_beta_eff; variant 0 = diagonal,
   1 = isotropic).  -1 for an invalid descriptor or op, or an op the descriptor
   does not serve.
   Calls with T = 0 launch at most one small fill kernel. */
int kdn_kernel_launches(const kdn_desc_t *desc, int variant, int op);

/* Synchronises `stream`, then returns and clears the device status word kept
   in the first bytes of `workspace`: KDN_OK; KDN_ERR_RANGE when a fused kernel
   met a chunk whose cumulative decay left its range; or KDN_ERR_TIMEOUT when a bounded
   device-side wait of the most recent kdn_*_fwd / kdn_*_bwd call on that
   workspace gave up.  Each of those calls clears the word before it starts. */
kdn_status_t kdn_get_device_status(void *workspace, void *stream);

/* Self-test of the device-side failure reporting: clears the status word of
   `workspace` (any workspace of at least 256 bytes, 256-byte aligned) and
   launches one small kernel. Thread 0 waits, with the bounded wait every
   kernel of this library uses, on an mbarrier phase that nothing completes.
   After 4096 polls, well under a millisecond, the kernel records
   KDN_ERR_TIMEOUT in the word and returns normally, so the CUDA context stays
   usable.
   kdn_get_device_status(workspace, stream) then returns KDN_ERR_TIMEOUT.
   Returns KDN_ERR_INVALID_ARG for a null or misaligned workspace. */
kdn_status_t kdn_selftest_wait_timeout(void *workspace, void *stream);

/* ==========================================================================
 * Operators of the hybrid layer: the paper's hybrid backbone alternates the
 * mixers above with sliding-window attention, each behind a pre-norm on the
 * residual stream.  Same conventions (ownership, streams, errors, alignment).
 *
 * Sliding-window attention with sinks.  Query i of a sequence of len tokens
 * (i < len) sees key j when j <= i and (j > i - window or j < sinks): the last
 * `window` tokens up to itself, and the first `sinks` tokens for good.
 *   s_ij = scale q_i.k_j;  lse_i = log sum_j exp s_ij;  o_i = sum_j exp(s_ij - lse_i) v_j
 * over the keys i sees.  H query heads share Hk key/value heads: query head h
 * reads kv head h / (H / Hk).
 *   Layouts  q, o, dO, dq [B, T, H, d];  k, v, dk, dv [B, T, Hk, d]
 *            lse [B, H, T] float32;  lens [B] int32, NULL -> every len = T
 *            (values are clamped to [0, T])
 *            cache kc, vc [B, Hk, sinks + window, d];  pos [B] int32
 *   Padding  Rows at and past len see nothing and are seen by nothing: their o
 *            and gradients are 0, their lse is -inf, and what q, k, v and dO
 *            hold there (NaN included) is never used.
 *   Values   Live tokens (before len) are taken to be finite.  A NaN or an infinity in
 *            one's k, v, q or dO reaches what its definition names and may also reach
 *            queries and keys that do not see it (a weight of zero times it).
 *   Dtypes   q, k, v, dO, o, the caches and the gradients have desc->dtype.  Scores,
 *            softmax statistics and all sums are float32; with bfloat16 the
 *            weights (and in the backward dS) are rounded to bfloat16 as operands
 *            of the second products.
 *   Sizes    d in {32, 64, 128}; H a multiple of Hk (0 heads only where both are
 *            0); T >= 0, at most 2^21; B, H <= 65535; B*H*T <= 2^31 - 1; window
 *            >= 1, sinks >= 0, window + sinks <= 2^30.
 *   Memory   Outputs overlap neither inputs nor one another (kernels of a call overlap).
 *   Order    Every sum has a fixed order: the same call gives the same bits.
 */
typedef struct {
  int B, T, H, Hk, d; /* batch, tokens, query heads, kv heads, head dimension */
  int window;         /* keys a query sees, itself included */
  int sinks;          /* first tokens that every later query sees too */
  int dtype;          /* kdn_dtype_t of q, k, v, o, dO, gradients and caches */
  float scale;        /* > 0; NaN -> 1/sqrt(d) */
} kdn_swa_desc_t;

/* Workspace bytes of kdn_swa_fwd / kdn_swa_bwd (256-byte aligned, contents
   need no initialisation; its first word is the device status that
   kdn_get_device_status reads).  The backward takes two floats a query head and token and at
   most 160 MB beside them, whatever the window and the sinks.  0 for a descriptor
   that is invalid or not served. */
size_t kdn_swa_fwd_workspace_bytes(const kdn_swa_desc_t *desc);
size_t kdn_swa_bwd_workspace_bytes(const kdn_swa_desc_t *desc);

/* Forward.  lse NULL -> not written (kdn_swa_bwd needs it). */
kdn_status_t kdn_swa_fwd(const kdn_swa_desc_t *desc, const void *q, const void *k,
                         const void *v, const int *lens, void *o, float *lse,
                         void *workspace, size_t workspace_bytes, void *stream);

/* Gradients of <dO, o> with respect to q, k and v from the forward's o and lse
   (same descriptor, inputs and lens).  dk and dv are sums over the query heads
   that share a kv head. */
kdn_status_t kdn_swa_bwd(const kdn_swa_desc_t *desc, const void *q, const void *k,
                         const void *v, const int *lens, const void *o, const float *lse,
                         const void *dO, void *dq, void *dk, void *dv, void *workspace,
                         size_t workspace_bytes, void *stream);

/* The bounded cache of decode: like the mixers' memory its size does not grow
   with the context.  Token t lives in slot t if t < sinks, else in slot
   sinks + (t - sinks) mod window.  kdn_swa_cache_fill copies into it the tokens
   of a prompt (k, v [B, T, Hk, d], lens) that a later token can still see; slots
   that no token of the prompt belongs to are left untouched. */
kdn_status_t kdn_swa_cache_fill(const kdn_swa_desc_t *desc, const void *k, const void *v,
                                const int *lens, void *kc, void *vc, void *stream);

/* One decode token of every sequence: q [B, H, d], k, v [B, Hk, d] are the token at
   position pos[b] (the number of tokens before it).  Its k and v are written into
   the cache and o [B, H, d] is its attention over the tokens it sees, itself
   included.  pos[b] < 0: sequence b is idle, its o is 0 and its cache untouched.
   pos is read on the device and not changed.  Slots that hold no token yet are
   never used, whatever they hold.  desc->T is ignored; needs no workspace. */
kdn_status_t kdn_swa_decode_step(const kdn_swa_desc_t *desc, const void *q, const void *k,
                                 const void *v, void *kc, void *vc, const int *pos,
                                 void *o, void *stream);

/* Residual addition and RMS norm of `rows` rows of D columns:
     h = x + res;  rstd = (mean_c h^2 + eps)^-1/2;  y = h rstd w
   in float32, each output rounded once (y from the unrounded h).
     out_dtype = dtype: y has the activations' type.
     out_dtype = KDN_F8E4M3: y holds e4m3 bytes q with y ~ q * scale,
       scale = max |y| / 448 over the row (block 0) or over each 128 columns
       (block 128; the last block may be shorter), 1 where that maximum is 0 or
       not finite; below float32's normal range it is rounded up and so never 0.
       scales [rows] or [rows, ceil(D / 128)] float32.
   Sizes: D a multiple of 8, at most 16384; rows at most 2^31 - 1. */
typedef struct {
  long long rows;
  int D;
  int dtype;     /* kdn_dtype_t of x, res, h, w, dy, dh, dx: KDN_F32 or KDN_BF16 */
  int out_dtype; /* kdn_dtype_t of y: dtype or KDN_F8E4M3 */
  int block;     /* columns a scale: 0 (the row) or 128; KDN_F8E4M3 only */
  float eps;     /* >= 0 */
} kdn_norm_desc_t;

/* res NULL -> h = x.  h, rstd [rows] NULL -> not written.  h may be x or res. */
kdn_status_t kdn_add_rmsnorm_fwd(const kdn_norm_desc_t *desc, const void *x, const void *res,
                                 const void *w, void *y, void *h, float *rstd,
                                 float *scales, void *stream);

/* Gradients: h and rstd are the forward's, dy the gradient of y, dh that of h from
   the residual stream (NULL -> 0).  dx is the gradient of x and of res alike; dw
   [D] float32.  dx may be dy or dh.  desc->out_dtype must be dtype (the gradient with
   respect to the unquantised y). */
size_t kdn_add_rmsnorm_bwd_workspace_bytes(const kdn_norm_desc_t *desc);
kdn_status_t kdn_add_rmsnorm_bwd(const kdn_norm_desc_t *desc, const void *h, const void *w,
                                 const float *rstd, const void *dy, const void *dh, void *dx,
                                 float *dw, void *workspace, size_t workspace_bytes,
                                 void *stream);

/* Rotary positions of queries and keys.  Of a head's d channels the first `rot` are turned
   in pairs, pair i of a token at position p by the angle p f_i, and multiplied by mscale; the
   others are copied:
     y1 = mscale (x1 cos p f_i - x2 sin p f_i),  y2 = mscale (x1 sin p f_i + x2 cos p f_i)
   with (x1, x2) channels (i, i + rot/2), or (2i, 2i + 1) when interleaved.

   kdn_rope_freqs (host only, no CUDA call) fills a table of rot/2 frequencies,
     f_i = base^(-2i / rot)                                   factor = 1
     f_i = base^(-2i / rot) ((1 - w_i) / factor + w_i)        factor > 1: longer contexts
     w_i = (r_i - beta_slow) / (beta_fast - beta_slow) clipped to [0, 1],  r_i = trained f_i / 2 pi
   (trained = 0: w_i = 0, every position divided by factor): a pair that makes more than beta_fast
   turns over the trained length is kept, one that makes fewer than beta_slow interpolated.
   An entry is f_i / 2 pi, a fraction of a turn, in units of 2^-64; a caller may fill a table of
   its own (any frequency is taken modulo one turn a position).  *mscale (NULL: not wanted) is
   0.1 ln factor + 1 when trained > 0 and factor > 1, else 1.
   The angle of a position is that entry times the position modulo 2^64, which is exact: positions
   of any size (negative ones turn backwards) lose nothing. */
typedef struct {
  int rot;                     /* turned channels: even, 2..256 */
  double base;                 /* > 1 */
  double factor;               /* >= 1 */
  double trained;              /* >= 0: tokens of the trained context */
  double beta_fast, beta_slow; /* beta_fast > beta_slow >= 0 */
} kdn_rope_freqs_t;
kdn_status_t kdn_rope_freqs(const kdn_rope_freqs_t *f, unsigned long long *turns, float *mscale);

/* Layouts  q, qo [B, T, H, d]; k, ko [B, T, Hk, d] (Hk = 0: none).  Rows of tokens may lie
              apart: ldq, ldk, ldqo, ldko elements from one token's row to the next (0: heads * d).
              A single token of every sequence has T = 1.
            turns  host memory, rot/2 entries, read before the call returns
            pos    [B] int32, the position of each sequence's first token (NULL: 0); with
                   pos_per_token [B, T], that of every token
            lens   [B] int32, NULL -> every len = T (values are clamped to [0, T])
   Padding  Rows at and past len are never read; their outputs are 0.
   Dtypes   KDN_F32 or KDN_BF16; float32 arithmetic, each output rounded once.
   Sizes    d a multiple of 8, at most 256; rot even, 2..d; T at most 2^21; H, Hk <= 65535;
            B*T <= 2^31 - 1.
   Memory   qo may be q (with the same row distance) and ko may be k; otherwise outputs overlap
            neither inputs nor one another (KDN_ERR_INVALID_ARG). */
typedef struct {
  int B, T, H, Hk, d;
  int rot;
  int interleaved;   /* 1: pairs are neighbouring channels; 0: half of rot apart */
  int pos_per_token; /* 1: pos is [B, T]; 0: [B] */
  int dtype;
  float mscale;      /* finite */
  long long ldq, ldk, ldqo, ldko;
} kdn_rope_desc_t;
kdn_status_t kdn_rope_fwd(const kdn_rope_desc_t *desc, const unsigned long long *turns, const void *q,
                          const void *k, const int *pos, const int *lens, void *qo, void *ko, void *stream);

/* Gradients: dqo, dko are those of qo, ko (row distances ldqo, ldko), dq and dk those of q and k (ldq,
   ldk): the same turns backwards.  dq may be dqo and dk dko, as above. */
kdn_status_t kdn_rope_bwd(const kdn_rope_desc_t *desc, const unsigned long long *turns, const void *dqo,
                          const void *dko, const int *pos, const int *lens, void *dq, void *dk, void *stream);

/* Gated feed-forward block of `rows` tokens:
     g = x Wg^T,  u = x Wu^T,  h = act(g) u,  y = h Wd^T
     KDN_ACT_SILU: act(g) = g s(g);  KDN_ACT_GELU: g s(2 z), z = sqrt(2/pi) (g + 0.044715 g^3), which
     is the tanh form g (1 + tanh z) / 2;  s(z) = 1 / (1 + e^-z)
   Layouts  x, y, dy, dx [rows, D];  wg, wu, dwg, dwu [F, D];  wd, dwd [D, F];  g, u, h [rows, F]
   Dtypes   desc->dtype throughout, the weights' gradients desc->dw_dtype (dtype or KDN_F32).  Sums and
            the activation are float32; with bfloat16 h and, in the backward, dg and du are rounded to
            bfloat16 as operands of the products behind them, and the backward reads g and u as stored.
            With float32 and more than 16 rows a product's operands are taken as three bfloat16s, which is
            exact to 2^-27 for magnitudes above 1e-33, and the workspace holds them (6 bytes an element of x,
            the weights and h, in the backward also of dy, dg and du).
   Sums     The tensor cores truncate: with bfloat16 a sum loses up to 2^-23 of its accumulator for every 16 terms.
            With float32 weights' gradients an accumulator takes 512 terms, and what it holds is added in float32, rounded
            to nearest; with bfloat16 ones and for y and dx it takes up to 65536 (or 4096 of a longer sum, through
            float32 in the workspace), for g, u and dh all D.
   Values   Inputs are taken to be finite.
   Sizes    D and F multiples of 8, at most 2^20; rows at most 2^31 - 1.
   Memory   Outputs and the workspace overlap neither inputs nor one another: KDN_ERR_INVALID_ARG otherwise.
   Order    Every sum has a fixed order: the same call gives the same bits. */
typedef enum { KDN_ACT_SILU = 0, KDN_ACT_GELU = 1 } kdn_act_t;
typedef struct {
  long long rows;
  int D, F;
  int dtype;    /* kdn_dtype_t: KDN_F32 or KDN_BF16 */
  int act;      /* kdn_act_t */
  int dw_dtype; /* kdn_dtype_t of dwg, dwu, dwd: dtype or KDN_F32 */
} kdn_ffn_desc_t;

/* Workspace bytes (256-byte aligned, contents need no initialisation; its first word is the device
   status that kdn_get_device_status reads).  0 for a descriptor that is invalid or not served. */
size_t kdn_ffn_fwd_workspace_bytes(const kdn_ffn_desc_t *desc);
size_t kdn_ffn_bwd_workspace_bytes(const kdn_ffn_desc_t *desc);

/* Forward.  g and u NULL (both) -> not written (kdn_ffn_bwd needs them); h is always written. */
kdn_status_t kdn_ffn_fwd(const kdn_ffn_desc_t *desc, const void *x, const void *wg, const void *wu,
                         const void *wd, void *g, void *u, void *h, void *y, void *workspace,
                         size_t workspace_bytes, void *stream);

/* Gradients of <dy, y> with respect to x and the weights from the forward's g, u and h. */
kdn_status_t kdn_ffn_bwd(const kdn_ffn_desc_t *desc, const void *x, const void *wg, const void *wu,
                         const void *wd, const void *g, const void *u, const void *h, const void *dy,
                         void *dx, void *dwg, void *dwu, void *dwd, void *workspace,
                         size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* KDN_H */
