/*
 * kla.h - C ABI of the MI355X (gfx950) Kaczmarz Linear Attention hot path.
 *
 * The library computes, per sequence and per head, the gated delta-rule
 * recurrence of the paper (Sec. 3.1 eq. (3), Sec. 3.3 Algorithm 1):
 *
 *     S~   = alpha_t S_{t-1}                      alpha_t = exp(log_alpha_t)
 *     e_t  = v_t - S~^T k_t
 *     beta = eta_t / (||k_t||^2 + eps)            (beta := 0 when the denominator is 0)
 *     S_t  = S~ + beta k_t e_t^T
 *     o_t  = S_t^T q_t                            (no query normalisation in the plain entry points;
 *                                                  the *_opts ones offer Sec. 3.3's o_t / ||q_t||)
 *
 * with the state S a d_k x d_v matrix (Sec. 2), stored row-major with d_v
 * contiguous, always fp32.  The same map written for R = S^T is eq. (5).
 *
 * Conventions for every entry point
 *   - All data pointers are DEVICE pointers unless a parameter says "host".
 *   - The caller owns every buffer and keeps it alive until the stream has
 *     passed the call.  The library allocates and frees nothing and is thread-safe; the
 *     only state it keeps is, per device, the address of the scratch array of
 *     kla_chunk_fwd_static; it reads nothing from the environment.  Work is enqueued on `hip_stream`
 *     (a hipStream_t, NULL = the default stream); the call returns without
 *     waiting for it.
 *   - Return value: KLA_OK or a negative kla_status.  A validation failure is
 *     reported before anything is launched and leaves all outputs untouched.  A
 *     failed launch is reported as KLA_ERR_HIP.
 *   - q, k, v, o share one element type (kla_dtype).  Gates, eps, states are fp32.
 *   - Token-major layout: a tensor "[N, T, H, D]" is contiguous with D fastest.
 *     Data pointers must be 16-byte aligned.
 *   - Supported shapes: dk in {64, 128}; dv in {64, 128, 256}; chunk == 64.
 */
#ifndef KLA_H
#define KLA_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Element type of q, k, v, o.  Passed as a plain int, so that a value that is neither of the two comes back as
 * KLA_ERR_DTYPE (an enum parameter holding any other value is undefined behaviour in C++). */
enum { KLA_F32 = 0, KLA_BF16 = 1 };
typedef int kla_dtype;

typedef enum {
    KLA_OK = 0,
    KLA_ERR_NULL = -1,       /* a required pointer is NULL                               */
    KLA_ERR_SHAPE = -2,      /* unsupported or inconsistent sizes, or eps < 0            */
    KLA_ERR_DTYPE = -3,      /* unknown kla_dtype                                        */
    KLA_ERR_ALIGN = -4,      /* a data pointer is not 16-byte aligned                    */
    KLA_ERR_WORKSPACE = -5,  /* workspace missing or smaller than the query reports      */
    KLA_ERR_SEQLENS = -6,    /* host cu_seqlens not starting at 0, decreasing, or != T   */
    KLA_ERR_HIP = -7         /* the HIP runtime refused a launch                         */
} kla_status;

/* Human-readable name of a status code (static storage, never NULL). */
const char *kla_status_string(int code);

/*
 * Bytes of device scratch kla_chunk_fwd needs for these sizes (0 on invalid sizes).  It covers the per-chunk
 * objects of eqs. (6)-(7) and, for a small bf16 batch of long sequences, the per-segment state maps of the
 * segment-parallel scan (where the fused bf16 kernel runs, which keeps those objects on chip, only a token 256
 * bytes); ask again whenever a size or the element type changes.
 * For a packed batch pass the host copy of cu_seqlens and n_seq > 0 (then N must be 1
 * and T the total token count); otherwise cu_seqlens_host = NULL, n_seq = 0.
 */
size_t kla_chunk_fwd_workspace_bytes(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                                     const int32_t *cu_seqlens_host, int n_seq);

/*
 * Chunkwise-parallel forward (Sec. 4, Algorithm 1 right panel, eqs. (6)-(8)): for every
 * sequence and head, the outputs o_t of all tokens and the state after the last token.
 * The result equals the token loop above; chunks of 64 tokens are counted from each
 * sequence's own first token and never straddle sequences; a sequence of any length >= 0 is
 * accepted (a short last chunk is handled inside the kernels).
 *
 *   q, k        [N, T, H, dk]  dt         in
 *   v           [N, T, H, dv]  dt         in
 *   log_alpha   [N, T, H]      fp32       in   natural log of the decay gate (<= 0 expected)
 *   eta         [N, T, H]      fp32       in   write gate (0..1 expected)
 *   eps                                   in   stabiliser of eq. (3), >= 0
 *   h0          [n_states, H, dk, dv] fp32 in  initial states, or NULL for zeros
 *   o           [N, T, H, dv]  dt         out  must not alias an input
 *   hT          [n_states, H, dk, dv] fp32 out final states, or NULL if unwanted; may alias h0
 *   cu_seqlens_dev  [n_seq+1] int32 device, or NULL for a fixed-length batch
 *   cu_seqlens_host same values on the host (used for grid sizing and validation), or NULL
 *   n_seq       number of packed sequences; 0 for fixed length.  If n_seq > 0 then N == 1,
 *               T is the total token count and n_states = n_seq; otherwise n_states = N.
 *   workspace   device scratch of at least kla_chunk_fwd_workspace_bytes(...) bytes,
 *               256-byte aligned; contents undefined on return.
 */
int kla_chunk_fwd(const void *q, const void *k, const void *v,
                  const float *log_alpha, const float *eta, float eps,
                  const float *h0, void *o, float *hT,
                  const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                  int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * kla_chunk_fwd for callers that cannot allocate device memory and have no workspace to hand over: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Same arguments, results and error
 * codes as kla_chunk_fwd (same kernels) without `workspace` / `workspace_bytes`: whatever kla_chunk_fwd would
 * keep in its workspace - the per-chunk objects of the two-kernel form (fp32 inputs, wide value heads), the maps
 * and states of the segment-parallel scan - goes to a fixed scratch array of KLA_STATIC_SCRATCH_BYTES that is part
 * of the library's device image (every GPU the library is used on holds its own copy from the first use there
 * until the process ends).  The call allocates and frees nothing, neither directly nor through another library.
 *   - A problem whose kla_chunk_fwd_workspace_bytes(...) exceeds KLA_STATIC_SCRATCH_BYTES (the scan order of a packed
 *     batch, at most 1 KiB, does not count) is refused with KLA_ERR_WORKSPACE before anything is launched (32 MiB holds about 2 400 chunk-heads of the two-kernel form
 *     in bf16, 1 200 in fp32; bf16 problems that run the fused kernel need none of it and are never refused).
 *   - The first call on a device looks up the device address of the array (one hipGetSymbolAddress, which may load
 *     the library's code onto that device): make it outside any stream capture.  KLA_ERR_HIP if the lookup fails.
 *   - All calls on one GPU share the one array: two calls that may overlap in time on the same GPU (different
 *     streams, or different threads) race; calls on one stream, or on different GPUs, do not.  Nothing in the
 *     array has to start at zero, every call writes what it reads.
 */
#define KLA_STATIC_SCRATCH_BYTES (32u << 20)
int kla_chunk_fwd_static(const void *q, const void *k, const void *v,
                         const float *log_alpha, const float *eta, float eps,
                         const float *h0, void *o, float *hT,
                         const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                         int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                         void *hip_stream);

/*
 * One recurrent decode step (Algorithm 1 left panel) for B*H independent states.
 *
 *   q, k        [B, H, dk] dt     in
 *   v           [B, H, dv] dt     in
 *   log_alpha, eta [B, H]  fp32   in
 *   S           [B, H, dk, dv] fp32   in/out, updated IN PLACE to S_t
 *   o           [B, H, dv] dt     out
 */
int kla_decode_step(const void *q, const void *k, const void *v,
                    const float *log_alpha, const float *eta, float eps,
                    float *S, void *o,
                    int B, int H, int dk, int dv, kla_dtype dt, void *hip_stream);

/*
 * Options of the *_opts entry points (bit flags; any other bit is KLA_ERR_SHAPE).
 *   KLA_OPT_NORMALIZE_Q  the read-out of Sec. 3.3 / Algorithm 1 (left) as printed,
 *                        o_t = S_t^T q_t / ||q_t||, with o_t = 0 for a zero query; the norm is
 *                        taken over the stored q in fp32.  States are not affected.
 *   KLA_OPT_GDN_BETA     beta_t = eta_t: the gated delta rule the paper starts from (Table 2; the
 *                        "w/o normalization" row of its ablation) instead of eq. (3); eps is
 *                        then unused.
 */
enum { KLA_OPT_NORMALIZE_Q = 1, KLA_OPT_GDN_BETA = 2 };

/*
 * Tuning fields of the same `opts` argument (bits 8..25), for tests and A/B measurements: every setting computes
 * the same results up to rounding, 0 in a field is the library's own choice (the measured best), and a value
 * outside a field's range is KLA_ERR_SHAPE.  They replace any reading of the environment: a call's behaviour
 * depends on its arguments alone.  The workspace needed depends on some of them (segments, the generic and
 * unfused forms), so pass the same `opts` to the *_workspace_bytes_opts query and to the call.
 *   KLA_TUNE_SCAN_WAVES(n)     n = 1, 2, 4: compute waves (16 state columns each) per workgroup of the scan stage
 *   KLA_TUNE_SCAN_SEGMENTS(n)  n = 1: never cut sequences for the segment-parallel scan; n = 2..16: cut into n
 *   KLA_TUNE_GENERIC_SCAN / _INTRA / _BWD   bf16 inputs through plain forms of the kernels, their reference
 *   KLA_TUNE_UNFUSED           bf16 forward as two kernels (intra-chunk stage, then scan) where one fused kernel would run
 *   KLA_TUNE_FUSED             bf16 forward as the one fused kernel wherever it can run (one or two compute waves per
 *                              workgroup, no segments), also where the two-kernel form is the library's choice.  The
 *                              two round different operands to 16 bits (the off-diagonal blocks of I + L; V - D K S)
 *   KLA_TUNE_DECODE_SLICE(n)   n = 32, 64, 128, 256: state columns per workgroup of the decode step
 *   KLA_TUNE_DECODE_NT(n)      n = 0..3: bit 0 non-temporal state loads, bit 1 non-temporal state stores
 */
#define KLA_TUNE_SCAN_WAVES(n)    ((unsigned)((n) == 4 ? 3 : (n)) << 8)
#define KLA_TUNE_SCAN_SEGMENTS(n) ((unsigned)(n) << 10)
#define KLA_TUNE_GENERIC_SCAN     (1u << 15)
#define KLA_TUNE_GENERIC_INTRA    (1u << 16)
#define KLA_TUNE_GENERIC_BWD      (1u << 17)
#define KLA_TUNE_DECODE_SLICE(n)  ((unsigned)((n) == 32 ? 1 : (n) == 64 ? 2 : (n) == 128 ? 3 : (n) == 256 ? 4 : 7) << 18)
#define KLA_TUNE_DECODE_NT(n)     ((unsigned)((n) + 1) << 21)
#define KLA_TUNE_UNFUSED          (1u << 24)
#define KLA_TUNE_FUSED            (1u << 25)

/* Workspace of kla_chunk_fwd_opts(..., opts) / kla_chunk_bwd_opts(..., opts) (0 on invalid sizes or fields);
 * the plain queries are these with opts = 0. */
size_t kla_chunk_fwd_workspace_bytes_opts(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                                          const int32_t *cu_seqlens_host, int n_seq, unsigned opts);
size_t kla_chunk_bwd_workspace_bytes_opts(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                                          const int32_t *cu_seqlens_host, int n_seq, unsigned opts);

/* kla_chunk_fwd with options; kla_chunk_fwd(...) is kla_chunk_fwd_opts(..., 0).  Same workspace. */
int kla_chunk_fwd_opts(const void *q, const void *k, const void *v,
                       const float *log_alpha, const float *eta, float eps,
                       const float *h0, void *o, float *hT,
                       const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                       int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                       void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/* kla_decode_step with options; kla_decode_step(...) is kla_decode_step_opts(..., 0). */
int kla_decode_step_opts(const void *q, const void *k, const void *v,
                         const float *log_alpha, const float *eta, float eps,
                         float *S, void *o,
                         int B, int H, int dk, int dv, kla_dtype dt, void *hip_stream, unsigned opts);

/*
 * Backward pass of kla_chunk_fwd (no options): gradients of
 *     L = sum_t <d_o_t, o_t> + sum <d_hT, hT>
 * with respect to q, k, v, log_alpha, eta and h0.  The paper trains with this operator but states
 * only its forward map (Algorithm 1; eqs. (3), (6)-(8)); the gradients are those equations
 * differentiated chunk by chunk, including the dependence of beta_t on k_t through eq. (3)
 * (d beta / d k = -2 eta k / (||k||^2 + eps)^2), which the delta rule with beta = eta does not have.
 * The forward quantities are recomputed, not saved: only the inputs of the forward call are needed.
 *
 *   q, k, v, log_alpha, eta, eps, h0, cu_seqlens_*, n_seq, N, T, H, dk, dv, chunk, dt: as in kla_chunk_fwd
 *   d_o         [N, T, H, dv]  dt                in   gradient of the outputs
 *   d_hT        [n_states, H, dk, dv] fp32       in   gradient of the final states, or NULL for zeros
 *   dq, dk_     [N, T, H, dk]  dt                out
 *   dv_         [N, T, H, dv]  dt                out
 *   dlog_alpha, deta  [N, T, H] fp32             out
 *   dh0         [n_states, H, dk, dv] fp32       out  or NULL if unwanted
 *   workspace   device scratch of at least kla_chunk_bwd_workspace_bytes(...) bytes, 256-byte aligned.
 *               It holds, per chunk and head, the incoming state and the gradient of the outgoing state
 *               (dk x dv each, in dt) and three [N, T, H, dv] arrays in dt (two for bf16), so it is much larger
 *               than the forward's: about (2 * dk * dv / 64 + 3 * dv) * sizeof(dt) bytes per token and head.
 *               For a small bf16 batch of long sequences it also holds the per-segment maps and states of the
 *               segment-parallel sweeps (as in kla_chunk_fwd).
 * Outputs must not alias inputs or each other.  Same error codes and conventions as kla_chunk_fwd;
 * rows of the outputs are written for every token of every sequence, nothing else is touched.
 * The result is deterministic (no atomics).
 */
size_t kla_chunk_bwd_workspace_bytes(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                                     const int32_t *cu_seqlens_host, int n_seq);
int kla_chunk_bwd(const void *q, const void *k, const void *v,
                  const float *log_alpha, const float *eta, float eps,
                  const float *h0, const void *d_o, const float *d_hT,
                  void *dq, void *dk_, void *dv_, float *dlog_alpha, float *deta, float *dh0,
                  const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                  int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                  void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * kla_chunk_bwd with options: the backward of kla_chunk_fwd_opts(..., opts), same option bits.
 *   KLA_OPT_GDN_BETA     beta_t = eta_t: d eta = d beta and dk loses its term through the coefficient.
 *   KLA_OPT_NORMALIZE_Q  d_o is the gradient of o_t = S_t^T q_t / ||q_t|| (Sec. 3.3); dq is the gradient with respect to
 *                        the stored q (orthogonal to q_t, since o_t does not depend on the length of q_t), 0 for a zero
 *                        query.
 * kla_chunk_bwd(...) is kla_chunk_bwd_opts(..., 0).  Same workspace.
 */
int kla_chunk_bwd_opts(const void *q, const void *k, const void *v,
                       const float *log_alpha, const float *eta, float eps,
                       const float *h0, const void *d_o, const float *d_hT,
                       void *dq, void *dk_, void *dv_, float *dlog_alpha, float *deta, float *dh0,
                       const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                       int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                       void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/*
 * A training step calls both directions on the same inputs, and the backward begins by recomputing what the forward had in
 * its hands: the per-chunk operands, the incoming state of every chunk, the right-hand sides X of eq. (6).  This pair passes them
 * on instead.  kla_chunk_fwd_save is kla_chunk_fwd_opts (same outputs, bit for bit, same workspace) and also fills `saved`;
 * kla_chunk_bwd_saved is kla_chunk_bwd_opts (same gradients, bit for bit) from the unchanged inputs of that forward and `saved`,
 * which it only reads.
 *   saved            device memory, 256-byte aligned, of at least kla_chunk_saved_bytes(...) bytes: about
 *                    (dk * dv / 64 + dv + 154) * sizeof(dt) bytes per token and head (fp32: one dv more).  0: this call
 *                    cannot leave its intermediates (shapes whose forward runs as one kernel or in segments, batches without a
 *                    token, more than KLA_SAVED_MAX_BYTES, the plain kernels); the pair then returns KLA_ERR_SHAPE.
 *   workspace        of kla_chunk_bwd_saved: kla_chunk_bwd_saved_workspace_bytes(...)
 * The size arguments, the offsets of a packed batch (on host and device) and opts have to be those of the forward: what it left
 * behind is laid out by them.
 */
#define KLA_SAVED_MAX_BYTES (1024u << 20)
size_t kla_chunk_saved_bytes(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                             const int32_t *cu_seqlens_host, int n_seq, unsigned opts);
size_t kla_chunk_bwd_saved_workspace_bytes(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                                           const int32_t *cu_seqlens_host, int n_seq, unsigned opts);
int kla_chunk_fwd_save(const void *q, const void *k, const void *v,
                       const float *log_alpha, const float *eta, float eps,
                       const float *h0, void *o, float *hT,
                       const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                       int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                       void *workspace, size_t workspace_bytes, void *saved, size_t saved_bytes,
                       void *hip_stream, unsigned opts);
int kla_chunk_bwd_saved(const void *q, const void *k, const void *v,
                        const float *log_alpha, const float *eta, float eps,
                        const float *h0, const void *d_o, const float *d_hT,
                        void *dq, void *dk_, void *dv_, float *dlog_alpha, float *deta, float *dh0,
                        const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                        int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                        void *workspace, size_t workspace_bytes, const void *saved, size_t saved_bytes,
                        void *hip_stream, unsigned opts);

/*
 * Diagonal gating (App. B, "Extension to diagonal gating"; App. A, decay-agnostic remark): the decay operator is
 * D_t = diag(alpha_t) with one decay per key channel, S~ = diag(alpha_t) S_{t-1} (row i of the d_k x d_v state is
 * scaled by alpha_t[i]); the residual, the Kaczmarz coefficient of eq. (3), the write and the read-out are unchanged.
 * Inside a chunk gamma_i becomes a vector and every decay ratio acts elementwise inside the inner products
 * (L_ij = beta_i sum_c k_ic k_jc gamma_ic/gamma_jc, and likewise for A o Q K^T, the right-hand side and eq. (8)).
 *
 *   log_alpha   [N, T, H, dk] fp32 (chunk forward) or [B, H, dk] fp32 (decode step): natural log of alpha_t per channel
 * Every other argument, the conventions and the error codes are those of kla_chunk_fwd / kla_decode_step.  The
 * workspace (kla_chunk_fwd_diag_workspace_bytes) also holds three [N, T, H, dk] arrays in dt: the keys and queries
 * with the chunk-local decay folded in, which the scan stage consumes.
 */
size_t kla_chunk_fwd_diag_workspace_bytes(int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                                          const int32_t *cu_seqlens_host, int n_seq);
int kla_chunk_fwd_diag(const void *q, const void *k, const void *v,
                       const float *log_alpha, const float *eta, float eps,
                       const float *h0, void *o, float *hT,
                       const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                       int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                       void *workspace, size_t workspace_bytes, void *hip_stream);
int kla_decode_step_diag(const void *q, const void *k, const void *v,
                         const float *log_alpha, const float *eta, float eps,
                         float *S, void *o,
                         int B, int H, int dk, int dv, kla_dtype dt, void *hip_stream);

/* The two diagonal-gating calls with the option bits of kla_chunk_fwd_opts (same meaning: Sec. 3.3 read-out, Table 2's
 * beta_t = eta_t); kla_chunk_fwd_diag(...) and kla_decode_step_diag(...) are these with opts = 0.  Same workspace. */
int kla_chunk_fwd_diag_opts(const void *q, const void *k, const void *v,
                            const float *log_alpha, const float *eta, float eps,
                            const float *h0, void *o, float *hT,
                            const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                            int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                            void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);
int kla_decode_step_diag_opts(const void *q, const void *k, const void *v,
                              const float *log_alpha, const float *eta, float eps,
                              float *S, void *o,
                              int B, int H, int dk, int dv, kla_dtype dt, void *hip_stream, unsigned opts);

/*
 * The Kaczmarz coefficient alone (eq. (3)): beta[i] = eta[i] / (||k_i||^2 + eps), 0 when the
 * denominator is 0, for n_token_heads rows of dk elements.
 *   k [n_token_heads, dk] dt in;  eta [n_token_heads] fp32 in;  beta [n_token_heads] fp32 out.
 */
int kla_beta(const void *k, const float *eta, float eps, float *beta,
             long n_token_heads, int dk, kla_dtype dt, void *hip_stream);

/* ------------------------------------------------------------------------------------------------------------------
 * The operators around the recurrence in a layer: the short convolution ahead of it, another recurrence for hybrid
 * layers, and the norms before and after a block.  The conventions above hold, except:
 *   - Inputs whose row stride ld_* (elements from one token to the next) is an argument may be column ranges of a wider
 *     tensor, e.g. of the output of one projection for several of them; a row itself is contiguous.  Everything else is
 *     contiguous, and so are all outputs.  An output must not overlap an input, except where it says so.
 *   - Data pointers have to be aligned to their element only (A, states and checkpoints: 16 bytes);
 *     rows may start at any element and have any width.
 *   - Parameters (weights, biases, scales) and their gradients are fp32.
 * All sums, states and norms are fp32; an output is rounded to dt once.  Results are deterministic (no atomics).
 * ------------------------------------------------------------------------------------------------------------------ */
enum { KLA_LAYER_SILU = 1,        /* kla_conv_*: y = p sigmoid(p) instead of y = p                                         */
       KLA_LAYER_SOFTPLUS = 2,    /* kla_ssm_*: delta = log(1 + exp(raw + bias)) instead of raw + bias                     */
       KLA_LAYER_SIGMOID = 4,     /* kla_gated_norm_*: the gate's activation is sigmoid(g) instead of g sigmoid(g)         */
       KLA_LAYER_GATE_FIRST = 8   /* kla_gated_norm_*: the gate multiplies what is normalised instead of the result        */ };

/*
 * Short causal convolution of every channel:  p_t[d] = bias[d] + sum_j weight[d][j] x_{t-W+1+j}[d],  y = p sigmoid(p) or p.
 * Before a sequence's first token stands its state, the last W - 1 inputs of the tokens before, oldest first (or zeros).
 *   x           [N, T, D] dt, rows ld_x apart       in
 *   weight      [D, W], bias [D] or NULL            in
 *   state       [n_states, W-1, D] dt or NULL       in   n_states, packed batches: as in kla_chunk_fwd
 *   y           [N, T, D] dt                        out  (y == x: KLA_ERR_SHAPE)
 *   state_out   [n_states, W-1, D] dt or NULL       out  the last W - 1 inputs (state_out == state: KLA_ERR_SHAPE)
 * W in 2..4, D in 1..2^30.
 */
int kla_conv_fwd(const void *x, long ld_x, const float *weight, const float *bias, const void *state,
                 void *y, void *state_out,
                 const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                 int N, int T, int D, int W, kla_dtype dt, void *hip_stream, unsigned opts);

/* Gradients of sum <d_y, y> + sum <d_state_out, state_out> (d_state_out NULL: zeros) from the inputs of the forward.
 * d_y, dx [N, T, D] contiguous; dbias, d_state NULL if unwanted; workspace 256-byte aligned.  dx == x, dx == d_y, d_state == state,
 * d_state == d_state_out: KLA_ERR_SHAPE. */
size_t kla_conv_bwd_workspace_bytes(int N, int T, int D, int W);
int kla_conv_bwd(const void *x, long ld_x, const float *weight, const float *bias, const void *state,
                 const void *d_y, const void *d_state_out,
                 void *dx, float *dweight, float *dbias, void *d_state,
                 const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                 int N, int T, int D, int W, kla_dtype dt,
                 void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/* One token for B sequences: x [B, D], y [B, D], state [B, W-1, D] updated in place. */
int kla_conv_step(const void *x, long ld_x, const float *weight, const float *bias, void *state, void *y,
                  int B, int D, int W, kla_dtype dt, void *hip_stream, unsigned opts);

/*
 * Selective state space scan, one decay per channel and state:
 *     delta_t = softplus(raw_t + delta_bias) (or without softplus)
 *     h_t[d][n] = exp(delta_t[d] A[d][n]) h_{t-1}[d][n] + delta_t[d] u_t[d] B_t[n]
 *     y_t[d] = (sum_n C_t[n] h_t[d][n] + skip[d] u_t[d]) z_t[d] sigmoid(z_t[d])
 *   u, delta (raw), z   [N, T, D] dt, rows ld_u, ld_delta, ld_z apart   in   z NULL: no gate
 *   A           [D, S]                                                  in   (negative expected)
 *   B, C        [N, T, G, S] dt, tokens ld_B, ld_C apart                in   group g serves channels g D/G .. (g+1) D/G - 1
 *   skip, delta_bias [D]                                                in   or NULL
 *   h0          [n_states, D, S] fp32                                   in   or NULL for zeros
 *   y           [N, T, D] dt                                            out
 *   hT          [n_states, D, S] fp32                                   out  or NULL; may alias h0
 *   saved       kla_ssm_saved_bytes(...): the states at every 16th token (every 8th from S = 32 on), for the backward; or NULL
 * S in {8, 16, 32, 64}; D a multiple of G; D and the row strides at most 2^24; at most 65535 sequences and groups (kla_ssm_step: any
 * strides, number of sequences and groups).
 */
size_t kla_ssm_fwd_workspace_bytes(int N, int T, int D, int G, int S, const int32_t *cu_seqlens_host, int n_seq);
size_t kla_ssm_saved_bytes(int N, int T, int D, int G, int S, const int32_t *cu_seqlens_host, int n_seq);
int kla_ssm_fwd(const void *u, long ld_u, const void *delta, long ld_delta, const float *A,
                const void *B, long ld_B, const void *C, long ld_C,
                const float *skip, const void *z, long ld_z, const float *delta_bias, const float *h0,
                void *y, float *hT, float *saved, size_t saved_bytes,
                const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                int N, int T, int D, int G, int S, kla_dtype dt,
                void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/* Gradients of sum <d_y, y> + sum <d_hT, hT> (d_hT NULL: zeros) from the inputs of the forward.  The workspace holds the parts of dB
 * and dC that 32 channels give each: 8 S bytes per token for each 32 channels.  saved: what a forward with these
 * arguments left, or NULL (it is formed again, in the workspace).  du, ddelta, dz [N, T, D], dB, dC [N, T, G, S] contiguous; dz
 * needed iff z; dskip, ddelta_bias, dh0 NULL if unwanted. */
size_t kla_ssm_bwd_workspace_bytes(int N, int T, int D, int G, int S, const int32_t *cu_seqlens_host, int n_seq,
                                   int has_saved);
int kla_ssm_bwd(const void *u, long ld_u, const void *delta, long ld_delta, const float *A,
                const void *B, long ld_B, const void *C, long ld_C,
                const float *skip, const void *z, long ld_z, const float *delta_bias, const float *h0,
                const void *d_y, const float *d_hT, const float *saved, size_t saved_bytes,
                void *du, void *ddelta, float *dA, void *dB, void *dC, float *dskip, void *dz, float *ddelta_bias, float *dh0,
                const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                int N, int T, int D, int G, int S, kla_dtype dt,
                void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/* One token for N sequences: u, delta, z, y [N, D], B, C [N, G, S]; h [N, D, S] fp32 updated in place. */
int kla_ssm_step(const void *u, long ld_u, const void *delta, long ld_delta, const float *A,
                 const void *B, long ld_B, const void *C, long ld_C,
                 const float *skip, const void *z, long ld_z, const float *delta_bias, float *h, void *y,
                 int N, int D, int G, int S, kla_dtype dt, void *hip_stream, unsigned opts);

/*
 * Before a block: the residual stream plus the scaled output of the block before, and its RMS norm.
 *     r' = residual + scale x,   y = weight r' / sqrt(mean(r'^2) + eps)        (0 for a row of zeros with eps = 0;
 * the squares are fp32: elements below 2^-75 count as zeros there, and a row's sum of squares has to stay below 2^128)
 *   x           [M, D] dt, rows ld_x apart          in
 *   residual    [M, D] res_dt                       in   or NULL: r' = scale x
 *   scale       [D] or NULL for ones, weight [D]    in
 *   y           [M, D] dt                           out  of the unrounded r'
 *   residual_out [M, D] res_dt                      out  r', or NULL if unwanted; may alias residual
 * res_dt: dt or fp32.  D at most 8192.
 */
int kla_add_norm_fwd(const void *x, long ld_x, const void *residual, const float *scale, const float *weight, float eps,
                     void *y, void *residual_out, long M, int D, kla_dtype dt, kla_dtype res_dt, void *hip_stream);

/* Gradients of sum <d_y, y> + sum <d_residual_out, r'> (d_residual_out NULL: zeros).  dscale, d_residual NULL if unwanted;
 * d_residual may alias d_residual_out. */
size_t kla_add_norm_bwd_workspace_bytes(long M, int D, kla_dtype dt);
int kla_add_norm_bwd(const void *x, long ld_x, const void *residual, const float *scale, const float *weight, float eps,
                     const void *d_y, const void *d_residual_out,
                     void *dx, void *d_residual, float *dscale, float *dweight,
                     long M, int D, kla_dtype dt, kla_dtype res_dt,
                     void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * After a block: RMS norm of every head, times the activated gate (or, KLA_LAYER_GATE_FIRST, of the head times the gate).
 *     y = weight n act(gate), n = x / sqrt(mean(x^2) + eps);    or  y = weight n, n of x act(gate)
 *   x, gate     [M, H, D] dt, tokens ld_x, ld_gate apart   in
 *   weight      [D]                                        in   the same for all heads
 *   y           [M, H, D] dt                               out
 * D at most 8192.
 */
int kla_gated_norm_fwd(const void *x, long ld_x, const void *gate, long ld_gate, const float *weight, float eps, void *y,
                       long M, int H, int D, kla_dtype dt, void *hip_stream, unsigned opts);
size_t kla_gated_norm_bwd_workspace_bytes(long M, int H, int D, kla_dtype dt);
int kla_gated_norm_bwd(const void *x, long ld_x, const void *gate, long ld_gate, const float *weight, float eps,
                       const void *d_y, void *dx, void *d_gate, float *dweight, long M, int H, int D, kla_dtype dt,
                       void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/* ------------------------------------------------------------------------------------------------------------------
 * Softmax attention, the other mixing layer of hybrid stacks: over whole sequences (forward and backward), and for new
 * tokens over a paged cache of earlier ones.  Query i of a sequence sees keys j of the same sequence:
 *     s_ij = scale q_i . k_j,   p_ij = exp(s_ij) / sum_j exp(s_ij),   o_i = sum_j p_ij v_j,   lse_i = log sum_j exp(s_ij)
 * with KLA_ATTN_CAUSAL j <= i only, and with window > 0 (causal only) j > i - window only.  H query heads share Hk key heads,
 * H a multiple of Hk: query head h reads key head h / (H / Hk).
 *   - q [N, T, H, D], k, v [N, T, Hk, D] dt: tokens ld_q, ld_k, ld_v elements apart (column ranges of a wider tensor), the heads of a
 *     token contiguous.  D is 64 or 128.  Rows start at multiples of 16 bytes: pointers and strides are (else KLA_ERR_ALIGN).
 *   - T H / Hk at most 2^30, H / Hk at most 2^16, H D and strides at most 2^24 elements, scale positive and finite.
 *   - Scores, softmax and sums are fp32; weights are rounded to dt where they are multiplied with values, outputs once.
 *     Results are deterministic (no atomics).  A key that a query does not see has no part in its row, also where it holds a NaN.  A
 *     row whose scores are all -inf, or one of whose scores is +inf or NaN, is NaN; an infinite value makes o infinite, or a NaN where
 *     its weight is 0 in fp32.
 *   - An output must not overlap an input.
 * ------------------------------------------------------------------------------------------------------------------ */
enum { KLA_ATTN_CAUSAL = 1 };

/*   o           [N, T, H, D] dt                     out
 *   lse         [N, T, H] fp32                      out  or NULL if unwanted; what the backward takes
 *   rest        [N, T, H, D] bf16                   out  or NULL if unwanted: what the rounding of o leaves out (dt = bf16 only, else
 *                                                        KLA_ERR_DTYPE), for a backward whose dq and dk do not carry that rounding */
int kla_attn_fwd(const void *q, long ld_q, const void *k, long ld_k, const void *v, long ld_v,
                 void *o, float *lse, void *rest, float scale, int window,
                 const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                 int N, int T, int H, int Hk, int D, kla_dtype dt, void *hip_stream, unsigned opts);

/* Gradients of sum <d_o, o> from the inputs and outputs of the forward (o, lse and, unless NULL, rest).
 *   o, d_o, rest [N, T, H, D] dt, lse [N, T, H] fp32   in   contiguous
 *   dq [N, T, H, D], dk, dv [N, T, Hk, D] dt        out  contiguous
 * workspace 256-byte aligned. */
size_t kla_attn_bwd_workspace_bytes(int N, int T, int H, int Hk, int D, const int32_t *cu_seqlens_host, int n_seq, kla_dtype dt);
int kla_attn_bwd(const void *q, long ld_q, const void *k, long ld_k, const void *v, long ld_v,
                 const void *o, const float *lse, const void *rest, const void *d_o, void *dq, void *dk, void *dv,
                 float scale, int window,
                 const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                 int N, int T, int H, int Hk, int D, kla_dtype dt,
                 void *workspace, size_t workspace_bytes, void *hip_stream, unsigned opts);

/* New tokens of n_seq (packed) or N sequences behind `cached` earlier ones each: token t of sequence s stands at position cached[s] + t
 * and sees the sequence's cached tokens and the new ones up to itself (and in its window).  The keys and values of the new tokens are
 * stored in the cache too; `cached` stays as it is, for the other layers of a step.
 *   k_cache, v_cache [n_pages, Hk, page, D] dt      in/out  page a power of two, 16 to 1024
 *   page_table  [sequences, max_pages] int32        in   device; rows ld_table apart: entry p holds the page of positions p page ..
 *   cached      [sequences] int32                   in   device; taken as at least 0 and at most max_pages page
 *   o           [N, T, H, D] dt, lse [N, T, H] fp32 or NULL    out
 *   max_len     a bound of cached + new tokens for how the work is cut (tiles of 32 or 128 query rows, parts of the keys): results beyond
 *               it are right, but slower, and so may be those of sequences far below it
 * Entries matter for positions below `cached` in some query's window, and for new tokens.  Others in the row's first max_pages may be read
 * too, and the pages that they name, without a part in any result.  An entry that is no page (below 0 or
 * from n_pages on) reads as the nearest page that is one, and nothing is stored through it; nor are new tokens at positions from
 * max_pages page on.  A page that new tokens go to must not be read or written through another entry in the same call.
 * max_pages page at most 2^30.  workspace 256-byte aligned. */
size_t kla_attn_extend_workspace_bytes(int N, int T, int H, int Hk, int D, const int32_t *cu_seqlens_host, int n_seq,
                                       int window, int max_len, kla_dtype dt);
int kla_attn_extend(const void *q, long ld_q, const void *k, long ld_k, const void *v, long ld_v,
                    void *k_cache, void *v_cache, const int32_t *page_table, long ld_table, const int32_t *cached,
                    void *o, float *lse, float scale, int window,
                    const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                    int N, int T, int H, int Hk, int D, int n_pages, int page, int max_pages, int max_len,
                    kla_dtype dt, void *workspace, size_t workspace_bytes, void *hip_stream);

/* One new token for B sequences: q, o [B, H, D], k, v [B, Hk, D]; workspace as for kla_attn_extend, N = B and T = 1. */
int kla_attn_step(const void *q, long ld_q, const void *k, long ld_k, const void *v, long ld_v,
                  void *k_cache, void *v_cache, const int32_t *page_table, long ld_table, const int32_t *cached,
                  void *o, float scale, int window, int B, int H, int Hk, int D, int n_pages, int page, int max_pages,
                  int max_len, kla_dtype dt, void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Test hook: the per-chunk objects the first stage of kla_chunk_fwd leaves in its workspace,
 * unpacked to plain row-major fp32 so that they can be compared one by one with eqs. (6)-(7).
 * Arguments as in kla_chunk_fwd.  For every chunk c (global chunk index, sequences in order)
 * and head h:
 *   Tb_out  [n_chunks, H, 64, 64]  (I + B(A^- o K K^T))^{-1} B, i.e. the solve of eq. (6) as a matrix
 *   P_out   [n_chunks, H, 64, 64]  A o Q K^T (lower triangle incl. diagonal) of eq. (7)
 *   g_out   [n_chunks, H, 64]      chunk-local running sum of log_alpha (log gamma_i)
 * Rows and columns beyond a short last chunk are zero (g repeats its last value).
 * The values are those the second stage of the two-kernel form consumes (rounded to dt for dt = bf16); workspace
 * from kla_chunk_fwd_workspace_bytes_opts(..., KLA_TUNE_UNFUSED) with dv = 64.
 */
int kla_debug_intra_chunk(const void *q, const void *k,
                          const float *log_alpha, const float *eta, float eps,
                          float *Tb_out, float *P_out, float *g_out,
                          const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                          int N, int T, int H, int dk, int chunk, kla_dtype dt,
                          void *workspace, size_t workspace_bytes, void *hip_stream);

/*
 * Profiling hook: one stage of the two-kernel form of kla_chunk_fwd alone (KLA_TUNE_UNFUSED; workspace from
 * kla_chunk_fwd_workspace_bytes_opts(..., KLA_TUNE_UNFUSED)), so that each kernel can be timed between two
 * events.  Arguments as in kla_chunk_fwd.  stage = 1: the intra-chunk stage (fills the workspace);
 * stage = 2: the scan stage (consumes a workspace that stage 1 filled for the same inputs, writes
 * o and hT).  Any other stage is KLA_ERR_SHAPE.
 */
int kla_debug_chunk_stage(const void *q, const void *k, const void *v,
                          const float *log_alpha, const float *eta, float eps,
                          const float *h0, void *o, float *hT,
                          const int32_t *cu_seqlens_dev, const int32_t *cu_seqlens_host, int n_seq,
                          int N, int T, int H, int dk, int dv, int chunk, kla_dtype dt,
                          void *workspace, size_t workspace_bytes, void *hip_stream, int stage);

/*
 * Measurement hook: what this GPU delivers for the access patterns the rooflines of the hot path are quoted
 * against (none of the method's arithmetic runs).  bench.py reports the results as second denominators beside the
 * published peaks.
 *   kind 0  in-place streaming, x <- 2 x over `bytes` of fp32 at buf (a multiple of 65536): every byte read once and
 *           written once, one workgroup per 64 KiB with all loads first, as in the decode step; iters != 0 selects
 *           non-temporal loads and stores.  aux unused.
 *   kind 1  read-only streaming of `bytes` at buf; aux receives bytes / 16384 floats.
 *   kind 2  dense bf16 matrix pipe: `bytes` workgroups of four waves, each wave `iters` rounds of eight
 *           independent 16x16x32 products (16384 flop each per wave); aux receives 256 floats per workgroup.
 *   kind 3  the copy wave of the chunk kernels alone: 256 workgroups, 64 steps; per step one wave brings n copies of
 *           1 KiB (256-byte rows 2 KiB apart; four workgroups of an XCD share the rows) from buf into LDS through a
 *           ring one or two steps deep, one barrier per step.  iters = n + 256 (depth - 1), n one of 16, 32, 48, 60;
 *           `bytes` = size of buf, at least n x 4 MiB (else KLA_ERR_WORKSPACE).  aux unused.
 */
int kla_debug_peak_probe(int kind, void *buf, void *aux, size_t bytes, int iters, void *hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* KLA_H */
