/*
 * favor.h - C ABI of libfavor, FAVOR attention (Fast Attention Via Orthogonal
 * Random features, arXiv 2006.03555) for AMD MI355X (gfx950).
 *
 * Every tensor argument is a DEVICE pointer owned by the caller; the library
 * never allocates, frees or retains device memory (scratch is the caller's
 * workspace; the one exception is the static scratch array each GPU holds for
 * favor_attn_both_noalloc). Every call is asynchronous: work is enqueued on `stream`
 * (NULL = the default stream) and nothing waits.
 *
 * Errors: arguments are validated completely before anything is launched. On
 * failure a call returns a non-zero favor_status, writes no output and records
 * a message retrievable with favor_last_error() (per thread). A failed launch
 * returns FAVOR_ERR_DEVICE. Numerical outcomes are not errors: a denominator
 * D-hat that is zero gives IEEE Inf/NaN rows exactly as the formulas do.
 *
 * Layouts (row-major, contiguous, 16-byte aligned):
 *   Q, K, V, out   [B][H][L][d]      in_dtype (out: out_dtype)
 *   W              [H][M][d]  float  rows omega_m of the random-feature matrix
 *   b              [H][M]     float  phases b_m
 *   X' (features)  [B][H][L][M]      out_dtype
 *   state          [B][H][M][d+1] float, column d holds sum_j K'_j (the "1" column)
 * One draw (W, b) per head is shared by every batch entry.
 *
 * Supported: d = 64; M a multiple of 16 from 16 to 256 (the kernels work on M
 * rounded up to 64, 128 or 256 rows, the rows past M being padding whose
 * features are zero, so every array above keeps M; the causal scan with F32
 * inputs and M > 128 runs as two passes over the feature halves);
 * 0 <= L <= 2^30 (any length, ragged tails handled; L = 0 is a no-op); B, H >= 0,
 * B*H <= 65535; in_dtype F32 or BF16; out_dtype F32 or BF16. F32 inputs use
 * fp32 matrix cores and a cosine of at most 1.4e-7 absolute error (rms 2.0e-8);
 * BF16 inputs use bf16 matrix cores with fp32 accumulation, the hardware cosine
 * and bf16 features.
 */
#ifndef FAVOR_H
#define FAVOR_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define FAVOR_API __attribute__((visibility("default")))
#else
#define FAVOR_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

/* The HIP runtime's stream handle (the same declaration as in
 * hip/hip_runtime_api.h, so either header may come first). NULL is the default
 * stream. */
struct ihipStream_t;
typedef struct ihipStream_t *hipStream_t;

typedef enum {
  FAVOR_OK = 0,
  FAVOR_ERR_INVALID_ARGUMENT = 1,  /* null/misaligned pointer, negative size, bad enum */
  FAVOR_ERR_UNSUPPORTED = 2,       /* valid but not implemented (d, M, dtype combo)    */
  FAVOR_ERR_WORKSPACE_TOO_SMALL = 3,
  FAVOR_ERR_DEVICE = 4             /* a HIP launch or runtime call failed               */
} favor_status;

typedef enum { FAVOR_F32 = 0, FAVOR_BF16 = 1 } favor_dtype;

typedef enum {
  FAVOR_RF_ORTHO_CHI = 0,   /* R-ORF blocks, rows scaled by independent chi_d norms (default) */
  FAVOR_RF_ORTHO_FIXED = 1, /* R-ORF blocks, every row scaled to norm sqrt(d)                  */
  FAVOR_RF_IID = 2,         /* unstructured i.i.d. N(0, I_d) rows                              */
  FAVOR_RF_HADAMARD = 3,    /* H-ORF blocks sqrt(d) H D3 H D2 H D1 (Sec. 2.4 (2))              */
  FAVOR_RF_GIVENS = 4       /* G-ORF blocks sqrt(d) G_1 ... G_K, K = 2 d log2 d (Sec. 2.4 (2)) */
} favor_rf_kind;

/* Feature kernel (Sec. 2.2, Eq. interesting):
 *   SOFTMAX  Gaussian-kernel features for softmax attention (Sec. 2.3):
 *            phi(x)_m = exp(||x~||^2 / 2) sqrt(2/M) cos(omega_m . x~ + b_m)
 *   RELU     generalized attention with f = ReLU, g = h = 1 (the paper's
 *            "Performer-ReLU", App. B): phi(x)_m = ReLU(omega_m . x~) / sqrt(M)
 *            + kernel_eps; the phases b are not used. */
typedef enum { FAVOR_KERNEL_SOFTMAX = 0, FAVOR_KERNEL_RELU = 1 } favor_kernel;

typedef struct {
  int32_t B, H, L, d, M;
  favor_dtype in_dtype;     /* Q, K, V (and X for the feature map) */
  favor_dtype out_dtype;    /* out, X'                             */
  float input_scale;        /* x~ = input_scale * x. d^-1/4 evaluates the paper's
                               exp(Q K^T / sqrt d) (Sec. 2.1) on the given Q, K.  */
  float denom_eps;          /* added to D-hat before dividing; 0 = Algorithm 1      */
  int32_t chunk;            /* causal chunk length T: tokens per step of the
                               prefix-sum scan (Sec. 2.5.1): 64 (four 16-token
                               matrix-core blocks in the intra-chunk product) or,
                               for bf16 inputs, 32; 0 = the library's choice (of
                               the scan's form as well as its step; fp32: 64).
                               Other values,
                               and 32 with fp32 inputs in a causal call, return
                               FAVOR_ERR_UNSUPPORTED. The result is the same sum
                               in another grouping                                 */
  int32_t kernel;           /* favor_kernel; 0 (zero-initialised) = SOFTMAX         */
  int32_t no_renormalize;   /* 0 = out = Buf3 / (buf4 + denom_eps) (Algorithm 1);
                               1 = out = Buf3 = Q' K'^T V ("renormalize_attention"
                               off, App. B; denom_eps is then unused)             */
  float kernel_eps;         /* RELU: added to every feature (App. B kernel_epsilon,
                               default 1e-3); ignored for SOFTMAX                  */
  int32_t segment;          /* causal: tokens per segment, the stretch of the
                               sequence one workgroup scans chunk by chunk from
                               the aggregate of the segments before it (a multiple
                               of 64, at most 2^30); 0 = library default (about one
                               workgroup per compute unit, two with T = 32 or,
                               chunk = 0, with bf16 inputs and M <= 128)           */
} favor_desc;

/*
 * favor_orf_draw - draw the random-feature matrix W [n_heads][M][d] and phases
 * b [n_heads][M] (Sec. 2.3 for the Gaussian-kernel features, Sec. 2.4 for the
 * orthogonal R-ORF construction).
 *
 * For each head h and block k < ceil(M/d): a d x d matrix of N(0,1) entries has
 * its rows orthonormalised in order by Gram-Schmidt (the orthogonal factor
 * with positive triangular diagonal); row m = k d + r is scaled by rho_m (kind
 * CHI: the norm of an independent N(0, I_d) vector; FIXED: sqrt(d)); the first
 * M stacked rows are kept. IID kind keeps the raw Gaussian rows. b_m = 2 pi u_m.
 * HADAMARD: block k = sqrt(d) H D3 H D2 H D1 with the normalised Sylvester-
 * Hadamard matrix H[i][j] = (-1)^popcount(i & j) / sqrt(d) and diagonals D_t of
 * signs: element (3 k + t) d + c of purpose 3 is +1 when its 32-bit word is
 * below 2^31, else -1. GIVENS: block k = sqrt(d) G_1 ... G_K, K = 2 d log2 d;
 * G_t rotates the (i, j) plane by theta (row vectors: v_i <- cos v_i + sin v_j,
 * v_j <- -sin v_i + cos v_j), from words x0, x1, x2 of call k K + t of purpose 4:
 * i = (x0 d) >> 32, j' = (x1 (d - 1)) >> 32, j = j' + [j' >= i],
 * theta = 2 pi (x2 + 0.5) 2^-32. Both are orthogonal with rows of norm sqrt(d).
 *
 * Random numbers: Philox4x64-10 (Salmon et al., SC'11), key (seed, 0), counter
 * (i, h, purpose, 0) with purpose 0 = Gaussian blocks, 1 = chi-norm Gaussians,
 * 2 = phases, 3 = Hadamard signs, 4 = Givens rotations. Call i yields four 64-bit words w0..w3, i.e. eight 32-bit words
 * x[2j] = low(wj), x[2j+1] = high(wj); stream element n is word n % 8 of call
 * n / 8; u = (x + 0.5) 2^-32; Gaussians by Box-Muller from uniform pairs
 * (u[2p], u[2p+1]): sqrt(-2 ln u[2p]) * (cos, sin)(2 pi u[2p+1]). Gaussian
 * element of block k, row r, column c: n = (k d + r) d + c; chi vector of row
 * m: n = m d + c; phase of row m: n = m. Uniforms, Gaussians and phases are
 * computed in fp32; the orthogonalisation, norms and scaling in fp64.
 *
 * Requires n_heads >= 0, d = 64, 1 <= M <= 4096. W, b: device, fp32; W 16-byte
 * aligned, b 4-byte aligned.
 */
FAVOR_API favor_status favor_orf_draw(uint64_t seed, int32_t n_heads, int32_t M, int32_t d,
                            favor_rf_kind kind, float *W, float *b, hipStream_t stream);

/*
 * favor_feature_map - X' = D_X X-hat, the paper's Q' = D_Q Q-hat (Sec. 2.3,
 * Eqs. dqdk and qkprime) with Gaussian-kernel features (c = sqrt 2, f = cos):
 *   X'[l][m] = exp(||x~_l||^2 / 2) * sqrt(2/M) * cos(omega_m . x~_l + b_m),
 *   x~_l = input_scale * X[l];
 * with g->kernel = FAVOR_KERNEL_RELU the generalized-attention features
 *   X'[l][m] = max(omega_m . x~_l, 0) / sqrt(M) + g->kernel_eps   (b unused).
 * X [B][H][L][d] in g->in_dtype -> Xprime [B][H][L][M] in g->out_dtype.
 * g->denom_eps, g->chunk and g->no_renormalize are ignored.
 */
FAVOR_API favor_status favor_feature_map(const favor_desc *g, const void *X, const float *W,
                               const float *b, void *Xprime, hipStream_t stream);

/*
 * favor_workspace_size - bytes of device workspace favor_attn_bidir (causal = 0),
 * favor_attn_causal (causal = 1, or any value other than 0 and 2) or
 * favor_attn_both (causal = 2) needs for descriptor g; 0 if g is invalid.
 * The workspace must be 256-byte aligned; its contents on entry do not matter.
 */
FAVOR_API size_t favor_workspace_size(const favor_desc *g, int causal);

/*
 * favor_attn_bidir - bidirectional FAVOR (Sec. 2.5, Algorithm 1):
 *   C = [V 1_L], Buf1 = K'^T C (M x (d+1)), Buf2 = Q' Buf1,
 *   out = diag(buf4 + denom_eps)^-1 Buf3 with [Buf3 buf4] = Buf2,
 * where Q', K' are the feature maps of favor_feature_map for g->kernel. With
 * g->no_renormalize = 1 the result is Buf3 itself. The L x L matrix Q' K'^T and
 * the L x M features are never stored. Deterministic (no atomics).
 */
FAVOR_API favor_status favor_attn_bidir(const favor_desc *g, const void *Q, const void *K,
                              const void *V, const float *W, const float *b, void *out,
                              void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_bidir_save - favor_attn_bidir that also writes, for the backward
 * pass, row_scale [B][H][L] fp32 (nullable): each row's 1 / (buf4 + denom_eps)
 * in units of the features without D_Q sqrt(2/M). Needs out_dtype == in_dtype;
 * row_scale is not written without renormalisation.
 */
FAVOR_API favor_status favor_attn_bidir_save(const favor_desc *g, const void *Q, const void *K,
                                             const void *V, const float *W, const float *b,
                                             void *out, float *row_scale, void *ws,
                                             size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_causal - unidirectional FAVOR by prefix sums (Sec. 2.5.1, Eq.
 * cumsum): row i of the result is (G^PS_i)^T Q'_i normalised as in Algorithm 1
 * (not normalised with g->no_renormalize = 1; features as for favor_attn_bidir),
 * G^PS_i = S_0 + sum_{j <= i} K'_j C_j^T (keys up to and including i). The
 * prefix tensor is never stored: workgroups scan chunks of tokens carrying an
 * M x (d+1) fp32 state.
 * state_in  (nullable) [B][H][M][d+1] fp32: S_0, the aggregate of earlier tokens.
 * state_out (nullable) [B][H][M][d+1] fp32: receives S_0 + sum over all L tokens,
 * so a long sequence can be processed in pieces. Deterministic (no atomics).
 */
FAVOR_API favor_status favor_attn_causal(const favor_desc *g, const void *Q, const void *K,
                               const void *V, const float *W, const float *b, void *out,
                               const float *state_in, float *state_out,
                               void *ws, size_t ws_bytes, hipStream_t stream);

/* favor_attn_causal_save - favor_attn_causal that also writes row_scale, as
 * favor_attn_bidir_save does. */
FAVOR_API favor_status favor_attn_causal_save(const favor_desc *g, const void *Q,
                                              const void *K, const void *V, const float *W,
                                              const float *b, void *out, const float *state_in,
                                              float *state_out, float *row_scale, void *ws,
                                              size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_both - both directions over the same Q, K, V in one call: the
 * results of favor_attn_bidir (out_bidir) and favor_attn_causal (out_causal,
 * with state_in / state_out as there; state_in affects the causal output only).
 * The bidirectional Buf1 = K'^T [V 1] is the causal aggregate over the whole
 * sequence (G^PS_L of Eq. cumsum), so one pass over the keys serves both:
 * the key features are built once per segment and the segment scan also
 * returns the total. Workspace: favor_workspace_size(g, 2). Deterministic.
 * row_scale_bidir, row_scale_causal (nullable): as for favor_attn_bidir_save.
 */
FAVOR_API favor_status favor_attn_both(const favor_desc *g, const void *Q, const void *K,
                                       const void *V, const float *W, const float *b,
                                       void *out_bidir, void *out_causal,
                                       const float *state_in, float *state_out,
                                       float *row_scale_bidir, float *row_scale_causal,
                                       void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_both_noalloc - favor_attn_both for callers that cannot allocate
 * device memory (code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc): the same arguments without ws / ws_bytes, and the same
 * results. The workspace is a static array of favor_noalloc_scratch_bytes()
 * bytes (32 MiB) that each GPU the library runs on holds from the first load of
 * the library's code there until the process ends; nothing is allocated or
 * freed by the call. A call whose favor_workspace_size(g, 2) exceeds it returns
 * FAVOR_ERR_WORKSPACE_TOO_SMALL and launches nothing. Every call on one GPU uses
 * that GPU's one array: calls that overlap on one GPU (concurrent streams,
 * threads) race on it and must be serialised by the caller. The array needs no
 * clearing (the kernels overwrite what they read). The current device is the
 * one whose array is used (the stream must belong to it).
 */
FAVOR_API favor_status favor_attn_both_noalloc(const favor_desc *g, const void *Q,
                                               const void *K, const void *V, const float *W,
                                               const float *b, void *out_bidir,
                                               void *out_causal, const float *state_in,
                                               float *state_out, float *row_scale_bidir,
                                               float *row_scale_causal, hipStream_t stream);

/* Size in bytes of favor_attn_both_noalloc's static scratch array. */
FAVOR_API size_t favor_noalloc_scratch_bytes(void);

/*
 * Backward pass (the paper trains through FAVOR and benchmarks its backward
 * pass, Sec. 4.1): gradients of a loss with respect to Q, K, V given
 * dout = dLoss/dout, for the same descriptor, inputs and features as the
 * forward call. Algorithm 1 and Eq. cumsum are taken in reverse:
 *   [dBuf3 dbuf4] from the normalisation (dBuf3 = dout / (buf4 + eps), dbuf4 =
 *   -(dout . out) / (buf4 + eps); dout and 0 without renormalisation),
 *   dQ' = dBuf2 Buf1^T, dBuf1 = Q'^T dBuf2, dK' = C dBuf1^T, dV = (K' dBuf1)[:, :d],
 * then through the feature maps. The forward quantities are recomputed (nothing
 * from the forward call is needed); W and b receive no gradient.
 * dout, dQ, dK, dV: [B][H][L][d] in in_dtype; out_dtype must equal in_dtype
 * (FAVOR_ERR_UNSUPPORTED otherwise). Every supported M; with fp32 inputs the
 * gradient kernels take 128 (bidirectional) or 64 (causal) features at a time
 * and add the slices' parts into dQ, dK, dV in a fixed order. Deterministic
 * (no atomics). dQ, dK, dV are written in full (ragged tails included).
 * Workspace: favor_backward_workspace_size(g, causal) bytes, 256-byte aligned
 * (causal: 0 bidirectional, 1 causal, 2 both directions in one call).
 * out and row_scale (both nullable, both or neither): the forward call's output
 * and row_scale for the same inputs, features and descriptor; given, the backward
 * skips recomputing them (their recomputation otherwise runs inside the call).
 * Not read without renormalisation.
 * fwd_ws, fwd_op: the workspace a forward call left behind and which call that
 * was (1 favor_attn_bidir or favor_attn_bidir_save, 2 favor_attn_causal or
 * favor_attn_causal_save, 3 favor_attn_both), or NULL and 0. The forward call must have had the same
 * descriptor, K, V, W, b (and, causal, the same state_in), completed in stream
 * order before, and its workspace must be unchanged since. Given, the backward
 * reads Buf1 (bidirectional: 1 or 3) or the segment prefixes (causal: 2 or 3),
 * the W'' fragments and b'' from it instead of recomputing them; fwd_ws is only
 * read. Other fwd_op values, or fwd_ws without fwd_op, are
 * FAVOR_ERR_INVALID_ARGUMENT.
 */
FAVOR_API size_t favor_backward_workspace_size(const favor_desc *g, int causal);

/* favor_attn_bidir_backward - gradients of favor_attn_bidir. */
FAVOR_API favor_status favor_attn_bidir_backward(const favor_desc *g, const void *Q,
                                                 const void *K, const void *V, const float *W,
                                                 const float *b, const void *dout,
                                                 const void *out, const float *row_scale,
                                                 const void *fwd_ws, int32_t fwd_op,
                                                 void *dQ, void *dK, void *dV, void *ws,
                                                 size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_causal_backward - gradients of favor_attn_causal (Eq. cumsum):
 * dQ'_i = G^PS_i dBuf2_i with the prefix aggregate, and with the suffix
 * R_j = dstate_out + sum_{i >= j} Q'_i dBuf2_i^T: dK'_j = R_j C_j,
 * dV_j = (R_j^T K'_j)[:d]. state_in (nullable) as in the forward call;
 * dstate_out (nullable) [B][H][M][d+1] fp32: the gradient reaching state_out;
 * dstate_in (nullable) [B][H][M][d+1] fp32: receives the gradient of state_in
 * (R_1), so a sequence processed in pieces is differentiated piece by piece
 * from the last. L = 0 copies dstate_out (or zeros) to dstate_in.
 */
FAVOR_API favor_status favor_attn_causal_backward(const favor_desc *g, const void *Q,
                                                  const void *K, const void *V, const float *W,
                                                  const float *b, const float *state_in,
                                                  const void *dout, const void *out,
                                                  const float *row_scale, const void *fwd_ws,
                                                  int32_t fwd_op, const float *dstate_out,
                                                  void *dQ, void *dK,
                                                  void *dV, float *dstate_in, void *ws,
                                                  size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_both_backward - gradients of favor_attn_both: of a loss that depends
 * on both outputs, given dout_bidir and dout_causal (Algorithm 1 and Eq. cumsum
 * in reverse, as the two calls above). dQ, dK, dV receive the sums of the two
 * directions' gradients. The key side is one pass: the bidirectional dBuf1 is
 * the aggregate every key of the sequence sees, so it is added to each key's
 * causal suffix R_j before dK'_j = R_j C_j and dV_j = (R_j^T K'_j)[:d]; dQ of the
 * causal direction is added onto the bidirectional one (bf16: one more
 * rounding). out_bidir with row_scale_bidir, and out_causal with
 * row_scale_causal: each pair nullable, both or neither, as the forward call
 * saved them. fwd_ws, fwd_op: a favor_attn_both call's workspace and 3, or NULL
 * and 0. state_in, dstate_out, dstate_in as for favor_attn_causal_backward
 * (dstate_in receives the causal direction's state gradient only; the
 * bidirectional output does not depend on state_in). Workspace:
 * favor_backward_workspace_size(g, 2) bytes, 256-byte aligned. Other
 * conditions and errors as for the two calls above.
 */
FAVOR_API favor_status favor_attn_both_backward(const favor_desc *g, const void *Q,
                                                const void *K, const void *V, const float *W,
                                                const float *b, const float *state_in,
                                                const void *dout_bidir, const void *dout_causal,
                                                const void *out_bidir,
                                                const float *row_scale_bidir,
                                                const void *out_causal,
                                                const float *row_scale_causal,
                                                const void *fwd_ws, int32_t fwd_op,
                                                const float *dstate_out, void *dQ, void *dK,
                                                void *dV, float *dstate_in, void *ws,
                                                size_t ws_bytes, hipStream_t stream);

/*
 * Linear attention with a decay per head (no random features: Q and K enter as they
 * are, for instance as favor_feature_map wrote them):
 *   S_t = a_h S_{t-1} + k_t v_t^T,   out_t = scale q_t^T S_t,   a_h = exp(log_decay[h]),
 * that is out_i = scale (sum_{j <= i} a^(i-j) (q_i . k_j) v_j + a^(i+1) q_i^T S_in).
 * log_decay [H] fp32: 0 keeps everything, -Inf only the token itself. A positive value
 * grows as the formula says up to 1.38 (while a^64, and scale a^64, are in fp32's range; in
 * sequences of fewer tokens, a^L); beyond it results may be Inf or NaN where the formula
 * is finite.
 *
 * Layouts: Q, K [B][H][L][dk], V, out [B][H][L][dv] with rows of contiguous elements and
 * any strides between them, in elements (favor_strides; all three 0 = the contiguous
 * layout above): [B][L][H][d] tensors, slices of one QKV projection and broadcast inputs
 * (a stride of 0) need no copy. Strides and base addresses are multiples of 16 bytes, and
 * tokens at most 2^25 bytes apart (FAVOR_ERR_UNSUPPORTED);
 * rows of an output must not share elements (FAVOR_ERR_INVALID_ARGUMENT), and outputs
 * must not overlap inputs. state [B][H][dk][dv] fp32, contiguous.
 *
 * Supported: dk and dv multiples of 8 up to 256; dtype (inputs, out, gradients) F32 or
 * BF16; 0 <= L <= 2^30; B*H <= 65535. F32 uses fp32 matrix cores, BF16 bf16 ones with
 * fp32 sums; states are fp32 throughout, and one that a call returns is as exact for BF16
 * inputs as for F32 ones. In BF16 pair weights and states enter the products of a row to
 * 16 bits, so that the row's own rounding is what it is off by, whatever its batch. (The
 * products in a state that the call does not return are taken to 16 bits too: the last bits
 * of such a call's outputs may differ from those of one that returns it.)
 *
 * lengths [B] int32 (nullable, device): sequence b has its first lengths[b] tokens
 * (values outside 0 .. L are taken as 0 or L), and rows behind them are padding: their
 * inputs are not read, their rows of out and of the gradients are written as zeros. A
 * NaN or infinity in a token reaches the results of its own chunk of 64 tokens and of
 * those behind it (dK, dV and dS_in: before it); in BF16 an infinity in a value or a state
 * may arrive there as NaN.
 */
typedef struct {
  int64_t batch, head, token;
} favor_strides;

typedef struct {
  int32_t B, H, L, dk, dv;
  favor_dtype dtype;        /* Q, K, V, out and the gradients */
  float scale;
  favor_strides q, k, v, out;
  favor_strides grad_out, grad_q, grad_k, grad_v;   /* read by the backward pass only */
} favor_decay_desc;

/* Bytes of device workspace for favor_attn_decay (backward = 0) or
 * favor_attn_decay_backward (1), 256-byte aligned; 0 if none is needed (then ws may be
 * NULL) or g is invalid. Its contents on entry do not matter. */
FAVOR_API size_t favor_decay_workspace_size(const favor_decay_desc *g, int backward);

/*
 * favor_attn_decay - the chunked form, for prompts and training. state_in (nullable): S
 * before the first token; state_out (nullable; may be state_in, and must not overlap it
 * otherwise): S after each sequence's last one, so a sequence can be processed in pieces.
 * Deterministic (no atomics).
 */
FAVOR_API favor_status favor_attn_decay(const favor_decay_desc *g, const void *Q,
                                        const void *K, const void *V, const float *log_decay,
                                        const int32_t *lengths, void *out,
                                        const float *state_in, float *state_out, void *ws,
                                        size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_decay_backward - gradients of a loss that depends on out and state_out, from
 * dout and dstate_out (nullable: zeros); state_in and lengths as in the forward call:
 *   dq_i = scale (sum_{j <= i} a^(i-j) (dout_i . v_j) k_j + a^(i+1) S_in dout_i)
 *   dk_j = scale sum_{i >= j} a^(i-j) (dout_i . v_j) q_i + a^(n-1-j) dS_out v_j
 *   dv_j = scale sum_{i >= j} a^(i-j) (q_i . k_j) dout_i + a^(n-1-j) dS_out^T k_j
 *   dS_in = a^n dS_out + scale sum_i a^(i+1) q_i dout_i^T
 * dstate_in (nullable; may be dstate_out; overlaps neither it nor state_in otherwise)
 * receives the gradient of state_in. Nothing from the forward call is needed. log_decay receives no gradient. For a broadcast input every
 * head (or batch entry) gets its own gradient, to be summed by the caller. Deterministic.
 */
FAVOR_API favor_status favor_attn_decay_backward(
    const favor_decay_desc *g, const void *Q, const void *K, const void *V,
    const float *log_decay, const int32_t *lengths, const float *state_in, const void *dout,
    const float *dstate_out, void *dQ, void *dK, void *dV, float *dstate_in, void *ws,
    size_t ws_bytes, hipStream_t stream);

/*
 * favor_attn_decay_step - the recurrent form, for single tokens: Q, K [B][H][dk], V, out
 * [B][H][dv], and the states state [n_slots][H][dk][dv] updated in place. g->L has no effect
 * (it must be in its range). Nor have token strides, except that a tensor whose three strides
 * are 0 is contiguous: one row for every sequence and head has batch = head = 0 and a token
 * stride that is not 0. slots [B] int32 (nullable, device): the place of
 * each sequence's state, NULL: state b is sequence b's (n_slots >= B). A sequence with a
 * place outside 0 .. n_slots - 1 (padding of a captured batch) has no state and out = 0.
 * Sequences that name the same place take their turns in order, as tokens of one sequence.
 */
FAVOR_API favor_status favor_attn_decay_step(const favor_decay_desc *g, const void *Q,
                                             const void *K, const void *V,
                                             const float *log_decay, const int32_t *slots,
                                             int32_t n_slots, float *state, void *out,
                                             hipStream_t stream);

/* Host-only validation of a descriptor for an operation (0 favor_attn_decay, 1 its
 * backward pass, 2 favor_attn_decay_step). */
FAVOR_API favor_status favor_validate_decay_desc(const favor_decay_desc *g, int op);

/*
 * favor_dropout - y_n = residual_n + [bits_n >= t] x_n / (1 - t / 2^16) with t = p 2^16
 * rounded to the nearest (ties to even): p is taken to 16 bits, and p >= 1 - 2^-17 drops
 * everything. residual nullable (0); y may be x or residual, and overlaps
 * neither otherwise. x, residual, y: n elements
 * of dtype, contiguous, 16-byte aligned. A dropped element is 0 whatever x holds.
 *
 * bits_n is 16-bit piece n % 8 of Philox4x32-10 (Salmon et al., SC'11) with key (seed low,
 * seed high) and counter (c low, c high, offset low, offset high), c = n / 8: pieces 2 j
 * and 2 j + 1 are the low and high half of word j. Calls with other (seed, offset) have
 * independent masks. The mask is not stored: the gradient is the same call on dy with
 * the same p, seed, offset and no residual. rng (nullable, device, 8-byte aligned): two
 * words {seed, offset} read by the kernel in place of the arguments, so that a captured
 * graph draws a new mask whenever the program changes them.
 */
FAVOR_API favor_status favor_dropout(const void *x, const void *residual, void *y, int64_t n,
                                     favor_dtype dtype, double p, uint64_t seed,
                                     uint64_t offset, const uint64_t *rng, hipStream_t stream);

/*
 * Short causal convolution, one filter per channel (the step in front of a selective scan):
 *   u_t = bias + sum_{j < width} w[j] x_{t - width + 1 + j},   y_t = u_t, or u_t sigmoid(u_t)
 * with the inputs before the first token from a state (zeros without one).
 *
 * Layouts: x, y [B][L][D] with rows of D contiguous elements and any strides between them, in
 * elements (favor_strides, head unused; all three 0 = contiguous), multiples of 16 bytes, so
 * that halves of one projection and transposed batches need no copy; outputs' rows must not
 * share elements, and outputs must not overlap inputs. weight [D][width] and bias [D]
 * (nullable) fp32. States [B][width - 1][D] in dtype, contiguous: the last width - 1 inputs,
 * the oldest first.
 *
 * Supported: width 2 to 8; D a multiple of 8 up to 65536; dtype (x, y, states and their
 * gradients) F32 or BF16, sums in fp32; 0 <= L <= 2^30, B <= 65535, L D <= 2^38, B L D <= 2^46.
 * lengths [B] int32 (nullable, device): as for favor_attn_decay: rows behind a sequence are not read
 * and their rows of y and dx are written as zeros.
 */
typedef struct {
  int32_t B, L, D, width;
  favor_dtype dtype;
  int32_t silu;                      /* 0: y = u */
  favor_strides x, y;
  favor_strides grad_y, grad_x;      /* read by the backward pass only */
} favor_conv_desc;

/* state_in (nullable), state_out (nullable; may be state_in, and overlaps it not otherwise). */
FAVOR_API favor_status favor_conv(const favor_conv_desc *g, const void *x, const float *weight,
                                  const float *bias, const int32_t *lengths, void *y,
                                  const void *state_in, void *state_out, hipStream_t stream);

/*
 * Gradients from dy and dstate_out (nullable: zeros) of x, weight [D][width], bias (dbias
 * nullable) and state_in (dstate_in nullable; overlaps neither state nor dstate_out). With no
 * sequence (B = 0) or no token the parameters' gradients are zeros.
 * Nothing from the forward call is needed. Deterministic. Workspace:
 * favor_conv_workspace_size(g) bytes, 256-byte aligned; its contents do not matter.
 */
FAVOR_API favor_status favor_conv_backward(const favor_conv_desc *g, const void *x,
                                           const float *weight, const float *bias,
                                           const int32_t *lengths, const void *state_in,
                                           const void *dy, const void *dstate_out, void *dx,
                                           float *dweight, float *dbias, void *dstate_in,
                                           void *ws, size_t ws_bytes, hipStream_t stream);
FAVOR_API size_t favor_conv_workspace_size(const favor_conv_desc *g);

/*
 * One token of B sequences: x, y [B][D] (batch strides; L has no effect within its range) and
 * the states [n_slots][width - 1][D], updated in place. slots as for favor_attn_decay_step: a
 * place outside 0 .. n_slots - 1 is padding and gives y = 0, sequences that name the same place
 * take their turns in order.
 */
FAVOR_API favor_status favor_conv_step(const favor_conv_desc *g, const void *x,
                                       const float *weight, const float *bias,
                                       const int32_t *slots, int32_t n_slots, void *state,
                                       void *y, hipStream_t stream);

/*
 * Selective state space scan, per channel d (in group g = d / (D / groups)) and state n:
 *   s_t = softplus(dt_t + dt_bias_d)   (softplus = 0: dt_t + dt_bias_d)
 *   h_t[n] = exp(s_t A[d][n]) h_{t-1}[n] + s_t x_t B_t[g][n]
 *   y_t = (sum_n C_t[g][n] h_t[n] + skip_d x_t) silu(z_t)
 * without the terms of a NULL dt_bias, skip or z.
 *
 * Layouts: x, dt, z, y [B][L][D] as for favor_conv; B, C [B][L][groups][N] with N contiguous
 * elements and any strides in elements (head: the group's), not aligned; tokens of all of them
 * at most 2^25 bytes apart. A [D][N], skip and dt_bias [D] fp32. States [B][D][N] fp32, contiguous.
 *
 * Supported: N from 1 to 256; D up to 65536 with D / groups a multiple of 8; dtype (x, dt, B,
 * C, z, y and their gradients) F32 or BF16; 0 <= L <= 2^30, B <= 65535, L D <= 2^38, B L D and
 * B L groups N <= 2^46. Steps, states and sums are fp32 for both, and what is below 2^-126 as an
 * exponential is 0. A is meant to be negative; for a positive one exp(A times the steps of any 128
 * tokens) has to be in fp32's range, and A must be finite. lengths as for favor_conv
 * (B's and C's padding is not read either, its gradients are zeros). A NaN or infinity reaches
 * the results of its own channel (in B or C: of its group) from its token on, and gradients as the
 * formulas carry it; in the backward pass it may reach all of its chunk of 128 tokens.
 */
typedef struct {
  int32_t B, L, D, N, groups;
  favor_dtype dtype;
  int32_t softplus;
  favor_strides x, dt, b, c, z, y;
  favor_strides grad_y, grad_x, grad_dt, grad_b, grad_c, grad_z;   /* backward pass only */
} favor_scan_desc;

/*
 * Bytes of device workspace for favor_selective_scan (backward = 0) or its backward pass (1),
 * 256-byte aligned; 0 if none is needed or g is invalid. Its contents do not matter. Backward, in
 * floats: 3 B chunks D N for states and dA (chunks of 128 tokens), and 2 B L groups N for dB and dC
 * for each workgroup of a group's channels: up to 128 channels of a large call with N <= 16, 32 of
 * others. So that part grows fourfold from N = 16 to 17, and B4 L4096 D4096 N64 takes 1.5 GB.
 */
FAVOR_API size_t favor_scan_workspace_size(const favor_scan_desc *g, int backward);

/* state_in (nullable), state_out (nullable; may be state_in, and overlaps it not otherwise):
 * the state before the first and after each sequence's last token. Deterministic. */
FAVOR_API favor_status favor_selective_scan(const favor_scan_desc *g, const void *x,
                                            const void *dt, const float *A, const void *Bm,
                                            const void *C, const float *skip, const void *z,
                                            const float *dt_bias, const int32_t *lengths,
                                            void *y, const float *state_in, float *state_out,
                                            void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * Gradients from dy and dstate_out (nullable: zeros): with e_t = dy_t silu(z_t), and
 * q_t = exp(s_t A) (C_t e_t + q_{t+1}) from the right (q behind the last token: dstate_out),
 *   dC = sum_d e h,  dB = sum_d (C e + q_{t+1}) s x,  dA = sum s_t q_t h_{t-1},  dstate_in = q_0
 *   ds = sum_n A q_t h_{t-1} + x sum_n (C e + q_{t+1}) B,  ddt = ds softplus'(dt + dt_bias)
 *   dx = s sum_n (C e + q_{t+1}) B + skip e,  dz = dy (C h + skip x) silu'(z),  dskip = sum e x
 * and ddt_bias = sum ddt. dskip, dz and ddt_bias are required where skip, z and dt_bias are
 * given, and not written otherwise. With no sequence (B = 0) or no token the parameters' gradients
 * are zeros. dstate_in (nullable) may be dstate_out, and overlaps
 * neither it nor state_in otherwise. Nothing from the forward call is needed. Deterministic.
 */
FAVOR_API favor_status favor_selective_scan_backward(
    const favor_scan_desc *g, const void *x, const void *dt, const float *A, const void *Bm,
    const void *C, const float *skip, const void *z, const float *dt_bias,
    const int32_t *lengths, const float *state_in, const void *dy, const float *dstate_out,
    void *dx, void *ddt, float *dA, void *dB, void *dC, float *dskip, void *dz,
    float *ddt_bias, float *dstate_in, void *ws, size_t ws_bytes, hipStream_t stream);

/* One token of B sequences: x, dt, z, y [B][D], Bm, C [B][groups][N] (token strides and L, within
 * its range, have no effect), the states [n_slots][D][N] updated in place; slots as for
 * favor_conv_step. */
FAVOR_API favor_status favor_selective_scan_step(const favor_scan_desc *g, const void *x,
                                                 const void *dt, const float *A, const void *Bm,
                                                 const void *C, const float *skip, const void *z,
                                                 const float *dt_bias, const int32_t *slots,
                                                 int32_t n_slots, float *state, void *y,
                                                 hipStream_t stream);

/* Host-only validation of a descriptor (op: 0 forward, 1 backward, 2 single tokens). */
FAVOR_API favor_status favor_validate_conv_desc(const favor_conv_desc *g, int op);
FAVOR_API favor_status favor_validate_scan_desc(const favor_scan_desc *g, int op);

/*
 * Beam search's choice of the next tokens: for each of B entries the n best of the K V
 * continuations by
 *   score(k, v) = scores[k] + x[k][v] - log sum_u exp x[k][u]
 * in falling order: out_scores [B][n] fp32, parent [B][n] (the beam k) and token [B][n] int32.
 * Ties go to the lower beam, then in one beam to the higher logit and the lower token. Sums of
 * exponentials are fp32 per lane and joined in 64 bits; scores are compared in 64 bits. In one
 * call equal rows have equal scores; how a row is cut depends on V and on B K, so with another
 * number of rows its score may be rounded otherwise. Logits of any size are taken.
 *
 * logits [B][K][V] of dtype, V contiguous, strides in elements (both 0 = contiguous), not
 * aligned: any V and slices of a padded vocabulary. scores [B][K] fp32. ended [B][K] bytes
 * (nullable): a beam that has ended (not 0) offers only itself, with end_token and its own
 * score, and its logits are not read. end_token < 0: there is none (then ended must be NULL).
 * Only scores that are finite in fp32 are offered: a beam of score -Inf, a token of logit -Inf and
 * a beam with a NaN or +Inf among its logits (whose sum is no number) offer nothing. Where fewer
 * than n are offered the rest has score -Inf, parent 0 and token end_token (0 without one).
 *
 * Supported: K and n up to 64, V from 1 to 2^30, B K <= 65535. Workspace:
 * favor_beam_workspace_size(g) bytes, 256-byte aligned; its contents do not matter.
 */
typedef struct {
  int32_t B, K, V, n;
  favor_dtype dtype;
  int64_t batch_stride, beam_stride;
  int32_t end_token;
} favor_beam_desc;

FAVOR_API favor_status favor_validate_beam_desc(const favor_beam_desc *g);   /* host only */
FAVOR_API size_t favor_beam_workspace_size(const favor_beam_desc *g);
FAVOR_API favor_status favor_beam_select(const favor_beam_desc *g, const void *logits,
                                         const float *scores, const uint8_t *ended,
                                         float *out_scores, int32_t *parent, int32_t *token,
                                         void *ws, size_t ws_bytes, hipStream_t stream);

/*
 * The states of pools (of favor_attn_decay_step, favor_conv_step, favor_selective_scan_step)
 * behind the chosen beams: beam j of entry b continues beam parent[b][j], whose state is at
 * place slots[b][parent[b][j]] of every pool (slots NULL: b K + the beam). A beam's first
 * child takes its place as it is; its other children, in order, take the places of the
 * entry's beams without children, in order, and the states are copied there, in place. So only
 * the states of dead beams are written, and new_slots [B][K] holds the same places as slots in
 * another order. A beam whose parent is outside 0 .. K - 1 takes a free place and its state
 * stays what it was there. Nothing is copied from or to places outside 0 .. n_slots - 1.
 * The places inside the pools that one call names must differ. new_slots must not overlap
 * slots or parent.
 *
 * pools: n_pools host descriptions, read during the call: data (16-byte aligned),
 * bytes_per_slot (a multiple of 16, up to 2^34) and n_slots; they must not overlap. K <= 64,
 * B K <= 65535. Up to 64 pools are one launch.
 */
typedef struct {
  void *data;
  int64_t bytes_per_slot;
  int32_t n_slots;
} favor_beam_pool;

FAVOR_API favor_status favor_beam_reorder(int32_t B, int32_t K, const int32_t *parent,
                                          const int32_t *slots, int32_t *new_slots,
                                          const favor_beam_pool *pools, int32_t n_pools,
                                          hipStream_t stream);

/* Host-only validation of a descriptor for an operation (0 feature map,
 * 1 bidirectional, 2 causal, 3 both, 4 bidirectional backward, 5 causal
 * backward, 6 backward of both directions); launches nothing and touches no
 * device. */
FAVOR_API favor_status favor_validate_desc(const favor_desc *g, int op);

FAVOR_API const char *favor_status_string(favor_status s);

/* Detail of the last failure on the calling thread ("" if none). */
FAVOR_API const char *favor_last_error(void);

/*
 * Per-kernel timing for benchmarks. While enabled, every kernel the library
 * launches is bracketed by two HIP events recorded on the launch stream (the
 * events come from a pool; nothing is allocated on the device). Reading
 * waits for the recorded events and returns, for kernel id k, the summed
 * milliseconds and launch count since the last reset. Ids run from 0 to
 * favor_timing_num_kernels() - 1; favor_timing_kernel_name(k) names them.
 * Not thread-safe with respect to concurrent launches from several threads.
 */
FAVOR_API favor_status favor_timing_enable(int on);
FAVOR_API favor_status favor_timing_reset(void);
FAVOR_API int32_t favor_timing_num_kernels(void);
FAVOR_API const char *favor_timing_kernel_name(int32_t k);
FAVOR_API favor_status favor_timing_read(int32_t k, double *ms, int64_t *count);

/*
 * Measurement probes for roofline reports (not part of the method): one launch
 * of 512 workgroups of 256 threads (two per CU) in which every wave issues
 * iters x 8 independent v_mfma_f32_16x16x32_bf16 (kind 0), every lane
 * evaluates iters x 8 independent hardware cosines (kind 1), or every lane
 * projects iters tokens onto M = 256 H-ORF rows the structured way, four blocks
 * of three 64-point Walsh-Hadamard transforms with sign flips in registers
 * (kind 2; the O(M log d) apply of Sec. 2.4, against which the dense matrix-core
 * projection of kind 0 is compared). Timing a launch and dividing
 * favor_probe_work(kind, iters) (FLOP for kind 0, cosines for kind 1, tokens
 * for kind 2) by its duration gives the rate this GPU reaches. sink: a device
 * buffer of at least 512 floats (never written for the probe's inputs).
 */
FAVOR_API favor_status favor_probe(int32_t kind, int32_t iters, float *sink, hipStream_t stream);
FAVOR_API double favor_probe_work(int32_t kind, int32_t iters);

/* ABI version of this header; bumped on any incompatible change. */
FAVOR_API int32_t favor_abi_version(void);

#define FAVOR_ABI_VERSION 7

#ifdef __cplusplus
}
#endif

#endif /* FAVOR_H */
