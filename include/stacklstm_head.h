/*
 * stacklstm_head.h -- C ABI of the operators between the states of a StackLSTM and its answers
 * (MI355X, gfx950; in the same library as stacklstm.h): layer norm, a linear layer with its
 * epilogue, the distillation loss of logits, and a beam search's step with the stacks' reordering.
 * h_top of stacklstm_fwd is a [T * B, H] matrix of rows for the first of them.
 *
 * Conventions for every entry point:
 *  - All array arguments are DEVICE pointers, owned by the caller; the library keeps none of them
 *    after the call returns and holds no state between calls, but for kernels' launch attributes,
 *    set once per device. Matrices are row-major. A matrix with an ld_ field in the dims may have
 *    that many elements from row to row (0: dense); the others are
 *    dense. Arrays need only their element's alignment; 16-byte aligned ones with strides of whole
 *    16 bytes get the fastest paths. A work space is 16-byte aligned.
 *  - Calls are asynchronous on `stream` (a hipStream_t; NULL = default stream) and never synchronise
 *    the host. They allocate nothing and may be captured into a graph.
 *  - Outputs are overwritten, not accumulated, and must not overlap inputs (exceptions are named).
 *  - SLSTM_F32 arrays hold float, SLSTM_BF16 arrays raw bfloat16; arrays declared float are 32-bit
 *    in both. Sums, softmax statistics, norms and products are held in 32 bits; a 16-bit output is
 *    rounded once (nearest even) unless a rounding is named.
 *  - Errors found by the argument checks (SLSTM_EINVAL, SLSTM_EWORKSPACE) launch nothing;
 *    SLSTM_EDEVICE reports a HIP runtime error. No exception crosses the ABI. Values in arrays
 *    are not checked on the host: an index out of range is left out, never followed.
 *  - Results are deterministic: equal calls give equal bits, whatever runs beside them.
 */
#ifndef STACKLSTM_HEAD_H
#define STACKLSTM_HEAD_H

#include "stacklstm.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { SLSTM_F32 = 0, SLSTM_BF16 = 1 } slstm_type;

/* ------------------------------------------------------------------ layer norm
 * s = x + res,  mean = mean(s),  rstd = 1 / sqrt(mean((s - mean)^2) + eps),
 * y = (s - mean) rstd gamma + beta, per row. */
typedef struct {
  int64_t rows;            /* 0 .. 2^31 - 1 */
  int32_t width;           /* 1 .. 8192 */
  int32_t type;            /* slstm_type of x, res, sum, y, dy, dsum, dx */
  float eps;               /* >= 0 */
  int64_t ld_x, ld_res, ld_dy;
} slstm_norm_dims;

/* Bytes of work space of stacklstm_norm_bwd (0 for invalid dims); the forward needs none. */
size_t stacklstm_norm_workspace_bytes(const slstm_norm_dims* d);

/*  x [rows, width]; res [rows, width] or NULL                      (read)
 *  gamma, beta [width] float, NULL = 1 and 0                       (read)
 *  sum [rows, width] or NULL: s, what a backward reads as its x    (written; only with res)
 *  y [rows, width]; mean, rstd [rows] float or NULL                (written)
 * y comes from s before s is rounded to `type`. */
int stacklstm_norm_fwd(const slstm_norm_dims* d, const void* x, const void* res, const float* gamma, const float* beta,
                       void* sum, void* y, float* mean, float* rstd, void* stream);

/*  x [rows, width]: s (the forward's sum, or its x without res); gamma, mean, rstd as there  (read)
 *  dy [rows, width]; dsum [rows, width] or NULL: gradient that reaches s past the norm       (read)
 *  dx [rows, width]: the gradient of s, hence of x and of res; dgamma, dbeta [width] float or NULL  (written)
 * workspace may be NULL where neither dgamma nor dbeta is asked for. */
int stacklstm_norm_bwd(const slstm_norm_dims* d, const void* x, const float* gamma, const float* mean, const float* rstd,
                       const void* dy, const void* dsum, void* dx, float* dgamma, float* dbeta, void* workspace,
                       size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ linear layer
 * z = x W + b,  y = act(z) + res.  Backward: dz = dy act'(z), dx = dz W^T, dW = x^T dz, db = sum dz. */
typedef enum {
  SLSTM_ACT_NONE = 0,
  SLSTM_ACT_RELU = 1,      /* derivative 0 at 0 */
  SLSTM_ACT_TANH = 2,
  SLSTM_ACT_SILU = 3,      /* z sigma(z) */
  SLSTM_ACT_GELU = 4       /* z/2 (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) */
} slstm_act;

/* Beside an slstm_act: with SLSTM_BF16 the backward's products take dz with 16 significant bits instead of 8, as two
 * bfloat16 matrices with a product each, summed in 32 bits before the one rounding. Twice the products' time. The forward,
 * SLSTM_F32 and SLSTM_ACT_NONE (dz is dy) have nothing to do with it. */
#define SLSTM_LINEAR_WIDE_DZ 0x100

typedef struct {
  int64_t M;               /* rows, 0 .. 2^30 */
  int32_t K, N;            /* inputs and outputs, 1 .. 2^24; y, x and W each of less than 2^31 - 2^19 tiles of 64 x 64 */
  int32_t type;            /* slstm_type of every array */
  int32_t act;             /* slstm_act, or that and SLSTM_LINEAR_WIDE_DZ */
  int64_t ld_x, ld_w, ld_res, ld_y, ld_dy;
} slstm_linear_dims;

/* Bytes of work space of stacklstm_linear_fwd / _bwd (0 for invalid dims). The two calls share
 * nothing in it. */
size_t stacklstm_linear_fwd_workspace_bytes(const slstm_linear_dims* d);
size_t stacklstm_linear_bwd_workspace_bytes(const slstm_linear_dims* d);

/*  x [M, K], W [K, N], b [N] or NULL, res [M, N] or NULL            (read)
 *  y [M, N]; z [M, N] or NULL: what a backward reads (act other than none)  (written)
 * Products are exact in 32 bits for SLSTM_BF16 operands and fp32 for SLSTM_F32 ones, sums fp32. y comes
 * from z before z is rounded to `type`. y may be res itself (same strides). */
int stacklstm_linear_fwd(const slstm_linear_dims* d, const void* x, const void* W, const void* b, const void* res, void* y,
                         void* z, void* workspace, size_t ws_bytes, void* stream);

/*  x, W as given to the forward; z as written by it (NULL with SLSTM_ACT_NONE)  (read)
 *  dy [M, N]                                                                 (read)
 *  dx [M, K], dW [K, N], db [N], each or NULL (dense)                        (written)
 * The gradient of res is dy. With SLSTM_BF16, dz is rounded to bfloat16 for the products of dx and dW (the
 * operands of the matrix units), unless SLSTM_LINEAR_WIDE_DZ is asked for; db sums it unrounded. */
int stacklstm_linear_bwd(const slstm_linear_dims* d, const void* x, const void* W, const void* z, const void* dy, void* dx,
                         void* dW, void* db, void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ distillation loss
 * Per row: p = softmax(value / tau) over the K entries that the teacher stored, q_tau = softmax(logits / tau),
 * q_1 = softmax(logits),
 *   loss = alpha tau^2 sum_j p_j (log p_j - log q_tau[index_j]) - (1 - alpha) log q_1[label]
 *   dloss/dlogits = alpha tau (q_tau sum_j p_j - sum_j p_j onehot(index_j)) + (1 - alpha) (q_1 - onehot(label))
 * An entry whose index is outside [0, V) is not there (p is over the others), a label outside [0, V) neither (its
 * term is 0). A row without entries and without a label has loss 0 and gradient 0, whatever its logits hold, and so is
 * the gradient of a row whose grad is 0. An entry with p = 0 adds nothing, also where its logit is -inf; entries that
 * are all -inf count as none. An index that occurs twice counts twice. */
typedef struct {
  int64_t rows;            /* 0 .. 2^31 - 1 */
  int32_t V;               /* 1 .. 2^22 */
  int32_t K;               /* entries of a row, 1 .. 256 */
  int32_t type;            /* slstm_type of logits and dlogits */
  float tau;               /* 1e-6 .. 1e6 */
  float alpha;             /* 0 .. 1 */
  int64_t ld_logits, ld_dlogits;
} slstm_distill_dims;

size_t stacklstm_distill_workspace_bytes(const slstm_distill_dims* d);

/*  logits [rows, V]; index [rows, K] int32, value [rows, K] float; label [rows] int32 or NULL   (read)
 *  loss [rows] float; stats [rows, 3] float or NULL: the largest logit m, log sum exp((logits - m) / tau)
 *  and log sum exp(logits - m), for a backward                                                  (written) */
int stacklstm_distill_fwd(const slstm_distill_dims* d, const void* logits, const int32_t* index, const float* value,
                          const int32_t* label, float* loss, float* stats, void* workspace, size_t ws_bytes, void* stream);

/* dlogits [rows, V] = grad[row] dloss/dlogits, grad [rows] float or NULL = 1; stats as written by the forward.
 * dlogits may be logits itself (same strides). */
int stacklstm_distill_bwd(const slstm_distill_dims* d, const void* logits, const int32_t* index, const float* value,
                          const int32_t* label, const float* stats, const float* grad, void* dlogits, void* stream);

/* Both in one pass over the logits, where grad is known beforehand (a mean over rows, a mask). dlogits may be logits
 * itself (same strides). */
int stacklstm_distill_step(const slstm_distill_dims* d, const void* logits, const int32_t* index, const float* value,
                           const int32_t* label, const float* grad, float* loss, void* dlogits, void* workspace,
                           size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ beam search
 * One step over B searches of K beams each: the continuation of beam k by token v has
 *   total = (logits[v] - lse) + score[k],   lse = log sum exp of the beam's (legal) logits,
 * in two fp32 additions; a finished beam (done) has the one continuation total = score[k], at the place of its token 0.
 * The K continuations with the largest totals are taken in falling order; ties go to the lower place k V + v. A total
 * of -inf or NaN is no continuation: a beam without legal tokens, with score -inf, or whose logits hold NaN or +inf
 * has none. */
typedef struct {
  int32_t B;               /* searches, >= 0; B K <= 2^31 - 1 */
  int32_t K;               /* beams, 1 .. 64 */
  int32_t V;               /* tokens or actions, 1 .. 2^22 */
  int32_t type;            /* slstm_type of logits */
  int32_t eos;             /* the token that finishes a beam, -1: none */
  int64_t ld_logits;
} slstm_beam_dims;

size_t stacklstm_beam_workspace_bytes(const slstm_beam_dims* d);

/*  logits [B K, V]; legal [B K, V] uint8 or NULL (0: not allowed)                        (read)
 *  score [B, K] float; done [B, K] uint8 or NULL (none is finished)                        (read)
 *  score_next [B, K] float; parent, token [B, K] int32; done_next [B, K] uint8             (written)
 * token is -1 for a finished beam that goes on. Where there are fewer than K continuations the places left have
 * score_next -inf, parent their own number, token -1, done_next 1. done_next: token == eos, or the parent was done. */
int stacklstm_beam_select(const slstm_beam_dims* d, const void* logits, const uint8_t* legal, const float* score,
                          const uint8_t* done, float* score_next, int32_t* parent, int32_t* token, uint8_t* done_next,
                          void* workspace, size_t ws_bytes, void* stream);

/* One array of per-beam state: [B K] rows of `slots` slots of slot_bytes bytes. */
typedef struct {
  const void* src;
  void* dst;               /* must not overlap any src, live or other dst of the call, nor parent (SLSTM_EINVAL) */
  int64_t slot_bytes;      /* >= 1; slots * slot_bytes <= 2^31 */
  int32_t slots;           /* >= 1; a stack of T + 1 states, or 1 */
  int32_t reserved;        /* 0 */
  const int32_t* live;     /* [B K] slots in use of each row of src, NULL: all; taken as 0 below 0, as slots above */
} slstm_beam_state;

#define SLSTM_BEAM_MAX_STATES 8

/* dst row (b, k) = src row (b, parent[b, k]), for up to SLSTM_BEAM_MAX_STATES arrays in one launch. Slots that are not
 * live in the parent's row are left as they were in dst, as is a row whose parent is outside [0, K). Uses B and K. */
int stacklstm_beam_reorder(const slstm_beam_dims* d, const int32_t* parent, const slstm_beam_state* states, int32_t count,
                           void* stream);

#ifdef __cplusplus
}
#endif
#endif /* STACKLSTM_HEAD_H */
