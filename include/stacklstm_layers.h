/*
 * stacklstm_layers.h -- C ABI of the layers around the states of a StackLSTM (MI355X, gfx950; in the same library as
 * stacklstm.h): attention to an encoder's states, log probabilities of tokens with entropy and best tokens, and dropout.
 *
 * The conventions are those of stacklstm_head.h: device pointers owned by the caller; calls are asynchronous on `stream`,
 * never synchronise the host, allocate nothing and may be captured into a graph; outputs are overwritten and must not overlap
 * inputs (exceptions are named); argument errors (SLSTM_EINVAL, SLSTM_EWORKSPACE) launch nothing; sums, softmax statistics and
 * products are held in 32 bits, a 16-bit output is rounded once unless a rounding is named; arrays need only their element's
 * alignment, a work space 16 bytes; results are deterministic. A work space holds nothing between calls, and two calls that
 * may run at once (on two streams, or two graphs) need one each. Calls run on the current device, which is to be the stream's.
 */
#ifndef STACKLSTM_LAYERS_H
#define STACKLSTM_LAYERS_H

#include "stacklstm_head.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ attention
 * Query t of sequence b and head h attends to the keys of head h / (Hq / Hk):
 *   x_j = scale q . k_j,  p = softmax of x over the keys that are there,  y = sum_j p_j v_j.
 * Backward, from dy:  dv_j = sum p_j dy,  s_j = p_j (dy . v_j - dy . y),  dq = scale sum_j s_j k_j,  dk_j = scale sum s_j q,
 * the sums of dk and dv over all queries and over the Hq / Hk heads that share the key.
 * A key is there if its place is below k_len[b] and its mask byte is not 0; what absent keys and values hold (NaN too) has no
 * effect, and their dk and dv are 0. A query at or past q_len[b], or one without keys, has y = 0 and dq = 0 and adds
 * nothing to dk and dv, whatever it holds. A key whose x is -inf has p = 0; a query all of whose x are -inf has y = 0 and dq = 0. */
typedef struct {
  int64_t b, t, h;         /* elements from one sequence, place and head to the next; the D elements of a head are neighbours */
} slstm_strides;

typedef struct {
  int32_t B;               /* sequences, >= 0 */
  int32_t Tq, Tk;          /* queries and keys of a sequence, 0 .. 2^24 */
  int32_t Hq, Hk;          /* heads of queries and of keys and values, 1 .. 2^16; Hq a multiple of Hk */
  int32_t D;               /* width of a head, 1 .. 256 */
  int32_t type;            /* slstm_type of every matrix */
  float scale;             /* -2^127 .. 2^127 */
  slstm_strides q, k, v, dy;        /* of inputs: >= 0, all three 0: dense [B, T, H, D]; a stride may be 0 (broadcast) */
  slstm_strides y, dq, dk, dv;      /* of outputs: all three 0: dense; no two elements at one place (SLSTM_EINVAL) */
} slstm_attend_dims;       /* B Tq Hq and B Tk Hk < 2^31; strides < 2^40 */

/* Floats of `stats` for a query and head (0 for invalid dims). */
int32_t stacklstm_attend_stats_width(const slstm_attend_dims* d);
/* Bytes of work space (0 for invalid dims). */
size_t stacklstm_attend_fwd_workspace_bytes(const slstm_attend_dims* d);
size_t stacklstm_attend_bwd_workspace_bytes(const slstm_attend_dims* d);

/*  q [B, Tq, Hq, D], k and v [B, Tk, Hk, D] (may be NULL with Tk = 0)                            (read)
 *  q_len, k_len [B] int32 or NULL: all (taken as 0 below 0, as Tq / Tk above)                      (read)
 *  mask [B, Tk] uint8 or NULL (0: not there)                                                      (read)
 *  y [B, Tq, Hq, D]; stats [B, Hq, Tq, stacklstm_attend_stats_width] float or NULL: the softmax's
 *  reference and sum, and what y's rounding to 16 bits takes off, for a backward                   (written)
 * With SLSTM_BF16 the p of a product with v are rounded to bfloat16, the operands of the matrix units. */
int stacklstm_attend_fwd(const slstm_attend_dims* d, const void* q, const void* k, const void* v, const int32_t* q_len,
                         const int32_t* k_len, const uint8_t* mask, void* y, float* stats, void* workspace, size_t ws_bytes,
                         void* stream);

/*  q, k, v, q_len, k_len, mask as given to the forward; y and stats as written by it; dy [B, Tq, Hq, D]   (read)
 *  dq [B, Tq, Hq, D]; dk, dv [B, Tk, Hk, D]                                                             (written)
 * With SLSTM_BF16, p and s are rounded to bfloat16 for the products. No output may be an input here. */
int stacklstm_attend_bwd(const slstm_attend_dims* d, const void* q, const void* k, const void* v, const int32_t* q_len,
                         const int32_t* k_len, const uint8_t* mask, const void* y, const float* stats, const void* dy, void* dq,
                         void* dk, void* dv, void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ log probabilities
 * Per row, with q = softmax of the logits over the tokens that are allowed:
 *   logp_g = log q[token_g],  entropy = -sum q log q,  and the N best tokens: those of the largest logits, falling, ties to
 *   the lower token, with their log q.
 *   dlogits = sum_g dlogp_g (onehot(token_g) - q) - dentropy q (log q + entropy)
 * A token outside [0, V) is not there: its logp is 0 and it has no gradient. One that is not allowed has logp -inf and no
 * gradient. Tokens given twice count twice. A logit of -inf has q = 0. Logits of -inf and NaN are never among the best; where
 * there are fewer than N the places left have index -1 and value -inf: what stacklstm_distill_* takes for entries that are not
 * there. A row without allowed tokens has entropy 0. A row with NaN or +inf has NaN logp and entropy. Where the dlogp of
 * all of a row's allowed tokens and its dentropy are 0, so is its gradient, whatever it holds. */
typedef struct {
  int64_t rows;            /* 0 .. 2^31 - 1 */
  int32_t V;               /* 1 .. 2^22 */
  int32_t G;               /* given tokens of a row, 0 .. 64 */
  int32_t N;               /* best tokens of a row, 0 .. 64 */
  int32_t type;            /* slstm_type of logits and dlogits */
  int64_t ld_logits, ld_dlogits;
} slstm_logprob_dims;

size_t stacklstm_logprob_workspace_bytes(const slstm_logprob_dims* d);

/*  logits [rows, V]; legal [rows, V] uint8 or NULL (0: not allowed); token [rows, G] int32 (NULL with G = 0)   (read)
 *  logp [rows, G] float (NULL with G = 0); entropy [rows] float or NULL; index [rows, N] int32, value [rows, N] float (NULL with
 *  N = 0); stats [rows, 3] float or NULL: the largest logit m, log sum exp(logits - m), and the entropy, for a backward  (written) */
int stacklstm_logprob_fwd(const slstm_logprob_dims* d, const void* logits, const uint8_t* legal, const int32_t* token,
                          float* logp, float* entropy, int32_t* index, float* value, float* stats, void* workspace,
                          size_t ws_bytes, void* stream);

/* dlogits [rows, V] from dlogp [rows, G] float (NULL: 0) and dentropy [rows] float (NULL: 0); stats as written by the forward.
 * dlogits may be logits itself (same strides). N is not looked at. */
int stacklstm_logprob_bwd(const slstm_logprob_dims* d, const void* logits, const uint8_t* legal, const int32_t* token,
                          const float* stats, const float* dlogp, const float* dentropy, void* dlogits, void* stream);

/* Both in one pass over the logits, where dlogp and dentropy are known beforehand (rewards, a mean over rows). dlogits may be
 * logits itself (same strides). */
int stacklstm_logprob_step(const slstm_logprob_dims* d, const void* logits, const uint8_t* legal, const int32_t* token,
                           const float* dlogp, const float* dentropy, float* logp, float* entropy, int32_t* index, float* value,
                           void* dlogits, void* workspace, size_t ws_bytes, void* stream);

/* ------------------------------------------------------------------ dropout
 *   y = keep x s + res,  dx = keep dy s,  s = 1 / (1 - p'),  p' = floor(65536 p + 1/2) / 65536,
 * keep is 1 with probability 1 - p'. What is dropped is 0 whatever x holds; with p' = 1 everything is. The mask is never stored:
 * element c of row r takes 16 bits of Philox4x32-10 (Salmon et al., 2011) with the key seed[0] (low word first) and the counter
 * words (c / 8, r, low and high word of seed[1]); elements 0 .. 7 of a group take the low half of output word 0, its high
 * half, the low half of word 1, and so on; an element is kept if its 16 bits are not below 65536 p'. */
typedef struct {
  int64_t rows;            /* 0 .. 2^31 - 1 */
  int32_t width;           /* 1 .. 2^24 */
  int32_t type;            /* slstm_type of every matrix */
  float p;                 /* 0 .. 1 */
  int64_t period;          /* 0, or: row r has the mask of row r % period (rows of one sequence in many steps: one mask for all) */
  int64_t ld_x, ld_res, ld_y;       /* ld_x: of x and of dy; ld_y: of y and of dx */
} slstm_dropout_dims;

/*  x [rows, width]; res [rows, width] or NULL; seed [2] int64: the generator's key and a step     (read)
 *  y [rows, width]                                                                               (written)
 * seed lies on the device, so that a captured graph takes another mask whenever it has been changed between replays. y may be x
 * or res itself (same strides). */
int stacklstm_dropout_fwd(const slstm_dropout_dims* d, const void* x, const void* res, const int64_t* seed, void* y,
                          void* stream);
/* dx [rows, width] from dy, with the forward's dims and seed; the gradient of res is dy. dx may be dy itself (same strides). */
int stacklstm_dropout_bwd(const slstm_dropout_dims* d, const void* dy, const int64_t* seed, void* dx, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* STACKLSTM_LAYERS_H */
