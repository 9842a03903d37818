/*
 * oob_layer.h -- C ABI of the operators of a transformer layer on one gfx950 GPU.
 *
 * The planner's input is a profile: the forward and backward time of every layer on d = 1..M GPUs
 * (F_{l,d}, B_{l,d} of Eq. 4).  These are the operators that such layers are made of, forward and
 * backward; a GPU's share of a layer on d GPUs is the same operators with 1/d of the columns or
 * heads.  Run and timed, they give the profile of a model on this GPU.
 *
 * Conventions: as in oob_plan.h -- plain C; array pointers are DEVICE pointers owned by the caller;
 * work is enqueued on `stream`; no call synchronises, copies to or from the host or allocates.
 * Argument errors are return codes (OOB_E* of oob_plan.h): OOB_EINVAL for arguments out of range,
 * OOB_ECAPACITY for a workspace that is too small.  A workspace starts at a multiple of 256 bytes,
 * holds nothing between calls, and may be used by the next call on the same stream.  Strides are in
 * elements.  Outputs must not overlap inputs or one another unless a call says so.  Every result is
 * the same in every run: sums are formed in a fixed order, no atomics.
 *
 * Types: OOB_BF16 and OOB_FP16 (all arrays of a call but those declared float), OOB_FP32 where a
 * call says so.  Sums, statistics and what lies between two products of one kernel are 32 bits;
 * results are rounded to the type once.
 */
#ifndef OOB_LAYER_H
#define OOB_LAYER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { OOB_BF16 = 0, OOB_FP16 = 1, OOB_FP32 = 2 };

/* ---- matrix product with bias, activation and residual --------------------------------------
 * z = x w^T + bias;  y = act(z) + residual.
 *   x [T][K], w [N][K], bias [N] or NULL, residual [T][N] or NULL (may be y itself, with its stride),
 *   y [T][N] out, z [T][N] out or NULL: what the backward pass needs where act is not NONE
 * Rows of below 2^24 values are accepted whatever their number.  Longer ones of x, w, and for the gradients dy: as long as the first 64
 * of them (fewer, where there are fewer), each rounded up to 8 values, lie within 2^31 bytes; otherwise OOB_EINVAL.
 * RELU max(z, 0); GELU z Phi(z), by the error function; GELU_TANH its form with tanh(sqrt(2 / pi) (z +
 * 0.044715 z^3)); SILU z / (1 + e^-z).  A NaN gives NaN, in value and slope. */
enum { OOB_ACT_NONE = 0, OOB_ACT_RELU = 1, OOB_ACT_GELU = 2, OOB_ACT_GELU_TANH = 3, OOB_ACT_SILU = 4, OOB_ACTS = 5 };

typedef struct oob_linear {
  int dtype, act;          /* OOB_BF16 or OOB_FP16; OOB_ACT_* */
  int64_t T, N, K;         /* T >= 0, N, K >= 1, each below 2^31 (see below for long rows) */
  const void *x, *w, *bias, *residual;
  void *y, *z;
  int64_t x_stride, w_stride, residual_stride, y_stride, z_stride;
} oob_linear;

size_t oob_layer_linear_workspace_size(const oob_linear *p); /* goes by sizes, strides and alignment; may be 0 */
int oob_layer_linear(const oob_linear *p, void *workspace, size_t bytes, void *stream);

/* dz = dy act'(z);  dx = dz w;  dw = dz^T x;  db = sum of dz over tokens.  dx, dw, db: each may be
 * NULL.  z is read where act is not NONE.  The residual's gradient is dy. */
typedef struct oob_linear_grad {
  int dtype, act;
  int64_t T, N, K;
  const void *dy, *x, *w, *z;
  void *dx, *dw, *db;
  int64_t dy_stride, x_stride, w_stride, z_stride, dx_stride, dw_stride;
} oob_linear_grad;

size_t oob_layer_linear_backward_workspace_size(const oob_linear_grad *p);
int oob_layer_linear_backward(const oob_linear_grad *p, void *workspace, size_t bytes, void *stream);

/* ---- norms before and after a block, its gate, residual scale and dropout ---------------------
 * A residual stream x [T][C] and a block's output z [T][C]:
 *   u = keep / (1 - p) * post(z) * post_weight + post_bias;  xp = alpha x + gate u;
 *   h = pre(xp) * weight + bias
 * with post NONE (u = keep / (1 - p) z), LAYER or RMS and pre LAYER or RMS: LAYER(v) = (v - mean) /
 * sqrt(variance + eps), RMS(v) = v / sqrt(mean of squares + eps).  weight, bias, post_weight, post_bias
 * [C]: each may be NULL (1, 0).  (keep multiplies post_bias too.)  gate [gates][C], T a
 * multiple of gates, above 0: gate g is that of rows g T / gates .. (g + 1) T / gates - 1; gates = 0: none.  keep: as in
 * oob_layer_dropout, element t C + c.  z NULL: xp is x itself and not written (post NONE, no gate, p 0,
 * alpha 1).  h is formed from xp before its rounding.
 * Types: OOB_BF16, OOB_FP16, OOB_FP32.  xp may be x (with stride C). */
enum { OOB_NORM_NONE = 0, OOB_NORM_LAYER = 1, OOB_NORM_RMS = 2 };
#define OOB_NORM_MAX_C 16384

typedef struct oob_norm {
  int dtype, pre, post;
  float eps, alpha, p;      /* eps >= 0; 0 <= p, rounded to a multiple of 2^-16 below 1 */
  int64_t T, C, gates;      /* T >= 0, 1 <= C <= OOB_NORM_MAX_C */
  uint64_t seed, offset;    /* of the dropout */
  const void *x, *z, *weight, *bias, *post_weight, *post_bias, *gate;
  int64_t x_stride, z_stride;
  void *xp, *h;             /* [T][C] out */
  float *saved;             /* [4][T] out ([2][T] where post is NONE): mean and 1 / deviation of pre, of post; or NULL.  The
                             * backward pass reads the means of LAYER norms */
} oob_norm;

int oob_layer_norm(const oob_norm *p, void *stream);

/* From the gradients of xp (dxp, NULL: zero) and h: those of x, z, and of the weights that are not
 * NULL.  Of p: x is xp (the forward call's result, x_stride its stride), saved and everything else as
 * in the forward call, xp and h are not used. */
typedef struct oob_norm_grad {
  const void *dxp, *dh;
  int64_t dxp_stride, dh_stride;
  void *dx, *dz;                                        /* [T][C] out; dz where there is a z */
  void *dweight, *dbias, *dpost_weight, *dpost_bias;    /* [C] out, each may be NULL */
  void *dgate;                                          /* [gates][C] out where there are gates */
} oob_norm_grad;

size_t oob_layer_norm_backward_workspace_size(const oob_norm *p);
int oob_layer_norm_backward(const oob_norm *p, const oob_norm_grad *g, void *workspace, size_t bytes, void *stream);

/* ---- attention ---------------------------------------------------------------------------------
 * B sequences of Sq queries and Sk keys, H heads of D values for queries and G for keys and values (head h
 * uses h / (H / G)).  Query i sees the keys j with begin_i <= j < end_i, key_begin (or 0) and key_end (or
 * Sk) [B][Sq]; causal: only those with j <= i + Sk - Sq as well.  Document, prefix and window masks are
 * such ranges.
 *   s_ij = scale q_i . k_j;  cap > 0: s_ij = cap tanh(s_ij / cap);  slopes [H] (or NULL): s_ij -= slope_h
 *   |i + Sk - Sq - j|;  o_i = sum_j softmax_j(s_ij) v_j;  lse_i = log sum_j e^s_ij
 * A query that sees no key has o = 0, lse = -inf and no part in any gradient, whatever it holds.  Keys that none of the
 * queries 128 t .. 128 t + 127 sees have no part in theirs, whatever they hold; others have to be finite, also for the
 * queries among those that do not see them.  The backward pass rounds p_ij (dout_i . v_j - dout_i . o_i) to the type: with
 * OOB_FP16 it has to stay below 65504.
 * q, o [B][Sq][H][D], k, v [B][Sk][G][D]: strides of a sequence, a row and a head, the last axis
 * contiguous; 0 for an axis of inputs that repeats, not of results (OOB_EINVAL).  k, v, and for the gradients q and dout, are copied where they do not start at 16 bytes, a stride is no multiple of
 * that or D none of 8, or rows lie 2^24 bytes apart; the heads of 32 rows (fewer, where there are fewer) then have to take less than 2^31 bytes. */
#define OOB_ATTENTION_MAX_D 128

typedef struct oob_attention {
  int dtype;                    /* OOB_BF16 or OOB_FP16 */
  int B, Sq, Sk, H, G, D;       /* B, Sq, Sk >= 0, Sq, Sk below 2^29; H a multiple of G >= 1; 1 <= D <= 128; B H (max(Sq, Sk) / 16 + 1) below 2^31 */
  int causal;
  float scale, cap;             /* scale > 0; cap 0: none */
  const void *q, *k, *v;
  const int32_t *key_begin, *key_end;
  const float *slopes;
  void *o;
  float *lse;                   /* [B][H][Sq] out, or NULL; read by the backward pass */
  int64_t q_stride[3], k_stride[3], v_stride[3], o_stride[3];
} oob_attention;

size_t oob_layer_attention_workspace_size(const oob_attention *p);
int oob_layer_attention(const oob_attention *p, void *workspace, size_t bytes, void *stream);

/* dq, dk, dv from dout, the gradient of o.  Of p: everything as in the forward call, o and lse its results. */
typedef struct oob_attention_grad {
  const void *dout;
  void *dq, *dk, *dv;
  int64_t dout_stride[3], dq_stride[3], dk_stride[3], dv_stride[3];
} oob_attention_grad;

size_t oob_layer_attention_backward_workspace_size(const oob_attention *p, const oob_attention_grad *g);
int oob_layer_attention_backward(const oob_attention *p, const oob_attention_grad *g, void *workspace, size_t bytes,
                                 void *stream);

/* ---- dropout -----------------------------------------------------------------------------------
 * y[i] = keep_i x[i] / (1 - p), n elements; y may be x.  keep_i: bits 16 (m % 4) .. + 15 of word m / 4,
 * m = offset + i, are not below round(65536 p), and 1 - p is that of the rounded p.  Word k is output
 * k of a SplitMix64 generator whose state starts at output function(seed).  The mask is never stored:
 * the backward pass is the same call on dy. */
int oob_layer_dropout(int dtype, const void *x, void *y, int64_t n, float p, uint64_t seed, uint64_t offset,
                      void *stream);

#ifdef __cplusplus
}
#endif
#endif
