/*
 * oob_expert.h -- C ABI of the operators of a layer with experts, and of clipping at the end of a step, on one gfx950 GPU.
 *
 * A layer with experts sends every token through few of many feed-forward blocks.  Scores choose them
 * (oob_expert_route), the chosen pairs (token, choice) are put in order of their experts
 * (oob_expert_rows), every expert's rows go through its own matrix (oob_expert_linear), and a token's
 * results are summed by their weights (oob_expert_sum).  A GPU's share of such a layer is the same
 * operators with some of the experts, or some of their columns.  Run and timed, they give the profile of
 * a model with experts.  oob_clip_* take the norm over all gradients of a step, and scale them.
 *
 * Conventions, types and errors: as in oob_layer.h.  Strides of rows are at least a row's length; those of logits, x, dy, y (of a sum), residual and dout, which
 * are only read, may be 0: one row for all.  Arrays of numbers of experts, rows and places are
 * int32.  What such an array holds out of range is never used as an address: each call says what it does
 * instead.
 */
#ifndef OOB_EXPERT_H
#define OOB_EXPERT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define OOB_EXPERT_MAX 1024 /* experts */
#define OOB_EXPERT_MAX_CHOICES 64 /* of a token */

/* ---- routing: experts and weights of every token --------------------------------------------------
 * l = logits[t], s = softmax(l) (SOFTMAX) or 1 / (1 + e^-l) (SIGMOID).  An expert whose l is -inf is closed:
 * s = 0, and it comes after all others.  A token all of whose experts are closed has weights 0.
 * What is compared: c = s + bias (compared in 64 bits), and l itself where there is neither a bias nor a
 * group (the same order).  NaN comes after everything, closed experts included.
 * groups > 1: experts are `groups` runs of E / groups; a group counts what its `group_best` largest c add
 * up to (NaN where fewer are numbers), and the keep_groups best groups take part, of equals those that come first.
 * experts[t]: the k largest c in falling order, of equals the first.  weights[t]: scale s of these, and with
 * renormalize scale s / (sum of s of these), formed from their logits alone whatever the size of s, 0 where all are closed. */
enum { OOB_ROUTE_SOFTMAX = 0, OOB_ROUTE_SIGMOID = 1 };

typedef struct oob_route {
  int dtype;                      /* of the logits: OOB_BF16, OOB_FP16, OOB_FP32 */
  int score, renormalize;         /* OOB_ROUTE_*; 0 or 1 */
  int E, k;                       /* 1 <= E <= OOB_EXPERT_MAX, 1 <= k <= min(OOB_EXPERT_MAX_CHOICES, keep_groups E / groups) */
  int groups, keep_groups, group_best; /* groups divide E, at most 64; 1 <= keep_groups <= groups; group_best 1 or 2 */
  float scale;                    /* finite */
  int64_t T;                      /* below 2^31 */
  const void *logits;             /* [T][E], rows logits_stride apart */
  int64_t logits_stride;
  const float *bias;              /* [E] or NULL */
  int32_t *experts;               /* [T][k] out */
  float *weights;                 /* [T][k] out */
} oob_route;

int oob_expert_route(const oob_route *p, void *stream);

/* The logits' gradient from that of the weights; the choice itself and the bias have none.  Reads p's dtype, score, renormalize, E, k,
 * scale, T, logits and experts (those of the forward call; a choice out of 0 .. E-1 has no part, an expert that is named twice has two).  Closed experts
 * get 0. */
int oob_expert_route_backward(const oob_route *p, const float *dweights, void *dlogits, int64_t dlogits_stride, void *stream);

/* ---- the chosen pairs in order of their experts ----------------------------------------------------
 * experts [n]: pair i takes expert experts[i].  Those of first .. first + E - 1 take part (all of them held here, or a
 * GPU's share); others, -1 for a token that goes nowhere, say, are left out.
 *   offsets [E + 1]: rows offsets[e] .. offsets[e + 1] - 1 are those of expert first + e;
 *   rows [n]: the pair of each row, pairs of one expert in their own order; -1 behind the last row;
 *   place [n]: the row of each pair, -1 for those left out. */
size_t oob_expert_rows_workspace_size(int64_t n, int E); /* may be 0 */
int oob_expert_rows(const int32_t *experts, int64_t n, int first, int E, int32_t *offsets, int32_t *rows, int32_t *place,
                    void *workspace, size_t bytes, void *stream); /* 0 <= n < 2^31, 1 <= E <= OOB_EXPERT_MAX */

/* ---- every expert's rows through its own matrix ----------------------------------------------------
 * Row r of expert e, offsets[e] <= r < offsets[e + 1]:  z[r] = x[token(r)] w[e]^T + bias[e];  y[r] = act(z[r]).
 * token(r) = rows[r] / per where rows is given (x [T][K], R = T per), r itself otherwise (x [R][K]).  Rows of y and z that
 * are no expert's stay as they are.  Offsets out of 0 .. R are taken as the nearest of these, a run that ends before it begins as empty; a row
 * whose token is out of 0 .. T-1 is one of zeros.  y and z share no memory with what is read (offsets and rows too) or with one another (OOB_EINVAL).  Rows that offsets give to two experts are undefined (nothing outside the arrays is touched). */
typedef struct oob_expert_linear_t {
  int dtype, act;          /* OOB_BF16 or OOB_FP16; OOB_ACT_* */
  int E, per;              /* experts, at most OOB_EXPERT_MAX; pairs of a token (rows NULL: 1) */
  int64_t R, T, N, K;      /* rows, rows of x (R = T per, so R where rows is NULL), below 2^31; N and K from 1 to 2^21 - 1 */
  const int32_t *offsets, *rows; /* [E + 1], [R] or NULL */
  const void *x, *w, *bias; /* w [E][N][K], bias [E][N] or NULL, contiguous but for w's strides */
  void *y, *z;             /* [R][N]; z or NULL: what the backward pass needs where act is not NONE (y without act otherwise) */
  int64_t x_stride, w_stride, expert_stride, y_stride, z_stride; /* w: between rows and between experts */
} oob_expert_linear_t;

size_t oob_expert_linear_workspace_size(const oob_expert_linear_t *p);
int oob_expert_linear(const oob_expert_linear_t *p, void *workspace, size_t bytes, void *stream);

/* dz = dy act'(z);  dx[r] = dz[r] w[e] (a row of x's gradient each: oob_expert_sum without weights adds those of a token);
 * dw[e] = sum of dz[r]^T x[token(r)], db[e] = sum of dz[r] over the rows of e, 0 where it has none.  dx, dw, db: each may be NULL.
 * Reads p's sizes, offsets, rows, x (for dw), w (for dx) and z; dx, dw and db share no memory with what is read or with one another (OOB_EINVAL). */
typedef struct oob_expert_linear_grad {
  const void *dy;          /* [R][N] */
  void *dx, *dw, *db;      /* [R][K], [E][N][K] contiguous, [E][N] */
  int64_t dy_stride, dx_stride;
} oob_expert_linear_grad;

size_t oob_expert_linear_backward_workspace_size(const oob_expert_linear_t *p, const oob_expert_linear_grad *g);
int oob_expert_linear_backward(const oob_expert_linear_t *p, const oob_expert_linear_grad *g, void *workspace, size_t bytes, void *stream);

/* ---- a token's results summed ----------------------------------------------------------------------
 * out[t] = residual[t] + sum over j < k of weights[t][j] y[place[t][j]], in the order of j; a place out of 0 .. R-1 has no part.  out shares no
 * memory with what is read (OOB_EINVAL), but may be the residual in its place. */
typedef struct oob_expert_sum_t {
  int dtype, k;            /* OOB_BF16, OOB_FP16, OOB_FP32; 1 <= k <= OOB_EXPERT_MAX_CHOICES */
  int64_t T, R, C;         /* each below 2^31, C >= 1 */
  const void *y;           /* [R][C] */
  const int32_t *place;    /* [T][k] */
  const float *weights;    /* [T][k] or NULL: 1 */
  const void *residual;    /* [T][C] or NULL */
  void *out;               /* [T][C]; may be residual, with its stride */
  int64_t y_stride, residual_stride, out_stride;
} oob_expert_sum_t;

int oob_expert_sum(const oob_expert_sum_t *p, void *stream);

/* dy[place[t][j]] = weights[t][j] dout[t];  dweights[t][j] = dout[t] . y[place[t][j]], 0 where the place is out of 0 .. R-1.  Rows of
 * dy that are nobody's stay as they are; no two places may be the same.  dy, dweights: one may be NULL; neither shares
 * memory with what is read (y for dweights alone) or with the other (OOB_EINVAL).  The residual's gradient is dout. */
int oob_expert_sum_backward(const oob_expert_sum_t *p, const void *dout, int64_t dout_stride, void *dy, int64_t dy_stride, float *dweights,
                            void *stream);

/* ---- the norm over many tensors, and clipping ------------------------------------------------------
 * The arrays below lie on the HOST and are read before the call returns: n tensors of sizes[i] values of types[i] (OOB_*), at from[i].
 * norm [1] (float, out): the root of the sum of all squares, squares summed in 64 bits (an infinity where it
 * passes 32 bits). */
size_t oob_clip_workspace_size(int n, const int64_t *sizes);
int oob_clip_norm(int n, const void *const *from, const int64_t *sizes, const int *types, float *norm, void *workspace, size_t bytes,
                  void *stream);
/* 1 where a tensor of `to` shares memory with another of them, with one of `from` that it does not lie on, or with the value `given` (may be NULL), 0
 * otherwise (host arrays; nothing is enqueued). */
int oob_clip_overlap(int n, const void *const *from, const void *const *to, const int64_t *sizes, const int *types, const float *given);
/* to[i] = from[i] factor, factor = max_norm / norm where norm > max_norm and finite, 1 otherwise.  to[i] may be from[i]: with a factor of
 * 1 nothing is written then.  given (float [1], on the device) is the norm if it is not NULL, one that several GPUs have added up, say; otherwise it is
 * that of oob_clip_norm, which is written to `norm`.  Where oob_clip_overlap is 1, or `norm` lies on a
 * tensor: OOB_EINVAL. */
int oob_clip_scale(int n, const void *const *from, void *const *to, const int64_t *sizes, const int *types, float max_norm,
                   const float *given, float *norm, void *workspace, size_t bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif
