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
 *   y [T][N] out, z [T][N] out or NULL: what the backward pass needs where act is not NONE */
enum { OOB_ACT_NONE = 0, OOB_ACT_RELU = 1, OOB_ACT_GELU = 2, OOB_ACT_GELU_TANH = 3, OOB_ACT_SILU = 4, OOB_ACTS = 5 };

typedef struct oob_linear {
  int dtype, act;          /* OOB_BF16 or OOB_FP16; OOB_ACT_* */
  int64_t T, N, K;         /* T >= 0, N, K >= 1, each below 2^31 */
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

#ifdef __cplusplus
}
#endif
#endif
