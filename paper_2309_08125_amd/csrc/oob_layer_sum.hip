/* The weighted sum of what a token's experts gave, and its gradients. */
#include "oob_expert.h"
#include "oob_layer_device.h"

namespace layer {
namespace {

/* A token takes `width` threads of a workgroup (a power of two), eight columns each at a time, eight choices' rows on their way together.  Memory bounds it: 4096
 * tokens, 8 choices, 4096 columns, bfloat16: 83 us (335 MB, 4.0 TB/s, behind the writes of what ran before), the gradients 107 us (570 MB, 5.3 TB/s). */
struct Sum {
  oob_expert_sum_t p;
  int width;
  const void *dout;
  void *dy;
  int64_t ld_dout, ld_dy;
  float *dweights;
};
constexpr int TOGETHER = 8; /* rows of y that are on their way at once */

/* WAVE: a wave has one token (rows of more than 256 values), and what goes by the token and its choices lies in scalar registers: the gradients take 69 vector
 * registers, seven waves a SIMD, and 107 us; 147, three and 122 otherwise. */
template <bool WAVE> __device__ inline int64_t token_of(const Sum &g) {
  int in = threadIdx.x / g.width;
  return (int64_t)blockIdx.x * (256 / g.width) + (WAVE ? uniform(in) : in);
}
/* Places and weights of choices from number j0 on; a place below 0 has no part.  All are asked for before the first is waited for. */
template <bool WAVE> __device__ __forceinline__ void places_of(const oob_expert_sum_t &p, int64_t t, int j0, int (&r)[TOGETHER], float (&w)[TOGETHER]) {
#pragma unroll
  for (int j = 0; j < TOGETHER; j++) r[j] = j0 + j < p.k ? p.place[t * p.k + j0 + j] : -1;
#pragma unroll
  for (int j = 0; j < TOGETHER; j++) w[j] = j0 + j >= p.k ? 0.f : p.weights ? p.weights[t * p.k + j0 + j] : 1.f;
#pragma unroll
  for (int j = 0; j < TOGETHER; j++) {
    if (WAVE) r[j] = uniform(r[j]), w[j] = __uint_as_float(uniform(__float_as_uint(w[j])));
    if (r[j] >= p.R) r[j] = -1;
  }
}

template <class E, bool WAVE> __global__ __launch_bounds__(256) void k_sum(Sum g) {
  const oob_expert_sum_t &p = g.p;
  int64_t t = token_of<WAVE>(g);
  int64_t c = ((int64_t)blockIdx.y * g.width + threadIdx.x % g.width) * 8, left = p.C - c;
  if (t >= p.T || left <= 0) return;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  typename Vec<E>::v8 res;
  if (p.residual) res = load8<E>((const E *)p.residual + t * p.residual_stride + c, left);
  for (int j0 = 0; j0 < p.k; j0 += TOGETHER) {
    typename Vec<E>::v8 y[TOGETHER];
    float w[TOGETHER];
    int r[TOGETHER];
    places_of<WAVE>(p, t, j0, r, w);
#pragma unroll
    for (int j = 0; j < TOGETHER; j++)
      if (r[j] >= 0) y[j] = load8<E>((const E *)p.y + r[j] * p.y_stride + c, left);
#pragma unroll
    for (int j = 0; j < TOGETHER; j++)
      if (r[j] >= 0)
        for (int e = 0; e < 8; e++) sum[e] += w[j] * (float)y[j][e];
  }
  typename Vec<E>::v8 out;
  for (int e = 0; e < 8; e++) out[e] = (E)(p.residual ? sum[e] + (float)res[e] : sum[e]);
  store8<E>((E *)p.out + t * p.out_stride + c, out, left);
}

/* dy[place] = w dout, dweights = dout . y[place]: a token's row of dout is read once for every TOGETHER choices. */
template <class E, bool WAVE> __global__ __launch_bounds__(256) void k_sum_grad(Sum g) {
  __shared__ float part[4][TOGETHER];
  const oob_expert_sum_t &p = g.p;
  int64_t t = token_of<WAVE>(g);
  bool live = t < p.T;
  int at = threadIdx.x % g.width;
  for (int j0 = 0; j0 < p.k; j0 += TOGETHER) {
    float w[TOGETHER], dot[TOGETHER];
    int r[TOGETHER];
#pragma unroll
    for (int j = 0; j < TOGETHER; j++) dot[j] = 0, r[j] = -1;
    if (live) places_of<WAVE>(p, t, j0, r, w);
    auto columns = [&](int64_t c, int64_t left) __attribute__((always_inline)) {
      typename Vec<E>::v8 y[TOGETHER], d = load8<E>((const E *)g.dout + t * g.ld_dout + c, left);
      if (g.dweights)
#pragma unroll
        for (int j = 0; j < TOGETHER; j++)
          if (r[j] >= 0) y[j] = load8<E>((const E *)p.y + r[j] * p.y_stride + c, left);
      if (g.dy)
#pragma unroll
        for (int j = 0; j < TOGETHER; j++) {
          if (r[j] < 0) continue;
          typename Vec<E>::v8 out;
          for (int e = 0; e < 8; e++) out[e] = (E)(w[j] * (float)d[e]);
          store8<E>((E *)g.dy + r[j] * g.ld_dy + c, out, left);
        }
      if (g.dweights)
#pragma unroll
        for (int j = 0; j < TOGETHER; j++)
          if (r[j] >= 0)
            for (int e = 0; e < 8; e++) dot[j] += (float)d[e] * (float)y[j][e]; /* past the row: zeros */
    };
    if (live)
      for (int64_t c = (int64_t)at * 8; c < p.C; c += g.width * 8) {
        if (p.C - c >= 8) columns(c, 8);
        else columns(c, p.C - c);
      }
    if (!g.dweights) continue;
    int run = g.width < 64 ? g.width : 64;
#pragma unroll
    for (int j = 0; j < TOGETHER; j++)
      for (int o = 1; o < run; o *= 2) dot[j] += __shfl_xor(dot[j], o);
    if (g.width > 64) { /* the sums of a token's waves, in their order */
      __syncthreads();
      if (lane() == 0)
#pragma unroll
        for (int j = 0; j < TOGETHER; j++) part[threadIdx.x / 64][j] = dot[j];
      __syncthreads();
      if (at == 0)
#pragma unroll
        for (int j = 0; j < TOGETHER; j++) { /* width is 128 or 256 */
          dot[j] = part[threadIdx.x / 64][j] + part[threadIdx.x / 64 + 1][j];
          if (g.width > 128) dot[j] += part[2][j], dot[j] += part[3][j];
        }
    }
    if (live && at == 0)
#pragma unroll
      for (int j = 0; j < TOGETHER; j++)
        if (j0 + j < p.k) g.dweights[t * p.k + j0 + j] = r[j] < 0 ? 0.f : dot[j];
  }
}

bool sum_ok(const oob_expert_sum_t *p, bool forward) {
  const int64_t most = (int64_t)1 << 31;
  if (!p || (p->dtype != OOB_BF16 && p->dtype != OOB_FP16 && p->dtype != OOB_FP32) || p->k < 1 || p->k > OOB_EXPERT_MAX_CHOICES) return false;
  if (p->T < 0 || p->R < 0 || p->C < 1 || p->T >= most || p->R >= most || p->C >= most) return false;
  if (p->T == 0) return true;
  size_t of = p->dtype == OOB_FP32 ? 4 : 2;
  if (!p->place || !multiple(p->place, 4) || !multiple(p->weights, 4)) return false;
  if (p->R && (!p->y || !readable(p->y_stride, p->C) || !multiple(p->y, of))) return false;
  if (!forward) return true;
  if (p->residual && (!readable(p->residual_stride, p->C) || !multiple(p->residual, of))) return false;
  return p->out && p->out_stride >= p->C && multiple(p->out, of);
}

/* The result on memory that other workgroups still read. */
bool out_shared(const oob_expert_sum_t *p) {
  const int64_t of = p->dtype == OOB_FP32 ? 4 : 2, cols = p->C * of, n = p->T * p->k * 4;
  Lies out{p->out, p->T, cols, p->out_stride * of}, res{p->residual, p->residual ? p->T : 0, cols, p->residual_stride * of};
  bool in_place = p->out == p->residual && (p->out_stride == p->residual_stride || p->T == 1);
  return share(out, {p->y, p->R, cols, p->y_stride * of}) || share(out, lies_flat(p->place, n)) || share(out, lies_flat(p->weights, n)) || (!in_place && share(out, res));
}

/* Threads of a token: those that its columns need, up to a workgroup. */
int width_of(int64_t C) {
  int w = 1;
  while (w < 256 && w * 8 < C) w *= 2;
  return w;
}

/* The same operands from token t on, as many as a launch takes: it has less than 2^32 threads. */
template <class E> Sum part_of(const Sum &g, int64_t t, int64_t n) {
  Sum q = g;
  oob_expert_sum_t &p = q.p;
  p.T = g.p.T - t < n ? g.p.T - t : n, p.place += t * p.k;
  if (p.weights) p.weights += t * p.k;
  if (p.residual) p.residual = (const E *)p.residual + t * p.residual_stride;
  if (p.out) p.out = (E *)p.out + t * p.out_stride;
  if (q.dout) q.dout = (const E *)q.dout + t * q.ld_dout;
  if (q.dweights) q.dweights += t * p.k;
  return q;
}
template <class E> void sum(const Sum &all, hipStream_t st) {
  int64_t per = 256 / all.width, n = per << 23;
  for (int64_t t = 0; t < all.p.T; t += n) {
    Sum g = part_of<E>(all, t, n);
    dim3 grid((unsigned)((g.p.T + per - 1) / per), (unsigned)((g.p.C + g.width * 8 - 1) / (g.width * 8)));
    if (g.width >= 64) k_sum<E, true><<<grid, 256, 0, st>>>(g);
    else k_sum<E, false><<<grid, 256, 0, st>>>(g);
  }
}
template <class E> void sum_grad(const Sum &all, hipStream_t st) {
  int64_t per = 256 / all.width, n = per << 23;
  for (int64_t t = 0; t < all.p.T; t += n) {
    Sum g = part_of<E>(all, t, n);
    unsigned groups = (unsigned)((g.p.T + per - 1) / per);
    if (g.width >= 64) k_sum_grad<E, true><<<groups, 256, 0, st>>>(g);
    else k_sum_grad<E, false><<<groups, 256, 0, st>>>(g);
  }
}

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" int oob_expert_sum(const oob_expert_sum_t *p, void *stream) {
  if (!sum_ok(p, true)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  if (out_shared(p)) return OOB_EINVAL;
  Sum g{};
  g.p = *p, g.width = width_of(p->C);
  if ((p->C + g.width * 8 - 1) / (g.width * 8) > 65535) return OOB_EINVAL; /* rows of 2^27 values */
  hipStream_t st = (hipStream_t)stream;
  if (p->dtype == OOB_BF16) sum<bf16>(g, st);
  else if (p->dtype == OOB_FP16) sum<fp16>(g, st);
  else sum<float>(g, st);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

extern "C" int oob_expert_sum_backward(const oob_expert_sum_t *p, const void *dout, int64_t dout_stride, void *dy, int64_t dy_stride, float *dweights,
                                       void *stream) {
  if (!sum_ok(p, false)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  size_t of = p->dtype == OOB_FP32 ? 4 : 2;
  if (!dout || !readable(dout_stride, p->C) || !multiple(dout, of) || (!dy && !dweights)) return OOB_EINVAL;
  if ((dy && (dy_stride < p->C || !multiple(dy, of))) || !multiple(dweights, 4)) return OOB_EINVAL;
  const int64_t cols = p->C * (int64_t)of, n = p->T * p->k * 4;
  Lies rows{dy, dy ? p->R : 0, cols, dy_stride * (int64_t)of}, dots = lies_flat(dweights, n);
  for (Lies to : {rows, dots})
    if (share(to, {dout, p->T, cols, dout_stride * (int64_t)of}) || (dweights && share(to, {p->y, p->R, cols, p->y_stride * (int64_t)of})) || share(to, lies_flat(p->place, n)) ||
        share(to, lies_flat(p->weights, n)))
      return OOB_EINVAL;
  if (share(rows, dots)) return OOB_EINVAL;
  Sum g{*p, width_of(p->C), dout, dy, dout_stride, dy_stride, dweights};
  hipStream_t st = (hipStream_t)stream;
  if (p->dtype == OOB_BF16) sum_grad<bf16>(g, st);
  else if (p->dtype == OOB_FP16) sum_grad<fp16>(g, st);
  else sum_grad<float>(g, st);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}
