/* Norms around a block with its gate, residual scale and dropout, their gradients, and dropout alone. */
#include "oob_layer_device.h"

namespace layer {

struct Norm {
  const void *x, *z, *w, *b, *pw, *pb, *gate;
  void *xp, *h;
  float *mean, *rstd, *pmean, *prstd; /* [T] each; the p's belong to the norm behind the block */
  int64_t T, C, ldx, ldz, rows_per_gate;
  int pre, post;
  float eps, alpha;
  Dropout drop;
};

struct NormGrad {
  Norm n; /* xp is read (from its place in x: n.x) */
  const void *dxp, *dh;
  int64_t ld_dxp, ld_dh;
  void *dx, *dz, *dgate;
  float *sums;        /* [workgroups][2 or 4][C]: dw, db, dpw, dpb */
  float *gate_sums;   /* [workgroups][C], or null: a workgroup has whole groups and writes dgate itself */
  int64_t rows;       /* of a workgroup */
  int64_t workgroups_per_gate;
};

/* Sums of N values over the WAVES waves that share a row, in every lane. */
template <int WAVES, int N> __device__ inline void sum_row(float (&v)[N], float *part, int &turn) {
  static_assert(N <= 6, "places");
  for (int k = 32; k > 0; k >>= 1)
    for (int i = 0; i < N; i++) v[i] += __shfl_xor(v[i], k);
  if (WAVES == 1) return;
  float *p = part + turn * WAVES * 6; /* two places in turn: a place is written again only behind a barrier that everybody passed after reading it */
  turn ^= 1;
  if (lane() == 0)
    for (int i = 0; i < N; i++) p[threadIdx.x / 64 * 6 + i] = v[i];
  __syncthreads();
  for (int i = 0; i < N; i++) {
    float s = 0;
    for (int k = 0; k < WAVES; k++) s += p[k * 6 + i];
    v[i] = s;
  }
}

/* Mean and 1 / deviation of a row held in registers: the deviation from the mean, not from the sum of squares. */
template <int WAVES, int V> __device__ inline void statistics(const float (&x)[V][8], int kind, int64_t C, float eps, int c0, float &mean, float &rstd, float *part, int &turn) {
  mean = 0;
  if (kind == OOB_NORM_LAYER) {
    float s[1] = {0};
    for (int k = 0; k < V; k++)
      for (int e = 0; e < 8; e++) s[0] += x[k][e];
    sum_row<WAVES, 1>(s, part, turn);
    mean = s[0] / C;
  }
  float q[1] = {0};
  for (int k = 0; k < V; k++)
    for (int e = 0; e < 8; e++) {
      float d = c0 + k * WAVES * 512 + e < C ? x[k][e] - mean : 0.f;
      q[0] += d * d;
    }
  sum_row<WAVES, 1>(q, part, turn);
  rstd = 1 / sqrtf(q[0] / C + eps);
}

/* Eight of a vector, or a constant where there is none. */
template <class E> __device__ inline typename Vec<E>::v8 load8_or(const void *p, int64_t at, int64_t left, float otherwise) {
  if (p) return load8<E>((const E *)p + at, left);
  typename Vec<E>::v8 v;
  for (int e = 0; e < 8; e++) v[e] = (E)otherwise;
  return v;
}
template <class E> __device__ inline void widen(typename Vec<E>::v8 v, float (&f)[8]) {
  for (int e = 0; e < 8; e++) f[e] = (float)v[e];
}
template <class E> __device__ inline void narrow(const float (&f)[8], typename Vec<E>::v8 &v) {
  for (int e = 0; e < 8; e++) v[e] = (E)f[e];
}

/* A row by WAVES waves, V x 8 values a lane, all of them in registers from the one read to the one write.  A workgroup is at least four
 * waves: rows of one wave go four at a time. */
template <class E, int WAVES, int V> __global__ __launch_bounds__(WAVES < 4 ? 256 : WAVES * 64) void k_norm(Norm n) {
  constexpr int ROWS = WAVES == 1 ? 4 : 1;
  __shared__ float part[WAVES * 12];
  int turn = 0;
  int c0 = (WAVES == 1 ? lane() : threadIdx.x) * 8;
  const int64_t C = n.C;
  typename Vec<E>::v8 w[V], b[V];
  for (int k = 0; k < V; k++) {
    int64_t c = c0 + k * WAVES * 512;
    w[k] = load8_or<E>(n.w, c, C - c, 1.f);
    b[k] = load8_or<E>(n.b, c, C - c, 0.f);
  }
  typename Vec<E>::v8 vx[V], vz[V];
  auto load = [&](int64_t t) __attribute__((always_inline)) {
    for (int k = 0; k < V; k++) {
      int64_t c = c0 + k * WAVES * 512;
      vx[k] = load8<E>((const E *)n.x + t * n.ldx + c, C - c);
      if (n.z) vz[k] = load8<E>((const E *)n.z + t * n.ldz + c, C - c);
    }
  };
  int64_t t = (int64_t)blockIdx.x * ROWS + (WAVES == 1 ? threadIdx.x / 64 : 0), stride = (int64_t)gridDim.x * ROWS;
  if (t < n.T) load(t);
  for (; t < n.T; t += stride) {
    float x[V][8], u[V][8];
    for (int k = 0; k < V; k++) {
      widen<E>(vx[k], x[k]);
      if (n.z) widen<E>(vz[k], u[k]);
    }
    if (t + stride < n.T) load(t + stride); /* on its way while this row is worked on */
    if (n.z) {
      if (n.post != OOB_NORM_NONE) {
        float mean, rstd;
        statistics<WAVES, V>(u, n.post, C, n.eps, c0, mean, rstd, part, turn);
        for (int k = 0; k < V; k++) {
          int64_t c = c0 + k * WAVES * 512;
          typename Vec<E>::v8 pw = load8_or<E>(n.pw, c, C - c, 1.f), pb = load8_or<E>(n.pb, c, C - c, 0.f);
          for (int e = 0; e < 8; e++) u[k][e] = (u[k][e] - mean) * rstd * (float)pw[e] + (float)pb[e];
        }
        if (c0 == 0) {
          if (n.pmean) n.pmean[t] = mean;
          if (n.prstd) n.prstd[t] = rstd;
        }
      }
      for (int k = 0; k < V; k++) {
        int64_t c = c0 + k * WAVES * 512;
        if (n.drop.threshold) {
          uint64_t lo, hi;
          random8(n.drop, (uint64_t)t * C + c, lo, hi);
          for (int e = 0; e < 8; e++) u[k][e] *= keep(n.drop, lo, hi, e);
        }
        if (n.gate) {
          typename Vec<E>::v8 g = load8<E>((const E *)n.gate + t / n.rows_per_gate * C + c, C - c);
          for (int e = 0; e < 8; e++) u[k][e] *= (float)g[e];
        }
        typename Vec<E>::v8 out;
        for (int e = 0; e < 8; e++) x[k][e] = c + e < C ? n.alpha * x[k][e] + u[k][e] : 0.f;
        narrow<E>(x[k], out);
        store8<E>((E *)n.xp + t * C + c, out, C - c);
      }
    }
    float mean, rstd;
    statistics<WAVES, V>(x, n.pre, C, n.eps, c0, mean, rstd, part, turn);
    if (c0 == 0) {
      if (n.mean) n.mean[t] = mean;
      if (n.rstd) n.rstd[t] = rstd;
    }
    for (int k = 0; k < V; k++) {
      int64_t c = c0 + k * WAVES * 512;
      typename Vec<E>::v8 out;
      for (int e = 0; e < 8; e++) out[e] = (E)((x[k][e] - mean) * rstd * (float)w[k][e] + (float)b[k][e]);
      store8<E>((E *)n.h + t * C + c, out, C - c);
    }
  }
}

/* From a variance that its rounding may have made negative; a NaN stays one (fmaxf would give 0). */
__device__ inline float inverse_deviation(float variance, float eps) { return 1 / sqrtf((variance < 0 ? 0.f : variance) + eps); }

/* Backward.  With xhat = (x' - mean) rstd and c = dh w:  d = dx' + rstd (c - mean(c) - xhat mean(c xhat))  (rms: without mean(c)),
 * dx = alpha d, dw = sum dh xhat, db = sum dh.  Behind it, where there is more than the residual sum: du = d gate keep, dgate = sum d u,
 * and the norm behind the block the same way from zhat.  A workgroup takes a run of rows and keeps the sums of its columns in registers. */
template <class E, int WAVES, int V, bool POST, bool GATE> __global__ __launch_bounds__(WAVES * 64) void k_norm_grad(NormGrad g) {
  const Norm &n = g.n;
  __shared__ float part[WAVES * 12];
  int turn = 0;
  int c0 = threadIdx.x * 8;
  const int64_t C = n.C;
  float dw[V][8] = {}, db[V][8] = {}, dpw[POST ? V : 1][8] = {}, dpb[POST ? V : 1][8] = {}, dg[GATE ? V : 1][8] = {};
  int64_t t0 = (int64_t)blockIdx.x * g.rows, t1 = t0 + g.rows;
  if (GATE && g.workgroups_per_gate) { /* the runs of a group's rows end with it */
    int64_t first = blockIdx.x / g.workgroups_per_gate * n.rows_per_gate;
    t0 = first + blockIdx.x % g.workgroups_per_gate * g.rows;
    t1 = t0 + g.rows < first + n.rows_per_gate ? t0 + g.rows : first + n.rows_per_gate;
  }
  if (t1 > n.T) t1 = n.T;
  for (int64_t t = t0; t < t1; t++) {
    typename Vec<E>::v8 vx[V], vd[V], vh[V], vz[V];
    for (int k = 0; k < V; k++) {
      int64_t c = c0 + k * WAVES * 512;
      vx[k] = load8<E>((const E *)n.x + t * n.ldx + c, C - c);
      vh[k] = load8<E>((const E *)g.dh + t * g.ld_dh + c, C - c);
      vd[k] = load8_or<E>(g.dxp, t * g.ld_dxp + c, C - c, 0.f);
      if (POST || GATE) vz[k] = load8<E>((const E *)n.z + t * n.ldz + c, C - c);
    }
    /* The statistics are those of x' as it was stored, not of what it was before: with y = x' - (the forward pass's mean), the row's
     * mean is that mean + sum(y) / C, and all that is needed are the sums of y, y^2, c and c y. */
    float mean = n.pre == OOB_NORM_LAYER ? n.mean[t] : 0.f;
    float pmean = POST && n.post == OOB_NORM_LAYER ? n.pmean[t] : 0.f;
    float d[V][8], s[POST ? 6 : 4] = {};
    for (int k = 0; k < V; k++) {
      int64_t c = c0 + k * WAVES * 512;
      typename Vec<E>::v8 w = load8_or<E>(n.w, c, C - c, 1.f);
      for (int e = 0; e < 8; e++) {
        float y = c + e < C ? (float)vx[k][e] - mean : 0.f;
        float v = (float)vh[k][e] * (float)w[e];
        d[k][e] = v;
        s[0] += y;
        s[1] += y * y;
        s[2] += v;
        s[3] += v * y;
        if (POST) {
          float z = c + e < C ? (float)vz[k][e] - pmean : 0.f;
          s[4] += z;
          s[5] += z * z;
        }
      }
    }
    sum_row<WAVES, POST ? 6 : 4>(s, part, turn);
    float shift = n.pre == OOB_NORM_LAYER ? s[0] / C : 0.f;
    float rstd = inverse_deviation(s[1] / C - shift * shift, n.eps);
    float m0 = n.pre == OOB_NORM_LAYER ? s[2] / C : 0.f, m1 = rstd * (s[3] - shift * s[2]) / C;
    float pshift = 0, prstd = 0, q[2] = {0, 0}; /* the norm behind the block: its mean without the rounding to one number, as above */
    if (POST) {
      pshift = n.post == OOB_NORM_LAYER ? s[4] / C : 0.f;
      prstd = inverse_deviation(s[5] / C - pshift * pshift, n.eps);
    }
    for (int k = 0; k < V; k++) {
      int64_t c = c0 + k * WAVES * 512;
      typename Vec<E>::v8 out, gate, pw, pb;
      for (int e = 0; e < 8; e++) {
        float xhat = (((float)vx[k][e] - mean) - shift) * rstd; /* not less the sum of both: it would round */
        dw[k][e] += (float)vh[k][e] * xhat;
        db[k][e] += (float)vh[k][e];
        d[k][e] = (float)vd[k][e] + rstd * (d[k][e] - m0 - xhat * m1);
        out[e] = (E)(n.alpha * d[k][e]);
      }
      store8<E>((E *)g.dx + t * C + c, out, C - c);
      if (!g.dz) continue;
      float kept[8];
      if (n.drop.threshold) {
        uint64_t lo, hi;
        random8(n.drop, (uint64_t)t * C + c, lo, hi);
        for (int e = 0; e < 8; e++) kept[e] = keep(n.drop, lo, hi, e);
      } else
        for (int e = 0; e < 8; e++) kept[e] = 1;
      if (GATE) gate = load8<E>((const E *)n.gate + t / n.rows_per_gate * C + c, C - c);
      if (POST) pw = load8_or<E>(n.pw, c, C - c, 1.f);
      if (GATE && POST) pb = load8_or<E>(n.pb, c, C - c, 0.f);
      for (int e = 0; e < 8; e++) {
        bool in = c + e < C;
        float du = d[k][e] * kept[e];
        float z = POST || GATE ? (float)vz[k][e] : 0.f;
        float zhat = POST ? ((z - pmean) - pshift) * prstd : z;
        if (GATE) {
          float u = zhat;
          if (POST) u = zhat * (float)pw[e] + (float)pb[e];
          dg[k][e] += du * u;
          du *= (float)gate[e];
        }
        if (POST) {
          du = in ? du : 0.f;
          dpw[k][e] += du * zhat;
          dpb[k][e] += du;
          du *= (float)pw[e];
          q[0] += du;
          q[1] += du * zhat;
        }
        d[k][e] = du;
        out[e] = (E)du;
      }
      if (!POST) store8<E>((E *)g.dz + t * C + c, out, C - c);
    }
    if (POST && g.dz) {
      sum_row<WAVES, 2>(q, part, turn);
      float p0 = n.post == OOB_NORM_LAYER ? q[0] / C : 0.f, p1 = q[1] / C;
      for (int k = 0; k < V; k++) {
        int64_t c = c0 + k * WAVES * 512;
        typename Vec<E>::v8 out;
        for (int e = 0; e < 8; e++) out[e] = (E)(prstd * (d[k][e] - p0 - (((float)vz[k][e] - pmean) - pshift) * prstd * p1));
        store8<E>((E *)g.dz + t * C + c, out, C - c);
      }
    }
    if (GATE && !g.workgroups_per_gate && (t + 1) % n.rows_per_gate == 0)
      for (int k = 0; k < V; k++) {
        int64_t c = c0 + k * WAVES * 512;
        typename Vec<E>::v8 out;
        narrow<E>(dg[k], out);
        store8<E>((E *)g.dgate + t / n.rows_per_gate * C + c, out, C - c);
        for (int e = 0; e < 8; e++) dg[k][e] = 0;
      }
  }
  constexpr int S = POST ? 4 : 2;
  for (int k = 0; k < V; k++) {
    int64_t c = c0 + k * WAVES * 512;
    float *to = g.sums + (int64_t)blockIdx.x * S * C + c;
    auto put = [&](float *p, float (&f)[8]) {
      typename Vec<float>::v8 v;
      for (int e = 0; e < 8; e++) v[e] = f[e];
      store8<float>(p, v, C - c);
    };
    put(to, dw[k]);
    put(to + C, db[k]);
    if (POST) put(to + 2 * C, dpw[k]), put(to + 3 * C, dpb[k]);
    if (GATE && g.workgroups_per_gate) put(g.gate_sums + (int64_t)blockIdx.x * C + c, dg[k]);
  }
}

/* Sums over the workgroups: row y of the grid is one of the results. */
struct NormSums {
  const float *from[2]; /* [runs][kinds][C], and the gates' [groups][runs][C] */
  void *to[5];          /* dw, db, dpw, dpb, dgate */
  int64_t C, runs, gate_runs;
  int kinds;
};
template <class E> __global__ __launch_bounds__(256) void k_norm_sums(NormSums g) {
  __shared__ float part[4][64];
  int64_t c = (int64_t)blockIdx.x * 64 + lane();
  int y = blockIdx.y;
  E *to = (E *)g.to[y < g.kinds ? y : 4];
  if (!to) return;
  const float *p = g.from[0] + y * g.C;
  int64_t runs = g.runs, step = g.kinds * g.C;
  if (y >= g.kinds) p = g.from[1] + (y - g.kinds) * g.gate_runs * g.C, runs = g.gate_runs, step = g.C, to += (y - g.kinds) * g.C;
  float s = 0;
  if (c < g.C)
#pragma unroll 8
    for (int64_t r = threadIdx.x / 64; r < runs; r += 4) s += p[r * step + c];
  part[threadIdx.x / 64][lane()] = s;
  __syncthreads();
  if (threadIdx.x < 64 && c < g.C) to[c] = (E)((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]));
}

/* y = x keep / (1 - p).  Two 64-bit hashes for eight elements keep it bound by memory: 11 us for 16.8 M bfloat16 elements, 6.1 TB/s (part of
 * them still in the last-level cache). */
template <class E> __global__ __launch_bounds__(256) void k_dropout(const E *x, E *y, int64_t n, Dropout d) {
  for (int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8; i < n; i += (int64_t)gridDim.x * 2048) {
    typename Vec<E>::v8 v = load8<E>(x + i, n - i);
    uint64_t lo, hi;
    random8(d, i, lo, hi);
    for (int e = 0; e < 8; e++) v[e] = (E)((float)v[e] * keep(d, lo, hi, e));
    store8<E>(y + i, v, n - i);
  }
}

/* ---- host ---- */
static bool norm_ok(const oob_norm *p) {
  if (p->dtype < OOB_BF16 || p->dtype > OOB_FP32 || p->T < 0 || p->C < 1 || p->C > OOB_NORM_MAX_C || p->T >= ((int64_t)1 << 40)) return false;
  if ((p->pre != OOB_NORM_LAYER && p->pre != OOB_NORM_RMS) || p->post < OOB_NORM_NONE || p->post > OOB_NORM_RMS) return false;
  if (!(p->eps >= 0) || !(p->p >= 0 && p->p < 1) || (double)p->p * 65536 + 0.5 >= 65536) return false;
  if (p->gates < 0 || (p->gates > 0 && (!p->gate || p->T == 0 || p->T % p->gates != 0))) return false;
  if (p->T == 0) return true;
  size_t e = p->dtype == OOB_FP32 ? 4 : 2;
  for (const void *a : {p->x, p->z, p->weight, p->bias, p->post_weight, p->post_bias, p->gate, (const void *)p->xp, (const void *)p->h})
    if (!multiple(a, e)) return false;
  if (!multiple(p->saved, 4) || !p->x || p->x_stride < p->C) return false;
  if (p->z) return p->z_stride >= p->C;
  return p->post == OOB_NORM_NONE && !p->gates && p->p == 0 && p->alpha == 1;
}

static Norm norm_of(const oob_norm *p) {
  Norm n{};
  n.x = p->x, n.z = p->z, n.w = p->weight, n.b = p->bias, n.pw = p->post_weight, n.pb = p->post_bias, n.gate = p->gates ? p->gate : nullptr;
  n.xp = p->xp, n.h = p->h;
  if (p->saved) n.mean = p->saved, n.rstd = p->saved + p->T, n.pmean = p->saved + 2 * p->T, n.prstd = p->saved + 3 * p->T;
  if (p->post == OOB_NORM_NONE) n.pmean = n.prstd = nullptr;
  n.T = p->T, n.C = p->C, n.ldx = p->x_stride, n.ldz = p->z_stride, n.rows_per_gate = p->gates ? p->T / p->gates : 1;
  n.pre = p->pre, n.post = p->post, n.eps = p->eps, n.alpha = p->alpha;
  n.drop = dropout_of(p->p, p->seed, p->offset);
  return n;
}

template <class E> static void norm(const Norm &n, hipStream_t st) {
  /* Rows of up to 1024 by one wave: no barrier; wider ones by as many waves as keep a lane's part in 32 registers.  Workgroups (768 of eight
   * waves) go through the rows with the weights in registers and the next row on its way (4096 x 12288, bfloat16: 87 us with dropout and 82 without,
   * 4.6 and 4.9 TB/s, a large copy's rate; a quarter more by 2048 workgroups without the row ahead).  Four vectors a lane of 32-bit values do not
   * fit the registers: rows over 12 288 in float32 take 282 us (4096 x 16384, 3.8 TB/s). */
  int64_t need = (n.C + 511) / 512, rows = n.T < 2048 ? n.T : 2048, wide = n.T < 768 ? n.T : 768, rows4 = n.T < 8192 ? (n.T + 3) / 4 : 2048;
  if (need <= 1) k_norm<E, 1, 1><<<(unsigned)rows4, 256, 0, st>>>(n);
  else if (need <= 2) k_norm<E, 1, 2><<<(unsigned)rows4, 256, 0, st>>>(n);
  else if (need <= 4) k_norm<E, 4, 1><<<(unsigned)rows, 256, 0, st>>>(n);
  else if (need <= 8) k_norm<E, 4, 2><<<(unsigned)rows, 256, 0, st>>>(n);
  else if (need <= 16) k_norm<E, 8, 2><<<(unsigned)wide, 512, 0, st>>>(n);
  else if (need <= 24) k_norm<E, 8, 3><<<(unsigned)wide, 512, 0, st>>>(n);
  else k_norm<E, 8, 4><<<(unsigned)wide, 512, 0, st>>>(n);
}

struct Runs { int64_t workgroups, rows, per_gate; };

/* Workgroups of the backward pass: enough waves to fill the GPU, and no more: each leaves a row of sums per weight (4096 x 12288: 130 us
 * with 256 workgroups of eight waves, 141 with 512; 4096 x 4096: 47 us with 512 of four, 61 with 256; what is read and written at a copy's
 * rate would take 100 and 33 us; loading the next row ahead gained nothing).  Where there are gates, a workgroup's rows belong to one gate, or, with
 * more gates than workgroups, to whole gates. */
static Runs runs_of(int64_t T, int64_t C, int64_t gates) {
  const int64_t most = C > 4096 ? 256 : 512;
  if (gates > most) {
    int64_t per = (gates + most - 1) / most, rows = per * (T / gates);
    return {(T + rows - 1) / rows, rows, 0};
  }
  int64_t g = gates ? gates : 1, of = T / g; /* rows of a gate (T % g == 0) */
  int64_t per = most / g < of ? most / g : of;
  if (per < 1) per = 1;
  int64_t rows = (of + per - 1) / per;
  per = rows ? (of + rows - 1) / rows : 1;
  return {g * per, rows, per};
}

template <class E, bool POST, bool GATE> static void norm_grad(const NormGrad &g, unsigned n, hipStream_t st) {
  int64_t need = (g.n.C + 511) / 512;
  if (need <= 1) k_norm_grad<E, 1, 1, POST, GATE><<<n, 64, 0, st>>>(g);
  else if (need <= 2) k_norm_grad<E, 2, 1, POST, GATE><<<n, 128, 0, st>>>(g);
  else if (need <= 4) k_norm_grad<E, 4, 1, POST, GATE><<<n, 256, 0, st>>>(g);
  else if (need <= 8) k_norm_grad<E, 4, 2, POST, GATE><<<n, 256, 0, st>>>(g);
  else if (need <= 16) k_norm_grad<E, 8, 2, POST, GATE><<<n, 512, 0, st>>>(g);
  else if (need <= 24) k_norm_grad<E, 8, 3, POST, GATE><<<n, 512, 0, st>>>(g);
  else k_norm_grad<E, 8, 4, POST, GATE><<<n, 512, 0, st>>>(g);
}

template <class E> static int norm_backward(const oob_norm *p, const oob_norm_grad *q, Arena a, hipStream_t st) {
  Runs r = runs_of(p->T, p->C, p->gates);
  bool post = p->post != OOB_NORM_NONE, gate = p->gates > 0;
  int kinds = post ? 4 : 2;
  NormGrad g{};
  g.n = norm_of(p);
  g.dxp = q->dxp, g.ld_dxp = q->dxp_stride, g.dh = q->dh, g.ld_dh = q->dh_stride;
  g.dx = q->dx, g.dz = p->z ? q->dz : nullptr, g.dgate = q->dgate;
  g.sums = (float *)a.take((size_t)r.workgroups * kinds * p->C * 4);
  g.gate_sums = gate && r.per_gate ? (float *)a.take((size_t)r.workgroups * p->C * 4) : nullptr;
  g.rows = r.rows, g.workgroups_per_gate = r.per_gate;
  if (!a.ok()) return OOB_ECAPACITY;
  if (p->T) {
    unsigned n = (unsigned)r.workgroups;
    if (post && gate) norm_grad<E, true, true>(g, n, st);
    else if (post) norm_grad<E, true, false>(g, n, st);
    else if (gate) norm_grad<E, false, true>(g, n, st);
    else norm_grad<E, false, false>(g, n, st);
  }
  NormSums s{};
  s.from[0] = g.sums, s.from[1] = g.gate_sums, s.C = p->C, s.runs = p->T ? r.workgroups : 0, s.gate_runs = p->T ? r.per_gate : 0, s.kinds = kinds;
  s.to[0] = q->dweight, s.to[1] = q->dbias, s.to[2] = post ? q->dpost_weight : nullptr, s.to[3] = post ? q->dpost_bias : nullptr;
  s.to[4] = gate && r.per_gate ? q->dgate : nullptr;
  k_norm_sums<E><<<dim3((unsigned)((p->C + 63) / 64), (unsigned)(kinds + (s.to[4] ? p->gates : 0))), 256, 0, st>>>(s);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

static size_t norm_bytes(const oob_norm *p) {
  Runs r = runs_of(p->T, p->C, p->gates);
  Arena a{nullptr, 0, 0};
  a.take((size_t)r.workgroups * (p->post != OOB_NORM_NONE ? 4 : 2) * p->C * 4);
  if (p->gates && r.per_gate) a.take((size_t)r.workgroups * p->C * 4);
  return a.used;
}

}  // namespace layer

using namespace layer;

extern "C" int oob_layer_norm(const oob_norm *p, void *stream) {
  if (!p || !norm_ok(p)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  if (!p->h || (p->z && !p->xp)) return OOB_EINVAL;
  Norm n = norm_of(p);
  if (p->dtype == OOB_BF16) norm<bf16>(n, (hipStream_t)stream);
  else if (p->dtype == OOB_FP16) norm<fp16>(n, (hipStream_t)stream);
  else norm<float>(n, (hipStream_t)stream);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

extern "C" size_t oob_layer_norm_backward_workspace_size(const oob_norm *p) { return p && norm_ok(p) ? norm_bytes(p) : 0; }

extern "C" int oob_layer_norm_backward(const oob_norm *p, const oob_norm_grad *q, void *workspace, size_t bytes, void *stream) {
  if (!p || !q || !norm_ok(p)) return OOB_EINVAL;
  size_t e = p->dtype == OOB_FP32 ? 4 : 2;
  for (const void *a : {q->dxp, q->dh, (const void *)q->dx, (const void *)q->dz, (const void *)q->dweight, (const void *)q->dbias, (const void *)q->dpost_weight,
                        (const void *)q->dpost_bias, (const void *)q->dgate})
    if (!multiple(a, e)) return OOB_EINVAL;
  if (p->T && (!p->saved || !q->dh || q->dh_stride < p->C || (q->dxp && q->dxp_stride < p->C) || !q->dx || (p->z && !q->dz))) return OOB_EINVAL;
  if (p->gates && !q->dgate) return OOB_EINVAL;
  if (!multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = norm_bytes(p);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena a{(char *)workspace, bytes, 0};
  if (p->dtype == OOB_BF16) return norm_backward<bf16>(p, q, a, (hipStream_t)stream);
  if (p->dtype == OOB_FP16) return norm_backward<fp16>(p, q, a, (hipStream_t)stream);
  return norm_backward<float>(p, q, a, (hipStream_t)stream);
}

extern "C" int oob_layer_dropout(int dtype, const void *x, void *y, int64_t n, float p, uint64_t seed, uint64_t offset, void *stream) {
  if (dtype < OOB_BF16 || dtype > OOB_FP32 || n < 0 || !(p >= 0 && p < 1) || (double)p * 65536 + 0.5 >= 65536) return OOB_EINVAL;
  if (n == 0) return OOB_OK;
  size_t e = dtype == OOB_FP32 ? 4 : 2;
  if (!x || !y || !multiple(x, e) || !multiple(y, e)) return OOB_EINVAL;
  Dropout d = dropout_of(p, seed, offset);
  int64_t wgs = (n + 2047) / 2048;
  unsigned grid = (unsigned)(wgs < 4096 ? wgs : 4096);
  hipStream_t st = (hipStream_t)stream;
  if (dtype == OOB_BF16) k_dropout<bf16><<<grid, 256, 0, st>>>((const bf16 *)x, (bf16 *)y, n, d);
  else if (dtype == OOB_FP16) k_dropout<fp16><<<grid, 256, 0, st>>>((const fp16 *)x, (fp16 *)y, n, d);
  else k_dropout<float><<<grid, 256, 0, st>>>((const float *)x, (float *)y, n, d);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}
