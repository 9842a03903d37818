/* Attention over a range of keys per query, and its gradients. */
#include "oob_layer_device.h"

#include <math.h>

namespace layer {

struct Heads { const char *p; int64_t batch, row, head; }; /* [B][S][heads][D], strides in bytes */

struct Attention {
  Heads q, k, v, o;
  const int32_t *begin, *end;
  const float *slopes;
  float *lse;
  int B, Sq, Sk, H, G, D;
  int causal;
  float scale, cap;
  /* backward */
  Heads dout, dq, dk, dv;
  const float *delta;  /* [B][H][Sq]: do . o */
  const int4 *ranges;  /* [B][tiles of 64 queries]: smallest begin, largest end, largest begin, smallest end */
};

constexpr int KT = 64;      /* rows of a tile in LDS (keys; queries in dk, dv) */
constexpr int WAVES = 4, ROWS = WAVES * 32; /* queries (keys) of a workgroup: 32 a wave */
constexpr float LOG2E = 1.44269504f, LN2 = 0.69314718f;
constexpr int FAR = 0x3fffffff; /* the begin of a row that sees nothing */

/* Chunk c (16 bytes) of row r is at c ^ swizzle(r): sixteen rows' chunk c, and four rows' four chunks, lie in different banks. */
template <int DP> __device__ inline int swizzle(int r) {
  return DP == 128 ? (r & 3) << 2 | (r >> 2 & 3) : (r >> 1 & 1) << 2 | (r >> 2 & 3);
}

/* Keys that query i sees: begin <= j < end; none: FAR, 0. */
__device__ inline void key_range(const Attention &a, int b, int i, int &begin, int &end) {
  begin = FAR, end = 0;
  if (i >= a.Sq) return;
  int lo = 0, hi = a.Sk;
  if (a.causal) {
    int64_t e = (int64_t)i + a.Sk - a.Sq + 1;
    hi = e < hi ? (int)(e > 0 ? e : 0) : hi;
  }
  if (a.begin) lo = max(lo, a.begin[(int64_t)b * a.Sq + i]);
  if (a.end) hi = min(hi, a.end[(int64_t)b * a.Sq + i]);
  if (lo < hi) begin = lo, end = hi;
}

/* 64 rows of a head on their way to LDS. */
template <int DP> struct Rows {
  static constexpr int BYTES = KT * DP * 2, LOADS = BYTES / (WAVES * 64 * 16);
  uint32_t off[LOADS];
  int row[LOADS];
  __device__ void init(int64_t stride, int D) {
    for (int i = 0; i < LOADS; i++) {
      int p = (i * WAVES * 64 + threadIdx.x) * 16, r = p / (DP * 2), c = (p / 16 % (DP / 8)) ^ swizzle<DP>(r);
      row[i] = r;
      off[i] = c * 8 < D ? (uint32_t)(r * stride + c * 16) : OOB_LAYER_OUT;
    }
  }
  /* rows lo <= first + r < hi; zeros for the others */
  __device__ void load(const char *base, int64_t stride, lds_char *to, int first, int lo, int hi) {
    __amdgpu_buffer_rsrc_t r = buffer(base + first * stride);
    int wave = uniform(threadIdx.x / 64);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      int at = first + row[i];
      load_lds(r, to + (i * WAVES * 64 + wave * 64) * 16, at >= lo && at < hi ? off[i] : OOB_LAYER_OUT);
    }
  }
};

/* Fragments of a tile's 32 rows from r0 on.  Straight: row l % 32, columns 16 t + 8 (l / 32) .. + 7. */
template <class E, int DP> __device__ inline typename Vec<E>::v8 straight(lds_char *tile, int r0, int t) {
  int l = lane(), r = r0 + (l & 31);
  return lds_read8<E>(tile + r * DP * 2 + ((2 * t + (l >> 5)) ^ swizzle<DP>(r)) * 16);
}
/* Transposed: column d0 + l % 32, rows r0 + 4 (l / 32) .. + 3 and r0 + 8 + 4 (l / 32) .. + 3: the rows whose values of a product a lane
 * holds in eight registers in a row, so that they are the other operand as they are. */
template <class E, int DP> __device__ inline typename Vec<E>::v8 transposed(lds_char *tile, int r0, int d0) {
  int l = lane(), r = r0 + 4 * (l >> 5) + ((l & 15) >> 2), c = d0 / 8 + ((l >> 4) & 1) * 2 + ((l >> 1) & 1);
  lds_char *p = tile + r * DP * 2 + (c ^ swizzle<DP>(r)) * 16 + (l & 1) * 8;
  lds_char *q = tile + (r + 8) * DP * 2 + (c ^ swizzle<DP>(r + 8)) * 16 + (l & 1) * 8;
  return lds_read_tr<E>(p, q);
}

/* Row `i` of a head as the second operand of products over d: d = 16 t + 8 (l / 32) .. + 7. */
template <class E, int DP> __device__ inline void row_fragments(const Heads &h, int64_t at, int i, bool in, int D, typename Vec<E>::v8 (&f)[DP / 16]) {
  for (int t = 0; t < DP / 16; t++) {
    int d = 16 * t + 8 * (lane() >> 5);
    f[t] = load8<E>((const E *)(h.p + at + i * h.row) + d, in ? D - d : 0);
  }
}

template <class E> __device__ inline typename Vec<E>::v8 round8(const float *p) {
  typename Vec<E>::v8 v;
  for (int e = 0; e < 8; e++) v[e] = (E)p[e];
  return v;
}

/* Four consecutive values of a row. */
template <class E> __device__ inline void store4(char *row, int d, int D, float a, float b, float c, float e) {
  E *p = (E *)row + d;
  typedef typename Vec<E>::v4 v4 __attribute__((aligned(2)));
  if (d + 4 <= D) {
    v4 v = {(E)a, (E)b, (E)c, (E)e};
    *(v4 *)p = v;
  } else {
    if (d < D) p[0] = (E)a;
    if (d + 1 < D) p[1] = (E)b;
    if (d + 2 < D) p[2] = (E)c;
  }
}

/* Column `l % 32` of a transposed result (d in the registers) to its row. */
template <class E, int DP> __device__ inline void store_column(const f32x16 (&acc)[DP / 32], float by, char *row, int D) {
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r += 4)
      store4<E>(row, 32 * t + 8 * (r >> 2) + 4 * (lane() >> 5), D, acc[t][r] * by, acc[t][r + 1] * by, acc[t][r + 2] * by, acc[t][r + 3] * by);
}

__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float tanh_(float x) { return 1 - 2 * __builtin_amdgcn_rcpf(1 + exp2_(x * (2 * LOG2E))); }

/* Raw products to scores times log2 e, where there is a cap or a bias (with neither, the caller folds the scale into the exponent). */
__device__ inline float score(const Attention &a, float slope2, float raw, int distance) {
  float s = raw * a.scale;
  if (a.cap > 0) s = a.cap * tanh_(s / a.cap);
  return s * LOG2E - slope2 * abs(distance);
}

/* The smallest begin and largest end over the workgroup's rows (each wave's in its lanes). */
__device__ inline void join_ranges(int &lo, int &hi, int (*part)[2]) {
  int wave = threadIdx.x / 64;
  if (lane() == 0) part[wave][0] = lo, part[wave][1] = hi;
  __syncthreads();
  for (int w = 0; w < WAVES; w++) lo = min(lo, part[w][0]), hi = max(hi, part[w][1]);
  lo = uniform(lo), hi = uniform(hi);
}
__device__ inline int wave_min(int v) {
  for (int k = 32; k > 0; k >>= 1) v = min(v, __shfl_xor(v, k));
  return uniform(v);
}
__device__ inline int wave_max(int v) {
  for (int k = 32; k > 0; k >>= 1) v = max(v, __shfl_xor(v, k));
  return uniform(v);
}

/* Which (tile, head, sequence) a workgroup takes.  Heads vary slowest within an XCD's share, so that what it reads of keys and values
 * stays in its L2; the last tiles, which see most keys where a mask is causal, go first. */
__device__ inline void place(int tiles, int heads, int &tile, int &head, int &b) {
  int64_t id = xcd_order(blockIdx.x, gridDim.x);
  tile = tiles - 1 - (int)(id % tiles);
  head = (int)(id / tiles % heads);
  b = (int)(id / tiles / heads);
}

/* ---- forward ------------------------------------------------------------------------------------------------------------------
 * A wave has 32 queries, one a lane pair: scores are formed transposed (keys in the registers, the query in the lane), so that a
 * query's running maximum and sum are its lane's own and the exponentials are, as they lie, the second operand of o^T += v^T p^T. */
template <class E, int DP> __global__ __launch_bounds__(WAVES * 64, 2) void k_attention(Attention a) {
  using R = Rows<DP>;
  __shared__ __attribute__((aligned(1024))) char mem[4 * R::BYTES];
  __shared__ int part[WAVES][2];
  lds_char *lds = (lds_char *)mem;
  int tile, h, b;
  place((a.Sq + ROWS - 1) / ROWS, a.H, tile, h, b);
  int g = h / (a.H / a.G);
  int wave = uniform(threadIdx.x / 64), l = lane(), half = l >> 5;
  int i = tile * ROWS + wave * 32 + (l & 31), offset = a.Sk - a.Sq;
  int begin, end;
  key_range(a, b, i, begin, end);
  int wlo = wave_min(begin), whi = wave_max(end), full_lo = wave_max(begin), full_hi = wave_min(end);
  int lo = wlo, hi = whi;
  join_ranges(lo, hi, part);

  typename Vec<E>::v8 q[DP / 16];
  row_fragments<E, DP>(a.q, b * a.q.batch + h * a.q.head, i, begin < end, a.D, q);
  f32x16 acc[DP / 32];
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r++) acc[t][r] = 0;
  float top = -INFINITY, sum = 0;
  bool plain = !(a.cap > 0) && !a.slopes;
  float slope2 = a.slopes ? a.slopes[h] * LOG2E : 0.f, c = plain ? a.scale * LOG2E : 1.f;

  R rk, rv;
  rk.init(a.k.row, a.D);
  rv.init(a.v.row, a.D);
  const char *pk = a.k.p + b * a.k.batch + g * a.k.head, *pv = a.v.p + b * a.v.batch + g * a.v.head;
  int first = lo / KT, last = lo < hi ? (hi + KT - 1) / KT : first;
  if (first < last) {
    rk.load(pk, a.k.row, lds, first * KT, lo, hi);
    rv.load(pv, a.v.row, lds + R::BYTES, first * KT, lo, hi);
  }
  for (int t = first; t < last; t++) {
    wait_barrier();
    lds_char *K = lds + (t - first) % 2 * 2 * R::BYTES, *V = K + R::BYTES;
    if (t + 1 < last) {
      lds_char *next = lds + (t + 1 - first) % 2 * 2 * R::BYTES;
      rk.load(pk, a.k.row, next, (t + 1) * KT, lo, hi);
      rv.load(pv, a.v.row, next + R::BYTES, (t + 1) * KT, lo, hi);
    }
    int j0 = t * KT;
    if (j0 >= whi || j0 + KT <= wlo) continue;
    f32x16 s[2];
#pragma unroll
    for (int x = 0; x < 2; x++) {
      for (int r = 0; r < 16; r++) s[x][r] = 0;
#pragma unroll
      for (int d = 0; d < DP / 16; d++) s[x] = mfma(straight<E, DP>(K, 32 * x, d), q[d], s[x]);
    }
    if (!plain)
      for (int x = 0; x < 2; x++)
        for (int r = 0; r < 16; r++) s[x][r] = score(a, slope2, s[x][r], i + offset - (j0 + 32 * x + 8 * (r >> 2) + 4 * half + (r & 3)));
    if (j0 < full_lo || j0 + KT > full_hi)
      for (int x = 0; x < 2; x++)
        for (int r = 0; r < 16; r++) {
          int j = j0 + 32 * x + 8 * (r >> 2) + 4 * half + (r & 3);
          s[x][r] = j >= begin && j < end ? s[x][r] : -INFINITY;
        }
    float m = fmaxf(s[0][0], s[1][0]);
    for (int r = 1; r < 16; r++) m = fmaxf(m, fmaxf(s[0][r], s[1][r]));
    m = fmaxf(m, __shfl_xor(m, 32)) * c;
    /* The exponents' origin follows the maximum only when it has risen by 8: what was summed before is then scaled, and no
     * exponential passes 2^8. */
    if (__any(m > top + 8)) {
      float to = fmaxf(m, top), by = to == -INFINITY ? 1.f : exp2_(top - to);
      sum *= by;
      for (int d = 0; d < DP / 32; d++)
        for (int r = 0; r < 16; r++) acc[d][r] *= by;
      top = to;
    }
    float from = top == -INFINITY ? 0.f : top;
    float p[2][16];
    for (int x = 0; x < 2; x++)
      for (int r = 0; r < 16; r++) {
        p[x][r] = exp2_(s[x][r] * c - from);
        sum += p[x][r];
      }
#pragma unroll
    for (int x = 0; x < 2; x++)
#pragma unroll
      for (int k = 0; k < 2; k++) {
        typename Vec<E>::v8 w = round8<E>(p[x] + 8 * k);
#pragma unroll
        for (int d = 0; d < DP / 32; d++) acc[d] = mfma(transposed<E, DP>(V, 32 * x + 16 * k, 32 * d), w, acc[d]);
      }
  }
  sum += __shfl_xor(sum, 32);
  if (i < a.Sq) {
    store_column<E, DP>(acc, sum > 0 ? 1 / sum : (sum == 0 ? 0.f : sum), (char *)a.o.p + b * a.o.batch + h * a.o.head + i * a.o.row, a.D);
    if (a.lse && half == 0) a.lse[((int64_t)b * a.H + h) * a.Sq + i] = sum == 0 ? -INFINITY : (top + __builtin_amdgcn_logf(sum)) * LN2;
  }
}

/* ---- backward --------------------------------------------------------------------------------------------------------------- */
/* delta = do . o: 16 lanes a row, eight values each. */
template <class E> __global__ __launch_bounds__(256) void k_delta(Attention a, float *delta) {
  int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16, rows = (int64_t)a.B * a.H * a.Sq;
  if (row >= rows) return;
  int i = (int)(row % a.Sq), h = (int)(row / a.Sq % a.H), b = (int)(row / a.Sq / a.H), d = threadIdx.x % 16 * 8;
  float s = 0;
  typename Vec<E>::v8 x = load8<E>((const E *)(a.dout.p + b * a.dout.batch + h * a.dout.head + i * a.dout.row) + d, a.D - d);
  typename Vec<E>::v8 y = load8<E>((const E *)(a.o.p + b * a.o.batch + h * a.o.head + i * a.o.row) + d, a.D - d);
  for (int e = 0; e < 8; e++) s += (float)x[e] * (float)y[e];
  for (int k = 8; k > 0; k >>= 1) s += __shfl_xor(s, k);
  if (d == 0) delta[row] = s;
}

__global__ __launch_bounds__(64) void k_ranges(Attention a, int4 *ranges) {
  int tiles = (a.Sq + KT - 1) / KT, b = blockIdx.x / tiles, t = blockIdx.x % tiles;
  int begin, end;
  key_range(a, b, t * KT + (int)threadIdx.x, begin, end);
  int lo = wave_min(begin), hi = wave_max(end), flo = wave_max(begin), fhi = wave_min(end);
  if (threadIdx.x == 0) ranges[blockIdx.x] = make_int4(lo, hi, flo, fhi);
}

/* What a pair (query, key) gives: p = e^(s - lse) and ds = p (dp - delta) ds/draw, both 0 where the key is not seen. */
__device__ inline void pair(const Attention &a, bool plain, float c, float slope2, bool seen, int distance, float lse2, float delta, float raw, float dp,
                            float &p, float &ds) {
  float by = a.scale, e = raw * c;
  if (!plain) {
    float s = raw * a.scale;
    if (a.cap > 0) {
      float t = tanh_(s / a.cap);
      s = a.cap * t;
      by *= 1 - t * t;
    }
    e = s * LOG2E - slope2 * abs(distance);
  }
  p = exp2_(e - lse2);
  ds = p * (dp - delta) * by;
  p = seen ? p : 0.f;
  ds = seen ? ds : 0.f;
}

/* dq: as in the forward pass a wave has 32 queries, one a lane pair; dp^T = v do^T beside s^T = k q^T, then dq^T += k^T ds^T. */
template <class E, int DP> __global__ __launch_bounds__(WAVES * 64, 2) void k_attention_dq(Attention a) {
  using R = Rows<DP>;
  __shared__ __attribute__((aligned(1024))) char mem[4 * R::BYTES];
  __shared__ int part[WAVES][2];
  lds_char *lds = (lds_char *)mem;
  int tile, h, b;
  place((a.Sq + ROWS - 1) / ROWS, a.H, tile, h, b);
  int g = h / (a.H / a.G);
  int wave = uniform(threadIdx.x / 64), l = lane(), half = l >> 5;
  int i = tile * ROWS + wave * 32 + (l & 31), offset = a.Sk - a.Sq;
  int begin, end;
  key_range(a, b, i, begin, end);
  int wlo = wave_min(begin), whi = wave_max(end), full_lo = wave_max(begin), full_hi = wave_min(end);
  int lo = wlo, hi = whi;
  join_ranges(lo, hi, part);

  typename Vec<E>::v8 q[DP / 16], dout[DP / 16];
  row_fragments<E, DP>(a.q, b * a.q.batch + h * a.q.head, i, begin < end, a.D, q);
  row_fragments<E, DP>(a.dout, b * a.dout.batch + h * a.dout.head, i, begin < end, a.D, dout);
  float lse2 = 0, delta = 0;
  if (begin < end) {
    int64_t at = ((int64_t)b * a.H + h) * a.Sq + i;
    lse2 = a.lse[at] * LOG2E, delta = a.delta[at];
  }
  f32x16 acc[DP / 32];
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r++) acc[t][r] = 0;
  bool plain = !(a.cap > 0) && !a.slopes;
  float slope2 = a.slopes ? a.slopes[h] * LOG2E : 0.f, c = a.scale * LOG2E;

  R rk, rv;
  rk.init(a.k.row, a.D);
  rv.init(a.v.row, a.D);
  const char *pk = a.k.p + b * a.k.batch + g * a.k.head, *pv = a.v.p + b * a.v.batch + g * a.v.head;
  int first = lo / KT, last = lo < hi ? (hi + KT - 1) / KT : first;
  if (first < last) {
    rk.load(pk, a.k.row, lds, first * KT, lo, hi);
    rv.load(pv, a.v.row, lds + R::BYTES, first * KT, lo, hi);
  }
  for (int t = first; t < last; t++) {
    wait_barrier();
    lds_char *K = lds + (t - first) % 2 * 2 * R::BYTES, *V = K + R::BYTES;
    if (t + 1 < last) {
      lds_char *next = lds + (t + 1 - first) % 2 * 2 * R::BYTES;
      rk.load(pk, a.k.row, next, (t + 1) * KT, lo, hi);
      rv.load(pv, a.v.row, next + R::BYTES, (t + 1) * KT, lo, hi);
    }
    int j0 = t * KT;
    if (j0 >= whi || j0 + KT <= wlo) continue;
    bool all = j0 >= full_lo && j0 + KT <= full_hi;
#pragma unroll
    for (int x = 0; x < 2; x++) {
      f32x16 s, dp;
      for (int r = 0; r < 16; r++) s[r] = dp[r] = 0;
#pragma unroll
      for (int d = 0; d < DP / 16; d++) {
        s = mfma(straight<E, DP>(K, 32 * x, d), q[d], s);
        dp = mfma(straight<E, DP>(V, 32 * x, d), dout[d], dp);
      }
      float ds[16];
      for (int r = 0; r < 16; r++) {
        int j = j0 + 32 * x + 8 * (r >> 2) + 4 * half + (r & 3);
        float p;
        pair(a, plain, c, slope2, all || (j >= begin && j < end), i + offset - j, lse2, delta, s[r], dp[r], p, ds[r]);
      }
#pragma unroll
      for (int k = 0; k < 2; k++) {
        typename Vec<E>::v8 w = round8<E>(ds + 8 * k);
#pragma unroll
        for (int d = 0; d < DP / 32; d++) acc[d] = mfma(transposed<E, DP>(K, 32 * x + 16 * k, 32 * d), w, acc[d]);
      }
    }
  }
  if (i < a.Sq) store_column<E, DP>(acc, 1.f, (char *)a.dq.p + b * a.dq.batch + h * a.dq.head + i * a.dq.row, a.D);
}

/* dk, dv: a wave has 32 keys, one a lane pair, and meets all queries that see them, of every head that shares them, 64 at a time:
 * s = q k^T and dp = do v^T (queries in the registers), then dv^T += do^T p and dk^T += q^T ds. */
template <class E, int DP> __global__ __launch_bounds__(WAVES * 64, DP == 128 ? 1 : 2) void k_attention_dkv(Attention a) {
  using R = Rows<DP>;
  __shared__ __attribute__((aligned(1024))) char mem[4 * R::BYTES];
  __shared__ __attribute__((aligned(16))) float row_lse[2][KT], row_delta[2][KT];
  __shared__ __attribute__((aligned(16))) int row_begin[2][KT], row_end[2][KT];
  lds_char *lds = (lds_char *)mem;
  int tiles = (a.Sq + KT - 1) / KT, tile, g, b;
  place((a.Sk + ROWS - 1) / ROWS, a.G, tile, g, b);
  int wave = uniform(threadIdx.x / 64), l = lane(), half = l >> 5;
  int k0 = tile * ROWS, w0 = k0 + wave * 32, j = w0 + (l & 31), offset = a.Sk - a.Sq, shared = a.H / a.G;

  typename Vec<E>::v8 k[DP / 16], v[DP / 16];
  row_fragments<E, DP>(a.k, b * a.k.batch + g * a.k.head, j, j < a.Sk, a.D, k);
  row_fragments<E, DP>(a.v, b * a.v.batch + g * a.v.head, j, j < a.Sk, a.D, v);
  f32x16 dk[DP / 32], dv[DP / 32];
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r++) dk[t][r] = dv[t][r] = 0;
  bool plain = !(a.cap > 0) && !a.slopes;
  float c = a.scale * LOG2E;
  R rq, rd;
  rq.init(a.q.row, a.D);
  rd.init(a.dout.row, a.D);

  /* (head of the group, tile of queries) pairs in order, those that see none of the workgroup's keys left out */
  const int4 *ranges = a.ranges + (int64_t)b * tiles;
  auto next = [&](int at) {
    for (at++; at < shared * tiles; at++) {
      int4 r = ranges[at % tiles];
      if (r.x < k0 + ROWS && r.y > k0) break;
    }
    return at;
  };
  float in_lse = 0, in_delta = 0;
  int in_begin = FAR, in_end = 0;
  auto ask = [&](int at, int which) { /* rows that see nothing are zeros, whatever they hold */
    int h = g * shared + at / tiles, i0 = at % tiles * KT;
    lds_char *to = lds + which * 2 * R::BYTES;
    const char *pq = a.q.p + b * a.q.batch + h * a.q.head, *pd = a.dout.p + b * a.dout.batch + h * a.dout.head;
    if (ranges[at % tiles].z == FAR) { /* some row of the tile sees nothing, or there is none */
      __amdgpu_buffer_rsrc_t bq = buffer(pq + (int64_t)i0 * a.q.row), bd = buffer(pd + (int64_t)i0 * a.dout.row);
      for (int n = 0; n < R::LOADS; n++) {
        int lo, hi;
        key_range(a, b, i0 + rq.row[n], lo, hi);
        lds_char *place = to + (n * WAVES * 64 + wave * 64) * 16;
        load_lds(bq, place, lo < hi ? rq.off[n] : OOB_LAYER_OUT);
        load_lds(bd, place + R::BYTES, lo < hi ? rd.off[n] : OOB_LAYER_OUT);
      }
    } else {
      rq.load(pq, a.q.row, to, i0, 0, a.Sq);
      rd.load(pd, a.dout.row, to + R::BYTES, i0, 0, a.Sq);
    }
    if (threadIdx.x < KT) {
      int i = i0 + threadIdx.x;
      key_range(a, b, i, in_begin, in_end);
      in_lse = in_delta = 0;
      if (in_begin < in_end) {
        int64_t row = ((int64_t)b * a.H + h) * a.Sq + i;
        in_lse = a.lse[row] * LOG2E, in_delta = a.delta[row];
      }
    }
  };
  auto put = [&](int which) {
    if (threadIdx.x < KT) {
      row_lse[which][threadIdx.x] = in_lse, row_delta[which][threadIdx.x] = in_delta;
      row_begin[which][threadIdx.x] = in_begin, row_end[which][threadIdx.x] = in_end;
    }
  };

  int at = next(-1), buf = 0;
  if (at < shared * tiles) ask(at, 0);
  while (at < shared * tiles) {
    put(buf);
    __builtin_amdgcn_s_waitcnt(0xc07f); /* lgkmcnt(0): the row's numbers are in LDS */
    wait_barrier();
    int then = next(at);
    if (then < shared * tiles) ask(then, buf ^ 1);
    lds_char *Q = lds + buf * 2 * R::BYTES, *D = Q + R::BYTES;
    int4 range = ranges[at % tiles];
    int i0 = at % tiles * KT;
    float slope2 = a.slopes ? a.slopes[g * shared + at / tiles] * LOG2E : 0.f;
    if (w0 < range.y && w0 + 32 > range.x) {
      bool all = w0 >= range.z && w0 + 32 <= range.w;
#pragma unroll
      for (int x = 0; x < 2; x++) {
        f32x16 s, dp;
        for (int r = 0; r < 16; r++) s[r] = dp[r] = 0;
#pragma unroll
        for (int d = 0; d < DP / 16; d++) {
          s = mfma(straight<E, DP>(Q, 32 * x, d), k[d], s);
          dp = mfma(straight<E, DP>(D, 32 * x, d), v[d], dp);
        }
        float p[16], ds[16];
#pragma unroll
        for (int n = 0; n < 4; n++) {
          int row = 32 * x + 8 * n + 4 * half;
          float4 lse = *(const float4 *)(row_lse[buf] + row), delta = *(const float4 *)(row_delta[buf] + row);
          int4 lo = *(const int4 *)(row_begin[buf] + row), hi = *(const int4 *)(row_end[buf] + row);
          const float *pl = &lse.x, *pd = &delta.x;
          const int *pb = &lo.x, *pe = &hi.x;
#pragma unroll
          for (int e = 0; e < 4; e++)
            pair(a, plain, c, slope2, all || (j >= pb[e] && j < pe[e]), i0 + row + e + offset - j, pl[e], pd[e], s[4 * n + e], dp[4 * n + e], p[4 * n + e], ds[4 * n + e]);
        }
#pragma unroll
        for (int m = 0; m < 2; m++) {
          typename Vec<E>::v8 wp = round8<E>(p + 8 * m), ws = round8<E>(ds + 8 * m);
#pragma unroll
          for (int d = 0; d < DP / 32; d++) {
            dv[d] = mfma(transposed<E, DP>(D, 32 * x + 16 * m, 32 * d), wp, dv[d]);
            dk[d] = mfma(transposed<E, DP>(Q, 32 * x + 16 * m, 32 * d), ws, dk[d]);
          }
        }
      }
    }
    at = then, buf ^= 1;
  }
  if (j < a.Sk) {
    store_column<E, DP>(dk, 1.f, (char *)a.dk.p + b * a.dk.batch + g * a.dk.head + j * a.dk.row, a.D);
    store_column<E, DP>(dv, 1.f, (char *)a.dv.p + b * a.dv.batch + g * a.dv.head + j * a.dv.row, a.D);
  }
}

/* ---- heads that the loads cannot take (rows that do not start at 16 bytes, a width that is no multiple of 8) go to the workspace ---- */
struct PackHeads { Heads from; uint16_t *to; int B, S, N, D, ld; };
__global__ __launch_bounds__(256) void k_pack_heads(PackHeads p) {
  int per = p.ld / 8;
  int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, row = id / per;
  int c = (int)(id % per) * 8;
  if (row >= (int64_t)p.B * p.S * p.N) return;
  int n = (int)(row % p.N), s = (int)(row / p.N % p.S), b = (int)(row / p.N / p.S);
  const uint16_t *from = (const uint16_t *)(p.from.p + b * p.from.batch + s * p.from.row + n * p.from.head);
  i16x8 v;
  for (int e = 0; e < 8; e++) v[e] = c + e < p.D ? (short)from[c + e] : (short)0;
  *(i16x8 *)(p.to + row * p.ld + c) = v;
}

static Heads heads_of(const void *p, const int64_t (&stride)[3]) { return {(const char *)p, stride[0] * 2, stride[1] * 2, stride[2] * 2}; }

static bool loadable(const Heads &h, int D) {
  return D % 8 == 0 && multiple(h.p, 16) && h.batch % 16 == 0 && h.row % 16 == 0 && h.head % 16 == 0 && h.row < (1 << 24);
}
static size_t packed_bytes(int B, int S, int N, int D) { return (size_t)B * S * N * up(D, 8) * 2; }

static void pack(Heads &h, int B, int S, int N, int D, Arena &w, hipStream_t st) {
  if (loadable(h, D)) return;
  int ld = (int)up(D, 8);
  void *to = w.take(packed_bytes(B, S, N, D));
  int64_t n = (int64_t)B * S * N * (ld / 8);
  if (w.ok() && n) k_pack_heads<<<(unsigned)((n + 255) / 256), 256, 0, st>>>({h, (uint16_t *)to, B, S, N, D, ld});
  h = {(const char *)to, (int64_t)S * N * ld * 2, (int64_t)N * ld * 2, (int64_t)ld * 2};
}

static bool attention_ok(const oob_attention *p) {
  if ((p->dtype != OOB_BF16 && p->dtype != OOB_FP16) || p->B < 0 || p->Sq < 0 || p->Sk < 0 || p->H < 1 || p->G < 1 || p->H % p->G != 0) return false;
  if (p->D < 1 || p->D > OOB_ATTENTION_MAX_D || p->Sq >= (1 << 29) || p->Sk >= (1 << 29)) return false;
  if (!(p->scale > 0) || !(p->cap >= 0) || !(p->scale < INFINITY) || !(p->cap < INFINITY)) return false;
  int64_t wgs = (int64_t)p->B * p->H * ((p->Sq > p->Sk ? p->Sq : p->Sk) / 16 + 1);
  if (wgs >= ((int64_t)1 << 31)) return false;
  for (const int64_t(*s)[3] : {&p->q_stride, &p->k_stride, &p->v_stride, &p->o_stride})
    for (int i = 0; i < 3; i++)
      if ((*s)[i] < 0) return false;
  for (const void *q : {p->q, p->k, p->v, (const void *)p->o})
    if (!multiple(q, 2)) return false;
  return multiple(p->key_begin, 4) && multiple(p->key_end, 4) && multiple(p->slopes, 4) && multiple(p->lse, 4);
}

static Attention attention_of(const oob_attention *p) {
  Attention a{};
  a.q = heads_of(p->q, p->q_stride), a.k = heads_of(p->k, p->k_stride), a.v = heads_of(p->v, p->v_stride), a.o = heads_of(p->o, p->o_stride);
  a.begin = p->key_begin, a.end = p->key_end, a.slopes = p->slopes, a.lse = p->lse;
  a.B = p->B, a.Sq = p->Sq, a.Sk = p->Sk, a.H = p->H, a.G = p->G, a.D = p->D;
  a.causal = p->causal != 0, a.scale = p->scale, a.cap = p->cap;
  return a;
}

static size_t forward_bytes(const oob_attention *p) {
  Attention a = attention_of(p);
  Arena w{nullptr, 0, 0};
  for (const Heads &h : {a.k, a.v})
    if (!loadable(h, a.D)) w.take(packed_bytes(a.B, a.Sk, a.G, a.D));
  return w.used;
}

template <class E> static int forward(const oob_attention *p, Arena w, hipStream_t st) {
  Attention a = attention_of(p);
  pack(a.k, a.B, a.Sk, a.G, a.D, w, st);
  pack(a.v, a.B, a.Sk, a.G, a.D, w, st);
  if (!w.ok()) return OOB_ECAPACITY;
  unsigned n = (unsigned)((int64_t)a.B * a.H * ((a.Sq + ROWS - 1) / ROWS));
  if (n) {
    if (a.D <= 64) k_attention<E, 64><<<n, WAVES * 64, 0, st>>>(a);
    else k_attention<E, 128><<<n, WAVES * 64, 0, st>>>(a);
  }
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

static size_t backward_bytes(const oob_attention *p, const oob_attention_grad *q) {
  Attention a = attention_of(p);
  Arena w{nullptr, 0, 0};
  w.take((size_t)a.B * a.H * a.Sq * 4);
  w.take((size_t)a.B * ((a.Sq + KT - 1) / KT) * sizeof(int4));
  for (const Heads &h : {a.k, a.v})
    if (!loadable(h, a.D)) w.take(packed_bytes(a.B, a.Sk, a.G, a.D));
  for (const Heads &h : {a.q, heads_of(q->dout, q->dout_stride)})
    if (!loadable(h, a.D)) w.take(packed_bytes(a.B, a.Sq, a.H, a.D));
  return w.used;
}

template <class E> static int backward(const oob_attention *p, const oob_attention_grad *q, Arena w, hipStream_t st) {
  Attention a = attention_of(p);
  a.dout = heads_of(q->dout, q->dout_stride);
  a.dq = heads_of(q->dq, q->dq_stride), a.dk = heads_of(q->dk, q->dk_stride), a.dv = heads_of(q->dv, q->dv_stride);
  float *delta = (float *)w.take((size_t)a.B * a.H * a.Sq * 4);
  int4 *ranges = (int4 *)w.take((size_t)a.B * ((a.Sq + KT - 1) / KT) * sizeof(int4));
  a.delta = delta, a.ranges = ranges;
  if (!w.ok()) return OOB_ECAPACITY;
  int64_t rows = (int64_t)a.B * a.H * a.Sq;
  if (rows) {
    k_delta<E><<<(unsigned)((rows + 15) / 16), 256, 0, st>>>(a, delta);
    k_ranges<<<(unsigned)(a.B * ((a.Sq + KT - 1) / KT)), 64, 0, st>>>(a, ranges);
  }
  pack(a.k, a.B, a.Sk, a.G, a.D, w, st);
  pack(a.v, a.B, a.Sk, a.G, a.D, w, st);
  pack(a.q, a.B, a.Sq, a.H, a.D, w, st);
  pack(a.dout, a.B, a.Sq, a.H, a.D, w, st);
  if (!w.ok()) return OOB_ECAPACITY;
  unsigned nq = (unsigned)((int64_t)a.B * a.H * ((a.Sq + ROWS - 1) / ROWS)), nk = (unsigned)((int64_t)a.B * a.G * ((a.Sk + ROWS - 1) / ROWS));
  if (nk) {
    if (a.D <= 64) k_attention_dkv<E, 64><<<nk, WAVES * 64, 0, st>>>(a);
    else k_attention_dkv<E, 128><<<nk, WAVES * 64, 0, st>>>(a);
  }
  if (nq) {
    if (a.D <= 64) k_attention_dq<E, 64><<<nq, WAVES * 64, 0, st>>>(a);
    else k_attention_dq<E, 128><<<nq, WAVES * 64, 0, st>>>(a);
  }
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

static bool grads_ok(const oob_attention *p, const oob_attention_grad *q) {
  for (const int64_t(*s)[3] : {&q->dout_stride, &q->dq_stride, &q->dk_stride, &q->dv_stride})
    for (int i = 0; i < 3; i++)
      if ((*s)[i] < 0) return false;
  for (const void *x : {q->dout, (const void *)q->dq, (const void *)q->dk, (const void *)q->dv})
    if (!multiple(x, 2)) return false;
  if (p->B > 0 && p->Sq > 0 && (!p->q || !p->o || !p->lse || !q->dout || !q->dq)) return false;
  return !(p->B > 0 && p->Sk > 0 && (!p->k || !p->v || !q->dk || !q->dv));
}

}  // namespace layer

using namespace layer;

extern "C" size_t oob_layer_attention_workspace_size(const oob_attention *p) { return p && attention_ok(p) ? forward_bytes(p) : 0; }

extern "C" int oob_layer_attention(const oob_attention *p, void *workspace, size_t bytes, void *stream) {
  if (!p || !attention_ok(p) || !multiple(workspace, 256)) return OOB_EINVAL;
  if (p->B == 0 || p->Sq == 0) return OOB_OK;
  if (!p->q || !p->o || (p->Sk > 0 && (!p->k || !p->v))) return OOB_EINVAL;
  size_t need = forward_bytes(p);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? forward<bf16>(p, w, (hipStream_t)stream) : forward<fp16>(p, w, (hipStream_t)stream);
}

extern "C" size_t oob_layer_attention_backward_workspace_size(const oob_attention *p, const oob_attention_grad *q) {
  return p && q && attention_ok(p) && grads_ok(p, q) ? backward_bytes(p, q) : 0;
}

extern "C" int oob_layer_attention_backward(const oob_attention *p, const oob_attention_grad *q, void *workspace, size_t bytes, void *stream) {
  if (!p || !q || !attention_ok(p) || !grads_ok(p, q) || !multiple(workspace, 256)) return OOB_EINVAL;
  if (p->B == 0) return OOB_OK;
  size_t need = backward_bytes(p, q);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? backward<bf16>(p, q, w, (hipStream_t)stream) : backward<fp16>(p, q, w, (hipStream_t)stream);
}
