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
  const float *lse2, *delta; /* [B][H][Sq]: lse log2 e (0 where there is none), do . o */
  float *parts;              /* [2][H / G][B][Sk][G][D] or null: dk and dv of every head for itself, where they are shared and workgroups are few */
  const int4 *ranges;  /* [B][tiles of grad_tile queries]: smallest begin, largest end, largest begin, smallest end */
};

/* A workgroup is two teams of four waves on the same 128 rows (queries; keys in dk, dv): 32 rows a wave, the other side's tiles dealt to
 * the teams in turn, and what the teams have summed joined at the end.  The teams take turns at the matrix cores as well: a step is a phase
 * of matrix products and a phase of exponentials, a barrier behind each, and one team is a phase behind the other, so that each SIMD has
 * one wave in either phase.  (Waves w and w + 4 share a SIMD.) */
constexpr int TEAM = 256, THREADS = 2 * TEAM, ROWS = 128;
constexpr int KT = 64; /* keys of a tile in the forward pass */
constexpr int grad_tile(int DP) { return DP == 64 ? 64 : 32; } /* rows of a tile in the backward pass: what its products leave registers for */
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

/* N rows of a head on their way to a team's LDS, 16 (DP 128) or 32 rows a load: rows that far apart have the same swizzle, so that a lane
 * has one offset and the loads differ by a scalar.  Every load is issued, whether or not there are such rows: the waits count loads. */
template <int DP, int N> struct Rows {
  static constexpr int BYTES = N * DP * 2, LOADS = BYTES / (TEAM * 16), STEP = N / LOADS;
  uint32_t off;
  int row;
  __device__ void init(int64_t stride, int D) {
    int p = threadIdx.x % TEAM * 16, c = (p / 16 % (DP / 8)) ^ swizzle<DP>(p / (DP * 2));
    row = p / (DP * 2);
    off = c * 8 < D ? (uint32_t)(row * stride + c * 16) : OOB_LAYER_OUT;
  }
  /* rows lo <= first + r < hi; zeros for the others */
  __device__ void load(const char *base, int64_t stride, lds_char *to, int first, int lo, int hi) {
    if (first >= lo && first + N <= hi) load(base, stride, to, first, [](int) { return true; });
    else load(base, stride, to, first, [&](int at) { return at >= lo && at < hi; });
  }
  template <class F> __device__ void load(const char *base, int64_t stride, lds_char *to, int first, F in) {
    __amdgpu_buffer_rsrc_t r = buffer(base + first * stride);
    int wave = uniform(threadIdx.x % TEAM / 64);
#pragma unroll
    for (int i = 0; i < LOADS; i++)
      load_lds(r, to + (i * TEAM + wave * 64) * 16, in(first + row + i * STEP) ? off : OOB_LAYER_OUT, (uint32_t)(i * STEP * stride));
  }
};

/* A lane's places in a tile: everything else about an address is a constant, so that reads need no arithmetic.
 * Straight fragments: row r0 + l % 32, columns 16 t + 8 (l / 32) .. + 7.  Transposed: column d0 + l % 32, rows r0 + 4 (l / 32) .. + 3 and
 * r0 + 8 + 4 (l / 32) .. + 3: the rows whose values of a product a lane holds in eight registers in a row, so that those are the other
 * operand as they are.  (r0: a multiple of 32 and of 16; the swizzle of row r + 8 is that of row r with one bit flipped.) */
template <class E, int DP> struct Places {
  int s[DP / 16], t[DP / 32];
  __device__ void init() {
    int l = lane(), r = l & 31;
    for (int i = 0; i < DP / 16; i++) s[i] = r * DP * 2 + ((2 * i + (l >> 5)) ^ swizzle<DP>(r)) * 16;
    r = 4 * (l >> 5) + ((l & 15) >> 2);
    for (int i = 0; i < DP / 32; i++) t[i] = r * DP * 2 + ((4 * i + ((l >> 4) & 1) * 2 + ((l >> 1) & 1)) ^ swizzle<DP>(r)) * 16 + (l & 1) * 8;
  }
  __device__ typename Vec<E>::v8 straight(lds_char *lds, int tile, int r0, int i) const { return lds_read8<E>(lds + s[i] + (tile + r0 * DP * 2)); }
  __device__ typename Vec<E>::v8 transposed(lds_char *lds, int tile, int r0, int i) const {
    static_assert(DP == 64 || DP == 128, "rows 8 apart differ in bit 1 of the swizzle");
    return lds_read_tr<E>(lds + t[i] + (tile + r0 * DP * 2), lds + (t[i] ^ 32) + (tile + (r0 + 8) * DP * 2));
  }
};

/* The same in two registers: a chunk's number enters its place by exclusive or, so that every place is one such step from the first.
 * fresh() keeps the compiler from holding them all. */
template <class E, int DP> struct FewPlaces {
  int s, t;
  __device__ void init() {
    Places<E, DP> p;
    p.init();
    s = p.s[0], t = p.t[0];
  }
  __device__ void fresh() { asm volatile("" : "+v"(s), "+v"(t)); }
  __device__ typename Vec<E>::v8 straight(lds_char *lds, int tile, int r0, int i) const { return lds_read8<E>(lds + (s ^ 32 * i) + (tile + r0 * DP * 2)); }
  __device__ typename Vec<E>::v8 transposed(lds_char *lds, int tile, int r0, int i) const {
    return lds_read_tr<E>(lds + (t ^ 64 * i) + (tile + r0 * DP * 2), lds + (t ^ 64 * i ^ 32) + (tile + (r0 + 8) * DP * 2));
  }
};

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
  typedef typename Vec<E>::v4 v4 __attribute__((aligned(sizeof(E))));
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

template <int N> struct Int { static constexpr int value = N; };
__device__ inline float max3(float a, float b, float c) { return __builtin_elementwise_maximum(__builtin_elementwise_maximum(a, b), c); }
/* The larger of lanes l and l ^ 32. */
__device__ inline float max_halves(float x) {
  float y = __shfl_xor(x, 32);
  return max3(x, y, y);
}
__device__ inline float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float tanh_(float x) { return 1 - 2 * __builtin_amdgcn_rcpf(1 + exp2_(x * (2 * LOG2E))); }

/* Kinds of scores: the scale alone (folded into the exponent), capped, with a bias, both. */
constexpr int CAP = 1, BIAS = 2;

/* Of a raw product: the score times log2 e, and dscore / draw over the scale, where wanted. */
template <int KIND> __device__ inline float score(const Attention &a, float slope2, float raw, int distance, float &by) {
  by = 1;
  float s = raw * (a.scale * LOG2E);
  if (KIND & CAP) {
    float t = tanh_(raw * (a.scale / a.cap));
    s = a.cap * LOG2E * t;
    by = 1 - t * t;
  }
  if (KIND & BIAS) s -= slope2 * (float)abs(distance);
  return s;
}

/* Barriers between phases: what a wave has read from LDS before, nobody writes until all are behind.  Not a fence, which would wait for
 * the loads in flight too; nothing is moved from one phase to another, arithmetic neither. */
__device__ inline void phase() {
  __builtin_amdgcn_sched_barrier(0);
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
/* All but the last N loads of the wave have landed (N < 16). */
template <int N> __device__ inline void landed() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }

/* The smallest begin and largest end over the rows (each team has them all). */
__device__ inline void join_ranges(int &lo, int &hi, int (*part)[2]) {
  int wave = threadIdx.x / 64;
  if (lane() == 0) part[wave][0] = lo, part[wave][1] = hi;
  __syncthreads();
  for (int w = 0; w < 4; w++) lo = min(lo, part[w][0]), hi = max(hi, part[w][1]);
  lo = uniform(lo), hi = uniform(hi);
}

/* The ranges of a workgroup's queries may leave keys between the first and the last that none of them sees (padding between documents,
 * say).  Those are read as zeros: 0 times what they hold need not be 0.  Ranges that all begin with the first key or all end with the last
 * leave none, nor do those of which each touches that of the query before; only for others the tiles are looked at (2 x 4096 tokens, 16 heads
 * of 128, documents of 360 padded to 384: 75 to 76 us forward, 209 to 210 backward; of 60 to 64: 69 to 74 and 197 to 204; without holes the
 * question takes 1 us of a call: 4096 tokens, 12 heads of 64, a window of 512: 28.4 to 29.8). */
struct Holes { int2 of[ROWS]; int any[8]; };

/* Before join_ranges, whose barrier this needs. */
__device__ inline void note_ranges(const Attention &a, int b, int i, int begin, int end, Holes &holes) {
  bool apart = false;
  int row = i % ROWS;
  if (a.begin && (a.end || a.causal)) {
    if (row > 0 && begin < end) {
      int begin0, end0; /* none: FAR, 0 touches nothing */
      key_range(a, b, i - 1, begin0, end0);
      apart = begin0 > end || begin > end0;
    }
    holes.of[row] = make_int2(begin, end); /* by both teams, the same */
  }
  bool any = __any(apart);
  if (lane() == 0) holes.any[threadIdx.x / 64] = any;
}
__device__ inline bool has_holes(const Holes &holes) {
  int any = 0;
  for (int w = 0; w < 4; w++) any |= holes.any[w];
  return uniform(any);
}

/* Which of the keys first .. first + N - 1 (N up to 64) some query of the workgroup sees, bit by bit. */
template <int N> __device__ inline uint64_t seen_keys(const Holes &holes, int first) {
  uint64_t seen = 0;
  for (int r = 0; r < ROWS; r += 64) {
    int2 range = holes.of[r + lane()];
    int from = max(range.x - first, 0), to = min(range.y - first, N);
    if (from < to) seen |= (~(uint64_t)0 >> (64 - (to - from))) << from;
  }
  if (__any(seen == ~(uint64_t)0 >> (64 - N))) return ~(uint64_t)0;
  for (int k = 32; k > 0; k >>= 1) seen |= (uint64_t)__shfl_xor((unsigned long long)seen, k);
  return (uint64_t)(uint32_t)uniform((int)(seen >> 32)) << 32 | (uint32_t)uniform((int)seen);
}
__device__ inline int wave_min(int v) {
  for (int k = 32; k > 0; k >>= 1) v = min(v, __shfl_xor(v, k));
  return uniform(v);
}
__device__ inline int wave_max(int v) {
  for (int k = 32; k > 0; k >>= 1) v = max(v, __shfl_xor(v, k));
  return uniform(v);
}

/* Which (tile, head, sequence) a workgroup takes: tile by tile, all heads of one tile in a row.  Workgroups are dealt to the 8 XCDs in
 * turn, so that with a multiple of 8 heads an XCD sees only its own keys and values; the tiles that see most keys where a mask is causal
 * go first (the last of queries, the first of keys), so that short ones fill up what long ones leave. */
__device__ inline void place(int heads, int B, int id, int &tile, int &head, int &b) {
  int n = heads * B;
  tile = id / n;
  head = id % n % heads;
  b = id % n / heads;
}

/* ---- forward ------------------------------------------------------------------------------------------------------------------
 * A wave has 32 queries, one a lane pair: scores are formed transposed (keys in the registers, the query in the lane), so that a
 * query's running maximum and sum are its lane's own and the exponentials are, as they lie, the second operand of o^T += v^T p^T.
 * A step's products are the scores of its tile and o^T of the tile before.
 * Bound by the matrix cores and the exponentials in turn, and in every other step by a wait of the compiler's own for all loads before the
 * reads: 75 us for 4096 tokens, 12 heads of 128, causal; without a mask and 16 heads 139 us, 0.99 PFLOP/s (14 % more with the teams in step, 6 %
 * more without the order of reads and products below). */
template <class E, int DP, int KIND> __global__ __launch_bounds__(THREADS, 2) void k_attention(Attention a) {
  using R = Rows<DP, KT>;
  __shared__ __attribute__((aligned(1024))) char mem[8 * R::BYTES];
  __shared__ int part[8][2];
  __shared__ Holes ranges;
  int wave = uniform(threadIdx.x / 64), team = wave / 4, l = lane(), half = l >> 5;
  lds_char *lds = (lds_char *)mem + team * 4 * R::BYTES; /* keys of even steps, of odd ones, values of even steps, of odd ones */
  int tile, h, b;
  place(a.H, a.B, blockIdx.x, tile, h, b);
  tile = (a.Sq + ROWS - 1) / ROWS - 1 - tile;
  int g = h / (a.H / a.G);
  int i = tile * ROWS + wave % 4 * 32 + (l & 31), offset = a.Sk - a.Sq;
  int begin, end;
  key_range(a, b, i, begin, end);
  int wlo = wave_min(begin), whi = wave_max(end), full_lo = wave_max(begin), full_hi = wave_min(end);
  int lo = wlo, hi = whi;
  note_ranges(a, b, i, begin, end, ranges);
  join_ranges(lo, hi, part);
  const bool holes = has_holes(ranges);
  int first = lo / KT, tiles = lo < hi ? (hi + KT - 1) / KT - first : 0, steps = (tiles + 1) / 2;

  typename Vec<E>::v8 q[DP / 16];
  row_fragments<E, DP>(a.q, b * a.q.batch + h * a.q.head, i, begin < end, a.D, q);
  f32x16 acc[DP / 32];
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r++) acc[t][r] = 0;
  float top = -INFINITY, sum = 0;
  float slope2 = KIND & BIAS ? a.slopes[h] * LOG2E : 0.f;
  const float c = KIND ? 1.f : a.scale * LOG2E;

  Places<E, DP> at;
  at.init();
  R rk, rv;
  rk.init(a.k.row, a.D);
  rv.init(a.v.row, a.D);
  const char *pk = a.k.p + b * a.k.batch + g * a.k.head, *pv = a.v.p + b * a.v.batch + g * a.v.head;
  auto key0 = [&](int n) __attribute__((always_inline)) { return (first + 2 * n + team) * KT; };
  auto load_k = [&](int n, int which) __attribute__((always_inline)) { rk.load(pk, a.k.row, lds + which * R::BYTES, key0(n), lo, hi); };
  auto load_v = [&](int n, int which) __attribute__((always_inline)) {
    lds_char *to = lds + (2 + which) * R::BYTES;
    int from = key0(n);
    if (holes) { /* of values alone: what a key gives a score is replaced, not multiplied */
      uint64_t seen = seen_keys<KT>(ranges, from);
      rv.load(pv, a.v.row, to, from, [&](int at) { return at < hi && (seen >> (at - from) & 1); });
    } else rv.load(pv, a.v.row, to, from, lo, hi);
  };

  f32x16 s[2];
  typename Vec<E>::v8 p[4]; /* exponentials of the step before, rounded: the second operand of its product with v */
  auto scores = [&](int K) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2; x++) {
#pragma unroll
      for (int r = 0; r < 16; r++) s[x][r] = 0;
#pragma unroll
      for (int d = 0; d < DP / 16; d++) s[x] = mfma(at.straight(lds, K, 32 * x, d), q[d], s[x]);
    }
  };
  auto outputs = [&](int V) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 4; x++)
#pragma unroll
      for (int d = 0; d < DP / 32; d++) acc[d] = mfma(at.transposed(lds, V, 16 * x, d), p[x], acc[d]);
  };
  auto exponentials = [&](int n) __attribute__((always_inline)) {
    int j0 = key0(n), j1 = j0 + 4 * half;
    if (KIND) {
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          float by;
          s[x][r] = score<KIND>(a, slope2, s[x][r], i + offset - (j1 + 32 * x + 8 * (r >> 2) + (r & 3)), by);
        }
    }
    if (j0 < full_lo || j0 + KT > full_hi) {
#pragma unroll
      for (int x = 0; x < 2; x++)
#pragma unroll
        for (int r = 0; r < 16; r++) {
          int j = j1 + 32 * x + 8 * (r >> 2) + (r & 3);
          s[x][r] = j >= begin && j < end ? s[x][r] : -INFINITY;
        }
    }
    float m = max3(s[0][0], s[0][1], s[1][0]);
#pragma unroll
    for (int r = 2; r < 16; r += 2) m = max3(m, s[0][r], s[0][r + 1]);
#pragma unroll
    for (int r = 1; r < 15; r += 2) m = max3(m, s[1][r], s[1][r + 1]);
    m = max3(m, s[1][15], s[1][15]);
    m = max_halves(m) * c;
    /* The exponents' origin follows the maximum only when it has risen by 8: what was summed before is then scaled, and no
     * exponential passes 2^8. */
    if (__any(m > top + 8)) {
      float to = m > top ? m : top, by = to == -INFINITY ? 1.f : exp2_(top - to);
      sum *= by;
#pragma unroll
      for (int d = 0; d < DP / 32; d++)
#pragma unroll
        for (int r = 0; r < 16; r++) acc[d][r] *= by;
      top = to;
    }
    float from = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int x = 0; x < 4; x++)
#pragma unroll
      for (int r = 0; r < 8; r++) {
        float e = exp2_(s[x / 2][8 * (x % 2) + r] * c - from);
        sum += e;
        p[x][r] = (E)e; /* the matrix cores take 16 bits; the sum does not see this rounding */
      }
  };
  load_k(0, 0);
  load_k(1, 1);
  load_v(0, 0);
  landed<2 * R::LOADS>();
  phase();
  if (team) phase();
  auto step = [&](int n, auto which, auto begun) __attribute__((always_inline)) {
    constexpr int W = decltype(which)::value;
    scores(W * R::BYTES);
    if (begun.value) outputs((3 - W) * R::BYTES);
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
    for (int g = 0; g < DP / 8 - 4; g++) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if (begun.value) {
#pragma unroll
      for (int g = 0; g < DP / 8; g++) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, 4, 0);
    }
    phase();
    load_k(n + 2, W);
    load_v(n + 1, W ^ 1);
    exponentials(n);
    landed<2 * R::LOADS>();
    phase();
  };
  if (steps) {
    step(0, Int<0>(), Int<0>());
    int n = 1;
    for (; n + 1 < steps; n += 2) {
      step(n, Int<1>(), Int<1>());
      step(n + 1, Int<0>(), Int<1>());
    }
    if (n < steps) step(n, Int<1>(), Int<1>());
    outputs((steps % 2 ? 2 : 3) * R::BYTES);
  }
  if (!team) phase();

  /* what the second team has, through LDS, to the first */
  sum += __shfl_xor(sum, 32);
  landed<0>();
  phase();
  __attribute__((address_space(3))) float *other = (__attribute__((address_space(3))) float *)(lds_char *)mem + wave % 4 * (DP / 2 + 2) * 64 + l;
  if (team) {
#pragma unroll
    for (int d = 0; d < DP / 32; d++)
#pragma unroll
      for (int r = 0; r < 16; r++) other[(d * 16 + r) * 64] = acc[d][r];
    other[DP / 2 * 64] = top, other[(DP / 2 + 1) * 64] = sum;
  }
  phase();
  if (team) return;
  float top1 = other[DP / 2 * 64], sum1 = other[(DP / 2 + 1) * 64];
  float to = top > top1 ? top : top1, by = to == -INFINITY ? 1.f : exp2_(top - to), by1 = to == -INFINITY ? 1.f : exp2_(top1 - to);
  sum = sum * by + sum1 * by1;
  float over = sum > 0 ? 1 / sum : (sum == 0 ? 0.f : sum);
  by *= over, by1 *= over;
#pragma unroll
  for (int d = 0; d < DP / 32; d++)
#pragma unroll
    for (int r = 0; r < 16; r++) acc[d][r] = acc[d][r] * by + other[(d * 16 + r) * 64] * by1;
  if (i < a.Sq) {
    store_column<E, DP>(acc, 1.f, (char *)a.o.p + b * a.o.batch + h * a.o.head + i * a.o.row, a.D);
    if (a.lse && half == 0) a.lse[((int64_t)b * a.H + h) * a.Sq + i] = sum == 0 ? -INFINITY : (to + __builtin_amdgcn_logf(sum)) * LN2;
  }
}

/* ---- backward --------------------------------------------------------------------------------------------------------------- */
/* delta = do . o and lse in powers of 2: 16 lanes a row, eight values each.  o is read as it was returned, rounded: forming it again would be
 * the forward pass. */
template <class E> __global__ __launch_bounds__(256) void k_delta(Attention a, float *lse2, float *delta) {
  int64_t row = (int64_t)blockIdx.x * 16 + threadIdx.x / 16, rows = (int64_t)a.B * a.H * a.Sq;
  if (row >= rows) return;
  int i = (int)(row % a.Sq), h = (int)(row / a.Sq % a.H), b = (int)(row / a.Sq / a.H), d = threadIdx.x % 16 * 8;
  float s = 0;
  typename Vec<E>::v8 x = load8<E>((const E *)(a.dout.p + b * a.dout.batch + h * a.dout.head + i * a.dout.row) + d, a.D - d);
  typename Vec<E>::v8 y = load8<E>((const E *)(a.o.p + b * a.o.batch + h * a.o.head + i * a.o.row) + d, a.D - d);
  for (int e = 0; e < 8; e++) s += (float)x[e] * (float)y[e];
  for (int k = 8; k > 0; k >>= 1) s += __shfl_xor(s, k);
  if (d == 0) {
    float x = a.lse[row];
    delta[row] = s, lse2[row] = x == -INFINITY ? 0.f : x * LOG2E;
  }
}

__global__ __launch_bounds__(64) void k_ranges(Attention a, int4 *ranges, int rows) { /* tiles of 32 or 64 rows: two or one a wave */
  int tiles = (a.Sq + rows - 1) / rows, per = 64 / rows, groups = (tiles + per - 1) / per, b = blockIdx.x / groups, t = blockIdx.x % groups * per + lane() / rows;
  int begin, end;
  key_range(a, b, t * rows + lane() % rows, begin, end);
  int4 r = make_int4(begin, end, begin, end);
  for (int k = rows / 2; k > 0; k >>= 1) {
    r.x = min(r.x, __shfl_xor(r.x, k)), r.y = max(r.y, __shfl_xor(r.y, k));
    r.z = max(r.z, __shfl_xor(r.z, k)), r.w = min(r.w, __shfl_xor(r.w, k));
  }
  if (lane() % rows == 0 && t < tiles) ranges[(int64_t)b * tiles + t] = r;
}

/* What a pair (query, key) gives: p = e^(s - lse) and ds = p (dp - delta) ds/draw but for the scale, which the sums
 * get at the end.  Both are rounded to the type for the products behind: the matrix cores take 16 bits.  (float16: ds without the scale has to
 * stay below 65504, and keeps more of its small values than with it.) */
template <int KIND> __device__ inline void pair(const Attention &a, float slope2, int distance, float lse2, float delta, float raw, float dp, float &p, float &ds) {
  float by;
  p = exp2_(score<KIND>(a, slope2, raw, distance, by) - lse2);
  ds = p * (dp - delta);
  if (KIND & CAP) ds *= by;
}

/* The second team's sums to the first's, 16 registers x N at a time through LDS. */
template <int N> __device__ __forceinline__ void join_sums(f32x16 (&acc)[N], lds_char *mem, int wave) {
  __attribute__((address_space(3))) float *other = (__attribute__((address_space(3))) float *)mem + wave % 4 * N * 16 * 64 + lane();
  phase();
  if (wave >= 4)
#pragma unroll
    for (int d = 0; d < N; d++)
#pragma unroll
      for (int r = 0; r < 16; r++) other[(d * 16 + r) * 64] = acc[d][r];
  phase();
  if (wave < 4)
#pragma unroll
    for (int d = 0; d < N; d++)
#pragma unroll
      for (int r = 0; r < 16; r++) acc[d][r] += other[(d * 16 + r) * 64];
}

/* LDS of the backward pass: per team three tiles each of two streams (a tile is read in two steps), the numbers of a tile's queries
 * (lse, delta, begin, end); the join needs the first two streams' worth. */
template <int DP> struct GradLds {
  static constexpr int GT = grad_tile(DP), TILE = GT * DP * 2, NUMBERS = 4 * GT * 4, TEAM_BYTES = 6 * TILE + 3 * NUMBERS, BYTES = 2 * TEAM_BYTES;
  static_assert(BYTES >= 4 * DP / 2 * 64 * 4, "the join");
};

/* dq: as in the forward pass a wave has 32 queries, one a lane pair; dp^T = v do^T beside s^T = k q^T, and dq^T += k^T ds^T of the tile before. */
template <class E, int DP, int KIND> __device__ __forceinline__ void attention_dq(const Attention &a, lds_char *mem, int (*part)[2], Holes &ranges, int id) {
  constexpr int GT = grad_tile(DP), X = GT / 32;
  using R = Rows<DP, GT>;
  constexpr int TILE = R::BYTES;
  int wave = uniform(threadIdx.x / 64), team = wave / 4, l = lane(), half = l >> 5;
  lds_char *lds = mem + team * GradLds<DP>::TEAM_BYTES; /* three tiles of keys, three of values */
  int tile, h, b;
  place(a.H, a.B, id, tile, h, b);
  tile = (a.Sq + ROWS - 1) / ROWS - 1 - tile;
  int g = h / (a.H / a.G);
  int i = tile * ROWS + wave % 4 * 32 + (l & 31), offset = a.Sk - a.Sq;
  int begin, end;
  key_range(a, b, i, begin, end);
  int wlo = wave_min(begin), whi = wave_max(end), full_lo = wave_max(begin), full_hi = wave_min(end);
  int lo = wlo, hi = whi;
  note_ranges(a, b, i, begin, end, ranges);
  join_ranges(lo, hi, part);
  const bool holes = has_holes(ranges);
  int first = lo / GT, tiles = lo < hi ? (hi + GT - 1) / GT - first : 0, steps = (tiles + 1) / 2;

  typename Vec<E>::v8 q[DP / 16], dout[DP / 16];
  row_fragments<E, DP>(a.q, b * a.q.batch + h * a.q.head, i, begin < end, a.D, q);
  row_fragments<E, DP>(a.dout, b * a.dout.batch + h * a.dout.head, i, begin < end, a.D, dout);
  float lse2 = 0, delta = 0;
  if (begin < end) {
    int64_t row = ((int64_t)b * a.H + h) * a.Sq + i;
    lse2 = a.lse2[row], delta = a.delta[row];
  }
  f32x16 acc[DP / 32];
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r++) acc[t][r] = 0;
  float slope2 = KIND & BIAS ? a.slopes[h] * LOG2E : 0.f;

  Places<E, DP> at;
  at.init();
  R rk, rv;
  rk.init(a.k.row, a.D);
  rv.init(a.v.row, a.D);
  const char *pk = a.k.p + b * a.k.batch + g * a.k.head, *pv = a.v.p + b * a.v.batch + g * a.v.head;
  auto key0 = [&](int n) __attribute__((always_inline)) { return (first + 2 * n + team) * GT; };
  auto load = [&](int n, int which) __attribute__((always_inline)) {
    int from = key0(n);
    if (holes) { /* of keys alone: what the values give is replaced, not multiplied */
      uint64_t seen = seen_keys<GT>(ranges, from);
      rk.load(pk, a.k.row, lds + which * TILE, from, [&](int at) { return at < hi && (seen >> (at - from) & 1); });
    } else rk.load(pk, a.k.row, lds + which * TILE, from, lo, hi);
    rv.load(pv, a.v.row, lds + (3 + which) * TILE, from, lo, hi);
  };
  f32x16 s[X], dp[X];
  typename Vec<E>::v8 ds[2 * X]; /* of the step before */
  auto scores = [&](int K, int V) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < X; x++) {
#pragma unroll
      for (int r = 0; r < 16; r++) s[x][r] = dp[x][r] = 0;
#pragma unroll
      for (int d = 0; d < DP / 16; d++) {
        s[x] = mfma(at.straight(lds, K, 32 * x, d), q[d], s[x]);
        dp[x] = mfma(at.straight(lds, V, 32 * x, d), dout[d], dp[x]);
      }
    }
  };
  auto sums = [&](int K) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2 * X; x++)
#pragma unroll
      for (int d = 0; d < DP / 32; d++) acc[d] = mfma(at.transposed(lds, K, 16 * x, d), ds[x], acc[d]);
  };
  auto exponentials = [&](int n) __attribute__((always_inline)) {
    int j0 = key0(n), j1 = j0 + 4 * half;
    bool all = j0 >= full_lo && j0 + GT <= full_hi;
#pragma unroll
    for (int x = 0; x < X; x++) {
#pragma unroll
      for (int r = 0; r < 16; r++) {
        float p, d;
        pair<KIND>(a, slope2, i + offset - (j1 + 32 * x + 8 * (r >> 2) + (r & 3)), lse2, delta, s[x][r], dp[x][r], p, d);
        dp[x][r] = d;
      }
      if (!all) {
#pragma unroll
        for (int r = 0; r < 16; r++) {
          int j = j1 + 32 * x + 8 * (r >> 2) + (r & 3);
          dp[x][r] = j >= begin && j < end ? dp[x][r] : 0.f;
        }
      }
#pragma unroll
      for (int r = 0; r < 16; r++) ds[2 * x + r / 8][r % 8] = (E)dp[x][r];
    }
  };
  load(0, 0);
  load(1, 1);
  landed<2 * R::LOADS>();
  phase();
  if (team) phase();
  auto step = [&](int n, auto which, auto begun) __attribute__((always_inline)) {
    constexpr int W = decltype(which)::value;
    if (begun.value) sums((W + 2) % 3 * TILE);
    scores(W * TILE, (3 + W) * TILE);
    if (begun.value) {
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int g = 0; g < X * DP / 16 - 2; g++) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
#pragma unroll
      for (int g = 0; g < X * DP / 8; g++) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
    }
    phase();
    load(n + 2, (W + 2) % 3);
    exponentials(n);
    landed<2 * R::LOADS>();
    phase();
  };
  int n = 0;
  if (steps) {
    step(0, Int<0>(), Int<0>());
    for (n = 1; n + 2 < steps; n += 3) {
      step(n, Int<1>(), Int<1>());
      step(n + 1, Int<2>(), Int<1>());
      step(n + 2, Int<0>(), Int<1>());
    }
    if (n < steps) step(n++, Int<1>(), Int<1>());
    if (n < steps) step(n++, Int<2>(), Int<1>());
    sums((steps - 1) % 3 * TILE);
  }
  if (!team) phase();
  landed<0>();
  join_sums(acc, mem, wave);
  if (!team && i < a.Sq) store_column<E, DP>(acc, a.scale, (char *)a.dq.p + b * a.dq.batch + h * a.dq.head + i * a.dq.row, a.D);
}

/* dk, dv: a wave has 32 keys, one a lane pair, and meets the queries of every head that shares them, a tile at a time: s = q k^T and
 * dp = do v^T (queries in the registers), and dv^T += do^T p, dk^T += q^T ds of the tile before.  The tiles are those between the first and
 * the last that see any of the workgroup's keys. */
template <class E, int DP, int KIND> __device__ __forceinline__ void attention_dkv(const Attention &a, lds_char *mem, int (*part)[2], int id) {
  constexpr int GT = grad_tile(DP), X = GT / 32;
  using R = Rows<DP, GT>;
  constexpr int TILE = R::BYTES, NUMBERS = GradLds<DP>::NUMBERS;
  int wave = uniform(threadIdx.x / 64), team = wave / 4, l = lane(), half = l >> 5;
  lds_char *lds = mem + team * GradLds<DP>::TEAM_BYTES; /* three tiles of q, three of do, three times the numbers */
  int tiles = (a.Sq + GT - 1) / GT, tile, g, b;
  /* its heads: all that share the keys, or one of them */
  int shared = a.H / a.G, h0;
  if (a.parts) {
    place(a.H, a.B, id, tile, h0, b);
    g = h0 / shared;
    shared = 1;
  } else {
    place(a.G, a.B, id, tile, g, b);
    h0 = g * shared;
  }
  int k0 = tile * ROWS, w0 = k0 + wave % 4 * 32, j = w0 + (l & 31), offset = a.Sk - a.Sq;

  const int4 *ranges = a.ranges + (int64_t)b * tiles;
  int lo = FAR, hi = 0;
  for (int t = threadIdx.x % TEAM; t < tiles; t += TEAM) {
    int4 r = ranges[t];
    if (r.x < k0 + ROWS && r.y > k0) lo = min(lo, t), hi = t + 1;
  }
  lo = wave_min(lo), hi = wave_max(hi);
  join_ranges(lo, hi, part);
  int per = lo < hi ? hi - lo : 0, total = per * shared, steps = (total + 1) / 2;

  typename Vec<E>::v8 k[DP / 16], v[DP / 16];
  row_fragments<E, DP>(a.k, b * a.k.batch + g * a.k.head, j, j < a.Sk, a.D, k);
  row_fragments<E, DP>(a.v, b * a.v.batch + g * a.v.head, j, j < a.Sk, a.D, v);
  f32x16 dk[DP / 32], dv[DP / 32];
  for (int t = 0; t < DP / 32; t++)
    for (int r = 0; r < 16; r++) dk[t][r] = dv[t][r] = 0;
  FewPlaces<E, DP> at;
  at.init();
  R rq, rd;
  rq.init(a.q.row, a.D);
  rd.init(a.dout.row, a.D);

  /* a team's tiles: every other one of those of the first head, then of the next */
  struct Tile { int head, t; };
  auto advance = [&](Tile &x) __attribute__((always_inline)) {
    for (x.t += 2; per && x.t >= hi; x.head++) x.t -= per;
  };
  Tile ahead = {0, lo + team}; /* the one that is loaded next */
  if (per && ahead.t >= hi) ahead.t -= per, ahead.head++;
  Tile now = ahead;
  auto load = [&](int which) __attribute__((always_inline)) { /* rows that see nothing are zeros, whatever they hold; past the last head too */
    bool there = ahead.head < shared && per;
    int h = h0 + (there ? ahead.head : 0), i0 = there ? ahead.t * GT : 0, most = there ? a.Sq : 0;
    const char *pq = a.q.p + b * a.q.batch + h * a.q.head, *pd = a.dout.p + b * a.dout.batch + h * a.dout.head;
    lds_char *tq = lds + which * TILE, *td = lds + (3 + which) * TILE;
    if (there && ranges[ahead.t].z == FAR) { /* some row of the tile sees nothing, or there is none */
      auto in = [&](int i) {
        int from, to;
        key_range(a, b, i, from, to);
        return from < to;
      };
      rq.load(pq, a.q.row, tq, i0, in);
      rd.load(pd, a.dout.row, td, i0, in);
    } else {
      rq.load(pq, a.q.row, tq, i0, 0, most);
      rd.load(pd, a.dout.row, td, i0, 0, most);
    }
    /* a wave each for the rows' numbers */
    int64_t row = ((int64_t)b * a.H + h) * a.Sq + i0, at = (int64_t)b * a.Sq + i0;
    int w = wave % 4;
    const void *from = w == 0 ? (const void *)(a.lse2 + row) : w == 1 ? (const void *)(a.delta + row) : w == 2 ? (const void *)(a.begin + at) : (const void *)(a.end + at);
    bool in = (w < 2 || (w == 2 ? a.begin : a.end)) && l < GT && i0 + l < most;
    if (l < GT) load_lds4(buffer(from), lds + 6 * TILE + which * NUMBERS + w * GT * 4, in ? l * 4 : OOB_LAYER_OUT);
    advance(ahead);
  };
  constexpr int LOADS = 2 * R::LOADS + 1;

  f32x16 s[X], dp[X];
  typename Vec<E>::v8 wp[2 * X], ws[2 * X]; /* of the step before */
  auto scores = [&](int Q, int D) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < X; x++) {
#pragma unroll
      for (int r = 0; r < 16; r++) s[x][r] = dp[x][r] = 0;
#pragma unroll
      for (int d = 0; d < DP / 16; d++) {
        s[x] = mfma(at.straight(lds, Q, 32 * x, d), k[d], s[x]);
        dp[x] = mfma(at.straight(lds, D, 32 * x, d), v[d], dp[x]);
      }
    }
  };
  auto sums = [&](int Q) __attribute__((always_inline)) {
#pragma unroll
    for (int x = 0; x < 2 * X; x++)
#pragma unroll
      for (int d = 0; d < DP / 32; d++) {
        dv[d] = mfma(at.transposed(lds, Q + 3 * TILE, 16 * x, d), wp[x], dv[d]);
        dk[d] = mfma(at.transposed(lds, Q, 16 * x, d), ws[x], dk[d]);
      }
  };
  auto exponentials = [&](int N) __attribute__((always_inline)) {
    bool there = now.head < shared && per; /* a team may have a tile less than the other */
    int4 range = make_int4(0, 0, FAR, 0);
    if (there) range = ranges[now.t];
    int i0 = now.t * GT;
    float slope2 = 0;
    if (KIND & BIAS) slope2 = a.slopes[h0 + (there ? now.head : 0)] * LOG2E;
    bool all = w0 >= range.z && w0 + 32 <= range.w;
#pragma unroll
    for (int x = 0; x < X; x++) {
#pragma unroll
      for (int n = 0; n < 4; n++) {
        int row = 32 * x + 8 * n;
        f32x4 lse = lds_numbers<f32x4>(lds + 16 * half + (N + row * 4)), delta = lds_numbers<f32x4>(lds + 16 * half + (N + GT * 4 + row * 4));
#pragma unroll
        for (int e = 0; e < 4; e++) {
          float p, d;
          pair<KIND>(a, slope2, i0 + row + 4 * half + e + offset - j, lse[e], delta[e], s[x][4 * n + e], dp[x][4 * n + e], p, d);
          s[x][4 * n + e] = p, dp[x][4 * n + e] = d;
        }
      }
      if (!all) {
#pragma unroll
        for (int n = 0; n < 4; n++) {
          int row = 32 * x + 8 * n;
          i32x4 from = {0, 0, 0, 0}, to = {a.Sk, a.Sk, a.Sk, a.Sk};
          if (a.begin) from = lds_numbers<i32x4>(lds + 16 * half + (N + 2 * GT * 4 + row * 4));
          if (a.end) to = lds_numbers<i32x4>(lds + 16 * half + (N + 3 * GT * 4 + row * 4));
#pragma unroll
          for (int e = 0; e < 4; e++) {
            int i = i0 + row + 4 * half + e;
            bool seen = there && j >= from[e] && j < to[e] && i < a.Sq && (!a.causal || j - offset <= i);
            s[x][4 * n + e] = seen ? s[x][4 * n + e] : 0.f;
            dp[x][4 * n + e] = seen ? dp[x][4 * n + e] : 0.f;
          }
        }
      }
#pragma unroll
      for (int r = 0; r < 16; r++) wp[2 * x + r / 8][r % 8] = (E)s[x][r], ws[2 * x + r / 8][r % 8] = (E)dp[x][r];
    }
    advance(now);
  };
  load(0);
  load(1);
  landed<LOADS>();
  phase();
  if (team) phase();
  auto step = [&](int n, auto which, auto begun) __attribute__((always_inline)) {
    constexpr int W = decltype(which)::value;
    at.fresh();
    if (begun.value) sums((W + 2) % 3 * TILE);
    if (begun.value) {
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int g = 0; g < X * DP / 8 - 2; g++) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    scores(W * TILE, (3 + W) * TILE);
    __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
    for (int g = 0; g < X * DP / 8 - 2; g++) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x8, 2, 0);
    phase();
    load((W + 2) % 3);
    exponentials(6 * TILE + W * NUMBERS);
    landed<LOADS>();
    phase();
  };
  int n = 0;
  if (steps) {
    step(0, Int<0>(), Int<0>());
    for (n = 1; n + 2 < steps; n += 3) {
      step(n, Int<1>(), Int<1>());
      step(n + 1, Int<2>(), Int<1>());
      step(n + 2, Int<0>(), Int<1>());
    }
    if (n < steps) step(n++, Int<1>(), Int<1>());
    if (n < steps) step(n++, Int<2>(), Int<1>());
    sums((steps - 1) % 3 * TILE);
  }
  if (!team) phase();
  landed<0>();
  join_sums(dk, mem, wave);
  join_sums(dv, mem, wave);
  if (!team && j < a.Sk && a.parts) {
    int64_t per = (int64_t)a.B * a.Sk * a.G * a.D;
    float *to = a.parts + h0 % (a.H / a.G) * per + (((int64_t)b * a.Sk + j) * a.G + g) * a.D;
    store_column<float, DP>(dk, a.scale, (char *)to, a.D);
    store_column<float, DP>(dv, 1.f, (char *)(to + a.H / a.G * per), a.D);
  } else if (!team && j < a.Sk) {
    store_column<E, DP>(dk, a.scale, (char *)a.dk.p + b * a.dk.batch + g * a.dk.head + j * a.dk.row, a.D);
    store_column<E, DP>(dv, 1.f, (char *)a.dv.p + b * a.dv.batch + g * a.dv.head + j * a.dv.row, a.D);
  }
}

/* Both in one launch: the tiles of keys first, then those of queries fill up what the last of them leave idle.  Seven products a pair of
 * tiles where five would do if dq were added up by atomics, whose order changes sums: with delta and ranges 264 us for 4096 tokens, 12 heads of
 * 128, causal (a quarter more in two launches of one-team workgroups); without a mask and 16 heads 543 us, 0.63 PFLOP/s on the five.  For heads of 128
 * the steps of dk and dv are short of registers (34 spilled, 73 with a distance bias, 93 with a cap too) and wait for all loads three times: for the
 * ranges of the tile that is loaded next, for those of the present one, and for what was spilled. */
template <class E, int DP, int KIND> __global__ __launch_bounds__(THREADS, 2) void k_attention_grad(Attention a, int of_keys) {
  __shared__ __attribute__((aligned(1024))) char mem[GradLds<DP>::BYTES];
  __shared__ int part[8][2];
  __shared__ Holes ranges;
  if ((int)blockIdx.x < of_keys) attention_dkv<E, DP, KIND>(a, (lds_char *)mem, part, blockIdx.x);
  else attention_dq<E, DP, KIND>(a, (lds_char *)mem, part, ranges, blockIdx.x - of_keys);
}

/* dk and dv from those of the heads that share them. */
template <class E> __global__ __launch_bounds__(256) void k_join_heads(Attention a) {
  int64_t per = (int64_t)a.B * a.Sk * a.G * a.D, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= per) return;
  int shared = a.H / a.G, d = (int)(at % a.D), g = (int)(at / a.D % a.G), j = (int)(at / a.D / a.G % a.Sk), b = (int)(at / a.D / a.G / a.Sk);
  float dk = 0, dv = 0;
  for (int h = 0; h < shared; h++) dk += a.parts[h * per + at], dv += a.parts[(shared + h) * per + at];
  ((E *)(a.dk.p + b * a.dk.batch + g * a.dk.head + j * a.dk.row))[d] = (E)dk;
  ((E *)(a.dv.p + b * a.dv.batch + g * a.dv.head + j * a.dv.row))[d] = (E)dv;
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
/* Whether the loads' 32-bit offsets (up to 31 rows of a lane's own, 48 beside the bounds) reach the rows, copied where they have to be. */
static bool reachable(const Heads &h, int S, int N, int D) { return loadable(h, D) || (S < 32 ? S : 32) * (N * up(D, 8) * 2) < (int64_t)1 << 31; }
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
  const int64_t most = (int64_t)1 << 31, heads = (int64_t)p->B * p->H, wgs = (p->Sq > p->Sk ? p->Sq : p->Sk) / 16 + 1;
  if (heads >= most || heads * wgs >= most) return false;
  for (const int64_t(*s)[3] : {&p->q_stride, &p->k_stride, &p->v_stride, &p->o_stride})
    for (int i = 0; i < 3; i++)
      if ((*s)[i] < 0) return false;
  for (const void *q : {p->q, p->k, p->v, (const void *)p->o})
    if (!multiple(q, 2)) return false;
  return multiple(p->key_begin, 4) && multiple(p->key_end, 4) && multiple(p->slopes, 4) && multiple(p->lse, 4);
}

/* Whether a result's rows are each its own: an axis of stride 0 has them all in one place. */
static bool apart(const int64_t (&stride)[3], int B, int S, int N) { return (stride[0] || B < 2) && (stride[1] || S < 2) && (stride[2] || N < 2); }

static Attention attention_of(const oob_attention *p) {
  Attention a{};
  a.q = heads_of(p->q, p->q_stride), a.k = heads_of(p->k, p->k_stride), a.v = heads_of(p->v, p->v_stride), a.o = heads_of(p->o, p->o_stride);
  a.begin = p->key_begin, a.end = p->key_end, a.slopes = p->slopes, a.lse = p->lse;
  a.B = p->B, a.Sq = p->Sq, a.Sk = p->Sk, a.H = p->H, a.G = p->G, a.D = p->D;
  a.causal = p->causal != 0, a.scale = p->scale, a.cap = p->cap;
  return a;
}

template <class F> static void by_kind(const Attention &a, F f) {
  if (a.cap > 0 && a.slopes) f(Int<CAP | BIAS>());
  else if (a.cap > 0) f(Int<CAP>());
  else if (a.slopes) f(Int<BIAS>());
  else f(Int<0>());
}

static bool rows_ok(const oob_attention *p) {
  Attention a = attention_of(p);
  return reachable(a.k, a.Sk, a.G, a.D) && reachable(a.v, a.Sk, a.G, a.D);
}
static bool rows_ok(const oob_attention *p, const oob_attention_grad *q) {
  Attention a = attention_of(p);
  return rows_ok(p) && reachable(a.q, a.Sq, a.H, a.D) && reachable(heads_of(q->dout, q->dout_stride), a.Sq, a.H, a.D);
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
    by_kind(a, [&](auto kind) {
      constexpr int KIND = decltype(kind)::value;
      if (a.D <= 64) k_attention<E, 64, KIND><<<n, THREADS, 0, st>>>(a);
      else k_attention<E, 128, KIND><<<n, THREADS, 0, st>>>(a);
    });
  }
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

/* Heads that share keys: a workgroup goes through all of them, unless that leaves most of the GPU without work.  (2 sequences of 1531, 8
 * heads on 2, width 80: 48 workgroups, 423 us forward and backward; one for each head and a pass that adds: 228 us.) */
static bool by_head(const Attention &a) { return a.H > a.G && (int64_t)a.B * a.G * ((a.Sk + ROWS - 1) / ROWS) < 256; }
static size_t parts_bytes(const Attention &a) { return by_head(a) ? (size_t)2 * (a.H / a.G) * a.B * a.Sk * a.G * a.D * 4 : 0; }

static size_t backward_bytes(const oob_attention *p, const oob_attention_grad *q) {
  Attention a = attention_of(p);
  Arena w{nullptr, 0, 0};
  w.take((size_t)a.B * a.H * a.Sq * 8);
  w.take((size_t)a.B * ((a.Sq + 31) / 32) * sizeof(int4));
  w.take(parts_bytes(a));
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
  int64_t rows = (int64_t)a.B * a.H * a.Sq;
  float *lse2 = (float *)w.take((size_t)rows * 8), *delta = lse2 + rows;
  int4 *ranges = (int4 *)w.take((size_t)a.B * ((a.Sq + 31) / 32) * sizeof(int4));
  float *parts = (float *)w.take(parts_bytes(a));
  a.lse2 = lse2, a.delta = delta, a.ranges = ranges, a.parts = by_head(a) ? parts : nullptr;
  if (!w.ok()) return OOB_ECAPACITY;
  if (rows) {
    k_delta<E><<<(unsigned)((rows + 15) / 16), 256, 0, st>>>(a, lse2, delta);
    k_ranges<<<(unsigned)(a.B * ((a.Sq + 63) / 64)), 64, 0, st>>>(a, ranges, grad_tile(a.D <= 64 ? 64 : 128));
  }
  pack(a.k, a.B, a.Sk, a.G, a.D, w, st);
  pack(a.v, a.B, a.Sk, a.G, a.D, w, st);
  pack(a.q, a.B, a.Sq, a.H, a.D, w, st);
  pack(a.dout, a.B, a.Sq, a.H, a.D, w, st);
  if (!w.ok()) return OOB_ECAPACITY;
  unsigned nq = (unsigned)((int64_t)a.B * a.H * ((a.Sq + ROWS - 1) / ROWS)), nk = (unsigned)((int64_t)a.B * (a.parts ? a.H : a.G) * ((a.Sk + ROWS - 1) / ROWS));
  by_kind(a, [&](auto kind) {
    constexpr int KIND = decltype(kind)::value;
    if (nk + nq && a.D <= 64) k_attention_grad<E, 64, KIND><<<nk + nq, THREADS, 0, st>>>(a, (int)nk);
    else if (nk + nq) k_attention_grad<E, 128, KIND><<<nk + nq, THREADS, 0, st>>>(a, (int)nk);
  });
  if (nk && a.parts) k_join_heads<E><<<(unsigned)(((int64_t)a.B * a.Sk * a.G * a.D + 255) / 256), 256, 0, st>>>(a);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

static bool grads_ok(const oob_attention *p, const oob_attention_grad *q) {
  for (const int64_t(*s)[3] : {&q->dout_stride, &q->dq_stride, &q->dk_stride, &q->dv_stride})
    for (int i = 0; i < 3; i++)
      if ((*s)[i] < 0) return false;
  for (const void *x : {q->dout, (const void *)q->dq, (const void *)q->dk, (const void *)q->dv})
    if (!multiple(x, 2)) return false;
  if (!apart(q->dq_stride, p->B, p->Sq, p->H) || !apart(q->dk_stride, p->B, p->Sk, p->G) || !apart(q->dv_stride, p->B, p->Sk, p->G)) return false;
  if (p->B > 0 && p->Sq > 0 && (!p->q || !p->o || !p->lse || !q->dout || !q->dq)) return false;
  return !(p->B > 0 && p->Sk > 0 && (!p->k || !p->v || !q->dk || !q->dv));
}

}  // namespace layer

using namespace layer;

extern "C" size_t oob_layer_attention_workspace_size(const oob_attention *p) { return p && attention_ok(p) ? forward_bytes(p) : 0; }

extern "C" int oob_layer_attention(const oob_attention *p, void *workspace, size_t bytes, void *stream) {
  if (!p || !attention_ok(p) || !multiple(workspace, 256)) return OOB_EINVAL;
  if (p->B == 0 || p->Sq == 0) return OOB_OK;
  if (!p->q || !p->o || (p->Sk > 0 && (!p->k || !p->v)) || !rows_ok(p) || !apart(p->o_stride, p->B, p->Sq, p->H)) return OOB_EINVAL;
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
  if (!rows_ok(p, q)) return OOB_EINVAL;
  size_t need = backward_bytes(p, q);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? backward<bf16>(p, q, w, (hipStream_t)stream) : backward<fp16>(p, q, w, (hipStream_t)stream);
}
