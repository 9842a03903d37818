/* Routing to experts and the chosen pairs in order of their experts. */
#include "oob_expert.h"
#include "oob_layer_device.h"

#define OOB_LDS __attribute__((address_space(3)))

namespace layer {
namespace {

__device__ inline float logit(const void *p, int dtype, int64_t at) {
  if (dtype == OOB_FP32) return ((const float *)p)[at];
  return dtype == OOB_BF16 ? (float)((const bf16 *)p)[at] : (float)((const fp16 *)p)[at];
}
__device__ inline void put(void *p, int dtype, int64_t at, float v) {
  if (dtype == OOB_FP32) ((float *)p)[at] = v;
  else if (dtype == OOB_BF16) ((bf16 *)p)[at] = (bf16)v;
  else ((fp16 *)p)[at] = (fp16)v;
}

/* What a lane's partner holds at each level of a reduction over neighbouring lanes: within rows of 16 by DPP moves (swapped pairs, pairs of pairs, mirrored
 * halves and rows: below each level all lanes of a part hold the same), across them by the swaps of rows and of halves. */
template <class F> __device__ inline uint32_t over(uint32_t v, int lanes, F f) {
  if (lanes > 1) v = f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));
  if (lanes > 2) v = f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));
  if (lanes > 4) v = f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x141, 0xf, 0xf, true));
  if (lanes > 8) v = f(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x140, 0xf, 0xf, true));
  if (lanes > 16) {
    auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = f(r[0], r[1]);
  }
  if (lanes > 32) {
    auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = f(r[0], r[1]);
  }
  return v;
}
/* Over runs of `lanes` lanes (a power of two). */
__device__ inline uint32_t max_over(uint32_t v, int lanes) { return over(v, lanes, [](uint32_t a, uint32_t b) { return a > b ? a : b; }); }
__device__ inline int min_over(int v, int lanes) { /* of numbers that are not negative */
  return (int)over((uint32_t)v, lanes, [](uint32_t a, uint32_t b) { return a < b ? a : b; });
}
__device__ inline float max_over(float v, int lanes) {
  return __uint_as_float(over(__float_as_uint(v), lanes, [](uint32_t a, uint32_t b) { return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b))); }));
}
__device__ inline float sum_over(float v, int lanes) {
  return __uint_as_float(over(__float_as_uint(v), lanes, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ inline uint64_t max_over(uint64_t v, int lanes) { /* the larger high half, then the larger low half of those that have it */
  uint32_t hi = max_over((uint32_t)(v >> 32), lanes);
  uint32_t lo = max_over((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u, lanes);
  return (uint64_t)hi << 32 | lo;
}
__device__ inline double sum_over(double v, int lanes) {
  for (int o = 1; o < lanes; o *= 2) v += __shfl_xor(v, o);
  return v;
}
/* Numbers in the order of what they stand for: 0 is nothing (absent or taken), NaN above it, -inf and all else above that.  The five lowest bits of those of
 * 32 can give way to another number, and a NaN's is not 0 then either. */
__device__ inline uint32_t key_of(float v) {
  if (v != v) return 32;
  uint32_t b = __float_as_uint(v + 0.f); /* -0 is 0 */
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ inline uint64_t key_of(double v) {
  if (v != v) return 1;
  uint64_t b = (uint64_t)__double_as_longlong(v + 0.);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

/* The key of a closed expert among keys of 64 bits: after all others, one that a bias of -inf rules out among them, but before NaN.  (Those of 32 bits are never the
 * last word where two follow one another whose scores are -inf.) */
constexpr uint64_t CLOSED = 2;

/* sigmoid(l) e^-m: with m the largest min(l, 0) of several, their ratios keep all digits however small they are. */
__device__ inline float sigmoid_over(float l, float m) { return expf(fminf(l, 0.f) - m) / (1 + expf(-fabsf(l))); }

__device__ inline float value_of(uint32_t key) { return __uint_as_float(key >> 31 ? key & 0x7fffffffu : ~key); } /* of key_of(float), NaN aside */

/* ---- routing -------------------------------------------------------------------------------------------------------------
 * A token takes a run of lanes, each V neighbouring experts of one group: a choice is a maximum over registers, then over the run, and of those that hold it the
 * smallest number.  What bounds it is instructions (16384 tokens, 256 experts in 8 groups, float32: 1070 a wave of two tokens, 25 us; a large copy would read
 * the logits in 3.3): with four experts a lane reductions make most of them (46 us), with 16 too few waves hide each other's waits (28 us).
 * Scores with a bias, and sums of groups, are compared as 64-bit programs do, to the last digit.  They are formed in 32 bits first: only where two that are
 * compared lie closer than their errors allow is the token done again in 64 (16384 tokens, 256 experts in 8 groups: 23 us, 37 where every token is, with a bias of 5, say). */
struct Route {
  oob_route p;
  int lanes;    /* a token's: a power of two, at least k */
  int per;      /* experts of a group */
  int in_group; /* lanes of a group: a power of two */
  int whole, whole_bias; /* a lane's logits, biases can be loaded four at a time */
};

template <int V> struct Token {
  float x[V], bias[V]; /* logits, -inf: closed or absent; 0 without a bias */
  int there, group; /* so many of the V exist */
  int e0;
};

/* Whether b is more than a.  In 64 bits NaN is less than everything; in 32 a token that holds one is not sure (see below), and what is absent counts as -inf. */
__device__ inline bool more(float b, float a) { return b > a; }
__device__ inline bool more(double b, double a) { return b > a || a != a; }
template <class F> constexpr F NONE = sizeof(F) == 8 ? (F)NAN : (F)-INFINITY;

/* Keys of scores in type F (double, float), and the best two scores. */
template <class F, int V, class K> __device__ __forceinline__ F keys_of(const Route &r, const Token<V> &a, int L, float top, K (&key)[V], F &best, F &next) {
  F s[V], total = 0;
  for (int i = 0; i < V; i++) {
    if constexpr (sizeof(F) == 8) s[i] = a.x[i] == -INFINITY ? 0. : r.p.score == OOB_ROUTE_SOFTMAX ? exp((double)a.x[i] - (double)top) : 1 / (1 + exp(-(double)a.x[i]));
    else {
      float e = __builtin_amdgcn_exp2f((r.p.score == OOB_ROUTE_SOFTMAX ? a.x[i] - top : -a.x[i]) * 1.44269504f);
      s[i] = a.x[i] == -INFINITY ? 0.f : r.p.score == OOB_ROUTE_SOFTMAX ? e : __builtin_amdgcn_rcpf(1 + e);
    }
    total += s[i];
  }
  F part = 1;
  if (r.p.score == OOB_ROUTE_SOFTMAX) {
    total = sum_over(total, L);
    if constexpr (sizeof(F) == 4) part = 1 / total;
  }
  best = next = NONE<F>;
  for (int i = 0; i < V; i++) {
    F c = sizeof(F) == 8 && i >= a.there ? NONE<F> : (F)-INFINITY;
    if (a.x[i] != -INFINITY) {
      c = s[i];
      if (r.p.score == OOB_ROUTE_SOFTMAX) c = sizeof(F) == 8 ? s[i] / total : s[i] * part;
      if (r.p.bias) c += a.bias[i];
    }
    key[i] = i < a.there ? key_of(c) : 0;
    if constexpr (sizeof(F) == 8) key[i] = i < a.there && a.x[i] == -INFINITY ? CLOSED : key[i];
    F low = more(c, best) ? best : c;
    best = more(c, best) ? c : best;
    next = more(low, next) ? low : next;
  }
  return total;
}

/* By how much a score and a bias of at most 4 formed in 32 bits may be off: the sum of up to 1024 exponentials 2.2e-6 of itself (32 in a row in a lane, then 6
 * halvings: 37 roundings of 2^-24; 16 in a row 1.3e-6), the exponentials' arguments 4e-7, three more roundings 2e-7, the bias's addition 3e-7: 3.1e-6 in all.  Larger
 * biases are left to 64 bits. */
constexpr float OFF = 4e-6f, LARGE = 4.f;

/* Closes the experts of the groups that are not kept; false: in 32 bits, two groups' sums lie too close to tell. */
template <class F, int V, class K> __device__ __forceinline__ bool groups(const Route &r, const Token<V> &a, int L, K (&key)[V], F best, F next) {
  const oob_route &p = r.p;
  for (int o = 1; o < r.in_group; o *= 2) {
    F b = __shfl_xor(best, o), n = __shfl_xor(next, o);
    F low = more(b, best) ? best : b; /* second of the four: the lower first or one of the seconds */
    best = more(b, best) ? b : best;
    n = more(n, next) ? n : next;
    next = more(low, n) ? low : n;
  }
  K of = a.group < p.groups ? key_of(p.group_best == 2 && r.per > 1 ? best + next : best) : 0;
  bool kept = false, sure = true;
  K most = 0;
  for (int n = 0; n < p.keep_groups; n++) {
    most = max_over(of, L);
    int won = min_over(of == most ? a.group : 1 << 30, L);
    if (a.group == won) kept = true, of = 0;
  }
  if constexpr (sizeof(F) == 4) {
    K beyond = max_over(of, L);
    if (beyond) sure = value_of(most) - value_of(beyond) > 6 * OFF; /* two scores each, and their sum's rounding */
  }
  if (!kept)
    for (int i = 0; i < V; i++) key[i] = 0;
  return sure;
}

/* The k largest keys; lane j gets the number of choice j.  CHECK: keys of 32 bits whose lowest bits have given way to the number in the lane (no two of a lane
 * are alike then, which saves a third of the instructions); false where two in a row lie too close to tell. */
template <bool CHECK, int V, class K> __device__ __forceinline__ bool choose(const Route &r, const Token<V> &a, int L, K (&key)[V], int &expert) {
  const int l = lane() & (L - 1), k = r.p.k;
  bool sure = true;
  K last = 0;
  if constexpr (CHECK)
#pragma unroll
    for (int i = 0; i < V; i++) key[i] = key[i] ? (key[i] & ~(K)31) | (V - 1 - i) : 0;
  for (int j = 0; j < k + (CHECK ? 1 : 0); j++) {
    K best = key[0];
#pragma unroll
    for (int i = 1; i < V; i++) best = key[i] > best ? key[i] : best;
    K most = max_over(best, L); /* never 0: k experts are there */
    int number;
    if constexpr (CHECK) {
      /* 32 units of the last place of a number, 4e-6 of it, each; NaN and infinities that follow one another: not sure */
      if (j && most) sure = sure && value_of(last) - value_of(most) > 2 * OFF + 8e-6f * fabsf(value_of(last));
      last = most;
      if (j == k) break;
      number = min_over(best == most ? a.e0 + V - 1 - (int)(most & 31) : 1 << 30, L);
      if (number >= a.e0 && number < a.e0 + V)
#pragma unroll
        for (int i = 0; i < V; i++) key[i] = key[i] == most ? 0 : key[i];
    } else {
      int at = 1 << 30;
#pragma unroll
      for (int i = V - 1; i >= 0; i--) at = key[i] == most ? a.e0 + i : at;
      number = min_over(at, L);
      int in = number - a.e0;
#pragma unroll
      for (int i = 0; i < V; i++) key[i] = i == in ? 0 : key[i];
    }
    if (l == j) expert = number;
  }
  return sure;
}

/* LANES: a token's, where they are known (the reductions then have no branches); 0: r.lanes. 32 experts a lane: three waves a SIMD and 12 registers of the way through 64
 * bits in memory, 16384 tokens of 33 groups of 31 experts 146 us; two waves without it 185 us. */
template <int V, bool SCORES, int LANES> __global__ __launch_bounds__(256, V == 32 ? 3 : 1) void k_route(Route r) {
  const oob_route &p = r.p;
  const int L = LANES ? LANES : r.lanes, l = lane() & (L - 1);
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool live = t < p.T; /* runs of lanes as a whole: the others take part in the exchanges and write nothing */
  Token<V> a;
  int in = l % r.in_group * V;
  a.group = l / r.in_group, a.e0 = a.group * r.per + in;
  a.there = a.group < p.groups ? r.per - in : 0;
  int64_t at = t * p.logits_stride + a.e0;
  if (V % 4 == 0 && r.whole) {
#pragma unroll
    for (int q = 0; q < V; q += 4) {
      bool here = live && q < a.there;
      if (p.dtype == OOB_FP32) {
        f32x4 v = here ? *(const f32x4 *)((const float *)p.logits + at + q) : f32x4{0, 0, 0, 0};
        for (int i = 0; i < 4; i++) a.x[q + i] = here ? v[i] : -INFINITY;
      } else {
        uint64_t v = here ? *(const uint64_t *)((const uint16_t *)p.logits + at + q) : 0;
        for (int i = 0; i < 4; i++) {
          uint16_t h = (uint16_t)(v >> (16 * i));
          a.x[q + i] = !here ? -INFINITY : p.dtype == OOB_BF16 ? (float)__builtin_bit_cast(bf16, h) : (float)__builtin_bit_cast(fp16, h);
        }
      }
    }
  } else {
    for (int i = 0; i < V; i++) a.x[i] = live && i < a.there ? logit(p.logits, p.dtype, at + i) : -INFINITY;
  }
  if constexpr (SCORES) { /* all loads before the first is waited for */
    if (V % 4 == 0 && p.bias && r.whole_bias) {
#pragma unroll
      for (int q = 0; q < V; q += 4) {
        f32x4 v = q < a.there ? *(const f32x4 *)(p.bias + a.e0 + q) : f32x4{0, 0, 0, 0};
        for (int i = 0; i < 4; i++) a.bias[q + i] = v[i];
      }
    } else {
#pragma unroll
      for (int i = 0; i < V; i++) a.bias[i] = p.bias && i < a.there ? p.bias[a.e0 + i] : 0.f;
    }
  }
  float top = a.x[0];
  for (int i = 1; i < V; i++) top = fmaxf(top, a.x[i]);
  if (p.score == OOB_ROUTE_SOFTMAX) top = max_over(top, L);

  float all = 0;
  int expert = 0; /* lane j's: choice j */
  if constexpr (SCORES) {
    uint32_t key[V];
    float best, next;
    all = keys_of<float>(r, a, L, top, key, best, next);
    bool sure = true;
    if (p.bias)
#pragma unroll
      for (int i = 0; i < V; i++) sure &= fabsf(a.bias[i]) <= LARGE;
    if (p.groups > 1) sure = groups(r, a, L, key, best, next) && sure && all == all; /* NaN: some score is */
    sure = choose<true>(r, a, L, key, expert) && sure;
    if (__ballot(live && !sure)) {
#pragma unroll
      for (int i = 0; i < V; i++) asm("" : "+v"(a.x[i])); /* conditions on it are formed anew, not kept from above in scalar registers */
      uint64_t wide[V];
      double b, n;
      keys_of<double>(r, a, L, top, wide, b, n);
      if (p.groups > 1) groups(r, a, L, wide, b, n);
      choose<false>(r, a, L, wide, expert);
    }
  } else {
    uint32_t key[V];
    for (int i = 0; i < V; i++) key[i] = i < a.there ? key_of(a.x[i]) : 0;
    choose<false>(r, a, L, key, expert);
  }

  const bool has = l < p.k;
  float mine = live && has ? logit(p.logits, p.dtype, t * p.logits_stride + expert) : -INFINITY, w;
  if (p.renormalize) {
    float m = max_over(!has || mine != mine ? -INFINITY : p.score == OOB_ROUTE_SIGMOID ? fminf(mine, 0.f) : mine, L);
    float s = !has || mine == -INFINITY ? 0.f : p.score == OOB_ROUTE_SIGMOID ? sigmoid_over(mine, m) : expf(mine - m);
    float sum = sum_over(s, L);
    w = sum == 0 ? 0.f : s / sum;
  } else if (p.score == OOB_ROUTE_SIGMOID) {
    w = sigmoid_over(mine, 0.f);
  } else {
    if (!SCORES) {
      for (int i = 0; i < V; i++) all += a.x[i] == -INFINITY ? 0.f : expf(a.x[i] - top);
      all = sum_over(all, L);
    }
    w = mine == -INFINITY ? 0.f : expf(mine - top) / all;
  }
  if (live && has) {
    p.experts[t * p.k + l] = expert;
    p.weights[t * p.k + l] = w * p.scale;
  }
}

/* ---- its gradient: a token takes a run of lanes, lane j its choice j; the row is put together in LDS, where the choices add to it
 * one after the other.  16384 tokens, 256 experts, float32: 7.7 us, 16.8 MB of rows written at 2.2 TB/s. */
struct RouteGrad {
  oob_route p;
  const float *dweights;
  void *dlogits;
  int64_t ld;
  int lanes, whole; /* whole: rows of dlogits can be written four values at a time */
};

__global__ __launch_bounds__(256) void k_route_grad(RouteGrad g) {
  extern __shared__ float rows[];
  const oob_route &p = g.p;
  const int L = g.lanes, l = lane() & (L - 1);
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool live = t < p.T;
  volatile OOB_LDS float *row = (OOB_LDS float *)rows + threadIdx.x / L * p.E;

  int e = live && l < p.k ? p.experts[t * p.k + l] : -1;
  bool has = e >= 0 && e < p.E;
  float x = has ? logit(p.logits, p.dtype, t * p.logits_stride + e) : -INFINITY, d = has ? g.dweights[t * p.k + l] * p.scale : 0.f;
  float add = 0;
  const bool whole = p.score == OOB_ROUTE_SOFTMAX && !p.renormalize; /* the only case in which an expert that was not chosen has a gradient */
  if (whole) {
    float top = -INFINITY, all = 0;
    for (int i = l; i < p.E; i += L) {
      float v = live ? logit(p.logits, p.dtype, t * p.logits_stride + i) : -INFINITY;
      row[i] = v;
      top = fmaxf(top, v);
    }
    top = max_over(top, L);
    for (int i = l; i < p.E; i += L) {
      float s = row[i] == -INFINITY ? 0.f : expf(row[i] - top);
      row[i] = s;
      all += s;
    }
    all = sum_over(all, L);
    add = x == -INFINITY ? 0.f : expf(x - top) / all * d;
    float dot = all == 0 ? 0.f : sum_over(add, L) / all;
    for (int i = l; i < p.E; i += L) row[i] = row[i] == 0 ? 0.f : -row[i] * dot;
  } else {
    bool sig = p.score == OOB_ROUTE_SIGMOID;
    if (p.renormalize) {
      float m = max_over(x != x ? -INFINITY : sig ? fminf(x, 0.f) : x, L);
      float s = x == -INFINITY ? 0.f : sig ? sigmoid_over(x, m) : expf(x - m);
      float all = sum_over(s, L);
      s = all == 0 ? 0.f : s / all;
      float dot = sum_over(s == 0 ? 0.f : s * d, L);
      add = s == 0 ? 0.f : s * (d - dot) * (sig ? sigmoid_over(-x, 0.f) : 1.f);
    } else {
      float q = expf(-fabsf(x)); /* s (1 - s) = q / (1 + q)^2 */
      add = x == -INFINITY ? 0.f : d * q / ((1 + q) * (1 + q));
    }
    for (int i = l; i < p.E; i += L) row[i] = 0;
  }
  __builtin_amdgcn_wave_barrier();
  for (int j = 0; j < p.k; j++) {
    if (l == j && has) row[e] += add;
    __builtin_amdgcn_wave_barrier();
  }
  if (!live) return;
  if (g.whole && p.dtype == OOB_FP32) {
    for (int i = 4 * l; i < p.E; i += 4 * L) *(f32x4 *)((float *)g.dlogits + t * g.ld + i) = f32x4{row[i], row[i + 1], row[i + 2], row[i + 3]};
  } else if (g.whole) {
    for (int i = 4 * l; i < p.E; i += 4 * L) {
      uint64_t v = 0;
      for (int e = 0; e < 4; e++)
        v |= (uint64_t)(p.dtype == OOB_BF16 ? __builtin_bit_cast(uint16_t, (bf16)row[i + e]) : __builtin_bit_cast(uint16_t, (fp16)row[i + e])) << (16 * e);
      *(uint64_t *)((uint16_t *)g.dlogits + t * g.ld + i) = v;
    }
  } else {
    for (int i = l; i < p.E; i += L) put(g.dlogits, p.dtype, t * g.ld + i, row[i]);
  }
}

/* Tokens of a launch, which has less than 2^32 threads. */
int64_t tokens_of(int lanes) { return ((int64_t)1 << 31) / lanes; }
/* The same operands from token t on, n of them. */
oob_route part_of(const oob_route &p, int64_t t, int64_t n) {
  oob_route q = p;
  q.T = p.T - t < n ? p.T - t : n;
  q.logits = (const char *)p.logits + t * p.logits_stride * (p.dtype == OOB_FP32 ? 4 : 2), q.experts += t * p.k;
  if (p.weights) q.weights += t * p.k;
  return q;
}

int ceil2(int n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

bool route_ok(const oob_route *p, bool forward) {
  if (!p || (p->dtype != OOB_BF16 && p->dtype != OOB_FP16 && p->dtype != OOB_FP32)) return false;
  if ((p->score != OOB_ROUTE_SOFTMAX && p->score != OOB_ROUTE_SIGMOID) || (p->renormalize != 0 && p->renormalize != 1)) return false;
  if (p->E < 1 || p->E > OOB_EXPERT_MAX || p->k < 1 || p->k > OOB_EXPERT_MAX_CHOICES || p->k > p->E) return false;
  if (!(p->scale - p->scale == 0) || p->T < 0 || p->T >= (int64_t)1 << 31) return false;
  if (forward) {
    if (p->groups < 1 || p->groups > 64 || p->E % p->groups || p->keep_groups < 1 || p->keep_groups > p->groups) return false;
    if (p->group_best < 1 || p->group_best > 2 || p->k > p->keep_groups * (p->E / p->groups)) return false;
  }
  if (p->T == 0) return true;
  size_t of = p->dtype == OOB_FP32 ? 4 : 2;
  if (!p->logits || !readable(p->logits_stride, p->E) || !p->experts || !multiple(p->logits, of) || !multiple(p->experts, 4)) return false;
  return !forward || (p->weights && multiple(p->weights, 4) && multiple(p->bias, 4));
}

template <int V, int LANES> void route(const Route &r, hipStream_t st) {
  unsigned n = (unsigned)((r.p.T * r.lanes + 255) / 256);
  if (r.p.bias || r.p.groups > 1) k_route<V, true, LANES><<<n, 256, 0, st>>>(r);
  else k_route<V, false, LANES><<<n, 256, 0, st>>>(r);
}
/* Where tokens fill the GPU (V is 8 then, unless groups are small or experts many) and have eight lanes or more, their number is compiled in: 65536 tokens, 8 of 64, 128, 256 and 512
 * experts in 8 groups 20, 32, 58 and 110 us, with lanes as a number 23, 37, 63 and 118; without groups and bias 9, 16, 33 and 68 against 10, 18, 35 and 71.  Fewer lanes take less than
 * the host's call. */
template <int V> void route(const Route &r, hipStream_t st) {
  if constexpr (V == 8) {
    if (r.lanes == 8) return route<V, 8>(r, st);
    if (r.lanes == 16) return route<V, 16>(r, st);
    if (r.lanes == 32) return route<V, 32>(r, st);
    if (r.lanes == 64) return route<V, 64>(r, st);
  }
  route<V, 0>(r, st);
}

/* ---- the chosen pairs in order of their experts ------------------------------------------------------------------------
 * A stable sort by counting.  A workgroup takes a run of pairs, each of its 16 waves up to 8 times 64 neighbours: a pair's rank among the 64 of the same
 * expert comes from votes over the expert's bits, among the wave's before them from the wave's own counts in LDS.  Where there are more pairs than one
 * workgroup takes, a first launch leaves every run's counts, and each workgroup of the second adds up all runs' and those of the runs before its own.
 * What bounds it is the way of a few dependent steps: 131 072 pairs, 32 of 256 experts 3.8 + 6.2 us, 8192 pairs of 8 experts, one workgroup, 8.8 us, which saves a
 * launch (3 us of the host's time). */
struct Rows {
  const int32_t *experts;
  int64_t n, per; /* pairs, pairs of a run */
  int first, E, runs, bits;
  int32_t *offsets, *rows, *place, *counts; /* counts [runs][E] */
};
constexpr int WAVES = 16, THREADS = WAVES * 64, ROUNDS = 8;
constexpr int64_t PAIRS = THREADS * ROUNDS; /* that a workgroup takes at a time */

/* The lanes of the wave that hold the same number of `bits` bits. */
__device__ inline uint64_t alike(int e, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; b++) {
    uint64_t set = __ballot(e >> b & 1);
    m &= e >> b & 1 ? set : ~set;
  }
  return m;
}
__device__ inline int expert_of(const Rows &r, int64_t i, int64_t end) { /* E: left out */
  if (i >= end) return r.E;
  int64_t e = (int64_t)r.experts[i] - r.first;
  return e >= 0 && e < r.E ? (int)e : r.E;
}

/* Counts per wave in LDS; a chunk has up to PAIRS pairs, a wave `rounds` times 64 of them in a row. */
struct Counts { uint16_t of[WAVES][OOB_EXPERT_MAX + 2]; };

__device__ inline void count(const Rows &r, int64_t from, int64_t end, int rounds, Counts &c, int (&e)[ROUNDS], int (&rank)[ROUNDS]) {
  int wave = threadIdx.x / 64;
  volatile OOB_LDS uint16_t *mine = (OOB_LDS uint16_t *)c.of[wave];
  int64_t at = from + (int64_t)wave * rounds * 64 + lane();
#pragma unroll
  for (int i = 0; i < ROUNDS; i++) e[i] = i < rounds ? expert_of(r, at + i * 64, end) : r.E;
  for (int x = lane(); x <= r.E; x += 64) mine[x] = 0;
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int i = 0; i < ROUNDS; i++) {
    if (i >= rounds) break;
    uint64_t same = alike(e[i], r.bits);
    int before = mine[e[i]], in = __popcll(same & ((1ull << lane()) - 1));
    rank[i] = before + in;
    __builtin_amdgcn_wave_barrier();
    if (in == 0) mine[e[i]] = (uint16_t)(before + __popcll(same));
    __builtin_amdgcn_wave_barrier();
  }
  __syncthreads();
}
/* The counts of this thread's expert over the waves; they become what the waves before have. */
__device__ inline int waves_before(const Rows &r, Counts &c) {
  int all = 0;
  if ((int)threadIdx.x < r.E)
#pragma unroll
    for (int w = 0; w < WAVES; w++) {
      int n = c.of[w][threadIdx.x];
      c.of[w][threadIdx.x] = (uint16_t)all;
      all += n;
    }
  return all;
}
__device__ inline int rounds_of(int64_t pairs) { return pairs >= PAIRS ? ROUNDS : (int)((pairs + THREADS - 1) / THREADS); }

__global__ __launch_bounds__(THREADS) void k_rows_count(Rows r) {
  __shared__ Counts c;
  int64_t from = blockIdx.x * r.per, end = from + r.per < r.n ? from + r.per : r.n;
  int all = 0, e[ROUNDS], rank[ROUNDS];
  for (; from < end; from += PAIRS) {
    count(r, from, end, rounds_of(end - from), c, e, rank);
    all += waves_before(r, c);
    __syncthreads();
  }
  if ((int)threadIdx.x < r.E) r.counts[(int64_t)blockIdx.x * r.E + threadIdx.x] = all;
}

__global__ __launch_bounds__(THREADS) void k_rows(Rows r) {
  __shared__ Counts c;
  __shared__ int base[OOB_EXPERT_MAX + 1], total_of[OOB_EXPERT_MAX], sums[WAVES];
  int64_t from = blockIdx.x * r.per, end = from + r.per < r.n ? from + r.per : r.n;
  int e[ROUNDS], rank[ROUNDS], all = 0, before = 0, here = 0; /* of this thread's expert: pairs, those of earlier runs, those of this chunk */
  if (r.runs == 1) {
    count(r, from, end, rounds_of(end - from), c, e, rank);
    all = here = waves_before(r, c);
  } else {
    /* all threads share the counts: the threads of an expert every so many runs; whole numbers, so that the order of their additions does not count */
    int stride = 1;
    while (stride < r.E) stride *= 2;
    int x = threadIdx.x % stride, part = threadIdx.x / stride, parts = THREADS / stride;
    if ((int)threadIdx.x < r.E) base[threadIdx.x] = total_of[threadIdx.x] = 0;
    __syncthreads();
    if (x < r.E) {
#pragma unroll 8
      for (int i = part; i < r.runs; i += parts) {
        int n = r.counts[(int64_t)i * r.E + x];
        if (i < (int)blockIdx.x) before += n;
        all += n;
      }
      atomicAdd(base + x, before);
      atomicAdd(total_of + x, all);
    }
    __syncthreads();
    all = before = 0;
    if ((int)threadIdx.x < r.E) before = base[threadIdx.x], all = total_of[threadIdx.x];
  }
  int upto = all; /* pairs of the experts up to this thread's */
  for (int o = 1; o < 64; o *= 2) {
    int u = __shfl_up(upto, o);
    if (lane() >= o) upto += u;
  }
  if (lane() == 63) sums[threadIdx.x / 64] = upto;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < WAVES; w++) {
    if (w < (int)threadIdx.x / 64) upto += sums[w];
    total += sums[w];
  }
  if ((int)threadIdx.x < r.E) {
    base[threadIdx.x] = upto - all + before;
    if (blockIdx.x == 0) {
      r.offsets[threadIdx.x + 1] = upto;
      if (threadIdx.x == 0) r.offsets[0] = 0;
    }
  }
  for (bool counted = r.runs == 1; from < end; from += PAIRS, counted = false) {
    int rounds = rounds_of(end - from), wave = threadIdx.x / 64;
    if (!counted) {
      count(r, from, end, rounds, c, e, rank);
      here = waves_before(r, c);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < ROUNDS; i++) {
      int64_t at = from + ((int64_t)wave * rounds + i) * 64 + lane();
      if (i < rounds && at < end) {
        int row = e[i] < r.E ? base[e[i]] + c.of[wave][e[i]] + rank[i] : -1;
        r.place[at] = row;
        if (row >= 0) r.rows[row] = (int32_t)at;
        if (at >= total) r.rows[at] = -1; /* rows behind the last: no pair goes there */
      }
    }
    __syncthreads();
    if ((int)threadIdx.x < r.E) base[threadIdx.x] += here;
  }
}

/* One workgroup does what it takes at a time alone; beyond, runs of 1024 pairs or more, 256 at most. */
int64_t run_of(int64_t n) {
  if (n <= PAIRS) return PAIRS;
  int64_t run = up((n + 255) / 256, THREADS);
  return run <= PAIRS ? run : up(run, PAIRS);
}

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" int oob_expert_route(const oob_route *p, void *stream) {
  if (!route_ok(p, true)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  Route r{*p, 0, p->E / p->groups, 0, 0, 0};
  int groups = ceil2(p->groups), least = ceil2(p->k); /* lanes of a token: a power of two of them for each group */
  /* eight experts a lane where the waves fill the GPU all the same, four otherwise (16 tokens: 2.6 us) */
  int in_group = ceil2((r.per + 7) / 8);
  if (p->T * groups * in_group < 64 * 2048) in_group = ceil2((r.per + 3) / 4);
  while (groups * in_group > 64) in_group /= 2;
  while (groups * in_group < least) in_group *= 2;
  r.lanes = groups * in_group, r.in_group = in_group;
  int v = (r.per + in_group - 1) / in_group;
  size_t four = p->dtype == OOB_FP32 ? 16 : 8;
  r.whole = r.per % 4 == 0 && multiple(p->logits, four) && p->logits_stride % 4 == 0;
  r.whole_bias = r.per % 4 == 0 && multiple(p->bias, 16);
  hipStream_t st = (hipStream_t)stream;
  for (int64_t t = 0, n = tokens_of(r.lanes); t < p->T; t += n) {
    r.p = part_of(*p, t, n);
    if (v <= 1) route<1>(r, st);
    else if (v <= 2) route<2>(r, st);
    else if (v <= 4) route<4>(r, st);
    else if (v <= 8) route<8>(r, st);
    else if (v <= 16) route<16>(r, st);
    else route<32>(r, st);
  }
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

extern "C" int oob_expert_route_backward(const oob_route *p, const float *dweights, void *dlogits, int64_t dlogits_stride, void *stream) {
  if (!route_ok(p, false)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  size_t of = p->dtype == OOB_FP32 ? 4 : 2;
  if (!dweights || !dlogits || dlogits_stride < p->E || !multiple(dweights, 4) || !multiple(dlogits, of)) return OOB_EINVAL;
  RouteGrad g{*p, dweights, dlogits, dlogits_stride, 0, p->E % 4 == 0 && dlogits_stride % 4 == 0 && multiple(dlogits, 4 * of)};
  int lanes = ceil2((p->E + 7) / 8), least = ceil2(p->k);
  g.lanes = lanes > 64 ? 64 : lanes < least ? least : lanes;
  for (int64_t t = 0, n = tokens_of(g.lanes); t < p->T; t += n) {
    g.p = part_of(*p, t, n), g.dweights = dweights + t * p->k, g.dlogits = (char *)dlogits + t * dlogits_stride * of;
    k_route_grad<<<(unsigned)((g.p.T * g.lanes + 255) / 256), 256, 256 / g.lanes * p->E * 4, (hipStream_t)stream>>>(g);
  }
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

extern "C" size_t oob_expert_rows_workspace_size(int64_t n, int E) {
  if (n < 1 || n >= (int64_t)1 << 31 || E < 1 || E > OOB_EXPERT_MAX) return 0;
  int64_t runs = (n + run_of(n) - 1) / run_of(n);
  return runs == 1 ? 0 : (size_t)up(runs * E * 4, 256);
}

extern "C" int oob_expert_rows(const int32_t *experts, int64_t n, int first, int E, int32_t *offsets, int32_t *rows, int32_t *place, void *workspace,
                               size_t bytes, void *stream) {
  if (n < 0 || n >= (int64_t)1 << 31 || E < 1 || E > OOB_EXPERT_MAX || !offsets || (n && (!experts || !rows || !place))) return OOB_EINVAL;
  if (!multiple(experts, 4) || !multiple(offsets, 4) || !multiple(rows, 4) || !multiple(place, 4) || !multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = oob_expert_rows_workspace_size(n, E);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Rows r{experts, n, run_of(n), first, E, 1, 0, offsets, rows, place, (int32_t *)workspace};
  if (n) r.runs = (int)((n + r.per - 1) / r.per);
  while (1 << r.bits <= E) r.bits++; /* E itself stands for those left out */
  hipStream_t st = (hipStream_t)stream;
  if (r.runs > 1) k_rows_count<<<r.runs, THREADS, 0, st>>>(r);
  k_rows<<<r.runs, THREADS, 0, st>>>(r);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}
