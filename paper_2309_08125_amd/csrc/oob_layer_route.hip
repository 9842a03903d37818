/* Routing to experts and the chosen pairs in order of their experts. */
#include "oob_expert.h"
#include "oob_layer_device.h"

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

/* Over runs of `lanes` lanes (a power of two). */
template <class K> __device__ inline K max_over(K v, int lanes) {
  for (int o = 1; o < lanes; o *= 2) {
    K u = __shfl_xor(v, o);
    v = u > v ? u : v;
  }
  return v;
}
template <class K> __device__ inline K sum_over(K v, int lanes) {
  for (int o = 1; o < lanes; o *= 2) v += __shfl_xor(v, o);
  return v;
}
/* The first lane of this lane's run for which `is` holds, counted in the run; -1: none. */
__device__ inline int first_of(bool is, int lanes) {
  uint64_t who = __ballot(is) >> (lane() & ~(lanes - 1));
  if (lanes < 64) who &= (1ull << lanes) - 1;
  return __ffsll((unsigned long long)who) - 1;
}

/* Numbers in the order of what they stand for: 0 is nothing (absent or taken), 1 a NaN, -inf and all else above. */
__device__ inline uint32_t key_of(float v) {
  if (v != v) return 1;
  uint32_t b = __float_as_uint(v + 0.f); /* -0 is 0 */
  return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ inline uint64_t key_of(double v) {
  if (v != v) return 1;
  uint64_t b = (uint64_t)__double_as_longlong(v + 0.);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

/* sigmoid(l) e^-m: with m the largest min(l, 0) of several, their ratios keep all digits however small they are. */
__device__ inline float sigmoid_over(float l, float m) { return expf(fminf(l, 0.f) - m) / (1 + expf(-fabsf(l))); }

/* ---- routing -------------------------------------------------------------------------------------------------------------
 * A token takes a run of lanes, each V neighbouring experts of one group: a choice is a maximum over registers, then over the run; of
 * equals the first expert is that of the first lane that holds it, which a vote finds. */
struct Route {
  oob_route p;
  int lanes;    /* a token's: a power of two, at least k */
  int per;      /* experts of a group */
  int in_group; /* lanes of a group: a power of two */
};

template <int V, bool SCORES> __global__ __launch_bounds__(256) void k_route(Route r) {
  using K = std::conditional_t<SCORES, uint64_t, uint32_t>;
  const oob_route &p = r.p;
  const int L = r.lanes, l = lane() & (L - 1);
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool live = t < p.T; /* runs of lanes as a whole: the others take part in the exchanges and write nothing */
  const int group = l / r.in_group, in = l % r.in_group * V, e0 = group * r.per + in;
  const int there = group < p.groups ? r.per - in : 0; /* of this lane's experts: so many exist */
  float x[V], top = -INFINITY;
  for (int i = 0; i < V; i++) {
    x[i] = live && i < there ? logit(p.logits, p.dtype, t * p.logits_stride + e0 + i) : -INFINITY;
    top = fmaxf(top, x[i]);
  }
  if (p.score == OOB_ROUTE_SOFTMAX) top = max_over(top, L);

  K key[V];
  double total = 0; /* of softmax */
  if constexpr (SCORES) { /* in 64 bits: sums of a score and a bias that lie close are told apart as a 64-bit program does */
    double s[V];
    for (int i = 0; i < V; i++) {
      s[i] = x[i] == -INFINITY ? 0. : p.score == OOB_ROUTE_SOFTMAX ? exp((double)x[i] - (double)top) : 1 / (1 + exp(-(double)x[i]));
      total += s[i];
    }
    if (p.score == OOB_ROUTE_SOFTMAX) total = sum_over(total, L);
    double best = -INFINITY, next = -INFINITY; /* of the group */
    for (int i = 0; i < V; i++) {
      double c = -INFINITY;
      if (x[i] != -INFINITY) {
        c = p.score == OOB_ROUTE_SOFTMAX ? s[i] / total : s[i];
        if (p.bias) c += p.bias[e0 + i];
      }
      key[i] = i < there ? key_of(c) : 0;
      if (c > best) next = best, best = c;
      else if (c > next) next = c;
    }
    if (p.groups > 1) {
      for (int o = 1; o < r.in_group; o *= 2) {
        double b = __shfl_xor(best, o), n = __shfl_xor(next, o);
        double low = b > best ? best : b; /* second of the four: the lower first or one of the seconds */
        best = b > best ? b : best;
        n = n > next ? n : next;
        next = low > n ? low : n;
      }
      uint64_t of = group < p.groups ? key_of(p.group_best == 2 && r.per > 1 ? best + next : best) : 0;
      bool kept = false;
      for (int n = 0; n < p.keep_groups; n++) {
        int won = first_of(of == max_over(of, L), L) / r.in_group;
        if (group == won) kept = true, of = 0;
      }
      if (!kept)
        for (int i = 0; i < V; i++) key[i] = 0;
    }
  } else {
    for (int i = 0; i < V; i++) key[i] = i < there ? key_of(x[i]) : 0;
  }

  float mine = -INFINITY; /* lane j gets the logit of choice j */
  for (int j = 0; j < p.k; j++) {
    K best = key[0];
    for (int i = 1; i < V; i++) best = key[i] > best ? key[i] : best;
    K most = max_over(best, L);
    int won = first_of(best == most, L), at = 0; /* the maximum is never 0: k experts are there */
    float value = 0;
    if (l == won) {
      for (int i = V - 1; i >= 0; i--)
        if (key[i] == most) at = i, value = x[i];
      for (int i = 0; i < V; i++)
        if (i == at) key[i] = 0;
    }
    int from = (lane() & ~(L - 1)) + won;
    value = __shfl(value, from);
    int number = __shfl(e0 + at, from);
    if (l == j) {
      mine = value;
      if (live) p.experts[t * p.k + j] = number;
    }
  }

  const bool has = l < p.k;
  float w;
  if (p.renormalize) {
    float m = max_over(!has || mine != mine ? -INFINITY : p.score == OOB_ROUTE_SIGMOID ? fminf(mine, 0.f) : mine, L);
    float s = !has || mine == -INFINITY ? 0.f : p.score == OOB_ROUTE_SIGMOID ? sigmoid_over(mine, m) : expf(mine - m);
    float all = sum_over(s, L);
    w = all == 0 ? 0.f : s / all;
  } else if (p.score == OOB_ROUTE_SIGMOID) {
    w = sigmoid_over(mine, 0.f);
  } else {
    float all = (float)total;
    if (!SCORES) {
      for (int i = 0; i < V; i++) all += x[i] == -INFINITY ? 0.f : expf(x[i] - top);
      all = sum_over(all, L);
    }
    w = mine == -INFINITY ? 0.f : expf(mine - top) / all;
  }
  if (live && has) p.weights[t * p.k + l] = w * p.scale;
}

/* ---- its gradient: a token takes a run of lanes, lane j its choice j; the row is put together in LDS, where the choices add to it
 * one after the other. */
struct RouteGrad {
  oob_route p;
  const float *dweights;
  void *dlogits;
  int64_t ld;
  int lanes;
};

__global__ __launch_bounds__(256) void k_route_grad(RouteGrad g) {
  extern __shared__ float rows[];
  const oob_route &p = g.p;
  const int L = g.lanes, l = lane() & (L - 1);
  const int64_t t = ((int64_t)blockIdx.x * 256 + threadIdx.x) / L;
  const bool live = t < p.T;
  volatile float *row = rows + threadIdx.x / L * p.E;

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
  if (live)
    for (int i = l; i < p.E; i += L) put(g.dlogits, p.dtype, t * g.ld + i, row[i]);
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
  if (!p->logits || p->logits_stride < p->E || !p->experts || !multiple(p->logits, of) || !multiple(p->experts, 4)) return false;
  return !forward || (p->weights && multiple(p->weights, 4) && multiple(p->bias, 4));
}

template <int V> void route(const Route &r, hipStream_t st) {
  unsigned n = (unsigned)((r.p.T * r.lanes + 255) / 256);
  if (r.p.bias || r.p.groups > 1) k_route<V, true><<<n, 256, 0, st>>>(r);
  else k_route<V, false><<<n, 256, 0, st>>>(r);
}

/* ---- the chosen pairs in order of their experts ------------------------------------------------------------------------
 * A stable sort by counting.  A workgroup takes a run of pairs, 1024 at a time, a wave 64 of them; a pair's rank among the wave's of the same
 * expert comes from votes over the expert's bits, the counts of the waves lie in LDS.  Where there are more pairs than one workgroup takes, a first launch
 * leaves every run's counts, and each workgroup of the second adds up those of the runs before its own. */
struct Rows {
  const int32_t *experts;
  int64_t n, per; /* pairs, pairs of a run (a multiple of 1024) */
  int first, E, runs, bits;
  int32_t *offsets, *rows, *place, *counts; /* counts [runs][E] */
};
constexpr int PAIRS = 1024, WAVES = PAIRS / 64;

/* The lanes of the wave that hold the same number of `bits` bits. */
__device__ inline uint64_t alike(int e, int bits) {
  uint64_t m = ~0ull;
  for (int b = 0; b < bits; b++) {
    uint64_t set = __ballot(e >> b & 1);
    m &= e >> b & 1 ? set : ~set;
  }
  return m;
}
__device__ inline int expert_of(const Rows &r, int64_t i) { /* E: left out */
  if (i >= r.n) return r.E;
  int64_t e = (int64_t)r.experts[i] - r.first;
  return e >= 0 && e < r.E ? (int)e : r.E;
}

/* Counts of a run's experts to `count` in LDS [E + 1]. */
__device__ inline void count_run(const Rows &r, int64_t from, int64_t to, int *count) {
  for (int e = threadIdx.x; e <= r.E; e += PAIRS) count[e] = 0;
  __syncthreads();
  for (int64_t at = from; at < to; at += PAIRS) {
    int e = expert_of(r, at + threadIdx.x);
    uint64_t same = alike(e, r.bits);
    if (__ffsll((unsigned long long)same) - 1 == lane()) atomicAdd(count + e, __popcll(same)); /* whole numbers: their order does not count */
  }
  __syncthreads();
}

__global__ __launch_bounds__(PAIRS) void k_rows_count(Rows r) {
  __shared__ int count[OOB_EXPERT_MAX + 1];
  int64_t from = blockIdx.x * r.per, to = from + r.per < r.n ? from + r.per : r.n;
  count_run(r, from, to, count);
  for (int e = threadIdx.x; e < r.E; e += PAIRS) r.counts[(int64_t)blockIdx.x * r.E + e] = count[e];
}

__global__ __launch_bounds__(PAIRS) void k_rows(Rows r) {
  __shared__ int base[OOB_EXPERT_MAX + 1];             /* the next row of each expert; before that, this run's counts */
  __shared__ uint16_t of_wave[WAVES][OOB_EXPERT_MAX + 2]; /* counts of a wave, then what the waves before it have */
  __shared__ int sums[WAVES];
  int64_t from = blockIdx.x * r.per, to = from + r.per < r.n ? from + r.per : r.n;
  int all = 0, before = 0; /* of this thread's expert: pairs, and those of earlier runs */
  if (r.runs == 1) {
    count_run(r, from, to, base);
    if ((int)threadIdx.x < r.E) all = base[threadIdx.x];
    __syncthreads();
  } else if ((int)threadIdx.x < r.E) {
    for (int i = 0; i < r.runs; i++) {
      int c = r.counts[(int64_t)i * r.E + threadIdx.x];
      if (i < (int)blockIdx.x) before += c;
      all += c;
    }
  }
  int end = all; /* of the experts up to this thread's */
  for (int o = 1; o < 64; o *= 2) {
    int u = __shfl_up(end, o);
    if (lane() >= o) end += u;
  }
  if (lane() == 63) sums[threadIdx.x / 64] = end;
  __syncthreads();
  int total = 0;
  for (int w = 0; w < WAVES; w++) {
    if (w < (int)threadIdx.x / 64) end += sums[w];
    total += sums[w];
  }
  if ((int)threadIdx.x < r.E) {
    base[threadIdx.x] = end - all + before;
    if (blockIdx.x == 0) {
      r.offsets[threadIdx.x + 1] = end;
      if (threadIdx.x == 0) r.offsets[0] = 0;
    }
  }
  __syncthreads();
  for (int64_t at = from; at < to; at += PAIRS) {
    int64_t i = at + threadIdx.x;
    int e = expert_of(r, i), wave = threadIdx.x / 64;
    uint64_t same = alike(e, r.bits);
    int rank = __popcll(same & ((1ull << lane()) - 1));
    for (int x = threadIdx.x; x < WAVES * (r.E + 1); x += PAIRS) of_wave[x / (r.E + 1)][x % (r.E + 1)] = 0;
    __syncthreads();
    if (rank == 0) of_wave[wave][e] = (uint16_t)__popcll(same);
    __syncthreads();
    int more = 0;
    if ((int)threadIdx.x < r.E)
      for (int w = 0; w < WAVES; w++) {
        int c = of_wave[w][threadIdx.x];
        of_wave[w][threadIdx.x] = (uint16_t)more;
        more += c;
      }
    __syncthreads();
    if (i < r.n) {
      int row = e < r.E ? base[e] + of_wave[wave][e] + rank : -1;
      r.place[i] = row;
      if (row >= 0) r.rows[row] = (int32_t)i;
      if (i >= total) r.rows[i] = -1; /* rows behind the last: no pair goes there */
    }
    __syncthreads();
    if ((int)threadIdx.x < r.E) base[threadIdx.x] += more;
  }
}

/* Pairs of a run: one workgroup does the smallest numbers alone; beyond, 1024 each as long as there are no more than 256 runs. */
int64_t run_of(int64_t n) { return n <= PAIRS * 2 ? up(n, PAIRS) : up((n + 255) / 256, PAIRS); }

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" int oob_expert_route(const oob_route *p, void *stream) {
  if (!route_ok(p, true)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  Route r{*p, 0, p->E / p->groups, 0};
  int groups = ceil2(p->groups), least = ceil2(p->k); /* lanes of a token: a power of two of them for each group */
  int in_group = ceil2((r.per + 3) / 4);              /* four experts a lane where there are enough lanes */
  while (groups * in_group > 64) in_group /= 2;
  while (groups * in_group < least) in_group *= 2;
  r.lanes = groups * in_group, r.in_group = in_group;
  int v = (r.per + in_group - 1) / in_group;
  hipStream_t st = (hipStream_t)stream;
  if (v <= 1) route<1>(r, st);
  else if (v <= 2) route<2>(r, st);
  else if (v <= 4) route<4>(r, st);
  else if (v <= 8) route<8>(r, st);
  else if (v <= 16) route<16>(r, st);
  else route<32>(r, st);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

extern "C" int oob_expert_route_backward(const oob_route *p, const float *dweights, void *dlogits, int64_t dlogits_stride, void *stream) {
  if (!route_ok(p, false)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  size_t of = p->dtype == OOB_FP32 ? 4 : 2;
  if (!dweights || !dlogits || dlogits_stride < p->E || !multiple(dweights, 4) || !multiple(dlogits, of)) return OOB_EINVAL;
  RouteGrad g{*p, dweights, dlogits, dlogits_stride, 0};
  int lanes = ceil2((p->E + 7) / 8), least = ceil2(p->k);
  g.lanes = lanes > 64 ? 64 : lanes < least ? least : lanes;
  unsigned n = (unsigned)((p->T * g.lanes + 255) / 256);
  k_route_grad<<<n, 256, 256 / g.lanes * p->E * 4, (hipStream_t)stream>>>(g);
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
  Rows r{experts, n, n ? run_of(n) : PAIRS, first, E, 1, 0, offsets, rows, place, (int32_t *)workspace};
  if (n) r.runs = (int)((n + r.per - 1) / r.per);
  while (1 << r.bits <= E) r.bits++; /* E itself stands for those left out */
  hipStream_t st = (hipStream_t)stream;
  if (r.runs > 1) k_rows_count<<<r.runs, PAIRS, 0, st>>>(r);
  k_rows<<<r.runs, PAIRS, 0, st>>>(r);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}
