/* The norm over many tensors, and the tensors scaled so that it does not pass a bound. */
#include <algorithm>
#include <utility>
#include <vector>

#include "oob_expert.h"
#include "oob_layer_device.h"

namespace layer {
namespace {

/* Tensors of one launch: their addresses travel with the launch's arguments (4 KB), nothing is copied to the device.  Few tensors take a launch with fewer
 * arguments, which is quicker to enqueue. */
constexpr int TENSORS = 112, FEW = 24;
constexpr int64_t CHUNK = 32768; /* values a workgroup takes at a time */
constexpr int64_t MOST = 0x7f000000; /* chunks of a launch */
constexpr int GROUPS = 2048;     /* workgroups of a launch at most, so that every workgroup of the second pass can add up their sums itself */
template <int N> struct Tensors {
  const void *from[N];
  void *to[N];
  int64_t sizes[N];
  int32_t until[N]; /* chunks of the tensors up to this one */
  uint8_t types[N];
  int n;
};
static_assert(sizeof(Tensors<TENSORS>) <= 3800, "arguments of a launch");

template <int N> __device__ inline int find(const Tensors<N> &t, int chunk, int64_t &first) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    int mid = (lo + hi) / 2;
    if (chunk < t.until[mid]) hi = mid;
    else lo = mid + 1;
  }
  first = (int64_t)(chunk - (lo ? t.until[lo - 1] : 0)) * CHUNK;
  return lo;
}

/* Sum over the workgroup, in a fixed order. */
__device__ inline double total_of(double s) {
  __shared__ double part[4];
  for (int o = 1; o < 64; o *= 2) s += __shfl_xor(s, o);
  __syncthreads();
  if (lane() == 0) part[threadIdx.x / 64] = s;
  __syncthreads();
  return (part[0] + part[1]) + (part[2] + part[3]);
}

/* Memory bounds both passes: 805 million values of bfloat16 in 48 tensors 300 us (5.4 TB/s) and, out of place, 641 us (5.0 TB/s).
 * Squares are summed in 64 bits: those of bfloat16 and float32 pass the range of 32 (values beyond 1.8e19 or below 1e-19), and a sum of 10^9
 * terms its digits. */
template <class E> __device__ inline double squares(const E *from, int64_t size, int64_t first) {
  int64_t last = first + CHUNK < size ? first + CHUNK : size;
  double s = 0;
  for (int64_t i = first + threadIdx.x * 8; i < last; i += 256 * 8 * 4) {
    typename Vec<E>::v8 v[4]; /* four loads on their way */
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (i + u * 2048 < last) v[u] = load8<E>(from + i + u * 2048, last - (i + u * 2048));
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (i + u * 2048 < last)
        for (int e = 0; e < 8; e++) s += (double)(float)v[u][e] * (double)(float)v[u][e];
  }
  return s;
}

template <int N> __global__ __launch_bounds__(256) void k_squares(Tensors<N> t, double *sums) {
  double s = 0;
  for (int c = blockIdx.x; c < t.until[t.n - 1]; c += gridDim.x) {
    int64_t first;
    int i = find(t, c, first);
    if (t.types[i] == OOB_FP32) s += squares((const float *)t.from[i], t.sizes[i], first);
    else if (t.types[i] == OOB_BF16) s += squares((const bf16 *)t.from[i], t.sizes[i], first);
    else s += squares((const fp16 *)t.from[i], t.sizes[i], first);
  }
  s = total_of(s);
  if (threadIdx.x == 0) sums[blockIdx.x] = s;
}

__device__ inline double add_up(const double *sums, int n) {
  double s = 0;
  for (int i = threadIdx.x; i < n; i += 256) s += sums[i];
  return total_of(s);
}

__global__ __launch_bounds__(256) void k_norm(const double *sums, int n, float *norm) {
  double s = sqrt(add_up(sums, n));
  if (threadIdx.x == 0) *norm = (float)s;
}

template <class E, class F> __device__ inline void scale(const E *from, E *to, int64_t size, int64_t first, F factor) {
  int64_t last = first + CHUNK < size ? first + CHUNK : size;
  for (int64_t i = first + threadIdx.x * 8; i < last; i += 256 * 8 * 4) {
    typename Vec<E>::v8 v[4];
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (i + u * 2048 < last) v[u] = load8<E>(from + i + u * 2048, last - (i + u * 2048));
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (i + u * 2048 < last) {
        if (factor != 1)
          for (int e = 0; e < 8; e++) v[u][e] = (E)(float)((F)(float)v[u][e] * factor);
        store8<E>(to + i + u * 2048, v[u], last - (i + u * 2048));
      }
  }
}

template <int N, class F> __device__ inline void scale_one(const Tensors<N> &t, int i, int64_t first, F factor) {
  if (t.types[i] == OOB_FP32) scale((const float *)t.from[i], (float *)t.to[i], t.sizes[i], first, factor);
  else if (t.types[i] == OOB_BF16) scale((const bf16 *)t.from[i], (bf16 *)t.to[i], t.sizes[i], first, factor);
  else scale((const fp16 *)t.from[i], (fp16 *)t.to[i], t.sizes[i], first, factor);
}

/* Each workgroup adds up the first pass's sums itself, in the same order, in place of a launch between the two. */
template <int N> __global__ __launch_bounds__(256) void k_scale(Tensors<N> t, const double *sums, int n, float max_norm, const float *given, float *norm) {
  float s = given ? *given : (float)sqrt(add_up(sums, n)); /* as it is returned: one that is given back does the same */
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = s;
  double factor = s > max_norm && s < INFINITY ? (double)max_norm / s : 1;
  bool small = factor < 0x1p-126; /* below, 32 bits lose its digits: the products are formed in 64 */
  int chunks = t.until[t.n - 1];
  for (int c = chunks - 1 - (int)blockIdx.x; c >= 0; c -= gridDim.x) { /* from the end: what was read last is still in the last-level cache */
    int64_t first;
    int i = find(t, c, first);
    if ((float)factor == 1.f && t.to[i] == t.from[i]) continue;
    if (small) scale_one(t, i, first, factor);
    else scale_one(t, i, first, (float)factor);
  }
}

bool tensors_ok(int n, const void *const *from, void *const *to, const int64_t *sizes, const int *types) {
  if (n < 0 || (n && (!from || !sizes || !types))) return false;
  for (int i = 0; i < n; i++) {
    if (types[i] != OOB_BF16 && types[i] != OOB_FP16 && types[i] != OOB_FP32) return false;
    size_t of = types[i] == OOB_FP32 ? 4 : 2;
    if (sizes[i] < 0 || sizes[i] >= (int64_t)1 << 40) return false;
    if (sizes[i] && (!from[i] || !multiple(from[i], of) || (to && (!to[i] || !multiple(to[i], of))))) return false;
  }
  return true;
}

/* Memory that is written and written or read by others. */
bool overlap(int n, const void *const *from, const void *const *to, const int64_t *sizes, const int *types, const void *given) try {
  using Part = std::pair<uintptr_t, uintptr_t>;
  std::vector<Part> parts;
  auto part = [&](const void *p, int i) { return Part{(uintptr_t)p, (uintptr_t)p + (uintptr_t)sizes[i] * (types[i] == OOB_FP32 ? 4 : 2)}; };
  for (int i = 0; i < n; i++)
    if (sizes[i]) parts.push_back(part(to[i], i));
  std::sort(parts.begin(), parts.end());
  for (size_t i = 1; i < parts.size(); i++)
    if (parts[i].first < parts[i - 1].second) return true;
  auto written = [&](Part p) { /* the parts do not overlap: only the last that begins before p's end can reach into it */
    auto after = std::lower_bound(parts.begin(), parts.end(), Part{p.second, 0});
    return after != parts.begin() && std::prev(after)->second > p.first;
  };
  for (int i = 0; i < n; i++)
    if (sizes[i] && from[i] != to[i] && written(part(from[i], i))) return true;
  return given && written({(uintptr_t)given, (uintptr_t)given + 4});
} catch (...) { /* no host memory: refused, nothing passes the C entry */
  return true;
}

/* The norm is written while other workgroups still read and write the tensors. */
bool norm_shared(int n, const void *const *from, const int64_t *sizes, const int *types, const float *norm) {
  for (int i = 0; i < n; i++)
    if (share({norm, 1, 4, 0}, lies_flat(from[i], sizes[i] * (types[i] == OOB_FP32 ? 4 : 2)))) return true;
  return false;
}

/* The next launch's tensors from number `at` on: those with values, as many as fit. */
template <int N> bool next(int &at, int n, const void *const *from, void *const *to, const int64_t *sizes, const int *types, Tensors<N> &t) {
  int64_t chunks = 0;
  for (t.n = 0; at < n && t.n < N; at++) {
    if (sizes[at] > 0) {
      int64_t more = (sizes[at] + CHUNK - 1) / CHUNK;
      if (chunks + more > MOST) break;
      chunks += more;
      t.from[t.n] = from[at], t.to[t.n] = to ? to[at] : nullptr;
      t.sizes[t.n] = sizes[at], t.until[t.n] = (int32_t)chunks, t.types[t.n] = (uint8_t)types[at];
      t.n++;
    }
  }
  return t.n > 0;
}
int groups_of(int64_t chunks) { return chunks < GROUPS ? (int)chunks : GROUPS; }

/* Sums of the first pass at most: every launch's workgroups, in launches of either kind. */
int64_t sums_of(int n, const int64_t *sizes) {
  int64_t chunks = 0, launches = n <= FEW ? 1 : (n + TENSORS - 1) / TENSORS;
  for (int i = 0; i < n; i++) chunks += (sizes[i] + CHUNK - 1) / CHUNK;
  launches += chunks / (MOST / 2); /* a launch that ends early holds more than half of what it may */
  return chunks < launches * GROUPS ? chunks : launches * GROUPS;
}

template <int N> int first_pass(int n, const void *const *from, const int64_t *sizes, const int *types, double *sums, hipStream_t st) {
  Tensors<N> t;
  int at = 0, done = 0;
  while (next(at, n, from, nullptr, sizes, types, t)) {
    int groups = groups_of(t.until[t.n - 1]);
    k_squares<<<groups, 256, 0, st>>>(t, sums + done);
    done += groups;
  }
  return done;
}
int first_pass(int n, const void *const *from, const int64_t *sizes, const int *types, double *sums, hipStream_t st) {
  return n <= FEW ? first_pass<FEW>(n, from, sizes, types, sums, st) : first_pass<TENSORS>(n, from, sizes, types, sums, st);
}

template <int N> int second_pass(int n, const void *const *from, void *const *to, const int64_t *sizes, const int *types, const double *sums, int count,
                                 float max_norm, const float *given, float *norm, hipStream_t st) {
  Tensors<N> t;
  int at = 0, launches = 0;
  while (next(at, n, from, to, sizes, types, t)) {
    k_scale<<<groups_of(t.until[t.n - 1]), 256, 0, st>>>(t, sums, count, max_norm, given, launches ? nullptr : norm);
    launches++;
  }
  return launches;
}

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" size_t oob_clip_workspace_size(int n, const int64_t *sizes) {
  if (n < 0 || !sizes) return 0;
  for (int i = 0; i < n; i++)
    if (sizes[i] < 0 || sizes[i] >= (int64_t)1 << 40) return 0;
  return (size_t)up(sums_of(n, sizes) * 8, 256);
}

extern "C" int oob_clip_overlap(int n, const void *const *from, const void *const *to, const int64_t *sizes, const int *types, const float *given) {
  return n > 0 && from && to && sizes && types && overlap(n, from, to, sizes, types, given);
}

extern "C" int oob_clip_norm(int n, const void *const *from, const int64_t *sizes, const int *types, float *norm, void *workspace, size_t bytes,
                             void *stream) {
  if (!tensors_ok(n, from, nullptr, sizes, types) || !norm || !multiple(norm, 4) || !multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = n ? oob_clip_workspace_size(n, sizes) : 0;
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  hipStream_t st = (hipStream_t)stream;
  int sums = first_pass(n, from, sizes, types, (double *)workspace, st);
  k_norm<<<1, 256, 0, st>>>((const double *)workspace, sums, norm);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

extern "C" int oob_clip_scale(int n, const void *const *from, void *const *to, const int64_t *sizes, const int *types, float max_norm,
                              const float *given, float *norm, void *workspace, size_t bytes, void *stream) {
  if (!tensors_ok(n, from, to, sizes, types) || (n && !to) || !(max_norm >= 0) || !multiple(workspace, 256)) return OOB_EINVAL;
  if (!multiple(given, 4) || !multiple(norm, 4) || (!given && !norm) || overlap(n, from, to, sizes, types, given)) return OOB_EINVAL;
  size_t need = n && !given ? oob_clip_workspace_size(n, sizes) : 0;
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  if (!given && (norm_shared(n, from, sizes, types, norm) || norm_shared(n, to, sizes, types, norm))) return OOB_EINVAL;
  hipStream_t st = (hipStream_t)stream;
  double *sums = (double *)workspace;
  int count = given ? 0 : first_pass(n, from, sizes, types, sums, st);
  if (given) norm = nullptr;
  int launches = n <= FEW ? second_pass<FEW>(n, from, to, sizes, types, sums, count, max_norm, given, norm, st)
                          : second_pass<TENSORS>(n, from, to, sizes, types, sums, count, max_norm, given, norm, st);
  if (norm && !launches) k_norm<<<1, 256, 0, st>>>(sums, 0, norm);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}
