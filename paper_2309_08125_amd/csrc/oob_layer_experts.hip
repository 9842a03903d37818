/* Every expert's rows through its own matrix, y[r] = act(x[token(r)] W[e]^T + b[e]), and the gradients. */
#include "oob_expert.h"
#include "oob_layer_product.h"

namespace layer {
namespace {

/* ---- which rows are whose --------------------------------------------------------------------------------------------------
 * The host knows the number of rows, not how they divide: launches are as large as the worst division needs (a partly filled tile
 * for every expert), and each workgroup finds its expert from the offsets, a run of experts per lane, and leaves if there is nothing for it. */
struct Division { const int32_t *offsets; int E; int64_t R; };

__device__ inline int64_t bound(const Division &d, int e) {
  int64_t o = d.offsets[e];
  return o < 0 ? 0 : o > d.R ? d.R : o;
}
__device__ inline int64_t rows_of(const Division &d, int e, int64_t &first) {
  first = bound(d, e);
  int64_t n = bound(d, e + 1) - first;
  return n > 0 ? n : 0;
}

struct Found { int expert, first, rows, part; }; /* expert: -1 past the last; part: which of the expert's pieces */

/* Piece id_of(pieces of all) where an expert with n rows has pieces_of(n); the same for all lanes of the wave, in scalar registers. */
template <class P, class I> __device__ inline Found find(const Division &d, P pieces_of, I id_of) {
  int per = (d.E + 63) / 64, e0 = lane() * per;
  int64_t mine = 0, first;
  for (int i = 0; i < per; i++)
    if (e0 + i < d.E) mine += pieces_of(rows_of(d, e0 + i, first));
  int64_t end = mine;
  for (int o = 1; o < 64; o *= 2) {
    int64_t u = __shfl_up(end, o);
    if (lane() >= o) end += u;
  }
  Found f{-1, 0, 0, 0};
  int64_t all = __shfl(end, 63);
  int total = uniform((int)(all < 0x7fffffff ? all : 0x7fffffff)), id = id_of(total); /* no launch has more workgroups */
  if (id >= total) return f;
  int owner = __ffsll((unsigned long long)__ballot(end > id)) - 1;
  int64_t at = id - (end - mine), rows = 0;
  int e = e0;
  if (lane() == owner)
    for (int i = 0; i < per; i++) {
      rows = rows_of(d, e0 + i, first);
      int64_t n = pieces_of(rows);
      e = e0 + i;
      if (at < n) break;
      at -= n;
    }
  f.expert = uniform(__shfl(e, owner));
  f.first = uniform(__shfl((int)first, owner)), f.rows = uniform(__shfl((int)rows, owner)), f.part = uniform(__shfl((int)at, owner));
  return f;
}

/* ---- the products: the tiles of a dense product (oob_layer_product.h), an expert's rows in place of all ---------------------- */
struct Experts {
  Product g; /* A: rows of all experts (or of x, where they are gathered); B, bias: of expert 0 */
  Division d;
  const int32_t *rows; /* gathered: row r of A is that of token rows[r] / per */
  int per;
  int64_t T, expert_stride; /* elements of B between experts */
  int ids; /* numbers of tiles: as many as there can be */
};

/* An operand's tile of ROWS x KSTEP on its way to LDS, laid out as Tile has it: the 16 bytes that a lane takes with its i-th load lie a fixed way from those
 * of its first, so that it holds one offset, not one for each. */
template <class E, int ROWS, int THREADS, bool KC> struct Strip {
  static constexpr int BYTES = ROWS * KSTEP * 2, LOADS = BYTES / (THREADS * 16), APART = KC ? THREADS * 16 / 128 : THREADS * 16 / (ROWS * 2);
  static_assert(APART % (KC ? 16 : 4) == 0, "the exchange of chunks is the same for all of a lane's loads");
  uint32_t off, way; /* byte offset of the first from the start of the step, bytes to the next */
  int k, row, left;  /* first k of the 16 bytes (k contiguous) or row of k; row of m (k contiguous), rows there are */

  __device__ void init(int64_t ld, int64_t rows) { /* rows: of m (n), from the tile's first on */
    int p = threadIdx.x * 16;
    left = (int)(rows < ROWS ? rows : ROWS), way = (uint32_t)(APART * ld * 2);
    if (KC) {
      int r = p / 128, c = (p / 16 % 8) ^ (r / 2 % 8);
      k = c * 8, row = r, off = (uint32_t)(r * ld * 2 + c * 16);
    } else {
      constexpr int CH = ROWS / 8;
      int r = p / (ROWS * 2), c = (p / 16 % CH) ^ (ROWS == 64 ? r / 2 % 2 * 4 : r % 4 * 4);
      k = r, row = 0, off = c * 8 < left ? (uint32_t)(r * ld * 2 + c * 16) : OOB_LAYER_OUT;
    }
  }
  /* Asks for the step that starts at `base`; kleft: values of k there are from here on, 0 or less: zeros land, nothing is read. */
  __device__ void load(const char *base, lds_char *to, int kleft) {
    __amdgpu_buffer_rsrc_t r = buffer(base);
    int wave = uniform(threadIdx.x / 64);
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      bool in = KC ? k < kleft && row + i * APART < left : k + i * APART < kleft;
      load_lds(r, to + (i * THREADS + wave * 64) * 16, in ? off : OOB_LAYER_OUT, i * way);
    }
  }
};

/* Rows of k that lie anywhere: each lane's offsets come from the rows' tokens. */
template <class E, int ROWS, int THREADS> struct Gathered {
  static constexpr int BYTES = ROWS * KSTEP * 2, LOADS = BYTES / (THREADS * 16);
  uint32_t off[LOADS];
  int k;
  __device__ void init(int64_t ld, int64_t left, const int32_t *rows, int per, int64_t T) {
#pragma unroll
    for (int i = 0; i < LOADS; i++) {
      int p = (i * THREADS + threadIdx.x) * 16, r = p / 128, c = (p / 16 % 8) ^ (r / 2 % 8);
      k = c * 8; /* the same for all */
      int t = r < left ? rows[r] : -1;
      t = t < 0 ? -1 : t / per;
      off[i] = t >= 0 && t < T ? (uint32_t)(t * ld * 2 + c * 16) : OOB_LAYER_OUT;
    }
  }
  __device__ void load(const char *base, lds_char *to, int kleft) {
    __amdgpu_buffer_rsrc_t r = buffer(base);
    int wave = uniform(threadIdx.x / 64);
#pragma unroll
    for (int i = 0; i < LOADS; i++) load_lds(r, to + (i * THREADS + wave * 64) * 16, k < kleft ? off[i] : OOB_LAYER_OUT);
  }
};

/* Waits until no more than `most` of the wave's loads and none of its reads of LDS are on the way, then for the workgroup. */
template <int most> __device__ inline void wait_but() {
  static_assert(most < 64, "six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0x0070 | (most & 15) | (most >> 4) << 14); /* vmcnt(most) lgkmcnt(0), expcnt as it is */
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

/* The sums of one tile over `steps` steps of k, the first BUFFERS of which lie in LDS; load(buffer) asks for the next.  Each buffer is an array of its own: the
 * compiler then knows that a read of one does not wait for the loads to the others.  A step's last products run behind the barrier that frees its
 * buffer: while they do, the first fragments of the next step are read and the loads of a later one are asked for.  At the end nobody reads the buffers any more.
 * Small tiles have four buffers: their steps are shorter than the way from memory. */
template <class E, int TM, int TN, int WM, int WN, bool AK, bool BK, int BUFFERS, class TA, class TB, class L>
__device__ __forceinline__ void multiply(L &load, int steps, lds_char *const (&buffers)[BUFFERS], f32x16 (&acc)[TM / WM / 32][TN / WN / 32]) {
  constexpr int FM = TM / WM / 32, FN = TN / WN / 32, READS = FM * (AK ? 1 : 2) + FN * (BK ? 1 : 2), LOADS = TA::LOADS + TB::LOADS;
  int wave = uniform(threadIdx.x / 64), wm = wave / WN, wn = wave % WN;
  Fragment<E, TM, FM, AK> fa;
  Fragment<E, TN, FN, BK> fb;
  fa.init(wm * FM * 32);
  fb.init(wn * FN * 32);
#pragma unroll
  for (int i = 0; i < FM; i++)
#pragma unroll
    for (int j = 0; j < FN; j++) acc[i][j] = f32x16{0};
  using V = typename Vec<E>::v8;
  V a0[FM], b0[FN], a1[FM], b1[FN];
  auto fetch = [&](lds_char *from, int s, V(&a)[FM], V(&b)[FN]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FM; i++) a[i] = fa.read(from, i, s);
#pragma unroll
    for (int j = 0; j < FN; j++) b[j] = fb.read(from + TA::BYTES, j, s);
  };
  auto products = [&](V(&a)[FM], V(&b)[FN]) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < FM; i++)
#pragma unroll
      for (int j = 0; j < FN; j++) acc[i][j] = mfma(b[j], a[i], acc[i][j]); /* lane: m, registers: n */
  };
  constexpr int EVERY = (READS + FM * FN - 1) / (FM * FN);
  auto order = [&]() __attribute__((always_inline)) { /* reads of the next fragments between the products */
#pragma unroll
    for (int g = 0; g < FM * FN; g++) {
      if (g * EVERY < READS) __builtin_amdgcn_sched_group_barrier(0x100, EVERY, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    }
  };
  auto front = [&](lds_char *now) __attribute__((always_inline)) { /* products 0 .. 2 of a step, reads of 1 .. 3 */
    __builtin_amdgcn_sched_barrier(0);
    fetch(now, 1, a1, b1);
    products(a0, b0);
    order();
    fetch(now, 2, a0, b0);
    products(a1, b1);
    order();
    fetch(now, 3, a1, b1);
    products(a0, b0);
    order();
  };
  auto back = [&](lds_char *now, lds_char *next) __attribute__((always_inline)) { /* product 3, read 0 of the next step */
    wait_but<(BUFFERS - 2) * LOADS>(); /* the next step's loads have landed, and nobody reads this buffer any more */
    fetch(next, 0, a0, b0);
    load(now);
    products(a1, b1);
#pragma unroll
    for (int g = 0; g < FM * FN; g++) {
      if (g * EVERY < READS) __builtin_amdgcn_sched_group_barrier(0x100, EVERY, 0);
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x10, (LOADS + FM * FN - 1) / (FM * FN), 0);
    }
  };
  fetch(buffers[0], 0, a0, b0);
  front(buffers[0]);
  /* the loop begins where loads are waited for: the compiler waits for all of them at its head whatever is on the way */
  int left = steps - 1;
  for (; left >= BUFFERS; left -= BUFFERS) {
#pragma unroll
    for (int i = 0; i < BUFFERS; i++) {
      back(buffers[i], buffers[(i + 1) % BUFFERS]);
      front(buffers[(i + 1) % BUFFERS]);
    }
  }
#pragma unroll
  for (int i = 0; i < BUFFERS - 1; i++)
    if (left > i) {
      back(buffers[i], buffers[i + 1]);
      front(buffers[i + 1]);
    }
  products(a1, b1);
  wait_barrier(); /* the loads past the last step have landed: the next tile's may be asked for */
}

/* A tile's sums through the epilogue, from the registers that the products leave them in: a lane has a row and, of 16 neighbouring columns, two times four.
 * An exchange between the halves of the wave makes them eight in a row, 16 bytes of C a store.  Nothing goes through LDS, so that the next tile's
 * first loads are on their way meanwhile.  FULL: all rows and columns are there, so that every wave makes STORES stores at least, which the wait behind counts on. */
template <int TM, int TN, int WM, int WN> constexpr int STORES = TM / WM / 32 * (TN / WN / 32) * 2;
template <class E, int ACT, bool FULL, int TM, int TN, int WM, int WN>
__device__ __forceinline__ void finish(const Product &g, f32x16 (&acc)[TM / WM / 32][TN / WN / 32], const E *bias, E *C, int64_t row, int left, int64_t n0) {
  constexpr int FM = TM / WM / 32, FN = TN / WN / 32;
  int wave = uniform(threadIdx.x / 64), wm = wave / WN, wn = wave % WN, l = lane();
  int64_t n1 = n0 + wn * FN * 32 + l / 32 * 8;
  typename Vec<E>::v8 add[FN][2];
  if (bias)
#pragma unroll
    for (int j = 0; j < FN; j++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        int64_t n = n1 + j * 32 + h * 16;
        if (FULL || n < g.N) add[j][h] = load8<E>(bias + n, FULL ? 8 : g.N - n);
      }
#pragma unroll
  for (int i = 0; i < FM; i++) {
    int m = (wm * FM + i) * 32 + (l & 31);
#pragma unroll
    for (int j = 0; j < FN; j++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        float v[8];
#pragma unroll
        for (int e = 0; e < 4; e++) {
          auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][8 * h + e]), __float_as_uint(acc[i][j][8 * h + 4 + e]), false, false);
          v[e] = __uint_as_float(two[0]), v[4 + e] = __uint_as_float(two[1]);
        }
        int64_t n = n1 + j * 32 + h * 16, at = row + m;
        if (!FULL && (m >= left || n >= g.N)) continue;
        typename Vec<E>::v8 out;
        if (bias)
#pragma unroll
          for (int e = 0; e < 8; e++) v[e] += (float)add[j][h][e];
        if (g.Z) { /* rounded to the type, as y is: half the memory between the passes; act' sees the rounding, act does not */
#pragma unroll
          for (int e = 0; e < 8; e++) out[e] = (E)v[e];
          store8<E>((E *)g.Z + at * g.ldz + n, out, FULL ? 8 : g.N - n);
        }
#pragma unroll
        for (int e = 0; e < 8; e++) out[e] = (E)activate(v[e], ACT);
        store8<E>(C + at * g.ldc + n, out, FULL ? 8 : g.N - n);
      }
  }
}

/* The same eight columns of a row, as sums that are not complete: TM x TN floats. */
template <int TM, int TN, int WM, int WN>
__device__ __forceinline__ void leave(f32x16 (&acc)[TM / WM / 32][TN / WN / 32], float *to, int left) {
  constexpr int FM = TM / WM / 32, FN = TN / WN / 32;
  int wave = uniform(threadIdx.x / 64), wm = wave / WN, wn = wave % WN, l = lane();
#pragma unroll
  for (int i = 0; i < FM; i++) {
    int m = (wm * FM + i) * 32 + (l & 31);
#pragma unroll
    for (int j = 0; j < FN; j++)
#pragma unroll
      for (int h = 0; h < 2; h++) {
        f32x4 lo, hi;
#pragma unroll
        for (int e = 0; e < 4; e++) {
          auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(acc[i][j][8 * h + e]), __float_as_uint(acc[i][j][8 * h + 4 + e]), false, false);
          lo[e] = __uint_as_float(two[0]), hi[e] = __uint_as_float(two[1]);
        }
        if (m >= left) continue;
        f32x4 *at = (f32x4 *)(to + (int64_t)m * TN + wn * FN * 32 + j * 32 + h * 16 + l / 32 * 8);
        at[0] = lo, at[1] = hi;
      }
  }
}

/* Where a workgroup's tile lies; expert -1: nowhere. */
struct Where { int expert, left, k, part; int64_t row, n0; const char *pa, *pb; }; /* rows of C from `row` on; k: depth; part: where its sums are left */

/* Rows of y (BK: W as it is), of dx (W by its columns) or, DW, the matrices dw[e] = dz^T x over the rows of e.  A workgroup takes one tile after the other, every
 * gridDim-th: the first loads of the next are asked for before the present one's epilogue.
 * 8192 rows, 8 experts, 4096 x 8192, bfloat16 (550 GFLOP each): y 620 us, dx 510, dw 555; a library's eight products of 1024 rows, without bias, activation and z, 497, 622 and 618.  Of
 * the time that a unit has a tile the matrix cores are busy 59 % (y), 76 % (dx's whole rounds) and 51 % (dw), at 2.0, 1.75 and 2.0 GHz.  Few rows: 16 tokens, 8 experts of 2048 x 2048: 13.2 us,
 * 5.1 TB/s of matrices (two buffers: 19.2).
 * Large tiles that are left over from whole rounds of the GPU, where they would keep few compute units busy for a round, are left to a second launch (REST), in which k
 * is divided among several workgroups that leave their sums, and a third that joins them.  8192 rows, 8 experts, 4096 x 8192, dx: 576 tiles,
 * 508 us; 597 without (the quarters of the 64 tiles left over, done as tiles of 128: 566). */
constexpr int UNITS = 256;
struct Rest { int whole, tiles, splits; }; /* of all large tiles the first `whole` are done one a workgroup */
__device__ inline Rest rest_of(int total, int steps) {
  int rest = total > UNITS ? total % UNITS : 0, splits = rest ? UNITS / rest : 1;
  if (splits > 8) splits = 8;
  if (splits > steps / 16) splits = steps / 16; /* a part of 16 steps takes as long as its sums' way to memory and back */
  return splits < 2 ? Rest{total, 0, 1} : Rest{total - rest, rest, splits};
}

template <class E, int TM, int TN, int WM, int WN, bool BK, bool GATHER, bool DW, bool REST>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_experts(Experts x) {
  constexpr int THREADS = WM * WN * 64;
  constexpr bool AK = !DW;
  using TA = std::conditional_t<GATHER, Gathered<E, TM, THREADS>, Strip<E, TM, THREADS, AK>>;
  using TB = Strip<E, TN, THREADS, BK>;
  constexpr int BUFFERS = TM == 64 ? 4 : 2, SIZE = TA::BYTES + TB::BYTES;
  __shared__ __attribute__((aligned(1024))) char first_[SIZE], second_[SIZE], third_[BUFFERS > 2 ? SIZE : 1024], fourth_[BUFFERS > 2 ? SIZE : 1024];
  lds_char *const all[4] = {(lds_char *)first_, (lds_char *)second_, (lds_char *)third_, (lds_char *)fourth_};
  lds_char *const(&buffers)[BUFFERS] = reinterpret_cast<lds_char *const(&)[BUFFERS]>(all);
  const Product &g = x.g;
  const int64_t da = AK ? KSTEP * 2 : KSTEP * 2 * g.lda, db = BK ? KSTEP * 2 : KSTEP * 2 * g.ldb;

  /* within an expert bands of eight rows of tiles, as in the dense product */
  auto band = [&](int tile, int tm, int tn, int &m, int &n) {
    int in = tile % (8 * tn), first = tile / (8 * tn) * 8, high = tm - first < 8 ? tm - first : 8;
    m = first + in % high, n = in / high;
  };
  auto locate = [&](int id) -> Where {
    Where w{};
    int m, n;
    if constexpr (DW) { /* every XCD gets an eighth of each expert's tiles, neighbours of one another: experts differ in rows */
      int per = g.tiles_m * g.tiles_n, part = (per + 7) / 8, in_e = id % (8 * part), tile = in_e % 8 * part + in_e / 8;
      w.expert = tile < per ? id / (8 * part) : -1;
      if (w.expert < 0) return w;
      band(tile, g.tiles_m, g.tiles_n, m, n);
      int64_t first, rows = rows_of(x.d, w.expert, first), m0 = (int64_t)m * TM;
      first = uniform((int)first), w.k = uniform((int)rows);
      w.n0 = (int64_t)n * TN, w.left = (int)(g.M - m0 < TM ? g.M - m0 : TM), w.row = (int64_t)w.expert * g.M + m0;
      w.pa = (const char *)g.A + (first * g.lda + m0) * 2, w.pb = (const char *)g.B + (first * g.ldb + w.n0) * 2;
    } else {
      int64_t tn = g.tiles_n;
      int steps = (int)((g.K + KSTEP - 1) / KSTEP), first = 0, last = steps;
      Found f = find(x.d, [&](int64_t r) { return (r + TM - 1) / TM * tn; }, [&](int total) {
        Rest r = TM == 256 ? rest_of(total, steps) : Rest{total, 0, 1};
        if (!REST) return id < r.whole ? (int)xcd_order(id, r.whole) : total;
        if (id >= r.tiles * r.splits) return total;
        w.part = (int)xcd_order(id, r.tiles * r.splits);
        int split = w.part / r.tiles;
        first = steps * split / r.splits, last = steps * (split + 1) / r.splits;
        return r.whole + w.part % r.tiles;
      });
      w.expert = f.expert;
      if (w.expert < 0) return w;
      band(f.part, (int)(((int64_t)f.rows + TM - 1) / TM), (int)tn, m, n);
      int64_t m0 = (int64_t)m * TM;
      w.n0 = (int64_t)n * TN;
      w.left = f.rows - m0 < TM ? (int)(f.rows - m0) : TM, w.row = f.first + m0;
      w.k = (last == steps ? (int)g.K : last * KSTEP) - first * KSTEP;
      w.pa = (const char *)g.A + (GATHER ? 0 : w.row * g.lda * 2) + first * da;
      w.pb = (const char *)g.B + (f.expert * x.expert_stride + (BK ? w.n0 * g.ldb : w.n0)) * 2 + first * db;
    }
    return w;
  };
  auto next_of = [&](int &id) -> Where { /* the next tile from number `id` on that is one */
    Where w{};
    w.expert = -1;
    for (; id < x.ids; id += gridDim.x) {
      w = locate(id);
      if (w.expert >= 0 || !DW) break;
    }
    id += gridDim.x;
    return w;
  };

  TA ta;
  TB tb;
  int kleft, id = blockIdx.x;
  const char *pa, *pb;
  auto load = [&](lds_char *to) __attribute__((always_inline)) { /* past the last step: nothing is read, zeros land */
    ta.load(pa, to, kleft);
    tb.load(pb, to + TA::BYTES, kleft);
    pa += da, pb += db, kleft -= KSTEP;
  };
  auto begin = [&](const Where &w) __attribute__((always_inline)) {
    if constexpr (GATHER) ta.init(g.lda, w.left, x.rows + w.row, x.per, x.T);
    else ta.init(g.lda, w.left);
    tb.init(g.ldb, g.N - w.n0);
    pa = w.pa, pb = w.pb, kleft = w.k;
#pragma unroll
    for (int i = 0; i < BUFFERS; i++) load(buffers[i]);
  };
  Where w = next_of(id);
  if (w.expert < 0) return;
  begin(w);
  wait_barrier();
  for (;;) {
    Where then = next_of(id);
    f32x16 acc[TM / WM / 32][TN / WN / 32];
    multiply<E, TM, TN, WM, WN, AK, BK, BUFFERS, TA, TB>(load, (w.k + KSTEP - 1) / KSTEP, buffers, acc);
    if (then.expert >= 0) begin(then);
    const E *bias = g.bias ? (const E *)g.bias + (int64_t)w.expert * g.N : nullptr;
    if constexpr (REST) {
      leave<TM, TN, WM, WN>(acc, g.partial + (int64_t)w.part * TM * TN, w.left);
      wait_barrier();
    } else if (w.left == TM && w.n0 + TN <= g.N) {
#define OOB_FINISH(ACT, FULL) finish<E, ACT, FULL, TM, TN, WM, WN>(g, acc, bias, (E *)g.C, w.row, w.left, w.n0)
      switch (g.act) {
        case OOB_ACT_RELU: OOB_FINISH(OOB_ACT_RELU, true); break;
        case OOB_ACT_SILU: OOB_FINISH(OOB_ACT_SILU, true); break;
        case OOB_ACT_GELU: OOB_FINISH(OOB_ACT_GELU, true); break;
        case OOB_ACT_GELU_TANH: OOB_FINISH(OOB_ACT_GELU_TANH, true); break;
        default: OOB_FINISH(OOB_ACT_NONE, true);
      }
      /* The next tile's loads, which are older than the stores, have landed; the stores need not have.  They are counted in order, so that with two buffers the next tile's first
       * step waits for them (vmcnt(0) in `back`); with four they have two steps' time. */
      wait_but<STORES<TM, TN, WM, WN>>();
    } else {
      switch (g.act) {
        case OOB_ACT_RELU: OOB_FINISH(OOB_ACT_RELU, false); break;
        case OOB_ACT_SILU: OOB_FINISH(OOB_ACT_SILU, false); break;
        case OOB_ACT_GELU: OOB_FINISH(OOB_ACT_GELU, false); break;
        case OOB_ACT_GELU_TANH: OOB_FINISH(OOB_ACT_GELU_TANH, false); break;
        default: OOB_FINISH(OOB_ACT_NONE, false);
      }
      wait_barrier();
#undef OOB_FINISH
    }
    if (then.expert < 0) return;
    w = then;
  }
}

/* Joins what REST left: 32 workgroups a tile, eight values a thread. */
template <class E> __global__ __launch_bounds__(256) void k_experts_join(Experts x) {
  constexpr int TILE = 256;
  const Product &g = x.g;
  int64_t tn = g.tiles_n;
  int tile = blockIdx.x / 32, at = (int)(blockIdx.x % 32 * 256 + threadIdx.x) * 8, steps = (int)((g.K + KSTEP - 1) / KSTEP);
  Rest r{};
  Found f = find(x.d, [&](int64_t n) { return (n + TILE - 1) / TILE * tn; }, [&](int total) {
    r = rest_of(total, steps);
    return tile < r.tiles ? r.whole + tile : total;
  });
  if (f.expert < 0) return;
  int tm = (int)(((int64_t)f.rows + TILE - 1) / TILE), in = f.part % (8 * (int)tn), band = f.part / (8 * (int)tn) * 8, high = tm - band < 8 ? tm - band : 8;
  int64_t m = (int64_t)(band + in % high) * TILE + at / TILE, n = (int64_t)(in / high) * TILE + at % TILE;
  if (m >= f.rows || n >= g.N) return;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (int s = 0; s < r.splits; s++) {
    const f32x4 *p = (const f32x4 *)(g.partial + ((int64_t)s * r.tiles + tile) * TILE * TILE + at);
    f32x4 lo = p[0], hi = p[1];
    for (int e = 0; e < 4; e++) v[e] += lo[e], v[4 + e] += hi[e];
  }
  Product one = g;
  if (g.bias) one.bias = (const E *)g.bias + (int64_t)f.expert * g.N;
  epilogue<E>(one, f.first + m, n, v);
}

/* ---- rows of another pitch or order in the workspace: what the tiles' loads cannot take as it lies ------------------------------
 * Rows of a multiple of 8 with zeros behind.  Row r comes from token rows[r] / per (rows given), or from part r / of, row r % of. */
struct Packed {
  const uint16_t *from;
  uint16_t *to;
  int64_t n, of, part_stride, cols, ld, ld_to, T;
  const int32_t *rows, *offsets; /* offsets: only rows below the largest one are anybody's */
  int per, E;
};

/* Two matrices in one launch, w and x: the first takes workgroups below `first`. */
struct Packs { Packed p[2]; int64_t first; };

template <int THREADS> __device__ __forceinline__ void pack_rows(const Packs &packs, int64_t group) {
  const bool second = group >= packs.first;
  const Packed &p = packs.p[second];
  int64_t per = p.ld_to / 8, id = (group - (second ? packs.first : 0)) * THREADS + threadIdx.x, r = id / per, c = id % per * 8;
  if (p.offsets) {
    int end = 0;
    for (int e = lane(); e <= p.E; e += 64) end = max(end, p.offsets[e]);
    for (int o = 1; o < 64; o *= 2) end = max(end, __shfl_xor(end, o));
    if (r >= end) return;
  }
  if (r >= p.n) return;
  int64_t at = -1;
  if (p.rows) {
    int64_t t = p.rows[r] < 0 ? -1 : p.rows[r] / p.per;
    if (t >= 0 && t < p.T) at = t * p.ld;
  } else {
    at = r / p.of * p.part_stride + r % p.of * p.ld;
  }
  i16x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
  if (at >= 0) v = __builtin_bit_cast(i16x8, load8<fp16>((const fp16 *)p.from + at + c, p.cols - c));
  *(i16x8 *)(p.to + r * p.ld_to + c) = v;
}
__global__ __launch_bounds__(256) void k_pack_rows(Packs packs) { pack_rows<256>(packs, blockIdx.x); }

/* ---- dz = dy act'(z) and the sums of its columns, runs of an expert's rows -------------------------------------------------- */
struct ActGrad {
  Division d;
  const void *dy, *z;
  void *dz; /* rows of a multiple of 8; null: act is none, dz is dy */
  int64_t ld_dy, ld_z, ld_dz, N;
  float *sums; /* [runs][N] or null */
  int rows;    /* of a run */
  int64_t runs; /* there is room for */
};

template <class E, int ACT> __global__ __launch_bounds__(256) void k_experts_act(ActGrad g) {
  __shared__ float part[4][512 + 8];
  Found f = find(g.d, [&](int64_t n) { return (n + g.rows - 1) / g.rows; }, [&](int) { return (int)blockIdx.y; });
  if (f.expert < 0) return;
  int64_t n = (int64_t)blockIdx.x * 512 + lane() * 8, left = g.N - n;
  int64_t t1 = (int64_t)(f.part + 1) * g.rows < f.rows ? f.first + (int64_t)(f.part + 1) * g.rows : (int64_t)f.first + f.rows;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int64_t stop = left > 0 ? t1 : 0;
  for (int64_t t0 = f.first + (int64_t)f.part * g.rows + threadIdx.x / 64; t0 < stop; t0 += 16) {
    typename Vec<E>::v8 d[4], z[4], out; /* four rows on their way before the first is worked on */
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (t0 + 4 * u < stop) {
        d[u] = load8<E>((const E *)g.dy + (t0 + 4 * u) * g.ld_dy + n, left);
        if (ACT != OOB_ACT_NONE) z[u] = load8<E>((const E *)g.z + (t0 + 4 * u) * g.ld_z + n, left);
      }
#pragma unroll
    for (int u = 0; u < 4; u++) {
      if (t0 + 4 * u >= stop) continue;
      for (int e = 0; e < 8; e++) {
        float v = (float)d[u][e] * (ACT == OOB_ACT_NONE ? 1.f : slope((float)z[u][e], ACT));
        out[e] = (E)v; /* the matrix cores take 16 bits: dx and dw see this rounding, the bias's gradient does not */
        sum[e] += v;
      }
      if (g.dz) store8<E>((E *)g.dz + (t0 + 4 * u) * g.ld_dz + n, out, 8); /* past N: zeros */
    }
  }
  if (!g.sums) return;
  for (int e = 0; e < 8; e++) part[threadIdx.x / 64][lane() * 8 + e] = sum[e];
  __syncthreads();
  for (int c = threadIdx.x; c < 512; c += 256) {
    int64_t at = (int64_t)blockIdx.x * 512 + c;
    if (at < g.N) g.sums[blockIdx.y * g.N + at] = (part[0][c] + part[1][c]) + (part[2][c] + part[3][c]);
  }
}

/* Few rows in all: an expert's 64 columns to a workgroup of 16 waves, 128 rows of them at a time, twice over on their way; its sums are db, and nothing is
 * joined in a launch of its own; copies of w and x go along.  1206 rows, 7 experts, 1021 columns, float16, with copies of 15 MB: 12.9 us; 23.1 in three launches.
 * 2048 rows, 8 experts, 1024 columns, without copies: 4.9 us evenly divided, 17.2 where one has all; 8.7 and 16.9 in two launches (8192 rows: 11.2 and 61 against 16.0 and 50). */
constexpr int64_t FEW_ROWS = 2048;
constexpr int FEW_THREADS = 1024;
template <class E, int ACT> __global__ __launch_bounds__(FEW_THREADS) void k_experts_act_few(ActGrad g, E *db, Packs packs) {
  constexpr int DEEP = 2, AT_ONCE = FEW_THREADS / 8, WAVES = FEW_THREADS / 64;
  __shared__ float part[WAVES][64];
  const int across = (int)((g.N + 63) / 64), e = blockIdx.x / across, at = threadIdx.x % 8 * 8;
  if (e >= g.d.E) {
    pack_rows<FEW_THREADS>(packs, blockIdx.x - across * g.d.E);
    return;
  }
  const int64_t n0 = (int64_t)(blockIdx.x % across) * 64;
  int64_t first, rows = rows_of(g.d, e, first), n = n0 + at, left = g.N - n;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int64_t stop = left > 0 ? first + rows : 0;
  for (int64_t t0 = first + threadIdx.x / 8; t0 < stop; t0 += AT_ONCE * DEEP) {
    typename Vec<E>::v8 d[DEEP], z[DEEP], out;
#pragma unroll
    for (int u = 0; u < DEEP; u++)
      if (t0 + AT_ONCE * u < stop) {
        d[u] = load8<E>((const E *)g.dy + (t0 + AT_ONCE * u) * g.ld_dy + n, left);
        if (ACT != OOB_ACT_NONE) z[u] = load8<E>((const E *)g.z + (t0 + AT_ONCE * u) * g.ld_z + n, left);
      }
#pragma unroll
    for (int u = 0; u < DEEP; u++) {
      if (t0 + AT_ONCE * u >= stop) continue;
      for (int i = 0; i < 8; i++) {
        float v = (float)d[u][i] * (ACT == OOB_ACT_NONE ? 1.f : slope((float)z[u][i], ACT));
        out[i] = (E)v; /* as above */
        sum[i] += v;
      }
      if (g.dz) store8<E>((E *)g.dz + (t0 + AT_ONCE * u) * g.ld_dz + n, out, 8);
    }
  }
  if (!db) return;
#pragma unroll
  for (int i = 0; i < 8; i++) {
    for (int o = 8; o < 64; o *= 2) sum[i] += __shfl_xor(sum[i], o);
    if (lane() < 8) part[threadIdx.x / 64][at + i] = sum[i];
  }
  __syncthreads();
  n = n0 + threadIdx.x;
  if (threadIdx.x < 64 && n < g.N) {
    float all = 0;
#pragma unroll
    for (int w = 0; w < WAVES; w++) all += part[w][threadIdx.x];
    db[e * g.N + n] = (E)all;
  }
}

/* db[e]: the sums of the expert's runs, in their order. */
template <class E> __global__ __launch_bounds__(256) void k_experts_db(ActGrad g, E *out) {
  __shared__ float part[4][64];
  int e = blockIdx.y;
  int64_t first, before = 0, n = (int64_t)blockIdx.x * 64 + lane();
  for (int i = lane(); i < e; i += 64) before += (rows_of(g.d, i, first) + g.rows - 1) / g.rows;
  for (int o = 1; o < 64; o *= 2) before += __shfl_xor(before, o);
  int64_t runs = (rows_of(g.d, e, first) + g.rows - 1) / g.rows;
  float s = 0;
  if (n < g.N)
    for (int64_t r = threadIdx.x / 64; r < runs && before + r < g.runs; r += 4) s += g.sums[(before + r) * g.N + n];
  part[threadIdx.x / 64][lane()] = s;
  __syncthreads();
  if (threadIdx.x < 64 && n < g.N) out[e * g.N + n] = (E)((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]));
}

/* ---- host -------------------------------------------------------------------------------------------------------------------- */
struct Operand { const void *p; int64_t ld, part; }; /* elements between rows and between experts */

bool loadable(const void *p, int64_t ld, int64_t cols) { return cols % 8 == 0 && multiple(p, 16) && ld % 8 == 0 && ld < (1 << 21); }
bool w_loadable(const oob_expert_linear_t *p) { return loadable(p->w, p->w_stride, p->K) && (p->expert_stride % 8 == 0 || p->E == 1); }
/* Rows of x as a forward tile takes them: where they lie, or gathered by 32-bit offsets from its start. */
bool x_loadable(const oob_expert_linear_t *p) {
  return loadable(p->x, p->x_stride, p->K) && (!p->rows || p->T * p->x_stride < (int64_t)1 << 30);
}

int64_t groups_of(const Packed &k, int threads) { return (k.n * (k.ld_to / 8) + threads - 1) / threads; }
Packs both(const Packed &a, const Packed &b, int threads) { return {{a, b}, groups_of(a, threads)}; }
void pack(const Packed &a, const Packed &b, hipStream_t st) {
  int64_t n = groups_of(a, 256) + groups_of(b, 256);
  if (n) k_pack_rows<<<(unsigned)n, 256, 0, st>>>(both(a, b, 256));
}
/* As the products take them, in the workspace where they have to be copied: `how` says so then (n is 0 otherwise). */
Operand plan_w(const oob_expert_linear_t *p, Arena &w, Packed &how) {
  how = Packed{};
  if (w_loadable(p)) return {p->w, p->w_stride, p->expert_stride};
  int64_t ld = up(p->K, 8);
  void *to = w.take((size_t)p->E * p->N * ld * 2);
  how = {(const uint16_t *)p->w, (uint16_t *)to, p->E * p->N, p->N, p->expert_stride, p->K, p->w_stride, ld, 0, nullptr, nullptr, 1, 0};
  return {to, ld, p->N * ld};
}
/* Rows of x in order of their experts. */
Operand plan_x(const oob_expert_linear_t *p, Arena &w, Packed &how) {
  how = Packed{};
  if (!p->rows && loadable(p->x, p->x_stride, p->K)) return {p->x, p->x_stride, 0};
  int64_t ld = up(p->K, 8);
  void *to = w.take((size_t)p->R * ld * 2);
  how = {(const uint16_t *)p->x, (uint16_t *)to, p->R, p->R, 0, p->K, p->x_stride, ld, p->T, p->rows, p->offsets, p->per, p->E};
  return {to, ld, 0};
}

int64_t tiles(int64_t n, int tile) { return (n + tile - 1) / tile; }

/* Tiles of R rows: as many as the worst division into E experts has. */
int64_t row_tiles(int64_t R, int E, int tile) { return R / tile + (R < E ? R : E); }

/* By the rows that an expert has on average, if all experts are here: where some are elsewhere R counts their pairs too, and the host does not know how many are not.  A tile of 256 is
 * then taken where few have rows: 4096 tokens, 2 choices, 2 of 8 experts here, 2048 x 2048 y 49 us, the middle one 32; 4 choices, 1 of 4 experts, 2048 x 512 41, the small one 18.  Where
 * there are enough of them it is the better one all the same: 4 choices, 32 of 128 experts, 2048 x 2048 82 us, the middle one 89; 2 of 8 experts, 4096 x 8192 153 and 159. */
int choose_tile(int64_t R, int E, int64_t N) {
  int64_t mean = R / E;
  if (mean >= 192 && tiles(R, 256) * tiles(N, 256) >= 112) return 256; /* 4096 rows, 8 experts, 2048 x 2048: 49 us, the middle one 56 (8192 rows in uneven runs: 99 and 85); of 64 tiles 77 and 55 */
  if (mean >= 96 && tiles(R, 128) * tiles(N, 128) >= 192) return 128;
  return 64;
}
int choose_dw(int64_t M, int64_t N, int E) {
  if (M >= 192 && N >= 192 && E * tiles(M, 256) * tiles(N, 256) >= 192) return 256;
  if (M >= 96 && N >= 96 && E * tiles(M, 128) * tiles(N, 128) >= 192) return 128;
  return 64;
}

/* Sums of tiles whose k is divided: room for as many parts as compute units where any division of the rows has more large tiles than these. */
size_t rest_bytes(int64_t R, int E, int64_t N, int64_t K) {
  return choose_tile(R, E, N) == 256 && row_tiles(R, E, 256) * tiles(N, 256) > UNITS && tiles(K, KSTEP) >= 32 ? (size_t)UNITS * 256 * 256 * 4 : 0;
}

template <class E, int TILE, int WN, bool BK, bool GATHER, bool DW> void launch(Experts x, hipStream_t st) {
  x.g.tiles_m = (int)tiles(x.g.M, TILE), x.g.tiles_n = (int)tiles(x.g.N, TILE);
  x.ids = (int)(DW ? x.d.E * up((int64_t)x.g.tiles_m * x.g.tiles_n, 8) : row_tiles(x.d.R, x.d.E, TILE) * x.g.tiles_n);
  int most = TILE == 256 ? 256 : 512; /* that run at once: one, two a compute unit */
  k_experts<E, TILE, TILE, 2, WN, BK, GATHER, DW, false><<<x.ids < most ? x.ids : most, 128 * WN, 0, st>>>(x);
  if constexpr (TILE == 256 && !DW)
    if (x.g.partial) {
      x.ids = UNITS;
      k_experts<E, TILE, TILE, 2, WN, BK, GATHER, false, true><<<UNITS, 128 * WN, 0, st>>>(x);
      k_experts_join<E><<<UNITS / 2 * 32, 256, 0, st>>>(x);
    }
}
template <class E, bool BK, bool GATHER, bool DW> int products(Experts x, hipStream_t st) {
  int tile = DW ? choose_dw(x.g.M, x.g.N, x.d.E) : choose_tile(x.d.R, x.d.E, x.g.N);
  if (tile == 256) launch<E, 256, 4, BK, GATHER, DW>(x, st);
  else if (tile == 128) launch<E, 128, 2, BK, GATHER, DW>(x, st);
  else launch<E, 64, 2, BK, GATHER, DW>(x, st);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

bool sizes_ok(const oob_expert_linear_t *p) {
  const int64_t most = (int64_t)1 << 31;
  return p && (p->dtype == OOB_BF16 || p->dtype == OOB_FP16) && p->act >= 0 && p->act < OOB_ACTS && p->E >= 1 && p->E <= OOB_EXPERT_MAX &&
         p->per >= 1 && p->R >= 0 && p->T >= 0 && p->N >= 1 && p->K >= 1 && p->R < most && p->T < most && p->N < (1 << 21) && p->K < (1 << 21) &&
         p->T * p->per == p->R && (p->rows || p->per == 1);
}
bool fits(int64_t tiles) { return tiles < (int64_t)1 << 31; }
/* Numbers of the smallest tiles, which are 32-bit; threads of the copies, 2^32 at most. */
bool launches_fit(const oob_expert_linear_t *p, bool forward) {
  int64_t most = (p->N > p->K ? p->N : p->K) + 64;
  bool x_lies = forward ? x_loadable(p) : !p->rows && loadable(p->x, p->x_stride, p->K);
  return fits(row_tiles(p->R, p->E, 64) * tiles(most, 64)) && fits(p->E * up(tiles(p->N, 64) * tiles(p->K, 64), 8)) &&
         ((w_loadable(p) ? 0 : p->E * p->N) + (x_lies ? 0 : p->R)) * (up(p->K, 8) / 8) < ((int64_t)1 << 32) - 512;
}

/* Where matrices lie. */
Lies lies(const void *p, int64_t rows, int64_t cols, int64_t ld) { return {p, rows, cols * 2, ld * 2}; }
/* On an expert's matrix: between those of far-apart experts there is room for others. */
bool on_w(const Lies &to, const oob_expert_linear_t *p) {
  if (!share(to, lies_flat(p->w, 2 * ((p->E - 1) * p->expert_stride + (p->N - 1) * p->w_stride + p->K)))) return false;
  if (p->expert_stride == p->N * p->w_stride) return share(to, lies(p->w, p->E * p->N, p->K, p->w_stride));
  for (int e = 0; e < p->E; e++)
    if (share(to, lies((const uint16_t *)p->w + e * p->expert_stride, p->N, p->K, p->w_stride))) return true;
  return false;
}
Lies lies_x(const oob_expert_linear_t *p) { return lies(p->x, p->x ? p->T : 0, p->K, p->x_stride); }
/* Offsets and rows are read by every workgroup, whenever it runs. */
bool on_numbers(const Lies &to, const oob_expert_linear_t *p) {
  return share(to, lies_flat(p->offsets, (p->E + 1) * 4)) || share(to, lies_flat(p->rows, p->R * 4));
}

struct Forward { Operand a, b; Packed x, w; float *rest; };
Forward plan(const oob_expert_linear_t *p, Arena &w) {
  Forward f{{p->x, p->x_stride, 0}, {}, {}, {}, nullptr};
  f.b = plan_w(p, w, f.w);
  if (!x_loadable(p)) f.a = plan_x(p, w, f.x);
  size_t rest = rest_bytes(p->R, p->E, p->N, p->K);
  if (rest) f.rest = (float *)w.take(rest);
  return f;
}

template <class E> int forward(const oob_expert_linear_t *p, Arena w, hipStream_t st) {
  Forward f = plan(p, w);
  if (!w.ok()) return OOB_ECAPACITY;
  pack(f.w, f.x, st);
  Experts x{};
  x.g.A = f.a.p, x.g.lda = f.a.ld, x.g.B = f.b.p, x.g.ldb = f.b.ld, x.expert_stride = f.b.part, x.g.partial = f.rest;
  x.g.N = p->N, x.g.K = p->K, x.g.bias = p->bias, x.g.C = p->y, x.g.ldc = p->y_stride, x.g.Z = p->z, x.g.ldz = p->z_stride, x.g.act = p->act;
  x.d = {p->offsets, p->E, p->R}, x.rows = p->rows, x.per = p->per, x.T = p->T;
  return p->rows && x_loadable(p) ? products<E, true, true, false>(x, st) : products<E, true, false, false>(x, st);
}

/* dz, the runs' sums, copies of w and x, sums of tiles whose depth is divided */
bool makes_dz(const oob_expert_linear_t *p, const oob_expert_linear_grad *g) {
  return (g->dx || g->dw) && (p->act != OOB_ACT_NONE || !loadable(g->dy, g->dy_stride, p->N));
}
int run_rows(const oob_expert_linear_t *p) { /* about 1024 workgroups, 16 rows at least; 65535 runs at most */
  int64_t r = up(p->R * tiles(p->N, 512) / 1024, 16), least = up(p->R / 32768, 16);
  r = r < 16 ? 16 : r > 4096 ? 4096 : r;
  return (int)(r < least ? least : r);
}
size_t sums_bytes(const oob_expert_linear_t *p) { return (size_t)row_tiles(p->R, p->E, run_rows(p)) * p->N * 4; }

bool few_rows(const oob_expert_linear_t *p) { return p->R <= FEW_ROWS && tiles(p->N, 64) * p->E + ((int64_t)p->E * p->N + p->R) * (up(p->K, 8) / 8) / FEW_THREADS < 1 << 21; }

struct Backward { Operand dz, w, x; Packed how_w, how_x; float *sums, *rest; };
Backward plan(const oob_expert_linear_t *p, const oob_expert_linear_grad *g, Arena &w) {
  Backward b{{g->dy, g->dy_stride, 0}, {}, {}, {}, {}, nullptr, nullptr};
  if (makes_dz(p, g)) b.dz = {w.take((size_t)p->R * up(p->N, 8) * 2), up(p->N, 8), 0};
  if (g->db && !few_rows(p)) b.sums = (float *)w.take(sums_bytes(p));
  if (g->dx) {
    b.w = plan_w(p, w, b.how_w);
    size_t rest = rest_bytes(p->R, p->E, p->K, p->N);
    if (rest) b.rest = (float *)w.take(rest);
  }
  if (g->dw) b.x = plan_x(p, w, b.how_x);
  return b;
}

template <class E> int backward(const oob_expert_linear_t *p, const oob_expert_linear_grad *g, Arena w, hipStream_t st) {
  bool makes = makes_dz(p, g);
  Backward b = plan(p, g, w);
  if (!w.ok()) return OOB_ECAPACITY;
  const bool few = few_rows(p);
  if (!p->R) b.how_w = b.how_x = Packed{};
  if (!few || !(makes || g->db)) { /* otherwise with dz, in one launch */
    pack(b.how_w, b.how_x, st);
    b.how_w = b.how_x = Packed{};
  }
  const Packs packs = both(b.how_w, b.how_x, FEW_THREADS);
  Operand dz = b.dz;
  float *sums = b.sums;
  Division d{p->offsets, p->E, p->R};
  if (makes || g->db) {
    ActGrad a{};
    a.d = d, a.dy = g->dy, a.ld_dy = g->dy_stride, a.z = p->z, a.ld_z = p->z_stride, a.N = p->N, a.sums = sums, a.rows = run_rows(p), a.runs = row_tiles(p->R, p->E, a.rows);
    a.dz = makes ? const_cast<void *>(dz.p) : nullptr, a.ld_dz = dz.ld;
    dim3 grid((unsigned)tiles(p->N, 512), (unsigned)a.runs);
    if (few) grid = dim3((unsigned)(tiles(p->N, 64) * p->E + packs.first + groups_of(b.how_x, FEW_THREADS)));
#define OOB_ACT_GRAD(ACT)                                                          \
  if (few) k_experts_act_few<E, ACT><<<grid, FEW_THREADS, 0, st>>>(a, (E *)g->db, packs);  \
  else k_experts_act<E, ACT><<<grid, 256, 0, st>>>(a);                             \
  break
    if (few || p->R) switch (p->act) {
      case OOB_ACT_RELU: OOB_ACT_GRAD(OOB_ACT_RELU);
      case OOB_ACT_GELU: OOB_ACT_GRAD(OOB_ACT_GELU);
      case OOB_ACT_GELU_TANH: OOB_ACT_GRAD(OOB_ACT_GELU_TANH);
      case OOB_ACT_SILU: OOB_ACT_GRAD(OOB_ACT_SILU);
      default: OOB_ACT_GRAD(OOB_ACT_NONE);
    }
#undef OOB_ACT_GRAD
    if (g->db && !few) k_experts_db<E><<<dim3((unsigned)tiles(p->N, 64), p->E), 256, 0, st>>>(a, (E *)g->db);
  }
  int rc = hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
  Experts x{};
  x.g.A = dz.p, x.g.lda = dz.ld, x.d = d;
  if (rc == OOB_OK && g->dx && p->R) {
    x.g.B = b.w.p, x.g.ldb = b.w.ld, x.expert_stride = b.w.part, x.g.partial = b.rest;
    x.g.N = p->K, x.g.K = p->N, x.g.C = g->dx, x.g.ldc = g->dx_stride;
    rc = products<E, false, false, false>(x, st);
  }
  if (rc == OOB_OK && g->dw) {
    x.g.B = b.x.p, x.g.ldb = b.x.ld, x.expert_stride = 0, x.g.partial = nullptr;
    x.g.M = p->N, x.g.N = p->K, x.g.K = 0, x.g.C = g->dw, x.g.ldc = p->K;
    rc = products<E, false, false, true>(x, st);
  }
  return rc;
}

size_t forward_bytes(const oob_expert_linear_t *p) {
  Arena w{nullptr, 0, 0};
  plan(p, w);
  return w.used;
}
size_t backward_bytes(const oob_expert_linear_t *p, const oob_expert_linear_grad *g) {
  Arena w{nullptr, 0, 0};
  plan(p, g, w);
  return w.used;
}

bool even(const void *p) { return multiple(p, 2); }

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" size_t oob_expert_linear_workspace_size(const oob_expert_linear_t *p) { return sizes_ok(p) && p->R ? forward_bytes(p) : 0; }

extern "C" int oob_expert_linear(const oob_expert_linear_t *p, void *workspace, size_t bytes, void *stream) {
  if (!sizes_ok(p) || !launches_fit(p, true)) return OOB_EINVAL;
  if (p->R == 0) return OOB_OK;
  if (!p->offsets || !p->x || !p->w || !p->y || !readable(p->x_stride, p->K) || p->w_stride < p->K || p->y_stride < p->N || p->expert_stride < 0) return OOB_EINVAL;
  if (p->z && p->z_stride < p->N) return OOB_EINVAL;
  if (!even(p->x) || !even(p->w) || !even(p->y) || !even(p->bias) || !even(p->z) || !multiple(p->offsets, 4) || !multiple(p->rows, 4)) return OOB_EINVAL;
  if (!multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = forward_bytes(p);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Lies y = lies(p->y, p->R, p->N, p->y_stride), z = lies(p->z, p->z ? p->R : 0, p->N, p->z_stride);
  for (Lies to : {y, z})
    if (share(to, lies_x(p)) || on_w(to, p) || share(to, lies_flat(p->bias, (int64_t)p->E * p->N * 2)) || on_numbers(to, p)) return OOB_EINVAL;
  if (share(y, z)) return OOB_EINVAL;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? forward<bf16>(p, w, (hipStream_t)stream) : forward<fp16>(p, w, (hipStream_t)stream);
}

extern "C" size_t oob_expert_linear_backward_workspace_size(const oob_expert_linear_t *p, const oob_expert_linear_grad *g) {
  return sizes_ok(p) && g ? backward_bytes(p, g) : 0;
}

extern "C" int oob_expert_linear_backward(const oob_expert_linear_t *p, const oob_expert_linear_grad *g, void *workspace, size_t bytes, void *stream) {
  if (!sizes_ok(p) || !g || !launches_fit(p, false) || !p->offsets) return OOB_EINVAL;
  if (p->R && (!g->dy || !readable(g->dy_stride, p->N) || (p->act != OOB_ACT_NONE && (!p->z || p->z_stride < p->N)))) return OOB_EINVAL;
  if (p->R && g->dx && (!p->w || p->w_stride < p->K || p->expert_stride < 0 || g->dx_stride < p->K)) return OOB_EINVAL;
  if (p->R && g->dw && (!p->x || !readable(p->x_stride, p->K))) return OOB_EINVAL;
  if (!even(g->dy) || !even(p->x) || !even(p->w) || !even(p->z) || !even(g->dx) || !even(g->dw) || !even(g->db)) return OOB_EINVAL;
  if (!multiple(p->offsets, 4) || !multiple(p->rows, 4) || !multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = backward_bytes(p, g);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Lies dx = lies(g->dx, g->dx ? p->R : 0, p->K, g->dx_stride), dw = lies_flat(g->dw, p->E * p->N * p->K * 2), db = lies_flat(g->db, p->E * p->N * 2);
  Lies dy = lies(g->dy, p->R, p->N, g->dy_stride), z = lies(p->z, p->z && p->act != OOB_ACT_NONE ? p->R : 0, p->N, p->z_stride);
  for (Lies to : {dx, dw, db})
    if (share(to, dy) || share(to, z) || (g->dx && on_w(to, p)) || (g->dw && share(to, lies_x(p))) || on_numbers(to, p)) return OOB_EINVAL;
  if (share(dx, dw) || share(dx, db) || share(dw, db)) return OOB_EINVAL;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? backward<bf16>(p, g, w, (hipStream_t)stream) : backward<fp16>(p, g, w, (hipStream_t)stream);
}
