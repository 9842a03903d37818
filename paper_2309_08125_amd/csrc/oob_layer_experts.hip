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
};

/* Rows of k that lie anywhere: each lane's offsets come from the rows' tokens. */
template <class E, int ROWS, int THREADS> struct Gathered : Tile<E, ROWS, THREADS, true> {
  __device__ void init(int64_t ld, int64_t left, const int32_t *rows, int per, int64_t T) {
    for (int i = 0; i < this->LOADS; i++) {
      int p = (i * THREADS + threadIdx.x) * 16, r = p / 128, c = (p / 16 % 8) ^ (r / 2 % 8);
      this->at[i] = c * 8;
      int64_t t = r < left ? rows[r] : -1;
      t = t < 0 ? -1 : t / per;
      this->off[i] = t >= 0 && t < T ? (uint32_t)(t * ld * 2 + c * 16) : OOB_LAYER_OUT;
    }
  }
};

/* The sums of one tile over `steps` steps: as in the dense product. */
template <class E, int TM, int TN, int WM, int WN, bool AK, bool BK, class TA, class TB>
__device__ inline void multiply(TA &ta, TB &tb, const char *pa, const char *pb, int64_t da, int64_t db, int64_t kleft, int steps, lds_char *lds,
                                f32x16 (&acc)[TM / WM / 32][TN / WN / 32]) {
  constexpr int FM = TM / WM / 32, FN = TN / WN / 32, STAGE = TA::BYTES + TB::BYTES;
  int wave = uniform(threadIdx.x / 64), wm = wave / WN, wn = wave % WN;
  Fragment<E, TM, FM, AK> fa;
  Fragment<E, TN, FN, BK> fb;
  fa.init(wm * FM * 32);
  fb.init(wn * FN * 32);
  for (int i = 0; i < FM; i++)
    for (int j = 0; j < FN; j++)
      for (int r = 0; r < 16; r++) acc[i][j][r] = 0;
  if (steps > 0) {
    ta.load(pa, lds, kleft);
    tb.load(pb, lds + TA::BYTES, kleft);
  }
  for (int t = 0; t < steps; t++) {
    wait_barrier(); /* the step's loads have landed, and nobody reads the other buffer any more */
    lds_char *now = lds + t % 2 * STAGE, *next = lds + (t + 1) % 2 * STAGE;
    pa += da, pb += db, kleft -= KSTEP;
    if (t + 1 < steps) {
      ta.load(pa, next, kleft);
      tb.load(pb, next + TA::BYTES, kleft);
    }
    typename Vec<E>::v8 a[2][FM], b[2][FN];
    auto fetch = [&](int s, int x) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < FM; i++) a[x][i] = fa.read(now, i, s);
#pragma unroll
      for (int j = 0; j < FN; j++) b[x][j] = fb.read(now + TA::BYTES, j, s);
    };
    fetch(0, 0);
#pragma unroll
    for (int s = 0; s < 4; s++) {
      if (s < 3) fetch(s + 1, (s + 1) % 2);
#pragma unroll
      for (int i = 0; i < FM; i++)
#pragma unroll
        for (int j = 0; j < FN; j++) acc[i][j] = mfma(b[s % 2][j], a[s % 2][i], acc[i][j]); /* lane: m, registers: n */
      constexpr int READS = FM * (AK ? 1 : 2) + FN * (BK ? 1 : 2); /* reads of the next fragments between the products */
      if (s == 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
      for (int g = 0; g < FM * FN; g++) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        if (s < 3 && g < READS) __builtin_amdgcn_sched_group_barrier(0x100, (READS + FM * FN - 1) / (FM * FN), 0);
      }
    }
  }
  __syncthreads();
}

/* A tile's sums through the epilogue: rows m0 .. m0 + left - 1 of C, 32 at a time through the wave's own part of LDS, so that a row of C
 * is written in one go. */
template <class E, int TM, int TN, int WM, int WN>
__device__ inline void finish(const Product &g, f32x16 (&acc)[TM / WM / 32][TN / WN / 32], lds_char *lds, int64_t m0, int64_t left, int64_t n0) {
  constexpr int FM = TM / WM / 32, FN = TN / WN / 32, PITCH = FN * 32 + 4, LPR = FN * 4, RPP = 64 / LPR;
  int wave = uniform(threadIdx.x / 64), wm = wave / WN, wn = wave % WN, l = lane();
  __attribute__((address_space(3))) float *stage = (__attribute__((address_space(3))) float *)lds + wave * 32 * PITCH;
#pragma unroll
  for (int i = 0; i < FM; i++) {
#pragma unroll
    for (int j = 0; j < FN; j++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        f32x4 v = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
        *(__attribute__((address_space(3))) f32x4 *)(stage + (l & 31) * PITCH + j * 32 + 8 * q + 4 * (l >> 5)) = v;
      }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int p = 0; p < 32 / RPP; p++) {
      int row = p * RPP + l / LPR, m = (wm * FM + i) * 32 + row;
      int64_t n = n0 + wn * FN * 32 + l % LPR * 8;
      float v[8];
      for (int e = 0; e < 8; e += 4) *(f32x4 *)(v + e) = *(__attribute__((address_space(3))) f32x4 *)(stage + row * PITCH + l % LPR * 8 + e);
      if (m < left && n < g.N) epilogue<E>(g, m0 + m, n, v);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  }
}

template <class E, int TM, int TN, int WM, int WN, bool AK, bool BK> constexpr int lds_bytes() {
  constexpr int stages = 2 * (TM + TN) * KSTEP * 2, out = WM * WN * 32 * (TN / WN + 4) * 4;
  return stages > out ? stages : out;
}

/* Rows of y (BK: W as it is) or of dx (W by its columns). */
template <class E, int TM, int TN, int WM, int WN, bool BK, bool GATHER>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_experts(Experts x) {
  __shared__ __attribute__((aligned(1024))) char mem[lds_bytes<E, TM, TN, WM, WN, true, BK>()];
  Product g = x.g;
  int64_t tn = g.tiles_n;
  Found f = find(x.d, [&](int64_t n) { return (n + TM - 1) / TM * tn; },
                 [&](int total) { return (int)blockIdx.x < total ? (int)xcd_order(blockIdx.x, total) : total; });
  if (f.expert < 0) return;
  /* within an expert bands of eight rows of tiles, as in the dense product */
  constexpr int BAND = 8;
  int tm = (int)(((int64_t)f.rows + TM - 1) / TM), tile = (int)f.part, band = tile / (BAND * (int)tn), in = tile - band * BAND * (int)tn;
  int high = tm - band * BAND < BAND ? tm - band * BAND : BAND;
  int64_t m0 = (int64_t)(band * BAND + in % high) * TM, n0 = (int64_t)(in / high) * TN, left = f.rows - m0, row = (int64_t)f.first + m0;

  Tile<E, TN, WM * WN * 64, BK> tb;
  tb.init(g.ldb, g.N - n0);
  const char *B = (const char *)g.B + f.expert * x.expert_stride * 2;
  const char *pb = B + (BK ? n0 * g.ldb : n0) * 2;
  int64_t db = BK ? KSTEP * 2 : KSTEP * 2 * g.ldb;
  int steps = (int)((g.K + KSTEP - 1) / KSTEP);
  f32x16 acc[TM / WM / 32][TN / WN / 32];
  if (GATHER) {
    Gathered<E, TM, WM * WN * 64> ta;
    ta.init(g.lda, left, x.rows + row, x.per, x.T);
    multiply<E, TM, TN, WM, WN, true, BK>(ta, tb, (const char *)g.A, pb, KSTEP * 2, db, g.K, steps, (lds_char *)mem, acc);
  } else {
    Tile<E, TM, WM * WN * 64, true> ta;
    ta.init(g.lda, left);
    multiply<E, TM, TN, WM, WN, true, BK>(ta, tb, (const char *)g.A + row * g.lda * 2, pb, KSTEP * 2, db, g.K, steps, (lds_char *)mem, acc);
  }
  if (g.bias) g.bias = (const E *)g.bias + f.expert * g.N;
  finish<E, TM, TN, WM, WN>(g, acc, (lds_char *)mem, row, left, n0);
}

/* dw[e] = dz^T x over the rows of e: A is dz, B is x, both with rows of k. */
template <class E, int TM, int TN, int WM, int WN> __global__ __launch_bounds__(WM *WN * 64, 2) void k_experts_dw(Experts x) {
  __shared__ __attribute__((aligned(1024))) char mem[lds_bytes<E, TM, TN, WM, WN, false, false>()];
  Product g = x.g;
  int64_t per = (int64_t)g.tiles_m * g.tiles_n, id = xcd_order(blockIdx.x, gridDim.x);
  int e = (int)(id / per), tile = (int)(id % per);
  constexpr int BAND = 8;
  int band = tile / (BAND * g.tiles_n), high = g.tiles_m - band * BAND < BAND ? g.tiles_m - band * BAND : BAND, in = tile - band * BAND * g.tiles_n;
  int64_t m0 = (int64_t)(band * BAND + in % high) * TM, n0 = (int64_t)(in / high) * TN;
  int64_t first, rows = rows_of(x.d, e, first);
  first = uniform((int)first), rows = uniform((int)rows);
  Tile<E, TM, WM * WN * 64, false> ta;
  Tile<E, TN, WM * WN * 64, false> tb;
  ta.init(g.lda, g.M - m0);
  tb.init(g.ldb, g.N - n0);
  f32x16 acc[TM / WM / 32][TN / WN / 32];
  multiply<E, TM, TN, WM, WN, false, false>(ta, tb, (const char *)g.A + (first * g.lda + m0) * 2, (const char *)g.B + (first * g.ldb + n0) * 2,
                                            KSTEP * 2 * g.lda, KSTEP * 2 * g.ldb, rows, (int)((rows + KSTEP - 1) / KSTEP), (lds_char *)mem, acc);
  g.C = (E *)g.C + (int64_t)e * g.M * g.ldc;
  finish<E, TM, TN, WM, WN>(g, acc, (lds_char *)mem, m0, g.M - m0, n0);
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

__global__ __launch_bounds__(256) void k_pack_rows(Packed p) {
  int64_t per = p.ld_to / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x, r = id / per, c = id % per * 8;
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

void pack(const Packed &k, hipStream_t st) {
  int64_t n = k.n * (k.ld_to / 8);
  if (n) k_pack_rows<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(k);
}
Operand pack_w(const oob_expert_linear_t *p, Arena &w, hipStream_t st) {
  if (w_loadable(p)) return {p->w, p->w_stride, p->expert_stride};
  int64_t ld = up(p->K, 8);
  void *to = w.take((size_t)p->E * p->N * ld * 2);
  if (w.ok() && w.base) pack({(const uint16_t *)p->w, (uint16_t *)to, p->E * p->N, p->N, p->expert_stride, p->K, p->w_stride, ld, 0, nullptr, nullptr, 1, 0}, st);
  return {to, ld, p->N * ld};
}
/* Rows of x in order of their experts. */
Operand pack_x(const oob_expert_linear_t *p, Arena &w, hipStream_t st) {
  if (!p->rows && loadable(p->x, p->x_stride, p->K)) return {p->x, p->x_stride, 0};
  int64_t ld = up(p->K, 8);
  void *to = w.take((size_t)p->R * ld * 2);
  if (w.ok() && w.base)
    pack({(const uint16_t *)p->x, (uint16_t *)to, p->R, p->R, 0, p->K, p->x_stride, ld, p->T, p->rows, p->offsets, p->per, p->E}, st);
  return {to, ld, 0};
}

int64_t tiles(int64_t n, int tile) { return (n + tile - 1) / tile; }

/* Tiles of R rows: as many as the worst division into E experts has. */
int64_t row_tiles(int64_t R, int E, int tile) { return R / tile + (R < E ? R : E); }

/* By the rows that an expert has on average. */
int choose_tile(int64_t R, int E, int64_t N) {
  int64_t mean = R / E;
  if (mean >= 192 && tiles(R, 256) * tiles(N, 256) >= 192) return 256;
  if (mean >= 96 && tiles(R, 128) * tiles(N, 128) >= 192) return 128;
  return 64;
}
int choose_dw(int64_t M, int64_t N, int E) {
  if (M >= 192 && N >= 192 && E * tiles(M, 256) * tiles(N, 256) >= 192) return 256;
  if (M >= 96 && N >= 96 && E * tiles(M, 128) * tiles(N, 128) >= 192) return 128;
  return 64;
}

template <class E, bool BK, bool GATHER> int products(Experts x, hipStream_t st) {
  int tile = choose_tile(x.d.R, x.d.E, x.g.N);
  x.g.tiles_n = (int)tiles(x.g.N, tile);
  unsigned n = (unsigned)(row_tiles(x.d.R, x.d.E, tile) * x.g.tiles_n);
  if (tile == 256) k_experts<E, 256, 256, 2, 4, BK, GATHER><<<n, 512, 0, st>>>(x);
  else if (tile == 128) k_experts<E, 128, 128, 2, 2, BK, GATHER><<<n, 256, 0, st>>>(x);
  else k_experts<E, 64, 64, 2, 2, BK, GATHER><<<n, 256, 0, st>>>(x);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}
template <class E> int products_dw(Experts x, hipStream_t st) {
  int tile = choose_dw(x.g.M, x.g.N, x.d.E);
  x.g.tiles_m = (int)tiles(x.g.M, tile), x.g.tiles_n = (int)tiles(x.g.N, tile);
  unsigned n = (unsigned)((int64_t)x.d.E * x.g.tiles_m * x.g.tiles_n);
  if (tile == 256) k_experts_dw<E, 256, 256, 2, 4><<<n, 512, 0, st>>>(x);
  else if (tile == 128) k_experts_dw<E, 128, 128, 2, 2><<<n, 256, 0, st>>>(x);
  else k_experts_dw<E, 64, 64, 2, 2><<<n, 256, 0, st>>>(x);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

bool sizes_ok(const oob_expert_linear_t *p) {
  const int64_t most = (int64_t)1 << 31;
  return p && (p->dtype == OOB_BF16 || p->dtype == OOB_FP16) && p->act >= 0 && p->act < OOB_ACTS && p->E >= 1 && p->E <= OOB_EXPERT_MAX &&
         p->per >= 1 && p->R >= 0 && p->T >= 0 && p->N >= 1 && p->K >= 1 && p->R < most && p->T < most && p->N < (1 << 21) && p->K < (1 << 21) &&
         (p->rows ? p->T * p->per == p->R : p->per == 1);
}
bool fits(int64_t blocks) { return blocks < (int64_t)1 << 31; }
/* Workgroups of the smallest tiles and of the copies, 256 threads each. */
bool launches_fit(const oob_expert_linear_t *p) {
  int64_t most = (p->N > p->K ? p->N : p->K) + 64;
  return fits(row_tiles(p->R, p->E, 64) * tiles(most, 64)) && fits(p->E * tiles(p->N, 64) * tiles(p->K, 64)) &&
         fits((p->R + p->E * p->N) * ((up(p->K, 8)) / 8) / 256 + 1);
}

size_t forward_bytes(const oob_expert_linear_t *p) {
  Arena w{nullptr, 0, 0};
  pack_w(p, w, nullptr);
  if (!x_loadable(p)) pack_x(p, w, nullptr);
  return w.used;
}

template <class E> int forward(const oob_expert_linear_t *p, Arena w, hipStream_t st) {
  Experts x{};
  Operand b = pack_w(p, w, st), a{p->x, p->x_stride, 0};
  bool gather = p->rows && x_loadable(p);
  if (!x_loadable(p)) a = pack_x(p, w, st);
  if (!w.ok()) return OOB_ECAPACITY;
  x.g.A = a.p, x.g.lda = a.ld, x.g.B = b.p, x.g.ldb = b.ld, x.expert_stride = b.part;
  x.g.N = p->N, x.g.K = p->K, x.g.bias = p->bias, x.g.C = p->y, x.g.ldc = p->y_stride, x.g.Z = p->z, x.g.ldz = p->z_stride, x.g.act = p->act;
  x.d = {p->offsets, p->E, p->R}, x.rows = p->rows, x.per = p->per, x.T = p->T;
  return gather ? products<E, true, true>(x, st) : products<E, true, false>(x, st);
}

/* dz, the runs' sums, then what the larger product takes */
bool makes_dz(const oob_expert_linear_t *p, const oob_expert_linear_grad *g) {
  return (g->dx || g->dw) && (p->act != OOB_ACT_NONE || !loadable(g->dy, g->dy_stride, p->N));
}
int run_rows(const oob_expert_linear_t *p) { /* about 1024 workgroups, 16 rows at least */
  int64_t r = up(p->R * tiles(p->N, 512) / 1024, 16);
  return (int)(r < 16 ? 16 : r > 4096 ? 4096 : r);
}
size_t sums_bytes(const oob_expert_linear_t *p) { return (size_t)row_tiles(p->R, p->E, run_rows(p)) * p->N * 4; }

size_t backward_bytes(const oob_expert_linear_t *p, const oob_expert_linear_grad *g) {
  Arena w{nullptr, 0, 0}, dx{nullptr, 0, 0}, dw{nullptr, 0, 0};
  if (makes_dz(p, g)) w.take((size_t)p->R * up(p->N, 8) * 2);
  if (g->db) w.take(sums_bytes(p));
  if (g->dx) pack_w(p, dx, nullptr);
  if (g->dw) pack_x(p, dw, nullptr);
  return w.used + (dx.used > dw.used ? dx.used : dw.used);
}

template <class E> int backward(const oob_expert_linear_t *p, const oob_expert_linear_grad *g, Arena w, hipStream_t st) {
  Operand dz{g->dy, g->dy_stride, 0};
  bool makes = makes_dz(p, g);
  if (makes) dz = {w.take((size_t)p->R * up(p->N, 8) * 2), up(p->N, 8), 0};
  float *sums = g->db ? (float *)w.take(sums_bytes(p)) : nullptr;
  if (!w.ok()) return OOB_ECAPACITY;
  Division d{p->offsets, p->E, p->R};
  if (makes || g->db) {
    ActGrad a{};
    a.d = d, a.dy = g->dy, a.ld_dy = g->dy_stride, a.z = p->z, a.ld_z = p->z_stride, a.N = p->N, a.sums = sums, a.rows = run_rows(p), a.runs = row_tiles(p->R, p->E, a.rows);
    a.dz = makes ? const_cast<void *>(dz.p) : nullptr, a.ld_dz = dz.ld;
    dim3 grid((unsigned)tiles(p->N, 512), (unsigned)a.runs);
    if (p->R) switch (p->act) {
      case OOB_ACT_RELU: k_experts_act<E, OOB_ACT_RELU><<<grid, 256, 0, st>>>(a); break;
      case OOB_ACT_GELU: k_experts_act<E, OOB_ACT_GELU><<<grid, 256, 0, st>>>(a); break;
      case OOB_ACT_GELU_TANH: k_experts_act<E, OOB_ACT_GELU_TANH><<<grid, 256, 0, st>>>(a); break;
      case OOB_ACT_SILU: k_experts_act<E, OOB_ACT_SILU><<<grid, 256, 0, st>>>(a); break;
      default: k_experts_act<E, OOB_ACT_NONE><<<grid, 256, 0, st>>>(a);
    }
    if (g->db) k_experts_db<E><<<dim3((unsigned)tiles(p->N, 64), p->E), 256, 0, st>>>(a, (E *)g->db);
  }
  int rc = hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
  if (rc == OOB_OK && g->dx && p->R) {
    Arena more = w; /* what one product takes is free again for the next on the stream */
    Operand b = pack_w(p, more, st);
    if (!more.ok()) return OOB_ECAPACITY;
    Experts x{};
    x.g.A = dz.p, x.g.lda = dz.ld, x.g.B = b.p, x.g.ldb = b.ld, x.expert_stride = b.part;
    x.g.N = p->K, x.g.K = p->N, x.g.C = g->dx, x.g.ldc = g->dx_stride, x.d = d;
    rc = products<E, false, false>(x, st);
  }
  if (rc == OOB_OK && g->dw) {
    Arena more = w;
    Operand b = pack_x(p, more, st);
    if (!more.ok()) return OOB_ECAPACITY;
    Experts x{};
    x.g.A = dz.p, x.g.lda = dz.ld, x.g.B = b.p, x.g.ldb = b.ld;
    x.g.M = p->N, x.g.N = p->K, x.g.C = g->dw, x.g.ldc = p->K, x.d = d;
    rc = products_dw<E>(x, st);
  }
  return rc;
}

bool even(const void *p) { return multiple(p, 2); }

}  // namespace
}  // namespace layer

using namespace layer;

extern "C" size_t oob_expert_linear_workspace_size(const oob_expert_linear_t *p) { return sizes_ok(p) && p->R ? forward_bytes(p) : 0; }

extern "C" int oob_expert_linear(const oob_expert_linear_t *p, void *workspace, size_t bytes, void *stream) {
  if (!sizes_ok(p) || !launches_fit(p)) return OOB_EINVAL;
  if (p->R == 0) return OOB_OK;
  if (!p->offsets || !p->x || !p->w || !p->y || p->x_stride < p->K || p->w_stride < p->K || p->y_stride < p->N || p->expert_stride < 0) return OOB_EINVAL;
  if (p->z && p->z_stride < p->N) return OOB_EINVAL;
  if (!even(p->x) || !even(p->w) || !even(p->y) || !even(p->bias) || !even(p->z) || !multiple(p->offsets, 4) || !multiple(p->rows, 4)) return OOB_EINVAL;
  if (!multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = forward_bytes(p);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? forward<bf16>(p, w, (hipStream_t)stream) : forward<fp16>(p, w, (hipStream_t)stream);
}

extern "C" size_t oob_expert_linear_backward_workspace_size(const oob_expert_linear_t *p, const oob_expert_linear_grad *g) {
  return sizes_ok(p) && g ? backward_bytes(p, g) : 0;
}

extern "C" int oob_expert_linear_backward(const oob_expert_linear_t *p, const oob_expert_linear_grad *g, void *workspace, size_t bytes, void *stream) {
  if (!sizes_ok(p) || !g || !launches_fit(p) || !fits(p->R * (p->N / 8 + 1) / 256) || !p->offsets) return OOB_EINVAL;
  if (row_tiles(p->R, p->E, run_rows(p)) > 65535 || p->E > 65535) return OOB_EINVAL;
  if (p->R && (!g->dy || g->dy_stride < p->N || (p->act != OOB_ACT_NONE && (!p->z || p->z_stride < p->N)))) return OOB_EINVAL;
  if (p->R && g->dx && (!p->w || p->w_stride < p->K || p->expert_stride < 0 || g->dx_stride < p->K)) return OOB_EINVAL;
  if (p->R && g->dw && (!p->x || p->x_stride < p->K)) return OOB_EINVAL;
  if (!even(g->dy) || !even(p->x) || !even(p->w) || !even(p->z) || !even(g->dx) || !even(g->dw) || !even(g->db)) return OOB_EINVAL;
  if (!multiple(p->offsets, 4) || !multiple(p->rows, 4) || !multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = backward_bytes(p, g);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? backward<bf16>(p, g, w, (hipStream_t)stream) : backward<fp16>(p, g, w, (hipStream_t)stream);
}
