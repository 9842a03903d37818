/* Matrix products of a transformer layer: y = act(x W^T + b) + r, and its gradients. */
#include "oob_layer_device.h"
#include "oob_layer_sizes.h"

namespace layer {

/* ---- the product -------------------------------------------------------------------------------------------------------
 * C[m][n] = sum_k A(m, k) B(n, k), each operand stored with k contiguous (rows of k) or with m (n) contiguous (rows of m per k): the
 * forward product and both gradients are one kernel, the m-contiguous operand read from LDS by transposing reads, no transposed copy.
 * Tiles go to LDS by loads that pass no registers, asked for a step ahead of the products; a wave's fragments are read one sub-step ahead (5 %).
 * In the gradients' products a step ahead is not reached: before the first transposing read of a step the compiler waits for all loads in
 * flight, since it cannot tell the LDS that they write from the LDS that is read.  4096 x 6144 x 12288: forward 504 us with its join (1.23 PFLOP/s,
 * matrix cores busy 63 % of the time, the rest mostly the barrier a step), dx 550 (1.12, 46 %), dw 590 (1.05, 48 %). */
struct Product {
  const void *A, *B;
  int64_t lda, ldb; /* elements between rows */
  int64_t M, N, K;
  /* epilogue: v = act(sum + bias[n]) + residual[m][n]; z gets sum + bias[n] */
  const void *bias, *residual;
  int64_t ldr;
  void *C, *Z;
  int64_t ldc, ldz;
  float *partial; /* [splits][rest][tile][tile]: sums of the tiles whose k is split, in place of the epilogue */
  int act, splits; /* splits: of the tiles from number `full` on */
  int full, rest;
  int tiles_m, tiles_n;
};

/* 1 / (1 + e^-x).  The reciprocal instruction (1 unit of 2^-23) in place of a division, which is ten: results are rounded to 16 bits. */
__device__ inline float sigmoid(float x) { return __builtin_amdgcn_rcpf(1 + __builtin_amdgcn_exp2f(x * -1.44269504f)); }

/* Phi(z), the normal distribution's, and bell = e^(-z^2 / 2).  Phi(-|z|) = bell t Q(t) with t = 1 / (1 + 0.32 |z|): Q is the polynomial of degree
 * 7 whose largest relative error over |z| <= 60 is least (4e-7, 8e-7 in 32 bits; found by linear programming on 1500 points).  1 + erf(z / sqrt(2))
 * has no digit left below z = -5.6, and erfcf takes 92 us for the gradient of 4096 x 6144 (its bias's alone) where this takes 43. */
__device__ inline float phi(float z, float &bell) {
  float t = __builtin_amdgcn_rcpf(1 + 0.32f * fabsf(z));
  float q = 0.03451068627f;
  q = q * t - 0.12242049668f;
  q = q * t + 0.10613986935f;
  q = q * t + 0.01553882127f;
  q = q * t + 0.09740863787f;
  q = q * t + 0.11342795430f;
  q = q * t + 0.12773489272f;
  q = q * t + 0.12765983351f;
  bell = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
  float tail = bell * t * q;
  return z < 0 ? tail : 1 - tail;
}

__device__ inline float activate(float z, int act) {
  switch (act) {
    case OOB_ACT_RELU: return z > 0 ? z : (z != z ? z : 0.f);
    case OOB_ACT_SILU: return z * sigmoid(z);
    case OOB_ACT_GELU: { float bell; return z * phi(z, bell); }
    case OOB_ACT_GELU_TANH: return z * sigmoid(1.5957691216f * (z + 0.044715f * z * z * z)); /* 0.5 (1 + tanh(u)) = sigmoid(2 u) */
    default: return z;
  }
}

/* act'(z).  Beyond +-1000 the smooth ones are 1 and 0 to the last bit, and their formulas would meet 0 times infinity: z of float16 is an
 * infinity from 65520 on, its square one of bfloat16 from 2^64 on. */
__device__ inline float slope(float z, int act) {
  if (act != OOB_ACT_NONE && act != OOB_ACT_RELU) z = __builtin_elementwise_minimum(__builtin_elementwise_maximum(z, -1000.f), 1000.f); /* NaN stays */
  switch (act) {
    case OOB_ACT_RELU: return z > 0 ? 1.f : (z != z ? z : 0.f);
    case OOB_ACT_SILU: { float e = sigmoid(z); return e * (1 + z * (1 - e)); }
    case OOB_ACT_GELU: { float bell, p = phi(z, bell); return p + z * 0.39894228f * bell; }
    case OOB_ACT_GELU_TANH: {
      float e = sigmoid(1.5957691216f * (z + 0.044715f * z * z * z)); /* its derivative is 2 e (1 - e) u' */
      return e + z * 2 * e * (1 - e) * 0.7978845608f * (1 + 0.134145f * z * z);
    }
    default: return 1.f;
  }
}

/* One operand's tile of ROWS (m or n) x KSTEP in LDS and the way from memory to there and to registers.
 * k contiguous: ROWS rows of 128 bytes, eight 16-byte chunks, chunk c of row r at c ^ (r / 2) % 8: sixteen lanes that read one chunk
 * of sixteen rows then meet all 64 banks.  m contiguous: KSTEP rows of 2 ROWS bytes, chunk c of row k at c ^ 4 (k % 4) (64-row tiles:
 * c ^ 4 (k / 2 % 2)): the four rows of a transposed read lie in different quarters of the banks. */
template <class E, int ROWS, int THREADS, bool KC> struct Tile {
  static constexpr int BYTES = ROWS * KSTEP * 2;
  static constexpr int LOADS = BYTES / (THREADS * 16);
  uint32_t off[LOADS]; /* this lane's byte offsets from the start of the step */
  int at[LOADS];       /* first k of the 16 bytes (k contiguous) or the row k */

  __device__ void init(int64_t ld, int64_t left) { /* left: rows (m or n) there are from the tile's first on */
    for (int i = 0; i < LOADS; i++) {
      int p = (i * THREADS + threadIdx.x) * 16;
      if (KC) {
        int r = p / 128, c = (p / 16 % 8) ^ (r / 2 % 8);
        at[i] = c * 8;
        off[i] = r < left ? (uint32_t)(r * ld * 2 + c * 16) : OOB_LAYER_OUT;
      } else {
        constexpr int CH = ROWS / 8;
        int k = p / (ROWS * 2), c = (p / 16 % CH) ^ (ROWS == 64 ? k / 2 % 2 * 4 : k % 4 * 4);
        at[i] = k;
        off[i] = c * 8 < left ? (uint32_t)(k * ld * 2 + c * 16) : OOB_LAYER_OUT;
      }
    }
  }
  /* Asks for the step that starts at `base`; kleft: values of k there are from here on. */
  __device__ void load(const char *base, lds_char *to, int64_t kleft) {
    __amdgpu_buffer_rsrc_t r = buffer(base);
    int wave = uniform(threadIdx.x / 64);
#pragma unroll
    for (int i = 0; i < LOADS; i++)
      load_lds(r, to + (i * THREADS + wave * 64) * 16, at[i] < kleft ? off[i] : OOB_LAYER_OUT);
  }
};

/* Fragment reads: the lane's byte offsets in a tile for a wave whose rows start at w0 (a multiple of 32). */
template <class E, int ROWS, int FR, bool KC> struct Fragment {
  int o[KC ? 4 : FR];
  __device__ void init(int w0) {
    int l = lane(), h = l >> 5;
    if (KC) {
      int r = w0 + (l & 31);
      for (int s = 0; s < 4; s++) o[s] = r * 128 + (((2 * s + h) ^ (r / 2 % 8)) * 16);
    } else {
      int j = (l & 15) >> 2, k = 8 * h + j;
      int x = ROWS == 64 ? k / 2 % 2 * 4 : k % 4 * 4;
      for (int i = 0; i < FR; i++) o[i] = k * ROWS * 2 + ((((w0 + 32 * i) / 8 + ((l >> 4) & 1) * 2 + ((l >> 1) & 1)) ^ x) * 16) + (l & 1) * 8;
    }
  }
  __device__ typename Vec<E>::v8 read(lds_char *tile, int i, int s) const {
    if (KC) return lds_read8<E>(tile + o[s] + i * 32 * 128);
    lds_char *p = tile + o[i] + s * 16 * ROWS * 2;
    return lds_read_tr<E>(p, p + 4 * ROWS * 2);
  }
};

/* Eight consecutive values of one row through the epilogue. */
template <class E> __device__ inline void epilogue(const Product &g, int64_t m, int64_t n, float *v) {
  int64_t left = g.N - n;
  if (g.bias) {
    const E *b = (const E *)g.bias + n;
    for (int e = 0; e < 8; e++) v[e] += e < left ? (float)b[e] : 0.f;
  }
  typename Vec<E>::v8 out;
  if (g.Z) { /* rounded to the type, as y is: half the memory between the passes; act' sees the rounding, act does not */
    for (int e = 0; e < 8; e++) out[e] = (E)v[e];
    store8<E>((E *)g.Z + m * g.ldz + n, out, left);
  }
  switch (g.act) { /* outside the loop: once for eight values */
    case OOB_ACT_RELU: for (int e = 0; e < 8; e++) v[e] = activate(v[e], OOB_ACT_RELU); break;
    case OOB_ACT_SILU: for (int e = 0; e < 8; e++) v[e] = activate(v[e], OOB_ACT_SILU); break;
    case OOB_ACT_GELU: for (int e = 0; e < 8; e++) v[e] = activate(v[e], OOB_ACT_GELU); break;
    case OOB_ACT_GELU_TANH: for (int e = 0; e < 8; e++) v[e] = activate(v[e], OOB_ACT_GELU_TANH); break;
  }
  if (g.residual) {
    typename Vec<E>::v8 r = load8<E>((const E *)g.residual + m * g.ldr + n, left);
    for (int e = 0; e < 8; e++) v[e] += (float)r[e];
  }
  for (int e = 0; e < 8; e++) out[e] = (E)v[e];
  store8<E>((E *)g.C + m * g.ldc + n, out, left);
}

/* Where a tile lies: bands of eight rows of tiles, so that consecutive workgroups of an XCD share rows of both operands in its L2. */
template <int TILE> __device__ inline void locate(const Product &g, int tile, int64_t &m0, int64_t &n0) {
  constexpr int BAND = 8;
  int band = tile / (BAND * g.tiles_n), high = g.tiles_m - band * BAND < BAND ? g.tiles_m - band * BAND : BAND, in = tile - band * BAND * g.tiles_n;
  m0 = (int64_t)(band * BAND + in % high) * TILE, n0 = (int64_t)(in / high) * TILE;
}

template <class E, int TM, int TN, int WM, int WN, bool AK, bool BK>
__global__ __launch_bounds__(WM *WN * 64, 2) void k_product(Product g) {
  constexpr int THREADS = WM * WN * 64, FM = TM / WM / 32, FN = TN / WN / 32;
  using TA = Tile<E, TM, THREADS, AK>;
  using TB = Tile<E, TN, THREADS, BK>;
  constexpr int STAGE = TA::BYTES + TB::BYTES, PITCH = FN * 32 + 4;
  constexpr int EPI = WM * WN * 32 * PITCH * 4;
  __shared__ __attribute__((aligned(1024))) char mem[2 * STAGE > EPI ? 2 * STAGE : EPI];
  lds_char *lds = (lds_char *)mem;

  int tile, split = 0, splits = 1;
  if ((int)blockIdx.x < g.full) {
    tile = (int)xcd_order(blockIdx.x, g.full);
  } else {
    int id = (int)xcd_order(blockIdx.x - g.full, (int64_t)g.rest * g.splits);
    tile = g.full + id % g.rest, split = id / g.rest, splits = g.splits;
  }
  int64_t m0, n0;
  locate<TM>(g, tile, m0, n0);

  int steps = (int)((g.K + KSTEP - 1) / KSTEP);
  int first = (int)((int64_t)steps * split / splits), last = (int)((int64_t)steps * (split + 1) / splits);

  TA ta;
  TB tb;
  ta.init(g.lda, g.M - m0);
  tb.init(g.ldb, g.N - n0);
  const char *pa = (const char *)g.A + (AK ? m0 * g.lda + (int64_t)first * KSTEP : (int64_t)first * KSTEP * g.lda + m0) * 2;
  const char *pb = (const char *)g.B + (BK ? n0 * g.ldb + (int64_t)first * KSTEP : (int64_t)first * KSTEP * g.ldb + n0) * 2;
  int64_t da = AK ? KSTEP * 2 : KSTEP * 2 * g.lda, db = BK ? KSTEP * 2 : KSTEP * 2 * g.ldb;
  int64_t kleft = g.K - (int64_t)first * KSTEP;

  int wave = uniform(threadIdx.x / 64), wm = wave / WN, wn = wave % WN;
  Fragment<E, TM, FM, AK> fa;
  Fragment<E, TN, FN, BK> fb;
  fa.init(wm * FM * 32);
  fb.init(wn * FN * 32);

  f32x16 acc[FM][FN];
  for (int i = 0; i < FM; i++)
    for (int j = 0; j < FN; j++)
      for (int r = 0; r < 16; r++) acc[i][j][r] = 0;

  if (first < last) {
    ta.load(pa, lds, kleft);
    tb.load(pb, lds + TA::BYTES, kleft);
  }
  for (int t = first; t < last; t++) {
    wait_barrier(); /* the step's loads have landed, and nobody reads the other buffer any more */
    lds_char *now = lds + (t - first) % 2 * STAGE, *next = lds + (t - first + 1) % 2 * STAGE;
    pa += da, pb += db, kleft -= KSTEP;
    if (t + 1 < last) {
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
      /* reads of the next fragments between the products */
      constexpr int READS = FM * (AK ? 1 : 2) + FN * (BK ? 1 : 2);
      if (s == 0) __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
#pragma unroll
      for (int g = 0; g < FM * FN; g++) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        if (s < 3 && g < READS) __builtin_amdgcn_sched_group_barrier(0x100, (READS + FM * FN - 1) / (FM * FN), 0);
      }
    }
  }
  __syncthreads();

  /* 32 rows of m at a time through the wave's own part of LDS, so that a row of C is written in one go */
  __attribute__((address_space(3))) float *stage = (__attribute__((address_space(3))) float *)lds + wave * 32 * PITCH;
  int l = lane();
  constexpr int LPR = FN * 4, RPP = 64 / LPR; /* lanes per row, rows per pass */
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
      int row = p * RPP + l / LPR;
      int64_t m = m0 + (wm * FM + i) * 32 + row, n = n0 + wn * FN * 32 + l % LPR * 8;
      float v[8];
      for (int e = 0; e < 8; e += 4) *(f32x4 *)(v + e) = *(__attribute__((address_space(3))) f32x4 *)(stage + row * PITCH + l % LPR * 8 + e);
      if (m < g.M && n < g.N) {
        if (splits > 1) {
          float *to = g.partial + ((int64_t)split * g.rest + (tile - g.full)) * TM * TN + (m - m0) * TN + (n - n0);
          for (int e = 0; e < 8; e += 4) *(f32x4 *)(to + e) = f32x4{v[e], v[e + 1], v[e + 2], v[e + 3]};
        } else {
          epilogue<E>(g, m, n, v);
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
  }
}

/* Joins the parts of the tiles whose k was split. */
template <class E, int TILE> __global__ __launch_bounds__(256) void k_join(Product g) {
  constexpr int PER = TILE * TILE / 8 / 256; /* workgroups a tile, eight values a thread */
  int tile = blockIdx.x / PER, at = (blockIdx.x % PER * 256 + threadIdx.x) * 8;
  int64_t m, n;
  locate<TILE>(g, g.full + tile, m, n);
  m += at / TILE, n += at % TILE;
  if (m >= g.M || n >= g.N) return;
  float v[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
  for (int s = 0; s < g.splits; s++) {
    const float *p = g.partial + ((int64_t)s * g.rest + tile) * TILE * TILE + at;
    f32x4 lo = *(const f32x4 *)p, hi = *(const f32x4 *)(p + 4);
    for (int e = 0; e < 4; e++) v[e] += lo[e], v[4 + e] += hi[e];
  }
  epilogue<E>(g, m, n, v);
}

/* ---- rows of another pitch: what the product's loads cannot take (rows that do not start at 16 bytes, a ragged contiguous axis)
 * goes to the workspace first, in rows of a multiple of 8 with zeros behind. */
struct Packed { const uint16_t *from; uint16_t *to; int64_t rows, cols, ld, ld_to; };

__global__ __launch_bounds__(256) void k_pack(Packed p) {
  int64_t per = p.ld_to / 8, id = (int64_t)blockIdx.x * 256 + threadIdx.x;
  int64_t r = id / per, c = id % per * 8;
  if (r >= p.rows) return;
  i16x8 v;
  for (int e = 0; e < 8; e++) v[e] = c + e < p.cols ? (short)p.from[r * p.ld + c + e] : (short)0;
  *(i16x8 *)(p.to + r * p.ld_to + c) = v;
}

/* ---- dz = dy act'(z), and the sums of its columns ------------------------------------------------------------------------
 * A workgroup takes 512 columns (64 lanes x 8) and a run of rows, four rows at a time, and leaves one row of sums. */
struct ActGrad {
  const void *dy, *z;
  void *dz; /* rows of a multiple of 8; null: act is none, dz is dy */
  int64_t ld_dy, ld_z, ld_dz, T, N;
  float *sums; /* [runs][N] or null */
  int64_t rows; /* of a run */
};

template <class E, int ACT> __global__ __launch_bounds__(256) void k_act_grad(ActGrad g) {
  __shared__ float part[4][512 + 8];
  int64_t n = (int64_t)blockIdx.x * 512 + lane() * 8, left = g.N - n;
  int64_t t1 = ((int64_t)blockIdx.y + 1) * g.rows < g.T ? ((int64_t)blockIdx.y + 1) * g.rows : g.T;
  float sum[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  const int64_t stop = left > 0 ? t1 : 0;
  for (int64_t t0 = (int64_t)blockIdx.y * g.rows + threadIdx.x / 64; t0 < stop; t0 += 16) {
    typename Vec<E>::v8 d[4], z[4], out; /* four rows on their way before the first is worked on */
#pragma unroll
    for (int u = 0; u < 4; u++)
      if (t0 + 4 * u < stop) {
        d[u] = load8<E>((const E *)g.dy + (t0 + 4 * u) * g.ld_dy + n, left);
        if (g.dz && ACT != OOB_ACT_NONE) z[u] = load8<E>((const E *)g.z + (t0 + 4 * u) * g.ld_z + n, left);
      }
#pragma unroll
    for (int u = 0; u < 4; u++) {
      if (t0 + 4 * u >= stop) continue;
      if (g.dz) {
        for (int e = 0; e < 8; e++) {
          float v = (float)d[u][e] * slope(ACT == OOB_ACT_NONE ? 0.f : (float)z[u][e], ACT);
          out[e] = (E)v; /* the matrix cores take 16 bits: dx and dw see this rounding */
          sum[e] += v;   /* the bias's gradient does not */
        }
        store8<E>((E *)g.dz + (t0 + 4 * u) * g.ld_dz + n, out, 8); /* past N: zeros */
      } else {
        for (int e = 0; e < 8; e++) sum[e] += (float)d[u][e];
      }
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

template <class E> __global__ __launch_bounds__(256) void k_sum_rows(const float *sums, int64_t runs, int64_t N, E *out) {
  __shared__ float part[4][64];
  int64_t n = (int64_t)blockIdx.x * 64 + lane();
  float s = 0;
  if (n < N)
    for (int64_t r = threadIdx.x / 64; r < runs; r += 4) s += sums[r * N + n];
  part[threadIdx.x / 64][lane()] = s;
  __syncthreads();
  if (threadIdx.x < 64 && n < N) out[n] = (E)((part[0][threadIdx.x] + part[1][threadIdx.x]) + (part[2][threadIdx.x] + part[3][threadIdx.x]));
}

/* ---- host ------------------------------------------------------------------------------------------------------------------ */
struct Operand { const void *p; int64_t ld, rows, cols; }; /* stored rows x cols, ld elements apart */

/* What the loads to LDS can take: 16-byte pieces of rows that end with the row, no long way between rows. */
static bool loadable(const Operand &o) { return o.cols % 8 == 0 && multiple(o.p, 16) && o.ld % 8 == 0 && o.ld < (1 << 21); }

static size_t partial_bytes(const Shape &s) { return s.rest ? (size_t)s.splits * s.rest * s.tile * s.tile * 4 : 0; }

/* As the product meets it: itself or its copy, ak: k contiguous. */
static Extent extent(const Operand &o, bool k_contiguous) { return {k_contiguous, o.rows, loadable(o) ? o.ld : up(o.cols, 8)}; }
static int largest_tile(const Operand &a, bool ak, const Operand &b, bool bk) { return largest_tile(extent(a, ak), extent(b, bk)); }

static size_t product_workspace(const Operand &a, bool ak, const Operand &b, bool bk, int64_t M, int64_t N, int64_t K) {
  Arena w{nullptr, 0, 0};
  if (!loadable(a)) w.take((size_t)a.rows * up(a.cols, 8) * 2);
  if (!loadable(b)) w.take((size_t)b.rows * up(b.cols, 8) * 2);
  Shape s = choose(M, N, K, largest_tile(a, ak, b, bk));
  w.take(partial_bytes(s));
  return w.used;
}

static Operand pack(const Operand &o, Arena &w, hipStream_t st) {
  if (loadable(o)) return o;
  int64_t ld = up(o.cols, 8);
  void *to = w.take((size_t)o.rows * ld * 2);
  int64_t n = o.rows * (ld / 8);
  if (n && w.ok()) k_pack<<<(unsigned)((n + 255) / 256), 256, 0, st>>>(Packed{(const uint16_t *)o.p, (uint16_t *)to, o.rows, o.cols, o.ld, ld});
  return {to, ld, o.rows, ld};
}

template <class E, bool AK, bool BK> static void launch(const Product &g, int tile, hipStream_t st) {
  unsigned n = (unsigned)(g.full + (int64_t)g.rest * g.splits);
  if (tile == 256) k_product<E, 256, 256, 2, 4, AK, BK><<<n, 512, 0, st>>>(g);
  else if (tile == 128) k_product<E, 128, 128, 2, 2, AK, BK><<<n, 256, 0, st>>>(g);
  else k_product<E, 64, 64, 2, 2, AK, BK><<<n, 256, 0, st>>>(g);
  if (g.rest && tile == 256) k_join<E, 256><<<(unsigned)g.rest * 32, 256, 0, st>>>(g);
  else if (g.rest) k_join<E, 64><<<(unsigned)g.rest * 2, 256, 0, st>>>(g);
}

/* The product with its operands as they are stored: ak (bk) says that k is contiguous.  The arena comes by value: what one product
 * takes is free again for the next on the stream, as the workspace's size has it. */
template <class E> static int product(Operand a, bool ak, Operand b, bool bk, Product g, Arena w, hipStream_t st) {
  if (g.M == 0 || g.N == 0) return OOB_OK;
  int largest = largest_tile(a, ak, b, bk);
  if (!largest) return OOB_EINVAL;
  Shape s = choose(g.M, g.N, g.K, largest);
  a = pack(a, w, st);
  b = pack(b, w, st);
  g.A = a.p, g.lda = a.ld, g.B = b.p, g.ldb = b.ld;
  g.splits = s.splits, g.full = s.full, g.rest = s.rest;
  g.partial = (float *)w.take(partial_bytes(s));
  if (!w.ok()) return OOB_ECAPACITY;
  g.tiles_m = (int)((g.M + s.tile - 1) / s.tile), g.tiles_n = (int)((g.N + s.tile - 1) / s.tile);
  if (ak && bk) launch<E, true, true>(g, s.tile, st);
  else if (ak) launch<E, true, false>(g, s.tile, st);
  else launch<E, false, false>(g, s.tile, st);
  return hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
}

static bool sizes_ok(int dtype, int act, int64_t T, int64_t N, int64_t K) {
  const int64_t most = (int64_t)1 << 31;
  return (dtype == OOB_BF16 || dtype == OOB_FP16) && act >= 0 && act < OOB_ACTS && T >= 0 && N >= 1 && K >= 1 && T < most && N < most && K < most;
}
static bool fits(int64_t a, int64_t b) { /* workgroups of the smallest tile and its parts */
  return ((a + 63) / 64) * ((b + 63) / 64) < ((int64_t)1 << 31) / 64;
}

static int64_t runs_of(int64_t T, int64_t N) { /* runs of rows of k_act_grad: about 1024 workgroups, 16 rows at least */
  int64_t r = 1024 / ((N + 511) / 512);
  if (r > (T + 15) / 16) r = (T + 15) / 16;
  return r < 1 ? 1 : r;
}

static size_t linear_bytes(const oob_linear *p) {
  return product_workspace({p->x, p->x_stride, p->T, p->K}, true, {p->w, p->w_stride, p->N, p->K}, true, p->T, p->N, p->K);
}

template <class E> static int linear(const oob_linear *p, Arena w, hipStream_t st) {
  Product g{};
  g.M = p->T, g.N = p->N, g.K = p->K;
  g.bias = p->bias, g.residual = p->residual, g.ldr = p->residual_stride;
  g.C = p->y, g.ldc = p->y_stride, g.Z = p->z, g.ldz = p->z_stride, g.act = p->act;
  return product<E>({p->x, p->x_stride, p->T, p->K}, true, {p->w, p->w_stride, p->N, p->K}, true, g, w, st);
}

/* dz in the workspace (rows of a multiple of 8, zeros behind) where there is an activation or the products cannot load dy as it is;
 * then the sums of the bias's gradient and what the larger product takes */
static bool makes_dz(const oob_linear_grad *p) { return p->act != OOB_ACT_NONE || !loadable({p->dy, p->dy_stride, p->T, p->N}); }
static Operand dz_of(const oob_linear_grad *p, Arena &w) {
  if (!makes_dz(p)) return {p->dy, p->dy_stride, p->T, p->N};
  int64_t ld = up(p->N, 8);
  return {w.take((size_t)p->T * ld * 2), ld, p->T, ld};
}

/* Whether the products' loads reach their rows. */
static bool rows_ok(const oob_linear *p) {
  return largest_tile({p->x, p->x_stride, p->T, p->K}, true, {p->w, p->w_stride, p->N, p->K}, true) > 0;
}
static bool rows_ok(const oob_linear_grad *p) {
  Arena none{nullptr, 0, 0};
  Operand dz = dz_of(p, none);
  return (!p->dx || !p->T || largest_tile(dz, true, {p->w, p->w_stride, p->N, p->K}, false) > 0) &&
         (!p->dw || largest_tile(dz, false, {p->x, p->x_stride, p->T, p->K}, false) > 0);
}

static size_t grad_bytes(const oob_linear_grad *p) {
  Arena w{nullptr, 0, 0};
  Operand dz = dz_of(p, w);
  if (p->db) w.take((size_t)runs_of(p->T, p->N) * p->N * 4);
  size_t dx = p->dx ? product_workspace(dz, true, {p->w, p->w_stride, p->N, p->K}, false, p->T, p->K, p->N) : 0;
  size_t dw = p->dw ? product_workspace(dz, false, {p->x, p->x_stride, p->T, p->K}, false, p->N, p->K, p->T) : 0;
  return w.used + (dx > dw ? dx : dw);
}

template <class E> static int linear_grad(const oob_linear_grad *p, Arena w, hipStream_t st) {
  Operand dz = dz_of(p, w);
  float *sums = p->db ? (float *)w.take((size_t)runs_of(p->T, p->N) * p->N * 4) : nullptr;
  if (!w.ok()) return OOB_ECAPACITY;
  bool makes = makes_dz(p);
  if (makes || sums) {
    ActGrad a{};
    a.dy = p->dy, a.ld_dy = p->dy_stride, a.z = p->z, a.ld_z = p->z_stride;
    a.dz = makes ? const_cast<void *>(dz.p) : nullptr, a.ld_dz = dz.ld;
    a.T = p->T, a.N = p->N, a.sums = sums;
    int64_t runs = runs_of(p->T, p->N);
    a.rows = (p->T + runs - 1) / runs;
    dim3 grid((unsigned)((p->N + 511) / 512), (unsigned)runs);
    switch (p->act) {
      case OOB_ACT_RELU: k_act_grad<E, OOB_ACT_RELU><<<grid, 256, 0, st>>>(a); break;
      case OOB_ACT_GELU: k_act_grad<E, OOB_ACT_GELU><<<grid, 256, 0, st>>>(a); break;
      case OOB_ACT_GELU_TANH: k_act_grad<E, OOB_ACT_GELU_TANH><<<grid, 256, 0, st>>>(a); break;
      case OOB_ACT_SILU: k_act_grad<E, OOB_ACT_SILU><<<grid, 256, 0, st>>>(a); break;
      default: k_act_grad<E, OOB_ACT_NONE><<<grid, 256, 0, st>>>(a);
    }
    if (sums) k_sum_rows<E><<<(unsigned)((p->N + 63) / 64), 256, 0, st>>>(sums, runs, p->N, (E *)p->db);
  }
  int rc = hipGetLastError() == hipSuccess ? OOB_OK : OOB_EHIP;
  if (rc == OOB_OK && p->dx) {
    Product g{};
    g.M = p->T, g.N = p->K, g.K = p->N, g.C = p->dx, g.ldc = p->dx_stride;
    rc = product<E>(dz, true, {p->w, p->w_stride, p->N, p->K}, false, g, w, st);
  }
  if (rc == OOB_OK && p->dw) {
    Product g{};
    g.M = p->N, g.N = p->K, g.K = p->T, g.C = p->dw, g.ldc = p->dw_stride;
    rc = product<E>(dz, false, {p->x, p->x_stride, p->T, p->K}, false, g, w, st);
  }
  return rc;
}

static bool even(const void *p) { return multiple(p, 2); }

}  // namespace layer

using namespace layer;

extern "C" size_t oob_layer_linear_workspace_size(const oob_linear *p) {
  return p && sizes_ok(p->dtype, p->act, p->T, p->N, p->K) ? linear_bytes(p) : 0;
}

extern "C" int oob_layer_linear(const oob_linear *p, void *workspace, size_t bytes, void *stream) {
  if (!p || !sizes_ok(p->dtype, p->act, p->T, p->N, p->K) || !fits(p->T, p->N)) return OOB_EINVAL;
  if (p->T == 0) return OOB_OK;
  if (!p->x || !p->w || !p->y || p->x_stride < p->K || p->w_stride < p->K || p->y_stride < p->N) return OOB_EINVAL;
  if ((p->residual && p->residual_stride < p->N) || (p->z && p->z_stride < p->N)) return OOB_EINVAL;
  if (!even(p->x) || !even(p->w) || !even(p->y) || !even(p->bias) || !even(p->residual) || !even(p->z)) return OOB_EINVAL;
  if (!rows_ok(p) || !multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = linear_bytes(p);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? linear<bf16>(p, w, (hipStream_t)stream) : linear<fp16>(p, w, (hipStream_t)stream);
}

extern "C" size_t oob_layer_linear_backward_workspace_size(const oob_linear_grad *p) {
  return p && sizes_ok(p->dtype, p->act, p->T, p->N, p->K) ? grad_bytes(p) : 0;
}

extern "C" int oob_layer_linear_backward(const oob_linear_grad *p, void *workspace, size_t bytes, void *stream) {
  if (!p || !sizes_ok(p->dtype, p->act, p->T, p->N, p->K) || !fits(p->T, p->N) || !fits(p->T, p->K) || !fits(p->N, p->K)) return OOB_EINVAL;
  if (p->T && (!p->dy || p->dy_stride < p->N)) return OOB_EINVAL;
  if (p->T && p->act != OOB_ACT_NONE && (!p->z || p->z_stride < p->N)) return OOB_EINVAL;
  if (p->T && p->dx && (!p->w || p->w_stride < p->K || p->dx_stride < p->K)) return OOB_EINVAL;
  if (p->dw && ((p->T && (!p->x || p->x_stride < p->K)) || p->dw_stride < p->K)) return OOB_EINVAL;
  if (!even(p->dy) || !even(p->x) || !even(p->w) || !even(p->z) || !even(p->dx) || !even(p->dw) || !even(p->db)) return OOB_EINVAL;
  if (!rows_ok(p) || !multiple(workspace, 256)) return OOB_EINVAL;
  size_t need = grad_bytes(p);
  if (need > bytes || (need && !workspace)) return OOB_ECAPACITY;
  Arena w{(char *)workspace, bytes, 0};
  return p->dtype == OOB_BF16 ? linear_grad<bf16>(p, w, (hipStream_t)stream) : linear_grad<fp16>(p, w, (hipStream_t)stream);
}
