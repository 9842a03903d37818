/* What the matrix products of a layer share, dense ones and experts': activations and their slopes, tiles on their way to LDS and to
 * registers, the epilogue. */
#ifndef OOB_LAYER_PRODUCT_H
#define OOB_LAYER_PRODUCT_H

#include "oob_layer_device.h"
#include "oob_layer_sizes.h"

namespace layer {

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

}  // namespace layer
#endif
