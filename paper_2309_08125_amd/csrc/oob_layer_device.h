/* Device helpers shared by the kernels of a transformer layer's operators: element types, matrix instructions, loads that go
 * straight to LDS. */
#ifndef OOB_LAYER_DEVICE_H
#define OOB_LAYER_DEVICE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "oob_layer.h"
#include "oob_plan.h"

namespace layer {

typedef __bf16 bf16;
typedef _Float16 fp16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

template <class E> struct Vec;
template <> struct Vec<bf16> { typedef bf16 v2 __attribute__((ext_vector_type(2))); typedef bf16 v4 __attribute__((ext_vector_type(4))); typedef bf16 v8 __attribute__((ext_vector_type(8))); };
template <> struct Vec<fp16> { typedef fp16 v2 __attribute__((ext_vector_type(2))); typedef fp16 v4 __attribute__((ext_vector_type(4))); typedef fp16 v8 __attribute__((ext_vector_type(8))); };
template <> struct Vec<float> { typedef float v2 __attribute__((ext_vector_type(2))); typedef float v4 __attribute__((ext_vector_type(4))); typedef float v8 __attribute__((ext_vector_type(8))); };

/* D[32][32] += A[32][16] B[16][32].  A: lane l holds row l % 32, k = 8 (l / 32) .. + 7; B: lane l holds column l % 32, the same k;
 * D: lane l holds column l % 32, register r row 8 (r / 4) + 4 (l / 32) + r % 4. */
__device__ inline f32x16 mfma(Vec<bf16>::v8 a, Vec<bf16>::v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma(Vec<fp16>::v8 a, Vec<fp16>::v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }

/* 16 bytes of LDS. */
template <class E> __device__ inline typename Vec<E>::v8 lds_read8(lds_char *p) {
  return *(__attribute__((address_space(3))) typename Vec<E>::v8 *)p;
}

/* Transposed reads: within 16 lanes that name a 4 x 16 matrix of 16-bit elements (lane j: row j / 4, columns 4 (j % 4) .. + 3), lane j
 * gets column j.  Two of them make the 8 values of k that a lane of a matrix instruction holds. */
template <class E> __device__ inline typename Vec<E>::v8 lds_read_tr(lds_char *p, lds_char *q) {
  i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)p);
  i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)q);
  return __builtin_bit_cast(typename Vec<E>::v8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

/* A buffer that starts at `base`.  Lanes in bounds have offsets below 2^31; a lane whose offset is OUT gets zeros. */
#define OOB_LAYER_OUT 0x80000000u
__device__ inline __amdgpu_buffer_rsrc_t buffer(const void *base) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(base), 0, 0x7fffffff, 0x00020000);
}

/* 64 lanes x 16 (4) bytes from `r` at each lane's offset, and `more` (which the bounds do not see), to 1024 (256) consecutive bytes of LDS. */
__device__ inline void load_lds(__amdgpu_buffer_rsrc_t r, lds_char *to, uint32_t offset, uint32_t more = 0) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)to, 16, offset, more, 0, 0);
}
__device__ inline void load_lds4(__amdgpu_buffer_rsrc_t r, lds_char *to, uint32_t offset) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)to, 4, offset, 0, 0, 0);
}
template <class V> __device__ inline V lds_numbers(lds_char *p) { return *(__attribute__((address_space(3))) V *)p; }

/* Waits for the loads in flight, then for the workgroup. */
__device__ inline void wait_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0f70); /* vmcnt(0), the others as they are */
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

__device__ inline int lane() { return threadIdx.x & 63; }
__device__ inline int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

/* Workgroups are dealt to the 8 XCDs in turn; gives consecutive work to each (a permutation of 0 .. n-1 for every n). */
__device__ inline int64_t xcd_order(int64_t id, int64_t n) {
  int64_t per = n / 8, more = n % 8, x = id % 8;
  return x * per + (x < more ? x : more) + id / 8;
}

/* Eight consecutive values of a row, `left` of them in it.  Rows start anywhere: memory takes 16-byte accesses at any address. */
template <class E> struct Loose { typedef typename Vec<E>::v8 v8 __attribute__((aligned(sizeof(E)))); };
#define OOB_GLOBAL __attribute__((address_space(1)))
template <class E> __device__ inline typename Vec<E>::v8 load8(const E *from, int64_t left) {
  const OOB_GLOBAL E *p = (const OOB_GLOBAL E *)from;
  if (left >= 8) return *(const OOB_GLOBAL typename Loose<E>::v8 *)p;
  typename Vec<E>::v8 v;
  for (int e = 0; e < 8; e++) v[e] = e < left ? p[e] : (E)0.f;
  return v;
}
template <class E> __device__ inline void store8(E *to, typename Vec<E>::v8 v, int64_t left) {
  OOB_GLOBAL E *p = (OOB_GLOBAL E *)to;
  if (left >= 8) *(OOB_GLOBAL typename Loose<E>::v8 *)p = v;
  else
    for (int e = 0; e < 8; e++)
      if (e < left) p[e] = v[e];
}

/* ---- random bits from a counter: word n of the SplitMix64 sequence (Steele, Lea, Flood 2014) whose state starts at `key` ---- */
__host__ __device__ inline uint64_t mix64(uint64_t z) {
  z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
  z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
  return z ^ (z >> 31);
}
struct Dropout {
  uint64_t key, offset;
  uint32_t threshold; /* an element is kept where its 16 bits are not below this; 0: no dropout */
  float scale;        /* 65536 / (65536 - threshold): the mean stays exactly, p being rounded to a multiple of 2^-16 */
};
static inline Dropout dropout_of(float p, uint64_t seed, uint64_t offset) {
  uint32_t t = (uint32_t)((double)p * 65536 + 0.5);
  return {mix64(seed), offset, t, (float)(65536.0 / (65536 - t))};
}
/* The 16 bits of elements i .. i + 7: element n has bits 16 (n % 4) .. + 15 of word n / 4. */
__device__ inline void random8(const Dropout &d, uint64_t i, uint64_t &lo, uint64_t &hi) {
  uint64_t n = d.offset + i;
  uint64_t at = d.key + ((n >> 2) + 1) * 0x9E3779B97F4A7C15ull;
  int shift = (int)(n & 3) * 16;
  lo = mix64(at);
  hi = mix64(at + 0x9E3779B97F4A7C15ull);
  if (shift) {
    uint64_t more = mix64(at + 2 * 0x9E3779B97F4A7C15ull);
    lo = lo >> shift | hi << (64 - shift);
    hi = hi >> shift | more << (64 - shift);
  }
}
/* keep / (1 - p) of element e of random8's */
__device__ inline float keep(const Dropout &d, uint64_t lo, uint64_t hi, int e) {
  uint32_t bits = (uint32_t)((e < 4 ? lo : hi) >> (e % 4 * 16)) & 0xffff;
  return bits >= d.threshold ? d.scale : 0.f;
}

/* ---- host ---- */
static inline int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

/* Memory handed out in order, 256 bytes apart; sizes alone when there is none.  ok() before anything that was taken is used. */
struct Arena {
  char *base;
  size_t size, used;
  void *take(size_t bytes) {
    void *p = base ? base + used : nullptr;
    used += (bytes + 255) / 256 * 256;
    return p;
  }
  bool ok() const { return used <= size; }
};

static inline bool multiple(const void *p, size_t of) { return (uintptr_t)p % of == 0; }

}  // namespace layer
#endif
