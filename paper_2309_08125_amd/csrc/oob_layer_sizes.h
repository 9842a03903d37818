/* Which launches a matrix product of a transformer layer (oob_layer_linear.hip) takes: plain C++, so that a CPU test compiles it too. */
#ifndef OOB_LAYER_SIZES_H
#define OOB_LAYER_SIZES_H

#include <stdint.h>

#include <initializer_list>

namespace layer {

constexpr int KSTEP = 64; /* depth of a step: 128-byte rows of k */

/* An operand as the loads meet it: rows (of m or n where k is contiguous, of k otherwise) ld elements apart. */
struct Extent { bool k_contiguous; int64_t rows, ld; };

/* A tile's loads have 32-bit byte offsets from its first element, in a buffer of 2^31 - 1 bytes: whether its rows lie near enough. */
inline bool reaches(int tile, const Extent &e) {
  int64_t most = e.k_contiguous ? tile : KSTEP, wide = e.k_contiguous ? KSTEP : tile;
  return ((e.rows < most ? e.rows : most) - 1) * e.ld + wide < (int64_t)1 << 30;
}
/* 0: not even the small one's */
inline int largest_tile(const Extent &a, const Extent &b) {
  for (int tile : {256, 128, 64})
    if (reaches(tile, a) && reaches(tile, b)) return tile;
  return 0;
}

struct Shape { int tile, splits, full, rest; };

/* Which tile, and which tiles' k is split into how many parts.  The large tile reads half as much per product as the middle one (4096 x
 * 12288 x 6144: 497 against 565 us), a workgroup of it takes a compute unit.  What is left of the last round of 256 is split so that all
 * units share it (4096 x 6144 x 12288, 384 tiles: 574 us in two rounds, 513 us in one and a half and the join), from parts of 40 steps on
 * (there, 10 steps a part lose 11 %, 20 are even, 30 gain 5 %, 40 gain 7 %); fewer tiles than units are split where that fills three quarters of
 * the units (2048 x 2048 x 12288: 103 us, the middle tile 134; 2560 x 2560: 153 and 151, but 81 and 69 at a k of 5120).  Below that the middle tile,
 * two workgroups a unit (4096 x 8192 x 2048: 163 us, the small one 245); where neither gives most units one, the small tile with k split
 * until there are two workgroups a unit and no part has under four steps (1024 x 2048 x 2048: 19 us, the middle one 26).  Tiles whose rows
 * reach too far are left out. */
inline Shape choose(int64_t M, int64_t N, int64_t K, int largest) {
  auto tiles = [&](int64_t t) { return ((M + t - 1) / t) * ((N + t - 1) / t); };
  int64_t steps = (K + KSTEP - 1) / KSTEP, n = tiles(256), rest = n % 256;
  int64_t s = rest ? 256 / rest : 1;
  if (s > steps / 40) s = steps / 40; /* see above */
  if (s > 8) s = 8;
  if (largest >= 256 && rest && s >= 2 && (n > 256 || rest * s >= 192)) return {256, (int)s, (int)(n - rest), (int)rest};
  if (largest >= 256 && n >= 192) return {256, 1, (int)n, 0};
  n = tiles(128);
  if (largest >= 128 && n >= 192) return {128, 1, (int)n, 0};
  n = tiles(64), s = 1;
  while (n * s < 512 && steps / (s * 2) >= 4 && s < 32) s *= 2;
  return s == 1 ? Shape{64, 1, (int)n, 0} : Shape{64, (int)s, 0, (int)n};
}

}  // namespace layer
#endif
