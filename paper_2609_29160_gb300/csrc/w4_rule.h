// Which kernel takes the rows of a product with a matrix in 4 bits.
#pragma once

#include <algorithm>
#include <cstdint>

namespace tre {

// Whether k_w4_few takes less than the tensor cores' kernel, by what both measured from a cold L2, on
// the device: it 7 us and 0.48, 0.72 or 0.82 us for each MB of codes and pass of up to 16, 24 or 32 rows;
// the other 8 us and 0.28 us for each 64 elements of k and round of its units (0.38 with groups of
// 64, 0.75 with 32). Groups of 128:
//   4,096 x 4,096    16 rows 13 against 26 us, 32 rows 15 against 26, 64 rows 22 against 26, 96 rows 29 against 26;
//   16,384 x 4,096   16 rows 24 against 26, 32 rows 36 against 28.
// Of 96 shapes (4,096 to 28,672 rows of 2,048 and 4,096, 9 to 112 rows of x, every group) four take the
// slower kernel: up to 96 rows by at most 4 us, 112 by 11 (4,096 x 4,096, groups of 32).
// tiles: of 16 rows of the matrix; chunks: of 64 elements of k.
inline bool few_is_quicker(int rows, int tiles, int chunks, int group, int sms) {
  if (rows <= 8) return true;
  if (rows > 96) return false;
  const float mb = tiles * 8.f * chunks * 64.f * 1e-6f;
  const float pass = rows <= 16 ? 0.48f : rows <= 24 ? 0.72f : 0.82f;
  const int pairs = std::max(1, sms / 2), rounds = ((tiles + 15) / 16 + pairs - 1) / pairs;
  const float stage = group == 32 ? 0.75f : group == 64 ? 0.38f : 0.28f;
  return 7.f + mb * pass * ((rows + 31) / 32) <= 8.f + rounds * chunks * stage;
}

}  // namespace tre
