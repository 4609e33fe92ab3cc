// Which kernel an 8-bit linear runs, and with which split over K: host arithmetic on sizes alone (no HIP).
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace qift {
namespace route {

constexpr int64_t kW8RowsMaxM = 64;   // qift_w8_rows.hip

// The tiled product: tiles of `tile` x `tile`, K cut into `parts`.
struct W8Plan {
  int tile, parts;
};
inline W8Plan w8_plan(int64_t N, int64_t M, int64_t K) {
  const int64_t big = ((N + 255) / 256) * ((M + 255) / 256);
  if (big >= 192) return {256, 1};
  const int64_t tiles = ((N + 127) / 128) * ((M + 127) / 128), steps = (K + 127) / 128;
  int64_t parts = 512 / tiles;
  if (parts > steps / 8) parts = steps / 8;
  return {128, parts < 2 ? 1 : (int)parts};
}
// Bytes of the parts' sums.
inline size_t w8_workspace(int64_t N, int64_t M, int64_t K) {
  if (M <= kW8RowsMaxM) return 0;
  const W8Plan p = w8_plan(N, M, K);
  return p.parts == 1 ? 0 : (size_t)p.parts * (size_t)M * (size_t)((N + 3) / 4 * 4) * sizeof(int32_t);
}

}  // namespace route
}  // namespace qift
