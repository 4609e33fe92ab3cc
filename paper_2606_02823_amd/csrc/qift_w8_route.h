// Which kernel an 8-bit linear runs, and with which split over K: host arithmetic on sizes alone (no HIP).
//
// What the kernels' times follow is the bytes that a CU takes in: about 27 a ns to registers (qift_w8_rows.hip) and up to
// 54 a ns to LDS (qift_w8_gemm.hip), whatever the matrix cores do meanwhile, and for few tokens the weights' bytes from
// memory.  So a plan is the least of the times below (ns), which were fitted to these measured ones (us, rows x K at tokens;
// estimates in brackets):
//   rows of 16: 4096 x 4096 at 1 token 5.9 (5.6), 28672 x 4096 24.1 (26), 4096 x 14336 13.5 (14), 4096 x 4096 at 32 8.4 (8.8),
//     28672 x 4096 at 16 35 (36); rows of 32: 6144 x 4096 at 24 10.3 (10)
//   128 x 32 tiles: 28672 x 4096 at 16 27 (27); 128 x 64: 2500 x 4096 at 600 15 (18), 4096 x 11008 at 333 41 (43), 4096 x 14336 at 64,
//     8 parts, 19 (20)
//   128 x 128: 4096 x 4096 at 1024 26 (30), 4096 x 11008 at 333 75 (73), in 2 parts 45 (46), in 5 33 (39)
//   256 x 256: 9000 x 4096 at 1500 56 (56), 4096 x 14336 at 2048 162 (164), in 2 parts 117 (126), 28672 x 4096 at 4096 412 (408)
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace qift {
namespace route {

constexpr int64_t kW8RowsMaxM = 32;   // two token tiles of 16
constexpr int kCus = 256;

struct W8Plan {
  int rows;         // weight rows of a workgroup of the rows kernel (16, 32 or 64); 0: the tiled product
  int bn, bm;       // its tiles
  int parts;        // parts of K
  double ns;        // estimate
};

inline int64_t w8_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline W8Plan w8_plan(int64_t N, int64_t M, int64_t K, bool split) {
  const int64_t steps = w8_ceil(K, 128);
  const double stream = (double)N * (double)K / 4800.0;   // the weights from memory
  W8Plan best = {0, 0, 0, 1, 1e300};
  if (M <= kW8RowsMaxM) {
    const int rows[] = {16, 32, 64};
    for (int r : rows) {
      if (r == 64 && M <= 16) continue;
      const int64_t count = w8_ceil(N, r), each = w8_ceil(count, kCus);
      const double in = (double)each * (double)(r + M) * (double)K / 27.0;
      const double out = stream * (double)(each * kCus) / (double)count;   // the fullest CU's part of the stream
      const double ns = 1500.0 + (in > out ? in : out);
      if (ns <= best.ns) best = {r, 0, 0, 1, ns};
    }
  }
  // step times of a CU with one and with two workgroups, and what a workgroup takes beside its steps
  const struct {
    int bn, bm;
    double one, two, fixed;
  } tiles[] = {{128, 32, 400, 750, 3500}, {128, 64, 450, 900, 4000}, {128, 128, 800, 1150, 4000}, {256, 256, 1450, 3100, 6000}};
  for (const auto& t : tiles) {
    if (t.bm < 64 && M > t.bm) continue;
    const int64_t count = w8_ceil(N, t.bn) * w8_ceil(M, t.bm);
    for (int p = 1; p <= (split ? 16 : 1); ++p) {
      if (p > 1 && (p > steps / 4 || count * p > 2 * kCus || M > 65535)) break;
      const int64_t each = w8_ceil(count * p, kCus);   // workgroups of the fullest CU
      const double turn = (double)w8_ceil(steps, p) * ((double)(each / 2) * t.two + (double)(each & 1) * t.one);
      const double rounds = t.bn == 256 ? (double)each : 1.0;   // (only these stand alone on their CU to the end)
      double ns = (turn > stream ? turn : stream) + rounds * t.fixed;
      if (p > 1) ns += 3000.0 + 8.0 * p * (double)M * (double)N / 5000.0;   // the sums out and in, and their launch
      if (ns < best.ns) best = {0, t.bn, t.bm, p, ns};
    }
  }
  return best;
}
// Bytes of the parts' sums.
inline size_t w8_workspace(const W8Plan& p, int64_t N, int64_t M) {
  return p.parts == 1 ? 0 : (size_t)p.parts * (size_t)M * (size_t)(w8_ceil(N, 4) * 4) * sizeof(int32_t);
}

}  // namespace route
}  // namespace qift
