// Which kernel an 8-bit linear runs, and with which split over K: host arithmetic on sizes alone (no HIP).
//
// What the kernels' times follow is the bytes that a CU takes in: about 27 a ns to registers (qift_w8_rows.hip) and up to
// 54 a ns to LDS (qift_w8_gemm.hip), whatever the matrix cores do meanwhile, and for few tokens the weights' bytes from
// memory.  So a plan is the least of the times below (ns), which were fitted to measured ones (us, rows x K at tokens, 1.2 GB of
// weights in turn, so that they come from HBM; estimates in brackets):
//   rows of 4: 1024 x 14336 at 1 token 8.9 (4.9; rows of 16 10.5); of 8: 2048 x 4096 5.0 (3.1; of 16 5.3); of 16: 4096 x 4096
//     5.9 (4.7), at 32 8.8 (8.8), 28672 x 4096 at 1 23.9 (24.4), 4096 x 14336 12.5 (12.6); of 20: 10240 x 4096 11.1 (9.7; of 16
//     12.1); of 24: 6144 x 4096 7.4 (6.2; of 16 8.6, of 32 8.0); of 40: 10000 x 2048 at 24 8.2 (7.5; of 64 9.3)
//   128 x 32 tiles: 28672 x 4096 at 16 27 to 29 (28; rows of 28 33); 128 x 64: 2500 x 4096 at 600 15 (17), 32003 x 4096 at 61 31 (32),
//     4096 x 14336 at 64 in 8 parts 19 (23)
//   256 x 128: 4096 x 4096 at 2048 36 (38), 4096 x 11008 at 333 in 5 parts 32 (39)
//   256 x 256: 9000 x 4096 at 1500 56 (57), 4096 x 14336 at 2048 162 (166), in 2 parts 117 (123), 28672 x 4096 at 4096 411 (399)
// Over 56 drawn sizes of 17 to 4096 tokens the plan took 1.016 times the best tile's and split's time on average, at most 1.11,
// over 80 of 1 to 32 tokens 1.010 times that of the best number of rows, at most 1.07.
#pragma once

#include <stddef.h>
#include <stdint.h>

namespace qift {
namespace route {

constexpr int64_t kW8RowsMaxM = 32;   // two token tiles of 16
constexpr int kCus = 256;

struct W8Plan {
  int rows;         // weight rows of a workgroup of the rows kernel (4, 8, .. 64); 0: the tiled product
  int bn, bm;       // its tiles
  int parts;        // parts of K
  double ns;        // estimate
};

inline int64_t w8_ceil(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline W8Plan w8_plan(int64_t N, int64_t M, int64_t K, bool split) {
  const int64_t steps = w8_ceil(K, 128);
  const double stream = (double)N * (double)K / 4800.0;   // the weights from memory
  W8Plan best = {0, 0, 0, 1, 1e300};
  // One workgroup to each CU, of as many rows as that takes, or a few of equal size; less than 16 rows use a part of the product's
  // tile only, which is no loss where the bytes count.  (Rows of 4 of a short K are slower: 512 x 256 2.8 against 2.6.)
  if (M <= kW8RowsMaxM) {
    for (int r = K <= 1024 ? 8 : 4; r <= (M <= 16 ? 32 : 64); r += 4) {
      const int64_t count = w8_ceil(N, r), each = w8_ceil(count, kCus);
      if ((r < 16 && each > 1) || (r % 16 && each > 4)) continue;
      const double in = (double)each * ((double)r + (each > 1 ? 1.3 : 1.0) * (double)M) * (double)K / (r > 32 ? 22.0 : 27.0);
      // the fullest CU's part of the stream; more than four to a CU queue up and even out
      const double part = each > 4 ? 1.0 : (double)(each * kCus) / (double)count;
      const double out = (double)N * (double)K / 5300.0 * part;
      const double ns = 1250.0 + 250.0 * (double)(each < 4 ? each : 4) + (in > out ? in : out);
      if (ns < best.ns) best = {r, 0, 0, 1, ns};
    }
  }
  // Times of a step of a CU with one workgroup, where at most half of the CUs have one (`few`) and where most do, and with two
  // side by side (0: they do not fit); and what a workgroup takes beside its steps.
  const struct {
    int bn, bm;
    double few, one, two, fixed;
  } tiles[] = {{128, 32, 400, 400, 750, 3500}, {128, 64, 420, 420, 880, 4000}, {256, 128, 680, 950, 0, 8000}, {256, 256, 1400, 1500, 0, 9000}};
  for (const auto& t : tiles) {
    if (t.bm < 64 && M > t.bm) continue;
    const int64_t count = w8_ceil(N, t.bn) * w8_ceil(M, t.bm);
    for (int p = 1; p <= (split ? 16 : 1); ++p) {
      if (p > 1 && (p > steps / 4 || count * p > 2 * kCus || M > 65535)) break;
      const int64_t each = w8_ceil(count * p, kCus);   // workgroups of the fullest CU
      const double one = count * p <= kCus / 2 ? t.few : t.one;
      const double turn = (double)w8_ceil(steps, p) * (t.two > 0 ? (double)(each / 2) * t.two + (double)(each & 1) * one : (double)each * one);
      const double rounds = t.two > 0 ? 1.0 : (double)each;
      // (of the stream too the CUs with more workgroups than the others have a larger part)
      const double out = each > 1 ? stream * (0.5 + 0.5 * (double)(each * kCus) / (double)(count * p)) : stream;
      double ns = (turn > out ? turn : out) + rounds * t.fixed;
      if (p > 1) ns += 3000.0 + 8.0 * p * (double)M * (double)N / 5000.0;   // the sums out and in, and their launch
      if (ns < best.ns) best = {0, t.bn, t.bm, p, ns};
    }
  }
  return best;
}
// Whether the rows kernel takes eight waves with units of 128 k rather than four with units of 256, for up to 16 tokens and 16
// rows: four (4096 x 14336 at one token 12.5 us; eight, with units of 256 too, 13.3) except where many workgroups queue for a CU
// (28672 x 4096 23.9 with eight against 25.5).
inline bool w8_eight_waves(const W8Plan& p, int64_t N, int64_t K) {
  return w8_ceil(N, p.rows) > 2 * kCus && K > 1024 && K <= 8192;
}
// Bytes of the parts' sums.
inline size_t w8_workspace(const W8Plan& p, int64_t N, int64_t M) {
  return p.parts == 1 ? 0 : (size_t)p.parts * (size_t)M * (size_t)(w8_ceil(N, 4) * 4) * sizeof(int32_t);
}

}  // namespace route
}  // namespace qift
