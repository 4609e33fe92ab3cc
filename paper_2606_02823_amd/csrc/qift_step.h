// Arithmetic of a serving step's plan, for the kernels and for host code (plain C++: compiled without a GPU too).
#pragma once

#include <math.h>

#include "qift_pages.h"

namespace qift {
namespace step {

constexpr int kSeqs = 256;   // sequences of a workgroup, one to a thread

// What one sequence asks for, from device data that may hold anything.  room = table_pages * page, below 2^31.
struct Ask {
  int32_t len, n;        // cached tokens, brought into [0, room]; new tokens, at least 0
  int32_t held, need;    // pages that hold the cached tokens; pages to take, 0 for a sequence that cannot be served
  bool fits, bad;        // its tokens fit its row of the table; one of its numbers is out of range
};
QIFT_HD int32_t pages_of(int32_t tokens, pages::Div page) {   // 0 <= tokens < 2^31
  const uint32_t whole = pages::quotient((uint32_t)tokens, page);
  return (int32_t)(whole + (whole * page.d != (uint32_t)tokens));
}
QIFT_HD Ask ask(int32_t len, int32_t n, int64_t room, pages::Div page) {
  Ask a;
  a.bad = len < 0 || (int64_t)len > room || n < 0;
  const bool len_ok = len >= 0 && (int64_t)len <= room;
  a.len = len < 0 ? 0 : (int64_t)len > room ? (int32_t)room : len;
  a.n = n < 0 ? 0 : n;
  a.fits = len_ok && (int64_t)a.len + a.n <= room;
  if (!a.fits && a.n > 0) a.bad = true;
  a.held = pages_of(a.len, page);
  a.need = a.fits ? pages_of(a.len + a.n, page) - a.held : 0;
  return a;
}
// Whether a sequence has its tokens in this step: start and base are the sums of the new tokens and of the pages that the
// sequences before it ask for.  Both only grow, so of the sequences that need pages those served are the first ones.
QIFT_HD bool served(const Ask& a, int64_t start, int64_t base, int64_t rows, int64_t depth) {
  return a.n > 0 && a.fits && start + a.n <= rows && (a.need == 0 || base + a.need <= depth);
}
// The pages taken up to this sequence's last, where it takes any (one that needs none is served however many those before it
// asked for in vain); a step takes the most of these.
QIFT_HD int64_t taken(const Ask& a, int64_t start, int64_t base, int64_t rows, int64_t depth) {
  return a.need > 0 && served(a, start, base, rows, depth) ? base + a.need : 0;
}
// Slot of the token at position pos whose page is `entry`; -1 where that is none or the slot has no 31 bits.
QIFT_HD int32_t slot_of(int32_t entry, uint32_t at, uint32_t page) {
  const int64_t s = (int64_t)entry * page + at;
  return entry < 0 || s > 0x7FFFFFFF ? -1 : (int32_t)s;
}
// The last of `count` + 1 ascending sums s (s[0] <= at < s[count]) that is at most `at`; a sequence of none is passed over.
QIFT_HD int32_t find(const int32_t* s, int32_t count, int32_t at) {
  int32_t lo = 0, hi = count;
  while (hi - lo > 1) {
    const int32_t mid = (lo + hi) >> 1;
    if (s[mid] <= at) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Head h of a row's Hq query and Hkv key heads, as a wave takes them four at a time; one past the last is the last again
// (read, not written), so that it is always a head that is there.
struct Head {
  int32_t own;       // among the queries' or the keys'
  bool have, key;
};
QIFT_HD Head head_of(int32_t h, int32_t Hq, int32_t Hkv) {
  const int32_t all = Hq + Hkv, in = h < all ? h : all - 1;
  const bool key = in >= Hq;
  return {key ? in - Hq : in, h < all, key};
}

// Rows of `bytes` each at a stride in memory (a view of stacked rows, or one row: an array).
struct View {
  uint64_t at;
  int64_t stride, bytes, rows;
};
// Whether two views share a byte.  Rows of one view do not overlap each other (the stride is at least a row).
inline bool overlap(const View& a, const View& b) {
  if (a.rows < 1 || b.rows < 1 || a.bytes < 1 || b.bytes < 1) return false;
  const int64_t d = (int64_t)(b.at - a.at);   // of b's first row from a's
  if (d >= (a.rows - 1) * a.stride + a.bytes || -d >= (b.rows - 1) * b.stride + b.bytes) return false;
  // a's row i begins at x = i a.stride - d from b's first: it meets the last of b's rows that begins before it ends, or none.
  // With one stride rows i and i + 1 lie alike, so that the first two tell.
  for (int64_t i = d < a.bytes ? 0 : (d - a.bytes) / a.stride + 1, n = 0; i < a.rows; ++i, ++n) {
    const int64_t x = i * a.stride - d;
    if (x >= (b.rows - 1) * b.stride + b.bytes || (n == 2 && a.stride == b.stride)) break;
    const int64_t below = (x + a.bytes - 1) / b.stride, j = below < b.rows ? below : b.rows - 1;
    if (x < j * b.stride + b.bytes) return true;
  }
  return false;
}

// Sine and cosine of position * freq, within 2^-22 for angles below kMaxAngle; NaN from there on and for a frequency that is no
// number.  The product is x + low exactly (55 bits at most), the remainder of x's division by pi / 2 is taken with pi / 2 in
// two parts (off by less than 2^-51), and the Taylor sums of the remainder, |r| <= pi / 4 + 2^-12, are cut where the next term is
// below 2^-29.
constexpr double kMaxAngle = 0x1p40;
QIFT_HD void turn(int32_t position, float freq, float& sine, float& cosine) {
  const double product = (double)position * (double)freq;
  const bool in = fabs(product) < kMaxAngle;
  const double x = in ? product : 0.0, low = in ? fma((double)position, (double)freq, -product) : 0.0;
  const double n = rint(x * 0x1.45f306dc9c883p-1);                       // 2 / pi
  const double r = fma(-n, 0x1.1a62633145c07p-54, fma(-n, 0x1.921fb54442d18p0, x)) + low;
  const int quadrant = (int)(n - 4.0 * floor(n * 0.25));
  const float f = (float)r, z = f * f;
  float s = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
  s = fmaf(s, z, 1.f / 120.f);
  s = fmaf(s, z, -1.f / 6.f);
  s = fmaf(s * z, f, f);
  float c = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
  c = fmaf(c, z, -1.f / 720.f);
  c = fmaf(c, z, 1.f / 24.f);
  c = fmaf(c, z, -0.5f);
  c = fmaf(c, z, 1.f);
  const float a = quadrant & 1 ? c : s, b = quadrant & 1 ? s : c;
  sine = !in ? NAN : quadrant & 2 ? -a : a;
  cosine = !in ? NAN : (quadrant + 1) & 2 ? -b : b;
}

}  // namespace step
}  // namespace qift
