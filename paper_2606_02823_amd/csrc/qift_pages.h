// Index arithmetic of the paged KV4 cache and of the attention over it, for the kernels and for host code
// (plain C++: compiled without a GPU too).
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define QIFT_HD __host__ __device__ __forceinline__
#else
#define QIFT_HD inline
#endif

namespace qift {
namespace pages {

// Division of x < 2^31 by a fixed d, 1 <= d < 2^31: with 2^s >= d the multiplier m = ceil(2^(31 + s) / d) has at most
// 32 bits and floor(x m / 2^(31 + s)) = floor(x / d) for every x below 2^31 (m d - 2^(31 + s) < d <= 2^s).
struct Div {
  uint32_t d, m, s;   // s: the shift left after the high word of the product
};
inline Div make_div(uint32_t d) {
  uint32_t s = 1;
  while (s < 31 && (uint32_t(1) << s) < d) ++s;
  if (d == 1) return {1, 0, 0};
  return {d, (uint32_t)(((uint64_t(1) << (31 + s)) + d - 1) / d), s - 1};
}
QIFT_HD uint32_t quotient(uint32_t x, Div v) {
  return v.d == 1 ? x : (uint32_t)(((uint64_t)x * v.m) >> 32) >> v.s;
}

// Row of a slot: rows are [pages][Hkv][page].  The caller has checked 0 <= slot < pages * page; rows stay below 2^31.
QIFT_HD uint32_t slot_row(uint32_t slot, Div page, uint32_t Hkv, uint32_t head) {
  const uint32_t p = quotient(slot, page);
  return (p * Hkv + head) * page.d + (slot - p * page.d);
}

// Row of token t of a sequence whose table entry for that token is `entry` (checked to name a page); tiles divides by the
// 16-token tiles of a page.
QIFT_HD uint32_t table_index(uint32_t t, Div tiles) { return quotient(t >> 4, tiles); }
QIFT_HD uint32_t token_row(uint32_t t, uint32_t entry, uint32_t Hkv, uint32_t head, Div tiles) {
  const uint32_t page = tiles.d * 16;
  return (entry * Hkv + head) * page + (t - table_index(t, tiles) * page);
}

// Nodes and tokens of one sequence, taken from device data that may hold anything: every count is brought into the
// range the launch was made for, and bad says that one was not.  The nodes stand where the starts put them: those past
// max_nodes or past the last row are left out with their tokens, which lie behind the others', and the others keep their
// places.  A sequence whose first row is none has no rows.
struct Seq {
  int32_t row0, n, len, ctx;   // first row of q, rows, cached tokens, tokens before the first node
  bool bad;
};
QIFT_HD Seq sequence(int32_t s0, int32_t s1, int32_t len, int32_t rows, int32_t max_nodes, int64_t most) {
  Seq q;
  const int64_t nodes = s1 < s0 ? 0 : (int64_t)s1 - s0;
  const bool none = s0 < 0 || s0 > rows;
  q.bad = none || s1 < s0 || s1 > rows || nodes > max_nodes || len < 0 || (int64_t)len > most;
  q.row0 = none ? 0 : s0;
  q.n = none ? 0 : rows - s0;
  if (q.n > max_nodes) q.n = max_nodes;
  if (q.n > nodes) q.n = (int32_t)nodes;
  q.len = len < 0 ? 0 : (int64_t)len > most ? (int32_t)most : len;
  q.ctx = q.len > nodes ? q.len - (int32_t)nodes : 0;
  if (nodes > q.n && q.len > q.ctx + q.n) q.len = q.ctx + q.n;
  return q;
}

// Tokens that the block of query rows [block_rows block, block_rows (block + 1)) reaches: without a mask a row sees
// nothing past its own node.
QIFT_HD int32_t last_token(const Seq& q, bool masked, Div group, int32_t block_rows, int32_t block) {
  if (masked) return q.len;
  int32_t node = (int32_t)quotient((uint32_t)((block + 1) * block_rows - 1), group);
  if (node > q.n - 1) node = q.n - 1;
  const int32_t end = q.ctx + node + 1;
  return end < q.len ? end : q.len;
}

// Which of the 64 tokens t0 .. t0 + 63 row `node` sees, without the end of the sequence: bit i is token t0 + i.
QIFT_HD uint64_t low_bits(int32_t n) { return n <= 0 ? 0 : n >= 64 ? ~uint64_t(0) : (uint64_t(1) << n) - 1; }
QIFT_HD uint64_t chain_bits(int32_t t0, int32_t ctx, int32_t node) { return low_bits(ctx + node + 1 - t0); }
// From the words of the row's mask: d0 = t0 - ctx is the node at token t0 (negative: tokens before the first node, all
// seen); w0 is mask word max(d0, 0) / 64 and w1 the next, 0 past the mask's words.
QIFT_HD uint64_t tree_bits(int32_t d0, uint64_t w0, uint64_t w1) {
  if (d0 <= -64) return ~uint64_t(0);
  if (d0 < 0) return low_bits(-d0) | (w0 << -d0);
  const int32_t sh = d0 & 63;
  return sh ? (w0 >> sh) | (w1 << (64 - sh)) : w0;
}

// How the attention cuts its work.  A workgroup takes a block of 16 rt query rows (a row is a node and a head of the KV
// head's group) of one KV head and sequence at a time (a unit), over tokens in rounds of 256: 64 for each of its four
// waves.  Few units: the rounds of all units, in order, are dealt out evenly to `shares` workgroups a block of rows, whatever
// the sequences' lengths are; a unit that more than one share covers is joined from partial records.  Beginning and ending a
// unit takes a workgroup longer than a round, so a unit is dealt out as its rounds and kBegin more before them (32
// ragged sequences of 8 heads, where a share may have eight short units: 52 us with 0, 46 with 1, 45 with 2).
// Many units: one workgroup takes a unit whole, which needs no second launch.  With two workgroups to a CU's place or more
// (16 trees of 64 nodes over 8192 tokens, 1024 blocks of units: 268 us, dealt out 274; 4 ragged chunks of 256: 62, 71), and
// with half of the places filled where sequences have few rounds (256 blocks, 673 tokens: 17 us, dealt out 24; 448, 1021
// tokens: 29, 40; 480, 332 tokens: 25, 29).  Below that dealing out wins on ragged sequences (256 units of 32 sequences of
// up to 8192 tokens: 45 us, whole 63; 280 blocks, 2999 tokens: 37, 39) and loses little on even ones (512 units of 2048
// tokens: 37.5, 35.2).  The host knows max_len alone, not how the lengths differ, and counts max_nodes for every sequence:
// from 1024 blocks on one long sequence among short ones, or a chunk's max_nodes beside single tokens, leaves most of the
// card idle behind a few workgroups (127 sequences of one token, 8 heads, one of 65536 tokens, the others up to 2000: 66 us, dealt out; 128 of
// them, whole: 420 us.  A chunk of 256 and 3 single tokens, all over 65536: 872 us).
constexpr int kStep = 64, kWaves = 4, kRound = kStep * kWaves;
constexpr int kMostShared = 512;   // sequences whose rounds are dealt out (every workgroup adds them up)
constexpr int kBegin = 2, kFewRounds = 4;
struct Plan {
  int32_t rt, blocks;   // row tiles of a workgroup, blocks of a KV head's rows
  int32_t shares;       // workgroups of a block of rows; 0: one to a unit
};
QIFT_HD int32_t rounds_of(int32_t len) { return len < 1 ? 1 : (int32_t)(((int64_t)len + kRound - 1) / kRound); }
inline int64_t dealt_below(int64_t max_len) { return max_len <= kFewRounds * kRound ? 256 : 1024; }   // units times blocks
inline Plan plan(int64_t B, int32_t Hkv, int32_t G, int32_t max_nodes, int64_t max_len) {
  Plan p;
  const int64_t rows = (int64_t)max_nodes * G;
  p.rt = rows <= 16 ? 1 : 2;
  p.blocks = (int32_t)((rows + 16 * p.rt - 1) / (16 * p.rt));
  const int64_t units = B * Hkv, rounds = (max_len + kRound - 1) / kRound;
  p.shares = 0;
  if (rounds > 1 && B <= kMostShared && units * p.blocks < dealt_below(max_len)) {
    int64_t n = 512 / p.blocks;                 // two workgroups to each of 256 CUs
    if (n > units * (rounds + kBegin)) n = units * (rounds + kBegin);
    p.shares = n < 1 ? 1 : (int32_t)n;
  }
  return p;
}
// What is dealt out: the slots of all units, kBegin and its rounds for each.  Share i of n has the slots [first_slot(i),
// first_slot(i + 1)) of W, at least one; of a unit whose slots it has from lo to hi - 1 (counted in the unit) it takes the
// rounds round_at(lo) .. round_at(hi) - 1, if any.
QIFT_HD int32_t slots_of(int32_t len) { return rounds_of(len) + kBegin; }
QIFT_HD int32_t used_shares(int64_t W, int32_t shares) { return W < shares ? (int32_t)W : shares; }
// The share and block of rows of workgroup g: group g is on XCD g mod 8, which has every eighth part, in order, of the shares'
// blocks.  A share past the last one: the workgroup has none.
struct Place {
  int32_t share, block;
};
QIFT_HD Place place(int32_t g, int32_t shares, int32_t blocks) {
  const int32_t all = shares * blocks, per = (all + 7) / 8, j = g / 8, n = g % 8 * per + j;
  if (j >= per || n >= all) return {shares, 0};
  return {n / blocks, n % blocks};
}
QIFT_HD int64_t first_slot(int64_t W, int32_t n, int32_t i) { return W * i / n; }
QIFT_HD int32_t round_at(int32_t slot) { return slot > kBegin ? slot - kBegin : 0; }
// Partial records: share i and unit u have number i + u (both grow along the rounds, so no two have the same), each
// 128 sums per row, then (after all sums) the rows' references and sums of exponentials, then each unit's first and last
// share.
inline int64_t records(const Plan& p, int64_t B, int32_t Hkv) { return p.shares == 0 ? 0 : p.shares + B * Hkv; }
inline int64_t workspace_words(const Plan& p, int64_t B, int32_t Hkv, int32_t G, int32_t max_nodes) {
  return p.shares == 0 ? 0 : records(p, B, Hkv) * ((int64_t)max_nodes * G) * 130 + 2 * B * Hkv;
}

// Words that are enough for every call with at most B sequences, max_nodes nodes and max_len tokens.  A call with fewer nodes
// may be dealt out where one with more is not, and has more shares of a block where it has fewer blocks, so each number of
// blocks is asked with the most nodes that it has and the most sequences that are dealt out then; a longer max_len only adds.
inline int64_t most_workspace_words(int64_t B, int32_t Hkv, int32_t G, int32_t max_nodes, int64_t max_len) {
  int64_t most = 0;
  for (int32_t nodes = max_nodes; nodes > 0;) {
    const Plan one = plan(1, Hkv, G, nodes, max_len);
    const int64_t per = (int64_t)Hkv * one.blocks;
    int64_t b = (dealt_below(max_len) - 1) / per;
    if (b > kMostShared) b = kMostShared;
    if (b > B) b = B;
    if (b > 0) {
      const int64_t w = workspace_words(plan(b, Hkv, G, nodes, max_len), b, Hkv, G, nodes);
      if (w > most) most = w;
    }
    nodes = one.rt == 1 ? 0 : one.blocks == 1 ? 16 / G : (one.blocks - 1) * 32 / G;
  }
  return most;
}

}  // namespace pages
}  // namespace qift
