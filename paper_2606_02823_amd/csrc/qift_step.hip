// A serving step's plan: where each new token of each sequence goes (slots, positions, first rows), the pages taken for
// them, and the pages of finished sequences given back.
//
// Both kernels are one launch that reads its sums afresh: a workgroup has 256 sequences (one to a thread), adds up what the
// sequences before them ask for, and takes every split-th part of their rows and pages.  Nothing waits for another
// workgroup and nothing is counted by atomics, so the results do not depend on the order in which workgroups run; the
// price is that the lengths are read by all (2000 sequences: 16 KB from the L2 of each XCD).
#include "qift_fwht.h"   // flag_error
#include "qift_internal.h"
#include "qift_step.h"

namespace qift {
namespace {

using step::kSeqs;
constexpr int kAhead = 8;   // sequences of a thread whose numbers are read at once

struct Sums {
  int64_t a, b;
};

// Sums of v over the threads before this one and, in all, over the workgroup's 256; and of `other` over the workgroup.  One
// barrier and one more before the next use of `part`.
struct Scan {
  Sums before, all, other;
};
__device__ __forceinline__ Scan scan(Sums v, Sums other, Sums (*part)[2]) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  Sums s = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t a = __shfl_up((long long)s.a, d), b = __shfl_up((long long)s.b, d);
    other.a += __shfl_xor((long long)other.a, d);
    other.b += __shfl_xor((long long)other.b, d);
    if (lane >= d) {
      s.a += a;
      s.b += b;
    }
  }
  if (lane == 63) {
    part[w][0] = s;
    part[w][1] = other;
  }
  __syncthreads();
  Scan r = {{s.a - v.a, s.b - v.b}, {0, 0}, {0, 0}};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (i < w) {
      r.before.a += part[i][0].a;
      r.before.b += part[i][0].b;
    }
    r.all.a += part[i][0].a;
    r.all.b += part[i][0].b;
    r.other.a += part[i][1].a;
    r.other.b += part[i][1].b;
  }
  return r;
}

__device__ __forceinline__ int64_t depth_of(const int32_t* count, int64_t capacity, bool& bad) {
  const int32_t c = *count;
  bad = c < 0 || c > capacity;
  return c < 0 ? 0 : c > capacity ? capacity : c;
}

// (a sequence past the last before this workgroup's reads that one again, so that no load waits behind a branch)
__device__ __forceinline__ int before_at(int b, int first) { return b < first ? b : first - 1; }

// Bound by latency: the lengths, the scan, the search, the table's or the stack's entry, the slot (61 sequences 4.8 us, an
// empty launch 2.3).
__global__ __launch_bounds__(kSeqs) void k_plan(PlanCall c, pages::Div page, int split, uint32_t* err) {
  __shared__ Sums part[4][2];
  __shared__ int32_t s_start[kSeqs + 1], s_base[kSeqs + 1];   // from the workgroup's first sequence on
  __shared__ int32_t s_len[kSeqs], s_held[kSeqs], s_served[kSeqs];
  const int t = threadIdx.x;
  const int chunk = blockIdx.x / split, sub = blockIdx.x - chunk * split;
  const int first = chunk * kSeqs;   // (at most 65535 sequences)
  const int64_t room = (int64_t)c.table_pages * page.d;
  const bool last = first + kSeqs >= c.B;
  bool bad;
  const int64_t b = first + t;
  const int32_t my_len = b < c.B ? c.lens[b] : 0, my_n = b < c.B ? c.counts[b] : 0;
  const int64_t depth = depth_of(c.free_count, c.capacity, bad);
  // the sequences before this workgroup's
  Sums before = {0, 0};
  for (int b0 = 0; b0 < first; b0 += kAhead * kSeqs) {
    int32_t len[kAhead], n[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int at = before_at(b0 + i * kSeqs + t, first);
      len[i] = c.lens[at];
      n[i] = c.counts[at];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const step::Ask a = step::ask(len[i], n[i], room, page);
      const bool in = b0 + i * kSeqs + t < first;
      before.a += in ? a.n : 0;
      before.b += in ? a.need : 0;
    }
  }
  // its own
  const step::Ask a = step::ask(my_len, my_n, room, page);
  const Scan sums = scan({a.n, a.need}, before, part);
  const Sums own = sums.before, all = sums.all;
  before = sums.other;
  const int64_t start = before.a + own.a, base = before.b + own.b;
  const bool served = step::served(a, start, base, c.rows, depth);
  // (sums past every row and every page are cut: nothing behind them is served)
  auto cut = [](int64_t v) { return (int32_t)(v < 0x7FFFFFFF ? v : 0x7FFFFFFF); };
  auto row = [&](int64_t v) { return (int32_t)(v < c.rows ? v : c.rows); };
  s_start[t] = row(start);
  s_base[t] = cut(own.b);
  s_len[t] = a.len;
  s_held[t] = a.held;
  s_served[t] = served;
  if (t == 0) {
    s_start[kSeqs] = row(before.a + all.a);
    s_base[kSeqs] = cut(all.b);
  }
  if (sub == 0 && b < c.B) {
    c.starts[b] = row(start);
    c.lens_out[b] = served ? a.len + a.n : a.len;
    bad |= a.bad || (a.n > 0 && !served);
  }
  __syncthreads();
  if (last && sub == 0) {
    // the pages taken: all that are asked for, or, where something was left out, those up to the last sequence that takes some
    int64_t taken = before.b + all.b;
    if (taken > depth || before.a + all.a > c.rows) {
      taken = 0;
      Sums run = {0, 0};
      for (int64_t at = 0; at < c.B; at += kSeqs) {
        step::Ask o = {0, 0, 0, 0, true, false};
        if (at + t < c.B) o = step::ask(c.lens[at + t], c.counts[at + t], room, page);
        const Scan round = scan({o.n, o.need}, {0, 0}, part);
        const Sums mine = round.before, sum = round.all;
        int64_t most = step::taken(o, run.a + mine.a, run.b + mine.b, c.rows, depth);
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
          const int64_t other = __shfl_xor((long long)most, d);
          most = other > most ? other : most;
        }
        __syncthreads();
        if ((t & 63) == 0) part[t >> 6][0].a = most;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) taken = part[i][0].a > taken ? part[i][0].a : taken;
        __syncthreads();
        run.a += sum.a;
        run.b += sum.b;
      }
    }
    if (t == 0) {
      c.starts[c.B] = row(before.a + all.a);
      *c.free_out = (int32_t)(depth - taken);
    }
  }
  // rows: those of the workgroup's sequences; behind the last sequence's there are none
  const int64_t end = last ? c.rows : s_start[kSeqs];
  for (int64_t r = s_start[0] + (int64_t)sub * kSeqs + t; r < end; r += (int64_t)split * kSeqs) {
    int32_t slot = -1, pos = -1;
    if (r < s_start[kSeqs]) {
      const int s = step::find(s_start, kSeqs, (int32_t)r);
      if (s_served[s]) {
        pos = s_len[s] + (int32_t)(r - s_start[s]);
        const uint32_t p = pages::quotient((uint32_t)pos, page);
        const int32_t entry = (int32_t)p < s_held[s] ? c.table[(int64_t)(first + s) * c.table_pages + p]
                                                     : c.free_pages[depth - 1 - (before.b + s_base[s] + ((int32_t)p - s_held[s]))];
        slot = step::slot_of(entry, (uint32_t)pos - p * page.d, page.d);
        bad |= slot < 0;
      }
    }
    c.slots[r] = slot;
    c.positions[r] = pos;
  }
  // pages taken (those of a sequence that is served lie within the stack, whatever the others ask for)
  const int64_t there = depth - before.b, asked = s_base[kSeqs] < there ? s_base[kSeqs] : there;
  for (int64_t f = (int64_t)sub * kSeqs + t; f < asked; f += (int64_t)split * kSeqs) {
    const int s = step::find(s_base, kSeqs, (int32_t)f);
    if (!s_served[s]) continue;
    const int32_t entry = c.free_pages[depth - 1 - (before.b + f)];
    c.table[(int64_t)(first + s) * c.table_pages + s_held[s] + (f - s_base[s])] = entry;
    bad |= entry < 0;
  }
  if (bad) dev::flag_error(err, kDevErrIndex);
}

__global__ __launch_bounds__(kSeqs) void k_release(ReleaseCall c, pages::Div page, int split, uint32_t* err) {
  __shared__ Sums part[4][2];
  __shared__ int32_t s_base[kSeqs + 1];
  const int t = threadIdx.x;
  const int chunk = blockIdx.x / split, sub = blockIdx.x - chunk * split;
  const int first = chunk * kSeqs;   // (at most 65535 sequences)
  const int64_t room = (int64_t)c.table_pages * page.d;
  const bool last = first + kSeqs >= c.B;
  bool bad;
  const int64_t b = first + t;
  const int32_t my_len = b < c.B ? c.lens[b] : 0;
  const bool done = b < c.B && c.done[b] != 0;
  const int64_t depth = depth_of(c.free_count, c.capacity, bad);
  Sums before = {0, 0};
  for (int b0 = 0; b0 < first; b0 += kAhead * kSeqs) {
    int32_t len[kAhead], over[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int at = before_at(b0 + i * kSeqs + t, first);
      len[i] = c.lens[at];
      over[i] = c.done[at];
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) before.a += over[i] && b0 + i * kSeqs + t < first ? step::ask(len[i], 0, room, page).held : 0;
  }
  const step::Ask a = step::ask(my_len, 0, room, page);
  const Scan sums = scan({done ? a.held : 0, 0}, before, part);
  const Sums own = sums.before, all = sums.all;
  before = sums.other;
  auto cut = [](int64_t v) { return (int32_t)(v < 0x7FFFFFFF ? v : 0x7FFFFFFF); };
  s_base[t] = cut(own.a);
  if (t == 0) s_base[kSeqs] = cut(all.a);
  if (sub == 0 && b < c.B) {
    c.lens_out[b] = done ? 0 : a.len;
    bad |= a.bad;
  }
  __syncthreads();
  if (last && sub == 0 && t == 0) {
    const int64_t n = depth + before.a + all.a;
    *c.free_out = (int32_t)(n < c.capacity ? n : c.capacity);
  }
  for (int64_t f = (int64_t)sub * kSeqs + t; f < s_base[kSeqs]; f += (int64_t)split * kSeqs) {
    const int s = step::find(s_base, kSeqs, (int32_t)f);
    const int64_t at = depth + before.a + f;
    const int32_t entry = c.table[(int64_t)(first + s) * c.table_pages + (f - s_base[s])];
    bad |= entry < 0 || at >= c.capacity;
    if (at < c.capacity) c.free_pages[at] = entry;
  }
  if (bad) dev::flag_error(err, kDevErrIndex);
}

// Parts of a workgroup's rows or pages, one to a thread, up to 8 workgroups to a CU: a row is a search and two reads, one behind
// the other (2000 sequences with 116000 rows 7.8 us; 11.3
// with four to a thread and the sequences before them read one by one)
int splits(int64_t items, int64_t chunks) {
  int64_t n = (items + chunks * kSeqs - 1) / (chunks * kSeqs);
  if (n > 2048 / chunks) n = 2048 / chunks;
  return n < 1 ? 1 : (int)n;
}

}  // namespace

hipError_t launch_plan_step(const PlanCall& a, hipStream_t s) {
  const int64_t chunks = a.B < 1 ? 1 : (a.B + kSeqs - 1) / kSeqs;
  const int split = splits(a.rows, chunks);
  hipLaunchKernelGGL(k_plan, dim3((unsigned)(chunks * split)), dim3(kSeqs), 0, s, a, pages::make_div((uint32_t)a.page), split,
                     device_error_word());
  return hipGetLastError();
}

hipError_t launch_release(const ReleaseCall& a, hipStream_t s) {
  const int64_t chunks = a.B < 1 ? 1 : (a.B + kSeqs - 1) / kSeqs;
  // how many pages are given back is device data; the tables' size is its bound
  const int split = splits((a.B < kSeqs * chunks ? a.B : kSeqs * chunks) * a.table_pages / 8, chunks);
  hipLaunchKernelGGL(k_release, dim3((unsigned)(chunks * split)), dim3(kSeqs), 0, s, a, pages::make_div((uint32_t)a.page), split,
                     device_error_word());
  return hipGetLastError();
}

}  // namespace qift
