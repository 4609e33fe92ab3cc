// C ABI of a serving step around the paged cache (include/qift_step.h): host-side validation, then dispatch.  Every check
// runs before the first HIP call.
#include <math.h>

#include "../../include/qift_step.h"
#include "qift_internal.h"
#include "qift_step.h"

namespace {

constexpr int64_t k31 = int64_t(1) << 31;

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

bool tables_ok(int64_t B, int32_t table_pages, int32_t page, int64_t capacity) {
  return B >= 0 && B <= 65535 && table_pages >= 1 && page >= 16 && page % 16 == 0 && (int64_t)table_pages * page < k31 &&
         capacity >= 0 && capacity < k31;
}

struct Words {   // an array of 32-bit numbers
  const void* p;
  int64_t n;
};

// Whether one of the first `outputs` arrays overlaps any other.  Every workgroup reads the inputs afresh and none waits for
// another, so such a call's results would depend on their order.
template <int N>
bool overlap(const Words (&a)[N], int outputs) {
  for (int i = 0; i < outputs; ++i)
    for (int j = i + 1; j < N; ++j) {
      const uintptr_t x = reinterpret_cast<uintptr_t>(a[i].p), y = reinterpret_cast<uintptr_t>(a[j].p);
      if (a[i].n > 0 && a[j].n > 0 && x < y + 4 * (uintptr_t)a[j].n && y < x + 4 * (uintptr_t)a[i].n) return true;
    }
  return false;
}

}  // namespace

extern "C" {

int qift_kv4_plan_step(const int32_t* lens, const int32_t* counts, int64_t B, int32_t* table, int32_t table_pages,
                       int32_t page, const int32_t* free_pages, const int32_t* free_count, int64_t capacity, int64_t rows,
                       int32_t* starts, int32_t* lens_out, int32_t* slots, int32_t* positions, int32_t* free_out,
                       qift_stream_t stream) {
  if (!tables_ok(B, table_pages, page, capacity) || rows < 0 || rows >= k31) return QIFT_ERR_SHAPE;
  if (!free_count || !starts || !free_out || (B > 0 && (!lens || !counts || !table || !lens_out)) ||
      (capacity > 0 && !free_pages) || (rows > 0 && (!slots || !positions)))
    return QIFT_ERR_NULL;
  if ((B > 0 && lens == lens_out) || free_count == free_out) return QIFT_ERR_SHAPE;
  const void* p[] = {lens, counts, table, free_pages, free_count, starts, lens_out, slots, positions, free_out};
  for (const void* x : p)
    if (!aligned(x, 4)) return QIFT_ERR_ALIGN;
  const Words arrays[] = {{table, B * table_pages}, {starts, B + 1}, {lens_out, B}, {slots, rows}, {positions, rows}, {free_out, 1},
                          {lens, B}, {counts, B}, {free_pages, capacity}, {free_count, 1}};
  if (overlap(arrays, 6)) return QIFT_ERR_SHAPE;
  return qift::report_hip(qift::launch_plan_step({lens, counts, table, free_pages, free_count, starts, lens_out, slots, positions,
                                                  free_out, B, rows, capacity, table_pages, page},
                                                 (hipStream_t)stream));
}

int qift_kv4_release(const int32_t* lens, const int32_t* done, int64_t B, const int32_t* table, int32_t table_pages,
                     int32_t page, int32_t* free_pages, const int32_t* free_count, int64_t capacity, int32_t* lens_out,
                     int32_t* free_out, qift_stream_t stream) {
  if (!tables_ok(B, table_pages, page, capacity)) return QIFT_ERR_SHAPE;
  if (!free_count || !free_out || (B > 0 && (!lens || !done || !table || !lens_out)) || (capacity > 0 && !free_pages))
    return QIFT_ERR_NULL;
  if ((B > 0 && lens == lens_out) || free_count == free_out) return QIFT_ERR_SHAPE;
  const void* p[] = {lens, done, table, free_pages, free_count, lens_out, free_out};
  for (const void* x : p)
    if (!aligned(x, 4)) return QIFT_ERR_ALIGN;
  const Words arrays[] = {{free_pages, capacity}, {lens_out, B}, {free_out, 1}, {lens, B}, {done, B}, {table, B * table_pages},
                          {free_count, 1}};
  if (overlap(arrays, 3)) return QIFT_ERR_SHAPE;
  return qift::report_hip(qift::launch_release(
      {lens, done, table, free_pages, free_count, lens_out, free_out, B, capacity, table_pages, page}, (hipStream_t)stream));
}

int qift_head_norm_rope(const qift_head_rope* rope, const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                        int32_t dtype, const int32_t* positions, int64_t rows, int32_t Hq, int32_t Hkv, void* q_out,
                        int64_t q_out_stride, void* k_out, int64_t k_out_stride, qift_stream_t stream) {
  if (!rope) return QIFT_ERR_NULL;
  if (dtype != QIFT_F16 && dtype != QIFT_BF16) return QIFT_ERR_FORMAT;
  if (rope->head_dim != 128 || rope->rot < 0 || rope->rot > 128 || rope->rot % 8) return QIFT_ERR_SHAPE;
  if ((rope->pairs != 0 && rope->pairs != 1) || !(rope->eps >= 0x1p-80f) || !isfinite(rope->eps)) return QIFT_ERR_SPEC;
  if (rows < 0 || Hq < 0 || Hkv < 0 || Hq > 65535 || Hkv > 65535 || Hq + Hkv < 1) return QIFT_ERR_SHAPE;
  const int64_t groups = (Hq + Hkv + 3) / 4;
  if (rows >= k31 || rows * groups + 3 >= (int64_t(1) << 26)) return QIFT_ERR_SHAPE;   // four waves to a workgroup: fewer than 2^32 threads
  const int64_t strides[] = {q_stride, q_out_stride, k_stride, k_out_stride};
  const void* rowsp[] = {q, q_out, k, k_out};
  for (int i = 0; i < 4; ++i) {
    const int64_t heads = i < 2 ? Hq : Hkv;
    if (heads > 0 && (strides[i] < heads * 128 || strides[i] >= k31)) return QIFT_ERR_SHAPE;
  }
  if (rows == 0) return QIFT_OK;
  if (!positions || (rope->rot > 0 && !rope->freq)) return QIFT_ERR_NULL;
  for (int i = 0; i < 4; ++i)
    if ((i < 2 ? Hq : Hkv) > 0 && !rowsp[i]) return QIFT_ERR_NULL;
  for (int i = 0; i < 4; ++i)
    if ((i < 2 ? Hq : Hkv) > 0 && (!aligned(rowsp[i], 16) || strides[i] % 8)) return QIFT_ERR_ALIGN;
  if (!aligned(positions, 4) || !aligned(rope->freq, 16) || !aligned(rope->q_weight, 16) || !aligned(rope->k_weight, 16))
    return QIFT_ERR_ALIGN;
  // each value is read before it is written where an output is its input; any other overlap of what is written races
  auto view = [](const void* p, int64_t stride, int64_t bytes, int64_t n) {
    return qift::step::View{reinterpret_cast<uintptr_t>(p), stride, bytes, n};
  };
  qift::step::View v[8];
  for (int i = 0; i < 4; ++i) v[i] = view(rowsp[i], 2 * strides[i], (i < 2 ? Hq : Hkv) * 256, rows);
  v[4] = view(positions, 4 * rows, 4 * rows, 1);
  v[5] = view(rope->freq, 256, rope->rot * 2, 1);
  v[6] = view(rope->q_weight, 256, rope->q_weight ? 256 : 0, 1);
  v[7] = view(rope->k_weight, 256, rope->k_weight ? 256 : 0, 1);
  for (int out = 1; out < 4; out += 2)
    for (int i = 0; i < 8; ++i) {
      const bool in_place = i == out - 1 && v[i].at == v[out].at && (rows == 1 || v[i].stride == v[out].stride);
      if (i != out && !in_place && qift::step::overlap(v[out], v[i])) return QIFT_ERR_SHAPE;
    }
  qift::RopeCall c;
  c.x[0] = static_cast<const uint16_t*>(q);
  c.x[1] = static_cast<const uint16_t*>(k);
  c.y[0] = static_cast<uint16_t*>(q_out);
  c.y[1] = static_cast<uint16_t*>(k_out);
  c.weight[0] = static_cast<const uint16_t*>(rope->q_weight);
  c.weight[1] = static_cast<const uint16_t*>(rope->k_weight);
  c.x_stride[0] = q_stride;
  c.x_stride[1] = k_stride;
  c.y_stride[0] = q_out_stride;
  c.y_stride[1] = k_out_stride;
  c.heads[0] = Hq;
  c.heads[1] = Hkv;
  c.positions = positions;
  c.freq = rope->freq;
  c.rows = rows;
  c.eps = rope->eps;
  c.rot = rope->rot;
  c.pairs = rope->pairs;
  c.dtype = dtype;
  return qift::report_hip(qift::launch_head_norm_rope(c, (hipStream_t)stream));
}

}  // extern "C"
