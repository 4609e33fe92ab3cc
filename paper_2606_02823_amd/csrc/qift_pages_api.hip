// C ABI of the paged KV4 cache (include/qift_pages.h): host-side validation, then dispatch.  Every check runs before
// the first HIP call.
#include "../../include/qift_pages.h"
#include "qift_internal.h"
#include "qift_pages.h"

static_assert(QIFT_F16 == qift::kF16 && QIFT_BF16 == qift::kBF16 && QIFT_F32 == qift::kF32, "element types");
static_assert(QIFT_DEVERR_INDEX == qift::kDevErrIndex, "error bit");

namespace {

constexpr int64_t k31 = int64_t(1) << 31;
constexpr int64_t kGroups = int64_t(1) << 24;   // workgroups along x: 256 threads each, fewer than 2^32 threads

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

int check_shape(const qift_kv4_pages* c) {
  if (!c) return QIFT_ERR_NULL;
  if (c->head_dim != 128 || c->reserved != 0 || c->pages < 1 || c->page < 16 || c->page % 16 || c->Hkv < 1 || c->Hkv > 65535)
    return QIFT_ERR_SHAPE;
  if (c->pages >= k31 || c->pages * c->page >= k31 || c->pages * c->page * c->Hkv >= k31) return QIFT_ERR_SHAPE;
  return QIFT_OK;
}
int check_pointers(const qift_kv4_pages* c) {
  const void* p[] = {c->k_codes, c->k_scales, c->k_zeros, c->v_codes, c->v_scales, c->v_zeros};
  for (const void* x : p)
    if (!x) return QIFT_ERR_NULL;
  for (const void* x : p)
    if (!aligned(x, 16)) return QIFT_ERR_ALIGN;
  return QIFT_OK;
}
qift::Kv4Pool pool(const qift_kv4_pages* c) {
  return {c->pages, c->page, c->Hkv, c->k_codes, c->k_scales, c->k_zeros, c->v_codes, c->v_scales, c->v_zeros};
}

bool tree_shape_ok(int64_t B, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t max_nodes, int64_t max_len) {
  if (head_dim != 128 || B < 0 || B > 65535 || Hkv < 1 || Hkv > 65535 || Hq < Hkv || Hq % Hkv || Hq / Hkv > 64) return false;
  if (max_nodes < 1 || max_nodes > 256 || max_len < 1 || max_len >= (int64_t(1) << 28)) return false;
  const qift::pages::Plan p = qift::pages::plan(B < 1 ? 1 : B, Hkv, Hq / Hkv, max_nodes, max_len);
  return ((p.shares ? p.shares : B * Hkv) + 8) * p.blocks < kGroups;
}

}  // namespace

extern "C" {

int qift_kv4_append(const qift_kv4_pages* cache, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                    int32_t dtype, const int32_t* slots, int64_t n, void* k_values, void* v_values,
                    qift_stream_t stream) {
  int st = check_shape(cache);
  if (st != QIFT_OK) return st;
  if (dtype != QIFT_F16 && dtype != QIFT_BF16) return QIFT_ERR_FORMAT;
  const int64_t width = (int64_t)cache->Hkv * 128;
  if (n < 0 || n >= k31 || k_stride < width || v_stride < width || k_stride >= k31 || v_stride >= k31) return QIFT_ERR_SHAPE;
  if ((n + 15) / 16 * 2 * cache->Hkv >= kGroups) return QIFT_ERR_SHAPE;   // one to 16 tokens, a head and a side
  if (n == 0) return QIFT_OK;
  if (!k || !v || !slots || (!k_values) != (!v_values)) return QIFT_ERR_NULL;
  st = check_pointers(cache);
  if (st != QIFT_OK) return st;
  if (!aligned(k, 16) || !aligned(v, 16) || k_stride % 8 || v_stride % 8 || !aligned(slots, 4) ||
      (k_values && (!aligned(k_values, 16) || !aligned(v_values, 16))))
    return QIFT_ERR_ALIGN;
  return qift::report_hip(qift::launch_kv4_append(
      pool(cache), static_cast<const uint16_t*>(k), static_cast<const uint16_t*>(v), k_stride, v_stride, dtype, slots, n,
      static_cast<uint16_t*>(k_values), static_cast<uint16_t*>(v_values), (hipStream_t)stream));
}

int qift_kv4_read(const qift_kv4_pages* cache, const int32_t* slots, int64_t n, int32_t dtype, void* k_values,
                  void* v_values, qift_stream_t stream) {
  int st = check_shape(cache);
  if (st != QIFT_OK) return st;
  if (dtype != QIFT_F16 && dtype != QIFT_BF16 && dtype != QIFT_F32) return QIFT_ERR_FORMAT;
  if (n < 0 || (n + 63) / 64 >= kGroups) return QIFT_ERR_SHAPE;   // 64 tokens to a workgroup
  if (n == 0) return QIFT_OK;
  if (!slots || !k_values || !v_values) return QIFT_ERR_NULL;
  st = check_pointers(cache);
  if (st != QIFT_OK) return st;
  if (!aligned(slots, 4) || !aligned(k_values, 16) || !aligned(v_values, 16)) return QIFT_ERR_ALIGN;
  return qift::report_hip(qift::launch_kv4_read(pool(cache), slots, n, dtype, k_values, v_values, (hipStream_t)stream));
}

size_t qift_kv4_attention_tree_workspace_bytes(int64_t B, int32_t Hq, int32_t Hkv, int32_t head_dim, int32_t max_nodes,
                                               int64_t max_len) {
  if (!tree_shape_ok(B, Hq, Hkv, head_dim, max_nodes, max_len) || B == 0) return 0;
  return (size_t)qift::pages::most_workspace_words(B, Hkv, Hq / Hkv, max_nodes, max_len) * sizeof(float);
}

int qift_kv4_attention_tree(const qift_kv4_pages* cache, const void* q, int64_t q_stride, int32_t dtype, int64_t rows,
                            const int32_t* table, int32_t table_pages, const int32_t* starts, const int32_t* lens,
                            int64_t B, int32_t Hq, int32_t max_nodes, int64_t max_len, const uint64_t* visible, void* out,
                            void* workspace, size_t workspace_bytes, qift_stream_t stream) {
  int st = check_shape(cache);
  if (st != QIFT_OK) return st;
  if (dtype != QIFT_F16 && dtype != QIFT_BF16) return QIFT_ERR_FORMAT;
  if (!tree_shape_ok(B, Hq, cache->Hkv, cache->head_dim, max_nodes, max_len)) return QIFT_ERR_SHAPE;
  if (rows < 0 || rows >= k31 || table_pages < 1 || q_stride < (int64_t)Hq * 128 || q_stride >= k31) return QIFT_ERR_SHAPE;
  if (B == 0 || rows == 0) return QIFT_OK;
  if (!q || !table || !starts || !lens || !out) return QIFT_ERR_NULL;
  st = check_pointers(cache);
  if (st != QIFT_OK) return st;
  const int32_t Hkv = cache->Hkv, G = Hq / Hkv;
  const size_t need =
      (size_t)qift::pages::workspace_words(qift::pages::plan(B, Hkv, G, max_nodes, max_len), B, Hkv, G, max_nodes) * sizeof(float);
  if (need > 0 && (!workspace || workspace_bytes < need)) return QIFT_ERR_WORKSPACE;
  if (!aligned(q, 16) || q_stride % 8 || !aligned(out, 16) || !aligned(table, 4) || !aligned(starts, 4) ||
      !aligned(lens, 4) || (visible && !aligned(visible, 8)) || (need > 0 && !aligned(workspace, 16)))
    return QIFT_ERR_ALIGN;
  qift::TreeCall a;
  a.c = pool(cache);
  a.q = static_cast<const uint16_t*>(q);
  a.q_stride = q_stride;
  a.rows = rows;
  a.B = B;
  a.max_len = max_len;
  a.table = table;
  a.starts = starts;
  a.lens = lens;
  a.visible = visible;
  a.out = static_cast<uint16_t*>(out);
  a.ws = static_cast<float*>(workspace);
  a.table_pages = table_pages;
  a.Hq = Hq;
  a.max_nodes = max_nodes;
  a.dtype = dtype;
  return qift::report_hip(qift::launch_kv4_tree(a, (hipStream_t)stream));
}

}  // extern "C"
