// C ABI of the 8-bit linear (include/qift_w8.h): host-side validation, then dispatch.  Every check runs before the first HIP
// call.
#include "../../include/qift_w8.h"
#include "qift_internal.h"

namespace {

constexpr int64_t k31 = int64_t(1) << 31;
constexpr int64_t kRows24 = int64_t(1) << 24, kTokens23 = int64_t(1) << 23;   // workgroups of 256 and of 512: fewer than 2^32 threads
constexpr int64_t kMaxK = 131072;   // 127 * 127 * K stays below 2^31

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

bool clip_ok(int32_t flags, int* num, int* den) {
  *num = *den = 1;
  if (flags == 0) return true;
  if (flags & ~0xFFFF) return false;
  *num = (flags >> 8) & 0xFF;
  *den = flags & 0xFF;
  return *num >= 1 && *num <= *den && *den <= 16;
}

bool block_ok(int32_t b, int32_t most, int64_t K) { return b >= 2 && b <= most && (b & (b - 1)) == 0 && K % b == 0; }

bool shape_ok(int64_t N, int64_t K, int64_t M) {
  if (N < 1 || N >= k31 || K < 64 || K % 64 || K > kMaxK || M < 1 || M >= k31) return false;
  return ((N + 127) / 128) * ((M + 127) / 128) < (int64_t(1) << 20);   // fewer than 2^32 threads
}

}  // namespace

extern "C" {

int qift_quantize_weights8(const float* W, int64_t N, qift_hadamard_spec spec, int8_t* levels, uint16_t* scales,
                           qift_stream_t stream) {
  if (!W || !levels || !scales) return QIFT_ERR_NULL;
  if (N < 1 || N >= kRows24 || spec.K < 64 || spec.K % 64 || spec.K > qift::kWquantMaxK || N * spec.K >= k31) return QIFT_ERR_SHAPE;
  if (!block_ok(spec.block, 4096, spec.K) || spec.flags != 0) return QIFT_ERR_SPEC;
  if (!aligned16(W) || !aligned16(levels) || !aligned16(scales)) return QIFT_ERR_ALIGN;
  return qift::report_hip(qift::launch_quantize_weights8(W, N, spec.K, spec.block, levels, scales, (hipStream_t)stream));
}

int qift_rotate_quant_act8(const uint16_t* x, int64_t M, qift_hadamard_spec spec, int8_t* act_q, float* act_scale,
                           qift_stream_t stream) {
  if (!x || !act_q || !act_scale) return QIFT_ERR_NULL;
  if (M < 1 || M >= kTokens23 || spec.K < 64 || spec.K % 64 || spec.K > qift::kActMaxK) return QIFT_ERR_SHAPE;
  const bool bf16 = (spec.flags & QIFT_SPEC_BF16) != 0;
  int num, den;
  if (!block_ok(spec.block, 8192, spec.K) || !clip_ok(spec.flags & ~QIFT_SPEC_BF16, &num, &den)) return QIFT_ERR_SPEC;
  if (!aligned16(x) || !aligned16(act_q) || !aligned16(act_scale)) return QIFT_ERR_ALIGN;
  return qift::report_hip(
      qift::launch_rotate_quant_act8(x, M, spec.K, spec.block, num, den, act_q, act_scale, (hipStream_t)stream, bf16));
}

size_t qift_w8a8_workspace_bytes(const qift_w8* w, int64_t M) {
  return w && shape_ok(w->N, w->K, M) ? qift::route::w8_workspace(qift::route::w8_plan(w->N, M, w->K, true), w->N, M) : 0;
}

int qift_w8a8_linear(const qift_w8* w, const int8_t* act_q, const float* act_scale, int64_t M, int32_t dtype, void* out,
                     int32_t* acc_out, void* workspace, size_t workspace_bytes, qift_stream_t stream) {
  if (!w || !w->levels || !w->scales || !act_q || !act_scale || !out) return QIFT_ERR_NULL;
  if (dtype != QIFT_F16 && dtype != QIFT_BF16 && dtype != QIFT_F32) return QIFT_ERR_FORMAT;
  if (!shape_ok(w->N, w->K, M)) return QIFT_ERR_SHAPE;
  const qift::route::W8Plan plan = qift::route::w8_plan(w->N, M, w->K, workspace_bytes > 0);
  if (workspace_bytes > 0 && (!workspace || workspace_bytes < qift::route::w8_workspace(plan, w->N, M))) return QIFT_ERR_WORKSPACE;
  const void* p[] = {w->levels, w->scales, act_q, act_scale, out, acc_out, workspace};
  for (const void* x : p)
    if (!aligned16(x)) return QIFT_ERR_ALIGN;
  const qift::W8Call c = {w->levels, w->scales, w->N, w->K, act_q, act_scale, M, out, acc_out,
                          workspace_bytes > 0 ? workspace : nullptr, dtype};
  const hipStream_t s = (hipStream_t)stream;
  return qift::report_hip(plan.rows ? qift::launch_w8_rows(c, plan, s) : qift::launch_w8_gemm(c, plan, s));
}

}  // extern "C"
