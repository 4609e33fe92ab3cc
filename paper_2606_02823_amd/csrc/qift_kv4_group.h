// The 4-bit quantizer of one key or value vector (a group of 128 values) and the reductions over a wave's rows of 16
// lanes that it and the attention kernels use.
//
// 16 lanes per group, lane j holding values 8j .. 8j + 7.  In fp32, in this order, rounding half to even:
//   x_max = c max(max x, 0), x_min = c min(min x, 0) with c = fp32(0.95),
//   s = (x_max - x_min) / 15 (1 for a group of zeros), z = round(-x_min / s),
//   q = clip(round(x / s) + z, 0, 15),   reconstruction s (q - z).
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qift {
namespace {

constexpr int kD = 128;         // head dimension

typedef _Float16 v2h __attribute__((ext_vector_type(2)));

// Reductions by DPP moves within rows of 16 lanes (every lane gets its row's result) and lane reads across
// the four rows: a few cycles a step, where a shuffle through LDS takes about a hundred.
#define QIFT_DPP_B32(x, CTRL) __builtin_amdgcn_update_dpp(x, x, CTRL, 0xf, 0xf, false)
template <typename Op>
__device__ __forceinline__ int row_reduce(int x, Op op) {
  x = op(x, QIFT_DPP_B32(x, 0xb1));    // quad_perm [1,0,3,2]
  x = op(x, QIFT_DPP_B32(x, 0x4e));    // quad_perm [2,3,0,1]
  x = op(x, QIFT_DPP_B32(x, 0x141));   // row_half_mirror
  return op(x, QIFT_DPP_B32(x, 0x140));   // row_mirror
}

template <typename Op>
__device__ __forceinline__ float wave_reduce(float x, Op op) {   // every lane gets the wave's result
  const int r = row_reduce(__float_as_int(x), [&](int a, int b) {
    return __float_as_int(op(__int_as_float(a), __int_as_float(b)));
  });
  auto row = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(r, l)); };
  return op(op(row(0), row(16)), op(row(32), row(48)));
}
__device__ __forceinline__ float max_op(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float add_op(float a, float b) { return a + b; }

__device__ __forceinline__ v2h pk_max(v2h a, v2h b) { return __builtin_elementwise_max(a, b); }

// d / 15 correctly rounded for a finite d >= 0 that is 0 or far above the subnormals (the values here are
// fp16 times 0.95): the quotient by the rounded reciprocal, then one correction (checked against the
// division for every fp32 mantissa).
__device__ __forceinline__ float div15(float d) {
  constexpr float y = 1.0f / 15.0f;
  const float q = d * y;
  return d == INFINITY ? d : fmaf(fmaf(-q, 15.0f, d), y, q);
}

struct Kv4Group {
  float s, z;
  float q[8];   // the codes as whole numbers
  // as bytes, even values and odd ones, then two to a byte: values 8j .. 8j + 7
  __device__ __forceinline__ uint32_t codes() const {
    uint32_t even = 0, odd = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      if (e & 1) odd = __builtin_amdgcn_cvt_pk_u8_f32(q[e], e >> 1, odd);
      else even = __builtin_amdgcn_cvt_pk_u8_f32(q[e], e >> 1, even);
    }
    return even | (odd << 4);
  }
};

// The group whose 8 values of this lane are the 16 bytes u: fp16, or bf16.  Every lane of the wave takes part.
template <bool BF16>
__device__ __forceinline__ Kv4Group kv4_group(const uint4& u) {
  Kv4Group g;
  float v[8], top, bottom;
  if constexpr (BF16) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = __uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    top = bottom = v[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) {
      top = fmaxf(top, v[e]);
      bottom = fminf(bottom, v[e]);
    }
    auto f = [](int a) { return __int_as_float(a); };
    top = f(row_reduce(__float_as_int(top), [&](int a, int b) { return __float_as_int(fmaxf(f(a), f(b))); }));
    bottom = f(row_reduce(__float_as_int(bottom), [&](int a, int b) { return __float_as_int(fminf(f(a), f(b))); }));
  } else {
    const v2h h[4] = {__builtin_bit_cast(v2h, u.x), __builtin_bit_cast(v2h, u.y), __builtin_bit_cast(v2h, u.z),
                      __builtin_bit_cast(v2h, u.w)};
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)h[e >> 1][e & 1];
    // (max x, max -x) of the lane, then of its group's 16 lanes
    const v2h hx = pk_max(pk_max(h[0], h[1]), pk_max(h[2], h[3]));
    const v2h hn = pk_max(pk_max(-h[0], -h[1]), pk_max(-h[2], -h[3]));
    const v2h both = pk_max(v2h{hx[0], hn[0]}, v2h{hx[1], hn[1]});
    const v2h ext = __builtin_bit_cast(v2h, row_reduce(__builtin_bit_cast(int, both), [](int a, int b) {
                                         return __builtin_bit_cast(int, pk_max(__builtin_bit_cast(v2h, a), __builtin_bit_cast(v2h, b)));
                                       }));
    top = (float)ext[0];
    bottom = -(float)ext[1];
  }
  const float c = 0.95f;
  const float x_max = fmaxf(top, 0.f) * c, x_min = fminf(bottom, 0.f) * c;
  float s = BF16 ? (x_max - x_min) / 15.0f : div15(x_max - x_min);   // bf16 ranges reach fp32's subnormals
  if (s == 0.f) s = 1.f;
  // rint of the rounded quotient v / s without the division where it is clear: q0 = rint(v r), r the
  // approximate reciprocal, is that value when the residual v - q0 s lies inside half a step by more
  // than both roundings (|v / s| < 32 here); otherwise (a wave-uniform branch, rarely taken) divide.
  // The zero-point is decided the same way.
  const float inv = __builtin_amdgcn_rcpf(s);
  float qf[8];
  float z = rintf(-x_min * inv);
  float res = fabsf(fmaf(-z, s, -x_min));
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    qf[e] = rintf(v[e] * inv);
    res = fmaxf(res, fabsf(fmaf(-qf[e], s, v[e])));
  }
  const float half = (0.5f - 0x1p-16f) * s;
  bool divide = !(res < half);
  // (a bf16 group may have a step whose reciprocal or residuals leave the normal numbers)
  if (BF16) divide |= !(s > 0x1p-100f && s < 0x1p100f);
  if (__any(divide)) {
    z = rintf(-x_min / s);
#pragma unroll
    for (int e = 0; e < 8; ++e) qf[e] = rintf(v[e] / s);
  }
  z = fminf(fmaxf(z, 0.f), 15.f);
#pragma unroll
  for (int e = 0; e < 8; ++e) g.q[e] = fminf(fmaxf(qf[e] + z, 0.f), 15.f);
  g.s = s;
  g.z = z;
  return g;
}

}  // namespace
}  // namespace qift
