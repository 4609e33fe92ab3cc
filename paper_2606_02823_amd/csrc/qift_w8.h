// What the kernels of the 8-bit linear share: y[m, n] = s_w[n] s_x[m] sum_k level[n, k] q[m, k] over int8 levels and codes.
#pragma once

#include <type_traits>

#include "qift_fwht.h"   // buffer-load helpers
#include "qift_internal.h"
#include "qift_mma.h"

namespace qift {
namespace w8 {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));

constexpr int kAcc = 3;   // in place of an element type: the int32 sums themselves

// fp32(fp32(acc) s_x) s_w, each product rounded to fp32
__device__ __forceinline__ float scaled(int acc, float s_x, float s_w) {
  float t = (float)acc * s_x;
  asm volatile("" : "+v"(t));   // (not joined with the product or the conversion behind it, which would round once)
  t *= s_w;
  asm volatile("" : "+v"(t));
  return t;
}

// Four outputs as OT stores them: 8 bytes of fp16 or bf16 (to nearest, ties to even), 16 of fp32 or int32.
template <int OT>
using Quad = std::conditional_t<OT == kF16 || OT == kBF16, uint2, uint4>;
template <int OT>
__device__ __forceinline__ Quad<OT> quad(const int (&a)[4], float s_x, const float (&s_w)[4]) {
  if constexpr (OT == kAcc) {
    return make_uint4((uint32_t)a[0], (uint32_t)a[1], (uint32_t)a[2], (uint32_t)a[3]);
  } else {
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = scaled(a[i], s_x, s_w[i]);
    if constexpr (OT == kF32) {
      return make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
    } else {
      uint2 u;
      if constexpr (OT == kBF16) {
        asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(u.x) : "v"(y[0]), "v"(y[1]));
        asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(u.y) : "v"(y[2]), "v"(y[3]));
      } else {
        asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(u.x) : "v"(y[0]), "v"(y[1]));
        asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(u.y) : "v"(y[2]), "v"(y[3]));
      }
      return u;
    }
  }
}
template <int OT>
constexpr int size_of() { return OT == kF16 || OT == kBF16 ? 2 : 4; }

// Vectors at any multiple of two bytes: rows of y begin at m N, and the compiler stores such vectors whole on this target.
typedef uint32_t words2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t words4 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ void store_words(uint8_t* to, const uint2& v) { *reinterpret_cast<words2*>(to) = words2{v.x, v.y}; }
__device__ __forceinline__ void store_words(uint8_t* to, const uint4& v) {
  *reinterpret_cast<words4*>(to) = words4{v.x, v.y, v.z, v.w};
}
// The outputs n0 .. of token m that v holds, those below N.
template <int OT, typename V>
__device__ __forceinline__ void store_row(void* y, int64_t m, int64_t n0, int64_t N, const V& v) {
  constexpr int SZ = size_of<OT>(), E = sizeof(V) / SZ;
  uint8_t* to = static_cast<uint8_t*>(y) + (m * N + n0) * SZ;
  if (n0 + E <= N) {
    store_words(to, v);
    return;
  }
  const uint32_t* w = reinterpret_cast<const uint32_t*>(&v);
#pragma unroll
  for (int i = 0; i < E; ++i) {
    if (n0 + i >= N) break;
    if constexpr (SZ == 2) reinterpret_cast<uint16_t*>(to)[i] = (uint16_t)(w[i >> 1] >> (16 * (i & 1)));
    else reinterpret_cast<uint32_t*>(to)[i] = w[i];
  }
}

// The scales of rows n0 .. n0 + 3 (n0 a multiple of 4), as fp16 bits; zeros past the last row.
__device__ __forceinline__ uint2 load_scales(const uint16_t* sw, int64_t n0, int64_t N) {
  if (n0 + 4 <= N) return *reinterpret_cast<const uint2*>(sw + n0);
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = n0 + i < N ? sw[n0 + i] : 0u;
  return make_uint2(v[0] | (v[1] << 16), v[2] | (v[3] << 16));
}
__device__ __forceinline__ void scales4(uint2 u, float (&s)[4]) {
  const uint32_t w[2] = {u.x, u.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) s[i] = __half2float(__ushort_as_half((uint16_t)(w[i >> 1] >> (16 * (i & 1)))));
}

}  // namespace w8
}  // namespace qift
