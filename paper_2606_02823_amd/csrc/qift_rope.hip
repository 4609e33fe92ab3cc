// Norms of queries and keys for each head, and the rotation by position, in one pass over the rows.
//
//   y = x / sqrt(mean(x^2) + eps) * w      over the 128 values of a head (no weight: y = x)
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * freq[i]
// for the pairs i of the first rot values: values i and i + rot / 2, or 2 i and 2 i + 1.  fp32 throughout, the angle in fp64
// (step::turn); one rounding at the end.
#include "qift_fwht.h"
#include "qift_internal.h"
#include "qift_step.h"

namespace qift {
namespace {

constexpr int kHead = 128;

// Sum over the 16 lanes of a row of the wave, in every lane.
__device__ __forceinline__ float row_sum(float x) {
#define QIFT_ADD(CTRL) x += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, false))
  QIFT_ADD(0xb1);    // quad_perm [1,0,3,2]
  QIFT_ADD(0x4e);    // quad_perm [2,3,0,1]
  QIFT_ADD(0x141);   // row_half_mirror
  QIFT_ADD(0x140);   // row_mirror
#undef QIFT_ADD
  return x;
}

template <bool BF16>
__device__ __forceinline__ void unpack4(uint2 u, float (&v)[4]) {
  const uint32_t w[2] = {u.x, u.y};
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const uint32_t h = w[e >> 1];
    if constexpr (BF16) v[e] = __uint_as_float((e & 1) ? h & 0xFFFF0000u : h << 16);
    else v[e] = __half2float(__ushort_as_half((uint16_t)(h >> (16 * (e & 1)))));
  }
}
template <bool BF16>
__device__ __forceinline__ uint2 pack4(const float (&v)[4]) {   // to nearest, ties to even
  uint2 u;
  if constexpr (BF16) {
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(u.x) : "v"(v[0]), "v"(v[1]));
    asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(u.y) : "v"(v[2]), "v"(v[3]));
  } else {
    asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(u.x) : "v"(v[0]), "v"(v[1]));
    asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(u.y) : "v"(v[2]), "v"(v[3]));
  }
  return u;
}

// A wave takes up to 4 NG heads of one row, 16 lanes to a head; a lane has eight values as two fours, so that both values of
// its four pairs are its own: values 4 l and rot / 2 + 4 l on (PAIRS: 8 l and 8 l + 4 on), and past the rotated ones the rest.
// The four angles of a lane are the same for every head: lane (g, l) works out the g-th and the others read it from there.
// Bound by the bytes, each read and written once (16384 rows of 40 heads, 336 MB, 66.4 us, 5.05 TB/s).
template <bool BF16, bool PAIRS, int NG>
__global__ __launch_bounds__(256) void k_rope(RopeCall c, pages::Div per_row, uint32_t waves) {
  const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
  const uint32_t w = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
  if (w >= waves) return;
  const uint32_t row = pages::quotient(w, per_row), part = w - row * per_row.d;
  const int turning = c.rot >> 3;
  const bool turns = l < turning;
  int at0, at1;
  if constexpr (PAIRS) {
    at0 = 8 * l;
    at1 = at0 + 4;
  } else {
    at0 = turns ? 4 * l : c.rot + 4 * (l - turning);
    at1 = at0 + (turns ? c.rot / 2 : (kHead - c.rot) / 2);
  }
  const int32_t position = c.positions[row];
  const int first = (int)part * NG * 4, all = c.heads[0] + c.heads[1];
  uint2 u[NG][2];
  bool have[NG], key[NG];
  uint16_t* to[NG];
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    const int h = first + 4 * i + g;
    const step::Head head = step::head_of(h, c.heads[0], c.heads[1]);
    have[i] = head.have;
    key[i] = head.key;
    const int own = head.own;
    const uint16_t* from = (key[i] ? c.x[1] : c.x[0]) + (int64_t)row * (key[i] ? c.x_stride[1] : c.x_stride[0]) + own * kHead;
    to[i] = (key[i] ? c.y[1] : c.y[0]) + (int64_t)row * (key[i] ? c.y_stride[1] : c.y_stride[0]) + own * kHead;
    if (first + 4 * i >= all) break;   // (the wave has no such heads)
    u[i][0] = *reinterpret_cast<const uint2*>(from + at0);
    u[i][1] = *reinterpret_cast<const uint2*>(from + at1);
  }
  float sine = 0.f, cosine = 1.f;
  if (turns) step::turn(position, c.freq[4 * l + g], sine, cosine);
  float s[4], co[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s[j] = __shfl(sine, 16 * j + l);
    co[j] = __shfl(cosine, 16 * j + l);
  }
  float wt[2][2][4];
#pragma unroll
  for (int k = 0; k < 2; ++k)
    if (c.weight[k]) {
      unpack4<BF16>(*reinterpret_cast<const uint2*>(c.weight[k] + at0), wt[k][0]);
      unpack4<BF16>(*reinterpret_cast<const uint2*>(c.weight[k] + at1), wt[k][1]);
    }
#pragma unroll
  for (int i = 0; i < NG; ++i) {
    if (first + 4 * i >= all) break;
    float v[2][4];
    unpack4<BF16>(u[i][0], v[0]);
    unpack4<BF16>(u[i][1], v[1]);
    if (c.weight[0] || c.weight[1]) {
      float sq = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sq = fmaf(v[e >> 2][e & 3], v[e >> 2][e & 3], sq);
      const float r = rsqrtf(fmaf(row_sum(sq), 1.f / kHead, c.eps));
      if (key[i] ? c.weight[1] != nullptr : c.weight[0] != nullptr) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e >> 2][e & 3] *= r * (key[i] ? wt[1][e >> 2][e & 3] : wt[0][e >> 2][e & 3]);
      }
    }
    if (turns) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float& a = PAIRS ? v[j >> 1][2 * (j & 1)] : v[0][j];
        float& b = PAIRS ? v[j >> 1][2 * (j & 1) + 1] : v[1][j];
        const float a0 = a, b0 = b;
        a = fmaf(a0, co[j], -(b0 * s[j]));
        b = fmaf(a0, s[j], b0 * co[j]);
      }
    }
    uint2 o[2] = {pack4<BF16>(v[0]), pack4<BF16>(v[1])};
    if (position < 0) o[0] = o[1] = make_uint2(0u, 0u);   // padding
    if (have[i]) {
      if constexpr (PAIRS) {
        *reinterpret_cast<uint4*>(to[i] + at0) = make_uint4(o[0].x, o[0].y, o[1].x, o[1].y);
      } else {
        *reinterpret_cast<uint2*>(to[i] + at0) = o[0];
        *reinterpret_cast<uint2*>(to[i] + at1) = o[1];
      }
    }
  }
}

template <bool BF16, bool PAIRS, int NG>
hipError_t launch_n(const RopeCall& a, hipStream_t s) {
  const int64_t groups = (a.heads[0] + a.heads[1] + 3) / 4, per = (groups + NG - 1) / NG, waves = a.rows * per;
  hipLaunchKernelGGL((k_rope<BF16, PAIRS, NG>), dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, s, a,
                     pages::make_div((uint32_t)per), (uint32_t)waves);
  return hipGetLastError();
}
// Four heads to a wave until there are about 16 waves to each CU's SIMD; then as many as share the angles and keep loads
// in flight, without a rest where that goes (16384 rows of 40 heads, 336 MB: 4 heads to a wave 82.7 us, 8 70.6, 16 68.4, 20 66.4,
// 32 69.2; 5.05 TB/s, a large copy's rate being 5.10.  2999 rows of 64 heads, 98 MB: 4 23.0, 16 22.5).
template <bool BF16, bool PAIRS>
hipError_t launch_ng(const RopeCall& a, hipStream_t s) {
  const int64_t groups = (a.heads[0] + a.heads[1] + 3) / 4;
  if (a.rows * groups < 16384) return launch_n<BF16, PAIRS, 1>(a, s);
  return groups % 5 == 0 ? launch_n<BF16, PAIRS, 5>(a, s) : launch_n<BF16, PAIRS, 4>(a, s);
}

}  // namespace

hipError_t launch_head_norm_rope(const RopeCall& a, hipStream_t s) {
  if (a.dtype == kBF16) return a.pairs ? launch_ng<true, true>(a, s) : launch_ng<true, false>(a, s);
  return a.pairs ? launch_ng<false, true>(a, s) : launch_ng<false, false>(a, s);
}

}  // namespace qift
