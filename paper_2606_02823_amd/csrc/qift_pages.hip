// The paged KV4 cache: quantizing new tokens' keys and values into their slots, and reading slots back.
//
// Both work on tiles of 16 tokens of one KV head and one side (keys or values), a group of 16 lanes to a token, as
// kv4_group has it: a tile of consecutive slots then is 1 KB of codes, 64 bytes of scales and 16 of zero-points of one
// page, whole pieces of lines that one workgroup writes, while its 16 rows of the input are 256 bytes each.
#include "qift_internal.h"
#include "qift_kv4_group.h"
#include "qift_pages.h"

namespace qift {
namespace {

typedef _Float16 v8h __attribute__((ext_vector_type(8)));

// bf16 bits of a float, to nearest, ties to even (NaN stays one)
__device__ __forceinline__ uint32_t bf16_bits(float f) {
  const uint32_t u = __float_as_uint(f);
  return f == f ? (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16 : (u >> 16) | 0x40u;
}

// Eight values of a lane as 16 bytes of fp16 or bf16
template <int DT>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (DT == kBF16) {
      w[e] = bf16_bits(x[2 * e]) | (bf16_bits(x[2 * e + 1]) << 16);
    } else {
      const v2h h = {(_Float16)x[2 * e], (_Float16)x[2 * e + 1]};
      w[e] = __builtin_bit_cast(uint32_t, h);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// s (q - z) rounded to fp32.  (The value passes through a register that the compiler cannot see into: it would else join
// the product and the conversion to fp16 in one instruction with one rounding.)
__device__ __forceinline__ float value(float s, float d) {
  float y = s * d;
  asm("" : "+v"(y));
  return y;
}

struct Side {
  uint8_t* codes;
  float* scales;
  uint8_t* zeros;
};

// Workgroup (tile, head, side) of 16 tokens, its group of lanes l / 16 the token 16 tile + l / 16.
template <bool BF16>
__global__ __launch_bounds__(256) void k_append(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                int64_t ks, int64_t vs, const int32_t* __restrict__ slots, int n,
                                                pages::Div page, uint32_t Hkv, uint32_t capacity, Side kc, Side vc,
                                                uint16_t* __restrict__ kv, uint16_t* __restrict__ vv, uint32_t* err) {
  const int j = threadIdx.x & 15;
  const uint32_t head = blockIdx.y;
  const bool side = blockIdx.z != 0;
  const int64_t t = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const bool in = t < n;
  const uint16_t* x = (side ? v : k) + (in ? t : 0) * (side ? vs : ks) + head * kD;
  const uint4 u = reinterpret_cast<const uint4*>(x)[j];
  const int32_t slot = in ? slots[t] : -1;
  const Kv4Group g = kv4_group<BF16>(u);
  const bool write = slot >= 0 && (uint32_t)slot < capacity;
  if (slot >= 0 && !write && j == 0 && err) atomicOr(err, kDevErrIndex);
  const Side c = side ? vc : kc;
  if (write) {
    const uint32_t row = pages::slot_row((uint32_t)slot, page, Hkv, head);
    reinterpret_cast<uint32_t*>(c.codes + (uint64_t)row * (kD / 2))[j] = g.codes();
    if (j == 0) {
      c.scales[row] = g.s;
      c.zeros[row] = (uint8_t)g.z;
    }
  }
  if (kv && in) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = write ? value(g.s, g.q[e] - g.z) : 0.f;
    uint16_t* o = (side ? vv : kv) + (t * Hkv + head) * kD;
    reinterpret_cast<uint4*>(o)[j] = pack8<BF16 ? kBF16 : kF16>(y);
  }
}

template <int DT>
__global__ __launch_bounds__(256) void k_read(const int32_t* __restrict__ slots, int n, pages::Div page, uint32_t Hkv,
                                              uint32_t capacity, Side kc, Side vc, void* __restrict__ ko,
                                              void* __restrict__ vo, uint32_t* err) {
  const int j = threadIdx.x & 15;
  const uint32_t head = blockIdx.y;
  const bool side = blockIdx.z != 0;
  const int64_t t = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  if (t >= n) return;
  const int32_t slot = slots[t];
  const bool have = slot >= 0 && (uint32_t)slot < capacity;
  if (slot >= 0 && !have && j == 0 && err) atomicOr(err, kDevErrIndex);
  const Side c = side ? vc : kc;
  uint32_t w = 0;
  float s = 0.f, z = 0.f;
  if (have) {
    const uint32_t row = pages::slot_row((uint32_t)slot, page, Hkv, head);
    w = reinterpret_cast<const uint32_t*>(c.codes + (uint64_t)row * (kD / 2))[j];
    s = c.scales[row];
    z = (float)c.zeros[row];
  }
  float y[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) y[e] = value(s, (float)((w >> (4 * e)) & 15u) - z);
  const int64_t at = (t * Hkv + head) * kD;
  if constexpr (DT == kF32) {
    float4* o = reinterpret_cast<float4*>(static_cast<float*>(side ? vo : ko) + at) + 2 * j;
    o[0] = make_float4(y[0], y[1], y[2], y[3]);
    o[1] = make_float4(y[4], y[5], y[6], y[7]);
  } else {
    reinterpret_cast<uint4*>(static_cast<uint16_t*>(side ? vo : ko) + at)[j] = pack8<DT>(y);
  }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Pool& c, const uint16_t* k, const uint16_t* v, int64_t ks, int64_t vs, int dtype,
                             const int32_t* slots, int64_t n, uint16_t* kv, uint16_t* vv, hipStream_t s) {
  const dim3 grid((unsigned)((n + 15) / 16), (unsigned)c.Hkv, 2);
  const pages::Div page = pages::make_div((uint32_t)c.page);
  const uint32_t cap = (uint32_t)(c.pages * c.page);
  const Side kc = {c.kc, c.ks, c.kz}, vc = {c.vc, c.vs, c.vz};
  auto kernel = dtype == kBF16 ? k_append<true> : k_append<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, k, v, ks, vs, slots, (int)n, page, (uint32_t)c.Hkv, cap, kc, vc, kv, vv,
                     device_error_word());
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Pool& c, const int32_t* slots, int64_t n, int dtype, void* ko, void* vo,
                           hipStream_t s) {
  const dim3 grid((unsigned)((n + 15) / 16), (unsigned)c.Hkv, 2);
  const pages::Div page = pages::make_div((uint32_t)c.page);
  const uint32_t cap = (uint32_t)(c.pages * c.page);
  const Side kc = {c.kc, c.ks, c.kz}, vc = {c.vc, c.vs, c.vz};
  auto kernel = dtype == kF32 ? k_read<kF32> : dtype == kBF16 ? k_read<kBF16> : k_read<kF16>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, slots, (int)n, page, (uint32_t)c.Hkv, cap, kc, vc, ko, vo,
                     device_error_word());
  return hipGetLastError();
}

}  // namespace qift
