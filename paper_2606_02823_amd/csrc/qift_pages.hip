// The paged KV4 cache: quantizing new tokens' keys and values into their slots, and reading slots back.
//
// Both work on tiles of 16 tokens of one KV head and one side (keys or values), a group of 16 lanes to a token, as
// kv4_group has it: a tile of consecutive slots then is 1 KB of codes, 64 bytes of scales and 16 of zero-points of one
// page, whole pieces of lines that one workgroup writes, while its 16 rows of the input are 256 bytes each.
#include "qift_fwht.h"   // flag_error
#include "qift_internal.h"
#include "qift_kv4_group.h"
#include "qift_pages.h"

namespace qift {
namespace {

// Eight values of a lane as 16 bytes of fp16 or bf16, to nearest, ties to even.  (The conversions are written out: from
// the plain casts the compiler joins the product before them and the conversion to fp16 in one instruction with one
// rounding, where the value is the product rounded to fp32.)
template <int DT>
__device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    if constexpr (DT == kBF16) asm("v_cvt_pk_bf16_f32 %0, %1, %2" : "=v"(w[e]) : "v"(x[2 * e]), "v"(x[2 * e + 1]));
    else asm("v_cvt_pk_f16_f32 %0, %1, %2" : "=v"(w[e]) : "v"(x[2 * e]), "v"(x[2 * e + 1]));
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct Side {
  uint8_t* codes;
  float* scales;
  uint8_t* zeros;
};

// Workgroup (tile, side, head), heads fastest, of 16 tokens, its group of lanes l / 16 the token 16 tile + l / 16.  Bound by
// its bytes (without its arithmetic it takes as long), and those come best when the heads of a token are read together:
// 16384 tokens of 8 heads with the values written, 152 MB, 36.7 us with the tiles fastest, 32.1 so (4.7 TB/s; 31.0 us at a
// large copy's rate; all times here are of captured calls on two caches in turn, so that the Infinity Cache holds neither).
// More tiles to a workgroup, their loads ahead, were no faster.
template <bool BF16>
__global__ __launch_bounds__(256) void k_append(const uint16_t* __restrict__ k, const uint16_t* __restrict__ v,
                                                int64_t ks, int64_t vs, const int32_t* __restrict__ slots, int n,
                                                pages::Div page, pages::Div heads, uint32_t capacity, Side kc, Side vc,
                                                uint16_t* __restrict__ kv, uint16_t* __restrict__ vv, uint32_t* err) {
  const int j = threadIdx.x & 15;
  const uint32_t Hkv = heads.d, ts = pages::quotient(blockIdx.x, heads), head = blockIdx.x - ts * Hkv;
  const bool side = (ts & 1) != 0;
  const uint16_t* x = (side ? v : k) + head * kD + 8 * j;
  const Side c = side ? vc : kc;
  uint16_t* o = side ? vv : kv;
  const int64_t t = (int64_t)(ts >> 1) * 16 + (threadIdx.x >> 4), tr = t < n ? t : n - 1;   // rows past the last read it again
  const uint4 u = *reinterpret_cast<const uint4*>(x + tr * (side ? vs : ks));
  const int32_t slot = slots[tr];
  const Kv4Group g = kv4_group<BF16>(u);
  const bool in = t < n, write = in && slot >= 0 && (uint32_t)slot < capacity;
  if (in && slot >= 0 && !write && j == 0) dev::flag_error(err, kDevErrIndex);
  if (write) {
    const uint32_t row = pages::slot_row((uint32_t)slot, page, Hkv, head);
    reinterpret_cast<uint32_t*>(c.codes + (uint64_t)row * (kD / 2))[j] = g.codes();
    if (j == 0) {
      c.scales[row] = g.s;
      c.zeros[row] = (uint8_t)g.z;
    }
  }
  if (o && in) {
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = write ? g.s * (g.q[e] - g.z) : 0.f;
    *reinterpret_cast<uint4*>(o + (t * Hkv + head) * kD + 8 * j) = pack8<BF16 ? kBF16 : kF16>(y);
  }
}

// N tiles of 16 tokens of a head and side to a workgroup, every load sent before the first is used.  Bound by its bytes, most
// of them written: 32768 tokens of 8 heads to bf16, 170 MB, 36.6 us (4.7 TB/s; 34.7 us at a large copy's rate);
// here the tiles are fastest (heads fastest: 40 us).
template <int DT, int N>
__global__ __launch_bounds__(256) void k_read(const int32_t* __restrict__ slots, int n, pages::Div page, uint32_t Hkv,
                                              uint32_t capacity, Side kc, Side vc, void* __restrict__ ko,
                                              void* __restrict__ vo, uint32_t* err) {
  const int j = threadIdx.x & 15;
  const uint32_t head = blockIdx.y;
  const bool side = blockIdx.z != 0;
  const Side c = side ? vc : kc;
  void* o = side ? vo : ko;
  const int64_t t0 = (int64_t)blockIdx.x * (16 * N) + (threadIdx.x >> 4);
  int32_t slot[N];
  uint32_t w[N];
  float s[N], z[N];
#pragma unroll
  for (int i = 0; i < N; ++i) slot[i] = t0 + 16 * i < n ? slots[t0 + 16 * i] : -1;
#pragma unroll
  for (int i = 0; i < N; ++i) {   // what is no slot reads the cache's first row
    const bool have = slot[i] >= 0 && (uint32_t)slot[i] < capacity;
    if (slot[i] >= 0 && !have && j == 0) dev::flag_error(err, kDevErrIndex);
    const uint32_t row = have ? pages::slot_row((uint32_t)slot[i], page, Hkv, head) : 0u;
    w[i] = reinterpret_cast<const uint32_t*>(c.codes + (uint64_t)row * (kD / 2))[j];
    s[i] = c.scales[row];
    z[i] = (float)c.zeros[row];
    if (!have) slot[i] = -1;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t t = t0 + 16 * i;
    if (t >= n) continue;
    float y[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = slot[i] >= 0 ? s[i] * ((float)((w[i] >> (4 * e)) & 15u) - z[i]) : 0.f;
    const int64_t at = (t * Hkv + head) * kD + 8 * j;
    if constexpr (DT == kF32) {
      float4* p = reinterpret_cast<float4*>(static_cast<float*>(o) + at);
      p[0] = make_float4(y[0], y[1], y[2], y[3]);
      p[1] = make_float4(y[4], y[5], y[6], y[7]);
    } else {
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(o) + at) = pack8<DT>(y);
    }
  }
}

}  // namespace

hipError_t launch_kv4_append(const Kv4Pool& c, const uint16_t* k, const uint16_t* v, int64_t ks, int64_t vs, int dtype,
                             const int32_t* slots, int64_t n, uint16_t* kv, uint16_t* vv, hipStream_t s) {
  const dim3 grid((unsigned)((n + 15) / 16 * 2 * c.Hkv));
  const pages::Div page = pages::make_div((uint32_t)c.page);
  const uint32_t cap = (uint32_t)(c.pages * c.page);
  const Side kc = {c.kc, c.ks, c.kz}, vc = {c.vc, c.vs, c.vz};
  auto kernel = dtype == kBF16 ? k_append<true> : k_append<false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, k, v, ks, vs, slots, (int)n, page,
                     pages::make_div((uint32_t)c.Hkv), cap, kc, vc, kv, vv,
                     device_error_word());
  return hipGetLastError();
}

hipError_t launch_kv4_read(const Kv4Pool& c, const int32_t* slots, int64_t n, int dtype, void* ko, void* vo,
                           hipStream_t s) {
  // four tiles to a workgroup where that leaves at least four workgroups to a CU: 32768 tokens of 8 heads 46.4 -> 36.6 us,
  // 333 of 32 heads 4.1 against 4.5
  const bool wide = n * c.Hkv * 2 >= 65536;
  const dim3 grid((unsigned)((n + (wide ? 63 : 15)) / (wide ? 64 : 16)), (unsigned)c.Hkv, 2);
  const pages::Div page = pages::make_div((uint32_t)c.page);
  const uint32_t cap = (uint32_t)(c.pages * c.page);
  const Side kc = {c.kc, c.ks, c.kz}, vc = {c.vc, c.vs, c.vz};
  auto kernel = dtype == kF32    ? (wide ? k_read<kF32, 4> : k_read<kF32, 1>)
                : dtype == kBF16 ? (wide ? k_read<kBF16, 4> : k_read<kBF16, 1>)
                                 : (wide ? k_read<kF16, 4> : k_read<kF16, 1>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, slots, (int)n, page, (uint32_t)c.Hkv, cap, kc, vc, ko, vo,
                     device_error_word());
  return hipGetLastError();
}

}  // namespace qift
