// The 8-bit linear for up to 32 tokens: one pass over the weights, K cut into a slice for each wave.
#include "qift_w8.h"

namespace qift {
namespace {

using namespace w8;

// A workgroup owns `own` weight rows, a multiple of 4 and at most 16 RT, and all the tokens (TT tiles of 16); `own` is chosen
// so that the CUs have equal parts (6144 x 4096 at one token: 24 rows to each of 256 workgroups 7.4 us, 32 to 192 8.0).  Its
// waves take units of 64 U values of k in turn (unit u is wave u mod NWV's), so that together they read whole pieces of each
// row; weights and codes go straight to the operands of the 16 x 16 x 64 product (lane (r, g): row or token r, values 16 g ..
// 16 g + 15 of each 64), the next unit's loads sent before the present one is used.  The waves' sums meet in LDS, each wave
// adding up and storing some of the tiles.
// Bound by the weights' bytes with few tokens (28672 x 4096 at one 23.9 us, 4.9 TB/s; 4096 x 14336 12.5, 4.7; 4096 x 4096 5.9,
// of which 2.5 are the launch and the first loads), with more by what a CU takes into registers, about 27 bytes a ns
// (4096 x 4096 at 32 tokens 8.8 us): tiled products (qift_w8_gemm.hip) take over there.
template <int RT, int TT, int U, int NWV, int OT>
__global__ __launch_bounds__(64 * NWV) void k_w8_rows(const int8_t* __restrict__ W, const uint16_t* __restrict__ sw, int64_t N,
                                                      int K, int own, const int8_t* __restrict__ act, const float* __restrict__ sx,
                                                      int M, void* __restrict__ y, int32_t* __restrict__ acc_out) {
  __shared__ __align__(16) v4i part[NWV][RT * TT][64];
  const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n_base = (int64_t)blockIdx.x * own;
  const int rows = (int)(N - n_base < own ? N - n_base : own);
  const __amdgpu_buffer_rsrc_t wr = dev::make_rsrc(W + n_base * K, (uint32_t)rows * (uint32_t)K);
  const __amdgpu_buffer_rsrc_t ar = dev::make_rsrc(act, (uint32_t)M * (uint32_t)K);
  uint32_t wo[RT], ao[TT];
#pragma unroll
  for (int j = 0; j < RT; ++j) wo[j] = 16 * j + r < rows ? (uint32_t)(16 * j + r) * (uint32_t)K + 16u * g : dev::kOutOfRange;
#pragma unroll
  for (int t = 0; t < TT; ++t) ao[t] = 16 * t + r < M ? (uint32_t)(16 * t + r) * (uint32_t)K + 16u * g : dev::kOutOfRange;
  struct Unit {
    uint4 w[U][RT], a[U][TT];
  };
  // (K is a multiple of 64: what lies past it is out of range in whole 64s)
  auto load = [&](Unit& b, int k) {
#pragma unroll
    for (int s = 0; s < U; ++s) {
      const bool in = k + 64 * s < K;
#pragma unroll
      for (int j = 0; j < RT; ++j) b.w[s][j] = dev::bload16(wr, in ? wo[j] + (uint32_t)(k + 64 * s) : dev::kOutOfRange);
#pragma unroll
      for (int t = 0; t < TT; ++t) b.a[s][t] = dev::bload16(ar, in ? ao[t] + (uint32_t)(k + 64 * s) : dev::kOutOfRange);
    }
  };
  v4i acc[RT][TT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[j][t] = v4i{0, 0, 0, 0};
  auto use = [&](const Unit& b) {
#pragma unroll
    for (int s = 0; s < U; ++s)
#pragma unroll
      for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int t = 0; t < TT; ++t)
          acc[j][t] = mma::mfma_i8(v4i{(int)b.w[s][j].x, (int)b.w[s][j].y, (int)b.w[s][j].z, (int)b.w[s][j].w},
                                   v4i{(int)b.a[s][t].x, (int)b.a[s][t].y, (int)b.a[s][t].z, (int)b.a[s][t].w}, acc[j][t]);
  };
  constexpr int kStride = 64 * U * NWV;
  Unit u0, u1;
  int k = 64 * U * wave;
  load(u0, k);
  for (; k < K; k += 2 * kStride) {
    load(u1, k + kStride);
    use(u0);
    load(u0, k + 2 * kStride);
    use(u1);
  }
#pragma unroll
  for (int i = 0; i < RT * TT; ++i) part[wave][i][lane] = acc[i / TT][i % TT];
  __syncthreads();
  for (int i = wave; i < RT * TT; i += NWV) {
    v4i d = part[0][i][lane];
#pragma unroll
    for (int w = 1; w < NWV; ++w) d += part[w][i][lane];
    const int j = i / TT, t = i - j * TT, m = 16 * t + r;
    const int64_t n0 = n_base + 16 * j + 4 * g;
    if (m >= M || 16 * j + 4 * g >= rows) continue;
    const int a[4] = {d[0], d[1], d[2], d[3]};
    float s4[4];
    scales4(load_scales(sw, n0, N), s4);
    store_row<OT>(y, m, n0, N, quad<OT>(a, sx[m], s4));
    if (acc_out) store_row<kAcc>(acc_out, m, n0, N, quad<kAcc>(a, 0.f, s4));
  }
}

template <int RT, int TT, int U, int NWV>
hipError_t launch_rows(const W8Call& c, int rows, hipStream_t s) {
  const dim3 grid((unsigned)((c.N + rows - 1) / rows));
  auto kernel = c.dtype == kF32    ? k_w8_rows<RT, TT, U, NWV, kF32>
                : c.dtype == kBF16 ? k_w8_rows<RT, TT, U, NWV, kBF16>
                                   : k_w8_rows<RT, TT, U, NWV, kF16>;
  hipLaunchKernelGGL(kernel, grid, dim3(64 * NWV), 0, s, c.levels, c.scales, c.N, (int)c.K, rows, c.act, c.sx, (int)c.M, c.out,
                     c.acc);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w8_rows(const W8Call& c, const route::W8Plan& p, hipStream_t s) {
  if (c.M <= 16) {
    if (p.rows > 16) return launch_rows<2, 1, 4, 4>(c, p.rows, s);
    return route::w8_eight_waves(p, c.N, c.K) ? launch_rows<1, 1, 2, 8>(c, p.rows, s) : launch_rows<1, 1, 4, 4>(c, p.rows, s);
  }
  if (p.rows <= 16) return launch_rows<1, 2, 2, 4>(c, p.rows, s);
  return p.rows <= 32 ? launch_rows<2, 2, 2, 4>(c, p.rows, s) : launch_rows<4, 2, 2, 4>(c, p.rows, s);
}

}  // namespace qift
