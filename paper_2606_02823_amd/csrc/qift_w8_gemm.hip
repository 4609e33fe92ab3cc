// The 8-bit linear for more than 64 tokens: a tiled product on v_mfma_i32_32x32x32_i8.
#include "qift_w8.h"

namespace qift {
namespace {

using namespace w8;

__device__ __forceinline__ v16i mfma32_i8(v4i a, v4i b, v16i c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

constexpr int kBK = 128;   // k per step: a row of a tile is a line of memory

// slot of 16-byte column c of row r of a tile (8 and 16 consecutive rows spread over the banks)
__device__ __forceinline__ int slot(int r, int c) { return c ^ (((r >> 1) & 7) ^ ((r & 1) << 2)); }

// Tiles of 32 TN GN weight rows x 32 TM GM tokens, a wave to each of the GN x GM parts of TN x TM products.
// Both operands go to LDS without passing registers, a step ahead, in two buffers that are distinct arrays.  The barrier that
// hands a buffer over stands before the last quarter of a step's products: by then the step's operands are in registers, so
// the loads of the step after next go out into its buffer, and the first operands of the next step are read behind the
// remaining products.
// Workgroup z of `parts` takes an even part of the steps; with more than one, the int32 sums go to `y` as [parts][M][N4].
template <int TN, int TM, int GN, int GM, int OT>
__global__ __launch_bounds__(64 * GN * GM) void k_w8_gemm(const int8_t* __restrict__ W, const uint16_t* __restrict__ sw, int64_t N,
                                                          int K, const int8_t* __restrict__ act, const float* __restrict__ sx,
                                                          int64_t M, int tiles_n, int tiles_m, int parts, void* __restrict__ y,
                                                          int32_t* __restrict__ acc_out) {
  constexpr int NW = GN * GM, BN = 32 * TN * GN, BM = 32 * TM * GM;
  constexpr int NA = BN / (8 * NW), NB = BM / (8 * NW);   // direct-to-LDS loads of a wave and step, 8 rows each
  static_assert(NA * 8 * NW == BN && NB * 8 * NW == BM, "whole loads");
  __shared__ __align__(16) int8_t lds_a0[BN * kBK], lds_b0[BM * kBK];
  __shared__ __align__(16) int8_t lds_a1[BN * kBK], lds_b1[BM * kBK];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, h = lane >> 5;
  const int wn = wave / GM, wm = wave - wn * GM;
  // consecutive tiles of one XCD (workgroups go round the 8 XCDs) share weights and tokens in its L2
  int tn, tm, z;
  {
    const int T = tiles_n * tiles_m * parts;
    const int id = blockIdx.x, x = id & 7, base = T >> 3, rem = T & 7;
    int tile = x * base + (x < rem ? x : rem) + (id >> 3);
    z = tile / (tiles_n * tiles_m);
    tile -= z * (tiles_n * tiles_m);
    constexpr int GT = 8;
    const int grp = tile / (GT * tiles_n), first = grp * GT;
    const int width = tiles_m - first < GT ? tiles_m - first : GT;
    const int in = tile - grp * GT * tiles_n;
    tn = in / width;
    tm = first + in - tn * width;
  }
  const int64_t n_base = (int64_t)tn * BN, m_base = (int64_t)tm * BM;
  const int rows_n = (int)(N - n_base < BN ? N - n_base : BN), rows_m = (int)(M - m_base < BM ? M - m_base : BM);
  const int steps = (K + kBK - 1) / kBK;
  const int k_first = (int)((int64_t)steps * z / parts), k_end = (int)((int64_t)steps * (z + 1) / parts);

  const __amdgpu_buffer_rsrc_t wr = dev::make_rsrc(W + n_base * K, (uint32_t)rows_n * (uint32_t)K);
  const __amdgpu_buffer_rsrc_t ar = dev::make_rsrc(act + m_base * K, (uint32_t)rows_m * (uint32_t)K);
  // load q of a wave: rows 8 (NA wave + q) + lane / 8; adding 8 to a row flips column bit 2
  const int lrow = lane >> 3;
  const int col0 = 16 * slot(lrow, lane & 7);
  auto issue = [&](const __amdgpu_buffer_rsrc_t& rs, int count, int rows, int8_t* dst, int q, int kt) {
    const int row = 8 * (count * wave + q) + lrow, col = col0 ^ (64 * ((count * wave + q) & 1));
    const int k = kt * kBK + col;
    const uint32_t off = row < rows && k < K && kt < k_end ? (uint32_t)row * (uint32_t)K + (uint32_t)k : dev::kOutOfRange;
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)(dst + 1024 * (count * wave + q)), 16,
                                             off, 0, 0, 0);
  };
  auto issue_all = [&](int8_t* da, int8_t* db, int kt) {
#pragma unroll
    for (int q = 0; q < NA; ++q) issue(wr, NA, rows_n, da, q, kt);
#pragma unroll
    for (int q = 0; q < NB; ++q) issue(ar, NB, rows_m, db, q, kt);
    __builtin_amdgcn_sched_barrier(0);
  };

  v16i acc[TN][TM];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int t = 0; t < TM; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[j][t][i] = 0;

  int off[4];   // of operand s (values 32 s + 16 h .. of a row)
#pragma unroll
  for (int s = 0; s < 4; ++s) off[s] = r32 * kBK + 16 * slot(r32, 2 * s + h);
  v4i a[2][TN], b[2][TM];
  auto read = [&](const int8_t* ta, const int8_t* tb, int s, int to) {
#pragma unroll
    for (int t = 0; t < TM; ++t) b[to][t] = *reinterpret_cast<const v4i*>(tb + 32 * kBK * (TM * wm + t) + off[s]);
#pragma unroll
    for (int j = 0; j < TN; ++j) a[to][j] = *reinterpret_cast<const v4i*>(ta + 32 * kBK * (TN * wn + j) + off[s]);
  };
  auto products = [&](int from) {
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int i = 0; i < TM; ++i) {
        const int t = j & 1 ? TM - 1 - i : i;   // consecutive products share an operand
        acc[j][t] = mfma32_i8(a[from][j], b[from][t], acc[j][t]);
      }
  };
  auto step = [&](int8_t* ca, int8_t* cb, const int8_t* na, const int8_t* nb, int kt) {
#pragma unroll
    for (int s = 0; s < 3; ++s) {
      read(ca, cb, s + 1, (s + 1) & 1);
      products(s & 1);
      __builtin_amdgcn_sched_barrier(0);
    }
    __builtin_amdgcn_s_waitcnt(0x0070);   // the last operands are here, and the next step's tiles
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    issue_all(ca, cb, kt + 2);
    read(na, nb, 0, 0);
    products(1);
    __builtin_amdgcn_sched_barrier(0);
  };
  issue_all(lds_a0, lds_b0, k_first);
  __builtin_amdgcn_s_waitcnt(0x0070);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  issue_all(lds_a1, lds_b1, k_first + 1);
  read(lds_a0, lds_b0, 0, 0);
  int kt = k_first;
  for (; kt + 1 < k_end; kt += 2) {
    step(lds_a0, lds_b0, lds_a1, lds_b1, kt);
    step(lds_a1, lds_b1, lds_a0, lds_b0, kt + 1);
  }
  if (kt < k_end) step(lds_a0, lds_b0, lds_a1, lds_b1, kt);
  __builtin_amdgcn_s_waitcnt(0x0070);   // the loads past the end have landed before the buffers are used again
  __syncthreads();

  // D of tile (j, t): register 4 q + i of lane (token r32, half h) is row 32 j + 8 q + 4 h + i.  Through the wave's own part
  // of the idle buffers, a token tile at a time: rows of 32 TN outputs in chunks of 16 bytes, chunk c of token m in slot
  // c ^ m, then whole pieces of the rows of y.
  constexpr int SZ = size_of<OT>(), ROW = 32 * TN * SZ, CH = ROW / 16;
  static_assert(32 * ROW * NW <= 2 * (BN + BM) * kBK, "the waves' rows fit the buffers");
  constexpr int PER = BN * kBK / (32 * ROW);   // waves whose rows one of the weight buffers holds
  int8_t* mine;
  {
    constexpr int PB = BM * kBK / (32 * ROW);
    mine = wave < PER              ? lds_a0 + wave * 32 * ROW
           : wave < 2 * PER        ? lds_a1 + (wave - PER) * 32 * ROW
           : wave < 2 * PER + PB   ? lds_b0 + (wave - 2 * PER) * 32 * ROW
                                   : lds_b1 + (wave - 2 * PER - PB) * 32 * ROW;
  }
  const int64_t n_wave = n_base + 32 * TN * wn;
  const int64_t NY = OT == kAcc ? (N + 3) & ~int64_t(3) : N;
  uint8_t* out = static_cast<uint8_t*>(y) + (OT == kAcc ? (int64_t)z * M * NY * 4 : 0);
  const bool whole = NY % (16 / SZ) == 0;
  uint2 swq[TN][4];
#pragma unroll
  for (int j = 0; j < TN; ++j)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      swq[j][q] = OT == kAcc ? make_uint2(0u, 0u) : load_scales(sw, n_wave + 32 * j + 8 * q + 4 * h, N);
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int64_t m0 = m_base + 32 * (TM * wm + t);
    const float s_x = OT == kAcc ? 0.f : m0 + r32 < M ? sx[m0 + r32] : 0.f;
    if (t > 0) __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = 32 * j + 8 * q + 4 * h;
        float s4[4];
        scales4(swq[j][q], s4);
        const int d[4] = {acc[j][t][4 * q], acc[j][t][4 * q + 1], acc[j][t][4 * q + 2], acc[j][t][4 * q + 3]};
        const int at = n * SZ;
        *reinterpret_cast<Quad<OT>*>(mine + r32 * ROW + 16 * ((at >> 4) ^ (r32 & (CH - 1))) + (at & 15)) = quad<OT>(d, s_x, s4);
        if (OT != kAcc && acc_out && m0 + r32 < M && n_wave + n < N)
          store_quad<kAcc>(acc_out, m0 + r32, n_wave + n, N, quad<kAcc>(d, 0.f, s4));
      }
    __builtin_amdgcn_wave_barrier();
    if (whole) {
      constexpr int RI = 64 / CH;   // rows of one store
#pragma unroll
      for (int i = 0; i < 32 / RI; ++i) {
        const int rr = RI * i + lane / CH, c = lane % CH;
        const uint4 v = *reinterpret_cast<const uint4*>(mine + rr * ROW + 16 * (c ^ (rr & (CH - 1))));
        const int64_t m = m0 + rr, n = n_wave + c * (16 / SZ);
        if (m < M && n < NY) *reinterpret_cast<uint4*>(out + (m * NY + n) * SZ) = v;
      }
    } else {
#pragma unroll 4
      for (int i = 0; i < 32 * TN * 32 / 64; ++i) {
        const int rr = (64 * i) / (32 * TN) + (64 > 32 * TN ? lane / (32 * TN) : 0), n = (64 * i + lane) % (32 * TN);
        const int at = n * SZ;
        const int8_t* from = mine + rr * ROW + 16 * ((at >> 4) ^ (rr & (CH - 1))) + (at & 15);
        const int64_t m = m0 + rr;
        if (m < M && n_wave + n < N) {
          if constexpr (SZ == 2)
            *reinterpret_cast<uint16_t*>(out + (m * NY + n_wave + n) * 2) = *reinterpret_cast<const uint16_t*>(from);
          else
            *reinterpret_cast<uint32_t*>(out + (m * NY + n_wave + n) * 4) = *reinterpret_cast<const uint32_t*>(from);
        }
      }
    }
  }
}

// The parts' sums added up (int32: exact in any order), then the scales.
template <int OT>
__global__ __launch_bounds__(256) void k_w8_sum(const int32_t* __restrict__ ws, int parts, const uint16_t* __restrict__ sw,
                                                int64_t N, const float* __restrict__ sx, int64_t M, void* __restrict__ y,
                                                int32_t* __restrict__ acc_out) {
  const int64_t N4 = (N + 3) & ~int64_t(3);
  const int64_t n0 = 4 * ((int64_t)blockIdx.x * 256 + threadIdx.x), m = blockIdx.y;
  if (n0 >= N) return;
  int a[4] = {0, 0, 0, 0};
  for (int z = 0; z < parts; ++z) {
    const int4 v = *reinterpret_cast<const int4*>(ws + ((int64_t)z * M + m) * N4 + n0);
    a[0] += v.x;
    a[1] += v.y;
    a[2] += v.z;
    a[3] += v.w;
  }
  float s4[4];
  scales4(load_scales(sw, n0, N), s4);
  store_quad<OT>(y, m, n0, N, quad<OT>(a, sx[m], s4));
  if (acc_out) store_quad<kAcc>(acc_out, m, n0, N, quad<kAcc>(a, 0.f, s4));
}

template <int TN, int TM, int GN, int GM>
hipError_t launch_tiles(const W8Call& c, int parts, hipStream_t s) {
  constexpr int BN = 32 * TN * GN, BM = 32 * TM * GM;
  const int64_t tn = (c.N + BN - 1) / BN, tm = (c.M + BM - 1) / BM;
  const dim3 grid((unsigned)(tn * tm * parts)), block(64 * GN * GM);
  auto kernel = parts > 1            ? k_w8_gemm<TN, TM, GN, GM, kAcc>
                : c.dtype == kF32    ? k_w8_gemm<TN, TM, GN, GM, kF32>
                : c.dtype == kBF16   ? k_w8_gemm<TN, TM, GN, GM, kBF16>
                                     : k_w8_gemm<TN, TM, GN, GM, kF16>;
  hipLaunchKernelGGL(kernel, grid, block, 0, s, c.levels, c.scales, c.N, (int)c.K, c.act, c.sx, c.M, (int)tn, (int)tm, parts,
                     parts > 1 ? c.ws : c.out, c.acc);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || parts == 1) return e;
  auto sum = c.dtype == kF32 ? k_w8_sum<kF32> : c.dtype == kBF16 ? k_w8_sum<kBF16> : k_w8_sum<kF16>;
  hipLaunchKernelGGL(sum, dim3((unsigned)((c.N + 1023) / 1024), (unsigned)c.M), dim3(256), 0, s, static_cast<const int32_t*>(c.ws),
                     parts, c.scales, c.N, c.sx, c.M, c.out, c.acc);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_w8_gemm(const W8Call& c, const route::W8Plan& p, hipStream_t s) {
  return p.tile == 256 ? launch_tiles<4, 2, 2, 4>(c, p.parts, s) : launch_tiles<2, 2, 2, 2>(c, p.parts, s);
}

}  // namespace qift
