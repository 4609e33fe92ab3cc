// The 8-bit linear for prompts, for wide linears and for more than 32 tokens: a tiled product on v_mfma_i32_32x32x32_i8.
#include <utility>

#include "qift_w8.h"
#include "qift_waits.h"

namespace qift {
namespace {

using namespace w8;

__device__ __forceinline__ v16i mfma32_i8(v4i a, v4i b, v16i c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
}

// (a lambda that is not inlined early keeps what it refers to in memory)
#define QIFT_INLINE __attribute__((always_inline))

// f(0), f(1), .. with constants, so that every index is one
template <int... I, typename F>
__device__ __forceinline__ void each(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each(std::make_integer_sequence<int, N>(), f);
}
template <int V>
using Const = std::integral_constant<int, V>;

constexpr int kBK = 128;   // k per step: a row of a tile is a line of memory

// slot of 16-byte column c of row r of a tile (8 and 16 consecutive rows spread over the banks)
__device__ __forceinline__ int slot(int r, int c) { return c ^ (((r >> 1) & 7) ^ ((r & 1) << 2)); }

// Tiles of 32 TN GN weight rows x 32 TM GM tokens, a wave to each of the GN x GM parts of TN x TM products.
// Both operands go to LDS without passing registers, NS - 1 steps ahead, in NS buffers that are distinct arrays (so that the
// compiler sees that loads into one never alias reads from another, and adds no waits).  The barrier that hands a buffer over
// stands before the last quarter of a step's products: by then the step's operands are in registers, so the loads of step
// k + NS go out into its buffer, and the first operands of the next step are read between the remaining products.
// What bounds the largest tiles is the chip's power: the matrix units are busy 68 % of the time at 1.56 GHz (28672 x 4096 at
// 4096 tokens, 411 to 445 us from card to card, 2.2 to 2.3 POP/s; the library's 8192 x 8192 x 8192 2.42 to 2.55, this one at 4096
// tokens 2.53).  Of the 411 us 50 go into storing the outputs, 54 are lost to the loads and 26 to the reads of LDS.  The
// smaller tiles are bound by the bytes that a CU takes into LDS (2500 x 4096 at 600 tokens 15 us, 4096 x 11008 at 333 in five
// parts 32) or, with few tokens, by the weights' bytes (32003 x 4096 at 61 tokens 31 us, 4.2 TB/s).
// Workgroup z of `parts` takes an even part of the steps; with more than one, the int32 sums go to `y` as [parts][M][N4].
template <int TN, int TM, int GN, int GM, int NS, int OT>
__global__ __launch_bounds__(64 * GN * GM) void k_w8_gemm(const int8_t* __restrict__ W, const uint16_t* __restrict__ sw, int64_t N,
                                                          int K, const int8_t* __restrict__ act, const float* __restrict__ sx,
                                                          int64_t M, int tiles_n, int tiles_m, int parts, void* __restrict__ y,
                                                          int32_t* __restrict__ acc_out) {
  constexpr int NW = GN * GM, BN = 32 * TN * GN, BM = 32 * TM * GM;
  constexpr int NA = BN / (8 * NW), NB = BM / (8 * NW);   // direct-to-LDS loads of a wave and step, 8 rows each
  static_assert(NA * 8 * NW == BN && NB * 8 * NW == BM, "whole loads");
  static_assert((NS == 2 || NS == 3) && waits::w8_prologue(NS, NA + NB) < 64, "buffers, and six bits of vmcnt");
  __shared__ __align__(16) int8_t lds0[(BN + BM) * kBK];
  __shared__ __align__(16) int8_t lds1[(BN + BM) * kBK];
  __shared__ __align__(16) int8_t lds2[NS > 2 ? (BN + BM) * kBK : 16];
  __shared__ __align__(16) float s_sx[BM];
  __shared__ __align__(16) uint16_t s_sw[BN];
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
  const int k_first = steps * z / parts, k_end = steps * (z + 1) / parts;   // (at most 1024 steps and parts)

  const __amdgpu_buffer_rsrc_t wr = dev::make_rsrc(W + n_base * K, (uint32_t)rows_n * (uint32_t)K);
  const __amdgpu_buffer_rsrc_t ar = dev::make_rsrc(act + m_base * K, (uint32_t)rows_m * (uint32_t)K);
  // load q of a wave: rows 8 (NA wave + q) + lane / 8; adding 8 to a row flips column bit 2
  const int lrow = lane >> 3, col0 = 16 * slot(lrow, lane & 7);
  uint32_t at_a[NA], at_b[NB];
#pragma unroll
  for (int q = 0; q < NA; ++q) {
    const int p = NA * wave + q, row = 8 * p + lrow;
    at_a[q] = row < rows_n ? (uint32_t)row * (uint32_t)K + (uint32_t)(col0 ^ (64 * (p & 1))) : dev::kOutOfRange;
  }
#pragma unroll
  for (int q = 0; q < NB; ++q) {
    const int p = NB * wave + q, row = 8 * p + lrow;
    at_b[q] = row < rows_m ? (uint32_t)row * (uint32_t)K + (uint32_t)(col0 ^ (64 * (p & 1))) : dev::kOutOfRange;
  }
  auto send = [&](const __amdgpu_buffer_rsrc_t& rs, int8_t* dst, uint32_t from) QIFT_INLINE {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (__attribute__((address_space(3))) void*)dst, 16, from, 0, 0, 0);
  };
  const int k_stop = k_end * kBK < K ? k_end * kBK : K;
  // load i of a step: the weights' first, then the tokens'
  auto issue = [&](int8_t* dst, int k, auto i) QIFT_INLINE {
    constexpr bool weights = i < NA;
    const int p = weights ? NA * wave + i : NB * wave + i - NA;
    const bool in = k + (col0 ^ (64 * (p & 1))) < k_stop;
    if constexpr (weights) send(wr, dst + 1024 * p, in ? at_a[i] + (uint32_t)k : dev::kOutOfRange);
    else send(ar, dst + BN * kBK + 1024 * p, in ? at_b[i - NA] + (uint32_t)k : dev::kOutOfRange);
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
  // operand i of quarter s into register set `to`: the tokens' first, then the weights'
  auto read = [&](const int8_t* tile, auto s, auto to, auto i) QIFT_INLINE {
    if constexpr (i < TM) b[to][i] = *reinterpret_cast<const v4i*>(tile + BN * kBK + 32 * kBK * (TM * wm + i) + off[s]);
    else a[to][i - TM] = *reinterpret_cast<const v4i*>(tile + 32 * kBK * (TN * wn + i - TM) + off[s]);
  };
  constexpr int NP = TN * TM, NR = TN + TM, NL = NA + NB;   // products and operands of a quarter, loads of a step
  auto product = [&](auto from, auto i) QIFT_INLINE {
    constexpr int j = i / TM, t = j & 1 ? TM - 1 - i % TM : i % TM;   // consecutive products share an operand
    acc[j][t] = mfma32_i8(a[from][j], b[from][t], acc[j][t]);
  };
  // the products from number i0 on of the quarter in register set `from`, the reads of quarter s of `tile` into the other set
  // and the loads l0 .. l1 - 1 of the step at k spread between them
  auto quarter = [&](const int8_t* tile, auto s, auto from, auto i0, int8_t* dst, int k, auto l0, auto l1) QIFT_INLINE {
    each<NP - i0>([&](auto i) QIFT_INLINE {
      each<l1 - l0>([&](auto l) QIFT_INLINE {
        if constexpr (l * (NP - i0) / (l1 - l0) == i) issue(dst, k, Const<l0 + l>());
      });
      each<NR>([&](auto r) QIFT_INLINE {
        if constexpr (r * (NP - i0) / NR == i) read(tile, s, Const<1 - from>(), r);
      });
      product(from, Const<i0 + i>());
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  constexpr int FIRST = waits::w8_first(NL);   // loads that go out with the last quarter; the others with the next step's first
  // `last` is the buffer that the step before handed over
  auto step = [&](int8_t* cur, int8_t* nxt, int8_t* last, int kt) QIFT_INLINE {
    quarter(cur, Const<1>(), Const<0>(), Const<0>(), last, (kt - 1 + NS) * kBK, Const<FIRST>(), Const<NL>());
    quarter(cur, Const<2>(), Const<1>(), Const<0>(), last, 0, Const<0>(), Const<0>());
    quarter(cur, Const<3>(), Const<0>(), Const<0>(), last, 0, Const<0>(), Const<0>());
    __builtin_amdgcn_s_waitcnt(waits::encode(waits::w8_handover(NS, NL), true));   // the last operands, the next step's tiles
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    quarter(nxt, Const<0>(), Const<1>(), Const<0>(), cur, (kt + NS) * kBK, Const<0>(), Const<FIRST>());
  };
  // the tile's scales for the end (their loads go out before the tiles')
  static_assert(BN <= 64 * NW && BM <= 64 * NW, "a scale to a thread");
  float sx_pre = 0.f;
  uint16_t sw_pre = 0;
  if constexpr (OT != kAcc) {
    if (tid < rows_m) sx_pre = sx[m_base + tid];
    if (tid < rows_n) sw_pre = sw[n_base + tid];
  }
  __builtin_amdgcn_sched_barrier(0);
  int8_t* const lds_last = NS == 2 ? lds1 : lds2;
  each<NL>([&](auto i) QIFT_INLINE { issue(lds0, k_first * kBK, i); });
  if constexpr (NS > 2) each<NL>([&](auto i) QIFT_INLINE { issue(lds1, (k_first + 1) * kBK, i); });
  each<FIRST>([&](auto i) QIFT_INLINE { issue(lds_last, (k_first + NS - 1) * kBK, i); });
  __builtin_amdgcn_sched_barrier(0);
  if constexpr (OT != kAcc) {
    if (tid < BM) s_sx[tid] = sx_pre;
    if (tid < BN) s_sw[tid] = sw_pre;
  }
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(waits::encode(waits::w8_prologue(NS, NL), true));
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
  each<NR>([&](auto r) QIFT_INLINE { read(lds0, Const<0>(), Const<0>(), r); });
  // (steps past k_end, up to a whole round of the buffers, work on zeros)
  for (int kt = k_first; kt < k_end; kt += NS) {
    step(lds0, lds1, lds_last, kt);
    if constexpr (NS == 2) {
      step(lds1, lds0, lds0, kt + 1);
    } else {
      step(lds1, lds2, lds0, kt + 1);
      step(lds2, lds0, lds1, kt + 2);
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0070);   // the loads past the end have landed before the buffers are used again
  __syncthreads();

  // D of tile (j, t): register 4 q + i of lane (token r32, half h) is row 32 j + 8 q + 4 h + i.  Through the wave's own part
  // of the idle buffers, a token tile at a time: rows of 32 TN outputs in chunks of 16 bytes, chunk c of token m in slot
  // c ^ m, then 16-byte pieces of the rows of y, which begin at any place where N is no multiple of 8 (28671 x 4096 at 4096 tokens
  // 424 us; value by value 460).
  constexpr int SZ = size_of<OT>(), ROW = 32 * TN * SZ, CH = ROW / 16;
  constexpr int PER = (BN + BM) * kBK / (32 * ROW);   // waves whose rows one of the buffers holds
  static_assert(PER * NS >= NW, "the waves' rows fit the buffers");
  int8_t* const mine = (wave < PER ? lds0 : wave < 2 * PER ? lds1 : lds2) + wave % PER * (32 * ROW);
  const int64_t n_wave = n_base + 32 * TN * wn;
  const int64_t NY = OT == kAcc ? (N + 3) & ~int64_t(3) : N;
  constexpr int E = 16 / SZ;
  const int have = NY - n_wave > 32 * TN ? 32 * TN : NY > n_wave ? (int)(NY - n_wave) : 0, last = have / E * E, rest = have - last;
  uint8_t* out = static_cast<uint8_t*>(y) + (OT == kAcc ? (int64_t)z * M * NY * 4 : 0);
#pragma unroll
  for (int t = 0; t < TM; ++t) {
    const int64_t m0 = m_base + 32 * (TM * wm + t);
    const float s_x = OT == kAcc ? 0.f : s_sx[32 * (TM * wm + t) + r32];
    if (t > 0) __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < TN; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = 32 * j + 8 * q + 4 * h;
        float s4[4];
        scales4(OT == kAcc ? make_uint2(0u, 0u) : *reinterpret_cast<const uint2*>(s_sw + 32 * TN * wn + n), s4);
        const int d[4] = {acc[j][t][4 * q], acc[j][t][4 * q + 1], acc[j][t][4 * q + 2], acc[j][t][4 * q + 3]};
        const int at = n * SZ;
        *reinterpret_cast<Quad<OT>*>(mine + r32 * ROW + 16 * ((at >> 4) ^ (r32 & (CH - 1))) + (at & 15)) = quad<OT>(d, s_x, s4);
        if (OT != kAcc && acc_out && m0 + r32 < M && n_wave + n < N)
          store_row<kAcc>(acc_out, m0 + r32, n_wave + n, N, quad<kAcc>(d, 0.f, s4));
      }
    __builtin_amdgcn_wave_barrier();
    constexpr int RI = 64 / CH;   // rows of one store
#pragma unroll
    for (int i = 0; i < 32 / RI; ++i) {
      const int rr = RI * i + lane / CH, c = lane % CH;
      const uint4 v = *reinterpret_cast<const uint4*>(mine + rr * ROW + 16 * (c ^ (rr & (CH - 1))));
      const int64_t m = m0 + rr, n = n_wave + c * (16 / SZ);
      if (m < M && n + E <= NY) store_words(out + (m * NY + n) * SZ, v);
    }
    if (rest > 0) {   // the values of the last row of weights' piece that do not fill 16 bytes
#pragma unroll 1
      for (int i = 0; i < 32 * E / 64; ++i) {
        const int rr = (64 * i + lane) / E, n = last + (64 * i + lane) % E, place = n * SZ;
        const int8_t* from = mine + rr * ROW + 16 * ((place >> 4) ^ (rr & (CH - 1))) + (place & 15);
        if (m0 + rr < M && (64 * i + lane) % E < rest) {
          uint8_t* to = out + ((m0 + rr) * NY + n_wave + n) * SZ;
          if constexpr (SZ == 2) *reinterpret_cast<uint16_t*>(to) = *reinterpret_cast<const uint16_t*>(from);
          else *reinterpret_cast<uint32_t*>(to) = *reinterpret_cast<const uint32_t*>(from);
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
  for (int z0 = 0; z0 < parts; z0 += 4) {   // four parts' loads at once (one past the last: the last again, not added)
    int4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int z = z0 + i < parts ? z0 + i : parts - 1;
      v[i] = *reinterpret_cast<const int4*>(ws + ((int64_t)z * M + m) * N4 + n0);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (z0 + i < parts) {
        a[0] += v[i].x;
        a[1] += v[i].y;
        a[2] += v[i].z;
        a[3] += v[i].w;
      }
  }
  float s4[4];
  scales4(load_scales(sw, n0, N), s4);
  store_row<OT>(y, m, n0, N, quad<OT>(a, sx[m], s4));
  if (acc_out) store_row<kAcc>(acc_out, m, n0, N, quad<kAcc>(a, 0.f, s4));
}

template <int TN, int TM, int GN, int GM, int NS>
hipError_t launch_tiles(const W8Call& c, int parts, hipStream_t s) {
  constexpr int BN = 32 * TN * GN, BM = 32 * TM * GM;
  const int64_t tn = (c.N + BN - 1) / BN, tm = (c.M + BM - 1) / BM;
  const dim3 grid((unsigned)(tn * tm * parts)), block(64 * GN * GM);
  auto kernel = parts > 1            ? k_w8_gemm<TN, TM, GN, GM, NS, kAcc>
                : c.dtype == kF32    ? k_w8_gemm<TN, TM, GN, GM, NS, kF32>
                : c.dtype == kBF16   ? k_w8_gemm<TN, TM, GN, GM, NS, kBF16>
                                     : k_w8_gemm<TN, TM, GN, GM, NS, kF16>;
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
  if (p.bm == 256) return launch_tiles<4, 2, 2, 4, 2>(c, p.parts, s);
  if (p.bm == 128) return launch_tiles<2, 2, 4, 2, 3>(c, p.parts, s);
  return p.bm == 64 ? launch_tiles<1, 1, 4, 2, 3>(c, p.parts, s) : launch_tiles<1, 1, 4, 1, 3>(c, p.parts, s);
}

}  // namespace qift
