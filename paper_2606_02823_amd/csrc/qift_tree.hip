// Attention of several new tokens per sequence (one token, a chain, a tree of drafts, a chunk of a prompt) over the
// paged KV4 cache:
//   out[row][h] = sum_t p_t v_t,  p = softmax over the tokens the row sees of q . k_t / sqrt(128),
//   k_t = s_t (code - z_t) and v_t likewise.
// A KV head's query rows are its nodes times the G heads of its group.  Workgroup (chunk, KV head and sequence, block of
// rows) takes 16 RT rows over one chunk of tokens; its four waves take every fourth step of 64 tokens each, keep their own
// running maximum, sum of exponentials and output sums in registers, and meet once at the end, so the loop has no
// barrier and a step's codes are unpacked once for all rows.  Chunks of a long sequence are joined by k_tree_merge.
//
// Per step, with c = lane mod 16 and kg = lane / 16:
//   scores   D[token][row] on the f16 MFMA, A = 16 tokens x 32 dimensions of code - z (exact), B = the queries; lane
//            (c, kg) receives tokens 16 j + 4 kg + i (j, i = 0 .. 3) of row c;
//   softmax  in the lane.  What meets the value codes is w_t = p_t s_t, so the reference m of a row is a bound of
//            score + log2 s, not of the score: w = 2^(score + log2 s - m) then fits fp16 whatever the scales are, p = w / s
//            goes into the sum of exponentials, and sum w (code - z) / sum p is the result.  The reference only moves when
//            it is passed by 2^8, so most steps need no reduction across lanes and no rescaling;
//   values   D[dimension][row] += A[dimension][token] B[token][row], B = w as two fp16 parts (2^-21 relative), which the
//            lane holds in place: the contraction's order of tokens is the one the scores left, and the transposing
//            LDS read is given the rows of the lane's own 16 tokens, so no weight crosses lanes.
#include <type_traits>

#include "qift_fwht.h"
#include "qift_internal.h"
#include "qift_kv4_group.h"
#include "qift_pages.h"

namespace qift {
namespace {

using pages::kRound;
using pages::kStep;
using pages::kWaves;

typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));

constexpr float kLowest = -1e30f;   // the reference of a row that has seen nothing: finite, below any score
constexpr float kSlack = 8.f;       // how far, as a power of two, a weight may pass 1 before the reference moves
constexpr float kTop = 7.f;         // w at the reference is 2^kTop, so w < 2^(kSlack + kTop) = 2^15
// A vector of zeros has scale 1 whatever the scales around it, so kLeast stands for it in the reference (and for smaller
// scales: results below 2^-86 may be off).  Its p cannot be had from w, nor those of scales so far from 1 that w leaves
// fp32's range under another token's reference: from the first such token on a wave takes the exponentials of the
// scores too.
constexpr float kLeast = 0x1p-90f, kFar = 0x1p60f;

// x 2^d, also where 2^d alone is no normal number
__device__ __forceinline__ float scaled(float x, float d) {
  const float h = __builtin_amdgcn_exp2f(0.5f * d);
  return x * h * h;
}

struct TreeArgs {
  const uint8_t* kc;
  const float* ks;
  const uint8_t* kz;
  const uint8_t* vc;
  const float* vs;
  const uint8_t* vz;
  const uint16_t* q;
  int64_t q_stride;
  const int32_t* table;
  const int32_t* starts;
  const int32_t* lens;
  const uint64_t* visible;
  uint16_t* out;
  float* part;
  uint32_t* err;
  int64_t records;            // partial records: 128 sums each, then 2 statistics each
  int64_t most;               // tokens a sequence may have: min(max_len, table_pages page)
  pages::Div tiles, group;    // 16-token tiles of a page; heads of a group
  uint32_t pool_pages;
  int32_t Hkv, Hq, G, B, rows, table_pages, max_nodes, words, chunk, chunks, blocks, bf16;
};

// Eight codes of a word less their zero-points, as exact fp16: a code in bits 0-3 of a half under the exponent of
// 1024, one in bits 4-7 under that of 64; then the base, 1024 or 64 plus the zero-point, is subtracted.  Element e is
// nibble kNib[e].
constexpr int kNib[8] = {0, 4, 1, 5, 2, 6, 3, 7};
__device__ __forceinline__ v8h unpack(uint32_t w, v2h b0, v2h b1, v2h b2, v2h b3) {
  const uint32_t w8 = w >> 8;
  const v2h h0 = __builtin_bit_cast(v2h, (w & 0x000F000Fu) | 0x64006400u) - b0;
  const v2h h1 = __builtin_bit_cast(v2h, (w & 0x00F000F0u) | 0x54005400u) - b1;
  const v2h h2 = __builtin_bit_cast(v2h, (w8 & 0x000F000Fu) | 0x64006400u) - b2;
  const v2h h3 = __builtin_bit_cast(v2h, (w8 & 0x00F000F0u) | 0x54005400u) - b3;
  return v8h{h0[0], h0[1], h1[0], h1[1], h2[0], h2[1], h3[0], h3[1]};
}

// Where a wave's token lies: lane l holds the cache row of token t0 + l, 0 for one that is not there.
struct Rows {
  uint32_t row;
  bool ok;
};

// A wave's own staging area, and the area where the waves' sums meet
struct Stage {
  uint32_t v[kStep * kD / 8];   // value codes, 64 bytes a token, 16-byte pieces of row r at piece ^ (r / 16)
  float ks[kStep], ls[kStep], rs[kStep];   // key scale; log2 and reciprocal of the value scale
  uint32_t kz[kStep];           // 1024 + key zero-point as fp16, twice
  _Float16 vz[kStep];           // 1024 (tokens of odd place in their four: 64) + value zero-point, in the order of use
};
constexpr int kPad = kD + 4;
union Lds {
  Stage stage[kWaves];
  float sum[kWaves][16][kPad];
};

__device__ __forceinline__ uint16_t to_bits(float f, int bf16) {
  if (!bf16) return __builtin_bit_cast(uint16_t, (_Float16)f);
  const uint32_t u = __float_as_uint(f);
  return (uint16_t)(f == f ? (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16 : (u >> 16) | 0x40u);
}

template <int RT>
__global__ __launch_bounds__(256) void k_tree(TreeArgs a) {
  __shared__ __attribute__((aligned(16))) Lds lds;
  __shared__ float stat[2][kWaves][16 * RT];   // reference, sum of exponentials
  const int tid = threadIdx.x, lane = tid & 63, c = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // blocks of rows over the same chunk are 8 workgroups apart: one XCD, whose L2 then holds the chunk
  const uint32_t per = 8u * (uint32_t)a.blocks;
  const uint32_t unit = (blockIdx.x / per) * 8 + blockIdx.x % 8, block = (blockIdx.x % per) / 8;
  const uint32_t chunk = unit % (uint32_t)a.chunks, kvb = unit / (uint32_t)a.chunks;
  const int kv = (int)(kvb % (uint32_t)a.Hkv), b = (int)(kvb / (uint32_t)a.Hkv);
  if (b >= a.B) return;
  const pages::Seq sq = pages::sequence(a.starts[b], a.starts[b + 1], a.lens[b], a.rows, a.max_nodes, a.most);
  if (sq.bad && block == 0 && chunk == 0 && kv == 0 && tid == 0) dev::flag_error(a.err, kDevErrIndex);
  const int nrows = sq.n * a.G, r0 = (int)block * 16 * RT;
  if (r0 >= nrows) return;
  const int32_t end = pages::last_token(sq, a.visible != nullptr, a.group, 16 * RT, (int32_t)block);
  const int32_t t_lo = (int32_t)chunk * a.chunk;
  if (t_lo >= end && chunk > 0) return;
  const int32_t t_hi = end - t_lo < a.chunk ? end : t_lo + a.chunk;

  // ---- the queries: B operands, element e of step st is dimension 32 kg + 8 st + kNib[e] of row c
  v8h qb[RT][4];
  float rowf[RT];      // a row's scores as powers of two: raw score times this
  int32_t node[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + 16 * rt + c;
    const bool in = r < nrows;
    const int rr = in ? r : nrows - 1;
    node[rt] = (int32_t)pages::quotient((uint32_t)rr, a.group);
    const int h = kv * a.G + rr - node[rt] * a.G;
    const uint4* src = reinterpret_cast<const uint4*>(a.q + (int64_t)(sq.row0 + node[rt]) * a.q_stride + (int64_t)h * kD + 32 * kg);
    constexpr float unit_score = 0.088388347648318447f * 1.4426950408889634f;   // 1 / sqrt(128), log2 e
    uint4 u[4];
#pragma unroll
    for (int st = 0; st < 4; ++st) u[st] = in ? src[st] : make_uint4(0, 0, 0, 0);
    if (a.bf16) {
      // scaled by a power of two that brings the row's largest into [2^14, 2^15): 8 significant bits stay exact in
      // fp16 down to 2^-28 of it
      float top = 0.f;
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const uint32_t w[4] = {u[st].x, u[st].y, u[st].z, u[st].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) top = fmaxf(top, fabsf(__uint_as_float(e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16)));
      }
      top = fmaxf(top, __shfl_xor(top, 16));
      top = fmaxf(top, __shfl_xor(top, 32));
      const int ex = top > 0.f && top < INFINITY ? 14 - ilogbf(top) : 0;
      rowf[rt] = ldexpf(unit_score, -ex);
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const uint32_t w[4] = {u[st].x, u[st].y, u[st].z, u[st].w};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int n = kNib[e];
          qb[rt][st][e] = (_Float16)ldexpf(__uint_as_float(n & 1 ? w[n >> 1] & 0xFFFF0000u : w[n >> 1] << 16), ex);
        }
      }
    } else {
      rowf[rt] = unit_score;
#pragma unroll
      for (int st = 0; st < 4; ++st) {
        const v8h x = __builtin_bit_cast(v8h, u[st]);
#pragma unroll
        for (int e = 0; e < 8; ++e) qb[rt][st][e] = x[kNib[e]];
      }
    }
  }

  float m[RT], l[RT];
  v4f o[RT][8];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = kLowest;
    l[rt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) o[rt][dt] = v4f{0.f, 0.f, 0.f, 0.f};
  }
  bool direct = false;         // the sum of exponentials is taken of the scores, not of the weights
  Stage& sg = lds.stage[wave];
  const int32_t* table = a.table + (int64_t)b * a.table_pages;
  auto entry = [&](int32_t t0) {   // the table's entry of token t0 + lane (anything for a token that is not there)
    const int32_t t = t0 + lane;
    return table[t < t_hi ? pages::table_index((uint32_t)t, a.tiles) : 0u];
  };
  auto rows_of = [&](int32_t t0, int32_t e) {
    const int32_t t = t0 + lane;
    Rows r;
    r.ok = t < t_hi && (uint32_t)e < a.pool_pages;
    if (t < t_hi && !r.ok) dev::flag_error(a.err, kDevErrIndex);
    r.row = r.ok ? pages::token_row((uint32_t)t, (uint32_t)e, (uint32_t)a.Hkv, (uint32_t)kv, a.tiles) : 0u;
    return r;
  };
  // 16 tokens from row `first` on (a page holds whole tiles of 16, so all of them are rows of the cache)
  auto load_tile = [&](const uint8_t* codes, uint32_t first, int token, int piece) {
    return *reinterpret_cast<const uint4*>(codes + (uint64_t)(first + (uint32_t)token) * (kD / 2) + 16 * piece);
  };

  int32_t t0 = t_lo + wave * kStep;
  uint4 kw[4], vw[4];
  float ksl = 0.f, vsl = 0.f;
  uint32_t kzl = 0, vzl = 0;
  Rows cur{0, false};
  int32_t ahead = 0;           // the next step's table entry
  if (t0 < t_hi) {
    cur = rows_of(t0, entry(t0));
    ahead = entry(t0 + kRound);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)cur.row, 16 * j);
      vw[j] = load_tile(a.vc, first, lane >> 2, lane & 3);
    }
    ksl = a.ks[cur.row];
    vsl = a.vs[cur.row];
    kzl = a.kz[cur.row];
    vzl = a.vz[cur.row];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)cur.row, 16 * j);
      kw[j] = load_tile(a.kc, first, c, kg);
    }
  }

  for (; t0 < t_hi; t0 += kRound) {
    const uint64_t there = __ballot(cur.ok);
    // ---- stage the step's scales, zero-points and value codes (a wave's LDS operations keep their order)
    {
      float v = fmaxf(vsl, kLeast);
      const bool unit = vsl == 1.f && vzl == 0, far = vsl < INFINITY && !(vsl > 1.f / kFar && vsl < kFar);
      if (__any(cur.ok && (unit || far))) {
        // (a lane's token is t0 + lane; load u holds 16 bytes of token 16 u + lane / 4)
        uint32_t codes = 0;
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint64_t held = __ballot((vw[u].x | vw[u].y | vw[u].z | vw[u].w) != 0);
          if (lane >> 4 == u) codes = (uint32_t)(held >> (4 * c)) & 15u;
        }
        const bool zero = unit && codes == 0;
        if (zero) v = kLeast;
        direct |= __any(cur.ok && (zero || far));
      }
      sg.ks[lane] = ksl;
      sg.ls[lane] = __builtin_amdgcn_logf(v);
      sg.rs[lane] = cur.ok && !direct && vsl < INFINITY ? __builtin_amdgcn_rcpf(v) : 0.f;   // (NaN: w is NaN where it is seen)
      const _Float16 kb = (_Float16)(1024.f + (float)kzl);
      const v2h kb2 = {kb, kb};
      sg.kz[lane] = __builtin_bit_cast(uint32_t, kb2);
      // token 16 j + 4 g + i goes to pair i of half j / 2 of lane group g, element j mod 2
      const int tj = lane >> 4, tg = (lane >> 2) & 3, ti = lane & 3;
      sg.vz[tg * 16 + (tj >> 1) * 8 + ti * 2 + (tj & 1)] = (_Float16)((ti & 1 ? 64.f : 1024.f) + (float)vzl);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(&sg.v[(16 * j + (lane >> 2)) * (kD / 8) + 4 * ((lane & 3) ^ j)]) = vw[j];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // ---- the next step's loads, its key codes after this step's are used
    const int32_t tn = t0 + kRound;
    Rows nxt{0, false};
    if (tn < t_hi) {
      nxt = rows_of(tn, ahead);
      ahead = entry(tn + kRound);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)nxt.row, 16 * j);
        vw[j] = load_tile(a.vc, first, lane >> 2, lane & 3);
      }
      ksl = a.ks[nxt.row];
      vsl = a.vs[nxt.row];
      kzl = a.kz[nxt.row];
      vzl = a.vz[nxt.row];
    }
    // ---- scores
    v4f sc[RT][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const v2h b10 = __builtin_bit_cast(v2h, sg.kz[16 * j + c]);
      const v2h b6 = b10 - v2h{(_Float16)960.f, (_Float16)960.f};
      const uint32_t w[4] = {kw[j].x, kw[j].y, kw[j].z, kw[j].w};
      v8h ka[4];
#pragma unroll
      for (int st = 0; st < 4; ++st) ka[st] = unpack(w[st], b10, b6, b10, b6);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        v4f acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int st = 0; st < 4; ++st) acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(ka[st], qb[rt][st], acc, 0, 0, 0);
        sc[rt][j] = acc;
      }
    }
    if (tn < t_hi) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t first = (uint32_t)__builtin_amdgcn_readlane((int)nxt.row, 16 * j);
        kw[j] = load_tile(a.kc, first, c, kg);
      }
    }
    // ---- softmax: weights p s as two fp16 parts, B operands of the value phase
    v8h ahi[RT][2], alo[RT][2];
    auto softmax = [&](auto masked) {
      constexpr bool kMasked = decltype(masked)::value;
      v4f k4[4], l4[4], r4[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        k4[j] = *reinterpret_cast<const v4f*>(&sg.ks[16 * j + 4 * kg]);
        l4[j] = *reinterpret_cast<const v4f*>(&sg.ls[16 * j + 4 * kg]);
        r4[j] = *reinterpret_cast<const v4f*>(&sg.rs[16 * j + 4 * kg]);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        uint32_t seen[2] = {0, 0};   // bits 16 (j mod 2) + i of word j / 2: token 16 j + 4 kg + i
        if constexpr (kMasked) {
          uint64_t bits;
          if (a.visible) {
            const int32_t d0 = t0 - sq.ctx;
            uint64_t w0 = 0, w1 = 0;
            const int32_t k0 = d0 > 0 ? d0 >> 6 : 0;
            if (d0 > -64) {
              const uint64_t* row = a.visible + (int64_t)(sq.row0 + node[rt]) * a.words;
              if (k0 < a.words) w0 = row[k0];
              if (k0 + 1 < a.words) w1 = row[k0 + 1];
            }
            bits = pages::tree_bits(d0, w0, w1);
          } else {
            bits = pages::chain_bits(t0, sq.ctx, node[rt]);
          }
          bits = (bits & there) >> (4 * kg);
          seen[0] = (uint32_t)bits;
          seen[1] = (uint32_t)(bits >> 32);
        }
        float y[16], top = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v = fmaf(sc[rt][j][i] * k4[j][i], rowf[rt], l4[j][i]);
            if constexpr (kMasked) v = (seen[j >> 1] >> (16 * (j & 1) + i)) & 1u ? v : -INFINITY;
            y[4 * j + i] = v;
          }
#pragma unroll
        for (int e = 0; e < 16; ++e) top = fmaxf(top, y[e]);
        if (__any(top > m[rt] + (kTop + kSlack))) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float mn = fmaxf(m[rt], top - kTop), f = __builtin_amdgcn_exp2f(m[rt] - mn);
          l[rt] = scaled(l[rt], m[rt] - mn);
          m[rt] = mn;
#pragma unroll
          for (int dt = 0; dt < 8; ++dt) o[rt][dt] *= f;
        }
        float w[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          w[e] = __builtin_amdgcn_exp2f(y[e] - m[rt]);
          l[rt] = fmaf(w[e], r4[e >> 2][e & 3], l[rt]);
        }
        if constexpr (kMasked) {
          if (direct) {
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const float d = fmaf(sc[rt][e >> 2][e & 3] * k4[e >> 2][e & 3], rowf[rt], -m[rt]);
              l[rt] += (seen[e >> 3] >> (16 * ((e >> 2) & 1) + (e & 3))) & 1u ? __builtin_amdgcn_exp2f(d) : 0.f;
            }
          }
        }
        // half h, pair i: tokens 16 (2 h) + 4 kg + i and 16 (2 h + 1) + 4 kg + i
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float x = w[8 * h + i], z = w[8 * h + 4 + i];
            const v2h hi = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_pkrtz(x, z));
            const v2h lo = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_pkrtz(x - (float)hi[0], z - (float)hi[1]));
            ahi[rt][h][2 * i] = hi[0];
            ahi[rt][h][2 * i + 1] = hi[1];
            alo[rt][h][2 * i] = lo[0];
            alo[rt][h][2 * i + 1] = lo[1];
          }
      }
    };
    if (direct || there != ~uint64_t(0) || t0 + kStep > sq.ctx) softmax(std::integral_constant<bool, true>{});
    else softmax(std::integral_constant<bool, false>{});
    // ---- values: A = 16 dimensions x 32 tokens of code - z.  The transposing read hands lane (c, kg) the 16 codes of
    // dimension 16 dt + c whose rows the 16 lanes of its group name: token 16 (c / 4) + 4 kg + c mod 4, nibble c.
    {
      v2h bz[2][4];
      const uint4* z4 = reinterpret_cast<const uint4*>(&sg.vz[16 * kg]);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const uint4 z = z4[h];
        bz[h][0] = __builtin_bit_cast(v2h, z.x);
        bz[h][1] = __builtin_bit_cast(v2h, z.y);
        bz[h][2] = __builtin_bit_cast(v2h, z.z);
        bz[h][3] = __builtin_bit_cast(v2h, z.w);
      }
      const int row = 16 * (c >> 2) + 4 * kg + (c & 3);
#pragma unroll
      for (int dt = 0; dt < 8; ++dt) {
        const int off = row * (kD / 8) + 4 * ((dt >> 1) ^ (c >> 2)) + 2 * (dt & 1);
        const v2i t = __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) v2i*)(sg.v + off));
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const v8h va = unpack(h ? (uint32_t)t.y : (uint32_t)t.x, bz[h][0], bz[h][1], bz[h][2], bz[h][3]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, ahi[rt][h], o[rt][dt], 0, 0, 0);
            o[rt][dt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va, alo[rt][h], o[rt][dt], 0, 0, 0);
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    cur = nxt;
  }

  // ---- the four waves' sums meet under a common reference
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] += __shfl_xor(l[rt], 16);
    l[rt] += __shfl_xor(l[rt], 32);
    if (kg == 0) {
      stat[0][wave][16 * rt + c] = m[rt];
      stat[1][wave][16 * rt + c] = l[rt];
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    __syncthreads();   // the staging areas, or the last tile's sums, are no longer read
    float M = stat[0][0][16 * rt + c];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, stat[0][w][16 * rt + c]);
    const float f = __builtin_amdgcn_exp2f(m[rt] - M);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<v4f*>(&lds.sum[wave][c][16 * dt + 4 * kg]) = o[rt][dt] * f;
    __syncthreads();
    const int row = tid >> 4, d0 = (tid & 15) * 8, r = r0 + 16 * rt + row;
    float Mr = stat[0][0][16 * rt + row], L = 0.f;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) Mr = fmaxf(Mr, stat[0][w][16 * rt + row]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) L += scaled(stat[1][w][16 * rt + row], stat[0][w][16 * rt + row] - Mr);
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      v4f x = *reinterpret_cast<const v4f*>(&lds.sum[0][row][d0 + e]);
#pragma unroll
      for (int w = 1; w < kWaves; ++w) x += *reinterpret_cast<const v4f*>(&lds.sum[w][row][d0 + e]);
      s[e] = x[0];
      s[e + 1] = x[1];
      s[e + 2] = x[2];
      s[e + 3] = x[3];
    }
    if (r < nrows) {
      if (a.chunks == 1) {
        const int nd = (int)pages::quotient((uint32_t)r, a.group);
        const float inv = L == 0.f ? 0.f : 1.f / L;   // a row that sees nothing: 0
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = (uint32_t)to_bits(s[2 * e] * inv, a.bf16) | ((uint32_t)to_bits(s[2 * e + 1] * inv, a.bf16) << 16);
        uint16_t* y = a.out + ((int64_t)(sq.row0 + nd) * a.Hq + kv * a.G + (r - nd * a.G)) * kD + d0;
        *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        const int64_t rec = (((int64_t)b * a.Hkv + kv) * a.chunks + chunk) * ((int64_t)a.max_nodes * a.G) + r;
        float* y = a.part + rec * kD + d0;
        *reinterpret_cast<float4*>(y) = make_float4(s[0], s[1], s[2], s[3]);
        *reinterpret_cast<float4*>(y + 4) = make_float4(s[4], s[5], s[6], s[7]);
        if (d0 == 0) {
          a.part[a.records * kD + 2 * rec] = Mr;
          a.part[a.records * kD + 2 * rec + 1] = L;
        }
      }
    }
  }
}

// out = sum_c 2^(m_c - M) sums_c / sum_c 2^(m_c - M) l_c over the chunks c of a row's sequence.  32 lanes of four
// dimensions take a row, or `slices` times 32 lanes share its chunks.
__global__ __launch_bounds__(256) void k_tree_merge(TreeArgs a, int32_t block_rows, int32_t slices) {
  __shared__ v4f sum[8][32];
  const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
  const int kv = blockIdx.y, b = blockIdx.z;
  const pages::Seq sq = pages::sequence(a.starts[b], a.starts[b + 1], a.lens[b], a.rows, a.max_nodes, a.most);
  const int nrows = sq.n * a.G, first = (int)blockIdx.x * (8 / slices);
  if (first >= nrows) return;
  const int r = first + slot / slices, slice = slot % slices;
  const bool in = r < nrows;
  v4f acc = {0.f, 0.f, 0.f, 0.f};
  float L = 0.f;
  if (in) {
    const int32_t end = pages::last_token(sq, a.visible != nullptr, a.group, block_rows, r / block_rows);
    const int32_t n = (end + a.chunk - 1) / a.chunk;
    const int64_t R = (int64_t)a.max_nodes * a.G, rec = ((int64_t)b * a.Hkv + kv) * a.chunks * R + r;
    const float* st = a.part + a.records * kD + 2 * rec;
    float M = kLowest;
    for (int32_t i = lane; i < n; i += 32) M = fmaxf(M, st[2 * R * i]);
#pragma unroll
    for (int d = 16; d; d >>= 1) M = fmaxf(M, __shfl_xor(M, d));
    for (int32_t i = lane; i < n; i += 32) L += scaled(st[2 * R * i + 1], st[2 * R * i] - M);
#pragma unroll
    for (int d = 16; d; d >>= 1) L += __shfl_xor(L, d);
    const float* y = a.part + rec * kD + 4 * lane;
#pragma unroll 4
    for (int32_t i = slice; i < n; i += slices) {
      const float f = __builtin_amdgcn_exp2f(st[2 * R * i] - M);
      acc += *reinterpret_cast<const v4f*>(y + R * kD * i) * f;
    }
  }
  if (slices > 1) {
    sum[slot][lane] = acc;
    __syncthreads();
    if (slice) return;
    for (int s = 1; s < slices; ++s) acc += sum[slot + s][lane];
  }
  if (!in) return;
  const int nd = (int)pages::quotient((uint32_t)r, a.group);
  const float inv = L == 0.f ? 0.f : 1.f / L;
  uint2 w;
  w.x = (uint32_t)to_bits(acc[0] * inv, a.bf16) | ((uint32_t)to_bits(acc[1] * inv, a.bf16) << 16);
  w.y = (uint32_t)to_bits(acc[2] * inv, a.bf16) | ((uint32_t)to_bits(acc[3] * inv, a.bf16) << 16);
  *reinterpret_cast<uint2*>(a.out + ((int64_t)(sq.row0 + nd) * a.Hq + kv * a.G + (r - nd * a.G)) * kD + 4 * lane) = w;
}

}  // namespace

hipError_t launch_kv4_tree(const TreeCall& t, hipStream_t s) {
  const Kv4Pool& c = t.c;
  const int32_t G = t.Hq / c.Hkv;
  const pages::Plan p = pages::plan(t.B, c.Hkv, G, t.max_nodes, t.max_len);
  TreeArgs a;
  a.kc = c.kc;
  a.ks = c.ks;
  a.kz = c.kz;
  a.vc = c.vc;
  a.vs = c.vs;
  a.vz = c.vz;
  a.q = t.q;
  a.q_stride = t.q_stride;
  a.table = t.table;
  a.starts = t.starts;
  a.lens = t.lens;
  a.visible = t.visible;
  a.out = t.out;
  a.part = t.ws;
  a.err = device_error_word();
  a.records = pages::records(p, t.B, c.Hkv, G, t.max_nodes);
  const int64_t room = (int64_t)t.table_pages * c.page;
  a.most = t.max_len < room ? t.max_len : room;
  a.tiles = pages::make_div((uint32_t)c.page / 16);
  a.group = pages::make_div((uint32_t)G);
  a.pool_pages = (uint32_t)c.pages;
  a.Hkv = c.Hkv;
  a.Hq = t.Hq;
  a.G = G;
  a.B = (int32_t)t.B;
  a.rows = (int32_t)t.rows;
  a.table_pages = t.table_pages;
  a.max_nodes = t.max_nodes;
  a.words = (t.max_nodes + 63) / 64;
  a.chunk = p.chunk;
  a.chunks = p.chunks;
  a.blocks = p.blocks;
  a.bf16 = t.dtype == kBF16;
  const int64_t units = (t.B * c.Hkv * p.chunks + 7) / 8 * 8;
  const dim3 grid((unsigned)(units * p.blocks));
  auto kernel = p.rt == 1 ? k_tree<1> : k_tree<2>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.chunks == 1) return e;
  // rows of many chunks are shared by 8 slices, of few by 2
  const int32_t slices = p.chunks > 16 ? 8 : p.chunks > 4 ? 4 : 2;
  const int64_t R = (int64_t)t.max_nodes * G;
  const dim3 mgrid((unsigned)((R * slices + 7) / 8), (unsigned)c.Hkv, (unsigned)t.B);
  hipLaunchKernelGGL(k_tree_merge, mgrid, dim3(256), 0, s, a, 16 * p.rt, slices);
  return hipGetLastError();
}

}  // namespace qift
