// Attention of several new tokens per sequence (one token, a chain, a tree of drafts, a chunk of a prompt) over the
// paged KV4 cache:
//   out[row][h] = sum_t p_t v_t,  p = softmax over the tokens the row sees of q . k_t / sqrt(128),
//   k_t = s_t (code - z_t) and v_t likewise.
// A KV head's query rows are its nodes times the G heads of its group.  A workgroup takes 16 RT rows over a run of tokens
// of one sequence; its four waves take every fourth step of 64 tokens each, keep their own reference, sum of
// exponentials and output sums in registers, and meet once at the run's end, so the loop has no barrier and a step's
// codes are unpacked once for all rows.  The runs are even shares of all sequences' tokens (pages::Plan); those of one
// sequence are joined by k_tree_merge.
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
typedef _Float16 v4h __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

constexpr float kLowest = -0x1.fffffep127f;   // the reference of a row that has seen nothing: no finite score is below it
constexpr float kSlack = 8.f;       // how far, as a power of two, a weight may pass 1 before the reference moves
constexpr float kTop = 7.f;         // w at the reference is 2^kTop, so w < 2^(kSlack + kTop) = 2^15
// A vector of zeros has scale 1 whatever the scales around it, so kLeast stands for it in the reference (and for smaller
// scales: results below 2^-86 may be off).  Its w may then leave fp32's range where its p counts, and so may those of
// scales far from 1 under another token's reference (within [2^-50, 2^50] a p that is lost so is 2^-33 of another at most):
// from the first such token on a wave takes the p of a w that is 0 from the score.
constexpr float kLeast = 0x1p-90f, kFar = 0x1p50f;

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
  int64_t records;            // partial records times rows: 128 sums each, then 2 statistics each
  int64_t most;               // tokens a sequence may have: min(max_len, table_pages page)
  pages::Div tiles, group;    // 16-token tiles of a page; heads of a group
  uint32_t pool_pages;
  int32_t Hkv, Hq, G, B, rows, table_pages, max_nodes, words, shares, blocks, bf16;
};

// The kernel's arguments in constant memory, read where they are used: held in scalar registers from the start they
// would not leave the loop enough of those, and what does not fit takes vector registers.
typedef const __attribute__((address_space(4))) TreeArgs* ArgPtr;
__device__ __forceinline__ ArgPtr arguments() {
  uint64_t p = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));   // (another read is another value to the compiler)
  return (ArgPtr)p;
}
__device__ __forceinline__ pages::Div group_of(ArgPtr a) { return {a->group.d, a->group.m, a->group.s}; }
__device__ __forceinline__ pages::Div tiles_of(ArgPtr a) { return {a->tiles.d, a->tiles.m, a->tiles.s}; }

// The thread's number as a new value: what is computed from it stays where it is computed, instead of being carried in
// registers from the start of the kernel through its loops.
__device__ __forceinline__ int thread_again() {
  int t = threadIdx.x;
  asm volatile("" : "+v"(t));
  return t;
}

// Eight codes of a word less their zero-points, as exact fp16 operands: a code in bits 0-3 of a half under the exponent of
// 1024 is 1024 + code, one in bits 4-7 under that of 64 is 64 + code; then the base, 1024 or 64 plus the zero-point (exact for
// every byte), is subtracted.  Left in the operands, with its share taken from the sums by one more product, the base would
// save two of these nine instructions a word (16 trees of 64 nodes 264 us, then 255; chains of 5 for 16 sequences 37.3, 35.9;
// 32 ragged sequences 43.9, 42.0), but the sums would be of 64 to 79 times the weights and round as such: up to 2^-9 of the
// largest value was lost so over 65536 tokens whose first have nearly all of the weight.  Codes as subnormal numbers in a
// half's lowest bits would take five instructions, but the matrix instructions sum products of subnormals with errors up to
// 2^-17 of them.  Element e is nibble kNib[e].
constexpr int kNib[8] = {0, 4, 1, 5, 2, 6, 3, 7};
// Masks and exponents as register values the compiler knows nothing of: with literals it takes an and and an or for each
// pair of codes, from registers the one instruction that does both.
struct Bits {
  uint32_t m0, m1, e10, e6;
};
__device__ __forceinline__ Bits code_bits() {
  Bits k = {0x000F000Fu, 0x00F000F0u, 0x64006400u, 0x54005400u};
  asm("" : "+s"(k.m0), "+s"(k.m1), "+v"(k.e10), "+v"(k.e6));
  return k;
}
__device__ __forceinline__ v8h unpack(uint32_t w, const Bits& k, v2h b0, v2h b1, v2h b2, v2h b3) {
  const uint32_t w8 = w >> 8;
  const v2h h0 = __builtin_bit_cast(v2h, (w & k.m0) | k.e10) - b0;
  const v2h h1 = __builtin_bit_cast(v2h, (w & k.m1) | k.e6) - b1;
  const v2h h2 = __builtin_bit_cast(v2h, (w8 & k.m0) | k.e10) - b2;
  const v2h h3 = __builtin_bit_cast(v2h, (w8 & k.m1) | k.e6) - b3;
  return v8h{h0[0], h0[1], h1[0], h1[1], h2[0], h2[1], h3[0], h3[1]};
}

// One of the two elements of a word of queries
template <bool BF16>
__device__ __forceinline__ float element(uint32_t w, bool high) {
  if constexpr (BF16) return __uint_as_float(high ? w & 0xFFFF0000u : w << 16);
  const v2h h = __builtin_bit_cast(v2h, w);
  return (float)(high ? h[1] : h[0]);
}

// Largest of three, in one instruction (fmaxf would first quiet each operand); a NaN is passed over
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
  return r;
}
// x less one half of a pair of fp16 values, exact here, in one instruction
__device__ __forceinline__ float less_low(float x, v2h h) {
  float r;
  asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(x));
  return r;
}
__device__ __forceinline__ float less_high(float x, v2h h) {
  float r;
  asm("v_fma_mix_f32 %0, -%1, 1.0, %2 op_sel:[1,0,0] op_sel_hi:[1,0,0]" : "=v"(r) : "v"(h), "v"(x));
  return r;
}

// Where a wave's token lies: lane l holds the cache row of token t0 + l, 0 for one that is not there.
struct Rows {
  uint32_t row;
  bool ok;
};

// A wave's own staging area, and the area where the waves' sums meet
struct Stage {
  uint32_t v[kStep * kD / 8];   // value codes, 64 bytes a token, 16-byte pieces of row r at piece ^ (r / 16)
  float ks[kStep], ls[kStep], rs[kStep];   // key scale log2 e / sqrt(128); log2 and reciprocal of the value scale
  v4h kz[kStep];                // 1024 + key zero-point twice, 64 + key zero-point twice
  _Float16 vz[kStep];           // 1024 or 64 + value zero-point, in the order of use
};
constexpr int kPad = kD + 4;
union Lds {
  Stage stage[kWaves];
  float sum[kWaves][16][kPad];
};

__device__ __forceinline__ uint16_t to_bits(float f, bool bf16) {
  if (!bf16) return __builtin_bit_cast(uint16_t, (_Float16)f);
  const uint32_t u = __float_as_uint(f);
  return (uint16_t)(f == f ? (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16 : (u >> 16) | 0x40u);
}

__device__ __forceinline__ pages::Seq sequence_of(ArgPtr a, int b) {
  return pages::sequence(a->starts[b], a->starts[b + 1], a->lens[b], a->rows, a->max_nodes, a->most);
}
// All sequences, and the slots of those before each one (times Hkv: before its first KV head), by the first wave;
// sequences without nodes have none.
struct Sequences {
  int32_t before[pages::kMostShared + 1];
  int4 seq[pages::kMostShared];   // first row, nodes, length, context
};
// x of the lane and all lanes below it
__device__ __forceinline__ int32_t running_sum(int32_t x) {
#define QIFT_SUM(CTRL, ROWS) x += __builtin_amdgcn_update_dpp(0, x, CTRL, ROWS, 0xf, false)
  QIFT_SUM(0x111, 0xf);   // row_shr 1, 2, 4, 8
  QIFT_SUM(0x112, 0xf);
  QIFT_SUM(0x114, 0xf);
  QIFT_SUM(0x118, 0xf);
  QIFT_SUM(0x142, 0xa);   // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
  QIFT_SUM(0x143, 0xc);
#undef QIFT_SUM
  return x;
}
__device__ __forceinline__ void add_slots(ArgPtr a, Sequences& all, bool flag) {
  if (threadIdx.x < 64) {
    int32_t sum = 0;
    if (threadIdx.x == 0) all.before[0] = 0;
    const int B = a->B;
    for (int b0 = 0; b0 < B; b0 += 64) {
      const int b = b0 + (int)threadIdx.x;
      int32_t r = 0;
      if (b < B) {
        const pages::Seq sq = sequence_of(a, b);
        r = sq.n > 0 ? pages::slots_of(sq.len) : 0;
        all.seq[b] = make_int4(sq.row0, sq.n, sq.len, sq.ctx);
        if (flag && sq.bad) dev::flag_error(a->err, kDevErrIndex);
      }
      r = running_sum(r);
      if (b < B) all.before[b + 1] = sum + r;
      sum += __builtin_amdgcn_readlane(r, 63);
    }
  }
  __syncthreads();
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// A run of rounds of one unit for the 16 RT rows from r0 on; whole: the run is all of the unit, so its result is final.
struct Run {
  int b, kv, r0;
  int32_t lo, hi;    // rounds of 256 tokens
  bool whole;
  int64_t record;
};

template <int RT>
struct Tree {
  Lds lds;
  float stat[2][kWaves][16 * RT];   // reference, sum of exponentials
  float back[16 * RT];
};

template <int RT, bool BF16>
__device__ __forceinline__ void tree_run(Tree<RT>& sh, const pages::Seq& sq, const Run& run) {
  const int lane = thread_again() & 63, c = lane & 15, kg = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int b = run.b, kv = run.kv, r0 = run.r0;
  Lds& lds = sh.lds;
  auto& stat = sh.stat;
  const int32_t t_lo = run.lo * kRound;
  int32_t t_hi = run.hi * kRound;

  const ArgPtr a = arguments();
  {
    const int32_t end = pages::last_token(sq, a->visible != nullptr, group_of(a), 16 * RT, r0 / (16 * RT));
    if (end < t_hi) t_hi = end;
  }
  const int32_t* table = a->table + (int64_t)b * a->table_pages;
  const uint8_t *kc = a->kc, *kz = a->kz, *vc = a->vc, *vz = a->vz;
  const float *ks = a->ks, *vs = a->vs;
  const pages::Div tiles = tiles_of(a);
  const uint32_t pool_pages = a->pool_pages, Hkv = (uint32_t)a->Hkv;
  auto entry = [&](int32_t t0) {   // the table's entry of token t0 + lane (anything for a token that is not there)
    const int32_t t = t0 + lane;
    return table[t < t_hi ? pages::table_index((uint32_t)t, tiles) : 0u];
  };
  bool bad = false;            // a table entry that names no page
  auto rows_of = [&](int32_t t0, int32_t e) {
    const int32_t t = t0 + lane;
    Rows r;
    r.ok = t < t_hi && (uint32_t)e < pool_pages;
    bad |= t < t_hi && !r.ok;
    r.row = r.ok ? pages::token_row((uint32_t)t, (uint32_t)e, Hkv, (uint32_t)kv, tiles) : 0u;
    return r;
  };
  // A step's loads.  Its value codes, scales and zero-points go to LDS when it begins, its key codes are used from
  // registers; the next step's are sent once they are, without a branch (a step past the end reads the cache's first
  // rows).  A tile of 16 tokens is 1 KB from its first row on (a page holds whole tiles): a uniform address and a fixed
  // offset of the lane.
  uint4 vw[4], kw[4];
  float ksl, vsl;
  // (bytes, not words: those would be extended, and all loads waited for, in the middle of the step before; 32 ragged sequences
  // of one token 47 us instead of 43.9)
  uint8_t kzl, vzl;
  Rows cur{0, false};
  int32_t ahead = 0;           // the next step's table entry
  const uint32_t koff = 64u * (uint32_t)c + 16u * (uint32_t)kg, voff = 16u * (uint32_t)lane;
  auto load = [&](const Rows& r) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint64_t first = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)r.row, 16 * j) * (kD / 2);
      vw[j] = *reinterpret_cast<const uint4*>(vc + first + voff);
      kw[j] = *reinterpret_cast<const uint4*>(kc + first + koff);
    }
    ksl = ks[r.row];
    vsl = vs[r.row];
    kzl = kz[r.row];
    vzl = vz[r.row];
  };

  int32_t t0 = t_lo + wave * kStep;
  if (t0 < t_hi) {
    cur = rows_of(t0, entry(t0));
    ahead = entry(t0 + kRound);
    load(cur);
  }

  // ---- the queries: B operands, element e of step st is dimension 32 kg + 8 st + kNib[e] of row c.  A row whose largest is
  // outside [2^-4, 2^15) is brought to [2^14, 2^15) by a power of two.  A bf16 query below 2^-17 is off by 2^-25 at most then
  // (so is the last bit of an fp16 row that is scaled down), all others are exact.
  v8h qb[RT][4];
  bool ranged = false; // whether any row has a power of two to be taken back (sh.back; all waves write the same)
  int32_t node[RT];
  {
  const ArgPtr a = arguments();
  const pages::Div group = group_of(a);
  const int G = a->G, nrows = sq.n * G;
  const uint16_t* q = a->q;
  const int64_t stride = a->q_stride;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int r = r0 + 16 * rt + c;
    const bool in = r < nrows;
    const int rr = in ? r : nrows - 1;
    node[rt] = (int32_t)pages::quotient((uint32_t)rr, group);
    const int h = kv * G + rr - node[rt] * G;
    const v4u* src = reinterpret_cast<const v4u*>(q + (int64_t)(sq.row0 + node[rt]) * stride + (int64_t)h * kD + 32 * kg);
    v4u u[4];
    float top = 0.f;
#pragma unroll
    for (int st = 0; st < 4; ++st) u[st] = in ? src[st] : v4u{0, 0, 0, 0};
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int n = 0; n < 8; ++n) top = fmaxf(top, fabsf(element<BF16>(u[st][n >> 1], n & 1)));
    top = fmaxf(top, __shfl_xor(top, 16));
    top = fmaxf(top, __shfl_xor(top, 32));
    const int ex = top > 0.f && top < INFINITY && !(top >= 0x1p-4f && top < 0x1p15f) ? 14 - ilogbf(top) : 0;
    if (kg == 0) sh.back[16 * rt + c] = ldexpf(1.f, -ex);
    ranged |= __any(ex != 0);
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int n = kNib[e];
        qb[rt][st][e] = (_Float16)ldexpf(element<BF16>(u[st][n >> 1], n & 1), ex);
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
  const Bits bits = code_bits();
  bool direct = false;         // a weight that is 0 need not mean that p is
  Stage& sg = lds.stage[wave];
  auto step = [&](int32_t t0) {
    const uint64_t there = __ballot(cur.ok);
    // ---- stage the step's scales, zero-points and value codes (a wave's LDS operations keep their order)
    {
      float v = vsl < kLeast ? kLeast : vsl;   // (NaN stays: w is NaN where it is seen)
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
      constexpr float kScore = 0.088388347648318447f * 1.4426950408889634f;   // 1 / sqrt(128), log2 e
      sg.ks[lane] = ksl * kScore;
      sg.ls[lane] = __builtin_amdgcn_logf(v);
      sg.rs[lane] = vsl < INFINITY ? __builtin_amdgcn_rcpf(v) : 0.f; 
      const _Float16 z10 = (_Float16)(1024.f + (float)kzl), z6 = (_Float16)(64.f + (float)kzl);
      sg.kz[lane] = v4h{z10, z10, z6, z6};
      // token 16 j + 4 g + i goes to pair i of half j / 2 of lane group g, element j mod 2
      const int tj = lane >> 4, tg = (lane >> 2) & 3, ti = lane & 3;
      sg.vz[tg * 16 + (tj >> 1) * 8 + ti * 2 + (tj & 1)] = (_Float16)((ti & 1 ? 64.f : 1024.f) + (float)vzl);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint4*>(&sg.v[(16 * j + (lane >> 2)) * (kD / 8) + 4 * ((lane & 3) ^ j)]) = vw[j];
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    // ---- scores, at once as powers of two with the value's scale: y = score + log2 s of token 16 j + 4 kg + i.  Four
    // independent sums at a time: 4 / RT tiles of tokens.
    v4f y[RT][4];
    constexpr int TJ = 4 / RT;
#pragma unroll
    for (int j0 = 0; j0 < 4; j0 += TJ) {
      v4f acc[TJ][RT];
      v2h b10[TJ], b6[TJ];
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        const v4h z = sg.kz[16 * (j0 + j) + c];
        b10[j] = v2h{z[0], z[1]};
        b6[j] = v2h{z[2], z[3]};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[j][rt] = v4f{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
          const uint4& u = kw[j0 + j];
          const v8h kd = unpack(st == 0 ? u.x : st == 1 ? u.y : st == 2 ? u.z : u.w, bits, b10[j], b6[j], b10[j], b6[j]);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) acc[j][rt] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kd, qb[rt][st], acc[j][rt], 0, 0, 0);
        }
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        const v4f k4 = *reinterpret_cast<const v4f*>(&sg.ks[16 * (j0 + j) + 4 * kg]);
        const v4f l4 = *reinterpret_cast<const v4f*>(&sg.ls[16 * (j0 + j) + 4 * kg]);
        if (ranged) {
          // a power of two below 1 goes to the sums, one above 1 comes after the key's scale: no product leaves fp32's range
          // before the score does
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const float back = sh.back[16 * rt + c], down = fminf(back, 1.f), up = fmaxf(back, 1.f);
#pragma unroll
            for (int i = 0; i < 4; ++i) y[rt][j0 + j][i] = fmaf(acc[j][rt][i] * down * k4[i], up, l4[i]);
          }
        } else {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[rt][j0 + j][i] = fmaf(acc[j][rt][i], k4[i], l4[i]);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    // ---- the next step's loads
    const Rows nxt = rows_of(t0 + kRound, ahead);
    ahead = entry(t0 + 2 * kRound);
    load(nxt);
    __builtin_amdgcn_sched_barrier(0);
    // ---- what a row does not see
    if (there != ~uint64_t(0) || t0 + kStep > sq.ctx) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        uint64_t see;
        const ArgPtr a = arguments();
        const uint64_t* visible = a->visible;
        const int32_t words = a->words;
        if (visible) {
          const int32_t d0 = t0 - sq.ctx;
          uint64_t w0 = 0, w1 = 0;
          const int32_t k0 = d0 > 0 ? d0 >> 6 : 0;
          if (d0 > -64) {
            const uint64_t* row = visible + (int64_t)(sq.row0 + node[rt]) * words;
            if (k0 < words) w0 = row[k0];
            if (k0 + 1 < words) w1 = row[k0 + 1];
          }
          see = pages::tree_bits(d0, w0, w1);
        } else {
          see = pages::chain_bits(t0, sq.ctx, node[rt]);
        }
        see = (see & there) >> (4 * kg);   // bit 16 j + i: token 16 j + 4 kg + i
        const uint32_t seen[2] = {(uint32_t)see, (uint32_t)(see >> 32)};
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) y[rt][j][i] = (seen[j >> 1] >> (16 * (j & 1) + i)) & 1u ? y[rt][j][i] : -INFINITY;
      }
    }
    // ---- softmax: weights w as two fp16 parts, B operands of the value phase
    v8h ahi[RT][2], alo[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float top = -INFINITY;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = max3(max3(top, y[rt][j][0], y[rt][j][1]), y[rt][j][2], y[rt][j][3]);
      if (__any(top > m[rt] + (kTop + kSlack))) {
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float mn = fmaxf(m[rt], top - kTop), f = __builtin_amdgcn_exp2f(m[rt] - mn);
        l[rt] = scaled(l[rt], m[rt] - mn);
        m[rt] = mn;
#pragma unroll
        for (int dt = 0; dt < 8; ++dt) o[rt][dt] *= f;
      }
    }
    if (direct) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float base = m[rt];
        asm volatile("" : "+v"(base));   // (or the weights below would be kept in registers from here on)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const v4f l4 = *reinterpret_cast<const v4f*>(&sg.ls[16 * j + 4 * kg]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = __builtin_amdgcn_exp2f(y[rt][j][i] - l4[i] - base);
            const bool lost = __builtin_amdgcn_exp2f(y[rt][j][i] - base) == 0.f, seen = y[rt][j][i] > -INFINITY;
            l[rt] += lost & seen ? p : 0.f;
          }
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    }
    float add[RT];               // the step's sum of exponentials: the running one then rounds once a step, not 16 times
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) add[rt] = 0.f;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      // half h, pair i: tokens 16 (2 h) + 4 kg + i and 16 (2 h + 1) + 4 kg + i
      const v4f r0 = *reinterpret_cast<const v4f*>(&sg.rs[32 * h + 4 * kg]);
      const v4f r1 = *reinterpret_cast<const v4f*>(&sg.rs[32 * h + 16 + 4 * kg]);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = __builtin_amdgcn_exp2f(y[rt][2 * h][i] - m[rt]), z = __builtin_amdgcn_exp2f(y[rt][2 * h + 1][i] - m[rt]);
          add[rt] = fmaf(x, r0[i], add[rt]);
          add[rt] = fmaf(z, r1[i], add[rt]);
          const v2h hi = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_pkrtz(x, z));
          const v2h lo = __builtin_bit_cast(v2h, __builtin_amdgcn_cvt_pkrtz(less_low(x, hi), less_high(z, hi)));
          ahi[rt][h][2 * i] = hi[0];
          ahi[rt][h][2 * i + 1] = hi[1];
          alo[rt][h][2 * i] = lo[0];
          alo[rt][h][2 * i + 1] = lo[1];
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) l[rt] += add[rt];
    // ---- values: A = 16 dimensions x 32 tokens of code - z.  The transposing read hands lane (c, kg) the 16 codes of
    // dimension 16 dt + c whose rows the 16 lanes of its group name: token 16 (c / 4) + 4 kg + c mod 4, nibble c.
    {
      v8h bz[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) bz[h] = *reinterpret_cast<const v8h*>(&sg.vz[16 * kg + 8 * h]);
      const int row = 16 * (c >> 2) + 4 * kg + (c & 3);
      // Dimension tiles at a time, for four independent sums; the next ones' reads go ahead of them.
      constexpr int TD = 4 / RT;
      v2i t[2][TD];
      auto read = [&](int d0, v2i (&t)[TD]) {
#pragma unroll
        for (int d = 0; d < TD; ++d) {
          const int dt = d0 + d, off = row * (kD / 8) + 4 * ((dt >> 1) ^ (c >> 2)) + 2 * (dt & 1);
          t[d] = __builtin_amdgcn_ds_read_tr4_b64_v2i32((__attribute__((address_space(3))) v2i*)(sg.v + off));
        }
      };
      read(0, t[0]);
#pragma unroll
      for (int d0 = 0; d0 < 8; d0 += TD) {
        if (d0 + TD < 8) read(d0 + TD, t[(d0 / TD + 1) & 1]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          v8h va[TD];
#pragma unroll
          for (int d = 0; d < TD; ++d) {
            const v2i x = t[(d0 / TD) & 1][d];
            va[d] = unpack(h ? (uint32_t)x.y : (uint32_t)x.x, bits, v2h{bz[h][0], bz[h][1]}, v2h{bz[h][2], bz[h][3]},
                           v2h{bz[h][4], bz[h][5]}, v2h{bz[h][6], bz[h][7]});
          }
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int d = 0; d < TD; ++d)
#pragma unroll
              for (int rt = 0; rt < RT; ++rt)
                o[rt][d0 + d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(va[d], part ? alo[rt][h] : ahi[rt][h], o[rt][d0 + d], 0, 0, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    cur = nxt;
  };
  for (; t0 < t_hi; t0 += kRound) step(t0);

  const ArgPtr z = arguments();
  if (bad) dev::flag_error(z->err, kDevErrIndex);
  const int G = z->G, nrows = sq.n * G;
  const pages::Div group = group_of(z);
  const int tid = thread_again(), c2 = tid & 15, kg2 = (tid >> 4) & 3;

  // ---- the four waves' sums meet under a common reference
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] += __shfl_xor(l[rt], 16);
    l[rt] += __shfl_xor(l[rt], 32);
    if (kg2 == 0) {
      stat[0][wave][16 * rt + c2] = m[rt];
      stat[1][wave][16 * rt + c2] = l[rt];
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    __syncthreads();   // the staging areas, or the last tile's sums, are no longer read
    float M = stat[0][0][16 * rt + c2];
#pragma unroll
    for (int w = 1; w < kWaves; ++w) M = fmaxf(M, stat[0][w][16 * rt + c2]);
    const float f = __builtin_amdgcn_exp2f(m[rt] - M);
#pragma unroll
    for (int dt = 0; dt < 8; ++dt) *reinterpret_cast<v4f*>(&lds.sum[wave][c2][16 * dt + 4 * kg2]) = o[rt][dt] * f;
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
      if (run.whole) {
        const int nd = (int)pages::quotient((uint32_t)r, group);
        const float inv = L == 0.f ? 0.f : 1.f / L;   // a row that sees nothing: 0
        uint32_t w[4];
#pragma unroll
        for (int e = 0; e < 4; ++e)
          w[e] = (uint32_t)to_bits(s[2 * e] * inv, BF16) | ((uint32_t)to_bits(s[2 * e + 1] * inv, BF16) << 16);
        uint16_t* y = z->out + ((int64_t)(sq.row0 + nd) * z->Hq + kv * G + (r - nd * G)) * kD + d0;
        *reinterpret_cast<uint4*>(y) = make_uint4(w[0], w[1], w[2], w[3]);
      } else {
        const int64_t rec = run.record * ((int64_t)z->max_nodes * G) + r;
        float* y = z->part + rec * kD + d0;
        *reinterpret_cast<float4*>(y) = make_float4(s[0], s[1], s[2], s[3]);
        *reinterpret_cast<float4*>(y + 4) = make_float4(s[4], s[5], s[6], s[7]);
        if (d0 == 0) {
          z->part[z->records * kD + 2 * rec] = Mr;
          z->part[z->records * kD + 2 * rec + 1] = L;
        }
      }
    }
  }
}

// RT = 1 is bound by its loads: 32 ragged sequences of one token, 154 MB, 44 us with the second launch (3.5 TB/s); 16 chains
// of 5, 146 MB, 37 us (3.9).  RT = 2 is bound by the instructions a SIMD issues, 608 vector and 96 matrix ones a step of 64
// tokens: 16 trees of 64 nodes over 8192 tokens 264 us, 0.78 PFLOP/s of matrix instructions.  (Times of captured calls on
// two caches in turn.)  Two waves to a SIMD: the output sums, weights and the next step's codes take 242 registers.
template <int RT, bool BF16>
__global__ __launch_bounds__(256, 2) void k_tree(TreeArgs) {
  __shared__ __attribute__((aligned(16))) Tree<RT> sh;
  __shared__ Sequences all;
  const ArgPtr a = arguments();
  // Workgroups go to the XCDs in turn.  Blocks of rows over the same tokens are taken by one XCD, whose L2 then holds the
  // tokens.
  Run run;
  if (a->shares == 0) {
    const uint32_t per = 8u * (uint32_t)a->blocks;
    const uint32_t i = (blockIdx.x / per) * 8 + blockIdx.x % 8, block = (blockIdx.x % per) / 8;
    run.r0 = (int)block * 16 * RT;
    run.b = (int)(i / (uint32_t)a->Hkv);
    run.kv = (int)(i % (uint32_t)a->Hkv);
    if (run.b >= a->B) return;
    const pages::Seq sq = sequence_of(a, run.b);
    if (sq.bad && block == 0 && run.kv == 0 && threadIdx.x == 0) dev::flag_error(a->err, kDevErrIndex);
    if (run.r0 >= sq.n * a->G) return;
    run.lo = 0;
    run.hi = pages::rounds_of(sq.len);
    run.whole = true;
    run.record = 0;
    tree_run<RT, BF16>(sh, sq, run);
    return;
  }
  add_slots(a, all, blockIdx.x == 0);
  const int B = a->B, Hkv = a->Hkv;
  const int64_t W = (int64_t)uniform(all.before[B]) * Hkv;
  // An XCD has an eighth of all blocks of all shares, one share's blocks after another's: as many as it has room for, so that
  // none waits for another to end (4 sequences of 69 nodes and 2984 tokens, 16 heads a group, 35 blocks and 14 shares: 48
  // us; with whole shares to an XCD, some with two and some with one, 65).
  const int32_t shares = pages::used_shares(W, a->shares);
  const pages::Place mine = pages::place((int32_t)blockIdx.x, shares, a->blocks);
  if (mine.share >= shares) return;
  const int32_t i = mine.share, block = mine.block;
  run.r0 = block * 16 * RT;
  int64_t pos = pages::first_slot(W, shares, i);
  const int64_t stop = pages::first_slot(W, shares, i + 1);
  // the sequence of the share's first slot: as many as have all their slots before it (those without slots too)
  int b = 0;
  for (int b0 = 0; b0 < B; b0 += 64) {
    const int x = b0 + (int)(threadIdx.x & 63);
    b += __popcll(__ballot(x < B && (int64_t)all.before[x + 1] * Hkv <= pos));
  }
  for (b = uniform(b); pos < stop; ++b) {
    const int4 q = all.seq[b];
    const pages::Seq sq = {uniform(q.x), uniform(q.y), uniform(q.z), uniform(q.w), false};
    if (sq.n == 0) continue;
    const int32_t first = uniform(all.before[b]), rounds = pages::rounds_of(sq.len), n = pages::slots_of(sq.len);
    run.b = b;
    for (run.kv = (int)((uint32_t)(pos - (int64_t)first * Hkv) / (uint32_t)n); run.kv < Hkv && pos < stop; ++run.kv) {
      const int64_t at = (int64_t)first * Hkv + (int64_t)run.kv * n;
      const int32_t hi = stop - at < n ? (int32_t)(stop - at) : n;
      run.lo = pages::round_at((int32_t)(pos - at));
      run.hi = pages::round_at(hi);
      pos = at + hi;
      if (run.hi == run.lo) continue;
      run.whole = run.lo == 0 && run.hi == rounds;
      run.record = (int64_t)i + (int64_t)b * Hkv + run.kv;
      if (block == 0 && threadIdx.x == 0) {   // which shares have the unit, for k_tree_merge
        int32_t* units = reinterpret_cast<int32_t*>(a->part + a->records * (kD + 2)) + 2 * ((int64_t)b * Hkv + run.kv);
        if (run.lo == 0) units[0] = i;
        if (run.hi == rounds) units[1] = i;
      }
      if (run.r0 < sq.n * a->G) {
        tree_run<RT, BF16>(sh, sq, run);
        __syncthreads();
      }
    }
  }
}

// out = sum_i 2^(m_i - M) sums_i / sum_i 2^(m_i - M) l_i over the shares i that cover a row's unit, where there are more
// than one.  32 lanes of four dimensions take a row, or `slices` times 32 lanes share its records, four at a time with
// every load sent before the first is used (the call's second kernel mostly waits: each wait in a row costs it about
// a microsecond of its four).
constexpr int kJoin = 4;
__global__ __launch_bounds__(256) void k_tree_merge(TreeArgs a, int32_t slices) {
  __shared__ v4f sums[8][32];
  __shared__ float stats[2][8];
  const int lane = threadIdx.x & 31, slot = threadIdx.x >> 5;
  const int kv = blockIdx.y, b = blockIdx.z;
  const int64_t unit = (int64_t)b * a.Hkv + kv, R = (int64_t)a.max_nodes * a.G;
  const int32_t* units = reinterpret_cast<const int32_t*>(a.part + a.records * (kD + 2)) + 2 * unit;
  const int32_t i0 = units[0], count = units[1] - i0 + 1;   // (of a sequence without nodes: not written, and not used)
  const pages::Seq sq = sequence_of(arguments(), b);
  const int nrows = sq.n * a.G, first = (int)blockIdx.x * (8 / slices);
  if (first >= nrows || count == 1) return;
  const int r = first + slot / slices, slice = slot % slices;
  const bool in = r < nrows;
  v4f acc = {0.f, 0.f, 0.f, 0.f};
  float M = kLowest, L = 0.f;
  if (in) {
    const int64_t rec = (i0 + unit) * R + r;
    const float* st = a.part + a.records * kD + 2 * rec;
    const float* y = a.part + rec * kD + 4 * lane;
    for (int32_t c0 = slice; c0 < count; c0 += slices * kJoin) {
      v4f o[kJoin];
      float m[kJoin], l[kJoin];
#pragma unroll
      for (int j = 0; j < kJoin; ++j) {
        const int32_t c = c0 + slices * j < count ? c0 + slices * j : c0;   // past the last: the first again, without weight
        o[j] = *reinterpret_cast<const v4f*>(y + R * kD * c);
        m[j] = st[2 * R * c];
        l[j] = st[2 * R * c + 1];
      }
      float top = M;
#pragma unroll
      for (int j = 0; j < kJoin; ++j) top = fmaxf(top, m[j]);
      acc *= __builtin_amdgcn_exp2f(M - top);
      L = scaled(L, M - top);
#pragma unroll
      for (int j = 0; j < kJoin; ++j)
        if (c0 + slices * j < count) {
          acc += o[j] * __builtin_amdgcn_exp2f(m[j] - top);
          L += scaled(l[j], m[j] - top);
        }
      M = top;
    }
  }
  if (slices > 1) {
    sums[slot][lane] = acc;
    if (lane == 0) {
      stats[0][slot] = M;
      stats[1][slot] = L;
    }
    __syncthreads();
    if (slice) return;
    float top = M;
    for (int s = 1; s < slices; ++s) top = fmaxf(top, stats[0][slot + s]);
    acc *= __builtin_amdgcn_exp2f(M - top);
    L = scaled(L, M - top);
    for (int s = 1; s < slices; ++s) {
      const float m = stats[0][slot + s];
      acc += sums[slot + s][lane] * __builtin_amdgcn_exp2f(m - top);
      L += scaled(stats[1][slot + s], m - top);
    }
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
  a.records = pages::records(p, t.B, c.Hkv) * ((int64_t)t.max_nodes * G);
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
  a.shares = p.shares;
  a.blocks = p.blocks;
  a.bf16 = t.dtype == kBF16;
  const int64_t groups = p.shares ? ((int64_t)p.shares * p.blocks + 7) / 8 * 8 : (t.B * c.Hkv + 7) / 8 * 8 * p.blocks;
  const dim3 grid((unsigned)groups);
  auto kernel = p.rt == 1 ? (a.bf16 ? k_tree<1, true> : k_tree<1, false>) : a.bf16 ? k_tree<2, true> : k_tree<2, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.shares == 0) return e;
  // a row's records: about as many as there are shares to a unit, and one more
  const int64_t each = p.shares / (t.B * c.Hkv) + 2;
  const int32_t slices = each <= kJoin ? 1 : each <= 2 * kJoin ? 2 : each <= 4 * kJoin ? 4 : 8;
  const int64_t R = (int64_t)t.max_nodes * G;
  const dim3 mgrid((unsigned)((R * slices + 7) / 8), (unsigned)c.Hkv, (unsigned)t.B);
  hipLaunchKernelGGL(k_tree_merge, mgrid, dim3(256), 0, s, a, slices);
  return hipGetLastError();
}

}  // namespace qift
