/*
 * qift_pages.h - C ABI of the paged KV4 cache: quantizing the keys and values of new tokens into it,
 * reading them back, and attention of several new tokens per sequence over it.
 *
 * The cache holds what qift_kv4_quant makes of a key or value vector (Sec. 4.1 "Quantization
 * configuration", Sec. 3.3 Eq. (15)): 64 bytes of 4-bit codes, an fp32 scale and a zero-point byte
 * per token and KV head.  Its tokens live in pages of a common pool, so that many sequences grow
 * without moving: page p holds `page` tokens, and the slot number p * page + i names token i of it.
 * The conventions of qift.h hold: device pointers unless the comment says "host", asynchronous
 * calls on the given stream, no allocation, every host check before the first HIP call, and calls
 * that fail enqueue nothing.
 *
 * Slots, tables, starts and lens are read on the device, so the host cannot refuse what they hold.
 * The kernels never access memory outside the cache and the given rows for any content of theirs;
 * an entry outside its range is left out as described at each call and sets QIFT_DEVERR_INDEX in
 * the device error word (qift_device_error).
 */
#ifndef QIFT_PAGES_H
#define QIFT_PAGES_H

#include "qift.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bit of the device error word: a slot, a page number, a node count or a length outside its range. */
enum { QIFT_DEVERR_INDEX = 4 };

/* Element types of keys, values, queries and outputs. */
enum { QIFT_F16 = 0, QIFT_BF16 = 1, QIFT_F32 = 2 };

/*
 * A pool of pages (host; a non-owning view, every pointer device and 16-byte aligned).  Rows are
 * ordered [pages][Hkv][page], so that a KV head's tokens of one page are contiguous; a dense
 * head-major cache [B][Hkv][T] is the pool of B pages of T tokens.
 *   page      tokens of a page, a positive multiple of 16.
 *   Hkv       KV heads; head_dim is 128.
 *   Limits: pages * Hkv * page < 2^31 rows (137 GB of codes).  pages * page need not fit one sequence:
 *   a token's position never enters, only its slot.
 */
typedef struct {
  int64_t pages;
  int32_t page, Hkv, head_dim;
  int32_t reserved;                 /* 0 */
  uint8_t *k_codes;                 /* [rows][64] */
  float *k_scales;                  /* [rows]     */
  uint8_t *k_zeros;                 /* [rows]     */
  uint8_t *v_codes;
  float *v_scales;
  uint8_t *v_zeros;
} qift_kv4_pages;

/*
 * Quantize n tokens' keys and values into their slots, with the arithmetic of qift_kv4_quant
 * (x_max = c max(max x, 0), x_min = c min(min x, 0), c = fp32(0.95); s = (x_max - x_min) / 15, 1 for a
 * vector of zeros; z = round(-x_min / s); q = clip(round(x / s) + z, 0, 15); fp32, in that order,
 * halves to even): the same rows, bit for bit, that qift_kv4_quant writes for fp16.
 *   k, v       fp16 or bf16 rows: token t, head h starts at element t * stride + 128 h; 16-byte
 *              aligned, strides multiples of 8 and at least 128 Hkv (views of stacked q|k|v rows
 *              are taken as they are).  Values finite, |x| < 2^126.
 *   dtype      QIFT_F16 or QIFT_BF16.
 *   slots      int32 [n]: slot of each token.  A negative slot: the token is not written (padding).
 *              A slot at or past pages * page: not written, QIFT_DEVERR_INDEX.  A slot may appear once
 *              in a call: of two tokens with one slot, the row keeps parts of either.
 *   k_values, v_values   out, nullable (both or none): the values s (q - z) that the cache now
 *              stands for, [n][Hkv][128] in dtype (one rounding from fp32), for the attention of the
 *              prompt that is being written; zeros for a token that is not written.
 *   n = 0 does nothing.  Limits: ceil(n / 16) * Hkv < 2^23.
 */
int qift_kv4_append(const qift_kv4_pages *cache, const void *k, const void *v, int64_t k_stride,
                    int64_t v_stride, int32_t dtype, const int32_t *slots, int64_t n, void *k_values,
                    void *v_values, qift_stream_t stream);

/*
 * Read tokens back: k_values, v_values [n][Hkv][128] = s (code - z) of the given slots, computed in
 * fp32 and rounded once to dtype (QIFT_F16, QIFT_BF16, or QIFT_F32: the fp32 value itself).  A negative
 * slot gives zeros; a slot at or past pages * page zeros and QIFT_DEVERR_INDEX.  A slot may appear
 * any number of times.  n = 0 does nothing.  Limits: n <= 2^30 - 64.
 */
int qift_kv4_read(const qift_kv4_pages *cache, const int32_t *slots, int64_t n, int32_t dtype,
                  void *k_values, void *v_values, qift_stream_t stream);

/* Workspace bytes that are enough for every call of qift_kv4_attention_tree with these heads whose B, max_nodes
 * and max_len are at most these: it grows with each of them, and stays below 26 MB.  0 where no such call
 * needs any, and for an unsupported shape.  (A call asks for what its own limits need, which may be less: one
 * that has work for every CU without cutting sequences needs none.) */
size_t qift_kv4_attention_tree_workspace_bytes(int64_t B, int32_t Hq, int32_t Hkv, int32_t head_dim,
                                               int32_t max_nodes, int64_t max_len);

/*
 * Grouped-query attention of B sequences' new tokens over the paged cache.  Sequence b has lens[b]
 * cached tokens; the last n_b = starts[b+1] - starts[b] of them are its new tokens (its nodes), whose
 * queries are rows starts[b] .. starts[b+1] - 1 of q and whose keys and values are already in the
 * cache.  Position t of sequence b lies in page table[b][t / page] at t mod page.  With
 * ctx_b = lens[b] - n_b, row starts[b] + i sees
 *   every position t < ctx_b, and of its own sequence's nodes j (position ctx_b + j)
 *   those with bit j mod 64 of visible[starts[b] + i][j / 64] set, or, without a mask, j <= i:
 * one token (n_b = 1), a chain of drafts or a chunk of a prompt without a mask, a tree of drafts with
 * the bits of each node's ancestors and its own.  For query head h, kv = h / (Hq / Hkv):
 *   out[row][h] = sum_t p_t v_hat[t][kv],  p = softmax over the visible t of q[row][h] . k_hat[t][kv] / sqrt(128)
 * and 0 for a row that sees nothing.  What a row does not see never reaches its result, whatever it
 * holds (infinities, NaN, slots nothing was written to).
 *   q          fp16 or bf16: row r, head h starts at element r * q_stride + 128 h; 16-byte aligned,
 *              q_stride a multiple of 8 and at least 128 Hq.
 *   rows       rows of q and out; rows at or past starts[B] of out are left as they were.
 *   table      int32 [B][table_pages]; only the entries that positions below lens[b] need are read.
 *              An entry outside [0, pages): its positions are not seen, QIFT_DEVERR_INDEX.
 *   starts     int32 [B + 1], ascending from 0.  A sequence's nodes past max_nodes, and those at or past
 *              row `rows`, are left out, QIFT_DEVERR_INDEX: not computed and, whatever a mask says, not
 *              seen; its other nodes keep their places.  A sequence whose first row is outside [0, rows]
 *              has none of its rows computed, QIFT_DEVERR_INDEX.
 *   lens       int32 [B], n_b <= lens[b] <= max_len and lens[b] <= table_pages * page.  A length
 *              outside [0, that limit] is taken as the nearer end, QIFT_DEVERR_INDEX; for lens[b] < n_b
 *              the nodes past lens[b] have no position and are not seen.
 *              The new tokens have to be counted: of a sequence whose tokens were not written (one that
 *              qift_kv4_plan_step left out, whose length stays) the last n_b cached ones are taken for
 *              them, and its rows of out mean nothing.
 *   max_nodes, max_len   host: what n_b and lens[b] may reach in this call (they size the launch and
 *              the workspace, so a captured call serves any content up to them).
 *              They also decide how work is cut: from 1024 on of B * Hkv * ceil(max_nodes * Hq / Hkv / 32)
 *              (256 where max_len <= 1024), and for B > 512, each (sequence, KV head, 32 rows) is one
 *              workgroup's whatever its length, so a batch of very different lengths or node counts is
 *              faster in two calls then.
 *   visible    uint64 [rows][ceil(max_nodes / 64)], 8-byte aligned, nullable.
 *   out        out: [rows][Hq][128] in q's type.
 *   workspace  device scratch of qift_kv4_attention_tree_workspace_bytes bytes (16-byte aligned;
 *              NULL where that is 0): partial sums of parts of long sequences.  It belongs to one call
 *              at a time: calls that overlap, two captured graphs among them, need their own.
 * Arithmetic: products of exact fp16 operands (code - z, and the queries) summed in fp32; softmax statistics
 * and sums in fp32; weights p s as two fp16 parts (2^-21 relative).  A row whose largest query is outside
 * [2^-4, 2^15) is scaled by a power of two that brings it to [2^14, 2^15); a bf16 row's queries that are
 * below 2^-17 then, and those of an fp16 row that is scaled down below 2^-14, are off by 2^-25 at most, all
 * others exact.  The result is within half a step of its type and
 *   (2 (S + L) + 14 + lens[b] / 256) 2^-21
 * of the KV head's largest value, S the largest |q| |k_hat| / sqrt(128) of the row and L the largest |log2|
 * of a value scale that it sees: with u = 2^-24, a score takes 7 u S (four sums of products, the key's scale,
 * the conversion to a power of two, the value's scale), a weight 2 u L more, both count in the numerator and
 * in the denominator; a wave's sum of values has lens[b] / 64 instructions' roundings, its sum of weights
 * lens[b] / 256; the rest are the exponentials, the joining of waves and parts and the division.
 * Value scales under 2^-90 count as 2^-90.  A score that with log2 of its value's scale, both as powers of
 * two, is past fp32's lowest value counts as not seen; past its largest, the row is NaN.
 * B = 0 or rows = 0 does nothing.  Limits: 1 <= max_nodes <= 256, Hq a multiple of Hkv and
 * Hq / Hkv <= 64, B <= 65535, max_len < 2^28, rows < 2^31, B * Hkv * ceil(max_nodes * Hq / Hkv / 16) < 2^23.
 * Up to two launches.
 */
int qift_kv4_attention_tree(const qift_kv4_pages *cache, const void *q, int64_t q_stride, int32_t dtype,
                            int64_t rows, const int32_t *table, int32_t table_pages, const int32_t *starts,
                            const int32_t *lens, int64_t B, int32_t Hq, int32_t max_nodes, int64_t max_len,
                            const uint64_t *visible, void *out, void *workspace, size_t workspace_bytes,
                            qift_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* QIFT_PAGES_H */
