/*
 * qift_step.h - C ABI of a serving step around the paged cache (qift_pages.h): where the new tokens of each sequence go,
 * the pages that are taken and given back for them, and the norms and the rotation of queries and keys between the linear that
 * makes them and the cache.
 *
 * The conventions of qift.h hold: device pointers unless the comment says "host", asynchronous calls on the given
 * stream, no allocation, every host check before the first HIP call, and calls that fail enqueue nothing.  Lengths, counts,
 * tables and stacks are device data, which the kernels check themselves: nothing is read or written outside the given
 * arrays for any content of theirs, and what is out of its range sets QIFT_DEVERR_INDEX in the device error word.
 */
#ifndef QIFT_STEP_H
#define QIFT_STEP_H

#include "qift.h"
#include "qift_pages.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Plan of a step: block table, slots, positions and row starts of the new tokens of B sequences.  Sequence b has lens[b]
 * cached tokens in the pages table[b][0 .. ceil(lens[b] / page)) and gets counts[b] new ones, whose rows stand behind those of
 * the sequences before it.  Free pages are a stack, free_pages[0 .. *free_count), of which the sequences take from the top in
 * their order:
 *   starts[b]   = counts[0] + .. + counts[b - 1], starts[B] their sum (each at most `rows`)
 *   lens_out[b] = lens[b] + counts[b]
 *   the k-th page that is taken, counted over all sequences and along each, is free_pages[*free_count - 1 - k];
 *   table[b]    gets its pages behind those that it holds; its other entries are left as they are
 *   *free_out   = *free_count less the pages taken
 *   row starts[b] + i: positions = lens[b] + i, slots = table[b][positions / page] * page + positions mod page;
 *   rows at or past starts[B]: -1 in both.
 * slots, table, starts and lens_out are what qift_kv4_append and qift_kv4_attention_tree take (they read a table row no
 * further than lens_out), positions what qift_head_norm_rope takes.
 * A sequence is served whole or not at all.  Left out, with QIFT_DEVERR_INDEX, are: one whose tokens do not fit its row of
 * the table; one whose rows do not all lie below `rows`; one that needs pages where the stack does not hold them after
 * all the sequences before it (left out for their rows or for pages or not) have had theirs.  Its slots and positions
 * are -1, its lens_out is lens[b], and it takes no pages; its rows keep their places.  What the rest of the step makes of
 * those rows means nothing: qift_kv4_attention_tree has no way to see that they were left out, takes the last cached tokens for
 * them and fills their rows of its output.  A sequence has its outputs in this step where lens_out[b] is lens[b] + counts[b],
 * a row where its position is not negative; the others' outputs do not depend on what was left out.  A negative count counts as 0 and a
 * length outside [0, table_pages * page] as the nearer end (its sequence is left out), with QIFT_DEVERR_INDEX; so does a depth
 * outside [0, capacity].  A page number that is negative or whose slots have no 31 bits gives slots of -1 and QIFT_DEVERR_INDEX.
 *   lens, counts   int32 [B].
 *   table          int32 [B][table_pages], read and written.
 *   free_pages     int32 [capacity]; free_count int32 [1].
 *   page           tokens of a page, a positive multiple of 16.
 *   rows           entries of slots and positions.
 *   starts out: int32 [B + 1]; lens_out out: int32 [B]; slots, positions out: int32 [rows]; free_out out: int32 [1].
 *   Nothing that is written (the table and the outputs) may overlap another of the arrays, the inputs among them
 *   (QIFT_ERR_SHAPE): every workgroup reads those afresh.  A loop of steps has two of lens_out and free_out in turn.
 * B = 0 gives starts[0] = 0 and rows of -1.  All arrays 4-byte aligned.  Limits: B <= 65535, rows < 2^31,
 * table_pages * page < 2^31, capacity < 2^31.  One launch.
 */
int qift_kv4_plan_step(const int32_t *lens, const int32_t *counts, int64_t B, int32_t *table, int32_t table_pages,
                       int32_t page, const int32_t *free_pages, const int32_t *free_count, int64_t capacity, int64_t rows,
                       int32_t *starts, int32_t *lens_out, int32_t *slots, int32_t *positions, int32_t *free_out,
                       qift_stream_t stream);

/*
 * The pages of finished sequences go back on the stack: for each b with done[b] != 0, in order, the pages
 * table[b][0 .. ceil(lens[b] / page)) are written to free_pages from *free_count on; lens_out[b] = 0 for these and lens[b]
 * for the others, *free_out = *free_count plus the pages given back.  The table is left as it is.  Pages that several
 * sequences share are the caller's to count: each row that names one gives it back.
 * A length or depth outside its range is taken as in qift_kv4_plan_step; pages past the stack's capacity are dropped and a
 * negative page number is put back as it is, both with QIFT_DEVERR_INDEX.
 * free_pages, lens_out and free_out are written and overlap nothing else (QIFT_ERR_SHAPE).  Arguments, limits and alignment
 * as there.  B = 0 copies the depth.  One launch.
 */
int qift_kv4_release(const int32_t *lens, const int32_t *done, int64_t B, const int32_t *table, int32_t table_pages,
                     int32_t page, int32_t *free_pages, const int32_t *free_count, int64_t capacity, int32_t *lens_out,
                     int32_t *free_out, qift_stream_t stream);

/*
 * Norms and rotation of a model's heads (host; a non-owning view).
 *   rot        values of each head that are rotated, its first ones: a multiple of 8, 0 .. head_dim.
 *   pairs      0: value i is paired with value i + rot / 2; 1: value 2 i with value 2 i + 1.
 *   freq       fp32 [rot / 2]: the angle of pair i at position p is p * freq[i].  Angles are below 2^40 (for every position:
 *              |freq| < 512); a pair whose angle is not, or whose frequency is no number, gets NaN.
 *   q_weight, k_weight   [head_dim] in the type of the rows, nullable: without one those heads are not normed.
 *   eps        finite, at least 2^-80 (squares that fp32 cannot hold are then nothing beside it).
 */
typedef struct {
  int32_t head_dim;            /* 128 */
  int32_t rot, pairs;
  float eps;
  const float *freq;
  const void *q_weight, *k_weight;
} qift_head_rope;

/*
 * For each head x of a row at position p:
 *   y = x / sqrt(mean(x^2) + eps) * w      (y = x without a weight)
 *   (a, b) -> (a cos t - b sin t, a sin t + b cos t), t = p * freq[i], for each pair of the rotated values.
 * fp32, the angle's exact product reduced in fp64 (sine and cosine are within 2^-22), one rounding at the end.  The result
 * is within half a step of its type and 2^-19 (|a| + |b|) of the exact one, a and b the pair's normed values.  The sum
 * of a head's squares has to be finite in fp32.
 *   q, k        fp16 or bf16: row r, head h starts at element r * stride + 128 h; strides multiples of 8 and at least
 *               128 heads (views of stacked q|k|v rows are taken as they are).  Hq or Hkv may be 0 (its pointers are not
 *               looked at then), not both.
 *   dtype       QIFT_F16 or QIFT_BF16.
 *   positions   int32 [rows].  A negative position: the row is padding, its outputs are zeros.
 *   q_out, k_out   out: as q and k, with strides of their own; the input itself with the input's stride is taken (each
 *               value is read before it is written), any other overlap of an output with an array of the call is
 *               QIFT_ERR_SHAPE (rows of stacked views that lie between each other's are no overlap).
 * 16-byte aligned, positions 4.  rows = 0 does nothing.  Limits: rows * ceil((Hq + Hkv) / 4) <= 2^26 - 4.  One launch.
 */
int qift_head_norm_rope(const qift_head_rope *rope, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                        int32_t dtype, const int32_t *positions, int64_t rows, int32_t Hq, int32_t Hkv, void *q_out,
                        int64_t q_out_stride, void *k_out, int64_t k_out_stride, qift_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* QIFT_STEP_H */
