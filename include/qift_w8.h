/*
 * qift_w8.h - C ABI of the 8-bit linear (W8A8): the sibling of the 2- and 4-bit linears for the products that a model
 * keeps at more bits, such as the projections around the attention or the output head.  (The paper's schedules, Sec. 4.4, mix
 * 2 and 4 bits by layer; this linear is not among them.)
 *
 *   y[m, n] = s_w[n] * s_x[m] * sum_k level[n, k] * q[m, k]
 *
 * with 8-bit integers on both sides, one scale per output channel and one per token, and no zero-points.  The rotation
 * (Sec. 3.1) is that of the other linears: rows of the weights rotated offline, tokens online.
 * The conventions of qift.h hold: device pointers unless the comment says "host", 16-byte aligned, asynchronous calls on
 * the given stream, no allocation, every check before the first HIP call, and calls that fail enqueue nothing.
 */
#ifndef QIFT_W8_H
#define QIFT_W8_H

#include "qift.h"
#include "qift_pages.h"   /* the element types QIFT_F16, QIFT_BF16 and QIFT_F32 */

#ifdef __cplusplus
extern "C" {
#endif

/* 8-bit weights (host; a non-owning view): the levels are the operands of the product as they are, so nothing is
 * packed.  Limits: N < 2^31, K a positive multiple of 64 and at most 131072 (127 * 127 * K stays below 2^31). */
typedef struct {
  int64_t N, K;              /* output and input features                                        */
  const int8_t *levels;      /* [N][K], -127 .. 127                                              */
  const uint16_t *scales;    /* fp16 s_w[N]                                                      */
} qift_w8;

/*
 * Offline weight quantization (Eq. (1) with b = 8 on the symmetric range), as qift_quantize_weights does it for W4:
 * each row of the fp32 W [N][spec.K] rotated in fp64, s_w = fp16(max|w| / 127), q = clip(rne(w / s_w), -127, 127)
 * against the stored scale; a row whose stored scale is 0 gets zeros.
 *   spec, limits as for qift_quantize_weights (K a multiple of 64, at most 16384; block a power of two, 2..4096,
 *   dividing K; flags 0; N * K < 2^31), and N < 2^24.
 *   levels, scales   out: the fields of a qift_w8.
 */
int qift_quantize_weights8(const float *W, int64_t N, qift_hadamard_spec spec, int8_t *levels, uint16_t *scales,
                           qift_stream_t stream);

/*
 * Online rotation + per-token symmetric INT8 quantization: qift_rotate_quant_act with 127 in place of 7,
 *   q[m,k] = sign(X_k) * min(127, rne(127 |X_k| / (c A)))   decided exactly,
 *   s_x[m] = fp32( (A * num) / ((den * 127) * sqrt(b)) ),
 * X the rotated token, A = max_k |X_k| (A = 0 gives zeros and the scale 0), c = num / den from spec.flags, which take
 * QIFT_CLIP and QIFT_SPEC_BF16 as there (bf16 tokens by the reading of qift_rotate_quant_act_bf16).
 *   x          fp16 or bf16 [M][spec.K], finite.
 *   act_q      out: int8 [M][K], act_scale out: fp32 [M].
 * Limits: M < 2^23, spec.K <= 32768, block 2..8192.
 */
int qift_rotate_quant_act8(const uint16_t *x, int64_t M, qift_hadamard_spec spec, int8_t *act_q, float *act_scale,
                           qift_stream_t stream);

/* Workspace bytes of qift_w8a8_linear for these weights and M tokens (host query; 0 where it needs none, and for an
 * unsupported shape).  It is not monotonic in M (K is cut where that is faster): a server asks
 * once for each M that occurs and takes the largest, which serves them all. */
size_t qift_w8a8_workspace_bytes(const qift_w8 *w, int64_t M);

/*
 * The 8-bit linear:
 *   acc[m][n] = sum_k level[n][k] * act_q[m][k]   exact int32
 *   y[m][n]   = T( fp32( fp32(acc) * act_scale[m] ) * fp32(s_w[n]) ), the products rounded to fp32,
 *               T fp16, bf16 (to nearest, ties to even) or fp32 as dtype says.
 *   w          host: the weights.
 *   act_q, act_scale   the codes and scales of qift_rotate_quant_act8 (-128 is taken too; sums past int32 wrap).
 *   M          1 <= M < 2^31.
 *   dtype      QIFT_F16, QIFT_BF16 or QIFT_F32: the type of out (QIFT_ERR_FORMAT otherwise).
 *   out        out: [M][N].
 *   acc_out    out, nullable: int32 [M][N], the exact sums.
 *   workspace, workspace_bytes   optional: with at least qift_w8a8_workspace_bytes (where that is not 0) K is cut
 *              into parts whose int32 sums meet in the workspace; NULL / 0: one workgroup goes along all of K.  The results
 *              are the same bit for bit.  A non-zero size below the query is QIFT_ERR_WORKSPACE.  The workspace is
 *              overwritten and belongs to one call at a time: calls that overlap, two captured graphs among them, need their own.
 * Limits: ceil(N / 128) * ceil(M / 128) < 2^20.  Up to two launches.
 */
int qift_w8a8_linear(const qift_w8 *w, const int8_t *act_q, const float *act_scale, int64_t M, int32_t dtype,
                     void *out, int32_t *acc_out, void *workspace, size_t workspace_bytes, qift_stream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* QIFT_W8_H */
