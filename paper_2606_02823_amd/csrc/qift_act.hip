// Rotation + INT4 quantization of activations (kernels: qift_act.h).
#include "qift_act.h"

namespace qift {

double act_denominator(int block, int clip_den, int largest) {
  // the fixed divisor of the per-token scale, (den * Q) * sqrt(b), rounded in that order
  return ((double)clip_den * (double)largest) * sqrt((double)block);
}

hipError_t launch_rotate_quant_act(const uint16_t* x, int64_t M, int64_t K, int block, int clip_num,
                                   int clip_den, int8_t* act_q, float* act_scale, int32_t* act_sum,
                                   hipStream_t s, bool bf16) {
  return bf16 ? launch_rqa<true, 7>(x, M, K, block, clip_num, clip_den, act_q, act_scale, act_sum, s)
              : launch_rqa<false, 7>(x, M, K, block, clip_num, clip_den, act_q, act_scale, act_sum, s);
}

}  // namespace qift
