// Rotation + INT8 quantization of activations for the 8-bit linear (kernels: qift_act.h).
#include "qift_act.h"

namespace qift {

hipError_t launch_rotate_quant_act8(const uint16_t* x, int64_t M, int64_t K, int block, int clip_num, int clip_den,
                                    int8_t* act_q, float* act_scale, hipStream_t s, bool bf16) {
  return bf16 ? launch_rqa<true, 127>(x, M, K, block, clip_num, clip_den, act_q, act_scale, nullptr, s)
              : launch_rqa<false, 127>(x, M, K, block, clip_num, clip_den, act_q, act_scale, nullptr, s);
}

}  // namespace qift
