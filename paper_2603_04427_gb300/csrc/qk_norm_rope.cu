// Norm and rotation into strided tensors (the kernel is in qk_norm_rope.cuh).
#include "qk_norm_rope.cuh"

namespace tk {

cudaError_t launch_qk_norm_rope(const QkParams& params, int num_sms, cudaStream_t s) {
  QkParams p = params;
  if (p.x_f32)
    return p.o_f32 ? by_r<float, float, -1>(p, num_sms, s) : by_r<float, __nv_bfloat16, -1>(p, num_sms, s);
  return p.o_f32 ? by_r<__nv_bfloat16, float, -1>(p, num_sms, s)
                 : by_r<__nv_bfloat16, __nv_bfloat16, -1>(p, num_sms, s);
}

}  // namespace tk
