// Norm and rotation with keys and values written to the cache (the kernel is
// in qk_norm_rope.cuh).
#include "qk_norm_rope.cuh"

namespace tk {
namespace {

template <typename X>
cudaError_t by_format(QkParams& p, int num_sms, cudaStream_t s) {
  switch (p.k_fmt) {
    case 0: return by_r<X, __nv_bfloat16, 0>(p, num_sms, s);
    case 1: return by_r<X, __nv_bfloat16, 1>(p, num_sms, s);
    case 2: return by_r<X, __nv_bfloat16, 2>(p, num_sms, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_qk_norm_rope_append(const QkParams& params, int num_sms, cudaStream_t s) {
  QkParams p = params;
  return p.x_f32 ? by_format<float>(p, num_sms, s) : by_format<__nv_bfloat16>(p, num_sms, s);
}

}  // namespace tk
