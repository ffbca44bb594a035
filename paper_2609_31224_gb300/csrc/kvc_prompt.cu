// Attention over whole prompts (kvc_attn_prompt): the kernels' attributes and launches by element type
// (kvc_prompt_tc.cu: bfloat16, kvc_prompt_f32.cu: binary32).
#include "kvc_prompt.h"

namespace kvc {

cudaError_t prompt_attributes(const Dev& d) {
  const cudaError_t e = d.esz == 2 ? prompt_tc_attributes() : prompt_f32_attributes();
  return e != cudaSuccess ? e : weights_attributes(d);
}

cudaError_t launch_attn_prompt(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                               LaunchOrder* order, cudaStream_t s, int64_t* launches) {
  // (Both kernels wait for the one before them before they let the next one start.)
  const cudaError_t e = d.esz == 2 ? launch_prompt_tc(d, lim, layer, q, out, s)
                                   : launch_prompt_f32(d, lim, layer, q, out, s);
  *launches += e == cudaSuccess;
  order->launched(layer, false);
  return e;
}

}  // namespace kvc
