// Kernels of whole prompts on the tensor cores (bfloat16), launched by kvc_prompt.cu and kvc_weights.cu.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

cudaError_t prompt_tc_attributes();
cudaError_t launch_prompt_tc(const Dev& d, const Limits& lim, int layer, const void* q, void* out,
                             cudaStream_t s);

}  // namespace kvc
