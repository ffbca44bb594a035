// Kernels of whole prompts, launched by kvc_prompt.cu: tensor cores for bfloat16 (tcgen05) and binary32.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

cudaError_t prompt_tc_attributes();
cudaError_t launch_prompt_tc(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int parts,
                             int64_t items, cudaStream_t s, int64_t* launches);
cudaError_t prompt_f32_attributes();  // those of the weights too
cudaError_t launch_prompt_f32(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int parts,
                              int64_t items, cudaStream_t s, int64_t* launches);

}  // namespace kvc
