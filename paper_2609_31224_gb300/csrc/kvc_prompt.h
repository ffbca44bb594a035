// Kernels of whole prompts, launched by kvc_prompt.cu: tensor cores for bfloat16 (tcgen05) and binary32.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

// Items of one part that the partial slots hold (kvc_prompt_merge.cuh).
__host__ __device__ inline int part_items(const Dev& d) {
  return d.esz == 2 ? d.pf_slots / 2 : d.dec_slots * 4 / 128;
}
// Parts of `items` items of a launch made for `parts`.  All its kernels take it from the items that are there:
// a captured launch may be replayed behind a longer chunk, whose parts the slots would not hold.
__device__ inline int parts_now(const Dev& d, int parts, int items) {
  return parts * items <= part_items(d) ? parts : max(1, part_items(d) / items);
}

cudaError_t prompt_tc_attributes();
cudaError_t launch_prompt_tc(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int parts,
                             int64_t items, cudaStream_t s, int64_t* launches);
cudaError_t prompt_f32_attributes();  // those of the weights too
cudaError_t launch_prompt_f32(const Dev& d, const Limits& lim, int layer, const void* q, void* out, int parts,
                              int64_t items, cudaStream_t s, int64_t* launches);

}  // namespace kvc
