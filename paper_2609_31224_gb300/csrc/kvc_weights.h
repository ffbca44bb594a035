// Attention weights (kvc_attn_weights): scratch and the kernels of each kind of chunk.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

// The caller's scratch.
struct WeightsWork {
  float* scores;   // single tokens: scores [page][KV head][slot][4]; chunks: sums [plane][page][slot],
                   // at most 4 planes a KV head
  float* lse;      // chunks: [call row][query head]
  float2* whole;   // single tokens: (max, sum) [session of the call][query head] of pairs in one CTA
  float2* parts;   // and [2 a CTA][4] of the others' parts
};
constexpr int WEIGHTS_PARTS = 4096;  // parts of single tokens, at least twice the CTAs of a grid

cudaError_t weights_token_attributes(const Dev& d);
cudaError_t launch_weights_token(const Dev& d, const Limits& lim, int layer, const void* q,
                                 float* weights, const WeightsWork& work, int n_seq, bool early,
                                 cudaStream_t s, int64_t* launches);

}  // namespace kvc
