// Attention weights (kvc_attn_weights): scratch and the kernels of each kind of chunk.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

// The caller's scratch.
struct WeightsWork {
  float* scores;   // single tokens: scores [page][KV head][slot][4]; chunks: sums [plane][page][slot],
                   // at most 4 planes a KV head
  float2* stats;   // chunks: (max, sum) [part of the keys][call row][query head]
  float2* whole;   // single tokens: (max, sum) [session of the call][query head] of pairs in one CTA
  float2* parts;   // and [2 a CTA][4] of the others' parts
};
constexpr int WEIGHTS_PARTS = 4096;  // parts of single tokens, at least twice the CTAs of a grid

constexpr int WEIGHTS_STATS = 1 << 18;  // (max, sum) pairs beyond those of one part
constexpr int WEIGHTS_SHARES = 4;    // of a chunk's tokens, at most (planes of a KV head)

cudaError_t weights_tc_attributes();
// Row statistics and sums by key of chunks; parts of the keys and shares of the tokens.
cudaError_t launch_weights_tc(const Dev& d, const Limits& lim, int layer, const void* q,
                              const WeightsWork& work, int parts, int shares, cudaStream_t s,
                              int64_t* launches);
cudaError_t launch_weights_f32(const Dev& d, const Limits& lim, int layer, const void* q,
                               const WeightsWork& work, int parts, int shares, cudaStream_t s,
                               int64_t* launches);
cudaError_t weights_token_attributes(const Dev& d);
cudaError_t launch_weights_token(const Dev& d, const Limits& lim, int layer, const void* q,
                                 float* weights, const WeightsWork& work, int n_seq, bool early,
                                 cudaStream_t s, int64_t* launches);

}  // namespace kvc
