// Attention weights (kvc_attn_weights): scratch and the kernels of each kind of chunk.
#pragma once

#include "kvc_launch.cuh"

namespace kvc {

// The caller's scratch.
struct WeightsWork {
  float* scores;   // single tokens: scores [page][KV head][slot][4]; chunks: sums [plane][page][slot],
                   // at most 8 planes a KV head
  float2* stats;   // chunks: (max, sum) [part of the keys][call row][query head]
  float2* whole;   // single tokens: (max, sum) [session of the call][query head] of pairs in one CTA
  float2* parts;   // and [2 a CTA][4] of the others' parts
};
constexpr int WEIGHTS_PARTS = 4096;  // parts of single tokens, at least twice the CTAs of a grid

constexpr int WEIGHTS_STATS = 1 << 18;  // (max, sum) pairs beyond those of one part
constexpr int WEIGHTS_SHARES = 8;    // of a chunk's tokens, at most (planes of a KV head)

// Parts of the keys for `tokens` rows of a launch made for `parts`, as far as the pairs hold.  All its kernels
// take it from the tokens that are there: a captured launch may be replayed behind a longer chunk.
__host__ __device__ inline int stat_parts(const Dev& d, int parts, int tokens) {
  const int64_t pairs = (int64_t)d.max_tokens * d.q_heads + WEIGHTS_STATS, rows = (int64_t)tokens * d.q_heads;
  if (parts * rows <= pairs) return parts;
  return (int)(pairs / rows);  // (one part of max_tokens tokens always fits)
}

// log2 of a row's denominator from its parts' (max, sum), eight of them read at once (one after the other,
// nine parts held up a step of few items by 3 us).
__device__ inline float row_lse(const float2* row, size_t stride, int parts) {
  const float2 first = *row;
  if (parts == 1) return first.x + log2f(first.y);
  float m = first.x, l = first.y;
  for (int p0 = 1; p0 < parts; p0 += 8) {
    float2 o[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
      o[i] = p0 + i < parts ? row[(size_t)(p0 + i) * stride] : make_float2(-INFINITY, 0.f);
    float mn = m;
#pragma unroll
    for (int i = 0; i < 8; ++i) mn = fmaxf(mn, o[i].x);
    l *= exp2_safe(m, mn);
#pragma unroll
    for (int i = 0; i < 8; ++i) l += o[i].y * exp2_safe(o[i].x, mn);
    m = mn;
  }
  return m + log2f(l);
}

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
