// Attention weights in plain binary32 arithmetic, for the rare rows and keys that the kernels find to be NaN.
//
// The kernels take q (or both operands) in two pieces.  A key that holds -infinity scores -infinity against
// positive query elements, and weighs 0; but of the pieces' products one may be +infinity, or 0 times an infinity,
// and their sum NaN.  The same goes for the zero rows that fill a tile of queries.  So a NaN is formed again
// here from whole operands, and stays one where the definition has one.  A score takes about a microsecond.
#pragma once

#include "kvc_prompt_list.cuh"
#include "kvc_rope.cuh"
#include "kvc_weights.h"

namespace kvc {

namespace {

// q . k of one query head and key; scale: of q.
template <typename T, int D>
__device__ __noinline__ float plain_score(const T* q, const float2* cs, const T* k, float scale) {
  using C = Chunk16<T>;
  float s = 0.f;
#pragma unroll 1
  for (int c = 0; c < D / 2; c += C::N) {
    float a[C::N], b[C::N], ka[C::N], kb[C::N];
    C::unpack(*reinterpret_cast<const uint4*>(q + c), a);
    C::unpack(*reinterpret_cast<const uint4*>(q + c + D / 2), b);
    C::unpack(*reinterpret_cast<const uint4*>(k + c), ka);
    C::unpack(*reinterpret_cast<const uint4*>(k + c + D / 2), kb);
#pragma unroll
    for (int e = 0; e < C::N; ++e) {
      float x, y;
      rope_pair(a[e], b[e], cs[c + e], x, y);
      s = fmaf(x * scale, ka[e], s);
      s = fmaf(y * scale, kb[e], s);
    }
  }
  return s;
}

template <typename T, int D>
__device__ inline float plain_score(const Dev& d, const SeqInfo& si, int layer, int head, int tok, int g, const T* q,
                                    float scale, int page, int slot) {
  const T* row = q + ((size_t)(si.q_row0 + tok) * d.q_heads + head * (d.q_heads / d.kv_heads) + g) * D;
  return plain_score<T, D>(row, d.rope + (size_t)(si.pos_first + tok) * (D / 2),
                           reinterpret_cast<const T*>(d.pool) + pool_offset_elems(d, page, layer, 0, head, slot),
                           scale);
}

// (max, sum) of a row over blocks [b0, b1) of the nb that are there.
template <typename T, int D>
__device__ __noinline__ float2 plain_stat(const Dev& d, const SeqInfo& si, int layer, int head, int tok, int g,
                                          const T* q, float scale, int b0, int b1, int nb) {
  const int32_t* hrow = d.hist_pt + (size_t)si.sid * d.max_pages_per_session;
  const int32_t* lrow = d.live_pt + (size_t)si.sid * d.max_pages_per_session;
  float m = -INFINITY, l = 0.f;
  for (int b = b0; b < min(b1, nb); ++b) {
    const uint32_t seen = slots_seen(si, b, nb, si.n_hist + si.n_live - si.t + tok);
    const int page = block_page(si, hrow, lrow, b);
    for (int slot = 0; slot < PS; ++slot) {
      if (!(seen >> slot & 1)) continue;
      const float s = plain_score<T, D>(d, si, layer, head, tok, g, q, scale, page, slot);
      if (!(s < INFINITY)) return make_float2(0.f, NAN);
      const float to = fmaxf(m, s);
      l = l * exp2_safe(m, to) + exp2_safe(s, to);
      m = to;
    }
  }
  return make_float2(m, l);
}

// What a key draws from tokens [t0, t1) of the chunk.
template <typename T, int D>
__device__ __noinline__ float plain_sum(const Dev& d, const SeqInfo& si, int layer, int head, int page, int slot,
                                        int t0, int t1, const T* q, float scale, const float2* stats, int parts) {
  const int group = d.q_heads / d.kv_heads;
  const size_t stride = (size_t)d.g->total_tokens * d.q_heads;
  auto lse = [&](int tok, int g) {
    return row_lse(stats + (size_t)(si.q_row0 + tok) * d.q_heads + head * group + g, stride, parts);
  };
  for (int tok = t0; tok < t1; ++tok)
    for (int g = 0; g < group; ++g)
      if (isnan(lse(tok, g))) return NAN;
  double w = 0.0;
  for (int tok = t0; tok < t1; ++tok)
    for (int g = 0; g < group; ++g)
      w += exp2f(plain_score<T, D>(d, si, layer, head, tok, g, q, scale, page, slot) - lse(tok, g));
  return (float)w;
}

}  // namespace

}  // namespace kvc
