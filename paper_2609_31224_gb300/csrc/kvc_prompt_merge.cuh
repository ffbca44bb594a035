// Items of whole prompts whose keys are cut into parts, and their joining.
//
// A part's rows (128 of an item's tile) leave their sums of P V, not divided, and (reference, sum) of P:
// [slot][D / 4][128 rows][4] and [slot][128], in the prefill's partial slots (of binary32 contexts, which
// have none, the decode's).  The parts of a tile have the slots (item * parts + part) * TILES + tile.
// With M = max m_p a row is sum_p O_p 2^(m_p - M) divided by sum_p l_p 2^(m_p - M), in the order of the
// parts, so that results repeat.  The parts come from L2: 5 us a layer, mostly the launch.
#pragma once

#include "kvc_prompt.h"
#include "kvc_prompt_list.cuh"

namespace kvc {

namespace {

constexpr int PART_ROWS = 128;
// A part's rows of DIMS in quads (quad i of row r at [i * PART_ROWS + r]), and their (reference, sum).
template <int DIMS>
__device__ inline float4* part_rows(const Dev& d, int slot) {
  return reinterpret_cast<float4*>(DIMS == 64 ? d.dec_part_o : d.pf_part_o) + (size_t)slot * (DIMS / 4) * PART_ROWS;
}
template <int DIMS>
__device__ inline float2* part_sums(const Dev& d, int slot) {
  return (DIMS == 64 ? d.dec_part_ml : d.pf_part_ml) + (size_t)slot * PART_ROWS;
}

__device__ inline void put_row(float* to, const float (&v)[8]) {
  reinterpret_cast<float4*>(to)[0] = make_float4(v[0], v[1], v[2], v[3]);
  reinterpret_cast<float4*>(to)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ inline void put_row(__nv_bfloat16* to, const float (&v)[8]) {
  alignas(16) __nv_bfloat162 two[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) two[i] = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
  *reinterpret_cast<uint4*>(to) = *reinterpret_cast<const uint4*>(two);
}

// A CTA joins 16 dims of a tile's rows: a thread has 8 dims of one row.  Items are TILES tiles of 32 tokens
// of one session and KV head, last ones first; empty(si, t0, part, parts) says which of the parts left nothing.
constexpr int MERGE_THREADS = 2 * PART_ROWS;
template <typename T, int DIMS, int TILES, typename EmptyFn>
__device__ inline void merge_parts(const Dev& d, T* out, int most_parts, EmptyFn empty) {
  constexpr int TOKENS_ = 32, HEADS_ = PART_ROWS / TOKENS_, SLICES = DIMS / 16;
  __shared__ int s_group[GROUPS + 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, H = d.kv_heads;
  pdl_wait();
  pdl_launch_dependents();
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0;
  auto items_of = [&](int i) { return (d.seq[i].t + TILES * TOKENS_ - 1) / (TILES * TOKENS_) * H; };
  if (warp == 0) list_items(n_seq, lane, s_group, items_of);
  __syncthreads();
  const int parts = parts_now(d, most_parts, s_group[GROUPS]);
  if (parts == 1) return;  // (the items wrote their rows themselves)
  const int total = s_group[GROUPS] * TILES * SLICES;
  for (int at = blockIdx.x; at < total; at += gridDim.x) {
    const int item = at / (TILES * SLICES), x = at / SLICES % TILES, slice = at % SLICES;
    int in;
    const int seq = find_item(n_seq, lane, s_group, item, items_of, &in);
    const SeqInfo si = d.seq[seq];
    const int t0 = ((si.t + TILES * TOKENS_ - 1) / (TILES * TOKENS_) - 1 - in / H) * TILES * TOKENS_;
    const int r = threadIdx.x % PART_ROWS, tok = t0 + x * TOKENS_ + r / HEADS_;
    if (tok >= si.t) continue;
    const int quad = 4 * slice + 2 * (threadIdx.x / PART_ROWS);
    float m = -INFINITY, l = 0.f, o[8] = {};
    for (int p = 0; p < parts; ++p) {
      if (empty(si, t0, p, parts)) continue;
      const int slot = (item * parts + p) * TILES + x;
      const float2 ml = part_sums<DIMS>(d, slot)[r];
      const float4* row = part_rows<DIMS>(d, slot) + (size_t)quad * PART_ROWS + r;
      const float4 a = row[0], b = row[PART_ROWS];
      const float to = fmaxf(m, ml.x), f = exp2_safe(m, to), g = exp2_safe(ml.x, to);
      const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      l = l * f + ml.y * g;
#pragma unroll
      for (int i = 0; i < 8; ++i) o[i] = o[i] * f + v[i] * g;
      m = to;
    }
    const float inv = 1.f / l;
#pragma unroll
    for (int i = 0; i < 8; ++i) o[i] *= inv;
    put_row(out + ((size_t)(si.q_row0 + tok) * d.q_heads + in % H * HEADS_ + r % HEADS_) * DIMS + 4 * quad, o);
  }
}

// Its CTAs: one for each slice of up to `tiles` tiles.
inline int merge_grid(int64_t tiles, int dims) { return (int)std::min<int64_t>(tiles * (dims / 16), 4096); }

}  // namespace

}  // namespace kvc
