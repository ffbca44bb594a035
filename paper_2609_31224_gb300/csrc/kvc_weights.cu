// Attention weights that the resident positions draw (kvc_attn_weights): for the queries of the last
// append, w_j += sum over tokens t and query heads h of p_thj = 2^(s_thj - lse_th), where s are the
// scores in units of log2 (scaled by log2(e) / sqrt(D)) and lse_th = log2 sum_j 2^s_thj over the keys
// that t sees.  Everything is in binary32.
//
// Single tokens are in kvc_weights_token.cu.  Of chunks, a weight needs its row's sum first, so the scores
// are formed twice: the first kernel forms the rows' (max, sum), the second the sums over rows for each
// key, KV head and share of the chunk's tokens ("planes"; kvc_weights_tc.cu, kvc_prompt_f32.cu).  The one
// here adds the planes up in their order, so that results repeat.
#include <algorithm>

#include "kvc_weights.h"

namespace kvc {

namespace {

constexpr int THREADS = 256;

// The planes' sums of each resident position, added to what it weighs: blockIdx.y is the session of the
// call (the first of some, where a captured launch is replayed behind more of them).  SPLIT threads have every SPLIT-th plane of a position, so that few loads follow one another (one
// thread took 22 us for 64 planes of 4,000 positions); their sums are joined in order.
constexpr int SPLIT = 4, POSITIONS = THREADS / SPLIT;

__global__ void __launch_bounds__(THREADS) weights_add_kernel(Dev d, int planes, WeightsWork work,
                                                              float* weights) {
  __shared__ float s_sum[SPLIT][POSITIONS];
  const int x = threadIdx.x % POSITIONS, part = threadIdx.x / POSITIONS;
  pdl_wait();
  pdl_launch_dependents();
  SeqInfo si = d.seq[blockIdx.y];  // (asked for together with the counts)
  const int n_seq = d.g->total_tokens > 0 ? d.g->n_seq : 0;
  const size_t plane = (size_t)d.n_pages * PS;
  for (int seq = blockIdx.y; seq < n_seq; seq += gridDim.y) {
    if (seq >= (int)gridDim.y) si = d.seq[seq];
    for (int at0 = blockIdx.x * POSITIONS; at0 < si.n_blocks * PS; at0 += gridDim.x * POSITIONS) {
      const int at = at0 + x, blk = at / PS, slot = at % PS;
      const BlockRange br = blk < si.n_blocks ? block_range(si, blk) : BlockRange{0, 0, 0};
      const bool in = slot >= br.lo && slot < br.hi;
      float w = 0.f;
      int gs = 0;
      float* to = nullptr;
      if (in) {
        gs = block_page(si, d.hist_pt + (size_t)si.sid * d.max_pages_per_session,
                        d.live_pt + (size_t)si.sid * d.max_pages_per_session, blk) * PS + slot;
        if (part == 0) to = weights + (size_t)si.sid * d.max_positions + d.meta_pos[gs];
#pragma unroll 16
        for (int h = part; h < planes; h += SPLIT) w += work.scores[h * plane + gs];
      }
      s_sum[part][x] = w;
      __syncthreads();
      if (to) {
#pragma unroll
        for (int p = 1; p < SPLIT; ++p) w += s_sum[p][x];
        *to += w;
      }
      __syncthreads();
    }
  }
}

cudaError_t launch_add(const Dev& d, const Limits& lim, int planes, const WeightsWork& work, float* weights,
                       int n_seq, cudaStream_t s, int64_t* launches) {
  const dim3 grid(std::max(1, std::min(256, 8 * lim.sms / n_seq)), n_seq);
  const cudaError_t e = launch_ex(&weights_add_kernel, grid, dim3(THREADS), 0, s, true, d, planes, work,
                                  weights);
  *launches += e == cudaSuccess;
  return e;
}

// The parts of a scratch area, from its start; their bytes.
size_t lay_out(uint8_t* base, int64_t n_pages, int q_heads, int max_tokens, int max_seq, WeightsWork* w) {
  size_t off = 0;
  auto take = [&](size_t bytes) {
    uint8_t* p = base ? base + off : nullptr;
    off += (bytes + 255) / 256 * 256;
    return p;
  };
  uint8_t* scores = take((size_t)n_pages * PS * q_heads * 2 * sizeof(float));
  uint8_t* stats = take(((size_t)max_tokens * q_heads + WEIGHTS_STATS) * sizeof(float2));
  uint8_t* whole = take((size_t)max_seq * q_heads * sizeof(float2));
  uint8_t* parts = take((size_t)WEIGHTS_PARTS * 4 * sizeof(float2));
  if (w) {
    w->scores = reinterpret_cast<float*>(scores);
    w->stats = reinterpret_cast<float2*>(stats);
    w->whole = reinterpret_cast<float2*>(whole);
    w->parts = reinterpret_cast<float2*>(parts);
  }
  return off;
}

}  // namespace

size_t weights_work_bytes(const kvc_config& c) {
  return lay_out(nullptr, c.n_pages, c.q_heads, c.max_tokens_per_call, c.max_seq_per_call, nullptr);
}

cudaError_t weights_attributes(const Dev& d) {
  const cudaError_t e = d.esz == 2 ? weights_tc_attributes() : cudaSuccess;  // (binary32: prompt_f32_attributes)
  return e != cudaSuccess ? e : weights_token_attributes(d);
}

cudaError_t launch_attn_weights(const Dev& d, const Limits& lim, int layer, const void* q,
                                float* weights, void* work, int n_seq, int total, int max_t,
                                int pages_max, int64_t pages_sum, LaunchOrder* order, cudaStream_t s,
                                int64_t* launches) {
  WeightsWork w;
  lay_out(static_cast<uint8_t*>(work), d.n_pages, d.q_heads, d.max_tokens, d.max_seq, &w);
  // (Each kernel but an early one waits for the one before it before it lets the next one start.)
  if (max_t == 1) {
    const bool early = order->early(layer, false);
    const cudaError_t e = launch_weights_token(d, lim, layer, q, weights, w, n_seq, early, s, launches);
    if (e == cudaSuccess) order->launched(layer, false);
    return e;
  }
  // Where the chunk's rows alone are too few items (64 tokens of a KV head, or 32), the keys are cut into
  // parts of 32 pages or more (binary32: eight), two items an SM in all.  One session, 4,096 positions, 8 KV
  // heads (4), us a layer, against one part: a chunk of 8 tokens 51 -> 25 (256 -> 26), of 64 tokens
  // 70 -> 35 (268 -> 53); with bfloat16 parts of eight pages 29 and 47.
  // Where the keys are too few items (512, or 128), the tokens are cut into shares of at least four tiles: two
  // prompts of 3,001 and 940 tokens, 72 items, took 264, 206 and 175 us a layer with 2, 4 and 8 shares.
  const int64_t tokens = d.esz == 2 ? 64 : 32, pages = d.esz == 2 ? 32 : 8, ctas = lim.sms;
  const int64_t rows = ((int64_t)total + (tokens - 1) * n_seq) / tokens * d.kv_heads;
  const int64_t part = d.esz == 2 ? 32 : 8;
  int64_t parts = std::max<int64_t>(1, std::min<int64_t>(2 * ctas / rows, (pages_max + part - 1) / part));
  parts = stat_parts(d, (int)parts, total);
  const int64_t keys = (pages_sum / pages + n_seq) * d.kv_heads;
  int shares = 1;
  while (shares < WEIGHTS_SHARES && keys * shares < 4 * ctas && max_t / 32 > 4 * shares) shares *= 2;
  cudaError_t e = d.esz == 2 ? launch_weights_tc(d, lim, layer, q, w, (int)parts, shares, s, launches)
                             : launch_weights_f32(d, lim, layer, q, w, (int)parts, shares, s, launches);
  if (e == cudaSuccess) e = launch_add(d, lim, d.kv_heads * shares, w, weights, n_seq, s, launches);
  if (e == cudaSuccess) order->launched(layer, false);
  return e;
}

}  // namespace kvc
